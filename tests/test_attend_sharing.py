"""When a group of sequences has its shared prefix read once (prefix_pays): a rule on rows, members, length and type, on the CPU; and
the batches of attend_batches.py that are meant to share do."""
import pytest

from tests import attend_batches as ab
from tests.attend_walk import walk, walk_batch  # noqa: F401


@pytest.mark.parametrize("rows,members,d,fp8,no,yes", [
    # rows, members: tokens that are read by each member still, tokens that are read once
    (256, 64, 128, 0, 128, 512),        # 64 single tokens of four heads
    (1024, 64, 128, 0, 512, 2048),      # four tokens each
    (4096, 64, 128, 0, 1024, 8192),     # eight tokens of eight heads each
    (1536, 24, 128, 0, 512, 8192),
    (256, 64, 128, 1, 128, 1024),
    (256, 64, 64, 0, 64, 512),
    (1024, 64, 64, 0, 256, 4096),
    (32, 8, 128, 0, 64, 2048),
    (64, 64, 128, 0, 1, 512),           # one head
])
def test_short_prefixes_are_read_by_every_member(walk, rows, members, d, fp8, no, yes):  # noqa: F811
    assert not walk.pays(rows, members, no, d, fp8)
    assert walk.pays(rows, members, yes, d, fp8)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fp8", [0, 1])
def test_what_pays_for_a_prefix_pays_for_a_longer_one(walk, d, fp8):  # noqa: F811
    for members in (0, 1, 2, 3, 8, 24, 64, 700):
        for own in (1, 3, 4, 16, 17, 32, 33, 64, 127, 128, 300):
            before = 0
            for prefix in (-5, 0, 1, 63, 64, 65, 200, 1000, 5000, 40000, 0x7fff0000):
                now = walk.pays(own * members, members, prefix, d, fp8)
                assert now >= before
                # (never for rows that the reserved room does not count: 128 a member and more)
                assert not now or (prefix > 0 and walk.share(own * members, members))
                before = now


def test_rows_and_members_of_any_number_are_answered(walk):  # noqa: F811
    assert not walk.pays(0, 2, 1000, 128, 0) or walk.share(0, 2)
    assert walk.pays((1 << 31) - 1, (1 << 25), 0x7fff0000, 128, 0) in (0, 1)
    assert not walk.pays((1 << 31) - 1, 2, 0x7fff0000, 64, 1)


@pytest.mark.parametrize("batch", [b for b in ab.SHARED + ab.BLOCKS if b["groups"]], ids=lambda b: b["name"])
def test_batches_share_what_they_are_meant_to(walk, batch):  # noqa: F811
    w = walk_batch(walk, *ab.shape(batch))
    assert w["sharing"] == batch["sharing"]
