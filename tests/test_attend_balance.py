"""Blocks that sp_attend_plan lays end to end are cut into stretches of equal cost, whatever the batch: blocks of 17 to 32 rows are small ones,
so that they do not count towards the large blocks for which a workgroup each is the better way."""
import numpy as np
import pytest

from tests import test_attend_plan as plan
from tests.attend_walk import walk, walk_batch  # noqa: F401


@pytest.mark.parametrize("heads", [(32, 8), (8, 8), (128, 8), (24, 8), (7, 1), (1024, 1024), (64, 2)])
@pytest.mark.parametrize("kind", [(128, 0), (128, 1), (64, 0), (64, 1)])
def test_no_stretch_has_much_more_than_its_share(walk, heads, kind):  # noqa: F811
    (H, H_kv), (d, fp8), checked, between = heads, kind, 0, 0
    few = [([5, 6, 7, 8] * n, [300 + 41 * i for i in range(4 * n)], []) for n in (2, 20, 60, 150)]     # 17 to 32 rows with four heads to a KV head
    for new, length, groups in plan._batches() + few:
        w = walk_batch(walk, new, length, groups, H, H_kv, d, fp8)
        blocks, pieces = w["blocks"], w["pieces"]
        assert (np.diff(pieces[:, 3]) >= 0).all() and (len(pieces) == 0 or pieces[-1, 3] < w["n_stretches"])
        if not w["stretched"] or len(pieces) == 0:
            # a workgroup for each piece
            assert len(pieces) == 0 or w["n_stretches"] == len(pieces)
            continue
        # a piece costs its steps and its block's extra; a stretch's ends are whole steps, of which a piece has two at least (no step costs more than 8, no
        # block more than 12 besides): at either end two steps, and the extra of a block that is begun elsewhere
        cost = [int(blocks[x[0], 8]) + -(-(int(x[2]) - (int(x[1]) & ~63)) // 64) * int(blocks[x[0], 6]) for x in pieces]
        per = np.bincount(pieces[:, 3], weights=cost, minlength=w["n_stretches"])
        share = (blocks[:, 7] * blocks[:, 6] + blocks[:, 8]).sum() / w["n_stretches"]
        assert per.max() <= share + 2 * 12 + 2 * 2 * 8 + 1
        checked += 1
        between += bool(((w["nr"] > 16) & ~w["large"]).sum() * H_kv >= 3 * (768 if d == 64 else 256))
    assert checked >= 100 or H_kv == 1024       # (1024 KV heads: three rounds with the first large block)
    if heads in ((32, 8), (24, 8)):
        assert between                          # small blocks that would have gone the other way if they counted as large


def test_whole_prompts_are_taken_a_block_at_a_time(walk):  # noqa: F811
    """... from the last sequence's last block to the first's first: of one sequence the longest come first, of several as they lie."""
    w = walk_batch(walk, [20000], [20000], [], 32, 8, 128, 0)
    assert not w["stretched"] and (np.diff(w["blocks"][:, 3]) <= 0).all()
    new = [900, 2300, 800, 2300, 300]
    w = walk_batch(walk, new, new, [], 64, 16, 64, 0)
    assert not w["stretched"] and (np.diff(w["blocks"][:, 0]) <= 0).all()
    for s in range(5):
        keys = w["blocks"][w["blocks"][:, 0] == s, 3]
        assert (np.diff(keys) <= 0).all() and keys[0] == new[s]
