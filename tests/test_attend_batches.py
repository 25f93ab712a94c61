"""The batches of attend_batches.py take the way through the plan that they are there for: without this a change of the rules
could leave a way of the kernels without a test on the GPU."""
import pytest

from tests import attend_batches as ab
from tests.attend_walk import walk, walk_batch  # noqa: F401


@pytest.mark.parametrize("batch", ab.BLOCKS, ids=lambda b: b["name"])
def test_large_blocks_that_workgroups_take_one_at_a_time(walk, batch):  # noqa: F811
    w = walk_batch(walk, *ab.shape(batch))
    assert not w["stretched"]
    assert w["large"].sum() * batch["H_kv"] >= (2304 if batch["d"] == 64 else 768)
    cut, prefix = w["blocks"][:, 4] > 1, w["blocks"][:, 0] < w["n_prefix"]
    assert bool((cut & w["large"] & ~prefix).any()) == batch["cut"]
    assert bool((cut & w["large"] & prefix).any()) == batch["cut_prefix"]


@pytest.mark.parametrize("batch", ab.SHARED, ids=lambda b: b["name"])
def test_blocks_laid_end_to_end(walk, batch):  # noqa: F811
    w = walk_batch(walk, *ab.shape(batch))
    assert w["stretched"] and w["n_prefix"] == sum(batch["sharing"])
    assert (w["blocks"][:w["n_prefix"], 4] > 1).any() or w["n_prefix"] > 32    # a prefix is cut where there are not many
