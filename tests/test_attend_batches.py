"""The batches of attend_batches.py take the way through the plan that they are there for: without this a change of the rules
could leave a way of the kernels without a test on the GPU."""
import types

import numpy as np
import pytest
import torch

from tests import attend_batches as ab
from tests import test_gpu_attend_counts as counts
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


@pytest.mark.parametrize("m", [1, 2, 63, 70001, 99999])
def test_counting_notices_one_key(m):
    """What the counting tests on the GPU compare: right results pass, with every rounding that is allowed; a key missed, met twice or taken for another does not."""
    rng = np.random.default_rng(m)
    v = rng.integers(-8, 9, (m, 1, 128))
    v[-1], v[0] = 8, (-8 if m > 1 else 8)
    total, b = v.sum(0, keepdims=True).astype(np.float64), dict(H=2, H_kv=1)

    def result(sums, n):
        out = torch.from_numpy(np.repeat(sums / n, 2, axis=1).astype(np.float32)).to(torch.bfloat16)
        return types.SimpleNamespace(out=out, lse=torch.full((1, 2), float(np.log(n)) * (1 + 2.0 ** -23), dtype=torch.float32))
    counts._check(b, result(total, m), total, np.array([m]))
    for sums, n in ((total - v[-1], m - 1), (total + v[-1], m + 1), (total + 64 * v[-1], m + 64)):
        if n > 0:
            with pytest.raises(AssertionError):
                counts._check(b, result(sums, n), total, np.array([m]))
    if m > 1:
        with pytest.raises(AssertionError):
            counts._check(b, result(total + v[-1] - v[0], m), total, np.array([m]))
