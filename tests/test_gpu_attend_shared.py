"""GPU: sp_attend on groups whose prefixes are long enough to be read once for all members (test_attend_sharing.py holds the batches to that), against
the fp64 oracle."""
import numpy as np
import pytest

from tests import attend_batches as ab
from tests import test_gpu_attend as ga

pytestmark = pytest.mark.gpu


def case(b, seed):
    return ga._case(np.random.default_rng(seed), b["new"], b["length"], b["H"], b["H_kv"], b["d"], page=b["page"], bits=b["bits"], groups=b["groups"])


@pytest.mark.parametrize("batch", ab.SHARED, ids=lambda b: b["name"])
def test_shared_prefixes_that_are_read_once(batch):
    ga._run(case(batch, 31))


def test_a_captured_step_goes_over_from_reading_once_to_reading_by_each_member():
    """One graph, replayed while the prefix grows from nothing to all that the members share, and back."""
    import torch
    b = next(x for x in ab.SHARED if x["name"].startswith("prefix of 192 rows, 16 bits d 128"))
    c = case(b, 32)
    oracle = ga._oracle(c)
    plan, a = ga._device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
        a.run()
    for prefix in (0, 1, 65, 500, 1999, 2111, 640, 0, 2111):
        plan.prefix_len.fill_(prefix)
        a.out.fill_(7)
        a.lse.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        ga._check(c, a, oracle=oracle)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_bad_page_of_a_prefix_that_is_read_once_reaches_its_group_only(bits):
    import torch
    rng = np.random.default_rng(33)
    c = ga._case(rng, [1] * 16, [2000 + 13 * i for i in range(16)], 8, 2, 128, bits=bits, groups=[(0, 8, 1990), (8, 16, 1900)])
    oracle = ga._oracle(c)
    c["cache"].table[0, 100] = -1
    plan, a = ga._device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    assert a.out[:8].isnan().all() and a.lse[:8].isnan().all()
    ga._check(c, a, rows=list(range(8, 16)), oracle=oracle)
