"""GPU: sp_attend with more large blocks than are laid end to end, a workgroup for each (test_attend_batches.py holds the batches to that), against the
fp64 oracle; whole prompts against the same definition evaluated in fp64 on the GPU."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests import attend_batches as ab
from tests import cache_cases as cc
from tests import test_gpu_attend as ga
from tests.test_gpu_attend_shared import case

pytestmark = pytest.mark.gpu

BATCHES = [b for b in ab.BLOCKS if len(b["new"]) > 1]
PROMPTS = [b for b in ab.BLOCKS if len(b["new"]) == 1]


@pytest.mark.parametrize("batch", BATCHES, ids=lambda b: b["name"])
def test_a_large_block_to_a_workgroup(batch):
    ga._run(case(batch, 51))


def _on_the_gpu(c):
    """co.attend for one contiguous sequence whose tokens are all new, head by head in fp64."""
    import torch
    k, v = (torch.from_numpy(x).cuda() for x in c["cache"].values())
    q = torch.from_numpy(ga.bf16_bits_to_f64(c["q"])).cuda()
    n, H, d = c["length"][0], c["H"], q.shape[2]
    G = H // k.shape[1]
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse, reach = torch.full(q.shape[:2], -float("inf"), dtype=torch.float64, device="cuda"), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    for h in range(H):
        kh, vh = k[:n, h // G], v[:n, h // G]
        s = c["scale"] * torch.mm(q[:n, h], kh.t().contiguous())
        s.masked_fill_(hidden, -float("inf"))
        w = torch.softmax(s, -1)
        out[:n, h], size[:n, h] = torch.mm(w, vh), torch.mm(w, vh.abs())
        lse[:n, h] = torch.logsumexp(s, -1)
        a = c["scale"] * torch.mm(q[:n, h].abs(), kh.abs().t().contiguous())
        reach[:n, h] = a.masked_fill_(hidden, 0).amax(-1)
    return tuple(x.cpu().numpy() for x in (out, lse, size, reach))


def test_the_definition_on_the_gpu_is_the_oracle_s():
    c = ga._case(np.random.default_rng(52), [70], [70], 4, 2, 64, page=0)
    for got, want in zip(_on_the_gpu(c), co.attend(ga.bf16_bits_to_f64(c["q"]), *c["cache"].values(), cc.offsets([70]), [70], c["cache"].where(), c["scale"])):
        np.testing.assert_allclose(got, want, rtol=1e-11, atol=1e-13)


@pytest.mark.parametrize("batch", PROMPTS, ids=lambda b: b["name"])
def test_a_whole_prompt(batch):
    import torch
    c = case(batch, 53)
    plan, a = ga._device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    ga._check(c, a, oracle=_on_the_gpu(c))
