"""GPU: sp_verify where much of the vocabulary is masked (-infinity: the k likeliest, a grammar), so that whole strips of the row that a token is
sampled from have nothing; random numbers at the ends of their range; vocabularies of more strips than the last kernel has threads."""
import math

import numpy as np
import pytest

from tests import test_gpu_verify as checks

pytestmark = pytest.mark.gpu

LAST = 1 - 2.0 ** -24      # the largest random number
# tokens in front and at the end that are masked, a sequence each: parts of a strip (512 or 1024 tokens), strips, several, parts of the last strip
FRONT = [0, 37, 511, 512, 513, 600, 1024, 1025, 1100, 2048, 4096, 4500, 0, 0, 0, 300]
BEHIND = [0, 0, 0, 3, 40, 600, 100, 1100, 0, 0, 30, 4, 700, 1500, 4200, 4500]


def _masked(rng, V, n, front, behind, **kw):
    """Rows of a sequence, the target's and the draft's, masked alike; drafted tokens that are not, every other one the likeliest of its row, which stands."""
    c = checks._case(rng, n, V, **kw)
    t = 0
    for b, k in enumerate(n):
        lo, hi = front[b], V - behind[b]
        for j in range(k + 1):
            row = c["target"][t + b + j]
            row[:lo], row[hi:] = -math.inf, -math.inf
            if j < k:
                if c["draft"] is not None:
                    c["draft"][t + j][:lo], c["draft"][t + j][hi:] = -math.inf, -math.inf
                likeliest = (t + j) % 2 == 1
                c["tokens"][t + j] = int(row.float().argmax()) if likeliest else int(rng.integers(lo, hi))
                c["u"][t + j] *= 1e-3 if likeliest else 1.0
        t += k
    return c


# workgroups of the smaller and of the larger parts: up to 512 times 4096 logits, and more
@pytest.mark.parametrize("V,B", [(9000, 16), (128256, 7), (128255, 17), (9001, 176)])
@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("r", [0.0, LAST, None])
def test_whole_strips_masked(V, B, draft, bits, r):
    rng = np.random.default_rng(V + B)
    front, behind = ([x[b % 16] for b in range(B)] for x in (FRONT, BEHIND))
    n = [[1, 0, 2][b % 3] for b in range(B)]
    c = _masked(rng, V, n, front, behind, bits=bits, draft=draft)
    if r is not None:
        c["r"][:] = r
    v = checks._run(c)
    assert (v.n_accepted >= 0).all() and int(v.n_accepted.sum()) > 0


@pytest.mark.parametrize("r", [0.0, 0.5, LAST])
def test_one_token_that_is_not_masked(r):
    """The first, the last, and those at borders of strips: nothing else can be sampled."""
    rng = np.random.default_rng(1)
    V, at = 20011, [0, 511, 512, 1023, 1024, 10000, 20009, 20010]
    for bits in (16, 32):
        c = checks._case(rng, [0] * len(at), V, bits=bits)
        for b, k in enumerate(at):
            row = c["target"][b]
            keep = row[k].clone()
            row.fill_(-math.inf)
            row[k] = keep
        c["r"][:] = r
        assert checks._run(c).out_tokens.tolist() == at


@pytest.mark.parametrize("bits", [16, 32])
def test_probabilities_that_underflow(bits):
    """Temperatures at which all but the largest logits are below 2^-1021 of them: such tokens are not sampled at r = 0 either."""
    rng = np.random.default_rng(2)
    for r in (0.0, LAST):
        c = checks._case(rng, [1, 0, 2, 0], 6000, bits=bits, temperature=[1e-4, 1e-5, 1e-6, 1e-30])
        c["tokens"][:] = c["target"].float().argmax(dim=1)[[0, 3, 4]].int().cpu().numpy()
        c["r"][:] = r
        checks._run(c)


@pytest.mark.parametrize("B", [2, 8])
@pytest.mark.parametrize("draft", [True, False])
def test_more_strips_than_threads(B, draft):
    rng = np.random.default_rng(3)
    V = 300001
    c = _masked(rng, V, [1, 2] * (B // 2), [0, 3000] * (B // 2), [5000, 0] * (B // 2), draft=draft)
    for r in (None, 0.0, LAST):
        if r is not None:
            c["r"][:] = r
        checks._run(c)
