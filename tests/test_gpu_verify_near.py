"""GPU: sp_verify where decisions are near: a draft that is the target but for one token, and random numbers close to p / q."""
import math

import numpy as np
import pytest

from tests import test_gpu_verify as checks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [700, 50257])
def test_a_draft_that_differs_at_its_token_alone(V):
    """The drafted token twice as likely as with the target, and turned down: what is left is the same share of every other token."""
    rng = np.random.default_rng(4)
    c = checks._case(rng, [1] * 6, V, bits=32, near=0.0)
    c["draft"].copy_(c["target"][0::2])
    for b in range(6):
        x = int(c["target"][2 * b].argmax())
        c["tokens"][b] = x
        c["draft"][b, x] += math.log(2.0)
    c["u"][:] = 0.95
    v = checks._run(c)
    assert v.n_accepted.tolist() == [0] * 6
    assert (v.out_tokens.view(6, 2)[:, 0].cpu().numpy() != c["tokens"]).all()


def _sum_bound(V):
    """Of a row's sum of weights, relative: as checks._check derives it."""
    return 2.0 ** -22 * (1 + math.log2(V)) + 48 * 2.0 ** -24


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V", [300, 8193, 128256])
def test_tokens_stand_and_fall_next_to_the_border(V, bits):
    """u on both sides of p / q, off by the two sums' bounds, u's own rounding and what the check of the inputs asks for besides."""
    rng = np.random.default_rng(V)
    n = [1] * 24
    c = checks._case(rng, n, V, bits=bits, temperature=rng.choice([0.7, 1.0, 1.3], 24))
    target, draft = (c[k].double().cpu().numpy() for k in ("target", "draft"))
    off = 2 * _sum_bound(V) + 2.0 ** -23 + 1e-5
    want = []
    for b in range(24):
        t = float(np.float32(c["temperature"][b]))
        p, q = ((lambda w: w / w.sum())(np.exp((z - z.max()) / t)) for z in (target[2 * b], draft[b]))
        likely = np.argsort(-q)[:40]
        x = int(likely[np.argmax(p[likely] < 0.9 * q[likely])])      # the likeliest that the draft has more often
        assert p[x] < 0.9 * q[x]
        stands = b % 2 == 0
        c["tokens"][b], c["u"][b] = x, p[x] / q[x] * (1 - off if stands else 1 + off)
        want.append(int(stands))
    assert checks._run(c).n_accepted.tolist() == want
