"""What sp_verify refuses on the host, and its oracle against distributions worked out by hand.  No GPU needed."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import verify_oracle as vo
from paper_2502_02789_amd import binding as sp

P = 0x7000_0000_0000


def _args(**kw):
    a = sp.VerifyArgs()
    base = dict(B=3, V=1000, T=7, d_cu_draft=P, d_tokens=P + 64, d_target=P + 0x10000, target_stride=1000, d_draft=P + 0x20000, draft_stride=1000,
                d_temperature=P + 128, d_u=P + 192, d_r=P + 256, d_past_len=P + 320, d_n_accepted=P + 384, d_out_tokens=P + 448, d_logprob=P + 512,
                d_kept_len=P + 576, d_workspace=P + 0x100000, workspace_bytes=1 << 30)
    for k, v in dict(base, **kw).items():
        setattr(a, k, v)
    return a


BAD = [
    (sp.SP_EINVAL, dict(B=0)), (sp.SP_EINVAL, dict(V=0)), (sp.SP_EINVAL, dict(V=1 << 24)), (sp.SP_EINVAL, dict(T=-1)), (sp.SP_EINVAL, dict(T=1 << 24)),
    (sp.SP_EINVAL, dict(logits_dtype=2)), (sp.SP_EINVAL, dict(T=1 << 20, V=128256, target_stride=128256, draft_stride=128256)),
    (sp.SP_EINVAL, dict(B=1 << 20, V=128256, target_stride=128256, draft_stride=128256)), (sp.SP_ENULL, dict(d_cu_draft=None)), (sp.SP_ENULL, dict(d_target=None)),
    (sp.SP_ENULL, dict(d_tokens=None)), (sp.SP_ENULL, dict(d_u=None)), (sp.SP_ENULL, dict(d_r=None)), (sp.SP_ENULL, dict(d_n_accepted=None)),
    (sp.SP_ENULL, dict(d_out_tokens=None)), (sp.SP_ENULL, dict(d_past_len=None)), (sp.SP_ENULL, dict(d_kept_len=None)), (sp.SP_EINVAL, dict(target_stride=999)),
    (sp.SP_EINVAL, dict(draft_stride=999)), (sp.SP_EALIGN, dict(d_target=P + 1)), (sp.SP_EALIGN, dict(d_draft=P + 2, logits_dtype=sp.SP_LOGITS_F32)),
    (sp.SP_EWORKSPACE, dict(d_workspace=None)), (sp.SP_EWORKSPACE, dict(workspace_bytes=64)), (sp.SP_EALIGN, dict(d_workspace=P + 16)),
]


@pytest.mark.parametrize("status,change", BAD)
def test_refuses(status, change):
    assert sp.load_library().sp_verify(C.byref(_args(**change)), None) == status


def test_sizes():
    lib = sp.load_library()
    assert lib.sp_verify(None, None) == sp.SP_ENULL and lib.sp_verify_workspace_bytes(None) == 0
    for bad in (dict(B=0), dict(V=0), dict(T=-1), dict(logits_dtype=7)):
        assert sp.sp_verify_workspace_bytes(_args(**bad)) == 0
    assert 0 < sp.sp_verify_workspace_bytes(_args()) < sp.sp_verify_workspace_bytes(_args(T=70, B=30, V=128256))


def test_device_class_refuses_tensors_off_the_gpu():
    from paper_2502_02789_amd import device as dev
    cu = torch.tensor([0, 1], dtype=torch.int32)
    with pytest.raises(ValueError):
        dev.Verifier(torch.zeros(2, 10), cu[1:].clone(), cu, torch.zeros(1), torch.zeros(1))


def test_oracle_by_hand():
    """Target (.5, .3, .2), draft (.2, .5, .3): token 0 always stands, token 1 with probability .6, and what is left over the draft is token 0 alone."""
    p, q = np.log([[.5, .3, .2], [.1, .2, .7]]), np.log([[.2, .5, .3]])
    for token, u, r, want in ((0, .999, .05, [1, 0, 0]), (0, .0, .25, [1, 0, 1]), (0, .0, .31, [1, 0, 2]), (1, .59, .99, [1, 1, 2]),
                              (1, .61, .99, [0, 0, -1]), (2, .65, .2, [1, 2, 1]), (2, .67, .0, [0, 0, -1])):
        n, out, logprob, kept, margin = vo.verify(p, np.array([token]), [0, 1], np.array([u]), np.array([r]), draft=q, past_len=[40])
        assert [n[0], *out] == want and kept[0] == 41 + n[0] and margin > 0.004
        assert np.allclose(np.exp(logprob[0]), [.5, .3, .2][out[0]]) and np.isneginf(logprob[1]) == (n[0] == 0)
    # without a draft: token 2 stands with probability .2; what is left is (.5, .3) / .8
    for u, r, want in ((.19, 0, [1, 2, 0]), (.21, .62, [0, 0, -1]), (.21, .63, [0, 1, -1]), (.21, .999, [0, 1, -1])):
        n, out, *_ = vo.verify(p, np.array([2]), [0, 1], np.array([u]), np.array([r]))
        assert [n[0], *out] == want
    # temperature 0: the largest, the first of equal ones
    z = np.array([[1.0, 5.0, 5.0], [0, -1, 2]])
    for token, want in ((1, [1, 1, 2]), (2, [0, 1, -1]), (0, [0, 1, -1])):
        n, out, logprob, *_ = vo.verify(z, np.array([token]), [0, 1], np.array([.5]), np.array([.5]), draft=z[:1], temperature=[0.0])
        assert [n[0], *out] == want and logprob[0] == 0
    n, out, logprob, kept, _ = vo.verify(np.full((1, 3), -np.inf), np.zeros(0, int), [0, 0], [], np.array([.5]), past_len=[9])
    assert n[0] == -1 and out[0] == -1 and np.isnan(logprob[0]) and kept[0] == 9


def test_oracle_keeps_the_target_s_distribution():
    """Drawn from q and verified, the first token is distributed as p: over a grid of all (token, u, r)."""
    p, q = np.array([.5, .3, .15, .05]), np.array([.1, .4, .1, .4])
    count, steps = np.zeros(4), 40
    for token in range(4):
        for u in (np.arange(steps) + .5) / steps:
            for r in (np.arange(steps) + .5) / steps:
                _, out, *_ = vo.verify(np.log(np.stack([p, p])), np.array([token]), [0, 1], np.array([u]), np.array([r]), draft=np.log(q)[None])
                count[out[0]] += q[token] / steps ** 2
    assert np.abs(count - p).max() < 0.02
