"""GPU: sp_cache_append without rotation, or at position 0, leaves every bf16 value as it is (subnormals, infinities, zeros of either sign; a NaN stays one)."""
import numpy as np
import pytest

from tests import cache_cases as cc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rotated", [False, True])
def test_every_bf16_value_arrives(rotated):
    import torch
    from paper_2502_02789_amd import device as dev
    every = np.arange(65536, dtype=np.uint32).astype(np.uint16).reshape(1024, 1, 64)
    x = every.copy()
    if rotated:      # the other of a pair is zero: nothing but the value itself is added up (infinity times a sine of zero is none)
        x[:, :, 32:] = 0
        inf = (x & 0x7FFF) >= 0x7F80
        x[inf] = 0x7F7F
    t = dev.bf16_from_bits(x)
    kc = torch.zeros((64, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    table = cc.cuda_ints(np.arange(64)[None])
    pos = torch.zeros(1024, dtype=torch.int32, device="cuda") if rotated else None
    q = dev.CacheAppender(t, t, cc.cuda_ints([0, 1024]), kc, vc, q=t, pos=pos, rope_theta=5e5 if rotated else 0.0, block_table=table).run()
    torch.cuda.synchronize()
    for name, got in (("queries", q), ("keys", kc), ("values", vc)):
        got = cc.host_bits(got.reshape(1024, 1, 64), 16)
        nan, got_nan = (x & 0x7FFF) > 0x7F80, (got & 0x7FFF) > 0x7F80
        assert (nan == got_nan).all(), name
        same = (got == x) | nan
        if rotated and name != "values":
            same |= (x & 0x7FFF) == 0       # (the sign of a zero is that of a sum of zeros)
        assert same.all(), (name, np.argwhere(~same)[:3], x[~same][:3], got[~same][:3])
