"""GPU: sp_cache_append of more than 2^24 tokens into 4 bits, all but the last of which have no place in the cache: as many heads as leave a
workgroup one token in a smaller call."""
import numpy as np
import pytest

from oracle import mxfp4_oracle as mx
from oracle.specprefill_oracle import bf16_bits_to_f64
from tests import cache_cases as cc
from tests import mxfp4_cases as mc

pytestmark = pytest.mark.gpu


def test_more_tokens_than_a_launch_has_workgroups():
    import torch
    from paper_2502_02789_amd import device as dev
    T, H_kv, d, kept = (1 << 24) + 5, 49, 64, 200
    rng = np.random.default_rng(1)
    flat = cc.normal_bits(rng, (1, 1, 8 * kept + d * H_kv)).reshape(-1)
    base = torch.zeros(8 * T + d * H_kv, dtype=torch.bfloat16, device="cuda")
    base[8 * (T - kept):] = dev.bf16_from_bits(flat)
    x = base.as_strided((T, H_kv, d), (8, d, 1))          # (rows that lie in one another are inputs like any others)
    (kc, ks), (vc, vs) = (dev.mxfp4_cache(kept, H_kv, d) for _ in "kv")
    dev.CacheAppender(x, x, cc.cuda_ints([0, T]), kc, vc, cache_len=cc.cuda_ints([kept - T]), cu_cache=cc.cuda_ints([0, kept]), k_block_scale=ks,
                      v_block_scale=vs).run()
    torch.cuda.synchronize()
    rows = np.stack([flat[8 * t:8 * t + d * H_kv].reshape(H_kv, d) for t in range(kept)])
    codes, blocks = mx.quantise(bf16_bits_to_f64(rows).astype(np.float32))
    for c, s in ((kc, ks), (vc, vs)):
        assert (mc.host_codes(c) == codes).all() and (mc.host_scales(s) == blocks).all()
