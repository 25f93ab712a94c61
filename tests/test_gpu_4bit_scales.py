"""GPU: block scales that sp_cache_append writes during steps with drafted tokens, against the oracle's: keys and values, old and new tokens."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import mxfp4_oracle as mx
from tests import mxfp4_cases as mc
from tests import test_gpu_4bit_flow as flow

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
def test_scales_of_every_step(heads):
    """As many as two codes, or scales, of the keys may differ (a cosine that the device's and the host's fp64 round to different fp32 values), none of the
    values': these are not turned."""
    import torch
    past = [300, 17, 64, 1]
    s = flow._Step(heads, past, 3, 16, seed=3)
    H, H_kv, d = heads
    c, freq = s.cache, co.rope_frequencies(flow.THETA, d)
    last = s.last.cpu().numpy()
    for k in range(4):
        s.draw(k)
        s.step()
        torch.cuda.synchronize()
        ids = np.concatenate([last[:, None], s.tokens.cpu().numpy().reshape(s.B, s.n)], axis=1).reshape(-1)
        x = s.table[ids]
        before = c.k_blocks.copy()
        mx.append(x[:, :H], x[:, H:H + H_kv], x[:, H + H_kv:], s.cu_new.cpu().numpy(), past, None, freq, (c.k, c.k_blocks), (c.v, c.v_blocks), c.where())
        assert (c.k_blocks != before).any()
        for codes, blocks, got, scales, allowed, name in ((c.k, c.k_blocks, s.kc, "k_block_scale", 2, "keys"), (c.v, c.v_blocks, s.vc, "v_block_scale", 0, "values")):
            got, got_blocks = mc.host_codes(got), mc.host_scales(s.scales[scales])
            same = np.repeat(got_blocks == blocks, 32, axis=-1)
            assert (got_blocks != blocks).sum() <= allowed and ((got != codes) & same).sum() <= allowed, name
            codes[:], blocks[:] = got, got_blocks
        s.go_on()
        past = s.verify.kept_len.tolist()
        last = s.last.cpu().numpy()
