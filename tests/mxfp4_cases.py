"""Batches in 4-bit caches, laid out as cache_cases.Cache has them."""
import numpy as np

from oracle import mxfp4_oracle as mx
from tests import cache_cases as cc


class FourBitCache(cc.Cache):
    """k, v: codes [n_rows, H_kv, d], one to a byte; k_blocks, v_blocks: scales [n_rows, H_kv, d/32] of both sides of 1."""

    def __init__(self, rng, room, H_kv, d, page=0, extra_pages=2, groups=(), lo=120, hi=128):
        super().__init__(rng, room, H_kv, d, page, 8, extra_pages, groups)
        shape = (self.n_rows, H_kv, d)
        self.bits = 4
        self.k, self.v = (rng.integers(0, 16, shape).astype(np.uint8) for _ in range(2))
        self.k_blocks, self.v_blocks = (rng.integers(lo, hi, (self.n_rows, H_kv, d // 32)).astype(np.uint8) for _ in range(2))
        self.k_scale = self.v_scale = None

    def parts(self):
        return self.k, self.v, self.k_blocks, self.v_blocks

    def share(self, groups):
        for lo, hi, prefix in groups:
            src = self.rows(lo, prefix)
            for b in range(lo + 1, hi):
                dst = self.rows(b, prefix)
                for x in self.parts():
                    x[dst] = x[src]

    def spoil_unused(self, lens):
        """NaN scales wherever no token of the sequences lies."""
        used = np.zeros(self.n_rows, bool)
        for b, m in enumerate(lens):
            used[self.rows(b, m)] = True
        self.k_blocks[~used] = self.v_blocks[~used] = 255

    def values(self):
        return mx.values(self.k, self.k_blocks), mx.values(self.v, self.v_blocks)

    def device(self, head_major=False):
        import torch

        def put(x):
            t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
            t = t.view(-1, self.page, *t.shape[1:]) if self.page else t
            return t.transpose(-3, -2).contiguous().transpose(-3, -2) if head_major else t
        ints = lambda a: None if a is None else cc.cuda_ints(a)  # noqa: E731
        k, v = (put(mx.pack(x)).view(torch.float4_e2m1fn_x2) for x in (self.k, self.v))
        return (dict(block_table=ints(self.table), cu_cache=ints(self.cu_cache)), k, v,
                dict(k_block_scale=put(self.k_blocks), v_block_scale=put(self.v_blocks)))


def host_codes(t):
    """Device codes -> [n_rows, H_kv, d], one to a byte."""
    import torch
    a = t.view(torch.uint8).contiguous().cpu().numpy()
    return mx.unpack(a.reshape((-1,) + a.shape[-2:]))


def host_scales(t):
    import torch
    a = t.view(torch.uint8).contiguous().cpu().numpy()
    return a.reshape((-1,) + a.shape[-2:])
