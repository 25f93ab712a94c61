"""Shared pieces of the tests of sp_cache_append and sp_attend: batches laid out in caches, on the host and on the GPU."""
import numpy as np

from oracle import cache_oracle as co
from oracle.specprefill_oracle import bf16_bits_to_f64, fp8_e4m3_bits_to_f64


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def normal_bits(rng, shape, scale=1.0):
    return co.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


class Cache:
    """Room for len(room) sequences of room[b] tokens, filled with noise: paged (pages shuffled over a pool with pages to spare) or
    contiguous; bf16 bits or E4M3 codes.  k, v: [n_rows, H_kv, d]."""

    def __init__(self, rng, room, H_kv, d, page=0, bits=16, extra_pages=2, groups=()):
        self.page, self.bits, self.H_kv, self.d = page, bits, H_kv, d
        B = len(room)
        if page:
            need = [-(-m // page) for m in room]
            shared = [0] * B        # whole pages that a member has in common with the first of its group
            first = list(range(B))
            for lo, hi, prefix in groups:
                for b in range(lo, hi):
                    shared[b], first[b] = (prefix // page if b > lo else 0), lo
            n_pages = sum(n - s for n, s in zip(need, shared)) + extra_pages
            order = rng.permutation(n_pages).astype(np.int32)
            self.table = np.full((B, max(1, max(need))), -1, np.int32)     # behind a sequence's pages: no page
            used = 0
            for b in range(B):
                own = need[b] - shared[b]
                self.table[b, :shared[b]] = self.table[first[b], :shared[b]]
                self.table[b, shared[b]:need[b]] = order[used:used + own]
                used += own
            self.n_rows, self.cu_cache = n_pages * page, None
        else:
            self.table, self.cu_cache = None, offsets(room)
            self.n_rows = max(1, int(self.cu_cache[-1]))
        shape = (self.n_rows, H_kv, d)
        if bits == 8:
            self.k = rng.integers(0, 0x7F, shape).astype(np.uint8) | (rng.integers(0, 2, shape) << 7).astype(np.uint8)
            self.v = rng.integers(0, 0x7F, shape).astype(np.uint8) | (rng.integers(0, 2, shape) << 7).astype(np.uint8)
            self.k_scale = (0.002 + 0.004 * rng.random(H_kv)).astype(np.float32)
            self.v_scale = (0.002 + 0.004 * rng.random(H_kv)).astype(np.float32)
        else:
            self.k, self.v = normal_bits(rng, shape), normal_bits(rng, shape)
            self.k_scale = self.v_scale = None

    def where(self):
        return {"table": self.table, "page": self.page, "cu_cache": self.cu_cache, "n_rows": self.n_rows}

    def rows(self, b, m):
        return np.array([co.row_of(b, i, self.where()) for i in range(m)], dtype=np.int64)

    def share(self, groups):
        """The first tokens of every member become those of the first member of its group."""
        for lo, hi, prefix in groups:
            src = self.rows(lo, prefix)
            for b in range(lo + 1, hi):
                dst = self.rows(b, prefix)
                self.k[dst], self.v[dst] = self.k[src], self.v[src]

    def spoil_unused(self, lens):
        """NaN (or its code) wherever no token of the sequences lies."""
        used = np.zeros(self.n_rows, bool)
        for b, m in enumerate(lens):
            used[self.rows(b, m)] = True
        self.k[~used] = self.v[~used] = 0x7FC1 if self.bits == 16 else 0x7F

    def values(self):
        if self.bits == 8:
            return (fp8_e4m3_bits_to_f64(self.k) * self.k_scale.astype(np.float64)[:, None], fp8_e4m3_bits_to_f64(self.v) * self.v_scale.astype(np.float64)[:, None])
        return bf16_bits_to_f64(self.k), bf16_bits_to_f64(self.v)

    def device(self, head_major=False):
        """(keyword arguments of the device classes, k_cache, v_cache)."""
        import torch

        def put(x):
            t = torch.from_numpy(np.ascontiguousarray(x).view(np.int16 if self.bits == 16 else np.uint8)).cuda()
            t = t.view(torch.bfloat16) if self.bits == 16 else t
            t = t.view(-1, self.page, self.H_kv, self.d) if self.page else t
            if head_major:      # [.., H_kv, tokens, d] in memory
                t = t.transpose(-3, -2).contiguous().transpose(-3, -2)
            return t
        ints = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
        fl = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
        return dict(block_table=ints(self.table), cu_cache=ints(self.cu_cache)), put(self.k), put(self.v), dict(k_scale=fl(self.k_scale), v_scale=fl(self.v_scale))


def host_bits(t, bits):
    """Device cache -> [n_rows, H_kv, d] bit patterns."""
    import torch
    t = t.contiguous()
    a = (t.view(torch.int16) if bits == 16 else t.view(torch.uint8)).cpu().numpy()
    a = a.view(np.uint16) if bits == 16 else a
    return a.reshape((-1,) + a.shape[-2:])


def cuda_ints(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
