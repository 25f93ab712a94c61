"""CPU oracle of the 4-bit cache format (OCP Microscaling, MXFP4): E2M1 codes with one E8M0 scale to 32 elements.

TEST INFRASTRUCTURE ONLY, like cache_oracle.py: plain numpy definitions that share no code with the library.  Codes are held one to a
byte here (0..15), scales as their bytes.
"""
from __future__ import annotations

import numpy as np

from . import cache_oracle as co
from .specprefill_oracle import bf16_bits_to_f64

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_values(scales: np.ndarray) -> np.ndarray:
    s = np.asarray(scales, dtype=np.int64)
    return np.where(s == 255, np.nan, np.exp2((s - 127).astype(np.float64)))


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 [.., d] of codes [.., d] and scales [.., d/32]."""
    x = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return x * np.repeat(scale_values(scales), 32, axis=-1)


def quantise(x: np.ndarray):
    """fp32 [.., d] -> (codes [.., d], scales [.., d/32]).  Codes of a block whose scale is NaN mean nothing and come back as 0."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(axis=-1)
    bad = ~np.isfinite(top)
    e = np.full(top.shape, -125)
    for k in range(-124, 128):                     # the smallest exponent that will do
        e = np.where(7.0 * np.exp2(float(k - 1)) < np.where(bad, 0.0, top), k, e)
    y = np.where(bad[..., None], 0.0, blocks) / np.exp2(e.astype(np.float64))[..., None]
    a = np.minimum(np.abs(y), 6.0)
    hi = np.searchsorted(MAGNITUDES, a)
    lo = np.maximum(hi - 1, 0)
    below, above = a - MAGNITUDES[lo], MAGNITUDES[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.signbit(y), code | 8, code).astype(np.uint8)
    code[bad] = 0
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(codes: np.ndarray) -> np.ndarray:
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(packed: np.ndarray) -> np.ndarray:
    return np.stack([packed & 15, packed >> 4], axis=-1).reshape(*packed.shape[:-1], -1)


def append(q_bits, k_bits, v_bits, cu_new, cache_len, pos, inv_freq, k, v, cache):
    """As cache_oracle.append, into k and v = (codes, scales) [n_rows, H_kv, ..] in place."""
    q_out = np.zeros_like(q_bits)
    for b in range(len(cu_new) - 1):
        for t in range(int(cu_new[b]), int(cu_new[b + 1])):
            i = int(cache_len[b]) + t - int(cu_new[b])
            p = np.array([i if pos is None else int(pos[t])])

            def turned(x):
                return bf16_bits_to_f64(x).astype(np.float32) if inv_freq is None else co.rotate_f32(x, p, inv_freq)
            q_out[t] = co.f32_to_bf16_bits(turned(q_bits[t:t + 1]))[0]
            row = co.row_of(b, i, cache)
            if row is not None:
                k[0][row], k[1][row] = quantise(turned(k_bits[t:t + 1])[0])
                v[0][row], v[1][row] = quantise(bf16_bits_to_f64(v_bits[t]).astype(np.float32))
    return q_out
