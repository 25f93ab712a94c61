"""CPU oracle of the cache operators: appending keys and values to a cache, and attention over it.

TEST INFRASTRUCTURE ONLY, like specprefill_oracle.py: plain numpy definitions that share no code with the library.
The rotation follows its stated roundings (angle in fp64, cosine and sine rounded to fp32, products and their sum
separate fp32 operations); everything else is fp64 on the exactly converted inputs.
"""
from __future__ import annotations

import math

import numpy as np

from .specprefill_oracle import bf16_bits_to_f64, fp8_e4m3_bits_to_f64


def f32_to_bf16_bits(x: np.ndarray) -> np.ndarray:
    """fp32 -> bf16, nearest even (NaN keeps its sign and becomes quiet)."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = ((u.astype(np.uint64) + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), ((u >> 16) | 0x40).astype(np.uint16), r)


_E4M3 = fp8_e4m3_bits_to_f64(np.arange(0x7F, dtype=np.uint8))      # the finite magnitudes, ascending


def f32_to_e4m3_codes(x: np.ndarray) -> np.ndarray:
    """fp32 -> OCP E4M3, nearest (ties to the even code), beyond 448 the largest finite value, NaN -> 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=448.0, neginf=-448.0)), 448.0)
    hi = np.clip(np.searchsorted(_E4M3, a, side="left"), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _E4M3[lo], _E4M3[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = np.where(np.signbit(x), code | 0x80, code).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), code)


def rope_frequencies(theta: float, d: int) -> np.ndarray:
    return float(np.float32(theta)) ** (-np.arange(d // 2, dtype=np.float64) / (d // 2))


def rotate_f32(x_bits: np.ndarray, pos: np.ndarray, inv_freq: np.ndarray) -> np.ndarray:
    """bf16 bits [T, heads, d] turned to positions [T]: fp32 values before their last rounding."""
    x = bf16_bits_to_f64(x_bits).astype(np.float32)
    half = x.shape[-1] // 2
    angle = np.asarray(pos, dtype=np.float64)[:, None, None] * inv_freq
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin], axis=-1)


def row_of(b: int, i: int, cache: dict):
    """Row of the flat token axis that holds token i of sequence b, or None where there is no room or the page is bad.
    cache: {"table", "page", "n_rows"} or {"cu_cache", "n_rows"}."""
    if cache.get("table") is not None:
        table, page = cache["table"], cache["page"]
        if i < 0 or i >= table.shape[1] * page:
            return None
        p = int(table[b, i // page])
        return p * page + i % page if 0 <= p < cache["n_rows"] // page else None
    lo, hi = int(cache["cu_cache"][b]), int(cache["cu_cache"][b + 1])
    return lo + i if i >= 0 and lo >= 0 and lo + i < min(hi, cache["n_rows"]) else None


def append(q_bits, k_bits, v_bits, cu_new, cache_len, pos, inv_freq, k_rows, v_rows, cache, k_scale=None, v_scale=None):
    """k_rows, v_rows [n_rows, H_kv, d] (bf16 bits or E4M3 codes) are written in place; returns the rotated queries' bits.
    Rows of q at and beyond cu_new[-1] come back as zeros."""
    fp8 = k_rows.dtype == np.uint8
    q_out = None if q_bits is None else np.zeros_like(q_bits)
    for b in range(len(cu_new) - 1):
        for t in range(int(cu_new[b]), int(cu_new[b + 1])):
            i = int(cache_len[b]) + t - int(cu_new[b])
            p = np.array([i if pos is None else int(pos[t])])

            def turned(x):
                return bf16_bits_to_f64(x).astype(np.float32) if inv_freq is None else rotate_f32(x, p, inv_freq)
            if q_bits is not None:
                q_out[t] = f32_to_bf16_bits(turned(q_bits[t:t + 1]))[0]
            row = row_of(b, i, cache)
            if row is None:
                continue
            for rows, x, scale in ((k_rows, turned(k_bits[t:t + 1])[0], k_scale), (v_rows, bf16_bits_to_f64(v_bits[t]).astype(np.float32), v_scale)):
                if fp8:
                    s = np.ones(x.shape[0], np.float32) if scale is None else scale.astype(np.float32)
                    with np.errstate(divide="ignore", invalid="ignore"):
                        x = np.where(s[:, None] == 0, np.float32(0), x / s[:, None])
                    rows[row] = f32_to_e4m3_codes(x)
                else:
                    rows[row] = f32_to_bf16_bits(x)
    return q_out


def attend(q, k_rows, v_rows, cu_new, kv_len, cache, scale):
    """q fp64 [T, H, d]; k_rows, v_rows fp64 [n_rows, H_kv, d].  Returns out [T, H, d], lse [T, H], and for error bounds
    the weighted mean of |V| [T, H, d] and the largest sum of |q_i k_i| * scale of a row [T, H]."""
    T, H, d = q.shape
    H_kv = k_rows.shape[1]
    G = H // H_kv
    out, size = np.zeros((T, H, d)), np.zeros((T, H, d))
    lse, reach = np.full((T, H), -np.inf), np.zeros((T, H))
    for b in range(len(cu_new) - 1):
        t0, t1, m = int(cu_new[b]), int(cu_new[b + 1]), int(kv_len[b])
        n = t1 - t0
        if n == 0 or m == 0:
            continue
        rows = np.array([row_of(b, i, cache) for i in range(m)])
        visible = np.clip(m - n + np.arange(n) + 1, 0, m)
        for h in range(H):
            k, v = k_rows[rows, h // G], v_rows[rows, h // G]
            s = scale * (q[t0:t1, h] @ k.T)
            s[np.arange(m)[None, :] >= visible[:, None]] = -np.inf
            some = visible > 0
            s, t = s[some], np.arange(t0, t1)[some]
            top = s.max(axis=1, keepdims=True)
            w = np.exp(s - top)
            total = w.sum(axis=1, keepdims=True)
            out[t, h], size[t, h] = (w @ v) / total, (w @ np.abs(v)) / total
            lse[t, h] = (top + np.log(total))[:, 0]
            a = scale * (np.abs(q[t, h]) @ np.abs(k).T)
            a[np.arange(m)[None, :] >= visible[some][:, None]] = 0
            reach[t, h] = a.max(axis=1)
    return out, lse, size, reach


def attend_bounds(out, lse, size, reach, d, keys):
    """How far fp32 sums with weights in bf16 may be off, elementwise.  A logit: d products summed in fp32, (d + 4) 2^-24 of the sum of
    the products' magnitudes (the last four: scale, base, exp2's argument).  A weight is off by as much relatively, in
    numerator and denominator, and by exp2's 2^-22; to bf16 it is rounded by at most half a step, 2^-8 of itself.  Sums over `keys` terms in fp32 add
    2^-24 for each of log2-many levels at best and each term at worst.  The result's own rounding: 2^-8 of itself."""
    logit = (d + 4) * 2.0 ** -24 * reach + 2.0 ** -22
    terms = keys * 2.0 ** -24
    o = size * (2.0 ** -8 + 2 * logit[..., None] + 2 * terms) * 1.01 + np.abs(out) * 2.0 ** -8 + 1e-30
    with np.errstate(invalid="ignore"):
        l = logit + terms + 2.0 ** -22 * (1 + np.where(np.isfinite(lse), np.abs(lse), 0))
    return o, l


def softmax_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)
