"""CPU oracle of the verification of drafted tokens.  TEST INFRASTRUCTURE ONLY: the definition in fp64, row by row."""
from __future__ import annotations

import numpy as np


def log_probabilities(logits: np.ndarray, temperature: float):
    """fp64 log-probabilities of one row, or None if it has none (NaN, +infinity, nothing but -infinity)."""
    z = np.asarray(logits, dtype=np.float64)
    if np.isnan(z).any() or z.max() == np.inf or z.max() == -np.inf:
        return None
    if temperature == 0:
        out = np.full(len(z), -np.inf)
        out[int(np.argmax(z))] = 0.0               # (the first of equal ones)
        return out
    z = (z - z.max()) / temperature
    return z - np.log(np.exp(z).sum())


def verify(target, tokens, cu, u, r, draft=None, temperature=None, past_len=None):
    """n_accepted [B], out_tokens [T + B], logprob [T + B], kept_len [B], and how near the decisions were to a border."""
    B, T, V = len(cu) - 1, len(tokens), target.shape[1]
    n_accepted, kept = np.zeros(B, np.int64), np.zeros(B, np.int64)
    out, logprob = np.full(T + B, -1), np.full(T + B, -np.inf)
    margin = np.inf
    for b in range(B):
        t0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        t = 1.0 if temperature is None else float(temperature[b])
        first, a, y, wrong = t0 + b, 0, -1, not 0 <= t < np.inf
        logs = []
        while not wrong:
            lp = log_probabilities(target[first + a], t)
            if lp is None:
                wrong = True
                break
            if a == n:
                w = np.exp(lp)
            else:
                x = int(tokens[t0 + a])
                if not 0 <= x < V:
                    wrong = True
                    break
                q = np.zeros(V)
                if draft is None:
                    q[x] = 1.0
                else:
                    lq = log_probabilities(draft[t0 + a], t)
                    if lq is None:
                        wrong = True
                        break
                    q = np.exp(lq)
                p = np.exp(lp)
                if t > 0 and max(p[x], float(u[t0 + a]) * q[x]) > 0:
                    margin = min(margin, abs(float(u[t0 + a]) * q[x] - p[x]) / max(p[x], float(u[t0 + a]) * q[x]))
                if float(u[t0 + a]) * q[x] < p[x]:
                    out[first + a] = x
                    logs.append(lp[x])
                    a += 1
                    continue
                w = np.maximum(p - q, 0.0)
                if not w.sum() > 0:
                    w = p
            cum = np.cumsum(w)
            bound = float(r[b]) * cum[-1]
            hit = np.nonzero((cum > bound) & (w > 0))[0]
            y = int(hit[0]) if len(hit) else int(np.nonzero(w > 0)[0][-1])
            logs.append(lp[y])
            break
        rows = slice(first, first + n + 1)
        if wrong:
            n_accepted[b], out[rows], logprob[rows] = -1, -1, np.nan
        else:
            n_accepted[b], out[first + a] = a, y
            logprob[first:first + a + 1] = logs
        kept[b] = 0 if past_len is None else int(past_len[b]) + (0 if wrong else a + 1)
    return n_accepted, out, logprob, kept, margin
