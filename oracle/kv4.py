"""The 4-bit full-context cache and the verification of drafted tokens, from
their definitions (include/kvr.h): what a cache of fp32 rows stands for, and
attention, eviction and rejection sampling in 64 bits.  Test infrastructure
only."""
from __future__ import annotations

import numpy as np

GROUP = 64


def bf16(x):
    """float32 rounded to the nearest bfloat16 (ties to even), as float32."""
    x = np.ascontiguousarray(x, np.float32)
    b = x.view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32))


def quantise(x):
    """codes uint8 [..., d], m and s float32 (bf16 values) [..., d / 64]."""
    x = np.asarray(x, np.float32)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    fine = np.isfinite(y).all(-1)
    with np.errstate(all="ignore"):
        lo, hi = y.min(-1), y.max(-1)
        f = np.float32(1.0) / np.float32(15.0)
        m, s = bf16(lo), bf16(hi * f - lo * f)
        m = np.where(fine, m, np.float32(np.nan))
        s = np.where(fine, s, np.float32(0))
        c = np.rint((y - m[..., None]) / s[..., None])
        c = np.where(s[..., None] > 0, np.clip(c, 0, 15), 0)
    return c.reshape(x.shape).astype(np.uint8), m, s


def values(x):
    """What rows x [..., d] stand for once stored: m + s * c, rounded once to
    float32."""
    c, m, s = (np.asarray(a, np.float64) for a in quantise(x))
    y = c.reshape(*c.shape[:-1], c.shape[-1] // GROUP, GROUP)
    with np.errstate(over="ignore"):
        y = (y * s[..., None] + m[..., None]).astype(np.float32)
    return y.reshape(c.shape)


def attend(q, k, v, scale=None):
    """One unit in 64 bits: q [T][G][d] of the newest T tokens, k and v [n][d]
    (values).  Returns out [T][G][d], the rows' scores [n] and, per output, the
    probability-weighted mean of |v|."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, G, d = q.shape
    n = k.shape[0]
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, mag = np.zeros((T, G, d)), np.zeros((T, G, d))
    score = np.zeros(n)
    for t in range(T):
        end = n - T + t + 1
        if end <= 0:
            continue
        x = q[t] @ k[:end].T * scale
        p = np.exp(x - x.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[t], mag[t] = p @ v[:end], p @ np.abs(v[:end])
        score[:end] += p.mean(0)
    return out, score, mag


def evict(score, budget, window):
    """Positions kept of rows with these scores, ascending: the window newest
    and the budget highest-scored others, ties to the lower position; a NaN
    ranks above every number."""
    n = len(score)
    first = max(0, n - window)
    key = np.where(np.isnan(score[:first]), np.inf, score[:first])
    order = sorted(range(first),
                   key=lambda i: (not np.isnan(score[i]), -key[i], i))
    return np.array(sorted(order[:budget]) + list(range(first, n)), np.int64)


def _softmax(x, temperature):
    """None where the row has no softmax."""
    x = np.asarray(x, np.float64) / temperature
    if np.isnan(x).any() or not np.isfinite(x.max()):
        return None
    e = np.exp(x - x.max())
    return e / e.sum()


def verify(target, draft, tokens, u, race, temperature=1.0):
    """One sequence: target [n + 1][V], draft [n][V], tokens, u [n], race [V].
    Returns (accepted, next token)."""
    n, V = len(tokens), len(race)
    race = np.asarray(race, np.float64)
    for t in range(n):
        p, q = _softmax(target[t], temperature), _softmax(draft[t], temperature)
        if p is None or q is None or not 0 <= tokens[t] < V:
            return t, -1
        if not float(u[t]) * q[tokens[t]] < p[tokens[t]]:
            w = np.maximum(p - q, 0)
            return t, int(np.argmax((w if w.max() > 0 else p) / race))
    p = _softmax(target[n], temperature)
    return n, -1 if p is None else int(np.argmax(p / race))
