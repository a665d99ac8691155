"""The 4-bit cache's operators in plain numpy, 64 bits, one sequence and head at a time (tests only)."""
from __future__ import annotations

import math

import numpy as np


def bf16_round(x):
    """fp32 numbers to the nearest bf16, half to even, as fp32."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isfinite(x), r.view(np.float32), np.asarray(x, np.float32))


def quantise(x):
    """x [..., dh] (bf16 values): codes, s, m as the header defines them; NaN rows where it says so."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        m = x.min(-1, keepdims=True)
        rng = (x.max(-1, keepdims=True) - m).astype(np.float32)
        s = bf16_round((rng.astype(np.float64) / 15).astype(np.float32)).astype(np.float64)
        t = (x - m) / s
    bad = ~np.isfinite(x).all(-1, keepdims=True) | ~np.isfinite(rng)
    code = np.where(s > 0, np.minimum(np.rint(np.where(np.isfinite(t), t, 0.0)), 15), 0.0)
    code = np.where(bad, 0, code)
    return code, np.where(bad, np.nan, s), np.where(bad, np.nan, m)


def values(x):
    """What the cache gives back for x, in 64 bits."""
    code, s, m = quantise(x)
    return code * s + m


def values32(x):
    """The same with the one rounding of an fp32 result."""
    code, s, m = quantise(x)
    return (code * s + m).astype(np.float32)


def attention(q, k, v, scale):
    """q [rows, Hq, dh], k, v [keys, heads, dh] in 64 bits -> out, lse, weights per key [heads, keys]."""
    rows, hq, dh = q.shape
    n, heads = k.shape[0], k.shape[1]
    group = hq // heads
    out, lse = np.zeros((rows, hq, dh)), np.full((rows, hq), -np.inf)
    w = np.zeros((heads, n))
    if n == 0:
        return out, lse, w
    for h in range(hq):
        s = q[:, h] @ k[:, h // group].T * scale
        top = s.max(-1, keepdims=True)
        e = np.exp(s - top)
        total = e.sum(-1, keepdims=True)
        out[:, h] = e / total @ v[:, h // group]
        lse[:, h] = (top + np.log(total))[:, 0]
        w[h // group] += (e / total).sum(0)
    return out, lse, w


def keep(weights, positions, n, count, first, protect_from):
    """One head: index that each of the min(n, count) places is filled from."""
    m = min(n, count)
    guarded = [(positions[j] < first or positions[j] >= protect_from) for j in range(n)]
    w = [0.0 if math.isnan(x) else x for x in weights[:n]]
    nan = [math.isnan(x) for x in weights[:n]]
    order = sorted(range(n), key=lambda j: (not guarded[j], nan[j] and not guarded[j], 0.0 if guarded[j] else -w[j], j))
    chosen = set(order[:m])
    late = iter(sorted(j for j in chosen if j >= m))
    return [j if j in chosen else next(late) for j in range(m)]


def norm_rope(x, gain, positions, theta, eps):
    """x [rows, heads, dh]"""
    x = np.asarray(x, np.float64)
    h = x.shape[-1] // 2
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    a = np.asarray(positions, np.float64)[:, None] * float(theta) ** (-np.arange(h) / h)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    return np.concatenate((x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s), -1)
