"""The operators between the q/k/v and the o product of a decoder layer, from their definitions in float64 (numpy).  Test
infrastructure; shares nothing with the library."""
from __future__ import annotations

import numpy as np


def norm_rotate(x, positions=None, table=None, weight=None, eps=1e-6, interleaved=False):
    """x [rows, heads, head_dim]; what comes out before it is rounded, and for every element the magnitude of the terms it is made of."""
    x = np.asarray(x, np.float64).copy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    size = np.abs(x)
    if table is not None:
        half = table.shape[1]
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = (np.asarray(table, np.float64)[positions][:, None, :, j] for j in (0, 1))
        xa, xb = x[..., a].copy(), x[..., b].copy()
        x[..., a], x[..., b] = xa * c - xb * s, xa * s + xb * c
        size[..., a] = size[..., b] = np.abs(xa) + np.abs(xb)
    return x, size


def cache_groups(x):
    """(low, step, codes) of fp16 rows [..., D] in groups of 32: every operation a single fp32 operation."""
    g = np.asarray(x, np.float32).reshape(*np.shape(x)[:-1], np.shape(x)[-1] // 32, 32)
    bad = ~np.isfinite(g).all(axis=-1, keepdims=True)
    g = np.where(bad, np.float32(0), g)
    low = g.min(axis=-1, keepdims=True)
    step = ((g.max(axis=-1, keepdims=True) - low) / np.float32(15)).astype(np.float16)
    with np.errstate(over="ignore"):
        beyond = np.isinf((low.astype(np.float64) + 15.0 * step.astype(np.float64)).astype(np.float16))
    step = np.where(beyond, np.nextafter(step, np.float16(0)), step)
    wide = step.astype(np.float32)
    ratio = np.divide(g - low, wide, out=np.zeros_like(g), where=np.broadcast_to(wide > 0, g.shape))
    codes = np.minimum(np.rint(ratio), np.float32(15)).astype(np.uint8)
    low = np.where(bad, np.float16(np.nan), low.astype(np.float16))
    return low, step, codes


def cache_values(x):
    """fp16 values that cached rows stand for: low + code * step, rounded once (float64 holds the sum exactly)."""
    low, step, codes = cache_groups(x)
    return (low.astype(np.float64) + codes * step.astype(np.float64)).astype(np.float16).reshape(np.shape(x))


def attention(q, k, v, scale, seen):
    """q [rows, heads, D], k and v [tokens, kv heads, D], seen [rows]: how many tokens a row sees.  Returns the rows' results (0 for a row
    that sees nothing) and sum_j p_j |v_j|, by which errors are judged."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    per = q.shape[1] // k.shape[1] if k.shape[1] else 1
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for r in range(q.shape[0]):
        n = min(int(seen[r]), k.shape[0])
        if n <= 0:
            continue
        for h in range(q.shape[1]):
            s = k[:n, h // per] @ q[r, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h] = p @ v[:n, h // per]
            size[r, h] = p @ np.abs(v[:n, h // per])
    return out, size
