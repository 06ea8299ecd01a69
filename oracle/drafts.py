"""A decoding step of several drafted tokens over the 4-bit cache, from its definitions (numpy): norm and rotation with every rounding given, attention of a
tree's rows, verification, and which token a kept one is.  Test infrastructure; shares nothing with the library."""
from __future__ import annotations

import numpy as np


def norm_rotate_rounded(x, positions=None, table=None, weight=None, eps=1e-6, interleaved=False):
    """fp16 [rows, heads, head_dim]: the factor from float64, every other operation a single fp32 one, one rounding to fp16."""
    y = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        if weight is not None:
            mean = (np.asarray(x, np.float64) ** 2).mean(axis=-1, keepdims=True) + np.float64(np.float32(eps))
            y = y * ((1.0 / np.sqrt(mean)).astype(np.float32) * np.asarray(weight, np.float32))
        if table is not None and table.shape[1]:
            half = table.shape[1]
            i = np.arange(half)
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            known = (positions >= 0) & (positions < table.shape[0])
            turn = np.where(known[:, None, None], table[np.where(known, positions, 0)], np.float32(np.nan))[:, None]
            c, s, ya, yb = turn[..., 0], turn[..., 1], y[..., a], y[..., b]
            y = y.copy()
            y[..., a], y[..., b] = ya * c - yb * s, ya * s + yb * c
        return y.astype(np.float16)


def ancestors(parents):
    """bool [rows, rows]: which rows a row of a tree sees: itself and those above it."""
    n = len(parents)
    sees = np.zeros((n, n), bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def mask_words(sees, words):
    """int32 [rows, words] of bool [rows, rows]."""
    bits = np.zeros((sees.shape[0], 32 * words), np.uint64)
    n = min(sees.shape[1], 32 * words)
    bits[:, :n] = sees[:, :n]
    return (bits.reshape(-1, words, 32) << np.arange(32, dtype=np.uint64)).sum(axis=-1).astype(np.uint32).view(np.int32)


def tree_attention(q, k, v, scale, sees):
    """q [rows, heads, D], k and v [tokens, kv heads, D], sees [rows, rows]: the last `rows` tokens are those of the rows.  Results (0 for a row that sees nothing)
    and sum_j p_j |v_j|, by which errors are judged."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    n, tokens, per = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    allowed = np.ones((n, tokens), bool)
    for j in range(n):
        if 0 <= tokens - n + j < tokens:
            allowed[:, tokens - n + j] = sees[:, j]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for r in range(n):
        at = np.flatnonzero(allowed[r])
        if not len(at):
            continue
        for h in range(q.shape[1]):
            s = k[at, h // per] @ q[r, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h] = p @ v[at, h // per]
            size[r, h] = p @ np.abs(v[at, h // per])
    return out, size


def _weight(p):
    p = np.asarray(p, np.float64)
    return np.where((p > 0) & np.isfinite(p), p, 0.0)


def verify(target, tokens, uniforms, final, parents=None, draft=None):
    """One sequence: (way, token drawn behind it).  target and draft [rows, vocabulary]; parents None: a chain."""
    n, vocab = target.shape
    parents = list(range(-1, n - 1)) if parents is None else [int(p) for p in parents]
    row, way = 0, [0]
    while True:
        mass, tried, children, follows = 1.0, set(), [i for i in range(row + 1, n) if parents[i] == row], None
        for i in children:
            x = int(tokens[i])
            p = float(_weight(target[row, x])) if 0 <= x < vocab else 0.0
            if draft is not None:
                m = float(_weight(draft[i, x])) if 0 <= x < vocab else 1.0
            else:
                m, p = mass, 0.0 if x in tried else p
                mass -= p
            tried.add(x)
            if p > 0 and float(np.float64(uniforms[i])) * m < p:
                follows = i
                break
        if follows is None:
            break
        row = follows
        way.append(row)
    weights = _weight(target[row])
    if draft is not None:
        if row + 1 < n:
            weights = np.maximum(weights - _weight(draft[row + 1]), 0.0)
    else:
        weights[[x for x in tried if 0 <= x < vocab]] = 0.0
    if not (weights > 0).any():
        weights = _weight(target[row])
    positive = np.flatnonzero(weights > 0)
    if not len(positive):
        return way, -1
    sums = np.cumsum(weights)
    passes = np.flatnonzero((sums > np.float64(final) * sums[-1]) & (weights > 0))
    return way, int(passes[0] if len(passes) else positive[-1])


def kept(rows, path, accepted):
    """For each of the `rows` newest tokens of a sequence, which of them it is afterwards."""
    of = list(range(rows))
    for i in range(min(accepted, rows - 1) + 1):
        if i < path[i] < rows:
            of[i] = int(path[i])
    return of
