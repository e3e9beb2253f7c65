"""The serving operators in 64 bits, written from their definitions (NumPy, test infrastructure only).

A batch is a list of requests; the cache is k, v of pages x heads x slots x channels as numbers (an int8 cache times its
scales).  `bound` results give, per output, the sum of absolute terms that rounding errors scale with.
"""
from __future__ import annotations

import numpy as np


def turned(x, positions, cos, sin, interleaved, weight=None, eps=0.0):
    """x: tokens x heads x channels; positions: tokens.  Norm per head, then rotation of the first 2 cos.shape[1] channels."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if cos is None:
        return x
    half = cos.shape[1]
    c, s = np.asarray(cos, np.float64)[positions][:, None], np.asarray(sin, np.float64)[positions][:, None]
    first = 2 * np.arange(half) if interleaved else np.arange(half)
    second = first + (1 if interleaved else half)
    y = x.copy()
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def positions_of(start, kv_len, s):
    n = start[s + 1] - start[s]
    return np.arange(kv_len[s] - n, kv_len[s])


def visible(pos, keys, window, sinks):
    """Mask rows x keys: which keys the tokens at `pos` see."""
    j, p = np.arange(keys)[None], np.asarray(pos)[:, None]
    ok = j <= p
    if window > 0:
        ok &= (j > p - window) | (j < sinks)
    return ok


def attention(q, k, v, pages, start, kv_len, scale, window=0, sinks=0, n_pages=None):
    """q: tokens x heads x channels; returns (out, sum of p |v|), zeros where a token sees nothing.  Values that no token
    sees are not looked at."""
    n_pages = k.shape[0] if n_pages is None else n_pages
    heads, kv_heads, page = q.shape[1], k.shape[1], k.shape[2]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(len(kv_len)):
        n = int(kv_len[s])
        slots = np.arange(n)
        at = np.asarray(pages[s])[slots // page] if n else np.zeros(0, int)
        there = (at >= 0) & (at < n_pages)
        ok = visible(positions_of(start, kv_len, s), n, window, sinks) & there[None]
        seen = np.nonzero(ok.any(0))[0]
        if not len(seen):
            continue
        ok = ok[:, seen]
        for h in range(heads):
            kh = k[at[seen], h * kv_heads // heads, seen % page].astype(np.float64)
            vh = v[at[seen], h * kv_heads // heads, seen % page].astype(np.float64)
            logits = np.where(ok, q[start[s]:start[s + 1], h].astype(np.float64) @ kh.T * scale, -np.inf)
            some = ok.any(1)
            p = np.exp(logits - np.where(some, logits.max(1), 0.0)[:, None])
            p = p / np.where(some, p.sum(1), 1.0)[:, None]
            out[start[s]:start[s + 1], h] = p @ vh
            size[start[s]:start[s + 1], h] = p @ np.abs(vh)
    return out, size


def adapters(x, ids, A, B, scale, y0):
    """Returns (y, sum of absolute terms)."""
    x, y = np.asarray(x, np.float64), np.array(y0, np.float64)
    size = np.abs(y)
    for a in range(A.shape[0]):
        rows = np.nonzero(ids == a)[0]
        f = 1.0 if scale is None else float(scale[a])
        Aa, Ba = A[a].astype(np.float64), B[a].astype(np.float64)
        y[rows] += f * (x[rows] @ Aa.T @ Ba.T)
        size[rows] += abs(f) * (np.abs(x[rows]) @ np.abs(Aa).T @ np.abs(Ba).T)
    return y, size
