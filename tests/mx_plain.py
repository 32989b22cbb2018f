"""Microscaled 4-bit rows and drawing from scores, restated in numpy in 64 bits from their definitions."""
from __future__ import annotations

import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """(codes as bytes, scale bytes) of the rows of a float64 array, value by value: the nearest level, the even code of
    two that are as near."""
    n, d = x.shape
    steps = -(-d // 128)
    padded = np.zeros((n, 128 * steps))
    padded[:, :d] = x
    b = padded.reshape(n, 4 * steps, 32)
    with np.errstate(all="ignore"):
        amax = np.abs(b).max(axis=2)
        fine = np.isfinite(amax)
        e = np.where(fine & (amax > 0), np.frexp(np.where(fine, amax, 1.0))[1] - 1 - 2, -127)
        e = np.maximum(e, -127)
        y = np.where(fine[..., None], np.nan_to_num(b) / np.exp2(e.astype(np.float64))[..., None], 0.0)
        off = np.abs(np.abs(y)[..., None] - LEVELS)
        best = off.min(axis=-1, keepdims=True)
        even_first = np.where(off == best, np.arange(8) % 2, 9)
        code = even_first.argmin(axis=-1).astype(np.uint8)
    code |= (np.signbit(np.where(fine[..., None], b, 0.0)).astype(np.uint8) << 3)
    scale = np.where(fine, e + 127, 255).astype(np.uint8)
    scale[:, -(-d // 32):] = 0
    code = code.reshape(n, 128 * steps)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), scale


def values(codes, scales, d):
    """What codes and scale bytes stand for, in float64."""
    n = codes.shape[0]
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(n, 2 * codes.shape[1])
    v = np.where(c >= 8, -1.0, 1.0) * LEVELS[c & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v.reshape(n, scales.shape[1], 32) * s[..., None]).reshape(n, 2 * codes.shape[1])[:, :d]


def nearest(rows, queries, k, l2):
    """The k best of every query by (score downwards, id): ids, distances."""
    s = queries @ rows.T
    key = s - 0.5 * (rows ** 2).sum(1) if l2 else s
    out_i = np.full((len(queries), k), -1, np.int64)
    out_d = np.full((len(queries), k), np.inf)
    for q in range(len(queries)):
        ids = np.flatnonzero(key[q] > -np.inf)
        best = ids[np.lexsort((ids, -key[q][ids]))][:k]
        out_i[q, :len(best)] = best
        out_d[q, :len(best)] = (queries[q] ** 2).sum() - 2 * key[q][best] if l2 else -s[q][best]
    return out_i, out_d


def draw(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(id, log-probability) drawn from one row of float64 scores; (-1, -inf) without candidates."""
    ids = np.flatnonzero(z > -np.inf)
    if not len(ids):
        return -1, -math.inf
    ids = ids[np.lexsort((ids, -z[ids]))]
    if not temperature > 0:
        return int(ids[0]), 0.0
    best = z[ids[0]]
    with np.errstate(all="ignore"):
        w = np.where(z[ids] == best, 1.0, np.exp((z[ids] - best) / temperature) if best < np.inf else 0.0)
    if top_k > 0:
        ids, w = ids[:top_k], w[:top_k]
    if 0 < top_p < 1:
        keep = int(np.searchsorted(np.cumsum(w), top_p * math.fsum(w))) + 1
        ids, w = ids[:keep], w[:keep]
    if min_p > 0:
        keep = w >= min(min_p, 1.0)
        ids, w = ids[keep], w[keep]
    order = np.argsort(ids)
    ids, w = ids[order], w[order]
    at = int(np.searchsorted(np.cumsum(w), max(u, 0.0) * math.fsum(w), side="right")) if u < 1 else len(w) - 1
    at = min(at, int(np.flatnonzero(w)[-1]))
    return int(ids[at]), -math.log1p(math.fsum(np.delete(w, at)) / w[at])
