"""A step of beam search restated in numpy in 64 bits from its definition."""
from __future__ import annotations

import math

import numpy as np


def select(z, totals, beams, k, finished=None, pad=0):
    """(parents, ids, totals) of float64 scores (groups * beams, n)."""
    groups = len(z) // beams
    parents, ids = np.full((groups, k), -1, np.int64), np.full((groups, k), -1, np.int64)
    out = np.full((groups, k), -np.inf)
    for g in range(groups):
        v, b, s, j = [], [], [], []
        for i in range(beams):
            row, total = z[g * beams + i], totals[g * beams + i]
            if not total > -np.inf:
                continue
            if finished is not None and finished[g * beams + i]:
                v.append([total]), b.append([i]), s.append([0.0]), j.append([pad])
                continue
            at = np.flatnonzero(row > -np.inf)
            if not len(at):
                continue
            most = row[at].max()
            below = np.zeros(len(at))
            other = row[at] != most
            below[other] = row[at][other] - most
            w = np.exp(below)
            v.append(total + (below - math.log(math.fsum(w)))), b.append(np.full(len(at), i)), s.append(row[at]), j.append(at)
        if not v:
            continue
        v, b, s, j = (np.concatenate(x) for x in (v, b, s, j))
        keep = v > -np.inf
        v, b, s, j = v[keep], b[keep], s[keep], j[keep]
        order = np.lexsort((j, -s, b, -v))[:k]
        m = len(order)
        parents[g, :m], ids[g, :m], out[g, :m] = b[order], j[order], v[order]
    return parents, ids, out
