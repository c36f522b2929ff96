"""Plain 64-bit forms of the calls in include/mkv_beam.h, written from their
definitions (CPU, numpy), and the error bounds that go with them."""
import math

import numpy as np


def select(logits, score, done, end, n_out):
    """logits [b, k, v] (as read), score [b, k], done [b, k] or None: (parent, token, score, done, gap).  Every
    continuation's score in 64 bits, sorted; equal ones by beam and token.  gap: the least difference between neighbours
    of the order that decides the answer (infinite where they are exactly equal, which the tie rule settles)."""
    b, k, v = logits.shape
    parent, token = np.full((b, n_out), -1), np.full((b, n_out), -1)
    best, over, gap = np.full((b, n_out), -np.inf), np.zeros((b, n_out), int), np.inf
    for i in range(b):
        x = np.full((k, v), -np.inf)
        for j in range(k):
            s = float(score[i, j])
            if not (-np.inf < s < np.inf):
                continue
            if done is not None and done[i, j]:
                x[j, end] = s
                continue
            row = logits[i, j].astype(np.float64)
            if np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
                continue
            top = row.max()
            x[j] = s + ((row - top) - math.log(np.exp(row - top).sum()))  # (both may be far from 0)
        flat = x.ravel()
        order = np.lexsort((np.arange(flat.size), -flat))[:n_out + 1]
        order = order[flat[order] > -np.inf]
        near = flat[order[:-1]] - flat[order[1:]]
        if (near > 0).any():
            gap = min(gap, near[near > 0].min())
        order = order[:n_out]
        n = len(order)
        parent[i, :n], token[i, :n], best[i, :n] = order // v, order % v, flat[order]
        over[i, :n] = (token[i, :n] == end) | (False if done is None else done[i][parent[i, :n]] != 0)
    return parent, token, best, over, gap


def reorder(arrays, parent, lengths=None):
    """A layer's arrays [b * N, h, ...], each copied from its parent's slot: rows 0..lengths-1 of it where `lengths`
    ([b * N, h]) is given for that array, else whole."""
    b, n = parent.shape
    out = []
    for x, ln in zip(arrays, lengths or [None] * len(arrays)):
        y = x.copy()
        for i in range(b):
            if ((parent[i] < -1) | (parent[i] >= n)).any():
                continue
            for j in range(n):
                p = parent[i, j]
                if p < 0:
                    continue
                if ln is None:
                    y[i * n + j] = x[i * n + p]
                else:
                    for h in range(x.shape[1]):
                        m = min(max(int(ln[i * n + p, h]), 0), x.shape[2])
                        y[i * n + j, h, :m] = x[i * n + p, h, :m]
        out.append(y)
    return out
