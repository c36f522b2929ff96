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


def prefix(q, k_new, v_new, K, V, length, moments, order, tau, Kt, Vt, length_t, count):
    """One step of every sequence: q [b, N, g*h, d], k_new and v_new [b, N, h, d] or None, K, V [b, h, cap, d], length
    [b, h], moments None or (n, mu_k, mu_v, C), tails [b * N, h, cap_t, d] and [b * N, h]: (out, lse, bound of out,
    bound of lse) in 64 bits, one sequence and head at a time.

    Bounds: a score is a sum of d products whose rounding in 32 bits, in any
    order, is at most d 2^-24 times the sum of their magnitudes S; twice that
    (1.6e-5 S) for tensor cores that cut instead of rounding, plus 1e-5 for the exponential and the sums.  That
    moves lse by as much, a weight by as much relatively, and out by twice as much times the mean magnitude A of the
    values under the weights.  A weight enters rounded to bf16, 2^-8 of it, about a normaliser of the rounded weights:
    2^-8 (A + |out|); the output is rounded once more, 2^-8 |out|.  The moment term's value is a sum of d products with
    C' in two bf16 parts: 1.6e-5 of its magnitudes."""
    b, N, hq, d = q.shape
    h = K.shape[1]
    g, s = hq // h, 1 / math.sqrt(d)
    out, lse = np.zeros((b, N, hq, d)), np.full((b, N, hq), -np.inf)
    tol, tol_lse = np.zeros_like(out), np.zeros_like(lse)
    for bi in range(b):
        for i in range(int(count[bi])):
            for hi in range(h):
                m, mt = int(length[bi, hi]), int(length_t[bi * N + i, hi])
                keys, vals = [K[bi, hi, :m], Kt[bi * N + i, hi, :mt]], [V[bi, hi, :m], Vt[bi * N + i, hi, :mt]]
                if k_new is not None:
                    keys.append(k_new[bi, i, hi:hi + 1])
                    vals.append(v_new[bi, i, hi:hi + 1])
                keys, vals = np.concatenate(keys).astype(np.float64), np.concatenate(vals).astype(np.float64)
                qs = q[bi, i, hi * g:(hi + 1) * g].astype(np.float64)
                x, S, f = s * qs @ keys.T, s * np.abs(qs) @ np.abs(keys).T, None
                if moments is not None and moments[0][bi, hi] > 0:
                    n = float(moments[0][bi, hi])
                    mk, mv, C = (a[bi, hi].astype(np.float64) for a in moments[1:])
                    f, F = np.broadcast_to(mv, qs.shape), np.broadcast_to(np.abs(mv), qs.shape)
                    if order == 1:
                        C = np.where(np.abs(n * C) < tau, 0, C)
                        f, F = f + s * qs @ C.T, F + s * np.abs(qs) @ np.abs(C).T
                    x = np.concatenate([x, math.log(n) + s * qs @ mk[:, None]], 1)
                    S = np.concatenate([S, math.log(n) + s * np.abs(qs) @ np.abs(mk)[:, None]], 1)
                if x.shape[1] == 0:
                    continue
                top = x.max(1, keepdims=True)
                p = np.exp(x - top)
                z = p.sum(1, keepdims=True)
                p = p / z
                o, A = p[:, :len(vals)] @ vals, p[:, :len(vals)] @ np.abs(vals)
                sums = 0
                if f is not None:
                    o, A, sums = o + p[:, -1:] * f, A + p[:, -1:] * np.abs(f), 1.6e-5 * p[:, -1:] * F
                row = slice(hi * g, (hi + 1) * g)
                out[bi, i, row], lse[bi, i, row] = o, (top + np.log(z))[:, 0]
                off = 1.6e-5 * S.max(1) + 1e-5
                tol[bi, i, row] = 1.001 * 2.0 ** -8 * (2 * np.abs(o) + A) + 2 * off[:, None] * A + sums + 1e-30
                tol_lse[bi, i, row] = off
    return out, lse, tol, tol_lse
