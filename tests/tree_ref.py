"""Plain 64-bit forms of the calls in include/mkv_tree.h, written from their
definitions one node, head and key at a time (CPU, numpy), and the error
bounds that go with them."""
import math

import numpy as np


def visible(parents, count):
    """sees[b][i]: the nodes that node i of item b sees, by walking up (empty for nodes not in use)."""
    out = []
    for row, m in zip(np.asarray(parents).tolist(), np.asarray(count).tolist()):
        sees = []
        for i in range(len(row)):
            up, a = [], i
            while i < m and a >= 0:
                up.append(a)
                a = row[a]
            sees.append(sorted(up))
        out.append(sees)
    return out


def words(sees, n):
    """The uint32 mask words of those lists as int32 [b, n, ceil(n / 32)]."""
    w = np.zeros((len(sees), n, (n + 31) // 32), np.uint32)
    for b, rows in enumerate(sees):
        for i, row in enumerate(rows):
            for a in row:
                w[b, i, a // 32] |= np.uint32(1 << (a % 32))
    return w.view(np.int32)


def attend(q, k, v, sees, K, V, length, moments, order, tau, count):
    """q [b, N, g*h, d], k, v [b, N, h, d], K, V [b, h, cap, d], length [b, h], moments None or (n, mu_k, mu_v, C):
    (out, lse, bound of out, bound of lse) in 64 bits.

    Bounds: a score is a sum of d products whose rounding in 32 bits, in any
    order, is at most d 2^-24 times the sum of their magnitudes S; twice that
    (d = 128: 1.6e-5 S) for tensor cores that cut instead of rounding, plus
    1e-5 for the exponential and the sums.  That moves lse by as much and a
    weight by as much relatively, hence out by twice as much times the mean
    magnitude A of the values under the weights; weights enter rounded to
    bf16 (8 significant bits: 2^-8 A), the output is rounded to bf16 (2^-8
    |out|, one part in a thousand more for the two together).  The moment
    term's value is a sum of d products too: 1.6e-5 times its magnitudes."""
    b, N, hq, d = q.shape
    h = k.shape[2]
    g = hq // h
    s = 1 / math.sqrt(d)
    out, lse = np.zeros((b, N, hq, d)), np.full((b, N, hq), -np.inf)
    tol, tol_lse = np.zeros_like(out), np.zeros_like(lse)
    for bi in range(b):
        for i in range(int(count[bi])):
            see = sees[bi][i]
            for hi in range(h):
                m = int(length[bi, hi])
                keys = np.concatenate([K[bi, hi, :m], k[bi, see, hi]]).astype(np.float64)
                vals = np.concatenate([V[bi, hi, :m], v[bi, see, hi]]).astype(np.float64)
                qs = q[bi, i, hi * g:(hi + 1) * g].astype(np.float64)
                x, S = s * qs @ keys.T, s * np.abs(qs) @ np.abs(keys).T
                if moments is not None and moments[0][bi, hi] > 0:
                    n = float(moments[0][bi, hi])
                    mk, mv, C = (a[bi, hi].astype(np.float64) for a in moments[1:])
                    f, F = np.broadcast_to(mv, qs.shape), np.broadcast_to(np.abs(mv), qs.shape)
                    if order == 1:
                        C = np.where(np.abs(n * C) < tau, 0, C)
                        f, F = f + s * qs @ C.T, F + s * np.abs(qs) @ np.abs(C).T
                    x = np.concatenate([x, math.log(n) + s * qs @ mk[:, None]], 1)
                    S = np.concatenate([S, math.log(n) + s * np.abs(qs) @ np.abs(mk)[:, None]], 1)
                else:
                    f = None
                if x.shape[1] == 0:
                    continue
                top = x.max(1, keepdims=True)
                with np.errstate(invalid="ignore"):
                    p = np.exp(x - top)
                    z = p.sum(1, keepdims=True)
                    p = p / z
                    o = p[:, :len(vals)] @ vals + (p[:, -1:] * f if f is not None else 0)
                    A = p[:, :len(vals)] @ np.abs(vals) + (p[:, -1:] * np.abs(f) if f is not None else 0)
                    sums = 1.6e-5 * p[:, -1:] * F if f is not None else 0
                row = slice(hi * g, (hi + 1) * g)
                out[bi, i, row], lse[bi, i, row] = o, (top + np.log(z))[:, 0]
                off = 1.6e-5 * S.max(1) + 1e-5
                tol[bi, i, row] = 1.001 * 2.0 ** -8 * (np.abs(o) + A) + 2 * off[:, None] * A + sums + 1e-30
                tol_lse[bi, i, row] = off
    return out, lse, tol, tol_lse


def rotate(x, pos, inv_freq, axis, neighbours, inverse):
    """x [b, T, heads, d], pos int [axes, b, T]; every pair of dims turned by its own angle, in 64 bits."""
    y = x.astype(np.float64).copy()
    m = len(inv_freq)
    for f in range(m):
        a, c = (2 * f, 2 * f + 1) if neighbours else (f, f + m)
        ang = pos[axis[f]].astype(np.float64) * float(np.float32(inv_freq[f]))
        cos, sin = np.cos(ang)[..., None], np.sin(ang)[..., None] * (-1 if inverse else 1)
        y[..., a] = x[..., a] * cos - x[..., c] * sin
        y[..., c] = x[..., a] * sin + x[..., c] * cos
    return y
