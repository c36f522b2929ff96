"""Plain 64-bit forms of mkv_norm_rope and its gradient (CPU, numpy), written
from their definitions, and the error bounds that go with them.

Bounds.  In 32 bits a sum of up to 128 squares is off by at most 128 2^-24 of
itself, its root by half of that, and the function, the two products and the
rotation's products and sum add a few units of 2^-23: together below 2^-16 of
the magnitudes that enter (sums of magnitudes, where terms can cancel).  What
is rounded to bf16 is off by half a step, 2^-8 of itself, more."""
import numpy as np

U32, U16 = 2.0 ** -16, 1.001 * 2.0 ** -8


def pairs(m, neighbours):
    f = np.arange(m)
    return (2 * f, 2 * f + 1) if neighbours else (f, f + m)


def turn(x, pos, inv_freq, axis, neighbours, back=False, magnitudes=False):
    """x [b, T, heads, d] with every pair of dims turned; with `magnitudes`, the sum of the two products' magnitudes."""
    y, (a, c) = x.astype(np.float64).copy(), pairs(len(inv_freq), neighbours)
    angle = np.stack([pos[ax].astype(np.float64) * float(np.float32(w)) for w, ax in zip(inv_freq, axis)], -1)
    cos, sin = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None] * (-1 if back else 1)
    if magnitudes:
        cos, sin = np.abs(cos), np.abs(sin)
        y = np.abs(y)
        x0, x1 = y[..., a].copy(), y[..., c].copy()
        y[..., a], y[..., c] = x0 * cos + x1 * sin, x0 * sin + x1 * cos
    else:
        x0, x1 = y[..., a].copy(), y[..., c].copy()
        y[..., a], y[..., c] = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    return y


def _normed(x, eps):
    x = x.astype(np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps)))
    return x * r, r


def forward(x, w, eps, *rot):
    """(y, bound): x [b, T, heads, d], w [d] or [heads, d] or None."""
    w = np.ones(x.shape[-1]) if w is None else w.astype(np.float64)
    n = _normed(x, eps)[0] * w
    y = turn(n, *rot)
    return y, U16 * np.abs(y) + U32 * turn(n, *rot, magnitudes=True) + 1e-38


def backward(x, dy, w, eps, *rot):
    """(dx, bound, dw, bound): dw of w's shape (None where w is)."""
    wd = np.ones(x.shape[-1]) if w is None else w.astype(np.float64)
    xh, r = _normed(x, eps)
    dn = turn(dy, *rot, back=True)
    mag = turn(dy, *rot, back=True, magnitudes=True)
    gain, gmag = wd * dn, np.abs(wd) * mag
    dx = r * (gain - xh * (gain * xh).mean(-1, keepdims=True))
    tol = U16 * np.abs(dx) + U32 * r * (gmag + np.abs(xh) * (gmag * np.abs(xh)).mean(-1, keepdims=True)) + 1e-38
    if w is None:
        return dx, tol, None, None
    over = (0, 1) if w.ndim == 2 else (0, 1, 2)
    rows = np.prod([x.shape[i] for i in over])
    # (each of the sums' additions is off by at most 2^-24 of the sum of magnitudes)
    return dx, tol, (dn * xh).sum(over), (U32 + rows * 2.0 ** -24) * (mag * np.abs(xh)).sum(over) + 1e-38
