"""mkv_norm_rope and its gradient on the CPU: layouts, refusals of the C entry
points and of the binding, and the plain gradient against differences."""
import ctypes
import os

import numpy as np
import pytest
import torch

import norm_ref as R
from paper_2606_01563_gb300 import mkv

FAKE = 1 << 20  # never dereferenced: validation fails before any launch
OK, INVALID, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 6, 7


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mkv.LIB_PATH):
        from paper_2606_01563_gb300 import build
        build.build()
    return mkv.lib()


def test_layouts():
    assert ctypes.sizeof(mkv.mkv_norm_rope_tensor) == 96 and mkv.mkv_norm_rope_tensor.weight_head.offset == 80
    assert ctypes.sizeof(mkv.mkv_norm_rope_grad_tensor) == 136 and mkv.mkv_norm_rope_grad_tensor.dweight.offset == 128


def _params(rot=128, **fields):
    p = mkv.rope_params([0.5] * (rot // 2))
    for k, v in fields.items():
        setattr(p, k, v)
    return p


def test_forward_refusals(L):
    def call(b=1, t=4, d=128, pos=FAKE, p=None, eps=1e-6, n=1, x=(FAKE, FAKE, 2, 0, 256, 128, 0, 256, 128),
             w=(FAKE, 0, 0)):
        arr = (mkv.mkv_norm_rope_tensor * 4)(*[mkv.mkv_norm_rope_tensor(mkv.mkv_rope_tensor(*x), *w)] * 4)
        return L.mkv_norm_rope(b, t, d, pos, 0, 0, p or _params(), eps, n, arr, None)
    assert call(d=96) == UNSUPPORTED and call(b=0) == SHAPE and call(t=-1) == SHAPE and call(n=0) == SHAPE
    assert call(n=5) == SHAPE and call(b=1 << 20, t=1 << 12) == SHAPE
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert call(eps=eps) == INVALID
    assert call(pos=None) == INVALID and call(pos=FAKE + 2) == INVALID
    assert call(p=_params(inverse=1)) == INVALID and call(p=_params(rot_dim=24)) == INVALID
    assert call(p=_params(n_axes=0)) == INVALID and call(p=_params(neighbours=2)) == INVALID
    bad = [(None, FAKE), (FAKE, None), (FAKE + 8, FAKE), (FAKE, FAKE + 2)]
    assert all(call(x=(*y, 2, 0, 256, 128, 0, 256, 128)) == INVALID for y in bad)
    assert call(x=(FAKE, FAKE, 0, 0, 256, 128, 0, 256, 128)) == INVALID
    assert call(x=(FAKE, FAKE, 2, 0, 256, 127, 0, 256, 128)) == INVALID
    assert call(x=(FAKE, FAKE, 2, 0, 256, 128, 0, 256, 0)) == INVALID  # two heads written to one place
    assert call(b=2) == INVALID  # two batch items too
    assert call(w=(FAKE + 4, 0, 0)) == INVALID and call(w=(FAKE, 0, 2)) == INVALID
    for head in (64, 129, -8):
        assert call(w=(FAKE, head, 0)) == INVALID
    assert call(w=(None, 128, 0)) == INVALID
    assert call(x=(FAKE, FAKE, 40000, 0, 256, 128, 0, 256, 128), n=2) == SHAPE
    assert call(t=0, pos=None) == OK


def test_gradient_refusals(L):
    def make(x=FAKE, dy=FAKE, dx=FAKE, heads=2, strides=(0, 256, 128) * 3, w=FAKE, step=0, f32=0, dw=FAKE):
        return mkv.mkv_norm_rope_grad_tensor(x, dy, dx, heads, *strides, w, step, f32, dw)

    def size(b=1, t=4, d=128, n=1, **kw):
        return L.mkv_norm_rope_grad_workspace_size(b, t, d, n, (mkv.mkv_norm_rope_grad_tensor * 4)(*[make(**kw)] * 4))

    def call(b=1, t=4, d=128, pos=FAKE, p=None, eps=1e-6, n=1, ws=FAKE, wsb=1 << 40, **kw):
        arr = (mkv.mkv_norm_rope_grad_tensor * 4)(*[make(**kw)] * 4)
        return L.mkv_norm_rope_grad(b, t, d, pos, 0, 0, p or _params(), eps, n, arr, ws, wsb, None)
    assert call(d=80) == UNSUPPORTED and call(b=0) == SHAPE and call(n=5) == SHAPE and call(eps=0.0) == INVALID
    assert call(pos=None) == INVALID and call(p=_params(inverse=1)) == INVALID
    for name in ("x", "dy", "dx"):
        assert call(**{name: None}) == INVALID and call(**{name: FAKE + 8}) == INVALID
    assert call(heads=0) == INVALID and size(heads=0) == 0
    assert call(strides=(0, 256, 128) * 2 + (0, 256, 0)) == INVALID  # dx of two heads in one place
    assert call(strides=(0, 256, 4) + (0, 256, 128) * 2) == INVALID
    assert call(w=None) == INVALID  # a weight's gradient without the weight
    assert call(dw=FAKE + 2) == INVALID and call(step=120) == INVALID and call(f32=3) == INVALID
    assert call(heads=40000, n=2) == SHAPE and size(heads=40000, n=2) == 0
    assert size(d=96) == 0 and size(n=0) == 0 and size(b=0) == 0
    need = size()
    assert need >= 256 and call(wsb=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=FAKE + 64) == WORKSPACE
    assert call(t=0, dw=None, ws=None, pos=None) == OK


def test_an_eps_too_small_for_sums_of_squares_is_refused(L):
    """Below the least normal number squares that leave fp32's range would matter beside it."""
    fwd = (mkv.mkv_norm_rope_tensor * 1)(mkv.mkv_norm_rope_tensor(mkv.mkv_rope_tensor(FAKE, FAKE, 2, 0, 256, 128, 0, 256, 128), FAKE, 0, 0))
    bwd = (mkv.mkv_norm_rope_grad_tensor * 1)(mkv.mkv_norm_rope_grad_tensor(FAKE, FAKE, FAKE, 2, *(0, 256, 128) * 3, FAKE, 0, 0, None))
    for eps, tokens, want in ((2.0 ** -126, 0, OK), (2.0 ** -126 - 2.0 ** -149, 4, INVALID), (1e-40, 4, INVALID), (2.0 ** -149, 4, INVALID)):
        assert L.mkv_norm_rope(1, tokens, 128, FAKE, 0, 0, _params(), eps, 1, fwd, None) == want
        assert L.mkv_norm_rope_grad(1, tokens, 128, FAKE, 0, 0, _params(), eps, 1, bwd, FAKE, 1 << 40, None) == want


def test_outputs_in_one_place_are_refused(L):
    """Two tensors written to one place (each would leave parts of its own there), and a place that is read with other strides."""
    def fwd(*xs, t=4):
        arr = (mkv.mkv_norm_rope_tensor * len(xs))(*(mkv.mkv_norm_rope_tensor(mkv.mkv_rope_tensor(*x), FAKE, 0, 0) for x in xs))
        return L.mkv_norm_rope(1, t, 128, FAKE, 0, 0, _params(), 1e-6, len(xs), arr, None)

    def bwd(*xs, t=4):
        arr = (mkv.mkv_norm_rope_grad_tensor * len(xs))(*(mkv.mkv_norm_rope_grad_tensor(*x) for x in xs))
        return L.mkv_norm_rope_grad(1, t, 128, FAKE, 0, 0, _params(), 1e-6, len(xs), arr, None, 0, None)  # (no workspace: not launched)
    far, s = [FAKE * i for i in range(2, 8)], (0, 256, 128)
    assert fwd((FAKE, far[0], 2, *s, *s), (FAKE, far[0], 2, *s, *s)) == INVALID
    assert fwd((FAKE, FAKE, 2, *s, 0, 512, 128)) == INVALID and fwd((FAKE, FAKE, 2, *s, 0, 256, 256)) == INVALID

    def grad(x=FAKE, dy=far[0], dx=far[1], sx=s, sdy=s, sdx=s, heads=2, dw=far[2]):
        return x, dy, dx, heads, *sx, *sdy, *sdx, FAKE, 0, 0, dw
    other = dict(dx=far[3], dw=far[4])
    assert bwd(grad(), grad(**other)) == bwd(grad(dw=None), grad(dx=far[3])) == WORKSPACE
    assert bwd(grad(dw=None), grad(dx=far[3], dw=None), t=0) == OK
    assert bwd(grad(), grad(**{**other, "dx": far[1]})) == INVALID and bwd(grad(), grad(**{**other, "dw": far[2]})) == INVALID
    assert bwd(grad(), grad(**{**other, "dw": far[2]}), t=0) == INVALID  # (both would be zeros, but that is a caller's mistake too)
    for same in ("x", "dy"):
        place = {same: far[1]}
        assert bwd(grad(**place)) == bwd(grad(**place, heads=1, sdx=(0, 256, 0))) == WORKSPACE  # in place; a stride that is not used
        for strides in ((0, 512, 128), (0, 256, 136)):
            assert bwd(grad(**place, sdx=strides)) == INVALID


def test_binding_refusals():
    pos, p = torch.zeros(1, 1, 4, dtype=torch.int32), _params(64)
    x = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    w = torch.ones(64)
    for bad in (x.float(), x[:, :3], x[..., ::2], x[0]):
        with pytest.raises(ValueError):
            mkv.mkv_norm_rope(pos, p, [(x, bad, w)], 1e-6)
        with pytest.raises(ValueError):
            mkv.mkv_norm_rope_grad_workspace_size([(x, bad, x, w, None)])
    for bad in (w[:32], w.half(), w.double(), torch.ones(3, 64), torch.ones(64).expand(2, 64), torch.ones(128)[::2]):
        with pytest.raises(ValueError):
            mkv.mkv_norm_rope(pos, p, [(x, x, bad)], 1e-6)
    for dw in (torch.zeros(64).bfloat16(), torch.zeros(2, 64), torch.zeros(128)[::2]):
        with pytest.raises(ValueError):
            mkv.mkv_norm_rope_grad_workspace_size([(x, x, x, w, dw)])
    with pytest.raises(ValueError):
        mkv.mkv_norm_rope_grad_workspace_size([(x, x, x, None, torch.zeros(64))])
    for bad in (pos.long(), pos[:, :, ::2], pos[0], torch.zeros(0, 1, 4, dtype=torch.int32)):
        with pytest.raises(ValueError):
            mkv.mkv_norm_rope(bad, p, [(x, x, w)], 1e-6)
    with pytest.raises(ValueError):
        mkv.mkv_norm_rope(pos, p, [], 1e-6)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
def test_plain_gradient_against_differences(neighbours, per_head):
    rng = np.random.default_rng(3)
    b, t, h, d, m = 2, 3, 2, 64, 8
    rot = (rng.integers(-50, 50, (2, b, t)), rng.uniform(0.1, 1, m), [i % 2 for i in range(m)], neighbours)
    x, dy = rng.standard_normal((2, b, t, h, d))
    w = rng.standard_normal((h, d) if per_head else d)
    dx, _, dw, _ = R.backward(x, dy, w, 0.1, *rot)

    def loss(x, w):
        return (R.forward(x, w, 0.1, *rot)[0] * dy).sum()
    for _ in range(40):
        u, v = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
        s = 1e-5
        # central differences: off by s^2 times the third derivative, and 2^-53 of the loss over s
        got = (loss(x + s * u, w + s * v) - loss(x - s * u, w - s * v)) / (2 * s)
        want = (dx * u).sum() + (dw * v).sum()
        assert abs(got - want) <= 1e-6 * (1 + abs(dx * u).sum() + abs(dw * v).sum())
