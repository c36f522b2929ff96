"""mkv_norm_rope and mkv_norm_rope_grad on the GPU against plain 64-bit forms,
with the bounds that tests/norm_ref.py derives."""
import numpy as np
import pytest
import torch

import norm_ref as R
from paper_2606_01563_gb300 import mkv
from gpu_util import host

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _rot(rng, b, t, m, axes, neighbours, far=0):
    pos = rng.integers(-100, 5000, (axes, b, t)) + far
    inv = [float(np.float32(1e6 ** (-i / m))) for i in range(m)]
    return torch.tensor(pos.astype(np.int32)).cuda(), mkv.rope_params(inv, [i % axes for i in range(m)], neighbours), (
        pos, inv, [i % axes for i in range(m)], neighbours)


def _weights(gen, kind, heads, d):
    if kind == "none":
        return None
    w = torch.randn((heads, d) if "heads" in kind else (d,), generator=gen, device="cuda")
    return w if "f32" in kind else w.to(BF16)


def _close(got, ref, tol):
    got = host(got).astype(np.float64)
    off = np.abs(got - ref) - tol
    assert (off <= 0).all(), (np.unravel_index(off.argmax(), off.shape), off.max())


CASES = [  # b, t, heads of the tensors, d, rot, axes, neighbours, weights
    (1, 1, (4, 1), 128, 128, 1, False, "bf16"),
    (2, 3, (8, 2), 64, 64, 3, True, "f32"),
    (3, 67, (5,), 128, 48, 2, False, "bf16 heads"),
    (1, 131, (1, 2, 3, 4), 64, 16, 4, True, "f32 heads"),
    (2, 40, (16, 4), 128, 64, 1, True, "none"),
    (1, 700, (32, 8), 128, 128, 3, False, "bf16"),
    (65, 1, (7, 7), 64, 48, 1, False, "f32"),
]


@pytest.mark.parametrize("b,t,heads,d,rot,axes,neighbours,weights", CASES)
def test_forward_and_gradient(b, t, heads, d, rot, axes, neighbours, weights):
    rng = np.random.default_rng(b * 1000 + t)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(t)
    pos, p, plain = _rot(rng, b, t, rot // 2, axes, neighbours)
    eps = 1e-5
    total = sum(heads)
    fused = torch.randn(b, t, total + 3, d, generator=gen, device="cuda").to(BF16)  # (and heads that are no tensor's)
    grads = torch.randn(b, total, t, d, generator=gen, device="cuda").to(BF16).transpose(1, 2)
    out = torch.full((b, total + 1, t, d), 7.0, dtype=BF16, device="cuda").transpose(1, 2)
    dfused = torch.full_like(fused, 7.0)
    fwd, bwd, at = [], [], 0
    for h in heads:
        s = slice(at, at + h)
        w = _weights(gen, weights, h, d)
        dw = None if w is None else torch.empty(w.shape, dtype=F32, device="cuda")
        fwd.append((fused[:, :, s], out[:, :, s], w))
        bwd.append((fused[:, :, s], grads[:, :, s], dfused[:, :, s], w, dw))
        at += h
    mkv.mkv_norm_rope(pos, p, fwd, eps)
    ws = torch.full((mkv.mkv_norm_rope_grad_workspace_size(bwd),), 255, dtype=torch.uint8, device="cuda")
    mkv.mkv_norm_rope_grad(pos, p, bwd, eps, ws)
    for (x, y, w), (_, dy, dx, _, dw) in zip(fwd, bwd):
        wh = None if w is None else host(w)
        _close(y, *R.forward(host(x), wh, eps, *plain))
        dx_ref, dx_tol, dw_ref, dw_tol = R.backward(host(x), host(dy), wh, eps, *plain)
        _close(dx, dx_ref, dx_tol)
        if dw is not None:
            _close(dw, dw_ref, dw_tol)
    # nothing else was written
    assert (out[:, :, total:] == 7).all() and (dfused[:, :, total:] == 7).all()
    # again, into other memory: the same bits; without the weights' gradient, the same dx
    again = [(x, dy, torch.empty_like(dx), w, None if dw is None else torch.empty_like(dw)) for x, dy, dx, w, dw in bwd]
    mkv.mkv_norm_rope_grad(pos, p, again, eps, ws)
    for a, c in zip(bwd, again):
        assert torch.equal(a[2], c[2]) and (a[4] is None or torch.equal(a[4], c[4]))
    without = [(x, dy, torch.empty_like(dx), w, None) for x, dy, dx, w, _ in bwd]
    mkv.mkv_norm_rope_grad(pos, p, without, eps, ws)
    assert all(torch.equal(a[2], c[2]) for a, c in zip(bwd, without))


def test_in_place_and_broadcast_gradients():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    b, t, h, d = 2, 37, 6, 128
    pos, p, plain = _rot(np.random.default_rng(5), b, t, 32, 1, False)
    x = torch.randn(b, t, h, d, generator=gen, device="cuda").to(BF16)
    w = torch.randn(d, generator=gen, device="cuda").to(BF16)
    one = torch.randn(1, 1, h, d, generator=gen, device="cuda").to(BF16).expand(b, t, h, d)  # one gradient for all tokens
    dw, ref = torch.empty(d, device="cuda"), R.backward(host(x), host(one), host(w), 1e-6, *plain)
    ws = mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size([(x, one, x, w, dw)]))
    into_x = x.clone()
    mkv.mkv_norm_rope_grad(pos, p, [(into_x, one, into_x, w, dw)], 1e-6, ws)
    _close(into_x, ref[0], ref[1])
    _close(dw, ref[2], ref[3])
    into_dy = one.contiguous()
    mkv.mkv_norm_rope_grad(pos, p, [(x, into_dy, into_dy, w, None)], 1e-6, ws)
    assert torch.equal(into_dy, into_x)
    y = torch.empty_like(x)
    mkv.mkv_norm_rope(pos, p, [(x, y, w)], 1e-6)
    mkv.mkv_norm_rope(pos, p, [(x, x, w)], 1e-6)
    assert torch.equal(x, y)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_zeros_of_huge_values_and_not_finite(d):
    b, t, h = 1, 6, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    pos, p, plain = _rot(np.random.default_rng(d), b, t, d // 4, 1, False)
    x = torch.randn(b, t, h, d, generator=gen, device="cuda").to(BF16)
    x[0, 0], x[0, 1] = 0, x[0, 1] * 1e37  # (sums of squares past fp32's range)
    x[0, 2, 0] *= 3e-30
    dy = torch.randn(b, t, h, d, generator=gen, device="cuda").to(BF16)
    w = torch.ones(d, device="cuda")
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda")
    ws = mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size([(x, dy, dx, w, dw)]))
    call = [(x, dy, dx, w, dw)]
    mkv.mkv_norm_rope(pos, p, [(x, y, w)], 1e-6)
    mkv.mkv_norm_rope_grad(pos, p, call, 1e-6, ws)
    _close(y, *R.forward(host(x), host(w), 1e-6, *plain))
    ref = R.backward(host(x), host(dy), host(w), 1e-6, *plain)
    _close(dx, ref[0], ref[1])
    _close(dw, ref[2], ref[3])
    # a value that is not finite makes its own row NaN, and no other
    x[0, 4, 1, 3], x[0, 5, 2, 7] = float("inf"), float("nan")
    y2 = torch.empty_like(y)
    mkv.mkv_norm_rope(pos, p, [(x, y2, w)], 1e-6)
    odd = torch.zeros(t, h, dtype=torch.bool)
    odd[4, 1] = odd[5, 2] = True
    assert torch.equal(y2[0][~odd], y[0][~odd]) and not torch.isfinite(y2[0][odd]).any(-1).all()


@pytest.mark.parametrize("d", [64, 128])
def test_the_least_eps_and_rows_whose_squares_leave_the_range(d):
    """eps 2^-126, rows from 1e-17 down to bf16's least values: sums of squares from 1e-34 to nothing, which is 2^-24 of eps."""
    b, t, h, eps = 1, 40, 2, 2.0 ** -126
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d + 1)
    pos, p, plain = _rot(np.random.default_rng(d), b, t, d // 4, 1, True)
    size = 10.0 ** -torch.linspace(17, 40, t, device="cuda", dtype=torch.float64)
    x = (torch.randn(b, t, h, d, generator=gen, device="cuda").double() * size[:, None, None]).to(BF16)
    dy = torch.randn(b, t, h, d, generator=gen, device="cuda").to(BF16)
    w = torch.randn(d, generator=gen, device="cuda")
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda")
    call = [(x, dy, dx, w, dw)]
    mkv.mkv_norm_rope(pos, p, [(x, y, w)], eps)
    mkv.mkv_norm_rope_grad(pos, p, call, eps, mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size(call)))
    _close(y, *R.forward(host(x), host(w), eps, *plain))
    ref = R.backward(host(x), host(dy), host(w), eps, *plain)
    _close(dx, ref[0], ref[1])
    _close(dw, ref[2], ref[3])


def test_no_tokens():
    p, pos = mkv.rope_params([1.0] * 32), torch.zeros(1, 2, 0, dtype=torch.int32, device="cuda")
    x, w, dw = torch.zeros(2, 0, 3, 64, dtype=BF16, device="cuda"), torch.ones(3, 64, device="cuda"), torch.full((3, 64), 9.0, device="cuda")
    mkv.mkv_norm_rope(pos, p, [(x, x, w)], 1e-6)
    call = [(x, x, x, w, dw)]
    mkv.mkv_norm_rope_grad(pos, p, call, 1e-6, mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size(call)))
    assert (dw == 0).all()


def test_offsets_past_32_bits():
    """Two batch items 2^31 elements apart and a head 2^31 elements up."""
    d, far = 64, 2 ** 31
    big = torch.empty(far + 8192, dtype=BF16, device="cuda")
    x = big.as_strided((2, 3, 2, d), (far, 256, d, 1))
    y = big.as_strided((2, 3, 2, d), (1024, 256, far, 1), 2048)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x.copy_(torch.randn(2, 3, 2, d, generator=gen, device="cuda"))
    pos, p, plain = _rot(np.random.default_rng(1), 2, 3, 32, 1, True, far=2 ** 31 - 6000)
    ref = R.forward(host(x), None, 1e-6, *plain)
    dy = torch.randn(2, 3, 2, d, generator=gen, device="cuda").to(BF16)
    g = R.backward(host(x), host(dy), None, 1e-6, *plain)
    mkv.mkv_norm_rope(pos, p, [(x, y, None)], 1e-6)
    _close(y, *ref)
    call = [(x, dy, x, None, None)]
    mkv.mkv_norm_rope_grad(pos, p, call, 1e-6, mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size(call)))
    _close(x, g[0], g[1])


def test_captured_on_another_stream_beside_eager_calls():
    """A forward and backward pass in a graph, replayed, beside eager calls with a workspace of their own."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    b, t, h, d = 2, 50, 4, 128
    pos, p, plain = _rot(np.random.default_rng(9), b, t, 64, 1, False)
    x, dy = (torch.randn(b, t, h, d, generator=gen, device="cuda").to(BF16) for _ in range(2))
    w = torch.randn(h, d, generator=gen, device="cuda")
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(h, d, device="cuda")
    call = [(x, dy, dx, w, dw)]
    ws = [mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size(call)) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mkv.mkv_norm_rope(pos, p, [(x, y, w)], 1e-6, stream=side)
        mkv.mkv_norm_rope_grad(pos, p, call, 1e-6, ws[0], stream=side)
    x.mul_(-2)
    for _ in range(2):
        graph.replay()
        e = [(x, dy, torch.empty_like(dx), w, torch.empty_like(dw))]
        mkv.mkv_norm_rope_grad(pos, p, e, 1e-6, ws[1])
    torch.cuda.synchronize()
    _close(y, *R.forward(host(x), host(w), 1e-6, *plain))
    ref = R.backward(host(x), host(dy), host(w), 1e-6, *plain)
    _close(dx, ref[0], ref[1])
    _close(dw, ref[2], ref[3])
    assert torch.equal(e[0][2], dx) and torch.equal(e[0][4], dw)


def test_tensors_of_another_device_are_refused():
    p, pos = mkv.rope_params([1.0] * 32), torch.zeros(1, 1, 2, dtype=torch.int32)
    x = torch.zeros(1, 2, 1, 64, dtype=BF16)
    with pytest.raises(ValueError):
        mkv.mkv_norm_rope(pos, p, [(x, x, None)], 1e-6)
    with pytest.raises(ValueError):
        mkv.mkv_norm_rope(pos.cuda(), p, [(x.cuda(), x, None)], 1e-6)
    with pytest.raises(ValueError):
        mkv.mkv_norm_rope_grad(pos.cuda(), p, [(x.cuda(), x.cuda(), x.cuda(), torch.ones(64), None)], 1e-6, mkv.alloc_workspace(1 << 20))
