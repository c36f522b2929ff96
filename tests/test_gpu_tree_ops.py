"""Visibility words, positions and path commits of drafted trees
(mkv_tree_build, mkv_tree_commit) and rotary positions (mkv_rope) on the GPU,
against plain forms: the first two exactly, the rotation to one rounding."""
import numpy as np
import pytest
import torch

import tree_ref as R
from paper_2606_01563_gb300 import mkv
from paper_2606_01563_gb300.inputs import bf16_round
from gpu_util import bf16, host, i32

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------- build
def _build(parents, count=None, base=None, pos=True):
    b, n = parents.shape
    mask = torch.full((b, n, (n + 31) // 32), 7, dtype=torch.int32, device="cuda")
    at = torch.full((b, n), 7, dtype=torch.int32, device="cuda") if pos else None
    ws = mkv.alloc_workspace(256)
    mkv.mkv_tree_build(i32(parents), mask, at, ws, count=count, base=base)
    return mask.cpu().numpy(), None if at is None else at.cpu().numpy(), ws


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 128, 200, 255, 256])
@pytest.mark.parametrize("shape", ["random", "chain", "star", "roots"])
def test_build(n, shape):
    rng = np.random.default_rng(n)
    b = 4
    parents = np.array([[{"random": rng.integers(-1, i) if i else -1, "chain": i - 1, "star": 0 if i else -1,
                          "roots": -1}[shape] for i in range(n)] for _ in range(b)], np.int32)
    count = np.array([n, 0, max(1, n // 2), max(0, n - 1)], np.int32)
    base = np.array([0, 5, 2 ** 31 - 1 - n, -3], np.int32)
    mask, pos, ws = _build(parents, i32(count), i32(np.stack([base, base], 1))[:, 1])
    assert mkv.mkv_get_device_error(ws)[0] == 0
    sees = R.visible(parents, count)
    np.testing.assert_array_equal(mask, R.words(sees, n))
    np.testing.assert_array_equal(pos, base[:, None] + np.array([[max(0, len(s) - 1) for s in r] for r in sees]))


def test_build_without_options():
    parents = np.array([[-1, 0, 0, 1, 3]], np.int32)
    mask, _, ws = _build(parents, pos=False)
    assert mkv.mkv_get_device_error(ws)[0] == 0
    assert mask[0, :, 0].tolist() == [1, 3, 5, 11, 27]
    _, pos, _ = _build(parents)
    assert pos[0].tolist() == [0, 1, 1, 2, 3]


@pytest.mark.parametrize("bad", [2, 7, -2, 2 ** 31 - 1, -2 ** 31])
def test_build_takes_a_wrong_parent_for_none_and_records_it(bad):
    parents = np.array([[-1, 0, 1], [-1, 0, bad], [-1, -1, 1]], np.int32)
    mask, pos, ws = _build(parents)
    assert mkv.mkv_get_device_error(ws) == (1, 1)
    assert mask[..., 0].tolist() == [[1, 3, 7], [1, 3, 4], [1, 2, 6]] and pos[1].tolist() == [0, 1, 0]


@pytest.mark.parametrize("bad", [4, -1])
def test_build_records_a_wrong_count(bad):
    mask, _, ws = _build(np.array([[-1, 0, 1]], np.int32), i32(np.array([bad])))
    assert mkv.mkv_get_device_error(ws) == (1, 0)
    assert mask[0, :, 0].tolist() == ([1, 3, 7] if bad > 0 else [0, 0, 0])


# ------------------------------------------------------------------ commit
def _commit_case(seed, b, h, d, layers, n, most, rows, strided=False):
    rng = np.random.default_rng(seed)
    torch.manual_seed(seed)
    g = mkv.geom(b, h, 2, d)
    made = []
    for _ in range(layers):
        cache = mkv.alloc_cache(g, rows + most)
        cache.K.copy_(torch.randn(cache.K.shape))
        cache.V.copy_(torch.randn(cache.V.shape))
        cache.pos.copy_(torch.randint(0, 1000, cache.pos.shape))
        cache.len.copy_(torch.randint(0, rows + 1, (b, h)))
        cache.seen.copy_(torch.randint(1000, 5000, (b, h)))
        if strided:
            kv = torch.randn(b, n + 1, 2 * h + 1, d, device="cuda").bfloat16()
            made.append((cache, kv[:, 1:, :h], kv[:, 1:, h:2 * h]))
        else:
            made.append((cache, torch.randn(b, n, h, d, device="cuda").bfloat16(),
                         torch.randn(b, n, h, d, device="cuda").bfloat16()))
    path = rng.integers(0, n, (b, most)).astype(np.int32)
    taken = rng.integers(0, most + 1, b).astype(np.int32)
    return g, made, path, taken


def _snapshot(cache):
    return [x.cpu().clone() for x in (cache.K, cache.V, cache.pos, cache.len, cache.seen)]


def _expected(before, k, v, path, taken, skip=()):
    K, V, pos, length, seen = (x.clone() for x in before)
    for bi in range(K.shape[0]):
        for hi in range(K.shape[1]):
            if (bi, hi) in skip or bi in skip:
                continue
            at = int(length[bi, hi])
            for j in range(int(taken[bi])):
                K[bi, hi, at + j], V[bi, hi, at + j] = k[bi, path[bi, j], hi].cpu(), v[bi, path[bi, j], hi].cpu()
                pos[bi, hi, at + j] = int(seen[bi, hi]) + j
            length[bi, hi] += int(taken[bi])
            seen[bi, hi] += int(taken[bi])
    return K, V, pos, length, seen


@pytest.mark.parametrize("b,h,d,layers,n,most,rows,strided", [
    (1, 1, 64, 1, 1, 1, 0, False), (2, 3, 128, 3, 7, 5, 20, True), (4, 8, 128, 36, 64, 6, 30, False),
    (3, 2, 64, 33, 9, 9, 10, True), (2, 1, 128, 2, 256, 256, 40, False), (70, 8, 64, 2, 5, 3, 9, False)])
def test_commit(b, h, d, layers, n, most, rows, strided):
    g, made, path, taken = _commit_case(b + n, b, h, d, layers, n, most, rows, strided)
    before = [_snapshot(c) for c, _, _ in made]
    ws = mkv.alloc_workspace(256)
    mkv.mkv_tree_commit(g, mkv.tree_layers(made), i32(path), i32(taken), ws)
    assert mkv.mkv_get_device_error(ws)[0] == 0
    for (cache, k, v), was in zip(made, before):
        for got, want in zip(_snapshot(cache), _expected(was, k, v, path, taken)):
            assert torch.equal(got, want)


def test_commit_leaves_units_that_do_not_fit():
    g, made, path, taken = _commit_case(5, 2, 2, 64, 2, 6, 4, 10)
    taken[:] = 4
    cache = made[1][0]
    cache.len.copy_(torch.tensor([[10, 11], [2, 3]]))  # 11 + 4 rows do not fit 14
    made[0][0].len.fill_(3)
    before = [_snapshot(c) for c, _, _ in made]
    ws = mkv.alloc_workspace(256)
    mkv.mkv_tree_commit(g, mkv.tree_layers(made), i32(path), i32(taken), ws)
    assert mkv.mkv_get_device_error(ws) == (3, 1)
    for (c, k, v), was, skip in zip(made, before, [(), ((0, 1),)]):
        for got, want in zip(_snapshot(c), _expected(was, k, v, path, taken, skip)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("what,value", [("path", 6), ("path", -1), ("taken", 5), ("taken", -1)])
def test_commit_leaves_items_with_wrong_paths(what, value):
    g, made, path, taken = _commit_case(6, 2, 1, 64, 1, 6, 4, 10)
    taken[:] = 3
    made[0][0].len.fill_(5)
    if what == "path":
        path[1, 2] = value
    else:
        taken[1] = value
    before = _snapshot(made[0][0])
    ws = mkv.alloc_workspace(256)
    mkv.mkv_tree_commit(g, mkv.tree_layers(made), i32(path), i32(taken), ws)
    assert mkv.mkv_get_device_error(ws) == (1, 1)
    for got, want in zip(_snapshot(made[0][0]), _expected(before, *made[0][1:], path, taken, skip=(1,))):
        assert torch.equal(got, want)
    # a wrong entry past the path's end is not read
    path[1, :], taken[1] = [0, 1, 2, 99], 3
    before = _snapshot(made[0][0])
    mkv.mkv_tree_commit(g, mkv.tree_layers(made), i32(path), i32(taken), ws)
    assert mkv.mkv_get_device_error(ws)[0] == 0
    for got, want in zip(_snapshot(made[0][0]), _expected(before, *made[0][1:], path, taken)):
        assert torch.equal(got, want)


# -------------------------------------------------------------------- rope
# One rounding to bf16 (8 significant bits: 2^-8 of the result) of fp32 products whose sine and
# cosine are off by at most 2^-20 (sum of two products: 2^-19 of the pair's norm).
def _rope_close(got, ref, x, m, neighbours):
    x = np.abs(x)
    pair = np.zeros_like(ref)
    for f in range(m):
        a, c = (2 * f, 2 * f + 1) if neighbours else (f, f + m)
        pair[..., a] = pair[..., c] = np.hypot(x[..., a], x[..., c])
    err = np.abs(got.astype(np.float64) - ref)
    assert (err <= 1.001 * 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * pair).all(), err.max()


def _freqs(rot, base=1e6):
    return (base ** (-np.arange(rot // 2) * 2.0 / rot)).astype(np.float32)


@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 48), (128, 16), (64, 64), (64, 16)])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("axes,tokens,b", [(1, 1, 1), (3, 37, 2), (2, 5, 3), (4, 130, 1)])
def test_rope(d, rot, neighbours, axes, tokens, b):
    rng = np.random.default_rng(rot + tokens)
    heads = (5, 2)
    inv = _freqs(rot)
    axis = rng.integers(0, axes, rot // 2)
    axis[-1] = axes - 1
    pos = rng.integers(0, 5000, (axes, b, tokens)).astype(np.int32)
    xs = [bf16_round(rng.standard_normal((b, tokens, h, d))) for h in heads]
    p = mkv.rope_params(inv, axis, neighbours)
    for inverse in (False, True):
        dev = [bf16(x) for x in xs]
        outs = [torch.full_like(x, 9) for x in dev]
        mkv.mkv_rope(i32(pos), p, list(zip(dev, outs)), inverse=inverse)
        for x, y, was in zip(xs, outs, dev):
            ref = R.rotate(x, pos, inv, axis, neighbours, inverse)
            _rope_close(host(y), ref, x, rot // 2, neighbours)
            np.testing.assert_array_equal(host(y)[..., rot:], x[..., rot:])
            np.testing.assert_array_equal(host(was), x)
        # in place: the same bits
        mkv.mkv_rope(i32(pos), p, [(x, x) for x in dev], inverse=inverse)
        for x, y in zip(dev, outs):
            assert torch.equal(x, y)


@pytest.mark.parametrize("where", [131071, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, -77])
def test_rope_far_positions(where):
    """The angle keeps its digits at every position (a product in 32 bits has none left at 2^24)."""
    rng = np.random.default_rng(1)
    inv = _freqs(64, 1e4)
    inv[3:7] = 3.25, -0.5, 0.0, 1000.25
    pos = np.array([[[where]]], np.int32)
    x = bf16_round(rng.standard_normal((1, 1, 3, 64)))
    dx = bf16(x)
    mkv.mkv_rope(i32(pos), mkv.rope_params(inv), [(dx, dx)])
    # the reference's own product in 64 bits loses 2^-53 of up to 2^31 radians
    _rope_close(host(dx), R.rotate(x, pos, inv, np.zeros(32, int), False, False), x, 32, False)


def test_rope_layouts():
    """Projections behind one another in, head-major keys out (what mkv_compress reads), and back."""
    b, t, h, g, d = 2, 33, 3, 4, 128
    qk = torch.randn(b, t, h * (g + 1), d, device="cuda").bfloat16()
    q, k = qk[:, :, :h * g], qk[:, :, h * g:]
    pos = torch.arange(t, dtype=torch.int32, device="cuda").expand(3, b, t)  # the same on every axis and item
    inv = _freqs(d)
    p = mkv.rope_params(inv, np.arange(d // 2) % 3)
    q2, k2 = torch.empty(b, t, h * g, d, dtype=torch.bfloat16, device="cuda"), torch.empty(b, h, t, d, dtype=torch.bfloat16, device="cuda")
    mkv.mkv_rope(pos, p, [(q, q2), (k, k2.transpose(1, 2))])
    for x, y in ((q, q2), (k, k2.transpose(1, 2))):
        x = host(x)
        _rope_close(host(y), R.rotate(x, pos.cpu().numpy(), inv, np.arange(64) % 3, False, False), x, 64, False)
    # there and back: two roundings (each at most 2^-8 of a component, of a pair at most 2^-8 of its norm)
    back = torch.empty_like(qk)
    mkv.mkv_rope(pos, p, [(q2, back[:, :, :h * g]), (k2.transpose(1, 2), back[:, :, h * g:])], inverse=True)
    pair = torch.hypot(qk[..., :64].float(), qk[..., 64:].float()).repeat(1, 1, 1, 2)
    assert ((back.float() - qk.float()).abs() <= 2.0 ** -7 * 1.01 * pair + 1e-6).all()


def test_rope_gradient():
    """The inverse call is the transpose of the rotation: its product with a cotangent is the directional
    derivative of <cotangent, rope(x)> by differences."""
    rng = np.random.default_rng(4)
    b, t, h, d = 1, 9, 2, 64
    inv, axis = _freqs(48), np.arange(24) % 2
    pos = rng.integers(0, 300, (2, b, t)).astype(np.int32)
    x, w = rng.standard_normal((b, t, h, d)), bf16_round(rng.standard_normal((b, t, h, d)))
    p = mkv.rope_params(inv, axis, True)
    dw, grad = bf16(w), torch.empty(b, t, h, d, dtype=torch.bfloat16, device="cuda")
    mkv.mkv_rope(i32(pos), p, [(dw, grad)], inverse=True)
    got = host(grad).astype(np.float64)

    def value(y):
        return (w * R.rotate(y, pos, inv, axis, True, False)).sum()

    eps = 1e-4
    for _ in range(40):
        at = tuple(rng.integers(0, s) for s in x.shape)
        step = np.zeros_like(x)
        step[at] = eps
        diff = (value(x + step) - value(x - step)) / (2 * eps)  # exact for a linear map, to 1e-9
        assert abs(got[at] - diff) <= 1.001 * 2.0 ** -8 * abs(diff) + 2.0 ** -19 * np.abs(w).max() * 2 + 1e-8


def test_rope_of_no_tokens_and_far_offsets():
    p = mkv.rope_params(_freqs(64))
    e = torch.empty(2, 0, 3, 64, dtype=torch.bfloat16, device="cuda")
    mkv.mkv_rope(torch.empty(1, 2, 0, dtype=torch.int32, device="cuda"), p, [(e, e)])
    # tokens more than 2^31 elements apart
    big = torch.empty(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((1, 2, 2, 64), (0, 2 ** 31 + 1024, 64, 1))
    v = bf16_round(np.random.default_rng(2).standard_normal((1, 2, 2, 64)))
    x.copy_(bf16(v))
    pos = np.array([[[3, 4]]], np.int32)
    mkv.mkv_rope(i32(pos), p, [(x, x)])
    _rope_close(host(x), R.rotate(v, pos, _freqs(64), np.zeros(32, int), False, False), v, 32, False)


def test_rope_many_heads_and_tensors():
    rng = np.random.default_rng(7)
    inv = _freqs(128)
    pos = rng.integers(0, 100, (1, 2, 11)).astype(np.int32)
    for heads in ([1], [64, 8], [1, 2, 3, 5], [128]):
        xs = [bf16_round(rng.standard_normal((2, 11, h, 128))) for h in heads]
        dev = [bf16(x) for x in xs]
        mkv.mkv_rope(i32(pos), mkv.rope_params(inv), [(x, x) for x in dev])
        for x, y in zip(xs, dev):
            _rope_close(host(y), R.rotate(x, pos, inv, np.zeros(64, int), False, False), x, 64, False)
