"""mkv_beam_select and mkv_beam_reorder on the GPU against plain 64-bit forms.

Selection: a score's error is that of the joined fp32 terms (a few units of
2^-23 of the sum, 5e-7 after the log) and of its one rounding to fp32 (2^-24 of it).
Choices must be equal wherever the order's gaps are above 2e-6, which is checked for the inputs of each case."""
import numpy as np
import pytest
import torch

import beam_ref as R
from paper_2606_01563_gb300 import mkv
from gpu_util import host

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
INVALID, CAPACITY = 1, 3


def _select(logits, score, done, end, out, ws=None, **kw):
    b, k, v = logits.shape
    t = [torch.full((b, out), 99, dtype=I32, device="cuda") for _ in range(3)]
    best = torch.full((b, out), 99.0, device="cuda")
    if ws is None:
        ws = mkv.alloc_workspace(mkv.mkv_beam_select_workspace_size(b, k, v, out))
        ws[256:] = 255  # (only the error word has to be zero)
    mkv.mkv_beam_select(logits, score, t[0], t[1], best, ws, done=done, done_out=t[2], end_token=end, **kw)
    return t[0], t[1], best, t[2], ws


def _check(logits, score, done, end, out, error=0):
    parent, token, best, over, ws = _select(logits, score, done, end, out)
    rp, rt, rs, ro, gap = R.select(host(logits), host(score), None if done is None else host(done), end, out)
    assert gap > 2e-6, gap
    assert (host(parent) == rp).all() and (host(token) == rt).all() and (host(over) == ro).all()
    got, fine = host(best).astype(np.float64), np.isfinite(rs)
    assert (got[~fine] == rs[~fine]).all()
    assert (np.abs(got[fine] - rs[fine]) <= 5e-7 + 2.0 ** -24 * np.abs(rs[fine])).all()
    assert mkv.mkv_get_device_error(ws)[0] == error
    return parent, token, best


def _inputs(b, k, v, dtype, seed, padded=0, spread=3.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = (spread * torch.randn(b, k, v + padded, generator=gen, device="cuda")).to(dtype)[:, :, :v]
    return x, -5 * torch.rand(b, k, generator=gen, device="cuda"), gen


SELECT = [  # batch, beams, vocab, n_out, type, padding, ended beams
    (1, 1, 1, 1, F32, 0, 0), (1, 1, 2, 4, BF16, 0, 0), (3, 2, 7, 5, F32, 1, 1), (2, 4, 33, 8, BF16, 3, 1),
    (1, 5, 1000, 5, BF16, 0, 1), (2, 3, 8192, 6, F32, 0, 0), (2, 8, 8193, 16, BF16, 7, 1), (1, 1, 100003, 64, F32, 0, 0),
    (1, 64, 20011, 64, BF16, 0, 1), (40, 8, 5001, 16, F32, 2, 1), (5, 64, 700, 33, BF16, 1, 1), (1, 4, 262144, 8, BF16, 0, 0),
    (700, 2, 1025, 2, BF16, 0, 1),
]


@pytest.mark.parametrize("b,k,v,out,dtype,padded,ended", SELECT)
def test_select(b, k, v, out, dtype, padded, ended):
    logits, score, gen = _inputs(b, k, v, dtype, v + k, padded)
    done = (torch.rand(b, k, generator=gen, device="cuda") < 0.3).to(I32) if ended else None
    _check(logits, score, done, min(2, v - 1), out)


@pytest.mark.parametrize("v,out", [(30011, 64), (30011, 5), (9000, 33)])
@pytest.mark.parametrize("order", ["same", "ascending", "descending", "zeros of both signs", "one high run"])
def test_select_orders_that_fill_lists(v, out, order):
    """Logits of which many or all pass a list's bound, equal ones by the lower token; two beams of equal scores."""
    x = torch.zeros(1, 2, v, device="cuda")
    i = torch.arange(v, device="cuda", dtype=F32)
    if order == "ascending":
        x[:] = i / 16384 * 8
    elif order == "descending":
        x[:] = -i / 16384 * 8
    elif order == "zeros of both signs":
        x[..., ::3] = -0.0
    elif order == "one high run":
        x[..., 5000:5000 + 2 * out] = 3
    _check(x, torch.full((1, 2), -1.5, device="cuda"), None, -1, out)
    _check(x.to(BF16), torch.full((1, 2), -1.5, device="cuda"), None, 7, out)


@pytest.mark.parametrize("dtype,sizes", [(BF16, range(521, 577, 5)), (F32, range(257, 289, 3))])
def test_select_vocabularies_of_one_chunk_in_part_of_a_block(dtype, sizes):
    """One vector of 16 bytes in each of 65 to 72 threads: what they add decides whether it had fitted."""
    for v in sizes:
        logits, score, _ = _inputs(1, 2, v, dtype, v, padded=-v % 8)
        _check(logits, score, None, 2, 64)


@pytest.mark.parametrize("threads", range(64, 74))
def test_select_masks_that_leave_some_threads_a_token(threads):
    """A chunk in which as many threads have one permitted token, of several chunks."""
    v = 3 * 2048 + 1000
    logits, score, _ = _inputs(1, 2, v, BF16, threads, padded=8 - v % 8)
    at = torch.arange(threads, device="cuda") * 8
    mask = torch.full((v,), -float("inf"), device="cuda")
    for chunk in range(3):
        mask[chunk * 2048 + at + chunk] = 0
    _check(logits + mask.to(BF16), score, None, -1, 64)


@pytest.mark.parametrize("out", [48, 56, 64])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_many_blocks_with_long_lists(out, dtype):
    """48 batch items with the same logits and scores: the same bits of each, on every call.  Against one item's call
    the scores are within twice the bound (that call cuts its runs elsewhere, so its sums round differently)."""
    logits, score, _ = _inputs(1, 8, 20000, dtype, out)
    p, t, s = _check(logits, score, None, 2, out)
    first = None
    for _ in range(20):
        got = _select(logits.expand(48, -1, -1), score.expand(48, -1).contiguous(), None, 2, out)
        assert (got[0] == p).all() and (got[1] == t).all()
        assert ((got[2] - s).abs() <= 2 * (5e-7 + 2.0 ** -24 * s.abs())).all()
        first = got[2][:1] if first is None else first
        assert (got[2] == first).all()
        assert mkv.mkv_get_device_error(got[4])[0] == 0


def test_select_first_step_and_masks():
    """Beams that are not alive, tokens that are forbidden, and items with fewer continuations than slots."""
    logits, score, _ = _inputs(4, 4, 300, F32, 11)
    score[:, 1:] = -float("inf")
    logits[1, 0, 6:] = -float("inf")
    logits[2] = -float("inf")  # nothing but forbidden tokens
    score[3] = -float("inf")   # nobody alive
    logits[3, 1] = float("nan")  # (not read)
    p, t, _ = _check(logits, score, None, 3, 10)
    assert (p[1, 6:] == -1).all() and (p[2:] == -1).all() and (t[2:] == -1).all() and (p[0] == 0).all()
    _check(torch.finfo(F32).min * torch.ones_like(logits[:1]), score[:1], None, 3, 4)  # the type's lowest value
    done = torch.ones(1, 4, dtype=I32, device="cuda")  # all have ended: four continuations
    _check(logits[:1] * float("nan"), torch.tensor([[-4.0, -1.0, -2.5, -9.0]], device="cuda"), done, 299, 10)


def test_select_values_that_are_not_finite_are_recorded():
    for bad, row in ((float("nan"), 3), (float("inf"), 1)):
        logits, score, _ = _inputs(2, 3, 9000, BF16, 5)
        logits.view(6, -1)[row, 8500] = bad
        _check(logits, score, None, 2, 6, error=INVALID)
    logits, score, _ = _inputs(2, 3, 900, BF16, 6)
    for bad in (float("nan"), float("inf")):
        score[1, 2] = bad
        *_, ws = _select(logits, score, None, 2, 6)
        assert mkv.mkv_get_device_error(ws) == (INVALID, 5)
        _check(logits, score, None, 2, 6, error=INVALID)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_select_a_score_that_is_not_finite_of_a_beam_that_has_ended(bad):
    logits, score, _ = _inputs(2, 3, 900, BF16, 7)
    logits[1, 1] = float("nan")  # (an ended beam's logits do not matter)
    done = torch.tensor([[0, 0, 0], [0, 1, 1]], dtype=I32, device="cuda")
    _check(logits, score, done, 2, 6)
    score[1, 2] = bad
    *_, ws = _select(logits, score, done, 2, 6)
    assert mkv.mkv_get_device_error(ws) == (INVALID, 5)
    _check(logits, score, done, 2, 6, error=INVALID)


def test_select_a_nan_among_forbidden_tokens_before_the_first_logit():
    """A run's first 2048 tokens are forbidden but for a NaN, which what comes after must not hide."""
    for nan in (float("nan"), -float("nan")):
        logits, score, _ = _inputs(100, 8, 5001, F32, 17)
        logits[1, 3, :2048] = -float("inf")
        logits[1, 3, 5] = nan
        *_, ws = _select(logits, score, None, 2, 6)
        assert mkv.mkv_get_device_error(ws) == (INVALID, 11)
        _check(logits, score, None, 2, 6, error=INVALID)


def test_select_odd_addresses_strides_and_offsets_past_32_bits():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    for dtype in (BF16, F32):
        flat = torch.randn(40000, generator=gen, device="cuda").to(dtype)
        for shift in (1, 3, 5):
            view = flat[shift:shift + 2 * 3 * 5001].view(2, 3, 5001)
            _check(view, -torch.rand(2, 3, generator=gen, device="cuda"), None, 2, 7)
    one = torch.randn(1, 1, 4001, generator=gen, device="cuda")
    _check(one.expand(2, 3, -1), -torch.rand(2, 3, generator=gen, device="cuda"), None, 2, 7)  # shared logits
    far = 2 ** 31 + 8
    big = torch.empty(far + 20000, dtype=BF16, device="cuda")
    view = big.as_strided((2, 2, 5000), (far, 5000, 1))
    view.copy_(torch.randn(2, 2, 5000, generator=gen, device="cuda"))
    _check(view, -torch.rand(2, 2, generator=gen, device="cuda"), None, 2, 7)


@pytest.mark.parametrize("beams", [64, 1])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["equal", "random"])
def test_select_sums_over_the_largest_vocabulary(kind, dtype, beams):
    """2^24 tokens: with 64 beams (of the same logits) a thread has 4096 chunks of 16 of them.  Equal logits are the case in
    which the roundings of one running sum in 32 bits add up.

    A term's exponential is off by 2^-22 at most and its exponent by two roundings (2^-23 of at most 8 where it has
    weight: 5e-7 at the least weights, less elsewhere), the 16 terms' sum by seven additions (7 2^-24); nothing else is in 32 bits: 1e-6 in all."""
    v, out = 1 << 24, 6
    gen = torch.Generator(device="cuda")
    gen.manual_seed(v + beams)
    row = torch.full((v,), -0.3, device="cuda") if kind == "equal" else torch.randn(v, generator=gen, device="cuda")
    row = row.to(dtype)
    score = 16.6 - 50 * torch.arange(beams, device="cuda", dtype=F32)[None]  # (the first beam's are the best, near 0)
    parent, token, best, _, ws = _select(row.view(1, 1, v).expand(1, beams, -1), score, None, -1, out)
    x = host(row).astype(np.float64)
    log = float(x.max()) + np.log(np.exp(x - x.max()).sum())
    at = np.flatnonzero(x >= np.partition(x, -out)[-out])
    at = at[np.lexsort((at, -x[at]))][:out]
    want = host(score)[0, 0].astype(np.float64) + (x[at] - log)
    assert (host(parent) == 0).all() and (host(token)[0] == at).all()
    assert (np.abs(host(best)[0] - want) <= 1e-6 + 2.0 ** -24 * np.abs(want)).all(), np.abs(host(best)[0] - want).max()
    assert mkv.mkv_get_device_error(ws)[0] == 0


def test_select_in_place_in_a_graph_on_another_stream():
    b, k, v = 3, 6, 4000
    logits, score, gen = _inputs(b, k, v, BF16, 21)
    done = torch.zeros(b, k, dtype=I32, device="cuda")
    ref = [logits.clone(), score.clone(), done.clone()]
    parent, token = (torch.empty(b, k, dtype=I32, device="cuda") for _ in range(2))
    ws = mkv.alloc_workspace(mkv.mkv_beam_select_workspace_size(b, k, v, k))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        mkv.mkv_beam_select(logits, score, parent, token, score, ws, done=done, done_out=done, end_token=2, stream=side)
    for _ in range(3):
        graph.replay()
        want = R.select(host(ref[0]), host(ref[1]), host(ref[2]), 2, k)
        assert (host(parent) == want[0]).all() and (host(token) == want[1]).all() and (host(done) == want[3]).all()
        assert (np.abs(host(score) - want[2]) <= 5e-7 + 2.0 ** -24 * np.abs(want[2])).all()
        logits.copy_(3 * torch.randn(b, k, v, generator=gen, device="cuda"))
        ref = [logits.clone(), score.clone(), done.clone()]


# ----------------------------------------------------------------- reorder
def _layer(gen, states, h, cap, d, y, moments, ragged=True):
    def rand(*shape, dtype=F32):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    def ints(hi, *shape):
        return torch.randint(0, hi, shape, generator=gen, device="cuda", dtype=I32)
    c = mkv.Cache(rand(states, h, cap, d, dtype=BF16), rand(states, h, cap, d, dtype=BF16), ints(1000, states, h, cap),
                  ints(cap + 1, states, h) if ragged else torch.full((states, h), cap, dtype=I32, device="cuda"), ints(1000, states, h),
                  rand(states, h, cap, d) if y else None, ints(cap + 1, states, h) if y else None)
    m = mkv.Moments(ints(50, states, h), rand(states, h, d), rand(states, h, d), rand(states, h, d, d)) if moments else None
    return c, m


def _fields(c, m):
    rows = [c.K, c.V, c.pos] + ([c.y] if c.y is not None else [])
    whole = [c.len, c.seen] + ([c.y_len] if c.y is not None else []) + ([m.n, m.mu_k, m.mu_v, m.C] if m is not None else [])
    return rows, whole


def _bits(t):
    return (t.view(torch.int16) if t.dtype is BF16 else t).cpu().numpy()


def _reorder_and_check(layers, parent, h, d, error=0, **kw):
    b, n = parent.shape
    want = []
    for c, m in layers:
        rows, whole = _fields(c, m)
        ln, yl = host(c.len), None if c.y is None else host(c.y_len)
        want.append(R.reorder([_bits(t) for t in rows + whole], host(parent), [ln] * 3 + ([yl] if c.y is not None else []) + [None] * len(whole)))
    ws = mkv.alloc_workspace(256)
    mkv.mkv_beam_reorder(mkv.geom(b, h, 1, d), mkv.beam_layers(layers), parent, ws, **kw)
    for (c, m), w in zip(layers, want):
        rows, whole = _fields(c, m)
        for i, (t, x) in enumerate(zip(rows + whole, w)):
            assert (_bits(t) == x).all(), i
    code, info = mkv.mkv_get_device_error(ws)
    assert code == error
    return info


REORDER = [  # layers, batch, N, heads, capacity, dim, y, moments
    (1, 1, 1, 1, 5, 64, 0, 0), (3, 2, 4, 2, 33, 128, 0, 1), (2, 1, 8, 3, 200, 64, 1, 1), (66, 1, 3, 1, 7, 64, 0, 1),
    (1, 3, 37, 2, 65, 128, 1, 0), (1, 1, 256, 1, 90, 64, 1, 1), (2, 5, 16, 8, 1, 128, 0, 0), (1, 1, 2, 1, 3001, 128, 0, 1),
]


@pytest.mark.parametrize("layers,b,n,h,cap,d,y,moments", REORDER)
@pytest.mark.parametrize("kind", ["any", "cycle", "one for all", "pairs exchanged", "stay"])
def test_reorder(layers, b, n, h, cap, d, y, moments, kind):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + cap)
    states = [_layer(gen, b * n, h, cap, d, y, moments) for _ in range(layers)]
    i = torch.arange(n, device="cuda", dtype=I32)
    parent = {"any": lambda: torch.randint(-1, n, (b, n), generator=gen, device="cuda", dtype=I32),
              "cycle": lambda: ((i + 1) % n).expand(b, n), "one for all": lambda: torch.full((b, n), n - 1, dtype=I32, device="cuda"),
              "pairs exchanged": lambda: (i ^ 1).clamp(max=n - 1).expand(b, n), "stay": lambda: torch.full((b, n), -1, dtype=I32, device="cuda")}
    _reorder_and_check(states, parent[kind]().contiguous(), h, d)


def test_reorder_refuses_items_with_bad_parents_and_records_lengths():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    states = [_layer(gen, 12, 2, 20, 64, 1, 1) for _ in range(2)]
    for bad in (4, -2, 2 ** 31 - 1, -2 ** 31):
        parent = torch.randint(0, 4, (3, 4), generator=gen, device="cuda", dtype=I32)
        parent[1, 2] = bad
        assert _reorder_and_check(states, parent, 2, 64, error=INVALID) == 1
    parent = torch.tensor([[1, 0, 2, 3]] * 3, dtype=I32, device="cuda")
    states[0][0].len[5, 1] = 21  # past the capacity: its rows up to the end
    assert _reorder_and_check(states, parent, 2, 64, error=CAPACITY) == 11
    states[0][0].len[4, 1] = 20  # (slot 1's length went to slot 0)
    states[0][0].len[4, 0] = -3
    assert _reorder_and_check(states, parent, 2, 64, error=CAPACITY) == 8


def test_reorder_records_lengths_of_y():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    parent = torch.tensor([[1, 0, 2, 3]] * 3, dtype=I32, device="cuda")
    for slot, bad in ((5, 21), (4, -1), (5, 2 ** 31 - 1), (7, -2 ** 31)):  # (slot 7's state stays)
        states = [_layer(gen, 12, 2, 20, 64, 1, 0) for _ in range(2)]
        states[1][0].y_len[slot, 1] = bad
        assert _reorder_and_check(states, parent, 2, 64, error=CAPACITY) == 2 * slot + 1


def test_reorder_in_a_graph_after_a_selection():
    """Selection and reordering captured together on another stream; each replay permutes what the last one left."""
    b, k, v, h, cap, d = 2, 4, 500, 2, 40, 128
    logits, score, gen = _inputs(b, k, v, F32, 8)
    states = [_layer(gen, b * k, h, cap, d, 0, 1, ragged=False) for _ in range(3)]
    parent, token = (torch.empty(b, k, dtype=I32, device="cuda") for _ in range(2))
    best = torch.empty(b, k, device="cuda")
    ws = mkv.alloc_workspace(mkv.mkv_beam_select_workspace_size(b, k, v, k))
    packed, g = mkv.beam_layers(states), mkv.geom(b, h, 1, d)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        mkv.mkv_beam_select(logits, score, parent, token, best, ws, stream=side)
        mkv.mkv_beam_reorder(g, packed, parent, ws, stream=side)
    for _ in range(3):
        before = [[_bits(t) for t in sum(_fields(*s), [])] for s in states]
        graph.replay()
        for s, old in zip(states, before):
            for t, x in zip(sum(_fields(*s), []), R.reorder(old, host(parent))):
                assert (_bits(t) == x).all()
        logits.copy_(torch.randn(b, k, v, generator=gen, device="cuda"))


def test_tensors_of_another_device_are_refused():
    logits, score, _ = _inputs(1, 2, 50, F32, 1)
    with pytest.raises(ValueError):
        _select(logits.cpu(), score, None, -1, 2)
    c, _ = _layer(torch.Generator(device="cuda"), 2, 1, 4, 64, 0, 0)
    with pytest.raises(ValueError):
        mkv.beam_layers([(mkv.Cache(c.K.cpu(), c.V, c.pos, c.len, c.seen), None)])


def test_reorder_waits_that_run_out_are_recorded():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    states = [_layer(gen, 8, 2, 300, 64, 0, 1)]
    parent = torch.tensor([[1, 2, 3, 0]] * 2, dtype=I32, device="cuda")
    ws, old = mkv.alloc_workspace(256), mkv.mkv_debug_set_poll_limit(0)
    try:
        mkv.mkv_beam_reorder(mkv.geom(2, 2, 1, 64), mkv.beam_layers(states), parent, ws)
        assert mkv.mkv_get_device_error(ws)[0] == 5
    finally:
        mkv.mkv_debug_set_poll_limit(old)
    _reorder_and_check(states, parent, 2, 64)
