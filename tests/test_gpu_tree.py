"""Attention of drafted trees over the cache (mkv_tree_step) against a plain
64-bit form: sizes around every tile edge, all geometries, masks that hide
everything, forms of the moments, strides, unused memory full of NaN, values
that are not finite, and the bounds of tests/tree_ref.py."""
import math

import numpy as np
import pytest
import torch

import tree_ref as R
from paper_2606_01563_gb300 import mkv
from paper_2606_01563_gb300.inputs import bf16_round
from gpu_util import bf16, f32, host, i32

pytestmark = pytest.mark.gpu
TAU = 1e-6


class Case:
    """One layer's cache, moments and drafted nodes, on the host and on the GPU."""

    def __init__(self, seed, b=1, h=2, g=4, d=128, n=5, rows=100, cap=None, c="f32", order=1, masks="tree", ragged=False,
                 spare=float("nan")):
        rng = np.random.default_rng(seed)
        self.geo, self.n, self.c, self.order = (b, h, g, d), n, c, order
        self.g = mkv.geom(b, h, g, d)
        cap = cap or rows + 3
        self.cap = cap
        self.length = np.full((b, h), rows, np.int32)
        self.count = np.full(b, n, np.int32)
        if ragged:
            self.length = rng.integers(0, rows + 1, (b, h)).astype(np.int32)
            self.count = rng.integers(0, n + 1, b).astype(np.int32)
        scale = np.exp(rng.uniform(math.log(0.5), math.log(2.0), (b, h, 1, d)))
        self.K = bf16_round(rng.standard_normal((b, h, cap, d)) * scale)
        self.V = bf16_round(rng.standard_normal((b, h, cap, d)) + 0.25)
        self.q = bf16_round(rng.standard_normal((b, n, h * g, d)))
        self.k = bf16_round(rng.standard_normal((b, n, h, d)) * scale[:, None, :, 0])
        self.v = bf16_round(rng.standard_normal((b, n, h, d)) + 0.25)
        for bi in range(b):  # what is not in use holds anything
            for hi in range(h):
                self.K[bi, hi, self.length[bi, hi]:] = spare
                self.V[bi, hi, self.length[bi, hi]:] = spare
            for x in (self.q, self.k, self.v):
                x[bi, self.count[bi]:] = spare
        self.moments = None
        if c != "none":
            nn = rng.integers(1, 2000, (b, h)).astype(np.int32)
            if b * h > 1:
                nn.reshape(-1)[-1] = 0  # a unit that evicted nothing: its moments are not read
            mk, mv = 0.3 * rng.standard_normal((b, h, d)), 0.3 * rng.standard_normal((b, h, d))
            C = 0.2 * rng.standard_normal((b, h, d, d))
            C[rng.random(C.shape) < 0.05] = 1e-10  # clamped
            mk, mv, C = (x.astype(np.float32) for x in (mk, mv, C))
            if c == "bf16":
                self.C_used = bf16_round(C)
            elif c == "split":  # hi + lo words: 16 to 17 significant bits of the clamped values
                Cc = np.where(np.abs(C * nn[..., None, None].astype(np.float32)) < np.float32(TAU), 0, C)
                hi = bf16_round(Cc)
                self.C_used = hi + bf16_round(Cc - hi)
            else:
                self.C_used = C
            self.moments = (nn, mk, mv, C)
        if masks == "tree":
            parents = np.array([[rng.integers(-1, max(i, 0)) if i else -1 for i in range(n)] for _ in range(b)], np.int32)
            self.sees = R.visible(parents, self.count)
        else:
            see = {"none": lambda i: [], "self": lambda i: [i], "all": lambda i: list(range(n)),
                   "later": lambda i: list(range(i + 1, n)), "odd": lambda i: [a for a in range(n) if a % 2],
                   "random": lambda i: [a for a in range(n) if rng.random() < 0.5]}[masks]
            self.sees = [[see(i) for i in range(n)] for _ in range(b)]
        self.mask = R.words(self.sees, n)
        if n % 32:  # bits past the last node mean nothing
            self.mask[..., -1] |= np.int32(-1) << np.int32(n % 32)
        self.sees = [[[a for a in row if a < m] for row in rows_] for rows_, m in zip(self.sees, self.count.tolist())]

    def device(self, count=True, fused=False):
        b, h, g, d = self.geo
        self.cache = mkv.Cache(bf16(self.K), bf16(self.V), i32(np.zeros((b, h, self.cap))), i32(self.length),
                               i32(self.length + 7))
        self.mom, c16, split = None, None, None
        if self.moments is not None:
            nn, mk, mv, C = self.moments
            self.mom = mkv.Moments(i32(nn), f32(mk), f32(mv), f32(C))
            if self.c == "bf16":
                c16 = torch.empty(b, h, d, d, dtype=torch.bfloat16, device="cuda")
                mkv.mkv_moments_pack_bf16(self.g, self.mom, c16)
            if self.c == "split":
                split = torch.empty(b, h, d, d, dtype=torch.int32, device="cuda")
                mkv.mkv_moments_pack_split(self.g, self.mom, TAU, split)
        self.p = mkv.mkv_decode_params(0 if self.mom is None else 1, self.order, TAU,
                                       None if c16 is None else c16.data_ptr(), 0,
                                       None if split is None else split.data_ptr())
        self.held = (c16, split)
        self.tree = mkv.Tree(i32(self.mask), i32(self.count) if count else None)
        self.dq, self.dk, self.dv = bf16(self.q), bf16(self.k), bf16(self.v)
        if fused:  # one projection's output, batch items and nodes padded
            pad = torch.full((b, self.n + 3, h * (g + 2) + 1, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            x = pad[:, :self.n]
            x[:, :, :h * g], x[:, :, h * g:h * (g + 1)], x[:, :, h * (g + 1):-1] = self.dq, self.dk, self.dv
            self.dq, self.dk, self.dv = x[:, :, :h * g], x[:, :, h * g:h * (g + 1)], x[:, :, h * (g + 1):-1]
        self.out = torch.full((b, self.n, h * g, d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((b, self.n, h * g), 7.0, device="cuda")
        self.ws = mkv.alloc_workspace(mkv.mkv_tree_workspace_size(self.g, self.n, self.cap))
        return self

    def step(self, lse=True, stream=None):
        mkv.mkv_tree_step(self.g, self.tree, self.dq, self.dk, self.dv, self.cache, self.mom, self.p, self.out,
                          self.lse if lse else None, self.ws, stream=stream)

    def check(self, own_sum=False):
        """own_sum: the bound of the kernel's normaliser, the sum of the rounded weights: sum w (1 + d) v / sum w (1 + d)
        differs from sum w v by sum w d (v - out) to first order, at most 2^-8 (A + |out|) where the unrounded sum gives 2^-8 A."""
        assert mkv.mkv_get_device_error(self.ws)[0] == 0
        moments = None if self.moments is None else (*self.moments[:3], self.C_used)
        out, lse, tol, tol_lse = R.attend(self.q, self.k, self.v, self.sees, self.K, self.V, self.length, moments,
                                          self.order, TAU, self.count)
        got, got_lse = host(self.out).astype(np.float64), host(self.lse).astype(np.float64)
        nothing = np.isneginf(lse)
        assert (np.isneginf(got_lse) == nothing).all()
        assert (got[nothing] == 0).all()
        err = np.abs(got - out)
        if own_sum:
            tol = tol + 1.001 * 2.0 ** -8 * np.abs(out)
        assert np.isfinite(got).all()
        assert (err <= tol).all(), f"out: {np.max(err - tol)} over its bound, at {np.argwhere(err > tol)[:4].tolist()}"
        err = np.abs(got_lse[~nothing] - lse[~nothing])
        assert (err <= tol_lse[~nothing]).all(), f"lse: {err.max()}"

    def run(self, **kw):
        self.device(**kw).step()
        self.check()
        return self


@pytest.mark.parametrize("n", [1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256])
def test_node_counts(n):
    Case(n, h=1, g=2 if n > 100 else 4, n=n, rows=70).run()


@pytest.mark.parametrize("rows", [0, 1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 500, 1025])
@pytest.mark.parametrize("c", ["none", "f32"])
def test_cache_lengths(rows, c):
    Case(rows + 1, h=2, n=6, rows=rows, c=c).run()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 2, 4, 8])
@pytest.mark.parametrize("c,order", [("none", 1), ("f32", 1), ("f32", 0), ("bf16", 1), ("split", 1)])
def test_geometries_and_moment_forms(d, g, c, order):
    Case(g + d, b=2, h=3, g=g, d=d, n=21, rows=150, c=c, order=order, ragged=True).run()


@pytest.mark.parametrize("masks", ["none", "self", "all", "later", "odd", "random"])
@pytest.mark.parametrize("rows,c", [(0, "none"), (0, "f32"), (90, "none"), (200, "split")])
def test_masks(masks, rows, c):
    Case(3, h=2, n=37, rows=rows, c=c, masks=masks).run()


@pytest.mark.parametrize("masks", ["all", "random"])
def test_wide_masks(masks):
    Case(4, h=1, g=1, n=256, rows=3, c="none", masks=masks).run()
    Case(5, h=1, g=8, n=150, rows=0, c="none", masks=masks).run()


@pytest.mark.parametrize("seed", range(6))
def test_ragged_batches(seed):
    Case(seed, b=5, h=3, g=4, n=[1, 9, 33, 64, 70, 130][seed], rows=[5, 400, 130, 700, 64, 260][seed],
         c=["f32", "none", "split", "bf16", "f32", "none"][seed], ragged=True).run()


def test_many_units():
    """More units than SMs, of unequal lengths."""
    Case(11, b=40, h=8, g=1, d=64, n=3, rows=300, c="f32", ragged=True).run()


def test_long_cache_of_few_units():
    Case(12, b=1, h=1, g=4, n=8, rows=20000, c="f32").run()
    Case(13, b=1, h=2, g=8, n=40, rows=5003, c="none").run()


def test_capacity_far_above_the_length():
    """The split is made for the length, not the capacity."""
    Case(14, b=2, h=2, n=7, rows=40, cap=9000, c="f32").run()


def test_offsets_past_32_bits():
    b, h, d = 1, 9, 128
    cap = 2 ** 31 // (8 * d) + 64
    c = Case(15, b=b, h=h, g=2, d=d, n=4, rows=200, c="none").device()
    K = torch.empty(b, h, cap, d, dtype=torch.bfloat16, device="cuda")
    V = torch.empty(b, h, cap, d, dtype=torch.bfloat16, device="cuda")
    K[:, :, :203], V[:, :, :203] = c.cache.K, c.cache.V
    c.cache.K, c.cache.V = K, V
    c.ws = mkv.alloc_workspace(mkv.mkv_tree_workspace_size(c.g, c.n, cap))
    c.step()
    c.check()


@pytest.mark.parametrize("n", [1, 30])
def test_strided_nodes(n):
    Case(16, b=3, h=2, n=n, rows=77, ragged=n > 1).run(fused=True)


def test_without_count_and_lse():
    c = Case(17, b=2, n=9, rows=140).device(count=False)
    c.step(lse=False)
    assert (c.lse == 7.0).all()
    c.step()
    c.check()


def test_not_finite_values_reach_only_who_sees_them():
    """A node whose value is infinite or NaN, and one whose key is: the rows that see it follow the formula, the
    others are those of finite nodes."""
    clean = Case(18, h=2, n=40, rows=150, masks="random", c="f32").run()
    bad = Case(18, h=2, n=40, rows=150, masks="random", c="f32")
    bad.v[0, 5, 0, 3] = np.inf
    bad.v[0, 17, 0, 3] = -np.inf
    bad.v[0, 29, 1, 100] = np.nan
    bad.k[0, 33, 0, 8] = np.nan
    bad.device().step()
    assert mkv.mkv_get_device_error(bad.ws)[0] == 0
    got, ref = host(bad.out), host(clean.out)
    lse, ref_lse = host(bad.lse), host(clean.lse)
    for i in range(40):
        s = set(bad.sees[0][i])
        first = got[0, i, :4]  # query heads of KV head 0
        if 33 in s:
            assert np.isnan(first).all() and np.isnan(lse[0, i, :4]).all()
        else:
            want = ref[0, i, :4].copy()
            if 5 in s and 17 in s:
                want[:, 3] = np.nan
            elif 5 in s:
                want[:, 3] = np.inf
            elif 17 in s:
                want[:, 3] = -np.inf
            np.testing.assert_array_equal(first, want)
            np.testing.assert_array_equal(lse[0, i, :4], ref_lse[0, i, :4])
        want = ref[0, i, 4:].copy()
        if 29 in s:
            want[:, 100] = np.nan
        np.testing.assert_array_equal(got[0, i, 4:], want)
        np.testing.assert_array_equal(lse[0, i, 4:], ref_lse[0, i, 4:])


def test_large_scores():
    """Scores of hundreds: one key takes all the weight, and the reference moves from tile to tile."""
    c = Case(19, h=2, n=20, rows=600, c="f32")
    c.K[0, :, :600] *= 8
    c.K[0, :, :600] *= np.linspace(0.1, 2, 600)[None, :, None]
    c.K = bf16_round(c.K)
    c.q = bf16_round(c.q * 4)
    c.run()


def test_same_call_same_bits():
    c = Case(20, b=2, h=3, n=50, rows=900, ragged=True).run()
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(5):
        c.out.fill_(3)
        c.step()
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    c.check()


def test_single_chain_equals_decode_steps():
    """Nodes in a chain give what decoding them one by one gives, to bf16."""
    c = Case(21, h=2, n=4, rows=130, c="f32")
    c.sees = [[list(range(i + 1)) for i in range(4)]]
    c.mask = R.words(c.sees, 4)
    c.run()
    _, h, g, d = c.geo
    ws = mkv.alloc_workspace(mkv.mkv_decode_workspace_size(c.g, c.cap + 8))
    cache = mkv.alloc_cache(c.g, c.cap + 8)
    cache.K[:, :, :130], cache.V[:, :, :130] = c.cache.K[:, :, :130], c.cache.V[:, :, :130]
    cache.len.fill_(130)
    for i in range(4):
        out, lse = torch.empty(1, h * g, d, device="cuda"), torch.empty(1, h * g, device="cuda")
        mkv.mkv_decode_step(c.g, c.dq[:, i].contiguous(), c.dk[:, i].contiguous(), c.dv[:, i].contiguous(), cache, c.mom,
                            c.p, out, lse, ws)
        # the weights' and the output's roundings to bf16: 2^-8 of the mean magnitude of the values (below 1.5)
        # and of the output
        assert ((c.out[:, i].float() - out).abs() <= 2 ** -8 * (1.5 + out.abs())).all()
        torch.testing.assert_close(c.lse[:, i], lse, rtol=0, atol=1e-4)


def test_other_stream_and_graph():
    c = Case(22, b=2, n=30, rows=300, ragged=True).device()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.step()
    s.synchronize()
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for _ in range(3):
            c.step()
    c.out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    c.check()


def test_layer_chain_with_early_loads():
    """Layers one after another on their own caches, each launch released into the one before; two passes reuse the
    workspace."""
    cases = [Case(30 + i, b=2, h=4, n=20, rows=200 + 37 * i, c="f32", ragged=True).device() for i in range(6)]
    ws = max((c.ws for c in cases), key=lambda w: w.numel())
    for c in cases:
        c.p.early_load = 1
        c.ws = ws
    torch.cuda.synchronize()
    for _ in range(2):
        for c in cases:
            c.step()
    for c in cases:
        c.check()


def test_corrupt_lengths_and_counts_are_recorded():
    c = Case(23, b=2, h=2, n=5, rows=50, spare=0.0).device()
    c.cache.len[1, 0] = c.cap + 5
    c.step()
    assert mkv.mkv_get_device_error(c.ws) == (3, 2)
    c.cache.len[1, 0] = -4
    c.step()
    assert mkv.mkv_get_device_error(c.ws) == (3, 2)
    c.cache.len[1, 0] = 50
    c.tree.count[1] = 6
    c.step()
    code, unit = mkv.mkv_get_device_error(c.ws)
    assert code == 1 and unit in (2, 3)
    c.check()  # taken as all nodes
    c.tree.count[1] = 5
    c.step()
    c.check()


@pytest.mark.parametrize("rows,b,h,n", [(300, 1, 2, 9), (9000, 1, 2, 20), (2000, 2, 2, 100), (700, 30, 8, 40)])
def test_waits_that_run_out_are_reported_and_leave_the_context_usable(rows, b, h, n):
    """One item per CTA, the list of tiles with its merge, two row blocks, many items: with the poll limit at zero the
    first wait of every CTA gives up, and the same call is right again afterwards."""
    c = Case(rows, b=b, h=h, n=n, rows=rows, c="f32").device()
    default = mkv.mkv_debug_set_poll_limit(0)
    try:
        c.step()
        assert mkv.mkv_get_device_error(c.ws)[0] == 5
    finally:
        assert mkv.mkv_debug_set_poll_limit(default) == 0
    for _ in range(2):
        c.step()
    c.check()


@pytest.mark.parametrize("b,h,g,d,n,rows,c", [
    (1, 8, 4, 128, 33, 4200, "none"), (1, 8, 4, 128, 64, 9000, "f32"), (2, 5, 8, 64, 70, 3000, "split"),
    (1, 3, 1, 128, 256, 2500, "bf16"), (20, 8, 2, 64, 12, 2000, "f32"), (1, 1, 8, 128, 256, 700, "f32"),
    (3, 8, 4, 128, 40, 1500, "f32"), (25, 8, 4, 64, 40, 1300, "none")])
def test_every_plan(b, h, g, d, n, rows, c):
    """Whole items and lists, one and two row blocks, few items of many parts and many of few, several items in a
    CTA's run; unequal lengths and counts."""
    Case(rows + n, b=b, h=h, g=g, d=d, n=n, rows=rows, c=c, ragged=True).run()


def test_one_long_item_among_short_ones():
    """The list cuts the long item into many parts; the others are whole."""
    c = Case(77, b=12, h=2, g=2, d=128, n=6, rows=6000, c="f32")
    c.length[:] = 40
    c.length[5, 1] = 6000
    c.K[:, :, 40:] = np.where((np.arange(12)[:, None] == 5)[..., None, None] & (np.arange(2)[None, :] == 1)[..., None, None],
                              c.K[:, :, 40:], np.nan)
    c.V[:, :, 40:] = np.where(np.isnan(c.K[:, :, 40:]), np.nan, c.V[:, :, 40:])
    c.run()


def test_rows_that_see_nothing_in_a_cut_item():
    """Nodes that are not in use and nodes without a bit, in items that several CTAs share."""
    c = Case(78, b=1, h=2, n=50, rows=6000, c="none", masks="none")
    c.length[0, 1] = 0  # the second head's nodes see nothing at all
    c.K[0, 1], c.V[0, 1] = np.nan, np.nan
    c.count[0] = 41
    c.sees = [[[] for _ in range(50)]]
    c.run()


def test_units_beyond_the_list():
    """More than 4096 units: one item per CTA whatever their lengths."""
    c = Case(79, b=520, h=8, g=1, d=64, n=2, rows=24, c="none", ragged=True)
    c.run()


@pytest.mark.parametrize("c", ["none", "f32", "bf16", "split"])
@pytest.mark.parametrize("d,g,n,b", [(64, 4, 9, 30), (128, 4, 9, 30), (64, 8, 40, 30), (128, 8, 40, 30),
                                     (64, 4, 9, 20), (128, 4, 9, 20), (64, 8, 40, 25), (128, 8, 40, 25)])
def test_short_items_in_a_list(d, g, n, b, c):
    """Runs of many items of one to four tiles, as a long capacity with short contents has them: what is asked for
    ahead (tiles, the moment matrices' slots, the next queries) crosses item after item."""
    case = Case(d + n, b=b, h=8, g=g, d=d, n=n, rows=1700, c=c)
    rng = np.random.default_rng(n)
    case.length[:] = rng.choice([0, 1, 100, 128, 129, 300], size=case.length.shape)
    case.count[::5] = rng.integers(0, n + 1, size=case.count[::5].shape)
    case.sees = [[[a for a in row if a < m] for row in rows_] for rows_, m in zip(case.sees, case.count.tolist())]
    case.device()
    for _ in range(3):
        case.step()
    case.check(own_sum=True)
