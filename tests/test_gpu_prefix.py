"""mkv_prefix_step on the GPU against a plain 64-bit form, with the bounds that tests/beam_ref.py derives."""
import numpy as np
import pytest
import torch

import beam_ref as R
from paper_2606_01563_gb300 import mkv
from gpu_util import host

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
TAU = 1e-6
INVALID, CAPACITY, TIMEOUT = 1, 3, 5


class Case:
    """Random caches, tails and new tokens; rows past every length hold NaN, and so do sequences that are not in use."""

    def __init__(self, b, N, h, g, d, rows, tail, moments="f32", order=1, ragged=True, new=True, seed=0, loud=1.0, fused=True,
                 room=3):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed * 7919 + b * 31 + N)
        self.gen, self.order, self.geom, self.N = gen, order, mkv.geom(b, h, g, d), N
        nan = float("nan")

        def rand(*shape, dtype=BF16):
            return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

        def lengths(most, *shape):
            return torch.randint(0, most + 1, shape, generator=gen, device="cuda", dtype=I32) if ragged else torch.full(
                shape, most, dtype=I32, device="cuda")

        def cache(units, cap, ln):
            K, V = rand(units, h, cap, d), rand(units, h, cap, d)
            past = torch.arange(cap, device="cuda") >= ln[..., None]
            K[past], V[past] = nan, nan
            return mkv.Cache(K, V, torch.randint(0, 99, (units, h, cap), generator=gen, device="cuda", dtype=I32), ln,
                             torch.randint(0, 9999, (units, h), generator=gen, device="cuda", dtype=I32))
        self.prefix = cache(b, rows + 5, lengths(rows, b, h))
        self.tail = cache(b * N, tail + room, lengths(tail, b * N, h))
        self.count = torch.full((b,), N, dtype=I32, device="cuda")
        if ragged:
            self.count = torch.randint(0, N + 1, (b,), generator=gen, device="cuda", dtype=I32)
        self.count[0] = N
        self.mom, self.held = None, None
        p = mkv.mkv_decode_params(0, order, TAU)
        if moments != "none":
            C = 0.3 * rand(b, h, d, d, dtype=F32)
            C[..., ::3, ::5] *= 1e-9  # (below the clamp)
            n = torch.randint(0, 3000, (b, h), generator=gen, device="cuda", dtype=I32)
            n.view(-1)[-1] = 0 if b * h > 1 else 7
            self.mom = mkv.Moments(n, rand(b, h, d, dtype=F32), rand(b, h, d, dtype=F32), C)
            if moments == "bf16":
                self.held = torch.empty(b, h, d, d, dtype=BF16, device="cuda")
                mkv.mkv_moments_pack_bf16(self.geom, self.mom, self.held)
                p.C16 = self.held.data_ptr()
            elif moments == "split":
                self.held = torch.empty(b, h, d, d, dtype=I32, device="cuda")
                mkv.mkv_moments_pack_split(self.geom, self.mom, TAU, self.held)
                p.C_split = self.held.data_ptr()
            p.correction = 1
        self.p = p
        qkv = rand(b, N, h * (g + 2) if fused else h * g, d)
        qkv[:, :, :h * g] *= loud
        dead = torch.arange(N, device="cuda") >= self.count[:, None]
        qkv[dead] = nan
        self.q, self.k, self.v = qkv[:, :, :h * g], None, None
        if new:
            kv = qkv if fused else rand(b, N, 2 * h, d)
            at = h * g if fused else 0
            self.k, self.v = kv[:, :, at:at + h], kv[:, :, at + h:at + 2 * h]
        self.out = torch.full((b, N, h * g, d), nan, dtype=BF16, device="cuda")
        self.lse = torch.full((b, N, h * g), nan, device="cuda")
        self.ws = mkv.alloc_workspace(mkv.mkv_prefix_workspace_size(self.geom, N, self.prefix.capacity, self.tail.capacity))
        self.ws[256:] = 255

    def run(self, lse=True, **kw):
        mkv.mkv_prefix_step(self.geom, mkv.Seqs(self.N, self.count), self.q, self.k, self.v, self.prefix, self.mom, self.tail, self.p,
                            self.out, self.lse if lse else None, self.ws, **kw)

    def reference(self):
        m = None
        if self.mom is not None:
            C = host(self.held) if self.p.C16 else host(self.mom.C)
            m = (host(self.mom.n), host(self.mom.mu_k), host(self.mom.mu_v), C)
        c, t = self.prefix, self.tail
        return R.prefix(host(self.q), None if self.k is None else host(self.k), None if self.v is None else host(self.v), host(c.K),
                        host(c.V), host(c.len), m, self.order, TAU, host(t.K), host(t.V), host(t.len), host(self.count))

    def check(self, ref, error=0):
        out, lse, tol, tol_lse = ref
        got = host(self.out).astype(np.float64)
        off = np.abs(got - out) - tol
        at = np.argwhere(off > 0)
        assert not len(at), (len(at), off.max(), [np.unique(x).tolist()[:40] for x in at.T], mkv.mkv_get_device_error(self.ws))
        lsd = host(self.lse).astype(np.float64)
        none = np.isneginf(lse)
        assert (np.isneginf(lsd) == none).all()
        assert (np.abs(np.where(none, 0, lsd) - np.where(none, 0, lse)) <= tol_lse).all()
        assert mkv.mkv_get_device_error(self.ws)[0] == error

    def step_and_check(self):
        t = self.tail
        before = [x.clone() for x in (t.K, t.V, t.pos, t.len, t.seen)]
        shared = [x.clone() for x in (self.prefix.K, self.prefix.V, self.prefix.pos, self.prefix.len, self.prefix.seen)]
        ref = self.reference()
        self.run()
        self.check(ref)
        if self.k is not None:  # the tails with the new tokens, and nothing else
            b, N, h, d = self.k.shape
            live = (torch.arange(N, device="cuda") < self.count[:, None]).view(-1, 1).expand(-1, h)
            for x, y in zip(before[:2], (self.k, self.v)):
                at = before[3][live].long()
                rows = x[live]
                rows[torch.arange(len(at), device="cuda"), at] = y.reshape(b * N, h, d)[live]
                x[live] = rows
            rows = before[2][live]
            rows[torch.arange(len(rows), device="cuda"), before[3][live].long()] = before[4][live]
            before[2][live] = rows
            before[3][live] += 1
            before[4][live] += 1
        for x, y in zip(before, (t.K, t.V, t.pos, t.len, t.seen)):
            assert torch.equal(x.view(torch.int16) if x.dtype is BF16 else x, y.view(torch.int16) if y.dtype is BF16 else y)
        for x, y in zip(shared, (self.prefix.K, self.prefix.V, self.prefix.pos, self.prefix.len, self.prefix.seen)):
            assert torch.equal(x.view(torch.int16) if x.dtype is BF16 else x, y.view(torch.int16) if y.dtype is BF16 else y)


CASES = [  # b, N, heads, group, dim, rows, tail, moments, order
    (1, 1, 1, 1, 64, 1, 0, "none", 1), (1, 2, 2, 2, 64, 128, 3, "f32", 1), (2, 3, 2, 4, 128, 63, 64, "split", 1),
    (1, 5, 3, 2, 128, 65, 130, "bf16", 1), (3, 2, 2, 8, 64, 1000, 1, "f32", 0), (2, 9, 1, 4, 128, 300, 65, "f32", 1),
    (1, 33, 2, 1, 64, 129, 17, "split", 1), (4, 8, 8, 4, 128, 700, 100, "bf16", 1), (1, 130, 1, 2, 128, 257, 5, "none", 1),
    (2, 40, 2, 8, 128, 400, 40, "f32", 1), (1, 256, 1, 8, 64, 200, 9, "split", 0), (5, 16, 5, 1, 128, 31, 33, "f32", 1),
    (1, 4, 8, 4, 128, 9000, 0, "f32", 1), (40, 2, 8, 4, 64, 90, 70, "none", 1), (1, 17, 2, 8, 64, 5000, 300, "bf16", 1),
]


@pytest.mark.parametrize("b,N,h,g,d,rows,tail,moments,order", CASES)
@pytest.mark.parametrize("ragged", [True, False])
def test_step(b, N, h, g, d, rows, tail, moments, order, ragged):
    Case(b, N, h, g, d, rows, tail, moments, order, ragged, seed=rows, fused=N % 2 == 0).step_and_check()


def test_steps_append_one_after_another():
    c = Case(2, 5, 2, 4, 128, 190, 60, room=8, seed=1)
    for _ in range(7):
        c.step_and_check()
        c.q.copy_(torch.randn(c.q.shape, generator=c.gen, device="cuda"))
        c.k.copy_(torch.randn(c.k.shape, generator=c.gen, device="cuda"))


def test_without_new_tokens_and_without_anything():
    Case(2, 3, 2, 4, 128, 100, 70, new=False, seed=2).step_and_check()
    c = Case(2, 3, 2, 2, 64, 100, 70, moments="none", new=False, seed=3)
    for x in (c.prefix, c.tail):
        x.len.zero_()
    c.step_and_check()
    assert (c.out == 0).all() and torch.isneginf(c.lse).all()
    c = Case(1, 3, 1, 2, 64, 100, 70, moments="none", new=True, seed=4)  # new tokens alone
    for x in (c.prefix, c.tail):
        x.len.zero_()
    c.step_and_check()
    assert torch.equal(c.out, c.v.repeat_interleave(2, 2))


def test_large_scores_and_outputs_without_lse():
    c = Case(2, 6, 2, 4, 128, 500, 80, seed=5, loud=30.0)
    c.step_and_check()
    before = c.out.clone()
    c.tail.len -= 1  # the same step again
    c.tail.len.clamp_(min=0)
    c.run(lse=False)
    c = Case(2, 6, 2, 4, 128, 500, 80, seed=5, loud=30.0)
    c.run(lse=False)
    assert torch.equal(c.out.view(torch.int16), before.view(torch.int16)) and torch.isnan(c.lse).all()


def test_full_tails_and_lengths_out_of_range_are_recorded():
    c = Case(1, 3, 2, 2, 64, 40, 20, ragged=False, room=0, seed=6)  # no room for the new token, which is attended to
    ref, before = c.reference(), [x.clone() for x in (c.tail.K, c.tail.V, c.tail.pos, c.tail.len, c.tail.seen)]
    c.run()
    c.check(ref, error=CAPACITY)
    assert all(torch.equal(x, y) for x, y in zip(before, (c.tail.K, c.tail.V, c.tail.pos, c.tail.len, c.tail.seen)))
    for who in ("prefix", "tail"):
        c = Case(2, 3, 2, 2, 64, 40, 20, ragged=False, room=0, seed=7, new=False)
        x = getattr(c, who)
        x.K.copy_(torch.randn(x.K.shape, generator=c.gen, device="cuda"))
        x.V.copy_(torch.randn(x.V.shape, generator=c.gen, device="cuda"))
        x.len[1, 1], x.len[0, 0] = x.capacity, 0
        ref = c.reference()
        x.len[1, 1], x.len[0, 0] = 2 ** 31 - 1, -2 ** 31
        c.run()
        c.check(ref, error=CAPACITY)
    c = Case(2, 3, 2, 2, 64, 40, 20, ragged=False, seed=8)
    ref = c.reference()
    c.count[1] = 4
    c.run()
    c.check(ref, error=INVALID)


def test_values_that_are_not_finite_stay_with_who_sees_them():
    """An infinite value in one tail, and a NaN new token of one sequence: the others as before."""
    c, e = (Case(1, 6, 2, 4, 128, 200, 50, seed=9, ragged=False) for _ in range(2))
    e.tail.V[2, 1, 7, 5] = float("inf")
    e.k[0, 4, 0, 3] = float("nan")
    c.run()
    e.run()
    rows = torch.ones(6, 8, dtype=torch.bool)
    rows[2, 4:] = rows[4, :4] = False
    assert torch.equal(c.out[0][rows], e.out[0][rows]) and torch.equal(c.lse[0][rows], e.lse[0][rows])
    assert not torch.isfinite(e.out[0, 2, 4:, 5]).any() and torch.isnan(e.out[0, 4, :4]).all()


@pytest.mark.parametrize("dim,group", [(128, 4), (64, 8)])
def test_against_decode_steps_over_caches_of_their_own(dim, group):
    """Every sequence with a copy of the shared rows and its tail in one cache, decoded by mkv_decode_step."""
    b, N, h, rows, tail = 2, 4, 2, 150, 30
    c = Case(b, N, h, group, dim, rows, tail, seed=10, ragged=False)
    g = mkv.geom(b * N, h, group, dim)
    own = mkv.alloc_cache(g, rows + tail + 2)
    for x, y, z in ((own.K, c.prefix.K, c.tail.K), (own.V, c.prefix.V, c.tail.V)):
        x[:, :, :rows] = y[:, :, :rows].repeat_interleave(N, 0)
        x[:, :, rows:rows + tail] = z[:, :, :tail]
    own.len.fill_(rows + tail)
    mom = mkv.Moments(*(x.repeat_interleave(N, 0).contiguous() for x in (c.mom.n, c.mom.mu_k, c.mom.mu_v, c.mom.C)))
    out, lse = torch.empty(b * N, h * group, dim, device="cuda"), torch.empty(b * N, h * group, device="cuda")
    mkv.mkv_decode_step(g, c.q.reshape(b * N, h * group, dim).contiguous(), c.k.reshape(b * N, h, dim).contiguous(),
                        c.v.reshape(b * N, h, dim).contiguous(), own, mom, c.p, out, lse,
                        mkv.alloc_workspace(mkv.mkv_decode_workspace_size(g, own.capacity)))
    _, _, tol, tol_lse = c.reference()
    c.run()
    assert (np.abs(host(c.out).astype(np.float64) - host(out).reshape(tol.shape)) <= 2 * tol).all()
    assert (np.abs(host(c.lse).astype(np.float64) - host(lse).reshape(tol_lse.shape)) <= 2 * tol_lse).all()


def test_two_graphs_with_a_workspace_each_on_another_stream():
    """Two layers' steps captured, replayed in turn; each has its own workspace, as calls that may overlap must."""
    cases = [Case(2, 5, 2, 4, 128, 600, 30, seed=s, room=6) for s in (11, 12)]
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.run(stream=side)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        refs = [c.reference() for c in cases]
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for c, ref in zip(cases, refs):
            c.check(ref)


def test_one_workspace_for_smaller_calls():
    """Sized for the largest batch, number of sequences and capacities, used by smaller ones in turn."""
    big = Case(6, 20, 3, 4, 128, 900, 200, seed=13)
    big.step_and_check()
    for b, N, rows, tail in ((1, 1, 899, 200), (1, 20, 64, 1), (6, 3, 1, 150), (2, 20, 900, 0)):
        c = Case(b, N, 3, 4, 128, rows, tail, seed=14 + b)
        assert mkv.mkv_prefix_workspace_size(c.geom, N, c.prefix.capacity, c.tail.capacity) <= big.ws.numel()
        c.ws = big.ws
        c.step_and_check()


def test_waits_that_run_out_are_recorded():
    c = Case(2, 5, 2, 4, 128, 600, 100, seed=20)
    old = mkv.mkv_debug_set_poll_limit(0)
    try:
        c.run()
        assert mkv.mkv_get_device_error(c.ws)[0] == TIMEOUT
    finally:
        mkv.mkv_debug_set_poll_limit(old)
    c = Case(2, 5, 2, 4, 128, 600, 100, seed=20)
    c.step_and_check()


def test_tensors_of_another_device_are_refused():
    c = Case(1, 2, 1, 2, 64, 10, 2)
    c.out = c.out.cpu()
    with pytest.raises(ValueError):
        c.run()


# Many query rows over many shared rows, which the kernels of drafted trees take: the same columns as CASES.
MANY = [
    (2, 64, 8, 4, 128, 2000, 100, "f32", 1),   # one row block of 256, lengths from 0 on
    (1, 256, 4, 8, 64, 2000, 3, "bf16", 1),    # the most rows
    (3, 33, 8, 1, 128, 4900, 40, "split", 1),  # 33 rows
    (1, 40, 8, 2, 128, 10000, 300, "f32", 0), (60, 9, 8, 4, 128, 500, 70, "f32", 1),
    (2, 100, 6, 8, 64, 1600, 1, "split", 1), (1, 65, 8, 8, 128, 2000, 0, "none", 1),
    (140, 5, 8, 8, 128, 200, 2, "f32", 1),     # more units than a list of their runs is made for
]


@pytest.mark.parametrize("b,N,h,g,d,rows,tail,moments,order", MANY)
@pytest.mark.parametrize("ragged", [True, False])
def test_step_of_many_rows(b, N, h, g, d, rows, tail, moments, order, ragged):
    Case(b, N, h, g, d, rows, tail, moments, order, ragged, seed=rows, fused=N % 2 == 0).step_and_check()


def test_many_rows_with_nothing_shared():
    for moments, new in (("none", False), ("f32", True)):
        c = Case(2, 64, 8, 4, 128, 2000, 9, moments=moments, new=new, seed=30)
        c.prefix.len.zero_()
        c.prefix.K.fill_(float("nan"))
        c.prefix.V.fill_(float("nan"))
        c.tail.len[::3] = 0
        if c.mom is not None:
            c.mom.n[:, ::2] = 0
        c.step_and_check()


def test_many_rows_with_large_scores():
    Case(1, 64, 8, 8, 128, 2500, 80, seed=31, loud=30.0).step_and_check()


def test_many_rows_sizes_out_of_range_are_recorded():
    for who in ("prefix", "tail", "count"):
        c = Case(2, 64, 8, 4, 128, 2000, 20, ragged=False, seed=32, new=False)
        x = c.tail if who == "tail" else c.prefix
        for y in (x.K, x.V):
            y[1, 1] = torch.randn(y[1, 1].shape, generator=c.gen, device="cuda")
        if who != "count":
            x.len[1, 1], x.len[0, 0] = x.capacity, 0
        ref = c.reference()
        if who == "count":
            c.count[1] = 65
        else:
            x.len[1, 1], x.len[0, 0] = 2 ** 31 - 1, -2 ** 31
        c.run()
        c.check(ref, error=INVALID if who == "count" else CAPACITY)


def test_many_rows_captured_and_between_calls_of_few():
    """One workspace: a graph of the step of many rows, replayed in turn with eager steps of few."""
    big = Case(2, 64, 8, 4, 128, 2000, 30, seed=33, room=8)
    few = Case(2, 3, 8, 4, 128, 300, 30, seed=34, room=8)
    few.ws = big.ws
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        big.run(stream=side)
    for _ in range(3):
        ref, ref_few = big.reference(), few.reference()
        graph.replay()
        few.run()
        big.check(ref)
        few.check(ref_few)


def test_many_rows_give_the_same_bits_again():
    c = Case(2, 64, 8, 4, 128, 2000, 100, seed=35, new=False)
    c.run()
    out, lse = c.out.clone(), c.lse.clone()
    for _ in range(20):
        c.run()
        assert torch.equal(c.out.view(torch.int16), out.view(torch.int16)) and torch.equal(c.lse, lse)


def test_many_rows_waits_that_run_out_are_recorded():
    c = Case(2, 64, 8, 4, 128, 2000, 100, seed=36)
    old = mkv.mkv_debug_set_poll_limit(0)
    try:
        c.run()
        assert mkv.mkv_get_device_error(c.ws)[0] == TIMEOUT
    finally:
        mkv.mkv_debug_set_poll_limit(old)
    Case(2, 64, 8, 4, 128, 2000, 100, seed=36).step_and_check()
