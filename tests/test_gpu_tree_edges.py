"""Edges of the calls in include/mkv_tree.h that their other GPU tests leave
out, against the plain 64-bit forms of tests/tree_ref.py.

Bound: the kernel divides by the sum of its rounded weights, so its bound is
the one of Case.check(own_sum=True), everywhere here."""
import numpy as np
import pytest
import torch

import tree_ref as R
from paper_2606_01563_gb300 import mkv
from paper_2606_01563_gb300.inputs import bf16_round
from gpu_util import host
from test_gpu_tree import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,n,rows", [(32, 13, 1000), (40, 8, 900), (2, 20, 6000)])
def test_one_slot_of_moments_in_a_ring_of_six(b, n, rows):
    """16-bit moments with one row block shift the ring by an odd number before an item's last tiles: whole items and
    runs, many CTAs at once (copies late and out of order), the same bits in every call."""
    c = Case(b + n, b=b, h=8, g=4, d=128, n=n, rows=rows, c="bf16", ragged=True).device()
    c.step()
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(40):
        c.step()
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    c.check(own_sum=True)


@pytest.mark.parametrize("g,n,rows", [(4, 20, 127), (4, 70, 127), (1, 40, 100), (8, 20, 255)])
@pytest.mark.parametrize("d", [64, 128])
def test_reference_moves_several_times_in_a_masked_tile(g, n, rows, d):
    """One node of a warp has scores that rise by 50 octaves every 32 keys, so the warp's reference moves in every
    group of 32 columns; the other rows, whose scores rise by one or two, take O and the weights already written
    of the tile along each time."""
    c = Case(50 + n, h=2, g=g, d=d, n=n, rows=rows, c="none", masks="all")
    rng = np.random.default_rng(d)
    way = rng.choice([-1.0, 1.0], d) / np.sqrt(d)
    large = np.arange(n) % (32 // g) == 0
    c.q = bf16_round(rng.standard_normal(c.q.shape) + way)
    c.q[0, large] = bf16_round(40 * way * np.sqrt(d / 128))
    rise = 10 * np.sqrt(d / 128)
    c.K[:, :, :rows] = bf16_round(0.5 * rng.standard_normal((1, 2, rows, d)) + rise * (np.arange(rows) // 32)[:, None] * way)
    c.k = bf16_round(0.5 * rng.standard_normal(c.k.shape) + rise * (rows / 32 + np.arange(n) // 32)[:, None, None] * way)
    c.device().step()
    c.check(own_sum=True)


@pytest.mark.parametrize("b,h,n,rows,c", [(1, 2, 9, 300, "f32"),       # an item per CTA
                                          (1, 2, 20, 20000, "f32"),    # the list of tiles: 2 units in many parts
                                          (2, 8, 40, 3000, "none"),    # two row blocks
                                          (70, 8, 5, 600, "bf16")])    # more units than threads in a CTA
def test_a_length_that_changes_under_an_early_load_is_recorded(b, h, n, rows, c):
    """A decode step, whose kernel is still running, appends a row to the cache that the call behind it reads with
    early_load.  Either the call read the new length everywhere, then it is right, or MKV_ERR_INVALID_ARG is recorded;
    no wait runs out, and the same call without early_load is right afterwards."""
    case = Case(b + n, b=b, h=h, n=n, rows=rows, c=c, spare=0.0).device()
    _, _, g, d = case.geo
    ws = mkv.alloc_workspace(mkv.mkv_decode_workspace_size(case.g, case.cap))
    q, k, v = (x[:, 0].contiguous() for x in (case.dq, case.dk, case.dv))
    y = torch.empty(b, h * g, d, device="cuda")

    def pair():
        case.p.early_load = 0
        mkv.mkv_decode_step(case.g, q, k, v, case.cache, case.mom, case.p, y, None, ws)
        case.p.early_load = 1
        case.step()

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):  # (no host time between the two)
        pair()
    recorded = 0
    for _ in range(20):
        case.cache.len.fill_(rows)
        case.out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        code, _ = mkv.mkv_get_device_error(case.ws)
        assert code in (0, 1)
        assert (case.cache.len == rows + 1).all()
        out, lse = case.out.clone(), case.lse.clone()
        case.p.early_load = 0
        case.step()
        assert mkv.mkv_get_device_error(case.ws)[0] == 0
        if code == 0:
            assert torch.equal(out, case.out) and torch.equal(lse, case.lse)
        recorded += code
    print(f"{recorded} of 20 recorded")
    # lengths that stay: nothing is recorded, and the outputs are those of the call that waits
    case.p.early_load = 1
    out.copy_(case.out), lse.copy_(case.lse)
    torch.cuda.synchronize()
    case.step()
    assert mkv.mkv_get_device_error(case.ws)[0] == 0
    assert torch.equal(out, case.out) and torch.equal(lse, case.lse)


@pytest.mark.parametrize("masks,rows", [("tree", 100), ("self", 0), ("none", 0), ("all", 3000)])
@pytest.mark.parametrize("n", [9, 70])
@pytest.mark.parametrize("large_c", [False, True])
def test_a_moment_logit_of_minus_infinity_is_no_term(masks, rows, n, large_c):
    """q.mu_k below the range of 32 bits: the term has no weight, whatever its value, and a row that sees nothing
    else gets zeros and a log-normaliser of -infinity."""
    c = Case(60 + n, h=2, n=n, rows=rows, c="f32", masks=masks)
    c.q = np.abs(c.q) + np.float32(0.5)
    c.q = bf16_round(c.q)
    nn, mk, mv, C = c.moments
    nn[:] = 100
    mk[:] = -1e38
    if large_c:
        C[:] = 3e38  # its product with q overflows
    c.device().step()
    c.moments = None  # the reference's: no term
    c.check(own_sum=True)


@pytest.mark.parametrize("size", [2.0 ** 105, 2.0 ** -90])
@pytest.mark.parametrize("b,h,g,n,rows,c", [(1, 2, 4, 9, 300, "none"), (1, 2, 4, 9, 300, "f32"), (8, 8, 4, 64, 700, "none"),
                                            (1, 1, 4, 20, 6000, "none")])
def test_values_near_the_ends_of_the_range(size, b, h, g, n, rows, c):
    """Scores that rise by 20 to 35 octaves after the first tile, with values of 2^105 and 2^-90: no weighted sum
    leaves the range, as none does whose weights are at most 1."""
    case = Case(70 + n, b=b, h=h, g=g, n=n, rows=rows, c=c)
    rng = np.random.default_rng(1)
    way = rng.choice([-1.0, 1.0], 128) / np.sqrt(128)
    case.q = bf16_round(0.5 * rng.standard_normal(case.q.shape) + 4 * way)
    case.K[:, :, 128:rows] = bf16_round(0.5 * rng.standard_normal((b, h, rows - 128, 128)) + 55 * way)
    case.V[:, :, :rows] *= size
    case.v *= size
    if case.moments is not None:
        case.moments[2][:] *= size  # mu_v, C
        case.moments[3][:] *= size
        if size < 1:
            case.moments[0][:] = 0  # (tau would clamp such a C)
    case.device().step()
    case.check(own_sum=True)
    assert np.abs(host(case.out).astype(np.float64)).max() > size / 8


def test_one_workspace_for_trees_of_every_size():
    """A workspace of the largest tree's and capacity's size, with a guard behind it, serves smaller ones: lists and
    whole items, one and two row blocks, one after another."""
    size = mkv.mkv_tree_workspace_size(mkv.geom(4, 8, 4, 128), 256, 4096)
    room = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
    room[size:] = 77
    for b, n, rows, cap in [(4, 256, 4000, 4096), (4, 32, 2000, 2064), (4, 64, 2000, 2064), (1, 65, 1000, 1040),
                            (1, 128, 1000, 1040), (1, 8, 2200, 2304), (1, 1, 4000, 4096), (2, 9, 30, 4096), (4, 13, 700, 800)]:
        c = Case(b + n, b=b, h=8, g=4, n=n, rows=rows, cap=cap, c="f32" if n < 100 else "none", ragged=n < 256).device()
        c.ws = room[:size]
        c.step()
        if n < 256:
            c.check(own_sum=True)
    assert mkv.mkv_get_device_error(room)[0] == 0
    assert (room[size:] == 77).all()


def _not_finite(c, rng):
    """Puts values that are not finite, and a NaN key, into some units' nodes: what every row has to be is
    (key, {column: value}) per (item, KV head, node)."""
    b, h, _, d = c.geo
    bad_v, bad_k = {}, {}
    for bi in range(b):
        for hi in range(h):
            m = int(c.count[bi])
            if m < 3 or rng.random() < 0.4:
                continue
            for value in (np.inf, -np.inf, np.nan, np.inf):  # (of both node tiles where there are two)
                node = int(rng.integers(0, m)) if rng.random() < 0.5 else m - 1 - int(rng.integers(0, min(m, 5)))
                col = int(rng.choice([3, 3, 62, d - 1]))
                c.v[bi, node, hi, col] = value
                bad_v[bi, hi, node, col] = value
            if rng.random() < 0.3:
                node = int(rng.integers(0, m))
                c.k[bi, node, hi, 8] = np.nan
                bad_k[bi, hi, node] = True
    return bad_v, bad_k


@pytest.mark.parametrize("b,h,g,d,n,rows,masks,short", [
    (1, 2, 4, 128, 40, 6000, "random", False),   # cut items, one row block
    (1, 8, 4, 128, 64, 9000, "random", False),   # cut items, two row blocks
    (2, 8, 2, 128, 256, 500, "random", False),   # two node tiles, two row blocks, whole items
    (1, 2, 1, 64, 200, 4000, "tree", False),     # two node tiles in cut items
    (1, 1, 8, 128, 200, 300, "odd", False),      # several row blocks of one unit
    (30, 8, 4, 128, 9, 1700, "random", True),    # runs of short items: some units have such values, the next have none
    (30, 8, 8, 64, 40, 1700, "tree", True),
    (12, 8, 4, 64, 140, 900, "random", True)])
@pytest.mark.parametrize("moments", ["none", "f32"])
def test_not_finite_values_in_every_plan(b, h, g, d, n, rows, masks, short, moments):
    """As in whole items of one row block: they reach the rows that see them, and no others.  The others differ from
    those of a run without such values by one rounding at most (a row that holds a NaN may leave its warp's reference
    elsewhere)."""
    runs = []
    for bad in (False, True):
        c = Case(80 + n, b=b, h=h, g=g, d=d, n=n, rows=rows, c=moments, masks=masks, spare=0.0)
        rng = np.random.default_rng(n)
        if short:
            c.length[:] = rng.choice([0, 1, 100, 128, 129, 300], size=c.length.shape)
            c.count[::5] = rng.integers(0, n + 1, size=c.count[::5].shape)
            c.sees = [[[a for a in row if a < m] for row in rows_] for rows_, m in zip(c.sees, c.count.tolist())]
        if bad:
            bad_v, bad_k = _not_finite(c, rng)
            assert bad_v
        c.device().step()
        assert mkv.mkv_get_device_error(c.ws)[0] == 0
        runs.append((host(c.out).astype(np.float64), host(c.lse).astype(np.float64)))
    (want, want_lse), (got, got_lse) = runs
    with np.errstate(invalid="ignore"):
        for bi in range(b):
            for i in range(int(c.count[bi])):
                see = set(c.sees[bi][i])
                for (x, hi, node, col), _ in bad_v.items():
                    if x == bi and node in see:  # (the last one written there)
                        want[bi, i, hi * g:(hi + 1) * g, col] += c.v[bi, node, hi, col]
                for x, hi, node in bad_k:
                    if x == bi and node in see:
                        want[bi, i, hi * g:(hi + 1) * g], want_lse[bi, i, hi * g:(hi + 1) * g] = np.nan, np.nan
    assert (np.isnan(got) == np.isnan(want)).all() and (np.isnan(got_lse) == np.isnan(want_lse)).all()
    ok = ~np.isnan(want)
    fin = ok & np.isfinite(want)
    assert (got[ok & ~fin] == want[ok & ~fin]).all()
    assert (np.abs(got[fin] - want[fin]) <= 2.0 ** -8 * np.abs(want[fin]) + 1e-6).all()
    ok = np.isfinite(want_lse)
    assert (np.isneginf(got_lse) == np.isneginf(want_lse)).all()
    assert (np.abs(got_lse[ok] - want_lse[ok]) <= 1e-5).all()
    assert not np.isfinite(want).all()
