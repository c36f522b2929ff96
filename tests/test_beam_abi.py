"""include/mkv_beam.h: every declared function is exported and bound, the
header compiles as C99 and C++ with the layouts the binding declares, and bad
arguments are refused before anything is launched.  Runs on the CPU."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2606_01563_gb300 import mkv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20  # never dereferenced: validation fails before any launch
OK, INVALID, SHAPE, CAPACITY, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 6, 7


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mkv.LIB_PATH):
        from paper_2606_01563_gb300 import build
        build.build()
    return mkv.lib()


def test_select_refusals(L):
    S = mkv.mkv_beam_scores

    def call(b=2, beams=4, vocab=100, s=None, out=4, parent=FAKE, token=FAKE, score=FAKE, done=FAKE, ws=FAKE, wsb=1 << 40):
        s = s or S(FAKE, 0, 400, 100, FAKE, FAKE, 2)
        return L.mkv_beam_select(b, beams, vocab, ctypes.byref(s), out, parent, token, score, done, ws, wsb, None)
    for bad in (dict(b=0), dict(b=65536), dict(beams=0), dict(beams=65), dict(vocab=0), dict(vocab=(1 << 24) + 1),
                dict(out=0), dict(out=65)):
        assert call(**bad) == SHAPE, bad
    sizes = mkv.mkv_beam_select_workspace_size
    assert sizes(0, 4, 100, 4) == sizes(2, 65, 100, 4) == sizes(2, 4, 0, 4) == sizes(2, 4, 100, 65) == 0
    for name in ("parent", "token", "score"):
        assert call(**{name: None}) == INVALID and call(**{name: FAKE + 2}) == INVALID
    assert call(done=FAKE + 1) == INVALID
    assert L.mkv_beam_select(2, 4, 100, None, 4, FAKE, FAKE, FAKE, None, FAKE, 1 << 40, None) == INVALID
    for s in (S(None, 0, 0, 0, FAKE, None, 2), S(FAKE + 1, 0, 0, 0, FAKE, None, 2), S(FAKE + 2, 1, 0, 0, FAKE, None, 2),
              S(FAKE, 2, 0, 0, FAKE, None, 2), S(FAKE, 0, -1, 0, FAKE, None, 2), S(FAKE, 0, 0, -1, FAKE, None, 2),
              S(FAKE, 0, 0, 0, None, None, 2), S(FAKE, 0, 0, 0, FAKE + 2, None, 2), S(FAKE, 0, 0, 0, FAKE, FAKE + 3, 2),
              S(FAKE, 0, 0, 0, FAKE, None, 100), S(FAKE, 0, 0, 0, FAKE, None, -2), S(FAKE, 0, 0, 0, FAKE, FAKE, -1)):
        assert call(s=s) == INVALID
    need = sizes(2, 4, 100, 4)
    assert need >= 256 and call(ws=None) == WORKSPACE and call(ws=FAKE + 8) == WORKSPACE and call(wsb=need - 1) == WORKSPACE


def test_reorder_refusals(L):
    def call(g=mkv.geom(2, 3, 1, 128), n=4, layers=1, parent=FAKE, ws=FAKE, wsb=256, null=False,
             cache=mkv.mkv_cache(FAKE, FAKE, FAKE, FAKE, FAKE, 64), mom=mkv.mkv_moments()):
        arr = None if null else (mkv.mkv_beam_layer * 1)(mkv.mkv_beam_layer(cache, mom))
        return L.mkv_beam_reorder(g, n, layers, arr, parent, ws, wsb, None)
    assert call(g=mkv.geom(2, 3, 1, 96)) == UNSUPPORTED and call(g=mkv.geom(0, 3, 1, 64)) == SHAPE
    assert call(n=0) == SHAPE and call(n=257) == SHAPE and call(g=mkv.geom(8192, 8, 1, 64)) == SHAPE
    assert call(parent=None) == INVALID and call(parent=FAKE + 2) == INVALID and call(layers=-1) == INVALID
    assert call(null=True) == INVALID
    for cache in (mkv.mkv_cache(None, FAKE, FAKE, FAKE, FAKE, 64), mkv.mkv_cache(FAKE, FAKE + 8, FAKE, FAKE, FAKE, 64),
                  mkv.mkv_cache(FAKE, FAKE, FAKE, FAKE, FAKE, 0), mkv.mkv_cache(FAKE, FAKE, FAKE, FAKE, FAKE, 64, FAKE)):
        assert call(cache=cache) == INVALID
    assert call(mom=mkv.mkv_moments(FAKE, FAKE, FAKE, None)) == INVALID
    assert call(mom=mkv.mkv_moments(FAKE, FAKE, FAKE, FAKE + 8)) == INVALID
    assert call(ws=None) == WORKSPACE and call(wsb=255) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE
    assert call(layers=0) == OK  # nothing to launch


def test_reorder_refuses_a_state_twice(L):
    def layer(at, mom=None):
        return mkv.mkv_beam_layer(mkv.mkv_cache(at, at, FAKE, FAKE, FAKE, 64),
                                  mkv.mkv_moments() if mom is None else mkv.mkv_moments(mom, FAKE, FAKE, FAKE))
    far = FAKE + (1 << 20)
    for pair in ((layer(FAKE), layer(FAKE)), (layer(FAKE, FAKE), layer(far, FAKE))):
        arr = (mkv.mkv_beam_layer * 2)(*pair)
        assert L.mkv_beam_reorder(mkv.geom(2, 3, 1, 128), 4, 2, arr, FAKE, FAKE, 256, None) == INVALID


def test_reorder_refuses_any_array_in_two_layers(L):
    """Layers whose arrays are all their own, but one: as much a move at once as a whole cache twice."""
    cache = ("K", "V", "pos", "len", "seen", "y", "y_len")
    names = cache + ("n", "mu_k", "mu_v", "C")

    def call(take=None, give=None, have=names, layers=3):
        at = [{x: (1 + i * len(names) + names.index(x)) << 20 if x in have else None for x in names} for i in range(layers)]
        if take is not None:
            at[-1][take] = at[0][give or take]
        arr = (mkv.mkv_beam_layer * layers)(*(mkv.mkv_beam_layer(
            mkv.mkv_cache(a["K"], a["V"], a["pos"], a["len"], a["seen"], 64, a["y"], a["y_len"]),
            mkv.mkv_moments(a["n"], a["mu_k"], a["mu_v"], a["C"])) for a in at))
        return L.mkv_beam_reorder(mkv.geom(2, 3, 1, 128), 4, layers, arr, FAKE, None, 256, None)  # (no workspace: not launched)
    for have in (names, cache, cache[:5], cache[:5] + names[7:]):
        assert call(have=have) == WORKSPACE and call(have=have, layers=70) == WORKSPACE
        for name in have:
            assert call(name, have=have) == INVALID and call(name, have=have, layers=70) == INVALID, name
    for take, give in (("K", "V"), ("V", "K"), ("mu_k", "mu_v"), ("mu_v", "mu_k")):
        assert call(take, give) == INVALID


def test_select_binding_refusals():
    b, k, v = 2, 3, 50
    good = dict(logits=torch.zeros(b, k, v), score=torch.zeros(b, k), parent=torch.zeros(b, 4, dtype=torch.int32),
                token=torch.zeros(b, 4, dtype=torch.int32), score_out=torch.zeros(b, 4),
                done=torch.zeros(b, k, dtype=torch.int32), done_out=torch.zeros(b, 4, dtype=torch.int32))
    bad = dict(logits=(torch.zeros(b, k, v).half(), torch.zeros(b, k, 2 * v)[..., ::2], torch.zeros(b * k, v)),
               score=(torch.zeros(b, k).double(), torch.zeros(b, k + 1), torch.zeros(k, b).t()),
               parent=(torch.zeros(b, 4).long(), torch.zeros(b + 1, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)),
               token=(torch.zeros(b, 5, dtype=torch.int32),), score_out=(torch.zeros(b, 5),),
               done=(torch.zeros(b, k).bool(), torch.zeros(b, 4, dtype=torch.int32)),
               done_out=(torch.zeros(b, k, dtype=torch.int32),))
    for name, values in bad.items():
        for x in values:
            with pytest.raises(ValueError):
                mkv.mkv_beam_select(**{**good, name: x}, ws=torch.zeros(1 << 20, dtype=torch.uint8), end_token=2)


def test_reorder_binding_refusals():
    def cache(states=6, h=2, cap=5, d=64, **other):
        c = mkv.alloc_cache(mkv.geom(states, h, 1, d), cap, device="cpu", evict_state="y" in other)
        for k, v in other.items():
            setattr(c, k, v)
        return c
    i32 = dict(dtype=torch.int32)
    m = mkv.alloc_moments(mkv.geom(6, 2, 1, 64), device="cpu")
    bad = [cache(V=torch.zeros(6, 2, 4, 64).bfloat16()), cache(K=torch.zeros(6, 2, 5, 64)), cache(pos=torch.zeros(6, 2, 4, **i32)),
           cache(len=torch.zeros(6, 2)), cache(seen=torch.zeros(2, 6, **i32).t()), cache(y=torch.zeros(6, 2, 5, 64).bfloat16())]
    for c in bad:
        with pytest.raises(ValueError):
            mkv.beam_layers([(c, None)])
    with pytest.raises(ValueError):
        mkv.beam_layers([])
    for name, x in (("n", m.n.float()), ("mu_k", m.mu_k[:, :, :32]), ("C", m.C.transpose(2, 3))):
        with pytest.raises(ValueError):
            mkv.beam_layers([(cache(K=cache().K), mkv.Moments(**{**m.__dict__, name: x}))])


def test_every_declared_function_is_exported_and_bound(L):
    src = open(os.path.join(ROOT, "include", "mkv_beam.h")).read()
    names = set(re.findall(r"MKV_API\s+[\w\s\*]+?\b(mkv_\w+)\s*\(", src))
    assert names == set(mkv.BEAM_EXPORTS)
    for n in names:
        assert hasattr(L, n) and hasattr(mkv, n), n


CLIENT = r"""
#include <stddef.h>
#include <stdio.h>
#include "mkv_beam.h"
#define CHECK(c) do { if (!(c)) { printf("FAIL %d: %s\n", __LINE__, #c); return 1; } } while (0)
int main(void) {
  CHECK(sizeof(mkv_seqs) == 48 && offsetof(mkv_seqs, count) == 8 && offsetof(mkv_seqs, kv_batch) == 40);
  CHECK(sizeof(mkv_beam_scores) == 56 && offsetof(mkv_beam_scores, score) == 32 && offsetof(mkv_beam_scores, end_token) == 48);
  CHECK(sizeof(mkv_beam_layer) == 96 && offsetof(mkv_beam_layer, mom) == 64);
  CHECK(MKV_BEAM_MAX_SEQS == 256 && MKV_BEAM_MAX_BEAMS == 64 && MKV_BEAM_MAX_OUT == 64);
  return 0;
}
"""


@pytest.mark.parametrize("compiler,std,ext", [("gcc", "c99", "c"), ("g++", "c++17", "cpp")])
def test_header_layouts(tmp_path, compiler, std, ext):
    if shutil.which(compiler) is None:
        pytest.skip(f"no {compiler}")
    src = tmp_path / f"client.{ext}"
    src.write_text(CLIENT)
    exe = tmp_path / "client"
    subprocess.run([compiler, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
    assert [ctypes.sizeof(x) for x in (mkv.mkv_seqs, mkv.mkv_beam_scores, mkv.mkv_beam_layer)] == [48, 56, 96]


def test_prefix_refusals(L):
    C = mkv.mkv_cache

    def call(g=mkv.geom(2, 3, 4, 128), n=5, count=None, strides=(0, 0, 0, 0), q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE,
             prefix=C(FAKE, FAKE, FAKE, FAKE, FAKE, 64), tail=C(FAKE, FAKE, FAKE, FAKE, FAKE, 9), null=False,
             mom=mkv.mkv_moments(FAKE, FAKE, FAKE, FAKE), p=mkv.mkv_decode_params(1, 1, 1e-6), ws=FAKE, wsb=1 << 40):
        s = mkv.mkv_seqs(n, count, *strides)
        return L.mkv_prefix_step(g, None if null else ctypes.byref(s), q, k, v, ctypes.byref(prefix), mom, ctypes.byref(tail), p, out,
                                 lse, ws, wsb, None)
    assert call(g=mkv.geom(2, 3, 4, 96)) == UNSUPPORTED and call(g=mkv.geom(2, 3, 3, 128)) == SHAPE
    for n in (0, 257, -1):
        assert call(n=n) == SHAPE and mkv.mkv_prefix_workspace_size(mkv.geom(1, 1, 1, 64), n, 10, 10) == 0
    sizes = mkv.mkv_prefix_workspace_size
    assert sizes(mkv.geom(1, 1, 1, 64), 2, 0, 1) == sizes(mkv.geom(1, 1, 1, 64), 2, 1, 0) == sizes(mkv.geom(1, 1, 1, 80), 2, 1, 1) == 0
    assert call(null=True) == INVALID
    for name in ("q", "k", "v", "out"):
        assert call(**{name: None}) == INVALID and call(**{name: FAKE + 8}) == INVALID
    assert call(lse=FAKE + 2) == INVALID and call(count=FAKE + 1) == INVALID
    dq, dkv = 12 * 128, 3 * 128
    for strides in ((dq - 8, 0, 0, 0), (dq + 4, 0, 0, 0), (0, 5 * dq - 8, 0, 0), (0, 0, dkv - 8, 0), (0, 0, 0, 5 * dkv - 8),
                    (-8, 0, 0, 0), (0, 0, 1 << 40, 0)):
        assert call(strides=strides) == INVALID, strides
    for bad in (C(None, FAKE, FAKE, FAKE, FAKE, 64), C(FAKE, FAKE + 8, FAKE, FAKE, FAKE, 64), C(FAKE, FAKE, FAKE, FAKE, FAKE, 0)):
        assert call(prefix=bad) == INVALID and call(tail=bad) == INVALID
    assert call(prefix=C(FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 29)) == SHAPE  # rows past a tensor map's coordinates
    assert call(tail=C(FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 27)) == SHAPE
    assert call(mom=mkv.mkv_moments(FAKE, FAKE + 4, FAKE, FAKE)) == INVALID
    assert call(p=mkv.mkv_decode_params(2, 1, 1e-6)) == INVALID and call(p=mkv.mkv_decode_params(1, 1, -1.0)) == INVALID
    assert call(p=mkv.mkv_decode_params(1, 1, 1e-6, FAKE, 0, FAKE)) == INVALID
    need = sizes(mkv.geom(2, 3, 4, 128), 5, 64, 9)
    assert need >= 256 and call(wsb=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE


def test_prefix_binding_refusals():
    g = mkv.geom(2, 2, 2, 64)
    b16 = dict(dtype=torch.bfloat16)
    prefix, tail = mkv.alloc_cache(g, 8, device="cpu"), mkv.alloc_cache(mkv.geom(6, 2, 2, 64), 4, device="cpu")
    good = dict(seqs=mkv.Seqs(3), q=torch.zeros(2, 3, 4, 64, **b16), k_new=torch.zeros(2, 3, 2, 64, **b16),
                v_new=torch.zeros(2, 3, 2, 64, **b16), prefix=prefix, tail=tail, out=torch.zeros(2, 3, 4, 64, **b16),
                lse=torch.zeros(2, 3, 4))
    bad = dict(seqs=(mkv.Seqs(3, torch.zeros(2)), mkv.Seqs(3, torch.zeros(3, dtype=torch.int32)), mkv.Seqs(2)),
               q=(good["q"].float(), good["q"][:, :2], good["q"].transpose(2, 3), good["q"][:1].expand(2, -1, -1, -1),
                  good["q"][:, :1].expand(-1, 3, -1, -1), torch.zeros(2, 3, 4, 128, **b16)[..., ::2], torch.zeros(2, 3, 8, 64, **b16)[:, :, ::2]),
               k_new=(None, good["k_new"].half(), torch.zeros(2, 3, 4, 64, **b16)[:, :, :2]),
               v_new=(None, torch.zeros(2, 4, 2, 64, **b16)), out=(good["out"].float(), torch.zeros(2, 6, 4, 64, **b16)[:, ::2]),
               lse=(torch.zeros(2, 3, 2), torch.zeros(2, 3, 4, dtype=torch.float64)), prefix=(tail,), tail=(prefix,),
               mom=(mkv.alloc_moments(mkv.geom(2, 3, 2, 64), device="cpu"),))
    # a cache whose tensors are not dense slabs: a transposed view has its units in another order
    for name, x in (("K", torch.zeros(2, 6, 4, 64, **b16).transpose(0, 1)), ("V", torch.zeros(6, 2, 64, 4, **b16).transpose(2, 3)),
                    ("len", torch.zeros(2, 6, dtype=torch.int32).t()), ("pos", torch.zeros(6, 2, 8, dtype=torch.int32)[..., ::2]),
                    ("K", tail.K.float()), ("seen", tail.seen.long()), ("V", torch.zeros(6, 2, 5, 64, **b16))):
        bad["tail"] += (mkv.Cache(**{**tail.__dict__, name: x}),)
    for name, values in bad.items():
        for x in values:
            with pytest.raises(ValueError):
                mkv.mkv_prefix_step(g, **{"mom": None, **good, name: x}, p=mkv.mkv_decode_params(0, 1, 1e-6),
                                    ws=torch.zeros(1 << 20, dtype=torch.uint8))
