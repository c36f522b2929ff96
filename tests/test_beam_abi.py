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
