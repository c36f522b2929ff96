"""The beam search example's calls together: every step's outputs against a plain 64-bit form over each beam's own
history, and the tails after each reordering against that history, row by row."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import beam_ref as R
import norm_ref as NR
from paper_2606_01563_gb300 import mkv
from gpu_util import host

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("beam_search", os.path.join(ROOT, "examples", "beam_search.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("beams,dim,group", [(4, 128, 4), (9, 64, 8)])
def test_steps_against_each_beams_history(example, beams, dim, group):
    b, h, layers, T, steps, vocab = 2, 2, 2, 400, 6, 300
    s = example.BeamSearch(batch=b, beams=beams, heads=h, group=group, dim=dim, layers=layers, T=T, budget=64, vocab=vocab,
                           steps=steps, seed=beams)
    hq = h * group
    rows = [[[] for _ in range(beams)] for _ in range(b)]  # of every beam: (k, v) of every layer, a token each
    for step in range(steps):
        tokens, before = host(s.token), [x.clone() for x in (s.score, s.done)]
        out = s.attend().clone()
        assert mkv.mkv_get_device_error(s.ws)[0] == 0
        pos = np.full((1, b, beams), T + step)
        for i in range(layers):
            raw = host(s.table[i])[tokens]  # the tokens' projections, before norms and rotation
            rot = (pos, [s.rope.inv_freq[f] for f in range(dim // 2)], [0] * (dim // 2), False)
            for at, w in ((slice(0, hq), s.weights[i][0]), (slice(hq, hq + h), s.weights[i][1])):
                want, tol = NR.forward(raw[:, :, at], host(w), example.EPS, *rot)
                assert (np.abs(host(s.qkv[i])[:, :, at] - want) <= tol).all()
            q, k, v = (host(s.qkv[i])[:, :, at] for at in (slice(0, hq), slice(hq, hq + h), slice(hq + h, None)))
            Kt, Vt = np.zeros((b * beams, h, steps, dim)), np.zeros((b * beams, h, steps, dim))
            for bi in range(b):
                for j in range(beams):
                    for t, (kr, vr) in enumerate(rows[bi][j]):
                        Kt[bi * beams + j, :, t], Vt[bi * beams + j, :, t] = kr[i], vr[i]
            cache, mom = s.prompts[i]
            want, _, tol, _ = R.prefix(q, k, v, host(cache.K), host(cache.V), host(cache.len),
                                       tuple(host(x) for x in (mom.n, mom.mu_k, mom.mu_v, mom.C)), 1, example.TAU, Kt, Vt,
                                       np.full((b * beams, h), step), np.full(b, beams))
            assert (np.abs(host(out[i]).astype(np.float64) - want) <= tol).all(), (step, i)
        new = [[([host(s.qkv[i])[bi, j, hq:hq + h] for i in range(layers)], [host(s.qkv[i])[bi, j, hq + h:] for i in range(layers)])
                for j in range(beams)] for bi in range(b)]
        parent, token = s.choose()
        assert mkv.mkv_get_device_error(s.ws_select)[0] == 0
        want = R.select(host(s.logits), host(before[0]), host(before[1]), example.END, beams)
        assert want[4] > 2e-6  # (gaps that fp32 terms cannot close)
        assert (host(parent) == want[0]).all() and (host(token) == want[1]).all() and (host(s.done) == want[3]).all()
        rows = [[rows[bi][p] + [new[bi][p]] for p in host(parent)[bi]] for bi in range(b)]
        for i, tail in enumerate(s.tails):
            assert (tail.len == step + 1).all() and (tail.seen == T + step + 1).all()
            for bi in range(b):
                for j in range(beams):
                    u = bi * beams + j
                    assert (host(tail.pos)[u, :, :step + 1] == T + np.arange(step + 1)).all()
                    for t, (kr, vr) in enumerate(rows[bi][j]):
                        assert (host(tail.K)[u, :, t] == kr[i]).all() and (host(tail.V)[u, :, t] == vr[i]).all()


def test_example_runs(example, monkeypatch):
    real = example.BeamSearch
    monkeypatch.setattr(example, "BeamSearch", lambda **kw: real(batch=2, beams=3, heads=2, layers=2, T=300, budget=64, vocab=500, steps=16))
    example.main()
