"""include/mkv_tree.h: every declared function is exported and bound, the
header compiles as C99 and C++ with the layouts the binding declares, and bad
arguments are refused before anything is launched.  Runs on the CPU."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import tree_ref as R
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


def test_every_declared_function_is_exported_and_bound(L):
    src = open(os.path.join(ROOT, "include", "mkv_tree.h")).read()
    names = set(re.findall(r"MKV_API\s+[\w\s\*]+?\b(mkv_\w+)\s*\(", src))
    assert names == set(mkv.TREE_EXPORTS)
    for n in names:
        assert hasattr(L, n) and hasattr(mkv, n), n


CLIENT = r"""
#include <stddef.h>
#include <stdio.h>
#include "mkv_tree.h"
#define CHECK(c) do { if (!(c)) { printf("FAIL %d: %s\n", __LINE__, #c); return 1; } } while (0)
int main(void) {
  CHECK(sizeof(mkv_tree) == 56 && offsetof(mkv_tree, mask) == 16 && offsetof(mkv_tree, kv_batch) == 48);
  CHECK(sizeof(mkv_tree_layer) == 80 && offsetof(mkv_tree_layer, k) == 64);
  CHECK(sizeof(mkv_rope_params) == 16 + 512 && offsetof(mkv_rope_params, axis) == 272);
  CHECK(sizeof(mkv_rope_tensor) == 72 && offsetof(mkv_rope_tensor, in_batch) == 24);
  CHECK(MKV_TREE_MAX_NODES == 256);
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
    assert [ctypes.sizeof(x) for x in (mkv.mkv_tree, mkv.mkv_tree_layer, mkv.mkv_rope_params, mkv.mkv_rope_tensor)] == [
        56, 80, 528, 72]


def _step(L, g=None, tree=None, q=FAKE, k=FAKE, v=FAKE, cache=None, mom=None, p=None, out=FAKE, lse=FAKE, ws=FAKE,
          wsb=1 << 40):
    g = g or mkv.geom(2, 3, 4, 128)
    tree = tree or mkv.mkv_tree(8, None, FAKE, 0, 0, 0, 0)
    cache = cache or mkv.mkv_cache(FAKE, FAKE, FAKE, FAKE, FAKE, 64)
    mom = mom or mkv.mkv_moments(FAKE, FAKE, FAKE, FAKE)
    p = p or mkv.mkv_decode_params(1, 1, 1e-6)
    return L.mkv_tree_step(g, ctypes.byref(tree), q, k, v, ctypes.byref(cache), ctypes.byref(mom), ctypes.byref(p), out,
                           lse, ws, wsb, None)


def test_step_refusals(L):
    T = mkv.mkv_tree
    assert _step(L, g=mkv.geom(2, 3, 4, 96)) == UNSUPPORTED
    assert _step(L, g=mkv.geom(2, 3, 3, 128)) == SHAPE
    for n in (0, 257, -1):
        assert _step(L, tree=T(n, None, FAKE, 0, 0, 0, 0)) == SHAPE
        assert mkv.mkv_tree_workspace_size(mkv.geom(1, 1, 1, 64), n, 10) == 0
    assert mkv.mkv_tree_workspace_size(mkv.geom(1, 1, 1, 64), 5, 0) == 0
    assert mkv.mkv_tree_workspace_size(mkv.geom(1, 1, 1, 96), 5, 10) == 0
    for name in ("q", "k", "v", "out"):
        assert _step(L, **{name: None}) == INVALID
        assert _step(L, **{name: FAKE + 8}) == INVALID
    assert _step(L, lse=FAKE + 2) == INVALID
    assert _step(L, tree=T(8, None, None, 0, 0, 0, 0)) == INVALID
    assert _step(L, tree=T(8, None, FAKE + 1, 0, 0, 0, 0)) == INVALID
    assert _step(L, tree=T(8, FAKE + 1, FAKE, 0, 0, 0, 0)) == INVALID
    dense_q, dense_kv = 12 * 128, 3 * 128
    for strides in [(dense_q - 8, 0, 0, 0), (dense_q + 4, 0, 0, 0), (0, 8 * dense_q - 8, 0, 0), (0, 0, dense_kv - 8, 0),
                    (0, 0, dense_kv + 1, 0), (0, 0, 0, 8 * dense_kv - 8), (-8, 0, 0, 0), (1 << 40, 0, 0, 0)]:
        assert _step(L, tree=T(8, None, FAKE, *strides)) == INVALID, strides
    assert _step(L, mom=mkv.mkv_moments(FAKE, FAKE + 4, FAKE, FAKE)) == INVALID
    assert _step(L, p=mkv.mkv_decode_params(2, 1, 1e-6)) == INVALID
    assert _step(L, p=mkv.mkv_decode_params(1, 1, -1.0)) == INVALID
    assert _step(L, p=mkv.mkv_decode_params(1, 1, 1e-6, FAKE, 0, FAKE)) == INVALID
    assert _step(L, cache=mkv.mkv_cache(FAKE + 8, FAKE, FAKE, FAKE, FAKE, 64)) == INVALID
    assert _step(L, ws=None) == WORKSPACE
    assert _step(L, ws=FAKE + 128) == WORKSPACE
    need = mkv.mkv_tree_workspace_size(mkv.geom(2, 3, 4, 128), 8, 64)
    assert need >= 256 and _step(L, wsb=need - 1) == WORKSPACE


def test_build_refusals(L):
    def build(b=2, n=4, parents=FAKE, count=None, base=None, bs=0, mask=FAKE, pos=FAKE, ws=FAKE, wsb=256):
        return L.mkv_tree_build(b, n, parents, count, base, bs, mask, pos, ws, wsb, None)
    for b, n in ((0, 4), (65536, 4), (2, 0), (2, 257)):
        assert build(b=b, n=n) == SHAPE
    assert build(parents=None) == INVALID and build(mask=None) == INVALID and build(parents=FAKE + 2) == INVALID
    assert build(count=FAKE + 1) == INVALID and build(base=FAKE + 3) == INVALID and build(bs=-1) == INVALID
    assert build(ws=None) == WORKSPACE and build(wsb=255) == WORKSPACE and build(ws=FAKE + 4) == WORKSPACE


def test_commit_refusals(L):
    def commit(g=mkv.geom(2, 3, 4, 128), n=8, layers=1, path=FAKE, P=3, taken=FAKE, ws=FAKE, wsb=256, k=FAKE, kv=0,
               cache=mkv.mkv_cache(FAKE, FAKE, FAKE, FAKE, FAKE, 64), null=False):
        arr = (mkv.mkv_tree_layer * 1)(mkv.mkv_tree_layer(cache, k, FAKE))
        tree = mkv.mkv_tree(n, None, None, 0, 0, kv, 0)
        return L.mkv_tree_commit(g, ctypes.byref(tree), layers, None if null else arr, path, P, taken, ws, wsb, None)
    assert commit(g=mkv.geom(2, 3, 4, 80)) == UNSUPPORTED and commit(g=mkv.geom(0, 3, 4, 64)) == SHAPE
    assert commit(n=0) == SHAPE and commit(n=257) == SHAPE and commit(P=0) == SHAPE and commit(P=257) == SHAPE
    assert commit(path=None) == INVALID and commit(taken=None) == INVALID and commit(null=True) == INVALID
    assert commit(k=None) == INVALID and commit(k=FAKE + 8) == INVALID and commit(kv=100) == INVALID
    assert commit(layers=-1) == INVALID
    assert commit(cache=mkv.mkv_cache(FAKE, FAKE, None, FAKE, FAKE, 64)) == INVALID
    assert commit(ws=None) == WORKSPACE and commit(wsb=0) == WORKSPACE
    assert commit(layers=0) == OK  # nothing to launch


def test_rope_refusals(L):
    def rope(b=1, t=4, d=128, pos=FAKE, pa=0, pb=0, n=1, x=(FAKE, FAKE, 2, 0, 256, 128, 0, 256, 128), rot=128, axes=1,
             freq=1.0, axis=0, **flags):
        p = mkv.rope_params([freq] * (rot // 2), [axis] * (rot // 2))
        p.rot_dim, p.n_axes = rot, axes
        for name, v in flags.items():
            setattr(p, name, v)
        arr = (mkv.mkv_rope_tensor * 4)(*(mkv.mkv_rope_tensor(*x) for _ in range(4)))
        return L.mkv_rope(b, t, d, pos, pa, pb, ctypes.byref(p), n, arr, None)
    assert rope(d=96, rot=64) == UNSUPPORTED
    assert rope(b=0) == SHAPE and rope(t=-1) == SHAPE and rope(n=0) == SHAPE and rope(n=5) == SHAPE
    assert rope(b=65536, t=65536) == SHAPE
    assert rope(pos=None) == INVALID and rope(pos=FAKE + 2) == INVALID and rope(pa=-1) == INVALID
    for rot in (0, 8, 24, 72):
        assert rope(rot=rot) == INVALID, rot
    assert rope(d=64, rot=128) == INVALID
    assert rope(axes=0) == INVALID and rope(axes=5) == INVALID and rope(axes=2, axis=2) == INVALID
    assert rope(axis=-1) == INVALID and rope(inverse=2) == INVALID and rope(neighbours=-1) == INVALID
    for f in (float("nan"), float("inf"), 2.0 ** 21):
        assert rope(freq=f) == INVALID
    for x in [(None, FAKE, 2, 0, 256, 128, 0, 256, 128), (FAKE, FAKE + 8, 2, 0, 256, 128, 0, 256, 128),
              (FAKE, FAKE, 0, 0, 256, 128, 0, 256, 128), (FAKE, FAKE, 2, 0, 252, 128, 0, 256, 128),
              (FAKE, FAKE, 2, 0, 256, -128, 0, 256, 128), (FAKE, FAKE, 2, 0, 256, 128, 0, 0, 128),
              (FAKE, FAKE, 2, 0, 256, 128, 0, 256, 0)]:
        assert rope(x=x) == INVALID, x
    assert rope(b=2, x=(FAKE, FAKE, 2, 0, 256, 128, 0, 256, 128)) == INVALID  # two items written to one place
    assert rope(t=0) == OK  # nothing to launch


def test_binding_refuses_tensors_it_cannot_describe():
    g = mkv.geom(1, 2, 2, 64)
    cache, mom = mkv.alloc_cache(g, 8, "cpu"), None
    p, ws = mkv.mkv_decode_params(0, 1, 1e-6), torch.zeros(256, dtype=torch.uint8)
    bf = torch.bfloat16
    good = dict(q=torch.zeros(1, 3, 4, 64, dtype=bf), k=torch.zeros(1, 3, 2, 64, dtype=bf),
                v=torch.zeros(1, 3, 2, 64, dtype=bf), out=torch.zeros(1, 3, 4, 64, dtype=bf), lse=torch.zeros(1, 3, 4))
    tree = mkv.Tree(torch.zeros(1, 3, 1, dtype=torch.int32))

    def step(tree=tree, **kw):
        a = {**good, **kw}
        mkv.mkv_tree_step(g, tree, a["q"], a["k"], a["v"], cache, mom, p, a["out"], a["lse"], ws)

    for kw in [dict(q=good["q"].float()), dict(q=good["q"][:, :2]), dict(q=good["q"].transpose(2, 3)),
               dict(k=torch.zeros(1, 3, 2, 128, dtype=bf)[..., ::2]), dict(v=torch.zeros(1, 3, 4, 64, dtype=bf)[:, :, :2]),
               dict(out=good["out"].float()), dict(lse=torch.zeros(1, 3, 4, dtype=bf)),
               dict(tree=mkv.Tree(torch.zeros(1, 3, 2, dtype=torch.int32))),
               dict(tree=mkv.Tree(tree.mask, torch.zeros(1, dtype=torch.int64)))]:
        with pytest.raises(ValueError):
            step(**kw)
    with pytest.raises(ValueError):
        mkv.rope_params([1.0] * 65)
    x = torch.zeros(1, 3, 2, 64, dtype=bf)
    pos = torch.zeros(1, 1, 3, dtype=torch.int32)
    for bad in [(pos.long(), x, x), (pos, x.float(), x), (pos, x, x[:, :2]), (pos, x.transpose(2, 3), x.transpose(2, 3))]:
        with pytest.raises(ValueError):
            mkv.mkv_rope(bad[0], mkv.rope_params([1.0] * 32), [bad[1:]])


def test_reference_forms():
    """The 64-bit forms the GPU tests compare with, pinned by library attention and by complex rotation."""
    rng = np.random.default_rng(0)
    b, n, h, g, d, rows = 1, 5, 2, 2, 64, 9
    q, k, v = (rng.standard_normal((b, n, x, d)) for x in (h * g, h, h))
    K, V = rng.standard_normal((2, b, h, rows, d))
    parents = np.array([[-1, 0, 0, 2, -1]])
    sees = R.visible(parents, [n])
    assert sees == [[[0], [0, 1], [0, 2], [0, 2, 3], [4]]]
    assert R.words(sees, n)[0, :, 0].tolist() == [1, 3, 5, 13, 16]
    out, lse, _, _ = R.attend(q, k, v, sees, K, V, np.full((b, h), rows), None, 1, 0.0, [n])
    vis = torch.zeros(n, rows + n, dtype=torch.bool)
    vis[:, :rows] = True
    for i, s in enumerate(sees[0]):
        vis[i, [rows + a for a in s]] = True
    for hq in range(h * g):
        t = [torch.from_numpy(x) for x in (q[0, :, hq], np.concatenate([K[0, hq // g], k[0, :, hq // g]]),
                                           np.concatenate([V[0, hq // g], v[0, :, hq // g]]))]
        ref = torch.nn.functional.scaled_dot_product_attention(*(x[None] for x in t), attn_mask=vis[None])[0]
        np.testing.assert_allclose(out[0, :, hq], ref.numpy(), rtol=1e-12, atol=1e-12)
        z = torch.logsumexp((t[0] @ t[1].T / 8).masked_fill(~vis, -np.inf), -1)
        np.testing.assert_allclose(lse[0, :, hq], z.numpy(), rtol=1e-12)
    # the moment term of evicted tokens with one common key: n tokens at that key and the mean value
    key, vals = rng.standard_normal(d), rng.standard_normal((7, d))
    mom = (np.full((b, h), 7), np.tile(key, (b, h, 1)), np.tile(vals.mean(0), (b, h, 1)), np.zeros((b, h, d, d)))
    got = R.attend(q, k, v, sees, K, V, np.full((b, h), rows), mom, 1, 0.0, [n])
    K2, V2 = (np.concatenate([x, np.tile(y, (b, h, 1, 1))], 2) for x, y in ((K, np.tile(key, (7, 1))), (V, vals)))
    want = R.attend(q, k, v, sees, K2, V2, np.full((b, h), rows + 7), None, 1, 0.0, [n])
    np.testing.assert_allclose(got[0], want[0], rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(got[1], want[1], rtol=1e-12)
    x, pos, inv = rng.standard_normal((1, 3, 2, 64)), np.array([[[1, 5, 9]], [[2, 4, 8]]]), np.linspace(0.1, 1, 16)
    axis = np.arange(16) % 2
    y = R.rotate(x, pos, inv, axis, True, False)
    z = x[..., 0:32:2] + 1j * x[..., 1:32:2]
    turned = z * np.exp(1j * (pos[axis, 0].T * inv.astype(np.float32)))[None, :, None]
    np.testing.assert_allclose(y[..., 0:32:2] + 1j * y[..., 1:32:2], turned, rtol=1e-9)
    np.testing.assert_allclose(R.rotate(y, pos, inv, axis, True, True), x, rtol=1e-12)
