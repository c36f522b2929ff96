"""What the binding of include/mkv_tree.h makes of tensors' shapes and strides
(CPU): the library's functions are replaced by a recorder, so that nothing is
launched and the integers that would reach the C calls can be read."""
import ctypes

import pytest
import torch

from paper_2606_01563_gb300 import mkv

BF = torch.bfloat16


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(mkv, "lib", lambda: r)
    monkeypatch.setattr(mkv, "_stream", lambda stream: 0)
    return r


def _step(b, n, h, g, d, q=None, k=None, v=None):
    geo = mkv.geom(b, h, g, d)
    q = torch.zeros(b, n, h * g, d, dtype=BF) if q is None else q
    k = torch.zeros(b, n, h, d, dtype=BF) if k is None else k
    v = torch.zeros(b, n, h, d, dtype=BF) if v is None else v
    tree = mkv.Tree(torch.zeros(b, n, (n + 31) // 32, dtype=torch.int32))
    mkv.mkv_tree_step(geo, tree, q, k, v, mkv.alloc_cache(geo, 8, "cpu"), None, mkv.mkv_decode_params(0, 1, 1e-6),
                      torch.zeros(b, n, h * g, d, dtype=BF), None, torch.zeros(256, dtype=torch.uint8))


def _commit(b, n, h, d, k, v):
    geo = mkv.geom(b, h, 1, d)
    layers = mkv.tree_layers([(mkv.alloc_cache(geo, 8, "cpu"), k, v)])
    i32 = dict(dtype=torch.int32)
    mkv.mkv_tree_commit(geo, layers, torch.zeros(b, 2, **i32), torch.zeros(b, **i32), torch.zeros(256, dtype=torch.uint8))
    return layers


@pytest.mark.parametrize("over", ["batch", "nodes"])
@pytest.mark.parametrize("what", ["q", "k", "v", "kv"])
def test_expanded_tensors_are_refused(recorder, over, what):
    """The C calls take a stride of 0 for the dense one: an expanded tensor would be read past its end."""
    b, n, h, g, d = 4, 8, 2, 2, 64

    def expanded(heads):
        one = torch.zeros(1 if over == "batch" else b, 1 if over == "nodes" else n, heads, d, dtype=BF)
        return one.expand(b, n, heads, d)
    kw = {"q": expanded(h * g)} if what == "q" else {x: expanded(h) for x in what}
    with pytest.raises(ValueError):
        _step(b, n, h, g, d, **kw)
    if what != "q":
        k, v = (kw.get(x, torch.zeros(b, n, h, d, dtype=BF)) for x in "kv")
        with pytest.raises(ValueError):
            _commit(b, n, h, d, k, v)
    assert not recorder.calls


def test_strides_that_go_out(recorder):
    b, n, h, g, d = 3, 5, 2, 4, 64
    qkv = torch.zeros(b, n + 2, h * (g + 2), d, dtype=BF)[:, :n]
    q, k, v = qkv[:, :, :h * g], qkv[:, :, h * g:h * (g + 1)], qkv[:, :, h * (g + 1):]
    _step(b, n, h, g, d, q, k, v)
    name, args = recorder.calls.pop()
    row = h * (g + 2) * d
    assert name == "mkv_tree_step" and list(args[1])[3:] == [row, (n + 2) * row] * 2
    t = _commit(b, n, h, d, k, v).tree
    assert (t.kv_node, t.kv_batch) == (row, (n + 2) * row)


def test_extents_of_one_may_have_any_stride(recorder):
    h, g, d = 2, 2, 64
    x = torch.zeros(1, 1, h * g, d, dtype=BF).expand(1, 1, h * g, d).as_strided((1, 1, h * g, d), (0, 0, d, 1))
    k = torch.zeros(1, 1, h, d, dtype=BF).as_strided((1, 1, h, d), (0, 0, d, 1))
    _step(1, 1, h, g, d, x, k, k)
    assert list(recorder.calls.pop()[1][1])[3:] == [0, 0, 0, 0]
    assert isinstance(_commit(1, 1, h, d, k, k).array, ctypes.Array)


def test_keys_and_values_of_one_batch_item_from_two_parents(recorder):
    """Their strides differ only where an extent is one: the same addresses are meant."""
    n, h, g, d = 5, 2, 2, 64
    k = torch.zeros(1, n, h, d, dtype=BF)
    v = torch.zeros(1, n + 4, h, d, dtype=BF)[:, :n]
    assert k.stride() != v.stride()
    _step(1, n, h, g, d, k=k, v=v)
    assert list(recorder.calls.pop()[1][1])[5:] == [h * d, 0]
    _commit(1, n, h, d, k, v)
    one = torch.zeros(3, 1, 1, d, dtype=BF)  # one node, one head
    _step(3, 1, 1, g, d, k=one, v=one.as_strided((3, 1, 1, d), (d, 7, 7, 1)))
    assert list(recorder.calls.pop()[1][1])[5:] == [0, d]


@pytest.mark.parametrize("v", [torch.zeros(2, 6, 2, 64, dtype=BF)[:, :5], torch.zeros(2, 5, 3, 64, dtype=BF)[:, :, :2],
                               torch.zeros(2, 5, 2, 128, dtype=BF)[..., ::2], torch.zeros(2, 2, 5, 64, dtype=BF).transpose(1, 2)])
def test_keys_and_values_of_unlike_strides_are_refused(recorder, v):
    with pytest.raises(ValueError):
        _step(2, 5, 2, 2, 64, v=v)
    assert not recorder.calls


@pytest.mark.parametrize("geo", [(1, 2, 64), (2, 1, 64), (2, 2, 128)])
def test_layers_with_a_cache_of_another_geometry_are_refused(geo):
    """A commit would write past such a cache's end."""
    kv = torch.zeros(2, 3, 2, 64, dtype=BF)
    cache = mkv.alloc_cache(mkv.geom(geo[0], geo[1], 1, geo[2]), 8, "cpu")
    with pytest.raises(ValueError):
        mkv.tree_layers([(cache, kv, kv)])
    mkv.tree_layers([(mkv.alloc_cache(mkv.geom(2, 2, 1, 64), 8, "cpu"), kv, kv)])


@pytest.mark.parametrize("h,g,d", [(8, 4, 128), (2, 8, 64), (5, 1, 128), (1, 2, 64)])
def test_a_workspace_serves_every_smaller_call(h, g, d):
    """Sized once for the largest batch, tree and capacity; the plans of smaller ones may need parts where it needs none."""
    caps, nodes = [1, 64, 128, 129, 500, 1040, 2064, 2304, 9000, 131072], [1, 8, 16, 31, 32, 33, 64, 65, 100, 128, 200, 256]
    batches = [1, 2, 4, 9, 32, 100, 600]
    size = {(b, n, c): mkv.mkv_tree_workspace_size(mkv.geom(b, h, g, d), n, c) for b in batches for n in nodes for c in caps}
    for b, n, c in size:
        assert size[b, n, c] >= 256 and size[b, n, c] <= 50 << 20
        for smaller in ((x, n, c) for x in batches if x < b), ((b, x, c) for x in nodes if x < n), ((b, n, x) for x in caps if x < c):
            assert all(size[s] <= size[b, n, c] for s in smaller), (b, n, c)
