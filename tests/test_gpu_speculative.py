"""The speculative decoding example end to end: the nodes' outputs against a
plain 64-bit form, and the caches after a commit against those that decode
steps leave when they append the same tokens one by one."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import tree_ref as R
from paper_2606_01563_gb300 import mkv
from gpu_util import host

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TAU = 1e-6


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("speculative_step", os.path.join(ROOT, "examples", "speculative_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _state(layer):
    c, m = layer.cache, layer.mom
    return mkv.Cache(*(x.clone() for x in (c.K, c.V, c.pos, c.len, c.seen))), mkv.Moments(*(x.clone() for x in (m.n, m.mu_k, m.mu_v, m.C)))


@pytest.mark.parametrize("dim,group,nodes", [(128, 4, 24), (64, 8, 40)])
def test_step_against_plain_forms_and_decode_steps(example, dim, group, nodes):
    s = example.Speculation(batch=2, heads=2, group=group, dim=dim, layers=2, T=700, budget=96, nodes=nodes, seed=dim)
    for _ in range(2):
        s.draft()
        plain = s.qkv.clone()
        before = [_state(layer) for layer in s.layers]
        out = s.attend().clone()
        assert mkv.mkv_get_device_error(s.ws)[0] == 0
        sees = R.visible(s.parents.cpu().numpy(), s.count.cpu().numpy())
        pos = host(s.pos).astype(int)
        seen = host(before[0][0].seen)
        assert (pos == seen[:, :1] + np.array([[len(x) - 1 for x in rows] for rows in sees])).all()
        inv, axis = np.array(s.rope.inv_freq[:dim // 2]), np.array(s.rope.axis[:dim // 2])
        at = np.broadcast_to(pos, (3, *pos.shape))
        hq, h = s.q.shape[3], s.k.shape[3]
        for i, (cache, mom) in enumerate(before):
            # the rotation by its own bound: one rounding to bf16
            for got, x in ((s.q[i], plain[i, :, :, :hq]), (s.k[i], plain[i, :, :, hq:hq + h])):
                ref = R.rotate(host(x), at, inv, axis, False, False)
                assert (np.abs(host(got) - ref) <= 1.001 * 2.0 ** -8 * np.abs(ref) + 2.0 ** -16).all()
            ref, _, tol, _ = R.attend(host(s.q[i]), host(s.k[i]), host(plain[i, :, :, hq + h:]), sees, host(cache.K), host(cache.V),
                                      host(cache.len), tuple(host(x) for x in (mom.n, mom.mu_k, mom.mu_v, mom.C)), 1, TAU,
                                      s.count.cpu().numpy())
            assert (np.abs(host(out[i]).astype(np.float64) - ref) <= tol).all()
        path, taken = s.verify()
        s.accept(path, taken)
        # the same tokens appended by decode steps, then the same eviction
        for i, (layer, (cache, mom)) in enumerate(zip(s.layers, before)):
            g = s.g
            for item in range(g.batch):
                one = mkv.geom(1, g.n_kv_heads, g.group, g.head_dim)
                c1 = mkv.Cache(*(x[item:item + 1].clone() for x in (cache.K, cache.V, cache.pos, cache.len, cache.seen)))
                m1 = mkv.Moments(*(x[item:item + 1].clone() for x in (mom.n, mom.mu_k, mom.mu_v, mom.C)))
                ws = mkv.alloc_workspace(mkv.mkv_decode_workspace_size(one, c1.capacity))
                y = torch.empty(1, g.n_kv_heads * g.group, g.head_dim, device="cuda")
                nodes_ = path[item, :int(taken[item])].long()
                for step, node in enumerate(nodes_):
                    mkv.mkv_decode_step(one, s.q[i][item:item + 1, node].contiguous(), s.k[i][item:item + 1, node].contiguous(),
                                        s.v[i][item:item + 1, node].contiguous(), c1, m1, s.params, y, None, ws)
                    # a node of the path attends over what decoding it would: to the roundings of weights and output
                    assert ((out[i][item, node].float() - y[0]).abs() <= 2.0 ** -8 * (4.0 + y[0].abs())).all()
                mkv.mkv_evict_append(one, s.q[i][item:item + 1, nodes_[-1]].contiguous(), None, None, layer.budget, c1, m1, TAU,
                                     layer.ws_evict)
                for got, want in ((layer.cache.K, c1.K), (layer.cache.V, c1.V), (layer.cache.pos, c1.pos)):
                    assert torch.equal(got[item, :, :layer.budget], want[0, :, :layer.budget])
                for got, want in ((layer.cache.len, c1.len), (layer.cache.seen, c1.seen), (layer.mom.n, m1.n)):
                    assert torch.equal(got[item], want[0])
                # the same kernel on the same rows (another number of units per launch)
                for got, want in ((layer.mom.mu_k, m1.mu_k), (layer.mom.mu_v, m1.mu_v), (layer.mom.C, m1.C)):
                    torch.testing.assert_close(got[item], want[0], rtol=1e-4, atol=1e-5)
