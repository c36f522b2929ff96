"""One speculative decoding step over compressed caches, as a server makes it.

Prompt: rotary positions on queries and keys (time, height and width axes),
then one mkv_compress per layer.  Step: a drafted tree's visibility words and
positions (mkv_tree_build), and per layer the nodes' rotary positions
(mkv_rope) and their attention over the retained rows, the nodes they see and
the moment term (mkv_tree_step).  Then the accepted path goes into the caches
of all layers (mkv_tree_commit), and every layer is evicted back to its budget.

There is no model here: projections are random, and the "verifier" accepts the
path to each tree's last node.  python examples/speculative_step.py
prints the time of the step's calls.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_01563_gb300 import mkv  # noqa: E402

TAU = 1e-6


def frequencies(dim, base=1e6):
    """Inverse frequencies, and their axes: a quarter turns with time, the rest with height and width."""
    m = dim // 2
    inv = [base ** (-i / m) for i in range(m)]
    return mkv.rope_params(inv, [0] * (m // 4) + [1] * (m // 4 + m // 8) + [2] * (m - m // 2 - m // 8))


class Layer:
    """One attention layer's caches, moments and workspaces, from a random prompt of T tokens."""

    def __init__(self, g, T, budget, room, rope, gen):
        b, h, grp, d = g.batch, g.n_kv_heads, g.group, g.head_dim
        self.g, self.budget = g, budget
        qkv = torch.randn(b, T, h * (grp + 2), d, generator=gen, device="cuda").bfloat16()
        q, k = qkv[:, :, :h * grp], qkv[:, :, h * grp:h * (grp + 1)]
        pos = torch.arange(T, dtype=torch.int32, device="cuda").expand(3, b, T)  # text: the same on every axis
        K = torch.empty(b, h, T, d, dtype=torch.bfloat16, device="cuda")
        mkv.mkv_rope(pos, rope, [(q, q), (k, K.transpose(1, 2))])
        V = qkv[:, :, h * (grp + 1):].transpose(1, 2).contiguous()
        window = 16
        q_obs = q[:, -window:].view(b, window, h, grp, d).permute(0, 2, 3, 1, 4).contiguous()
        p = mkv.mkv_compress_params(budget, window, 1, 1, 1, 1, 1, TAU)
        self.cache, self.mom = mkv.alloc_cache(g, budget + room), mkv.alloc_moments(g)
        ws = mkv.alloc_workspace(mkv.mkv_compress_workspace_size(g, T, p))
        mkv.mkv_compress(g, T, K, V, q_obs, p, self.cache, self.mom, ws)
        self.ws_evict = mkv.alloc_workspace(mkv.mkv_evict_workspace_size(g, budget + room))


class Speculation:
    """What a server keeps for trees of N nodes over L layers."""

    def __init__(self, batch=2, heads=4, group=4, dim=128, layers=3, T=2048, budget=256, nodes=24, path=8, seed=0):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.g = mkv.geom(batch, heads, group, dim)
        self.rope, self.nodes, self.path = frequencies(dim), nodes, path
        self.layers = [Layer(self.g, T, budget, path, self.rope, self.gen) for _ in range(layers)]
        i32 = dict(dtype=torch.int32, device="cuda")
        self.parents = torch.full((batch, nodes), -1, **i32)
        self.count = torch.full((batch,), nodes, **i32)
        self.mask = torch.empty(batch, nodes, (nodes + 31) // 32, **i32)
        self.pos = torch.empty(batch, nodes, **i32)
        # every layer's projection of the nodes: queries, keys and values of all heads side by side
        self.qkv = torch.empty(layers, batch, nodes, heads * (group + 2), dim, dtype=torch.bfloat16, device="cuda")
        hq = heads * group
        self.q, self.k, self.v = self.qkv[:, :, :, :hq], self.qkv[:, :, :, hq:hq + heads], self.qkv[:, :, :, hq + heads:]
        self.out = torch.empty(layers, batch, nodes, hq, dim, dtype=torch.bfloat16, device="cuda")
        self.commit = mkv.tree_layers([(layer.cache, self.k[i], self.v[i]) for i, layer in enumerate(self.layers)])
        self.tree = mkv.Tree(self.mask, self.count)
        self.params = mkv.mkv_decode_params(1, 1, TAU)
        self.ws = mkv.alloc_workspace(mkv.mkv_tree_workspace_size(self.g, nodes, budget + path))

    def draft(self):
        """A random tree per batch item and its projections, not yet rotated."""
        u = torch.rand(self.parents.shape, generator=self.gen, device="cuda")
        self.parents.copy_(torch.floor(u * torch.arange(self.nodes, device="cuda")))
        self.parents[:, 0] = -1
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=self.gen, device="cuda"))

    def attend(self):
        """The nodes' attention outputs of every layer; the projections are rotated in place.  (In a model a layer's
        projection follows from the output of the layer before; here all are given.)"""
        first = self.layers[0].cache.seen[:, 0]
        mkv.mkv_tree_build(self.parents, self.mask, self.pos, self.ws, count=self.count, base=first)
        at = self.pos.expand(3, -1, -1)  # drafted text: the same position on every axis
        for i, layer in enumerate(self.layers):
            q, k, v = self.q[i], self.k[i], self.v[i]
            mkv.mkv_rope(at, self.rope, [(q, q), (k, k)])
            mkv.mkv_tree_step(self.g, self.tree, q, k, v, layer.cache, layer.mom, self.params, self.out[i], None, self.ws)
        return self.out

    def verify(self):
        """Stands for the verifier: accepts the path that leads to each tree's last node, cut to the room of a cache."""
        path = torch.zeros(self.g.batch, self.path, dtype=torch.int32)
        taken = torch.zeros(self.g.batch, dtype=torch.int32)
        for i, row in enumerate(self.parents.tolist()):
            node, up = self.nodes - 1, []
            while node >= 0:
                up.append(node)
                node = row[node]
            up = up[::-1][:self.path]
            path[i, :len(up)] = torch.tensor(up, dtype=torch.int32)
            taken[i] = len(up)
        return path.cuda(), taken.cuda()

    def accept(self, path, taken):
        """The accepted nodes into every layer's cache, then back to the budget; the last accepted node's query scores
        the rows."""
        mkv.mkv_tree_commit(self.g, self.commit, path, taken, self.ws)
        last = path.gather(1, (taken.long() - 1).clamp(min=0)[:, None]).long()[:, 0]
        rows = torch.arange(self.g.batch, device="cuda")
        for i, layer in enumerate(self.layers):
            mkv.mkv_evict_append(self.g, self.q[i][rows, last].contiguous(), None, None, layer.budget, layer.cache,
                                 layer.mom, TAU, layer.ws_evict)


def main():
    s = Speculation(layers=8, nodes=48)
    s.draft()
    s.attend()  # warm-up; then the step's calls of all layers as one graph
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.attend()
    s.accept(*s.verify())
    for step in range(4):
        s.draft()
        path, taken = s.verify()
        torch.cuda.synchronize()
        a, b, c = (torch.cuda.Event(enable_timing=True) for _ in range(3))
        a.record()
        graph.replay()
        b.record()
        s.accept(path, taken)
        c.record()
        torch.cuda.synchronize()
        print(f"step {step}: {len(s.layers)} layers, {s.nodes} nodes: attention {1e3 * a.elapsed_time(b):.0f} us, accepted "
              f"{taken.tolist()}, commit and eviction {1e3 * b.elapsed_time(c):.0f} us, "
              f"rows per head {int(s.layers[0].cache.len[0, 0])}, evicted {int(s.layers[0].mom.n[0, 0])}")
    code, info = mkv.mkv_get_device_error(s.ws)
    assert code == 0, (code, info)


if __name__ == "__main__":
    main()
