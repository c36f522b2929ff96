"""Beam search over one compressed prompt, as a server makes its steps.

Prompt: norms and rotary positions of queries and keys (mkv_norm_rope), then one
mkv_compress per layer; the retained rows and moments are held once per prompt.
Step: per layer the new tokens' norms and positions and their attention over the
prompt and their own tails (mkv_prefix_step), then the best continuations of
every prompt (mkv_beam_select) and the selected beams' tails in all layers
(mkv_beam_reorder).

There is no model here: a token's projections are rows of a random table, and logits a random
matrix times the last layer's output.  python examples/beam_search.py prints
the time of a step's calls.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_01563_gb300 import mkv  # noqa: E402

TAU, EPS, END = 1e-6, 1e-6, 1


class BeamSearch:
    """What a server keeps for `beams` beams of each of `batch` prompts over `layers` layers."""

    def __init__(self, batch=2, beams=4, heads=4, group=4, dim=128, layers=3, T=1500, budget=256, vocab=1000, steps=16,
                 seed=0):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.g, self.beams, self.heads_q, self.T = mkv.geom(batch, heads, group, dim), beams, heads * group, T
        self.rope = mkv.rope_params([1e6 ** (-2 * i / dim) for i in range(dim // 2)])
        bf, i32 = dict(dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.int32, device="cuda")
        self.weights = [[1 + 0.1 * self.randn(dim) for _ in ("q", "k")] for _ in range(layers)]
        self.table = self.randn(layers, vocab, heads * (group + 2), dim).bfloat16()
        self.head = self.randn(self.heads_q * dim, vocab).bfloat16() / 2
        self.prompts = [self.prompt(i, budget) for i in range(layers)]
        states = mkv.geom(batch * beams, heads, group, dim)
        self.tails = [mkv.alloc_cache(states, steps) for _ in range(layers)]
        for tail in self.tails:
            tail.seen.fill_(T)
        self.seqs, self.params = mkv.Seqs(beams), mkv.mkv_decode_params(1, 1, TAU)
        self.qkv = torch.empty(layers, batch, beams, heads * (group + 2), dim, **bf)
        self.out = torch.empty(layers, batch, beams, self.heads_q, dim, **bf)
        self.logits = torch.empty(batch, beams, vocab, **bf)
        # at first only one beam of a prompt is alive
        self.score = torch.full((batch, beams), -float("inf"), device="cuda")
        self.score[:, 0] = 0
        self.done, self.parent = (torch.zeros(batch, beams, **i32) for _ in range(2))
        self.token = torch.randint(2, vocab, (batch, 1), generator=self.gen, device="cuda").int().expand(-1, beams).contiguous()
        self.position = torch.full((batch, 1), T, **i32)
        self.states = mkv.beam_layers([(tail, None) for tail in self.tails])
        self.ws = mkv.alloc_workspace(mkv.mkv_prefix_workspace_size(self.g, beams, budget, steps))
        self.ws_select = mkv.alloc_workspace(mkv.mkv_beam_select_workspace_size(batch, beams, vocab, beams))

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda")

    def norm_rope(self, layer, pos, qkv, q_out, k_out):
        h, hq = self.g.n_kv_heads, self.heads_q
        wq, wk = self.weights[layer]
        mkv.mkv_norm_rope(pos, self.rope, [(qkv[:, :, :hq], q_out, wq), (qkv[:, :, hq:hq + h], k_out, wk)], EPS)

    def prompt(self, layer, budget):
        """A layer's retained rows and moments of random prompts."""
        g, T, window = self.g, self.T, 16
        b, h, d = g.batch, g.n_kv_heads, g.head_dim
        qkv = self.randn(b, T, h * (g.group + 2), d).bfloat16()
        q, K = torch.empty(b, T, self.heads_q, d, dtype=torch.bfloat16, device="cuda"), torch.empty(b, h, T, d, dtype=torch.bfloat16, device="cuda")
        pos = torch.arange(T, dtype=torch.int32, device="cuda").expand(1, b, T)
        self.norm_rope(layer, pos, qkv, q, K.transpose(1, 2))
        V = qkv[:, :, self.heads_q + h:].transpose(1, 2).contiguous()
        q_obs = q[:, -window:].view(b, window, h, g.group, d).permute(0, 2, 3, 1, 4).contiguous()
        p = mkv.mkv_compress_params(budget, window, 1, 1, 1, 1, 1, TAU)
        cache, mom = mkv.alloc_cache(g, budget), mkv.alloc_moments(g)
        mkv.mkv_compress(g, T, K, V, q_obs, p, cache, mom, mkv.alloc_workspace(mkv.mkv_compress_workspace_size(g, T, p)))
        return cache, mom

    def attend(self):
        """The beams' tokens through every layer's attention.  (In a model a layer's projection follows from the output
        of the layer before; here all are given.)"""
        h, hq = self.g.n_kv_heads, self.heads_q
        at = self.position.expand(-1, self.beams)[None]
        for i, ((cache, mom), tail) in enumerate(zip(self.prompts, self.tails)):
            qkv = self.qkv[i]
            torch.index_select(self.table[i], 0, self.token.view(-1), out=qkv.view(-1, *qkv.shape[2:]))
            q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + h], qkv[:, :, hq + h:]
            # (a token's beams stand for the tokens of a sequence: one position for all of them)
            self.norm_rope(i, at.contiguous(), qkv, q, k)
            mkv.mkv_prefix_step(self.g, self.seqs, q, k, v, cache, mom, tail, self.params, self.out[i], None, self.ws)
        torch.matmul(self.out[-1].flatten(2), self.head, out=self.logits)
        return self.out

    def choose(self):
        """The best continuations, their scores and ends, and their tails in every layer."""
        mkv.mkv_beam_select(self.logits, self.score, self.parent, self.token, self.score, self.ws_select, done=self.done,
                            done_out=self.done, end_token=END)
        mkv.mkv_beam_reorder(self.g, self.states, self.parent, self.ws_select)
        self.position += 1
        return self.parent, self.token


def main():
    s = BeamSearch(batch=4, beams=8, heads=8, layers=8, T=4096, budget=1024, vocab=32000, steps=64)
    s.attend()  # warm-up; then a step's calls of all layers as one graph
    s.choose()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.attend()
        s.choose()
    for step in range(4):
        torch.cuda.synchronize()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        print(f"step {step}: {len(s.tails)} layers, {s.beams} beams of {s.g.batch} prompts: {1e3 * a.elapsed_time(b):.0f} us, tails of "
              f"{int(s.tails[0].len[0, 0])} rows, parents {s.parent[0].tolist()}, best score {float(s.score[0, 0]):.2f}")
    for ws in (s.ws, s.ws_select):
        code, info = mkv.mkv_get_device_error(ws)
        assert code == 0, (code, info)


if __name__ == "__main__":
    main()
