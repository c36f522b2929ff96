"""Several continuations of one compressed prompt (beam search, parallel
sampling) and the queries and keys that go into them: the calls whose time is
watched, as a user's program makes them.

prefix     one decoding step of all sequences that share a prompt
           (mkv_prefix_step): attention over the prompt's retained cache and
           moments, read once for all of them, and over each sequence's own
           tail, which the new token joins.
select     beam search's selection over beams and vocabulary
           (mkv_beam_select): the best continuations of every batch item.
reorder    the selected beams' states in every layer, in place
           (mkv_beam_reorder): caches, and moments where there are any.
normrope   norms of queries and keys per head with the rotation by position in
           the same pass (mkv_norm_rope), and its gradient
           (mkv_norm_rope_grad).

`own` chooses between the framework's kernels and the plain form: elementary
torch operations in 32 bits (angles, and the selection's sums and scores, whose
order decides, in 64), rounded once at the end.
"""
import math

import torch

own = False

TAU = 1e-6
EPS = 1e-6
EVICTED = 1024  # tokens behind the moments of a cache
END = 2         # the token that ends a sequence
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


def _prefix(name, batch, seqs, heads, group, dim, rows, tail, c, ragged):
    return {"name": name, "kind": "prefix", "batch": batch, "seqs": seqs, "heads": heads, "group": group, "dim": dim,
            "rows": rows, "tail": tail, "c": c, "ragged": ragged}


def _select(name, batch, beams, out, vocab, type_, padded, first):
    return {"name": name, "kind": "select", "batch": batch, "beams": beams, "out": out, "vocab": vocab, "type": type_,
            "padded": padded, "first": first}


def _reorder(name, layers, batch, seqs, heads, dim, rows, moments, ragged):
    return {"name": name, "kind": "reorder", "layers": layers, "batch": batch, "seqs": seqs, "heads": heads, "dim": dim,
            "rows": rows, "moments": moments, "ragged": ragged}


def _normrope(name, batch, heads, group, dim, tokens, rot, axes, pairs, weights, type_, grad):
    return {"name": name, "kind": "normrope", "batch": batch, "heads": heads, "group": group, "dim": dim,
            "tokens": tokens, "rot": rot, "axes": axes, "pairs": pairs, "weights": weights, "type": type_, "grad": grad}


def listed():
    return [
        # the smallest step: two sequences of one short prompt in a small model's layer, tails just begun
        _prefix("prefix_d64_b1_s2_r128_t3", 1, 2, 2, 2, 64, 128, 3, "f32", 0),
        # beam search with 8 beams on one Qwen3-4B layer, batch 4, budget 1024, C' in operand form
        _prefix("prefix_b4_s8_r1024_t100", 4, 8, 8, 4, 128, 1024, 100, "split", 0),
        # sampling 13 answers to each of 8 prompts, unequal numbers, prompts and answers, 16-bit moments
        _prefix("prefix_b8_s13_r4001_t300", 8, 13, 8, 4, 128, 4001, 300, "bf16", 1),
        # 64 answers to each of two 32K prompts kept whole (no eviction yet): the most rows and products
        _prefix("prefix_b2_s64_r32768_t256", 2, 64, 8, 4, 128, 32768, 256, "none", 0),
        # one request with 4 beams, the first step: only beam 0 is alive
        _select("select_b1_k4_v32000", 1, 4, 4, 32000, "bf16", 0, 1),
        # a batch of 32 requests with 8 beams, twice as many candidates (half of them may end), an odd vocabulary in padded rows
        _select("select_b32_k8_v150001", 32, 8, 16, 150001, "bf16", 1, 0),
        # 4 beams' tails in all 36 Qwen3-4B layers
        _reorder("reorder_l36_b1_s4_r64", 36, 1, 4, 8, 128, 64, 0, 0),
        # beams that evict: caches and moments of 8 layers, 4 requests with 16 beams, unequal lengths
        _reorder("reorder_l8_b4_s16_r512_m", 8, 4, 16, 8, 128, 512, 1, 1),
        # one token of 32 sequences: latency counts
        _normrope("normrope_b32_t1", 32, 8, 4, 128, 1, 128, 1, "halves", "shared", "bf16", 0),
        # a prompt before compress: one Qwen3-4B layer, batch 4, 32K tokens
        _normrope("normrope_b4_t32768", 4, 8, 4, 128, 32768, 128, 1, "halves", "shared", "bf16", 0),
        # training: the gradient of a batch of no round length, half of the dims rotated, neighbours paired, fp32 weights
        _normrope("normrope_grad_b2_t8191_r64", 2, 8, 4, 128, 8191, 64, 1, "neighbours", "shared", "f32", 1),
        # fine-tuning on a short sequence, weights of each head's own, three position axes
        _normrope("normrope_grad_d64_b1_t509", 1, 4, 2, 64, 509, 64, 3, "halves", "heads", "bf16", 1),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _geometry(rng):
    """(heads, group, dim): mostly the 8B-class geometry, else another built one."""
    if rng.random() < 0.5:
        return 8, 4, 128
    return rng.choice([2, 4, 5, 8]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128])


def draw(rng):
    heads, group, dim = _geometry(rng)
    kind = rng.choice(["prefix", "prefix", "prefix", "select", "select", "reorder", "normrope", "normrope"])
    if kind == "prefix":
        batch, seqs = _logint(rng, 1, 16), _logint(rng, 1, 64)
        units = batch * heads
        rows = _logint(rng, 48, max(48, min(2 ** 26 // (units * dim), 2 ** 27 // (units * seqs * group), 65536)))
        tail = rng.choice([0, 1, _logint(rng, 2, max(2, min(1024, 2 ** 25 // (units * seqs * dim))))])
        case = _prefix("", batch, seqs, heads, group, dim, rows, tail, rng.choice(["none", "f32", "bf16", "split"]),
                       rng.choice([0, 1]))
    elif kind == "select":
        batch, beams = _logint(rng, 1, 64), _logint(rng, 1, 32)
        vocab = _logint(rng, 1000, min(262144, 38000000 // (batch * beams)))
        case = _select("", batch, beams, rng.choice([beams, 2 * beams]), vocab, rng.choice(["bf16", "bf16", "f32"]),
                       rng.choice([0, 1]), rng.choice([0, 0, 1]))
        if case["type"] == "f32" and batch * beams * vocab > 19000000:
            case["type"] = "bf16"
    elif kind == "reorder":
        batch, seqs, layers, moments = _logint(rng, 1, 16), _logint(rng, 2, 32), rng.randint(1, 36), rng.choice([0, 1])
        units = batch * seqs * heads * layers
        while units > 4096:
            layers = max(1, layers // 2)
            batch = batch if layers > 1 else max(1, batch // 2)
            units = batch * seqs * heads * layers
        rows = _logint(rng, 8, min(2048, 4096 * 512 // units))
        case = _reorder("", layers, batch, seqs, heads, dim, rows, moments, rng.choice([0, 1]))
    else:
        batch, rot, grad = _logint(rng, 1, 64), rng.choice([dim, dim, dim // 2, 48]), rng.choice([0, 1])
        most = 4 * 32768 * 40 * 128 // (batch * heads * (group + 1) * dim)
        tokens = rng.choice([1, _logint(rng, 2, most // (4 if grad else 2))])
        case = _normrope("", batch, heads, group, dim, tokens, rot, rng.choice([1, 1, 3]),
                         rng.choice(["halves", "neighbours"]), rng.choice(["shared", "shared", "heads"]),
                         rng.choice(["bf16", "f32"]), grad)
    case.pop("name", None)
    return case


# ------------------------------------------------------------------ inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 29)
    return gen


def _prepare_prefix(c, seed):
    gen = _generator(seed)
    b, n, h, g, d, rows, tail = (c[x] for x in ("batch", "seqs", "heads", "group", "dim", "rows", "tail"))
    units, cap, cap_t = b * h, rows + 16, tail + 8
    lo, hi = math.log(0.5), math.log(4.0)
    scale = torch.exp(lo + (hi - lo) * torch.rand(units, 1, d, generator=gen, device="cuda"))

    def keys(m):
        return (torch.randn(units, m, d, generator=gen, device="cuda") * scale).to(BF16)

    def values(m):
        return torch.randn(units, m, d, generator=gen, device="cuda").to(BF16)

    def lengths(m, *shape):
        return torch.randint(m // 2, m + 1, shape, generator=gen, device="cuda", dtype=I32) if c["ragged"] else torch.full(
            shape, m, dtype=I32, device="cuda")

    def by_sequence(x, m):
        return x.view(b, h, n, m, d).transpose(1, 2).reshape(b * n, h, m, d)

    K, V = keys(cap), values(cap)
    s = {"case": c, "K": K.view(b, h, cap, d), "V": V.view(b, h, cap, d), "len": lengths(rows, b, h)}
    s["pos"] = torch.arange(cap, dtype=I32, device="cuda").expand(b, h, cap).contiguous()
    s["seen"] = s["len"] + EVICTED
    if c["c"] != "none":
        ke, ve = keys(EVICTED).float(), values(EVICTED).float()
        mk, mv = ke.mean(1), ve.mean(1)
        cov = torch.bmm((ve - mv[:, None]).transpose(1, 2), ke - mk[:, None]) / EVICTED
        s["n"] = torch.full((b, h), EVICTED, dtype=I32, device="cuda")
        s["mu_k"], s["mu_v"], s["C"] = mk.view(b, h, d), mv.view(b, h, d), cov.view(b, h, d, d).contiguous()
    # the sequences' tails, and how long they were before this step (a sequence's heads agree)
    s["Kt"], s["Vt"] = by_sequence(keys(n * cap_t), cap_t), by_sequence(values(n * cap_t), cap_t)
    s["post"] = torch.zeros(b * n, h, cap_t, dtype=I32, device="cuda")
    before = lengths(tail, b * n, 1).expand(b * n, h)
    s["state0"] = torch.stack([before, before + rows + EVICTED]).contiguous()
    s["state"] = s["state0"].clone()  # len and seen of the tails
    s["count"] = lengths(n, b).clamp(min=1)
    # a query lies near the sum of three retained keys
    pick = torch.randint(0, rows, (units, n * g, 3), generator=gen, device="cuda")
    q = K[torch.arange(units, device="cuda")[:, None, None], pick].float().sum(2)
    q = math.sqrt(d) * q / torch.linalg.norm(q, dim=-1, keepdim=True)
    q = q + 0.3 * torch.randn(q.shape, generator=gen, device="cuda")
    q = q.view(b, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, h * g, d)
    # queries, keys and values of a token lie behind one another, as a fused projection leaves them
    qkv = torch.empty(b, n, h * (g + 2), d, dtype=BF16, device="cuda")
    qkv[:, :, :h * g] = q.to(BF16)
    qkv[:, :, h * g:h * (g + 1)] = keys(n).view(b, h, n, d).transpose(1, 2)
    qkv[:, :, h * (g + 1):] = values(n).view(b, h, n, d).transpose(1, 2)
    s["q"], s["k"], s["v"] = qkv[:, :, :h * g], qkv[:, :, h * g:h * (g + 1)], qkv[:, :, h * (g + 1):]
    if own:
        s["call"] = _prefix_call(s)
    return s


def _prefix_call(s):
    """What a program keeps beside a layer's caches: the binding's views of them, the moments in the form that is
    read, the outputs and the workspace."""
    from paper_2606_01563_gb300 import mkv
    c = s["case"]
    b, n, h, g, d = c["batch"], c["seqs"], c["heads"], c["group"], c["dim"]
    geom = mkv.geom(b, h, g, d)
    s["Kt"], s["Vt"] = s["Kt"].contiguous(), s["Vt"].contiguous()  # (of one prompt's sequences they are a transposed view)
    prefix = mkv.Cache(s["K"], s["V"], s["pos"], s["len"], s["seen"])
    tail = mkv.Cache(s["Kt"], s["Vt"], s["post"], s["state"][0], s["state"][1])
    mom, c16, split = None, None, None
    if c["c"] != "none":
        mom = mkv.Moments(s["n"], s["mu_k"], s["mu_v"], s["C"])
        if c["c"] == "bf16":
            c16 = torch.empty(b, h, d, d, dtype=BF16, device="cuda")
            mkv.mkv_moments_pack_bf16(geom, mom, c16)
        elif c["c"] == "split":
            split = torch.empty(b, h, d, d, dtype=I32, device="cuda")
            mkv.mkv_moments_pack_split(geom, mom, TAU, split)
    p = mkv.mkv_decode_params(0 if mom is None else 1, 1, TAU, None if c16 is None else c16.data_ptr(), 0,
                              None if split is None else split.data_ptr())
    return {"g": geom, "prefix": prefix, "tail": tail, "mom": mom, "p": p, "held": (c16, split),
            "seqs": mkv.Seqs(n, s["count"]),
            "out": torch.empty(b, n, h * g, d, dtype=BF16, device="cuda"),
            "lse": torch.empty(b, n, h * g, dtype=F32, device="cuda"),
            "ws": mkv.alloc_workspace(mkv.mkv_prefix_workspace_size(geom, n, prefix.capacity, tail.capacity))}


def _prepare_select(c, seed):
    gen = _generator(seed)
    b, k, v = c["batch"], c["beams"], c["vocab"]
    stride = -(-v // 64) * 64 if c["padded"] else v
    # a flat bulk and, per beam, a few dozen tokens that stand out, as a language model's next-token scores
    logits = 1.5 * torch.randn(b, k, stride, generator=gen, device="cuda")
    best = torch.randint(0, v, (b, k, 40), generator=gen, device="cuda")
    logits.scatter_add_(2, best, 6 + 6 * torch.rand(b, k, 40, generator=gen, device="cuda"))
    s = {"case": c, "logits": logits.to(BF16 if c["type"] == "bf16" else F32)[:, :, :v]}
    s["score"] = -20 - 4 * torch.rand(b, k, generator=gen, device="cuda")
    if c["first"]:
        s["score"][:, 1:] = -math.inf
        s["done"] = torch.zeros(b, k, dtype=I32, device="cuda")
    else:
        s["done"] = (torch.rand(b, k, generator=gen, device="cuda") < 0.15).to(I32)
    if own:
        from paper_2606_01563_gb300 import mkv
        i32 = dict(dtype=I32, device="cuda")
        s["parent"], s["token"], s["over"] = (torch.empty(b, c["out"], **i32) for _ in range(3))
        s["best"] = torch.empty(b, c["out"], dtype=F32, device="cuda")
        s["ws"] = mkv.alloc_workspace(mkv.mkv_beam_select_workspace_size(b, k, v, c["out"]))
    return s


def _prepare_reorder(c, seed):
    gen = _generator(seed)
    layers, b, n, h, d, rows = c["layers"], c["batch"], c["seqs"], c["heads"], c["dim"], c["rows"]
    cap = rows + 8

    def rand(*shape, dtype=BF16):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = {"case": c, "K": rand(layers, b * n, h, cap, d), "V": rand(layers, b * n, h, cap, d),
         "pos": torch.randint(0, 100000, (layers, b * n, h, cap), generator=gen, device="cuda", dtype=I32)}
    shape = (layers, b * n, h)
    s["len"] = torch.full(shape, rows, dtype=I32, device="cuda")
    if c["ragged"]:
        s["len"] = torch.randint(rows // 2, rows + 1, shape, generator=gen, device="cuda", dtype=I32)
    s["seen"] = s["len"] + EVICTED
    if c["moments"]:
        s["n"] = torch.randint(0, 2 * EVICTED, shape, generator=gen, device="cuda", dtype=I32)
        s["mu_k"], s["mu_v"] = rand(*shape, d, dtype=F32), rand(*shape, d, dtype=F32)
        s["C"] = rand(*shape, d, d, dtype=F32)
    s["parent"] = torch.randint(0, n, (b, n), generator=gen, device="cuda", dtype=I32)
    if own:
        from paper_2606_01563_gb300 import mkv
        s["g"] = mkv.geom(b, h, 1, d)
        s["layers"] = mkv.beam_layers(
            [(mkv.Cache(s["K"][l], s["V"][l], s["pos"][l], s["len"][l], s["seen"][l]),
              mkv.Moments(s["n"][l], s["mu_k"][l], s["mu_v"][l], s["C"][l]) if c["moments"] else None)
             for l in range(layers)])
        s["ws"] = mkv.alloc_workspace(256)
    return s


def _freqs(c):
    """Inverse frequencies (fp32) and the axis of each: one axis, or 1/4, 3/8 and 3/8 of them on three."""
    m = c["rot"] // 2
    inv = [float(x) for x in torch.tensor([1e6 ** (-i / m) for i in range(m)], dtype=F32)]
    ends = [m] if c["axes"] == 1 else [m // 4, m // 4 + 3 * m // 8, m]
    return inv, [sum(i >= e for e in ends) for i in range(m)]


def _prepare_normrope(c, seed):
    gen = _generator(seed)
    b, h, g, d, t = c["batch"], c["heads"], c["group"], c["dim"], c["tokens"]

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=BF16)

    inv, axis = _freqs(c)
    i = torch.arange(t, device="cuda")
    wide = max(1, int(math.sqrt(t)))
    start = torch.randint(0, 4096, (b, 1), generator=gen, device="cuda")  # what a sequence has seen
    pos = torch.stack([i] if c["axes"] == 1 else [i // (4 * wide), i // wide, i % wide])
    s = {"case": c, "pos": (pos[:, None] + start).to(I32), "inv": torch.tensor(inv, dtype=F32, device="cuda"),
         "axis": torch.tensor(axis, device="cuda")}
    for name, heads in (("q", h * g), ("k", h)):
        shape = (heads, d) if c["weights"] == "heads" else (d,)
        w = 1 + 0.3 * torch.randn(*shape, generator=gen, device="cuda")
        s["w" + name] = w.to(BF16 if c["type"] == "bf16" else F32)
    # queries and keys as a fused projection leaves them, of a size that varies by token
    qkv = rand(b, t, h * (g + 2), d) * torch.exp(torch.randn(b, t, 1, 1, generator=gen, device="cuda")).to(BF16)
    s["q"], s["k"] = qkv[:, :, :h * g], qkv[:, :, h * g:h * (g + 1)]
    if c["grad"]:  # the results' gradients, in the layouts that the forward pass wrote
        s["dyq"], s["dyk"] = rand(b, t, h * g, d), rand(b, h, t, d).transpose(1, 2)
    if own:
        from paper_2606_01563_gb300 import mkv
        s["p"] = mkv.rope_params(inv, axis, c["pairs"] == "neighbours")
        if c["grad"]:
            dqkv = torch.empty_like(qkv)
            s["dq"], s["dk"] = dqkv[:, :, :h * g], dqkv[:, :, h * g:h * (g + 1)]
            s["dwq"], s["dwk"] = (torch.empty(s[w].shape, dtype=F32, device="cuda") for w in ("wq", "wk"))
            tensors = [(s["q"], s["dyq"], s["dq"], s["wq"], s["dwq"]), (s["k"], s["dyk"], s["dk"], s["wk"], s["dwk"])]
            s["ws"] = mkv.alloc_workspace(mkv.mkv_norm_rope_grad_workspace_size(tensors))
        else:
            s["q_out"] = torch.empty(b, t, h * g, d, dtype=BF16, device="cuda")
            s["k_out"] = torch.empty(b, h, t, d, dtype=BF16, device="cuda").transpose(1, 2)
            tensors = [(s["q"], s["q_out"], s["wq"]), (s["k"], s["k_out"], s["wk"])]
        s["tensors"] = tensors
    return s


def prepare(case, seed):
    return {"prefix": _prepare_prefix, "select": _prepare_select, "reorder": _prepare_reorder,
            "normrope": _prepare_normrope}[case["kind"]](case, seed)


# --------------------------------------------------------------------- run
def _live(c, count):
    """[b, n]: the sequences in use."""
    return torch.arange(c["seqs"], device="cuda") < count[:, None]


def _plain_prefix(s):
    c = s["case"]
    b, n, h, g, d = c["batch"], c["seqs"], c["heads"], c["group"], c["dim"]
    live = _live(c, s["count"])
    s["state"].copy_(s["state0"])
    # the new tokens join the tails of the sequences in use
    cap_t = s["Kt"].shape[2]
    length, seen = s["state"][0], s["state"][1]
    at = torch.arange(cap_t, device="cuda")
    new = ((at == length[..., None]) & live.view(b * n, 1, 1))
    s["Kt"].copy_(torch.where(new[..., None], s["k"].reshape(b * n, h, 1, d), s["Kt"]))
    s["Vt"].copy_(torch.where(new[..., None], s["v"].reshape(b * n, h, 1, d), s["Vt"]))
    s["post"].copy_(torch.where(new, seen[..., None], s["post"]))
    s["state"] += live.view(1, b * n, 1).to(I32)
    dead = ~live.repeat_interleave(g, 1)[:, None, :, None]  # [b, 1, n g, 1]
    q = s["q"].float().view(b, n, h, g, d).permute(0, 2, 1, 3, 4).reshape(b, h, n * g, d) * d ** -0.5
    x = q @ s["K"].float().transpose(2, 3)
    x = x.masked_fill_((torch.arange(x.shape[-1], device="cuda") >= s["len"][..., None, None]) | dead, -math.inf)
    qt = q.view(b, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(b * n, h, g, d)
    y = (qt @ s["Kt"].float().transpose(2, 3)).masked_fill_(at >= length[..., None, None], -math.inf)

    def by_prompt(z):  # [b n, h, g, ...] -> [b, h, n g, ...]
        return z.view(b, n, h, g, -1).permute(0, 2, 1, 3, 4).reshape(b, h, n * g, -1)

    top = torch.maximum(x.amax(-1, keepdim=True), by_prompt(y.amax(-1, keepdim=True)).masked_fill(dead, -math.inf))
    if c["c"] != "none":
        e = torch.log(s["n"].float())[..., None, None] + q @ s["mu_k"][..., None]
        e = e.masked_fill_(dead, -math.inf)
        top = torch.maximum(top, e)
    ref = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    ref_t = ref.view(b, h, n, g, 1).permute(0, 2, 1, 3, 4).reshape(b * n, h, g, 1)
    x, y = (x - ref).exp_(), (y - ref_t).exp_()
    total = x.sum(-1, keepdim=True) + by_prompt(y.sum(-1, keepdim=True))
    out = x @ s["V"].float() + by_prompt(y @ s["Vt"].float())
    if c["c"] != "none":
        C = s["C"].to(BF16).float() if c["c"] == "bf16" else s["C"]
        C = torch.where((C * s["n"][..., None, None]).abs() < TAU, torch.zeros_like(C), C)
        w = (e - ref).exp_()
        total = total + w
        out = out + w * (s["mu_v"][:, :, None] + q @ C.transpose(2, 3))
    out = torch.where(dead, torch.zeros_like(out), out / total)
    lse = torch.where(dead, torch.full_like(total, -math.inf), ref + torch.log(total))[..., 0]
    return {"out": out.view(b, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, h * g, d).to(BF16),
            "lse": lse.view(b, h, n, g).permute(0, 2, 1, 3).reshape(b, n, h * g),
            "K": s["Kt"], "V": s["Vt"], "pos": s["post"], "state": s["state"]}


def _plain_select(s):
    c = s["case"]
    b, k, v = c["batch"], c["beams"], c["vocab"]
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    x = x - (top + torch.log(torch.exp(x - top).sum(-1, keepdim=True)))
    x = s["score"].double()[..., None] + x
    # a beam that has ended has one continuation, itself
    at = torch.arange(v, device="cuda")
    ended = torch.where(at == END, s["score"].double()[..., None], torch.full_like(x, -math.inf))
    x = torch.where(s["done"][..., None] != 0, ended, x).view(b, k * v)
    best, at = torch.sort(x, dim=-1, descending=True, stable=True)
    best, at = best[:, :c["out"]], at[:, :c["out"]]
    parent, token = at // v, at % v
    over = (s["done"].gather(1, parent) != 0) | (token == END)
    none = torch.isinf(best)  # fewer continuations than slots
    parent, token, over = parent.masked_fill(none, -1), token.masked_fill(none, -1), over & ~none
    return {"parent": parent.to(I32), "token": token.to(I32), "score": best.to(F32), "done": over.to(I32)}


def _plain_reorder(s):
    c = s["case"]
    layers, b, n, h = c["layers"], c["batch"], c["seqs"], c["heads"]
    at = (torch.arange(b, device="cuda")[:, None] * n + s["parent"]).view(-1)
    rows = torch.arange(s["K"].shape[3], device="cuda") < s["len"][:, at][..., None]
    s["K"].copy_(torch.where(rows[..., None], s["K"][:, at], s["K"]))
    s["V"].copy_(torch.where(rows[..., None], s["V"][:, at], s["V"]))
    s["pos"].copy_(torch.where(rows, s["pos"][:, at], s["pos"]))
    names = ["len", "seen"] + (["n", "mu_k", "mu_v", "C"] if c["moments"] else [])
    [s[x].copy_(s[x][:, at]) for x in names]


def _angles(s):
    c = s["case"]
    angle = s["pos"].double()[s["axis"]].permute(1, 2, 0) * s["inv"].double()  # [b, tokens, rot / 2]
    return torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]


def _turn(x, cos, sin, rot, neighbours):
    if neighbours:
        a, c = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - c * sin, a * sin + c * cos], -1).flatten(-2)
    else:
        a, c = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - c * sin, a * sin + c * cos], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_normrope(s):
    c = s["case"]
    cos, sin = _angles(s)
    rot, neighbours = c["rot"], c["pairs"] == "neighbours"

    def forward(x, w):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        return _turn(y, cos, sin, rot, neighbours).to(BF16)

    def backward(x, dy, w):
        x, dn = x.float(), _turn(dy.float(), cos, -sin, rot, neighbours)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        y, gain = x * r, dn * w.float()
        dx = r * (gain - y * (gain * y).mean(-1, keepdim=True))
        return dx.to(BF16), (dn * y).sum((0, 1) if w.dim() == 2 else (0, 1, 2))

    if not c["grad"]:
        return {"q": forward(s["q"], s["wq"]), "k": forward(s["k"], s["wk"]).transpose(1, 2).contiguous()}
    (dq, dwq), (dk, dwk) = backward(s["q"], s["dyq"], s["wq"]), backward(s["k"], s["dyk"], s["wk"])
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if kind == "reorder":
        if own:
            from paper_2606_01563_gb300 import mkv
            mkv.mkv_beam_reorder(s["g"], s["layers"], s["parent"], s["ws"])
        else:
            _plain_reorder(s)
        return {x: s[x] for x in ["K", "V", "pos", "len", "seen"] + (["n", "mu_k", "mu_v", "C"] if c["moments"] else [])}
    if not own:
        return {"prefix": _plain_prefix, "select": _plain_select, "normrope": _plain_normrope}[kind](s)
    from paper_2606_01563_gb300 import mkv
    if kind == "prefix":
        a = s["call"]
        s["state"].copy_(s["state0"])  # the tails as the step before left them
        mkv.mkv_prefix_step(a["g"], a["seqs"], s["q"], s["k"], s["v"], a["prefix"], a["mom"], a["tail"], a["p"],
                            a["out"], a["lse"], a["ws"])
        return {"out": a["out"], "lse": a["lse"], "K": s["Kt"], "V": s["Vt"], "pos": s["post"], "state": s["state"]}
    if kind == "select":
        mkv.mkv_beam_select(s["logits"], s["score"], s["parent"], s["token"], s["best"], s["ws"], done=s["done"],
                            done_out=s["over"], end_token=END)
        return {"parent": s["parent"], "token": s["token"], "score": s["best"], "done": s["over"]}
    if c["grad"]:
        mkv.mkv_norm_rope_grad(s["pos"], s["p"], s["tensors"], EPS, s["ws"])
        return {x: s[x] for x in ("dq", "dk", "dwq", "dwk")}
    mkv.mkv_norm_rope(s["pos"], s["p"], s["tensors"], EPS)
    return {"q": s["q_out"], "k": s["k_out"].transpose(1, 2)}


# -------------------------------------------------------------------- work
def work(case):
    c = case
    b = c["batch"]
    if c["kind"] == "select":
        rows = b * (1 if c["first"] else 0.85 * c["beams"])
        return {"bytes": int(rows * c["vocab"] * (2 if c["type"] == "bf16" else 4) + b * (8 * c["beams"] + 16 * c["out"])),
                "flops": int(4 * rows * c["vocab"])}
    h, d = c["heads"], c["dim"]
    share = 0.75 if c.get("ragged") else 1
    if c["kind"] == "reorder":
        n = c["seqs"]
        # a state that is some slot's parent is read once, and every slot but its own parent's is written
        read, written = b * (n - n * (1 - 1 / n) ** n), b * (n - 1)
        state = c["rows"] * share * (4 * d + 4) + 8 + (4 * d * d + 8 * d + 4 if c["moments"] else 0)
        return {"bytes": int(c["layers"] * h * state * (read + written)), "flops": 0}
    g = c["group"]
    if c["kind"] == "normrope":
        values = b * c["tokens"] * h * (g + 1) * d
        weights = (h * (g + 1) if c["weights"] == "heads" else 2) * d
        by = values * (6 if c["grad"] else 4) + 4 * c["axes"] * b * c["tokens"]
        by += weights * ((2 if c["type"] == "bf16" else 4) + (4 if c["grad"] else 0))
        return {"bytes": by, "flops": values * (14 if c["grad"] else 7)}
    n, units = c["seqs"], b * h
    live, rows, tail = n * share, c["rows"] * share, c["tail"] * share + 1
    moments = 0 if c["c"] == "none" else (d * d * (2 if c["c"] == "bf16" else 4) + 8 * d + 4)
    by = units * (rows * 4 * d + moments + 4) + units * live * (tail * 4 * d + 4 * d + 20)
    by += units * live * g * 2 * d + units * n * g * (2 * d + 4)
    fl = units * live * g * (4 * (rows + tail) * d + (2 * d * d if moments else 0))
    return {"bytes": int(by), "flops": int(fl)}


# ---------------------------------------------------------- 64-bit results
def _exact_prefix(c, seed):
    s = prepare(dict(c), seed)
    b, n, h, g, d = c["batch"], c["seqs"], c["heads"], c["group"], c["dim"]
    out = torch.zeros(b, n, h * g, d, dtype=F64, device="cuda")
    lse = torch.full((b, n, h * g), -math.inf, dtype=F64, device="cuda")
    for bi in range(b):
        m = int(s["count"][bi])
        for hi in range(h):
            length, heads = int(s["len"][bi, hi]), slice(hi * g, (hi + 1) * g)
            q = s["q"][bi, :m, heads].double() / math.sqrt(d)
            x = torch.einsum("igd,jd->igj", q, s["K"][bi, hi, :length].double())
            z = torch.logsumexp(x, -1)
            o = torch.einsum("igj,jd->igd", torch.softmax(x, -1), s["V"][bi, hi, :length].double())
            if c["c"] != "none":
                C = s["C"][bi, hi]
                C = (C.to(BF16) if c["c"] == "bf16" else C).double()
                C = torch.where((C * EVICTED).abs() < TAU, torch.zeros_like(C), C)
                e = math.log(EVICTED) + q @ s["mu_k"][bi, hi].double()
                both = torch.logaddexp(z, e)
                f = s["mu_v"][bi, hi].double() + q @ C.T
                o = o * torch.exp(z - both)[..., None] + f * torch.exp(e - both)[..., None]
                z = both
            # the tails with their new tokens
            own_len = s["state0"][0].view(b, n, h)[bi, :m, hi]
            keys = torch.cat([s["Kt"].view(b, n, h, -1, d)[bi, :m, hi], s["k"][bi, :m, hi, None]], 1).double()
            vals = torch.cat([s["Vt"].view(b, n, h, -1, d)[bi, :m, hi], s["v"][bi, :m, hi, None]], 1).double()
            y = torch.einsum("igd,ijd->igj", q, keys)
            hide = torch.arange(keys.shape[1] - 1, device="cuda") >= own_len[:, None]
            y[:, :, :-1].masked_fill_(hide[:, None], -math.inf)
            zt = torch.logsumexp(y, -1)
            ot = torch.einsum("igj,ijd->igd", torch.softmax(y, -1), vals)
            both = torch.logaddexp(z, zt)
            out[bi, :m, heads] = o * torch.exp(z - both)[..., None] + ot * torch.exp(zt - both)[..., None]
            lse[bi, :m, heads] = both
    return {"out": out, "lse": lse, "K": None, "V": None, "pos": None, "state": None}


def _exact_select(c, seed):
    s = prepare(dict(c), seed)
    v = c["vocab"]
    p = torch.log_softmax(s["logits"].double(), -1) + s["score"].double()[..., None]
    p = torch.where(s["done"].bool()[..., None], torch.full_like(p, -math.inf), p)
    p[..., END] = torch.where(s["done"].bool(), s["score"].double(), p[..., END])
    return {"parent": None, "token": None, "score": torch.topk(p.reshape(c["batch"], c["beams"] * v), c["out"]).values,
            "done": None}


def _exact_normrope(c, seed):
    s = prepare(dict(c), seed)
    m = c["rot"] // 2
    i = torch.arange(m, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["pairs"] == "neighbours" else (i, i + m)
    angle = s["pos"].double()[s["axis"]].permute(1, 2, 0) * s["inv"].double()
    z = torch.polar(torch.ones_like(angle), angle)[:, :, None]

    def turned(y, z):
        y = y.clone()
        pair = torch.complex(y[..., first], y[..., second]) * z
        y[..., first], y[..., second] = pair.real, pair.imag
        return y

    def normed(x):
        return x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + EPS)

    if not c["grad"]:
        return {"q": turned(normed(s["q"]) * s["wq"].double(), z),
                "k": turned(normed(s["k"]) * s["wk"].double(), z).transpose(1, 2)}
    found = {}
    for name in ("q", "k"):
        x, w = s[name].double(), s["w" + name].double()
        dn = turned(s["dy" + name].double(), z.conj())
        size = torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
        found["d" + name] = w * dn / size - x * (w * dn * x).mean(-1, keepdim=True) / size ** 3
        found["dw" + name] = (dn * x / size).flatten(0, 1).sum(0)
        if w.dim() == 1:
            found["dw" + name] = found["dw" + name].sum(0)
    return {x: found[x] for x in ("dq", "dk", "dwq", "dwk")}


def exact(case, seed):
    if case["kind"] == "reorder":
        return None  # copies
    return {"prefix": _exact_prefix, "select": _exact_select, "normrope": _exact_normrope}[case["kind"]](case, seed)
