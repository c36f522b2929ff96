"""Speculative decoding over a compressed cache, and rotary positions: the
calls whose time is watched, as a user's program makes them.

attend   attention of a tree of drafted tokens over one layer's retained cache
         and moments (mkv_tree_step): queries, keys and values of the nodes in,
         outputs and log-normalisers out.
rope     rotary positions of a layer's queries and keys (mkv_rope), forward
         into the layouts that the next call reads, or the gradient's way back.
build    the nodes' visibility words and positions from their parents
         (mkv_tree_build), once for a drafted tree.
commit   the accepted path's keys and values into every layer's cache
         (mkv_tree_commit), once for a verified tree.

`own` chooses between the framework's kernels and the plain form: elementary
torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

TAU = 1e-6
EVICTED = 1024  # tokens behind the moments of a cache
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _attend(name, batch, heads, group, dim, nodes, rows, c, ragged):
    return {"name": name, "kind": "attend", "batch": batch, "heads": heads, "group": group, "dim": dim, "nodes": nodes,
            "rows": rows, "c": c, "ragged": ragged}


def _rope(name, batch, heads, group, dim, tokens, rot, axes, spread, pairs, inverse):
    return {"name": name, "kind": "rope", "batch": batch, "heads": heads, "group": group, "dim": dim, "tokens": tokens,
            "rot": rot, "axes": axes, "spread": spread, "pairs": pairs, "inverse": inverse}


def listed():
    return [
        # the smallest call: one token, one sequence, a small model's layer with a budget of 128; latency counts
        _attend("attend_d64_b1_n1_r128", 1, 2, 2, 64, 1, 128, "f32", 0),
        # a serving step: a tree of 64 nodes on one Qwen3-4B layer, batch 4, budget 1024, C' in operand form
        _attend("attend_b4_n64_r1024", 4, 8, 4, 128, 64, 1024, "split", 0),
        # a large batch of small trees of unequal sizes over caches of unequal lengths, 16-bit moments
        _attend("attend_b32_n13_r1000", 32, 8, 4, 128, 13, 1000, "bf16", 1),
        # a 128K prompt kept whole (no eviction yet) and a tree of 33 nodes: the most bytes
        _attend("attend_b1_n33_r131072", 1, 8, 4, 128, 33, 131072, "none", 0),
        # wide trees (256 nodes) over the sweep's largest budget: the most products
        _attend("attend_b8_n256_r4096", 8, 8, 4, 128, 256, 4096, "f32", 0),
        # an image+text prompt before compress: one Qwen3-4B layer, batch 4, 32K tokens, time, height and width axes
        _rope("rope_b4_t32768_a3", 4, 8, 4, 128, 32768, 128, 3, "blocks", "halves", 0),
        # the gradient of a prompt of no round length, half of the dims rotated, neighbouring dims paired
        _rope("rope_grad_b2_t8191_r64", 2, 8, 4, 128, 8191, 64, 1, "blocks", "neighbours", 1),
        # the nodes of a drafted tree: a few tokens, axes dealt out in turn
        _rope("rope_b4_t64_a3", 4, 8, 4, 128, 64, 128, 3, "turns", "halves", 0),
        # the topology of one step's trees
        {"name": "build_b4_n64", "kind": "build", "batch": 4, "nodes": 64, "ragged": 0},
        {"name": "build_b64_n251", "kind": "build", "batch": 64, "nodes": 251, "ragged": 1},
        # accepted paths of up to 6 nodes into the caches of all 36 Qwen3-4B layers
        {"name": "commit_l36_b4_n64", "kind": "commit", "batch": 4, "heads": 8, "dim": 128, "layers": 36, "nodes": 64,
         "path": 6, "rows": 300},
        # the same for a large batch, fewer layers, longer paths
        {"name": "commit_l8_b32_n33", "kind": "commit", "batch": 32, "heads": 8, "dim": 128, "layers": 8, "nodes": 33,
         "path": 16, "rows": 200},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _geometry(rng):
    """(heads, group, dim): mostly the 8B-class geometry, else another built one."""
    if rng.random() < 0.5:
        return 8, 4, 128
    return rng.choice([2, 4, 5, 8]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128])


def draw(rng):
    heads, group, dim = _geometry(rng)
    kind = rng.choice(["attend", "attend", "attend", "attend", "rope", "rope", "build", "commit"])
    if kind == "attend":
        batch, nodes = _logint(rng, 1, 64), _logint(rng, 1, 256)
        units = batch * heads
        most = min(131072, 2 ** 20 // units * 128 // dim, 2 ** 28 // (units * nodes * group))
        rows = _logint(rng, 48, max(48, most))
        case = _attend("", batch, heads, group, dim, nodes, rows, rng.choice(["none", "f32", "bf16", "split"]),
                       rng.choice([0, 1]))
    elif kind == "rope":
        batch, rot = _logint(rng, 1, 16), rng.choice([dim, dim, dim // 2, 48])
        tokens = _logint(rng, 1, 4 * 32768 * 40 // (batch * heads * (group + 1)) // 4)
        axes = rng.choice([1, 2, 3, 3])
        case = _rope("", batch, heads, group, dim, tokens, rot, axes, rng.choice(["blocks", "turns"]),
                     rng.choice(["halves", "neighbours"]), rng.choice([0, 0, 1]))
    elif kind == "build":
        case = {"kind": "build", "batch": _logint(rng, 1, 128), "nodes": _logint(rng, 1, 256),
                "ragged": rng.choice([0, 1])}
    else:
        batch, layers = _logint(rng, 1, 32), rng.randint(1, 40)
        nodes = _logint(rng, 4, 256)
        case = {"kind": "commit", "batch": batch, "heads": heads, "dim": dim, "layers": layers, "nodes": nodes,
                "path": rng.randint(1, min(16, nodes)),
                "rows": _logint(rng, 20, max(20, 150000 // (batch * heads * layers)))}
    case.pop("name", None)
    return case


# ------------------------------------------------------------------ inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 17)
    return gen


def _parents(c, gen):
    """Random trees: node 0 is a root, node i hangs below an earlier one (or is another root)."""
    b, n = c["batch"], c["nodes"]
    u = torch.rand(b, n, generator=gen, device="cuda")
    i = torch.arange(n, device="cuda", dtype=F32)
    parents = (torch.floor(u * (i + 1)) - 1).to(I32)
    count = torch.full((b,), n, dtype=I32, device="cuda")
    if c["ragged"]:
        count = torch.randint(n // 2, n + 1, (b,), generator=gen, device="cuda", dtype=I32)
    return torch.minimum(parents, (i - 1).to(I32)), count


def _prepare_attend(c, seed):
    gen = _generator(seed)
    b, h, g, d, n, rows = c["batch"], c["heads"], c["group"], c["dim"], c["nodes"], c["rows"]
    units, cap = b * h, rows + 16
    lo, hi = math.log(0.5), math.log(4.0)
    scale = torch.exp(lo + (hi - lo) * torch.rand(units, 1, d, generator=gen, device="cuda"))

    def keys(m):
        return (torch.randn(units, m, d, generator=gen, device="cuda") * scale).to(BF16)

    def values(m):
        return torch.randn(units, m, d, generator=gen, device="cuda").to(BF16)

    K, V = keys(cap), values(cap)
    s = {"case": c, "K": K.view(b, h, cap, d), "V": V.view(b, h, cap, d)}
    s["len"] = torch.full((b, h), rows, dtype=I32, device="cuda")
    if c["ragged"]:
        s["len"] = torch.randint(rows // 2, rows + 1, (b, h), generator=gen, device="cuda", dtype=I32)
    s["pos"] = torch.arange(cap, dtype=I32, device="cuda").expand(b, h, cap).contiguous()
    s["seen"] = s["len"] + EVICTED
    if c["c"] != "none":
        ke, ve = keys(EVICTED).float(), values(EVICTED).float()
        mk, mv = ke.mean(1), ve.mean(1)
        cov = torch.bmm((ve - mv[:, None]).transpose(1, 2), ke - mk[:, None]) / EVICTED
        s["n"] = torch.full((b, h), EVICTED, dtype=I32, device="cuda")
        s["mu_k"], s["mu_v"], s["C"] = mk.view(b, h, d), mv.view(b, h, d), cov.view(b, h, d, d).contiguous()
    # a node's query lies near the sum of three retained keys, as a decode step's does
    pick = torch.randint(0, rows, (units, n * g, 3), generator=gen, device="cuda")
    q = K[torch.arange(units, device="cuda")[:, None, None], pick].float().sum(2)
    q = math.sqrt(d) * q / torch.linalg.norm(q, dim=-1, keepdim=True)
    q = q + 0.3 * torch.randn(q.shape, generator=gen, device="cuda")
    q = q.view(b, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, h * g, d)
    # queries, keys and values of a node lie behind one another, as a fused projection leaves them
    qkv = torch.empty(b, n, h * (g + 2), d, dtype=BF16, device="cuda")
    qkv[:, :, :h * g] = q.to(BF16)
    qkv[:, :, h * g:h * (g + 1)] = keys(n).view(b, h, n, d).transpose(1, 2)
    qkv[:, :, h * (g + 1):] = values(n).view(b, h, n, d).transpose(1, 2)
    s["q"], s["k"], s["v"] = qkv[:, :, :h * g], qkv[:, :, h * g:h * (g + 1)], qkv[:, :, h * (g + 1):]
    s["parents"], s["count"] = _parents(c, gen)
    s["mask"] = _plain_build(s["parents"], s["count"], torch.zeros_like(s["count"]))[0]
    if own:
        s["call"] = _attend_call(s)
    return s


def _attend_call(s):
    """What a program keeps beside a layer's cache: the binding's views of it, the moments in the form that is
    read, the outputs and the workspace."""
    from paper_2606_01563_gb300 import mkv
    c = s["case"]
    b, h, g, d, n = c["batch"], c["heads"], c["group"], c["dim"], c["nodes"]
    geom = mkv.geom(b, h, g, d)
    cache = mkv.Cache(s["K"], s["V"], s["pos"], s["len"], s["seen"])
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
    return {"g": geom, "cache": cache, "mom": mom, "p": p, "held": (c16, split),
            "tree": mkv.Tree(s["mask"], s["count"]),
            "out": torch.empty(b, n, h * g, d, dtype=BF16, device="cuda"),
            "lse": torch.empty(b, n, h * g, dtype=F32, device="cuda"),
            "ws": mkv.alloc_workspace(mkv.mkv_tree_workspace_size(geom, n, cache.capacity))}


def _positions(c, gen):
    """[axes, b, tokens]: text, an image whose patches share a time and count rows and columns, text again.  Each
    sequence starts at an offset of its own (what it has seen)."""
    b, t = c["batch"], c["tokens"]
    start = torch.randint(0, 4096, (b, 1), generator=gen, device="cuda")
    i = torch.arange(t, device="cuda")
    first, patches = t // 4, t // 2
    wide = max(1, int(math.sqrt(patches)))
    at = (i - first).clamp(0, max(0, patches - 1))
    image = (i >= first) & (i < first + patches)
    after = first + wide + (i - first - patches)
    text = torch.where(i < first, i, after)
    axes = [torch.where(image, x, text) for x in (torch.full_like(i, first), first + at // wide, first + at % wide)]
    pos = torch.stack([axes[a] if c["axes"] > 1 else i for a in range(c["axes"])])
    return (pos[:, None] + start).to(I32)


def _freqs(c):
    """Inverse frequencies (fp32) and the axis of each: in blocks of 1/4, 3/8 and 3/8 of them, or in turn."""
    m, axes = c["rot"] // 2, c["axes"]
    inv = [float(x) for x in torch.tensor([1e6 ** (-i / m) for i in range(m)], dtype=F32)]
    if c["spread"] == "turns":
        return inv, [i % axes for i in range(m)]
    ends = {1: [m], 2: [m // 2, m], 3: [m // 4, m // 4 + 3 * m // 8, m]}[axes]
    return inv, [sum(i >= e for e in ends) for i in range(m)]


def _prepare_rope(c, seed):
    gen = _generator(seed)
    b, h, g, d, t = c["batch"], c["heads"], c["group"], c["dim"], c["tokens"]

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=BF16)

    inv, axis = _freqs(c)
    s = {"case": c, "pos": _positions(c, gen), "inv": torch.tensor(inv, dtype=F32, device="cuda"),
         "axis": torch.tensor(axis, device="cuda")}
    # forward: projections of a token lie behind one another, keys go to the layout that compress reads;
    # backward: the gradients come in those layouts and go back
    if c["inverse"]:
        s["q"], s["k"] = rand(b, t, h * g, d), rand(b, h, t, d).transpose(1, 2)
    else:
        qk = rand(b, t, h * (g + 1), d)
        s["q"], s["k"] = qk[:, :, :h * g], qk[:, :, h * g:]
    if own:
        from paper_2606_01563_gb300 import mkv
        s["p"] = mkv.rope_params(inv, axis, c["pairs"] == "neighbours")
        if c["inverse"]:
            dqk = torch.empty(b, t, h * (g + 1), d, dtype=BF16, device="cuda")
            s["q_out"], s["k_out"] = dqk[:, :, :h * g], dqk[:, :, h * g:]
        else:
            s["q_out"] = torch.empty(b, t, h * g, d, dtype=BF16, device="cuda")
            s["k_out"] = torch.empty(b, h, t, d, dtype=BF16, device="cuda").transpose(1, 2)
    return s


def _prepare_build(c, seed):
    gen = _generator(seed)
    parents, count = _parents(c, gen)
    s = {"case": c, "parents": parents, "count": count}
    s["base"] = torch.randint(0, 100000, (c["batch"],), generator=gen, device="cuda", dtype=I32)
    if own:
        from paper_2606_01563_gb300 import mkv
        s["mask"] = torch.empty(c["batch"], c["nodes"], -(-c["nodes"] // 32), dtype=I32, device="cuda")
        s["pos"] = torch.empty(c["batch"], c["nodes"], dtype=I32, device="cuda")
        s["ws"] = mkv.alloc_workspace(256)
    return s


def _prepare_commit(c, seed):
    gen = _generator(seed)
    b, h, d, layers, n, most = c["batch"], c["heads"], c["dim"], c["layers"], c["nodes"], c["path"]
    cap = c["rows"] + most

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=BF16)

    s = {"case": c, "K": rand(layers, b, h, cap, d), "V": rand(layers, b, h, cap, d),
         "pos": torch.arange(cap, dtype=I32, device="cuda").expand(layers, b, h, cap).contiguous(),
         "k": rand(layers, b, n, h, d), "v": rand(layers, b, n, h, d)}
    s["len0"] = torch.randint(c["rows"] // 2, c["rows"] + 1, (layers, b, h), generator=gen, device="cuda", dtype=I32)
    s["state0"] = torch.stack([s["len0"], s["len0"] + EVICTED])
    s["state"] = s["state0"].clone()  # len and seen of every layer
    s["path"] = torch.argsort(torch.rand(b, n, generator=gen, device="cuda"))[:, :most].sort(1).values.to(I32)
    s["taken"] = torch.randint(0, most + 1, (b,), generator=gen, device="cuda", dtype=I32)
    if own:
        from paper_2606_01563_gb300 import mkv
        s["g"] = mkv.geom(b, h, 1, d)
        s["layers"] = mkv.tree_layers([(mkv.Cache(s["K"][l], s["V"][l], s["pos"][l], s["state"][0, l], s["state"][1, l]),
                                        s["k"][l], s["v"][l]) for l in range(layers)])
        s["ws"] = mkv.alloc_workspace(256)
    return s


def prepare(case, seed):
    return {"attend": _prepare_attend, "rope": _prepare_rope, "build": _prepare_build,
            "commit": _prepare_commit}[case["kind"]](case, seed)


# --------------------------------------------------------------------- run
def _visible(mask, count):
    """[b, n, n] truth values: node i sees node a (both in use)."""
    n = mask.shape[1]
    a = torch.arange(n, device="cuda")
    live = a < count[:, None]
    bits = (mask.long()[:, :, a // 32] >> (a % 32)) & 1
    return (bits != 0) & live[:, None, :] & live[:, :, None], live


def _plain_build(parents, count, base):
    """Ancestors by squaring the one-step relation; bits packed into 32-bit words."""
    b, n = parents.shape
    a = torch.arange(n, device="cuda")
    live = a < count[:, None]
    reach = ((parents[:, :, None] == a) | (a[:, None] == a)) & live[:, :, None] & live[:, None, :]
    reach = reach.float()
    steps = 1
    while steps < n:
        reach = (torch.bmm(reach, reach) > 0).float()
        steps *= 2
    seen = torch.nn.functional.pad(reach, (0, -n % 32)).view(b, n, -1, 32).long()
    words = (seen << torch.arange(32, device="cuda")).sum(-1)
    depth = (reach.sum(-1) - 1).clamp(min=0).to(I32)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(I32), base[:, None] + depth


def _plain_attend(s):
    c = s["case"]
    b, h, g, d, n = c["batch"], c["heads"], c["group"], c["dim"], c["nodes"]
    q = s["q"].float().view(b, n, h, g, d).permute(0, 2, 1, 3, 4).reshape(b, h, n * g, d) * d ** -0.5
    vis, live = _visible(s["mask"], s["count"])
    vis = vis.repeat_interleave(g, 1)[:, None]                    # [b, 1, n g, n]
    dead = ~live.repeat_interleave(g, 1)[:, None, :, None]        # [b, 1, n g, 1]
    x = q @ s["K"].float().transpose(2, 3)
    cap = x.shape[-1]
    x = x.masked_fill_((torch.arange(cap, device="cuda") >= s["len"][..., None, None]) | dead, -math.inf)
    y = (q @ s["k"].float().permute(0, 2, 3, 1)).masked_fill_(~vis, -math.inf)
    top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True))
    if c["c"] != "none":
        e = torch.log(s["n"].float())[..., None, None] + q @ s["mu_k"][..., None]
        e = e.masked_fill_(dead, -math.inf)
        top = torch.maximum(top, e)
    ref = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    x, y = (x - ref).exp_(), (y - ref).exp_()
    total = x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
    out = x @ s["V"].float() + y @ s["v"].float().transpose(1, 2)
    if c["c"] != "none":
        C = s["C"].to(BF16).float() if c["c"] == "bf16" else s["C"]
        C = torch.where((C * s["n"][..., None, None]).abs() < TAU, torch.zeros_like(C), C)
        w = (e - ref).exp_()
        total = total + w
        out = out + w * (s["mu_v"][:, :, None] + q @ C.transpose(2, 3))
    some = total > 0
    out = torch.where(some, out / torch.where(some, total, torch.ones_like(total)), torch.zeros_like(out))
    lse = torch.where(some, ref + torch.log(total), torch.full_like(total, -math.inf))[..., 0]
    return {"out": out.view(b, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, h * g, d).to(BF16),
            "lse": lse.view(b, h, n, g).permute(0, 2, 1, 3).reshape(b, n, h * g)}


def _rotate(x, cos, sin, rot, neighbours):
    if neighbours:
        a, c = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - c * sin, a * sin + c * cos], -1).flatten(-2)
    else:
        a, c = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - c * sin, a * sin + c * cos], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rope(s):
    c = s["case"]
    angle = s["pos"].float()[s["axis"]].permute(1, 2, 0) * s["inv"]  # [b, tokens, rot / 2]
    cos, sin = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    if c["inverse"]:
        sin = -sin
    q, k = (_rotate(x.float(), cos, sin, c["rot"], c["pairs"] == "neighbours").to(BF16) for x in (s["q"], s["k"]))
    return {"q": q, "k": k if c["inverse"] else k.transpose(1, 2).contiguous()}


def _plain_commit(s):
    c = s["case"]
    s["state"].copy_(s["state0"])
    length, seen = s["state"][0], s["state"][1]
    layers, b, h, d, most = c["layers"], c["batch"], c["heads"], c["dim"], c["path"]
    j = torch.arange(most, device="cuda")
    take = (j < s["taken"][:, None])[None, :, None].expand(layers, b, h, most)
    at = length[..., None].long() + j
    from_ = s["path"].long()[None, :, None, :, None].expand(layers, b, h, most, d)
    row = at[..., None].expand(-1, -1, -1, -1, d)
    s["K"].scatter_(3, row, torch.where(take[..., None], s["k"].transpose(2, 3).gather(3, from_), s["K"].gather(3, row)))
    s["V"].scatter_(3, row, torch.where(take[..., None], s["v"].transpose(2, 3).gather(3, from_), s["V"].gather(3, row)))
    s["pos"].scatter_(3, at, torch.where(take, (seen[..., None] + j).to(I32), s["pos"].gather(3, at)))
    s["state"] += s["taken"][None, None, :, None]


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if kind == "commit":
        if own:
            from paper_2606_01563_gb300 import mkv
            s["state"].copy_(s["state0"])  # the caches as the step before left them
            mkv.mkv_tree_commit(s["g"], s["layers"], s["path"], s["taken"], s["ws"])
        else:
            _plain_commit(s)
        return {n: s[n] for n in ("K", "V", "pos", "state")}
    if not own:
        if kind == "attend":
            return _plain_attend(s)
        if kind == "rope":
            return _plain_rope(s)
        mask, pos = _plain_build(s["parents"], s["count"], s["base"])
        return {"mask": mask, "pos": pos}
    from paper_2606_01563_gb300 import mkv
    if kind == "attend":
        a = s["call"]
        mkv.mkv_tree_step(a["g"], a["tree"], s["q"], s["k"], s["v"], a["cache"], a["mom"], a["p"], a["out"], a["lse"],
                          a["ws"])
        return {"out": a["out"], "lse": a["lse"]}
    if kind == "rope":
        mkv.mkv_rope(s["pos"], s["p"], [(s["q"], s["q_out"]), (s["k"], s["k_out"])], inverse=bool(c["inverse"]))
        return {"q": s["q_out"], "k": s["k_out"] if c["inverse"] else s["k_out"].transpose(1, 2)}
    mkv.mkv_tree_build(s["parents"], s["mask"], s["pos"], s["ws"], count=s["count"], base=s["base"])
    return {"mask": s["mask"], "pos": s["pos"]}


# -------------------------------------------------------------------- work
def work(case):
    c = case
    b, n = c["batch"], c.get("nodes", 0)
    if c["kind"] == "build":
        return {"bytes": b * n * 4 * (2 + -(-n // 32)) + 8 * b, "flops": 0}
    h, d = c["heads"], c["dim"]
    if c["kind"] == "commit":
        rows = c["layers"] * b * h * c["path"] / 2  # half of the longest path, on average
        return {"bytes": rows * (8 * d + 4) + c["layers"] * b * h * 16 + 4 * b * (c["path"] + 1), "flops": 0}
    g = c["group"]
    if c["kind"] == "rope":
        values = b * c["tokens"] * h * (g + 1) * d
        return {"bytes": 4 * values + 4 * c["axes"] * b * c["tokens"], "flops": 3 * values * c["rot"] // d}
    share = 0.75 if c["ragged"] else 1
    rows, live, units = c["rows"] * share, n * share, b * h
    moments = 0 if c["c"] == "none" else (d * d * (2 if c["c"] == "bf16" else 4) + 8 * d + 4)
    by = units * (rows * 4 * d + moments + 4) + b * live * h * 2 * d * (g + 2) + b * live * 4 * -(-n // 32)
    by += b * n * h * g * (2 * d + 4)
    fl = units * live * g * (4 * (rows + live) * d + (2 * d * d if moments else 0))
    return {"bytes": int(by), "flops": int(fl)}


# ---------------------------------------------------------- 64-bit results
def _ancestors(parents, count):
    """Per sequence, a list of each node's visible nodes (itself and up), by walking up on the host."""
    out = []
    for row, m in zip(parents.tolist(), count.tolist()):
        sees = []
        for i, p in enumerate(row):
            sees.append([] if i >= m else [i] + (sees[p] if p >= 0 else []))
        out.append(sees)
    return out


def _exact_attend(c, seed):
    s = prepare(dict(c), seed)
    b, h, g, d, n = c["batch"], c["heads"], c["group"], c["dim"], c["nodes"]
    sees = _ancestors(s["parents"], s["count"])
    out = torch.zeros(b, n, h * g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, n, h * g), -math.inf, dtype=torch.float64, device="cuda")
    for bi in range(b):
        m = int(s["count"][bi])
        if m == 0:
            continue
        hide = torch.ones(m, m, dtype=torch.bool)
        for i in range(m):
            hide[i, sees[bi][i]] = False
        hide = hide.cuda()
        for hi in range(h):
            length = int(s["len"][bi, hi])
            q = s["q"][bi, :m, hi * g:(hi + 1) * g].double() / math.sqrt(d)
            keys = torch.cat([s["K"][bi, hi, :length], s["k"][bi, :m, hi]]).double()
            vals = torch.cat([s["V"][bi, hi, :length], s["v"][bi, :m, hi]]).double()
            x = torch.einsum("igd,jd->igj", q, keys)
            x[:, :, length:].masked_fill_(hide[:, None, :], -math.inf)
            z = torch.logsumexp(x, -1)
            o = torch.einsum("igj,jd->igd", torch.softmax(x, -1), vals)
            if c["c"] != "none":
                C = s["C"][bi, hi]
                C = (C.to(BF16) if c["c"] == "bf16" else C).double()
                C = torch.where((C * EVICTED).abs() < TAU, torch.zeros_like(C), C)
                e = math.log(EVICTED) + q @ s["mu_k"][bi, hi].double()
                f = s["mu_v"][bi, hi].double() + q @ C.T
                both = torch.logaddexp(z, e)
                o = o * torch.exp(z - both)[..., None] + f * torch.exp(e - both)[..., None]
                z = both
            out[bi, :m, hi * g:(hi + 1) * g], lse[bi, :m, hi * g:(hi + 1) * g] = o, z
    return {"out": out, "lse": lse}


def _exact_rope(c, seed):
    s = prepare(dict(c), seed)
    m, turn = c["rot"] // 2, -1.0 if c["inverse"] else 1.0
    i = torch.arange(m, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["pairs"] == "neighbours" else (i, i + m)
    angle = turn * s["pos"].double()[s["axis"]].permute(1, 2, 0) * s["inv"].double()
    z = torch.polar(torch.ones_like(angle), angle)[:, :, None]

    def rotated(x):
        y = x.double()
        pair = torch.complex(y[..., first], y[..., second]) * z
        y[..., first], y[..., second] = pair.real, pair.imag
        return y

    k = rotated(s["k"])
    return {"q": rotated(s["q"]), "k": k if c["inverse"] else k.transpose(1, 2)}


def exact(case, seed):
    if case["kind"] == "attend":
        return _exact_attend(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(case, seed)
    return None  # whole numbers and copies
