"""Performance cases of the attention operators: rotary positions of several axes, norms of queries and keys with the
rotation in the same pass, and dot-product attention over a graph's edges.

`run` computes each operator in a plain form, elementary torch operations in 32 bits (angles in 64) rounded once at the
end, or, with `own` true, through this package.  The graphs are seeded stand-ins of the workloads that this
repository's generator and benchmark use: a citation-like power-law graph, a constant in-degree graph (nearest
neighbours of points), a sampled neighbourhood block, an R-MAT graph with the node and edge counts of the large
workload, and one node with a long neighbourhood.  Edge lists come "sorted" by (destination, source) or in "arrival"
order, a random one.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
BASE = 10000.0

# the large R-MAT workload
LARGE_N, LARGE_E = 232965, 114600000


def listed():
    return [
        # rotation of one new node's queries in a serving loop: latency is all there is
        {"name": "rotary_one_node", "op": "rotary", "dir": "fwd", "rows": 1, "heads": 8, "feat": 64,
         "pairs": "12,10,10", "interleaved": False, "pos": "f32", "dtype": "bf16"},
        # patches of a batch of images (height, width), rotation and its gradient
        {"name": "rotary_image_step", "op": "rotary", "dir": "step", "rows": 50176, "heads": 8, "feat": 32,
         "pairs": "8,8", "interleaved": True, "pos": "i32", "dtype": "f32"},
        # cells of a long video (time, height, width), wide heads of which a part turns
        {"name": "rotary_video", "op": "rotary", "dir": "fwd", "rows": 262144, "heads": 16, "feat": 128,
         "pairs": "16,20,20", "interleaved": False, "pos": "i32", "dtype": "bf16"},
        # queries and keys of one new node
        {"name": "norm_rotary_one_node", "op": "norm_rotary", "dir": "fwd", "rows": 1, "heads": 8, "kv_heads": 2,
         "feat": 64, "pairs": "12,10,10", "interleaved": False, "pos": "f32", "per_head": False, "dtype": "bf16"},
        # an odd width and odd counts, a training step in bf16
        {"name": "norm_rotary_odd_step", "op": "norm_rotary", "dir": "step", "rows": 20011, "heads": 6, "kv_heads": 3,
         "feat": 47, "pairs": "7,7,8", "interleaved": True, "pos": "f32", "per_head": True, "dtype": "bf16"},
        # every point of a large cloud, a training step
        {"name": "norm_rotary_points_step", "op": "norm_rotary", "dir": "step", "rows": 262144, "heads": 8,
         "kv_heads": 8, "feat": 32, "pairs": "6,5,5", "interleaved": False, "pos": "f32", "per_head": False,
         "dtype": "f32"},
        # attention of one new node over a long neighbourhood, inference
        {"name": "dot_one_node", "op": "dot", "dir": "fwd", "graph": "one", "order": "sorted", "n_src": 100000,
         "n_dst": 1, "e": 100000, "heads": 8, "kv_heads": 2, "feat": 64, "bias": "none", "dtype": "bf16"},
        # a training step on a citation graph as it came from its file
        {"name": "dot_citation_step", "op": "dot", "dir": "step", "graph": "chunglu", "order": "arrival",
         "n_src": 20000, "n_dst": 20000, "e": 109170, "heads": 8, "kv_heads": 8, "feat": 8, "bias": "none",
         "dtype": "f32"},
        # one layer of a mini-batch with masked edges and an odd width, inference
        {"name": "dot_block_masked", "op": "dot", "dir": "fwd", "graph": "block", "order": "sorted", "n_src": 90000,
         "n_dst": 10000, "e": 100000, "heads": 6, "kv_heads": 3, "feat": 47, "bias": "mask", "dtype": "f32"},
        # nearest neighbours of a point cloud, edge biases learnt, shared key heads, a training step in bf16
        {"name": "dot_points_step", "op": "dot", "dir": "step", "graph": "knn", "order": "sorted", "n_src": 262144,
         "n_dst": 262144, "e": 8388608, "heads": 8, "kv_heads": 2, "feat": 32, "bias": "heads", "dtype": "bf16"},
        # a training step on a skewed graph in arrival order
        {"name": "dot_skewed_step", "op": "dot", "dir": "step", "graph": "rmat", "order": "arrival",
         "n_src": LARGE_N, "n_dst": LARGE_N, "e": LARGE_E // 8, "heads": 8, "kv_heads": 8, "feat": 16, "bias": "none",
         "dtype": "f32"},
        # the large graph, inference in bf16, the largest case
        {"name": "dot_large", "op": "dot", "dir": "fwd", "graph": "rmat", "order": "sorted", "n_src": LARGE_N,
         "n_dst": LARGE_N, "e": LARGE_E, "heads": 8, "kv_heads": 8, "feat": 16, "bias": "none", "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_pairs(rng, feat):
    """Pairs of columns turned by each of one to four axes (part of the columns, now and then)."""
    most = feat // 2
    axes = rng.randint(1, min(4, most))
    turned = most if rng.random() < 0.6 else rng.randint(axes, most)
    cuts = sorted(rng.sample(range(1, turned), axes - 1)) if axes > 1 else []
    ends = cuts + [turned]
    return ",".join(str(b - a) for a, b in zip([0] + cuts, ends))


def draw(rng):
    """Another case: any operator, head layout, width (odd ones among them), type and graph family."""
    op = rng.choice(["rotary", "norm_rotary", "norm_rotary", "dot", "dot", "dot"])
    dtype = rng.choice(["f32", "bf16"])
    way = rng.choice(["fwd", "step"])
    heads = rng.choice([1, 2, 3, 4, 6, 8, 8, 16])
    feat = rng.choice([8, 16, 32, 64, 128, rng.randint(3, 160), rng.randint(3, 160)])
    kv_heads = rng.choice([h for h in range(1, heads + 1) if heads % h == 0] + [heads] * 2)
    if op != "dot":
        rows = _log_int(rng, 1, 262144)
        while rows * heads * feat > 262144 * 2048 // 2:
            rows //= 2
        case = {"op": op, "dir": way, "rows": rows, "heads": heads, "feat": feat, "pairs": _draw_pairs(rng, feat),
                "interleaved": rng.random() < 0.5, "pos": rng.choice(["f32", "i32"]), "dtype": dtype}
        if op == "norm_rotary":
            case["kv_heads"] = kv_heads
            case["per_head"] = rng.random() < 0.3
        return case
    order = rng.choice(["sorted", "arrival"])
    graph = rng.choice(["one", "chunglu", "block", "knn", "rmat", "rmat"])
    if graph == "one":
        n_src, n_dst = _log_int(rng, 1, 1000000), 1
        e, way = n_src, "fwd"
    elif graph == "chunglu":
        n_src = n_dst = _log_int(rng, 3000, 200000)
        e = n_dst + int(n_dst * rng.uniform(2.0, 9.0))
    elif graph == "block":
        n_dst = _log_int(rng, 300, 200000)
        fan = rng.randint(3, 25)
        n_src, e = n_dst * (fan - 1), n_dst * fan
    elif graph == "knn":
        n_src = n_dst = _log_int(rng, 10000, 300000)
        e = n_dst * rng.choice([8, 15, 16, 20, 32])
    else:
        n_src = n_dst = _log_int(rng, 50000, 1000000)
        e = min(int(n_dst * rng.uniform(10.0, 100.0)), LARGE_E // 4)
    # no drawn case costs more than the largest listed one
    most = LARGE_E * 128 // (16 if way == "step" else 4)
    while e * heads * feat > most:
        if feat > 16:
            feat //= 2
        else:
            heads //= 2
            kv_heads = max(1, min(kv_heads, heads))
            while heads % kv_heads:
                kv_heads -= 1
    return {"op": op, "dir": way, "graph": graph, "order": order, "n_src": n_src, "n_dst": n_dst, "e": e,
            "heads": heads, "kv_heads": kv_heads, "feat": feat, "bias": rng.choice(["none", "none", "heads", "mask"]),
            "dtype": dtype}


# ---------------------------------------------------------------------------
# inputs


def _exactly(keys, e, gen):
    """e of the sorted distinct keys, in order."""
    drop = torch.randperm(keys.numel(), device="cuda", generator=gen)[: keys.numel() - e]
    keep = torch.ones(keys.numel(), dtype=torch.bool, device="cuda")
    keep[drop] = False
    return keys[keep]


def _rmat_keys(n, e, gen, abc=(0.57, 0.19, 0.19)):
    """Sorted distinct keys dst * n + src of an R-MAT graph, ids at random."""
    a, b, c = abc
    levels = max(1, (n - 1).bit_length())
    relabel = torch.randperm(n, device="cuda", generator=gen)
    keys = torch.empty(0, dtype=torch.int64, device="cuda")
    want = e
    while keys.numel() < e:
        m = int(1.3 * want) + 4096
        src = torch.zeros(m, dtype=torch.int32, device="cuda")
        dst = torch.zeros(m, dtype=torch.int32, device="cuda")
        for _ in range(levels):
            r = torch.rand(m, device="cuda", generator=gen)
            src = 2 * src + (r >= a + b)
            dst = 2 * dst + (((r >= a) & (r < a + b)) | (r >= a + b + c))
        ok = (src < n) & (dst < n)
        new = relabel[dst[ok].long()] * n + relabel[src[ok].long()]
        keys = torch.unique(torch.cat([keys, new]))
        want = max(2 * (e - keys.numel()), 4096)
    return _exactly(keys, e, gen)


def _chunglu_keys(n, e, gen):
    """Sorted keys dst * n + src: power-law endpoints (exponent 2.5), no duplicates, one self-loop per node."""
    w = torch.arange(1, n + 1, device="cuda", dtype=torch.float64) ** (-1.0 / 1.5)
    cum = torch.cumsum(w, 0)
    relabel = torch.randperm(n, device="cuda", generator=gen)
    keys = torch.empty(0, dtype=torch.int64, device="cuda")
    while keys.numel() < e - n:
        u = torch.rand((2, 2 * (e - n)), device="cuda", dtype=torch.float64, generator=gen) * cum[-1]
        ends = relabel[torch.searchsorted(cum, u).clamp_(max=n - 1)]
        new = (ends[0] * n + ends[1])[ends[0] != ends[1]]
        keys = torch.unique(torch.cat([keys, new]))
    loops = torch.arange(n, device="cuda") * (n + 1)
    return torch.sort(torch.cat([_exactly(keys, e - n, gen), loops]))[0]


def _edges(case, gen):
    """(src, dst) int32 on the GPU, in the case's order."""
    kind, ns, nd, e = case["graph"], case["n_src"], case["n_dst"], case["e"]
    if kind == "rmat":
        keys = _rmat_keys(ns, e, gen)
    elif kind == "chunglu":
        keys = _chunglu_keys(ns, e, gen)
    elif kind == "one":
        keys = torch.arange(e, device="cuda")
    else:  # block and knn: e / nd random sources for each destination
        src = torch.randint(0, ns, (e,), device="cuda", generator=gen)
        keys = torch.sort(torch.arange(nd, device="cuda").repeat_interleave(e // nd) * ns + src)[0]
    if case["order"] == "arrival":
        keys = keys[torch.randperm(e, device="cuda", generator=gen)]
    return (keys % ns).int(), (keys // ns).int()


def _pairs(case):
    return [int(p) for p in case["pairs"].split(",")]


def _positions(case, gen):
    """Frames and cells of a grid, or coordinates of points."""
    n, axes = case["rows"], len(_pairs(case))
    if case["pos"] == "f32":
        return torch.randn((n, axes), device="cuda", generator=gen) * 20.0
    span = torch.tensor([100000, 1024, 1024, 64][:axes], device="cuda")
    return (torch.rand((n, axes), device="cuda", generator=gen, dtype=torch.float64) * span).int()


def _frequencies(pairs):
    """For each axis, a geometric row from 1 down to about 1 / BASE."""
    return torch.cat([BASE ** (-torch.arange(p, dtype=torch.float64) / p) for p in pairs]).float().cuda()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt, H, F, op = DTYPES[case["dtype"]], case["heads"], case["feat"], case["op"]
    step = case["dir"] == "step"
    t = {}

    def normal(*shape, dtype=dt):
        return torch.randn(shape, device="cuda", generator=gen).to(dtype)

    if op == "dot":
        K, e = case["kv_heads"], case["e"]
        t["src"], t["dst"] = _edges(case, gen)
        # (queries and keys of unit variance, as the norms leave them)
        t["q"], t["k"], t["v"] = normal(case["n_dst"], H, F), normal(case["n_src"], K, F), normal(case["n_src"], K, F)
        if case["bias"] != "none":
            b = torch.randn((e, H, 1), device="cuda", generator=gen)
            if case["bias"] == "mask":  # a fifth of the edges masked, and all of some destinations'
                gone = torch.rand(e, device="cuda", generator=gen) < 0.2
                gone |= (t["dst"] % 64) == 5
                b.masked_fill_(gone.view(e, 1, 1), -math.inf)
            t["bias"] = b.to(dt)
        if step:
            t["dout"] = normal(case["n_dst"], H, F)
        return t
    t["pos"] = _positions(case, gen)
    t["freq"] = _frequencies(_pairs(case))
    n = case["rows"]
    t["q"] = normal(n, H, F)
    if step:
        t["gq"] = normal(n, H, F)
    if op == "norm_rotary":
        K = case["kv_heads"]
        t["k"] = normal(n, K, F)
        t["wq"] = (1.0 + 0.2 * torch.randn((1, H if case["per_head"] else 1, F), device="cuda", generator=gen)).to(dt)
        t["wk"] = (1.0 + 0.2 * torch.randn((1, K if case["per_head"] else 1, F), device="cuda", generator=gen)).to(dt)
        if step:
            t["gk"] = normal(n, K, F)
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    state = {"case": case, "t": t}
    if own:
        from paper_1909_01315_amd import gnnk
        if case["op"] == "dot":
            state["g"] = gnnk.Graph.from_coo(t.pop("src"), t.pop("dst"), case["n_src"], case["n_dst"])
        else:
            state["rot"] = gnnk.Rotary(t["freq"], _pairs(case), interleaved=case["interleaved"])
    elif case["op"] == "dot":
        t["src"], t["dst"] = t["src"].long(), t["dst"].long()
    return state


# ---------------------------------------------------------------------------
# the plain form


def _angles(case, t):
    """cos and sin of every row's pairs, (rows, 1, pairs) in 32 bits (angles in 64)."""
    axis = torch.repeat_interleave(torch.arange(len(_pairs(case))), torch.tensor(_pairs(case))).cuda()
    theta = t["pos"].double()[:, axis] * t["freq"].double()
    return torch.cos(theta).float().unsqueeze(1), torch.sin(theta).float().unsqueeze(1)


def _turn(x, cos, sin, interleaved):
    """Columns (2i, 2i + 1), or (i, i + P), of the first 2P turned by the angles; the others as they are."""
    P = cos.shape[2]
    head, rest = x[..., : 2 * P], x[..., 2 * P:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = head[..., :P], head[..., P:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([y, rest], dim=-1)


def _plain_rotary(case, t):
    cos, sin = _angles(case, t)
    il, dt = case["interleaved"], t["q"].dtype
    got = {"out": _turn(t["q"].float(), cos, sin, il).to(dt)}
    if case["dir"] == "step":
        got["dx"] = _turn(t["gq"].float(), cos, -sin, il).to(dt)
    return got


def _plain_norm(x, w, g, cos, sin, il):
    dt, x, w = x.dtype, x.float(), w.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    out = _turn(x * r * w, cos, sin, il).to(dt)
    if g is None:
        return (out,)
    g = _turn(g.float(), cos, -sin, il)
    dw = (g * x * r).sum((0, 1) if w.shape[1] == 1 else 0).view(w.shape)
    gw = g * w
    dx = r * (gw - x * (r * r * (gw * x).mean(-1, keepdim=True)))
    return out, dx.to(dt), dw.to(dt)


def _plain_norm_rotary(case, t):
    cos, sin = _angles(case, t)
    got = {}
    for s in ("q", "k"):
        for name, x in zip((s, "d" + s, "dw" + s),
                           _plain_norm(t[s], t["w" + s], t.get("g" + s), cos, sin, case["interleaved"])):
            got[name] = x
    return got


def _plain_dot(case, t):
    """Softmax over the in-edges of each destination, some heads at a time where edges times columns are many."""
    src, dst, q, k, v = t["src"], t["dst"], t["q"], t["k"], t["v"]
    H, F, K, e, nd, ns = case["heads"], case["feat"], case["kv_heads"], case["e"], case["n_dst"], case["n_src"]
    rep, scale, dt = H // K, 1.0 / math.sqrt(F), q.dtype
    step = case["dir"] == "step"
    out = torch.empty((nd, H, F), device="cuda")
    if step:
        dq = torch.empty((nd, H, F), device="cuda")
        dk, dv = torch.zeros((ns, K, F), device="cuda"), torch.zeros((ns, K, F), device="cuda")
        db = torch.empty((e, H, 1), device="cuda") if "bias" in t else None
    per = max(1, min(H, (1 << 30) // max(e * F, 1)))
    for h0 in range(0, H, per):
        h1 = min(H, h0 + per)
        of = torch.arange(h0, h1, device="cuda") // rep
        qh = q[:, h0:h1].float()
        kh, vh = k[:, of].float(), v[:, of].float()
        s = (qh[dst] * kh[src]).sum(-1) * scale
        if "bias" in t:
            s = s + t["bias"][:, h0:h1, 0].float()
        at = dst.view(e, 1).expand(e, h1 - h0)
        top = torch.full((nd, h1 - h0), -math.inf, device="cuda").scatter_reduce_(0, at, s, "amax")
        top = torch.where(top == -math.inf, 0.0, top)
        a = torch.exp(s - top[dst])
        del s
        total = torch.zeros((nd, h1 - h0), device="cuda").index_add_(0, dst, a)
        a = a / torch.where(total == 0.0, 1.0, total)[dst]
        m = a.unsqueeze(-1) * vh[src]
        out[:, h0:h1] = torch.zeros((nd, h1 - h0, F), device="cuda").index_add_(0, dst, m)
        del m
        if step:
            z = t["dout"][:, h0:h1].float()
            da = (z[dst] * vh[src]).sum(-1)
            mean = torch.zeros((nd, h1 - h0), device="cuda").index_add_(0, dst, a * da)
            ds = a * (da - mean[dst])
            if db is not None:
                db[:, h0:h1, 0] = ds
            ds = (ds * scale).unsqueeze(-1)
            dq[:, h0:h1] = torch.zeros((nd, h1 - h0, F), device="cuda").index_add_(0, dst, ds * kh[src])
            dkh = torch.zeros((ns, h1 - h0, F), device="cuda").index_add_(0, src, ds * qh[dst])
            dvh = torch.zeros((ns, h1 - h0, F), device="cuda").index_add_(0, src, a.unsqueeze(-1) * z[dst])
            dk.index_add_(1, of, dkh)
            dv.index_add_(1, of, dvh)
    got = {"out": out.to(dt)}
    if step:
        got.update(dq=dq.to(dt), dk=dk.to(dt), dv=dv.to(dt))
        if db is not None:
            got["dbias"] = db.to(dt)
    return got


def _own_run(state):
    from paper_1909_01315_amd import gnnk
    case, t = state["case"], state["t"]
    step = case["dir"] == "step"
    if case["op"] == "rotary":
        got = {"out": gnnk.node_rotary(state["rot"], t["q"], t["pos"])}
        if step:
            got["dx"] = gnnk.node_rotary(state["rot"], t["gq"], t["pos"], inverse=True)
        return got
    if case["op"] == "norm_rotary":
        rot, pos = state["rot"], t["pos"]
        q, k = gnnk.node_norm_rotary(t["q"], t["wq"], t["k"], t["wk"], rot=rot, pos_q=pos, pos_k=pos, eps=EPS)
        if not step:
            return {"q": q, "k": k}
        dq, dwq, dk, dwk = gnnk.node_norm_rotary_backward(t["q"], t["wq"], t["gq"], t["k"], t["wk"], t["gk"], rot=rot,
                                                          pos_q=pos, pos_k=pos, eps=EPS)
        return {"q": q, "dq": dq, "dwq": dwq, "k": k, "dk": dk, "dwk": dwk}
    g, bias = state["g"], t.get("bias")
    if not step:
        return {"out": gnnk.dot_aggregate(g, t["q"], t["k"], t["v"], bias=bias)}
    out, stats = gnnk.dot_aggregate(g, t["q"], t["k"], t["v"], bias=bias, want_stats=True)
    dq, dk, dv, db = gnnk.dot_aggregate_backward(g, t["q"], t["k"], t["v"], out, stats, t["dout"], bias=bias)
    got = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if db is not None:
        got["dbias"] = db
    return got


def run(state):
    if own:
        return _own_run(state)
    case, t = state["case"], state["t"]
    return {"rotary": _plain_rotary, "norm_rotary": _plain_norm_rotary, "dot": _plain_dot}[case["op"]](case, t)


def work(case):
    """Bytes: every input and output of the forward, and of the gradients, once; for the attention also a pass over the
    graph's neighbour ids and row offsets in each direction.  Operations: two to a multiplication and addition."""
    s, H, F = (2 if case["dtype"] == "bf16" else 4), case["heads"], case["feat"]
    step = case["dir"] == "step"
    if case["op"] == "dot":
        K, e, ns, nd = case["kv_heads"], case["e"], case["n_src"], case["n_dst"]
        nodes = (nd * H + 2 * ns * K) * F * s
        edges = e * H * s if case["bias"] != "none" else 0
        fwd = nodes + nd * H * F * s + edges + 4 * e + 4 * (nd + 1)
        flops = 4.0 * e * H * F
        if not step:
            return {"bytes": float(fwd), "flops": flops}
        bwd = 2 * nodes + nd * H * F * s + 2 * edges + 4 * e + 4 * (ns + 1)
        return {"bytes": float(fwd + bwd), "flops": flops * 3.5}
    n, pairs = case["rows"], _pairs(case)
    angles = n * len(pairs) * 4
    if case["op"] == "rotary":
        one = 2 * n * H * F * s + angles
        return {"bytes": float(one * (2 if step else 1)), "flops": 6.0 * n * H * sum(pairs) * (2 if step else 1)}
    cols = n * (H + case["kv_heads"]) * F
    return {"bytes": float(2 * cols * s + angles + ((3 * cols * s + angles) if step else 0)),
            "flops": float(cols * (7 + (13 if step else 0)))}


# ---------------------------------------------------------------------------
# the same results in 64 bits


def _rotations(case, t):
    """exp(i theta) of every row and pair"""
    cols, p0 = [], 0
    for axis, p in enumerate(_pairs(case)):
        cols.append(t["pos"][:, axis].double().view(-1, 1) * t["freq"][p0:p0 + p].double().view(1, -1))
        p0 += p
    theta = torch.cat(cols, 1)
    return torch.polar(torch.ones_like(theta), theta).unsqueeze(1)


def _turned(x, by, interleaved):
    P = by.shape[-1]
    y = x.clone()
    first = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    z = torch.complex(x[..., first[0]].contiguous(), x[..., first[1]].contiguous()) * by
    y[..., first[0]], y[..., first[1]] = z.real, z.imag
    return y


def _exact_nodes(case, t):
    by, il = _rotations(case, t), case["interleaved"]
    step = case["dir"] == "step"
    if case["op"] == "rotary":
        got = {"out": _turned(t["q"].double(), by, il)}
        if step:
            got["dx"] = _turned(t["gq"].double(), by.conj(), il)
        return got
    got = {}
    for s in ("q", "k"):
        x, w = t[s].double(), t["w" + s].double()
        size = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS)
        unit = x / size
        got[s] = _turned(unit * w, by, il)
        if step:
            g = _turned(t["g" + s].double(), by.conj(), il)
            gu = g * w
            # the derivative of x / size in the direction of each column
            got["d" + s] = gu / size - unit * (gu * unit).mean(-1, keepdim=True) / size
            dw = (g * unit).sum(0, keepdim=True)
            got["dw" + s] = dw if w.shape[1] > 1 else dw.sum(1, keepdim=True)
    return got


def _exact_dot(case, t):
    """Head by head, the edges of a destination side by side (those of a source for its gradients)."""
    src, dst = t["src"].long(), t["dst"].long()
    H, F, K, nd, ns = case["heads"], case["feat"], case["kv_heads"], case["n_dst"], case["n_src"]
    step = case["dir"] == "step"
    order = torch.argsort(dst, stable=True)
    u, w = src[order], dst[order]
    sizes = torch.bincount(dst, minlength=nd)
    if step:
        back = torch.argsort(u, stable=True)
        outs = torch.bincount(src, minlength=ns)

    def rows(x, how="sum", lengths=sizes, initial=0.0):
        return torch.segment_reduce(x, how, lengths=lengths, axis=0, initial=initial, unsafe=True)

    def spread(weight, table, at, lengths, perm=None):
        parts = []
        for c in range(0, F, 16):
            m = table[:, c:c + 16].double()[at] * weight.unsqueeze(1)
            parts.append(rows(m if perm is None else m[perm], "sum", lengths))
        return torch.cat(parts, 1)

    def dots(x, y):
        total = torch.zeros(u.numel(), dtype=torch.float64, device="cuda")
        for c in range(0, F, 16):
            total += (x[:, c:c + 16].double()[w] * y[:, c:c + 16].double()[u]).sum(1)
        return total

    got = {"out": torch.empty((nd, H, F), dtype=torch.float64, device="cuda")}
    if step:
        got["dq"] = torch.empty((nd, H, F), dtype=torch.float64, device="cuda")
        for name in ("dk", "dv"):
            got[name] = torch.zeros((ns, K, F), dtype=torch.float64, device="cuda")
        if "bias" in t:
            got["dbias"] = torch.empty((case["e"], H, 1), dtype=torch.float64, device="cuda")
    for h in range(H):
        j = h // (H // K)
        s = dots(t["q"][:, h], t["k"][:, j]) / math.sqrt(F)
        if "bias" in t:
            s += t["bias"][:, h, 0].double()[order]
        top = rows(s, "max", initial=-math.inf)
        top[top == -math.inf] = 0.0
        a = torch.exp(s - top[w])
        total = rows(a)
        total[total == 0.0] = 1.0
        a /= total[w]
        got["out"][:, h] = spread(a, t["v"][:, j], u, sizes)
        if step:
            da = dots(t["dout"][:, h], t["v"][:, j])
            ds = a * (da - rows(a * da)[w])
            if "bias" in t:
                got["dbias"][order, h, 0] = ds
            ds /= math.sqrt(F)
            got["dq"][:, h] = spread(ds, t["k"][:, j], u, sizes)
            got["dk"][:, j] += spread(ds, t["q"][:, h], w, outs, back)
            got["dv"][:, j] += spread(a, t["dout"][:, h], w, outs, back)
    return got


def exact(case, seed):
    t = _inputs(case, seed)
    return _exact_dot(case, t) if case["op"] == "dot" else _exact_nodes(case, t)
