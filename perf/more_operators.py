"""Performance cases of the operators between attention layers: the residual stream's addition with the root mean
square norm of its rows (and the gradients of that), rows of 8-bit integers with a scale each, and the product of such
rows with 8-bit weights that have a scale for each output column.

`run` computes each operator in a plain form, elementary torch operations in 32 bits rounded once at the end, or, with
`own` true, through this package.  A row is a node; the widths are those of layers over a graph's nodes.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
# products of the largest case, columns of the largest norm: no drawn case costs more
MOST_PRODUCTS, MOST_NORMED = 16384 * 4096 * 4096, 65536 * 4096


def listed():
    return [
        # norm of one new node's row in a serving loop: latency is all there is
        {"name": "norm_one_node", "op": "norm", "dir": "fwd", "rows": 1, "cols": 256, "residual": True,
         "dtype": "bf16"},
        # an odd width (6 heads of 47) and an odd count, a training step in bf16
        {"name": "norm_odd_step", "op": "norm", "dir": "step", "rows": 20011, "cols": 282, "residual": True,
         "dtype": "bf16"},
        # every point of a large cloud, a training step
        {"name": "norm_points_step", "op": "norm", "dir": "step", "rows": 262144, "cols": 256, "residual": True,
         "dtype": "f32"},
        # wide rows, inference, the largest norm
        {"name": "norm_wide", "op": "norm", "dir": "fwd", "rows": 65536, "cols": 4096, "residual": True,
         "dtype": "bf16"},
        # queries, keys and values of one new node in one product
        {"name": "linear_one_node", "op": "linear", "rows": 1, "cols": 1024, "outs": 1536, "bias": False,
         "dtype": "bf16"},
        # features stored in 8 bits, odd widths, results for a loss in fp32
        {"name": "linear_odd", "op": "linear", "rows": 20011, "cols": 282, "outs": 141, "bias": True, "dtype": "f32"},
        # queries, keys and values of a point cloud: about as much to write as to multiply
        {"name": "linear_points", "op": "linear", "rows": 262144, "cols": 256, "outs": 768, "bias": False,
         "dtype": "bf16"},
        # a wide layer over a batch of nodes, bound by the multiplications, the largest case
        {"name": "linear_large", "op": "linear", "rows": 16384, "cols": 4096, "outs": 4096, "bias": True,
         "dtype": "bf16"},
        # the entry of a layer for one new node: residual, norm, rows in 8 bits, product
        {"name": "norm_linear_one_node", "op": "norm_linear", "rows": 1, "cols": 512, "outs": 768, "residual": True,
         "bias": False, "dtype": "bf16"},
        # the same for every node of the large graph
        {"name": "norm_linear_layer", "op": "norm_linear", "rows": 232965, "cols": 512, "outs": 512, "residual": True,
         "bias": False, "dtype": "bf16"},
        # the product after the attention for a few nodes asked for together
        {"name": "quant_linear_few", "op": "quant_linear", "rows": 37, "cols": 2048, "outs": 2048, "bias": False,
         "dtype": "bf16"},
        # the same for a sampled block, 8 heads of 47 columns in fp32
        {"name": "quant_linear_block", "op": "quant_linear", "rows": 100000, "cols": 376, "outs": 256, "bias": True,
         "dtype": "f32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, most):
    """Columns of a row: multiples of 64, heads of other widths, or any number."""
    kind = rng.random()
    if kind < 0.4:
        return 64 * _log_int(rng, 1, most // 64)
    if kind < 0.6:
        return rng.choice([2, 4, 6, 8]) * rng.choice([8, 12, 20, 40, 47, 80])
    return _log_int(rng, 16, most)


def draw(rng):
    """Another case: any operator, count of rows, widths (odd ones among them) and type."""
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "norm_linear", "quant_linear"])
    rows, cols, dtype = _log_int(rng, 1, 300000), _width(rng, 4096), rng.choice(["f32", "bf16"])
    if op == "norm":
        way = rng.choice(["fwd", "step"])
        # (a step in fp32 moves four times the bytes)
        while rows * cols > MOST_NORMED // ((2 if way == "step" else 1) * (2 if dtype == "f32" else 1)):
            rows //= 2
        return {"op": op, "dir": way, "rows": rows, "cols": cols, "residual": rng.random() < 0.7, "dtype": dtype}
    outs = _width(rng, 4096)
    while rows * cols * outs > MOST_PRODUCTS // 2 or rows * (cols + outs) > MOST_NORMED // 2:
        rows //= 2
    case = {"op": op, "rows": rows, "cols": cols, "outs": outs, "bias": rng.random() < 0.4, "dtype": dtype}
    if op == "norm_linear":
        case["residual"] = rng.random() < 0.7
    return case


# ---------------------------------------------------------------------------
# inputs


def _in_8_bits(x):
    """Rows as whole numbers of -127 to 127 and the scale of each."""
    scale = x.abs().amax(1) / 127.0
    return torch.round(x / scale.unsqueeze(1)).clamp_(-127, 127).to(torch.int8), scale


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt, op, n, k = DTYPES[case["dtype"]], case["op"], case["rows"], case["cols"]
    t = {}

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    if op == "linear":
        t["q"], t["s"] = _in_8_bits(normal(n, k))
    else:
        t["x"] = normal(n, k).to(dt)
    if case.get("residual"):  # the stream grows from layer to layer, a few of its columns more than the others
        wide = 1.0 + 7.0 * (torch.rand(k, device="cuda", generator=gen) < 0.01).float()
        t["r"] = (3.0 * normal(n, k) * wide).to(dt)
    if op in ("norm", "norm_linear"):
        t["w"] = (1.0 + 0.2 * normal(k)).to(dt)
    if case.get("dir") == "step":
        t["gy"] = normal(n, k).to(dt)
        if case["residual"]:  # what the later layers send back along the stream
            t["gh"] = normal(n, k).to(dt)
    if op != "norm":
        t["wq"], t["ws"] = _in_8_bits(normal(case["outs"], k) / math.sqrt(k))
        if case["bias"]:
            t["b"] = (0.5 * normal(case["outs"])).to(_out_type(case))
    return t


def _out_type(case):
    """The product's: the case's for 8-bit rows; after a norm or an attention, bf16."""
    return DTYPES[case["dtype"]] if case["op"] == "linear" else torch.bfloat16


def prepare(case, seed):
    t = _inputs(case, seed)
    state = {"case": case, "t": t}
    if own and "wq" in t:
        from paper_1909_01315_amd import gnnk
        state["weight"] = gnnk.Weight8(t.pop("wq"), t.pop("ws"))
    return state


# ---------------------------------------------------------------------------
# the plain form


def _plain_sum(t):
    return t["x"].float() + t["r"].float() if "r" in t else t["x"].float()


def _plain_norm(h, w):
    return h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * w.float()


def _plain_rows8(x):
    """Values and scales: a row's largest magnitude is 127 steps."""
    s = x.abs().amax(1, keepdim=True) / 127.0
    return torch.round(x / s), s


def _plain_product(case, t, q, s):
    out = (q @ t["wq"].float().t()) * s * t["ws"]
    if "b" in t:
        out = out + t["b"].float()
    return out.to(_out_type(case))


def _plain(case, t):
    op = case["op"]
    if op == "linear":
        return {"out": _plain_product(case, t, t["q"].float(), t["s"].unsqueeze(1))}
    h = _plain_sum(t)
    if op == "quant_linear":
        return {"out": _plain_product(case, t, *_plain_rows8(h))}
    y, dt, got = _plain_norm(h, t["w"]), t["x"].dtype, {}
    if "r" in t:
        got["h"] = h.to(dt)
    if op == "norm_linear":
        got["out"] = _plain_product(case, t, *_plain_rows8(y))
        return got
    got["y"] = y.to(dt)
    if case["dir"] == "step":
        g, w = t["gy"].float(), t["w"].float()
        rn = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        gw = g * w
        dx = rn * (gw - h * (rn * rn * (gw * h).mean(1, keepdim=True)))
        if "gh" in t:
            dx = dx + t["gh"].float()
        got["dx"] = dx.to(dt)
        got["dw"] = (g * h * rn).sum(0).to(dt)
    return got


def _own_run(state):
    from paper_1909_01315_amd import gnnk
    case, t = state["case"], state["t"]
    op, r, b = case["op"], t.get("r"), t.get("b")
    if op == "linear":
        return {"out": gnnk.node_linear_i8(state["weight"], t["q"], t["s"], bias=b, dtype=_out_type(case))}
    if op == "quant_linear":
        q, s = gnnk.node_quantize(t["x"])
        return {"out": gnnk.node_linear_i8(state["weight"], q, s, bias=b, dtype=_out_type(case))}
    if op == "norm_linear":
        got = {}
        if r is not None:
            q, s, got["h"] = gnnk.node_add_norm_i8(t["x"], r, t["w"], eps=EPS)
        else:
            q, s = gnnk.node_add_norm_i8(t["x"], None, t["w"], eps=EPS)
        got["out"] = gnnk.node_linear_i8(state["weight"], q, s, bias=b, dtype=_out_type(case))
        return got
    if r is not None:
        y, h = gnnk.node_add_norm(t["x"], r, t["w"], eps=EPS)
        got = {"h": h, "y": y}
    else:
        h = t["x"]
        got = {"y": gnnk.node_add_norm(h, None, t["w"], eps=EPS)}
    if case["dir"] == "step":
        got["dx"], got["dw"] = gnnk.node_add_norm_backward(h, t["w"], t["gy"], grad_sum=t.get("gh"), eps=EPS)
    return got


def run(state):
    return _own_run(state) if own else _plain(state["case"], state["t"])


def work(case):
    """Bytes: every input and output once (8-bit rows between two operators are neither).  Operations: two to a
    multiplication and addition of the product, those of the norms counted singly."""
    n, k, op = case["rows"], case["cols"], case["op"]
    s = 2 if case["dtype"] == "bf16" else 4
    streams = 2 if case.get("residual") else 0  # the residual read, the sum written
    if op == "norm":
        moved, flops = 2 + streams, 5.0
        if case["dir"] == "step":  # and the stream, two gradients and theirs
            moved, flops = moved + (4 if case["residual"] else 3), flops + 12.0
        return {"bytes": float(n * k * s * moved + k * s), "flops": flops * n * k}
    m = case["outs"]
    product = m * k + 4 * m + n * m * (s if op == "linear" else 2)
    if op == "linear":
        rows = n * k + 4 * n
    else:
        rows = n * k * s * ((1 + streams) if op == "norm_linear" else 1)
    return {"bytes": float(product + rows), "flops": 2.0 * n * k * m}


# ---------------------------------------------------------------------------
# the same results in 64 bits


def _exact_rows8(x):
    most = torch.maximum(x.amax(1, keepdim=True), -x.amin(1, keepdim=True))
    return torch.round(x * 127.0 / most), most / 127.0


def exact(case, seed):
    t, op = _inputs(case, seed), case["op"]

    def product(q, s):
        out = torch.mm(q * s, (t["wq"].double() * t["ws"].double().unsqueeze(1)).t().contiguous())
        return out.add_(t["b"].double()) if "b" in t else out

    if op == "linear":
        return {"out": product(t["q"].double(), t["s"].double().unsqueeze(1))}
    if op == "quant_linear":
        return {"out": product(*_exact_rows8(t["x"].double()))}
    got, h, w = {}, t["x"].double(), t["w"].double()
    if "r" in t:
        h = got["h"] = h + t["r"].double()
    size = torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["cols"] + EPS)
    unit = h / size
    if op == "norm_linear":
        got["out"] = product(*_exact_rows8(unit * w))
        return got
    got["y"] = unit * w
    if case["dir"] == "step":
        g = t["gy"].double()
        gu = g * w
        # the derivative of h / size: what is along the row's own direction does not count
        dx = (gu - unit * (gu * unit).mean(1, keepdim=True)) / size
        got["dx"] = dx + t["gh"].double() if "gh" in t else dx
        got["dw"] = torch.einsum("nk,nk->k", g, unit)
    return got
