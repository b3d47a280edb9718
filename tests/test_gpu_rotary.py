"""Rotary positions of several axes and norms of heads (node_rotary,
node_norm_rotary and its backward) against their formulas in 64 bits, within
bounds derived in tests/_heads.py and here."""
import numpy as np
import pytest
import torch

from paper_1909_01315_amd import gnnk, nn
from _heads import TURN_U, U32, angles, close, pair_size, turn

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g).to(dtype)


def positions(g, n, axes, kind):
    if kind == "i32":
        span = torch.tensor([2000000, 1024, 300, 7][:axes])
        return (torch.rand((n, axes), generator=g, dtype=torch.float64) * span).int()
    return torch.randn((n, axes), generator=g) * 30.0


def frequencies(pairs):
    return torch.cat([10000.0 ** (-torch.arange(p, dtype=torch.float64) / max(p, 1)) for p in pairs]).float()


def spread(t, pad):
    """t on the GPU in rows of a stride `pad` columns larger, off 16-byte alignment for an odd pad"""
    if pad == 0:
        return t.cuda()
    n, h, f = t.shape
    buf = torch.full((n, h * f + pad), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[:, pad // 2: pad // 2 + h * f].unflatten(1, (h, f))
    v.copy_(t)
    return v


# rows, heads, columns, pairs, interleaved
SHAPES = [
    (1, 8, 64, (12, 10, 10), False),
    (1, 1, 2, (1,), True),
    (3, 2, 3, (1,), False),          # an odd width: a column without a partner
    (1000, 3, 16, (4, 4), True),
    (777, 5, 47, (7, 7, 8), True),
    (777, 5, 47, (7, 7, 8), False),
    (130, 16, 32, (6, 5, 5), False),
    (64, 2, 128, (16, 20, 20), False),  # part of the head turns, 16 columns after
    (64, 2, 128, (16, 16, 16), True),
    (33, 300, 24, (4, 0, 4, 4), False),  # more heads than a block's groups, an axis without pairs
    (20, 2, 256, (64, 32, 32), True),
    (9, 1, 130, (65,), False),        # odd pairs, wider than one pass of single pairs
    (5, 2, 1030, (100, 100, 15), False),
    (4, 1, 2048, (1024,), True),
    (20000, 4, 8, (2, 1, 1), False),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,H,F,pairs,il", SHAPES)
def test_rotary(n, H, F, pairs, il, dtype):
    g = gen(n + F)
    x = normal(g, n, H, F, dtype=dtype)
    for kind, pad in (("i32", 0), ("f32", 3)):
        pos, freq = positions(g, n, len(pairs), kind), frequencies(pairs)
        rot = gnnk.Rotary(freq.cuda(), pairs, interleaved=il)
        theta = angles(pos, freq, pairs)
        xd, pd = spread(x, pad), pos.cuda()
        for inverse in (False, True):
            got = gnnk.node_rotary(rot, xd, pd, inverse=inverse)
            close(got, turn(x.double(), theta, il, inverse),
                  TURN_U * U32 * pair_size(x.double(), sum(pairs), il), f"rotary {kind} inverse={inverse}")
    P = sum(pairs)
    assert torch.equal(got[..., 2 * P:].cpu(), x[..., 2 * P:]), "columns after the pairs pass unchanged"


def test_rotary_writes_only_its_columns_and_passes_what_is_not_turned():
    pairs, H, F, n = (2, 2), 3, 11, 70
    g = gen(5)
    x = normal(g, n, H, F)
    x[3, 1, 9] = float("inf")
    x[4, 0, 10] = float("nan")
    rot = gnnk.Rotary(frequencies(pairs).cuda(), pairs)
    buf = torch.full((n + 2, H * F + 5), 7.0, device="cuda")
    out = buf[1:n + 1, 2:2 + H * F].unflatten(1, (H, F))
    pos = positions(g, n, 2, "f32")
    got = gnnk.node_rotary(rot, x.cuda(), pos.cuda(), out=out)
    assert got is out
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[1:n + 1, 2:2 + H * F] = True
    assert bool((buf[~inside] == 7.0).all())
    assert torch.equal(out[..., 8:].cpu().nan_to_num(1.5, 2.5), x[..., 8:].nan_to_num(1.5, 2.5))
    assert bool(torch.isfinite(out[..., :8]).all())
    # positions as a slice of a wider table
    wide = torch.zeros((n, 5), device="cuda")
    wide[:, 1:3] = pos.cuda()
    assert torch.equal(gnnk.node_rotary(rot, x.cuda(), wide[:, 1:3]).nan_to_num(3.5), out.nan_to_num(3.5))


def test_positions_at_the_ends_of_int32_and_many_heads():
    """An angle near 2^31 is off by 2.5 half steps of fp64 (the product, the
    constant's own, the product with it): 2.5 2^-53 2^31 = 10 u."""
    pairs, H, F, n = (4, 4), 1024, 16, 6
    g = gen(7)
    x = normal(g, n, H, F)
    ends = torch.tensor([-2 ** 31, 2 ** 31 - 1, 2 ** 31 - 2, 0, -1, 2 ** 30 + 1])
    pos, freq = torch.stack([ends, ends.flip(0)], 1).int(), frequencies(pairs)
    theta = angles(pos, freq, pairs)
    got = gnnk.node_rotary(gnnk.Rotary(freq.cuda(), pairs), x.cuda(), pos.cuda())
    close(got, turn(x.double(), theta, False), (TURN_U + 10) * U32 * pair_size(x.double(), 8, False), "rotary")


def test_rotary_of_no_rows():
    rot = gnnk.Rotary.geometric((2, 2))
    x = torch.empty((0, 2, 8), device="cuda")
    assert gnnk.node_rotary(rot, x, torch.empty((0, 2), device="cuda")).shape == (0, 2, 8)
    w = torch.ones(8, device="cuda")
    q, k = gnnk.node_norm_rotary(x, w, x, w)
    assert q.shape == k.shape == (0, 2, 8)
    for wq in (w, torch.ones((2, 8), device="cuda")):
        dq, dw = gnnk.node_norm_rotary_backward(x, wq, x)
        assert dq.shape == x.shape and dw.shape == wq.shape and bool((dw == 0).all())


# roundings of 1 / sqrt(mean(x^2) + eps): the squares' sum takes at most 38
# (16 terms a lane and pass and 6 steps across lanes, heads of at most 2,048
# columns), the mean and eps 3, all halved by the root; the root and division 1 each
R_U = 23


def norm_reference(x, w, theta, il, eps, g=None):
    """(out, bound) or with g (dx, bound, terms of dw, their bound), all in 64 bits before the sums over rows"""
    x, w = x.double(), w.double()
    P = theta.shape[-1] if theta is not None else 0
    size = lambda t: pair_size(t, P, il) if P else t.abs()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if g is None:
        y = x * r * w
        return (turn(y, theta, il) if P else y), (TURN_U + R_U + 2) * U32 * size(y)
    g0 = turn(g.double(), theta, il, inverse=True) if P else g.double()
    gs = size(g.double())
    gw, gws = g0 * w, gs * w.abs()
    dx = r * (gw - x * r * r * (gw * x).mean(-1, keepdim=True))
    # gw: 10 u; its sum with x: 49 u; r^2, the mean and their product: 50 u; the last product, difference and product
    # with r: 26 u
    m = r * r * (gws * x.abs()).mean(-1, keepdim=True)
    return dx, U32 * r * (36 * gws + 126 * x.abs() * m), g0 * x * r, 35 * U32 * gs * x.abs() * r


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("n,H,F,pairs,il", SHAPES + [(50, 4, 40, None, False), (200, 1, 5, None, False),
                                                        (40, 2, 1, None, False)])
def test_norm_rotary_and_gradients(n, H, F, pairs, il, per_head, dtype):
    g = gen(n * 3 + F)
    eps = 1e-5
    K = next(k for k in (H // 2, H // 3, 1) if k >= 1 and H % k == 0)
    nk = n + 7
    q, k = normal(g, n, H, F, dtype=dtype), normal(g, nk, K, F, dtype=dtype)
    q[n // 2] = 0.0  # a row of zeros
    gq, gk = normal(g, n, H, F, dtype=dtype), normal(g, nk, K, F, dtype=dtype)
    wq = (1.0 + 0.3 * normal(g, 1, H if per_head else 1, F)).to(dtype)
    wk = (1.0 + 0.3 * normal(g, 1, K if per_head else 1, F)).to(dtype)
    rot = pos_q = pos_k = tq = tk = None
    if pairs:
        freq = frequencies(pairs)
        pos_q, pos_k = positions(g, n, len(pairs), "f32"), positions(g, nk, len(pairs), "i32")
        rot = gnnk.Rotary(freq.cuda(), pairs, interleaved=il)
        tq, tk = angles(pos_q, freq, pairs), angles(pos_k, freq, pairs)
        pos_q, pos_k = pos_q.cuda(), pos_k.cuda()
    qd, kd, wqd, wkd = spread(q, 6), k.cuda(), wq.cuda(), wk.cuda()
    oq, ok = gnnk.node_norm_rotary(qd, wqd, kd, wkd, rot=rot, pos_q=pos_q, pos_k=pos_k, eps=eps)
    close(oq, *norm_reference(q, wq, tq, il, eps), "q")
    close(ok, *norm_reference(k, wk, tk, il, eps), "k")
    # one tensor alone, and without a weight
    close(gnnk.node_norm_rotary(kd, wkd, rot=rot, pos_q=pos_k, eps=eps), *norm_reference(k, wk, tk, il, eps), "k alone")
    one = torch.ones_like(wq)
    close(gnnk.node_norm_rotary(qd, None, rot=rot, pos_q=pos_q, eps=eps), *norm_reference(q, one, tq, il, eps),
          "q without a weight")
    dq, dwq, dk, dwk = gnnk.node_norm_rotary_backward(qd, wqd, spread(gq, 1), kd, wkd, gk.cuda(), rot=rot, pos_q=pos_q,
                                                      pos_k=pos_k, eps=eps)
    for got, dw, x, w, th, gr, name in ((dq, dwq, q, wq, tq, gq, "q"), (dk, dwk, k, wk, tk, gk, "k")):
        dx, bound, terms, tb = norm_reference(x, w, th, il, eps, gr)
        close(got, dx, bound, f"d{name}")
        dims = (0,) if per_head else (0, 1)
        assert dw.shape == w.shape
        close(dw, terms.sum(dims).view(w.shape), tb.sum(dims).view(w.shape), f"dw{name}")
    # weight gradients alone, data gradients alone
    a, b, c, d = gnnk.node_norm_rotary_backward(qd, wqd, gq.cuda(), kd, wkd, gk.cuda(), rot=rot, pos_q=pos_q,
                                                pos_k=pos_k, eps=eps, want_q=False, want_wk=False)
    assert a is None and d is None and torch.equal(b, dwq) and torch.equal(c, dk)


def test_weight_gradient_of_many_rows_is_the_same_every_time():
    g = gen(11)
    n, H, F = 300001, 4, 32
    x, gr = normal(g, n, H, F).cuda(), normal(g, n, H, F).cuda()
    w = torch.ones(F, device="cuda")
    rot = gnnk.Rotary.geometric((8, 8))
    pos = positions(g, n, 2, "f32").cuda()
    first = gnnk.node_norm_rotary_backward(x, w, gr, rot=rot, pos_q=pos)
    for _ in range(3):
        again = gnnk.node_norm_rotary_backward(x, w, gr, rot=rot, pos_q=pos)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    dx, bound, terms, tb = norm_reference(x.cpu(), w.cpu().view(1, 1, F), angles(pos, rot.freq, rot.pairs), False, 1e-6,
                                          gr.cpu())
    close(first[1], terms.sum((0, 1)), tb.sum((0, 1)), "dw of 1.2M heads")


def test_infinite_and_nan_values_stay_in_their_heads():
    g = gen(13)
    x = normal(g, 40, 4, 24)
    x[3, 1, 5], x[7, 2, 0] = float("inf"), float("nan")
    w = torch.ones(24)
    rot = gnnk.Rotary.geometric((6, 6))
    pos = positions(g, 40, 2, "f32")
    out = gnnk.node_norm_rotary(x.cuda(), w.cuda(), rot=rot, pos_q=pos.cuda()).cpu()
    bad = ~torch.isfinite(out).all(-1)
    want = torch.zeros(40, 4, dtype=torch.bool)
    want[3, 1] = want[7, 2] = True
    assert torch.equal(bad, want)


def test_differentiable_forms_match_differences():
    """Gradients of nn.rotary and nn.norm_rotary against central differences
    of their 64-bit forms along random directions."""
    g = gen(17)
    n, H, K, F, pairs, eps = 12, 4, 2, 20, (3, 4), 1e-4
    freq, pos = frequencies(pairs), positions(g, n, 2, "f32")
    theta = angles(pos, freq, pairs)
    rot = gnnk.Rotary(freq.cuda(), pairs)
    xs = [normal(g, n, H, F), 1 + 0.2 * normal(g, H, F), normal(g, n, K, F), 1 + 0.2 * normal(g, F)]
    cq, ck = normal(g, n, H, F), normal(g, n, K, F)
    leaves = [t.cuda().requires_grad_(True) for t in xs]
    q, k = nn.norm_rotary(*leaves, rot=rot, pos_q=pos.cuda(), pos_k=pos.cuda(), eps=eps)
    z = nn.rotary(rot, q, pos.cuda())
    ((z * cq.cuda()).sum() + (k * ck.cuda()).sum()).backward()

    def value(ts):
        a, wa, b, wb = ts
        f = lambda t, w: turn(t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * w, theta, False)
        return (turn(f(a, wa), theta, False) * cq.double()).sum() + (f(b, wb) * ck.double()).sum()

    for i, t in enumerate(xs):
        d = normal(g, *t.shape).double()
        h = 1e-5
        at = lambda s: value([u.double() + (s * h * d if j == i else 0.0) for j, u in enumerate(xs)])
        want = float((at(1) - at(-1)) / (2 * h))
        grad = leaves[i].grad.double().cpu()
        got = float((grad * d).sum())
        # fp32 gradients, at most 300 u of each term; differences exact to h^2
        assert abs(got - want) <= 300 * U32 * float((grad.abs() * d.abs()).sum()) + 1e-6 * (1 + abs(want)), i


def test_differentiable_norms_of_queries_alone():
    """Without keys the layer gives and derives the queries' part of the pair, also of two rows."""
    g = gen(23)
    rot = gnnk.Rotary.geometric((2, 2))
    for n in (2, 30):
        x, c, w = normal(g, n, 3, 8).cuda(), normal(g, n, 3, 8).cuda(), (1 + 0.2 * normal(g, 8)).cuda()
        pos = positions(g, n, 2, "f32").cuda()
        grads = []
        for k in (None, x):
            q, wq = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
            out = nn.norm_rotary(q, wq, k, None, rot=rot, pos_q=pos, pos_k=pos)
            out = out if k is None else out[0]
            (out * c).sum().backward()
            grads.append((out.detach(), q.grad, wq.grad))
        assert grads[0][0].shape == x.shape
        for a, b in zip(*grads):
            assert torch.equal(a, b)


def test_second_derivatives_are_refused():
    x = torch.randn(5, 2, 8, device="cuda", requires_grad=True)
    pos = torch.arange(5, device="cuda", dtype=torch.int32)
    rot = gnnk.Rotary.geometric((4,))
    for f in (lambda: nn.rotary(rot, x, pos), lambda: nn.norm_rotary(x, rot=rot, pos_q=pos)):
        (d,) = torch.autograd.grad((f() ** 2).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            (d ** 2).sum().backward()


def test_replays_on_another_stream_equal_eager():
    g = gen(19)
    n, H, F = 5000, 8, 32
    q, k, gq, gk = (normal(g, n, H, F).cuda() for _ in range(4))
    w = (1 + 0.1 * normal(g, F)).cuda()
    rot = gnnk.Rotary.geometric((6, 5, 5))
    pos = positions(g, n, 3, "f32").cuda()

    def step():
        a, b = gnnk.node_norm_rotary(q, w, k, w, rot=rot, pos_q=pos, pos_k=pos)
        return [a, b, gnnk.node_rotary(rot, a, pos),
                *gnnk.node_norm_rotary_backward(q, w, gq, k, w, gk, rot=rot, pos_q=pos, pos_k=pos)]

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = step()
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
        _ = (q * 2).sum().item()
