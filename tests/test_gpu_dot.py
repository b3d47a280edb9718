"""Dot-product attention over edges (dot_aggregate and its backward) against
its formulas in 64 bits, within the bounds of tests/_attention.py."""
import numpy as np
import pytest
import torch

from paper_1909_01315_amd import gnnk, nn
from _attention import Reference
from _heads import U32, close

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def reset_options():
    yield
    for key, value in (("seg_edges", 0), ("no_fast", 0), ("no_split", 0), ("small_deg", -1), ("order_edges", 0),
                       ("neighbour_lists", -1)):
        gnnk.set_option(key, value)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


class Graph:
    def __init__(self, src, dst, n_src, n_dst, ptr64=False):
        self.src, self.dst, self.n_src, self.n_dst = src.long(), dst.long(), n_src, n_dst
        self.e = src.numel()
        self.g = gnnk.Graph.from_coo(src.int().cuda(), dst.int().cuda(), n_src, n_dst, ptr64=ptr64)


def uniform(n_src=70, n_dst=60, e=900, seed=1):
    """a multigraph; the last rows of both sides have no edges"""
    g = gen(seed)
    return Graph(torch.randint(0, n_src - 3, (e,), generator=g), torch.randint(0, n_dst - 5, (e,), generator=g), n_src,
                 n_dst)


def hubs(seed=2):
    """one destination of 3,000 edges, one source of 2,500, rows of every length up to 70"""
    g = gen(seed)
    n = 400
    src = [torch.randint(0, n, (3000,), generator=g), torch.full((2500,), 7), torch.randint(0, n, (2415,), generator=g)]
    dst = [torch.full((3000,), 11), torch.randint(0, n, (2500,), generator=g),
           torch.arange(70).repeat_interleave(torch.arange(70))]
    src, dst = torch.cat(src), torch.cat(dst)
    p = torch.randperm(src.numel(), generator=g)
    return Graph(src[p], dst[p], n, n)


def one(n, seed=3):
    """one destination"""
    return Graph(torch.randperm(n, generator=gen(seed)), torch.zeros(n, dtype=torch.long), n, 1)


GRAPHS = {"uniform": uniform, "hubs": hubs, "one edge": lambda: one(1), "one row": lambda: one(5000),
          "no edges": lambda: Graph(torch.empty(0, dtype=torch.long), torch.empty(0, dtype=torch.long), 5, 4)}


def spread(t, pad):
    """t on the GPU in rows of a stride `pad` columns larger, off 16-byte alignment for an odd pad"""
    n, h, f = t.shape
    buf = torch.full((n, h * f + pad), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[:, pad // 2: pad // 2 + h * f].unflatten(1, (h, f))
    v.copy_(t)
    return v


def biases(gr, H, kind, dtype, seed):
    if kind is None:
        return None
    g = gen(seed)
    b = torch.randn((gr.e, 1 if kind == "shared" else H, 1), generator=g)
    if kind == "mask":
        gone = torch.rand(gr.e, generator=g) < 0.3
        gone |= gr.dst % 5 == 2  # all edges of a destination
        b[gone] = -torch.inf
    if kind == "lowest":
        b[torch.rand(gr.e, generator=g) < 0.3] = torch.finfo(dtype).min
        b[gr.dst % 5 == 2] = torch.finfo(dtype).min
    return b.to(dtype)


def check(gr, H, K, F, dtype, kind=None, pad=0, seed=5, scale=None, size=1.0):
    g = gen(seed)
    mk = lambda n, h: (size * torch.randn((n, h, F), generator=g)).to(dtype)
    q, k, v, dz = mk(gr.n_dst, H), mk(gr.n_src, K), mk(gr.n_src, K), mk(gr.n_dst, H)
    b = biases(gr, H, kind, dtype, seed + 1)
    ref = Reference(gr.src, gr.dst, gr.n_src, gr.n_dst, q, k, v, b, scale, dz)
    up = lambda t: spread(t, pad) if pad else t.cuda()
    qd, kd, vd, zd = up(q), up(k), up(v), up(dz)
    bd = b.cuda() if b is not None else None
    out, stats = gnnk.dot_aggregate(gr.g, qd, kd, vd, bias=bd, scale=scale, want_stats=True)
    close(out, ref.out, ref.out_bound, "out")
    live = ref.live & (ref.total > 0)
    st = stats.double().cpu()
    assert bool((st[~live] == 0).all())
    # the statistics: 1 / sum against the maximum that stands beside it
    mine = torch.exp(ref.top - st[..., 0]) * ref.total * st[..., 1]
    assert bool(((mine - 1).abs() <= ref.stats_bound + 4 * U32 * (1 + ref.top.abs()))[live].all()), "stats"
    assert torch.equal(gnnk.dot_aggregate(gr.g, qd, kd, vd, bias=bd, scale=scale), out)
    got = gnnk.dot_aggregate_backward(gr.g, qd, kd, vd, out, stats, zd, bias=bd, scale=scale)
    names = ("dq", "dk", "dv") + (("dbias",) if b is not None else ())
    for name, t in zip(names, got):
        close(t, getattr(ref, name), getattr(ref, name + "_bound"), name)
    assert (got[3] is None) == (b is None)
    # some gradients alone are the same gradients
    part = gnnk.dot_aggregate_backward(gr.g, qd, kd, vd, out, stats, zd, bias=bd, scale=scale, want_q=False,
                                       want_v=False)
    assert part[0] is None and part[2] is None and torch.equal(part[1], got[1])
    assert b is None or torch.equal(part[3], got[3])
    return out, got


SHAPES = [(1, 1, 1), (4, 4, 2), (3, 1, 3), (8, 8, 16), (8, 2, 32), (6, 3, 47), (3, 3, 5), (16, 16, 64), (2, 1, 256),
          (12, 4, 20), (5, 5, 24), (7, 7, 130)]


@pytest.mark.parametrize("kind", [None, "heads", "shared", "mask", "lowest"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,K,F", SHAPES + [(4, 2, 8)])
def test_small_rows(H, K, F, dtype, kind):
    check(uniform(), H, K, F, dtype, kind)


# query heads of a key head that are no multiple of what a lane takes, more
# than a wavefront holds, in narrow and wide heads
@pytest.mark.parametrize("kind", [None, "heads", "shared", "mask"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,K,F", [(3, 1, 64), (6, 2, 32), (12, 1, 8), (5, 1, 40), (7, 1, 16), (24, 2, 64), (10, 2, 3),
                                   (16, 1, 256), (11, 1, 100), (64, 1, 8), (32, 4, 128)])
def test_query_heads_of_a_key_head(H, K, F, dtype, kind):
    check(uniform(e=700), H, K, F, dtype, kind)
    gnnk.set_option("seg_edges", 64)
    check(hubs(), H, K, F, dtype, kind)


@pytest.mark.parametrize("no_fast", [0, 1])
@pytest.mark.parametrize("seg", [0, 64])
@pytest.mark.parametrize("H,K,F,dtype,kind", [
    (8, 8, 16, F32, None), (8, 2, 32, BF16, "heads"), (6, 3, 47, F32, "mask"), (16, 16, 64, F32, "shared"),
    (2, 2, 8, F32, "shared"), (1, 1, 4, F32, None), (4, 4, 8, BF16, "mask"), (2, 1, 256, BF16, None),
    (3, 3, 5, BF16, "heads"), (1, 1, 128, BF16, "mask")])
def test_hub_rows(H, K, F, dtype, kind, seg, no_fast):
    gnnk.set_option("seg_edges", seg)
    gnnk.set_option("no_fast", no_fast)
    gr = hubs()
    info = gr.g.info()
    assert info["hub_dst_rows"] > 0 and info["hub_src_rows"] > 0
    check(gr, H, K, F, dtype, kind)


@pytest.mark.parametrize("key,value", [("no_split", 1), ("small_deg", 0), ("small_deg", 4000)])
@pytest.mark.parametrize("H,K,F,dtype", [(8, 8, 16, F32), (4, 2, 24, BF16), (1, 1, 4, F32)])
def test_results_of_every_schedule(H, K, F, dtype, key, value):
    gnnk.set_option(key, value)
    check(hubs(), H, K, F, dtype, "heads")


@pytest.mark.parametrize("lists", [0, 3])
def test_rows_listed_by_neighbour(lists):
    gnnk.set_option("order_edges", 1)
    gnnk.set_option("neighbour_lists", lists)
    check(hubs(), 4, 2, 16, F32, "mask")


@pytest.mark.parametrize("name", list(GRAPHS))
@pytest.mark.parametrize("H,K,F,dtype,kind", [(8, 8, 16, F32, None), (8, 2, 64, BF16, "shared"), (3, 1, 7, F32, "heads")])
def test_graphs_from_no_edges_to_one_long_row(name, H, K, F, dtype, kind):
    check(GRAPHS[name](), H, K, F, dtype, kind)


@pytest.mark.parametrize("H,K,F,dtype,kind", [
    (1, 1, 256, F32, "heads"), (2, 1, 512, BF16, "shared"), (256, 256, 256, F32, "shared"), (128, 32, 512, BF16, "mask"),
    (1024, 8, 64, BF16, None), (300, 300, 1, F32, "shared")])
def test_widest_heads_and_rows(H, K, F, dtype, kind):
    check(uniform(30, 20, 60), H, K, F, dtype, kind)


@pytest.mark.parametrize("n_src,n_dst", [(0, 4), (5, 0), (0, 0)])
@pytest.mark.parametrize("shared", [False, True])
def test_graphs_without_a_side(n_src, n_dst, shared):
    none = torch.empty(0, dtype=torch.long)
    gr = Graph(none, none, n_src, n_dst)
    q, kv = torch.randn((n_dst, 4, 8), device="cuda"), torch.randn((n_src, 2, 8), device="cuda")
    b = torch.empty((0, 1 if shared else 4, 1), device="cuda")
    out, stats = gnnk.dot_aggregate(gr.g, q, kv, kv, bias=b, want_stats=True)
    assert out.shape == q.shape and bool((out == 0).all()) and bool((stats == 0).all())
    grads = gnnk.dot_aggregate_backward(gr.g, q, kv, kv, out, stats, q, bias=b)
    for t, x in zip(grads, (q, kv, kv, b)):
        assert t.shape == x.shape and bool((t == 0).all())


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("H,K,F,dtype", [(8, 8, 16, F32), (6, 3, 47, BF16), (4, 4, 8, BF16), (2, 2, 3, F32)])
def test_strided_rows_of_any_alignment(H, K, F, dtype, pad):
    check(uniform(), H, K, F, dtype, "heads", pad=pad)


def test_keys_and_values_as_parts_of_one_table():
    gr = uniform()
    g = gen(21)
    q, kv = torch.randn((gr.n_dst, 4, 16), generator=g).cuda(), torch.randn((gr.n_src, 8, 16), generator=g).cuda()
    got = gnnk.dot_aggregate(gr.g, q, kv[:, :4], kv[:, 4:])
    assert torch.equal(got, gnnk.dot_aggregate(gr.g, q, kv[:, :4].contiguous(), kv[:, 4:].contiguous()))


@pytest.mark.parametrize("scale,size", [(0.0, 1.0), (-0.7, 1.0), (4.0, 3.0), (1e-3, 1.0)])
def test_scales(scale, size):
    check(uniform(), 4, 4, 16, F32, "heads", scale=scale, size=size)


@pytest.mark.parametrize("seg", [0, 32])
def test_masked_edges_may_hold_anything(seg):
    """A source reached by masked edges alone holds NaN and infinities: no
    output or gradient sees them, and its own gradients are 0."""
    gnnk.set_option("seg_edges", seg)
    gr = hubs()
    g = gen(23)
    H, K, F = 4, 2, 12
    q, k, v, dz = (torch.randn((n, h, F), generator=g) for n, h in ((gr.n_dst, H), (gr.n_src, K), (gr.n_src, K),
                                                                    (gr.n_dst, H)))
    b = torch.randn((gr.e, H, 1), generator=g)
    b[(gr.src % 10 == 3)] = -torch.inf
    b[(gr.dst % 17 == 5)] = -torch.inf
    clean = Reference(gr.src, gr.dst, gr.n_src, gr.n_dst, q, k, v, b, None, dz)
    k[3::10], v[3::10] = float("nan"), float("inf")
    k[13::10] = -float("inf")
    # a destination with no unmasked edge may hold anything in its query too
    q[5::17], dz[5::17] = float("inf"), float("nan")
    out, stats = gnnk.dot_aggregate(gr.g, q.cuda(), k.cuda(), v.cuda(), bias=b.cuda(), want_stats=True)
    got = gnnk.dot_aggregate_backward(gr.g, q.cuda(), k.cuda(), v.cuda(), out, stats, dz.cuda(), bias=b.cuda())
    close(out, clean.out, clean.out_bound, "out")
    for name, t in zip(("dq", "dk", "dv", "dbias"), got):
        close(t, getattr(clean, name), getattr(clean, name + "_bound"), name)
    assert bool((got[1][3::10] == 0).all()) and bool((got[2][3::10] == 0).all())
    assert bool((out[5::17] == 0).all()) and bool((got[0][5::17] == 0).all())


def test_nan_reaches_only_rows_whose_edges_see_it():
    gr = uniform()
    g = gen(29)
    q, k, v = (torch.randn((n, 2, 10), generator=g) for n in (gr.n_dst, gr.n_src, gr.n_src))
    k[9, 1, 9] = float("nan")
    v[20, 0, 3] = float("inf")
    out = gnnk.dot_aggregate(gr.g, q.cuda(), k.cuda(), v.cuda()).cpu()
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[gr.dst[gr.src == 9], 1] = True
    want[gr.dst[gr.src == 20], 0, 3] = True
    assert torch.equal(bad, want)


def test_long_row_keeps_its_accuracy():
    """200,000 edges of one row, whole and in segments"""
    n, H, F = 200000, 2, 16
    g = gen(31)
    q, k, v = torch.randn((1, H, F), generator=g), torch.randn((n, H, F), generator=g), torch.rand((n, H, F), generator=g)
    for no_split in (0, 1):
        gnnk.set_option("no_split", no_split)
        gr = one(n)
        ref = Reference(gr.src, gr.dst, n, 1, q, k, v)
        out = gnnk.dot_aggregate(gr.g, q.cuda(), k.cuda(), v.cuda())
        # the values are positive: the numerator and the sum of weights each
        # take one rounding an edge and one a batch, over the 512 edges of a
        # segment at most (joined in fp64) or the row's eighth that a lane
        # group walks; the weights themselves are off as everywhere
        edges = n / 8 if no_split else 512
        weights = float(ref.stats_bound.max()) / 2 - U32 * (1.25 * n + 20)
        rel = float(((out.double().cpu() - ref.out).abs() / ref.out).max())
        assert rel <= 2 * (U32 * (1.25 * edges + 20) + weights), rel


def test_tables_past_32_bit_offsets():
    """Rows more than 4 GiB into their table (a view with a wide row stride)."""
    n, H, F = 70000, 1, 8
    stride = 34000  # 70,000 rows x 34,000 x 2 bytes = 4.8 GB
    g = gen(37)
    src = torch.cat([torch.arange(n - 64, n), torch.arange(32)])
    dst = torch.arange(96) % 3
    gr = Graph(src, dst, n, 3)
    table = torch.zeros((n, stride), dtype=BF16, device="cuda")
    kd, vd = table[:, 8:16].unflatten(1, (1, 8)), table[:, 101:109].unflatten(1, (1, 8))
    k, v = (torch.randn((n, H, F), generator=g).to(BF16) for _ in range(2))
    kd.copy_(k), vd.copy_(v)
    q, dz = (torch.randn((3, H, F), generator=g).to(BF16) for _ in range(2))
    ref = Reference(gr.src, gr.dst, n, 3, q, k, v, None, None, dz)
    out, stats = gnnk.dot_aggregate(gr.g, q.cuda(), kd, vd, want_stats=True)
    close(out, ref.out, ref.out_bound, "out")
    dq, dk, dv, _ = gnnk.dot_aggregate_backward(gr.g, q.cuda(), kd, vd, out, stats, dz.cuda())
    close(dq, ref.dq, ref.dq_bound, "dq")
    close(dk, ref.dk, ref.dk_bound, "dk")
    close(dv, ref.dv, ref.dv_bound, "dv")


def test_writes_only_its_columns():
    gr = hubs()
    H, K, F = 3, 3, 9
    g = gen(41)
    q, k, v = (torch.randn((n, 3, F), generator=g).cuda() for n in (gr.n_dst, gr.n_src, gr.n_src))
    buf = torch.full((gr.n_dst + 2, H * F + 6), 7.0, device="cuda")
    out = buf[1:-1, 3:3 + H * F].unflatten(1, (H, F))
    gnnk.dot_aggregate(gr.g, q, k, v, out=out)
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[1:-1, 3:3 + H * F] = True
    assert bool((buf[~inside] == 7.0).all())
    assert torch.equal(out, gnnk.dot_aggregate(gr.g, q, k, v))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,K,F,shared", [(8, 2, 16, False), (6, 3, 47, True), (3, 3, 5, False)])
def test_strided_bias_statistics_and_gradients(H, K, F, shared, dtype):
    """Every tensor of a call in wider rows: the same values, and nothing else written."""
    gnnk.set_option("seg_edges", 64)
    gr = hubs()
    g = gen(41)
    mk = lambda n, h, f=F: torch.randn((n, h, f), generator=g).to(dtype)
    q, k, v, z, b = mk(gr.n_dst, H), mk(gr.n_src, K), mk(gr.n_src, K), mk(gr.n_dst, H), mk(gr.e, 1 if shared else H, 1)
    up = [t.cuda() for t in (q, k, v, z, b)]
    out, stats = gnnk.dot_aggregate(gr.g, *up[:3], bias=up[4], want_stats=True)
    want = gnnk.dot_aggregate_backward(gr.g, *up[:3], out, stats, up[3], bias=up[4])
    wide = [spread(t, 5) for t in (q, k, v, z, b)]
    bufs = [torch.full((t.shape[0], t.shape[1] * t.shape[2] + 3), 7.0, dtype=t.dtype, device="cuda")
            for t in (out, stats, *want)]
    view = [w[:, 1: w.shape[1] - 2].unflatten(1, t.shape[1:]) for w, t in zip(bufs, (out, stats, *want))]
    gnnk.dot_aggregate(gr.g, *wide[:3], bias=wide[4], out=view[0], stats=view[1])
    d = gnnk._desc
    gnnk._run(gr.g, None, gnnk.load().dot_aggregate_backward, gr.g.handle, *(d(t) for t in wide[:3]), d(wide[4]),
              F ** -0.5, d(view[0]), d(view[1]), d(wide[3]), *(d(t) for t in view[2:]))
    for w, x, t in zip(bufs, view, (out, stats, *want)):
        assert torch.equal(x, t)
        assert bool((w[:, 0] == 7).all()) and bool((w[:, -2:] == 7).all())


def test_refusals():
    gr = uniform()
    ones = lambda n, h, f, t=F32: torch.ones((n, h, f), dtype=t, device="cuda")
    nd, ns, e = gr.n_dst, gr.n_src, gr.e
    q, k, v = ones(nd, 4, 8), ones(ns, 2, 8), ones(ns, 2, 8)

    def refused(status, *a, **kw):
        with pytest.raises(gnnk.GnnkError) as err:
            gnnk.dot_aggregate(gr.g, *a, **kw)
        assert err.value.status == status, err.value

    refused(gnnk.EINVAL, ones(nd + 1, 4, 8), k, v)
    refused(gnnk.EINVAL, q, ones(nd, 2, 8), v)
    refused(gnnk.EINVAL, q, ones(ns, 3, 8), ones(ns, 3, 8))       # 3 does not divide 4
    refused(gnnk.EINVAL, q, k, ones(ns, 2, 4))
    refused(gnnk.EINVAL, q, k, v.bfloat16())
    refused(gnnk.EINVAL, q, k, v, bias=ones(e, 2, 1))
    refused(gnnk.EINVAL, q, k, v, bias=ones(e, 4, 8))
    refused(gnnk.EINVAL, q, k, v, bias=ones(e - 1, 1, 1))
    refused(gnnk.EINVAL, q, k, v, stats=ones(nd, 4, 2, BF16))
    refused(gnnk.EUNSUPPORTED, ones(nd, 1, 257), ones(ns, 1, 257), ones(ns, 1, 257))
    refused(gnnk.EUNSUPPORTED, *(ones(n, 1, 513, BF16) for n in (nd, ns, ns)))
    out, stats = gnnk.dot_aggregate(gr.g, q, k, v, want_stats=True)
    for bad in (dict(grad_out=ones(nd, 4, 4)), dict(stats=None), dict(out=ones(nd, 2, 8))):
        a = dict(out=out, stats=stats, grad_out=q)
        a.update(bad)
        with pytest.raises((gnnk.GnnkError, AttributeError)):
            gnnk.dot_aggregate_backward(gr.g, q, k, v, **a)
    with pytest.raises(ValueError):
        gnnk.dot_aggregate(gr.g, q.cpu(), k, v)


def test_scratch_bound_covers_the_calls():
    import ctypes
    gnnk.set_option("seg_edges", 64)
    gr = hubs()
    lib = gnnk.load()
    s = torch.cuda.Stream()
    for H, K, F, shared in ((8, 2, 16, True), (16, 16, 64, True), (1, 1, 1, False)):
        g = gen(43)
        q, z = (torch.randn((gr.n_dst, H, F), generator=g).cuda() for _ in range(2))
        k, v = (torch.randn((gr.n_src, K, F), generator=g).cuda() for _ in range(2))
        b = torch.randn((gr.e, 1 if shared else H, 1), generator=g).cuda()
        out, stats = gnnk.dot_aggregate(gr.g, q, k, v, bias=b, want_stats=True)
        want = gnnk.dot_aggregate_backward(gr.g, q, k, v, out, stats, z, bias=b)
        torch.cuda.synchronize()
        d = gnnk._desc
        mine = [torch.full_like(t, 3.0) for t in want]
        call = lambda: lib.dot_aggregate_backward(gr.g.handle, d(q), d(k), d(v), d(b), F ** -0.5, d(out), d(stats),
                                                  d(z), *(d(t) for t in mine), s.cuda_stream)
        lib.graph_attach_scratch(gr.g.handle, s.cuda_stream, None, 0)
        assert call() == gnnk.ENOMEM
        need = ctypes.c_size_t(0)
        assert lib.gnnk_scratch_needed(ctypes.byref(need)) == gnnk.OK
        assert 0 < need.value <= gr.g.scratch_bytes(H * F, wide_sums=shared)
        s.synchronize()
        assert all(bool((t == 3.0).all()) for t in mine), "nothing may run when the call is short of scratch"
        buf = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert lib.graph_attach_scratch(gr.g.handle, s.cuda_stream, buf.data_ptr(), need.value) == gnnk.OK
        assert call() == gnnk.OK
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(mine, want))
        lib.graph_attach_scratch(gr.g.handle, s.cuda_stream, None, 0)


def test_replays_and_two_streams_equal_eager():
    gnnk.set_option("seg_edges", 64)
    gr = hubs()
    g = gen(47)
    H, K, F = 8, 4, 16
    q, z = (torch.randn((gr.n_dst, H, F), generator=g).cuda() for _ in range(2))
    k, v = (torch.randn((gr.n_src, K, F), generator=g).cuda() for _ in range(2))
    b = torch.randn((gr.e, 1, 1), generator=g).cuda()

    def step():
        out, stats = gnnk.dot_aggregate(gr.g, q, k, v, bias=b, want_stats=True)
        return [out, stats, *gnnk.dot_aggregate_backward(gr.g, q, k, v, out, stats, z, bias=b)]

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            both.append(step())
    torch.cuda.synchronize()
    for got in both:
        assert all(torch.equal(x, y) for x, y in zip(got, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        outs = step()
    for _ in range(4):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, eager))
        _ = (q * 2).sum().item()


def test_a_larger_call_leaves_a_captured_one_its_scratch():
    """Scratch grows for an eager call on the stream of a captured one: a
    replay afterwards writes into no tensor that lives since."""
    gnnk.set_option("seg_edges", 64)
    gr = hubs()
    g = gen(61)
    mk = lambda h, f: tuple(torch.randn((gr.n_dst, h, f), generator=g).cuda() for _ in range(3))
    small, large = mk(2, 16), mk(16, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = gnnk.dot_aggregate(gr.g, *small)
    torch.cuda.synchronize()
    before = gr.g._lent[s.cuda_stream]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = gnnk.dot_aggregate(gr.g, *small)
    with torch.cuda.stream(s):
        gnnk.dot_aggregate(gr.g, *large)
        after = gr.g._lent[s.cuda_stream]
        size = before.numel()
        assert after.numel() >= 2 * size
        del before
        since = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(3):
        got.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert all(bool((t == 7).all()) for t in since)


def test_second_derivatives_are_refused():
    gr = uniform()
    q, k = (torch.randn(n, 2, 8, device="cuda", requires_grad=True) for n in (gr.n_dst, gr.n_src))
    (d,) = torch.autograd.grad((nn.dot_aggregate(gr.g, q, k, k) ** 2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        (d ** 2).sum().backward()


@pytest.mark.parametrize("shared", [False, True])
def test_differentiable_form_matches_differences(shared):
    gr = uniform(20, 15, 120)
    g = gen(53)
    H, K, F = 4, 2, 6
    xs = [torch.randn(s, generator=g) for s in ((gr.n_dst, H, F), (gr.n_src, K, F), (gr.n_src, K, F),
                                                (gr.e, 1 if shared else H, 1))]
    c = torch.randn((gr.n_dst, H, F), generator=g)
    leaves = [t.cuda().requires_grad_(True) for t in xs]
    (nn.dot_aggregate(gr.g, *leaves) * c.cuda()).sum().backward()

    def value(ts):
        return (Reference(gr.src, gr.dst, gr.n_src, gr.n_dst, *ts).out * c.double()).sum()

    for i, t in enumerate(xs):
        d = torch.randn(t.shape, generator=g).double()
        h = 1e-5
        at = lambda s: value([u.double() + (s * h * d if j == i else 0.0) for j, u in enumerate(xs)])
        want = float((at(1) - at(-1)) / (2 * h))
        grad = leaves[i].grad.double().cpu()
        got = float((grad * d).sum())
        assert abs(got - want) <= 300 * U32 * float((grad.abs() * d.abs()).sum()) + 1e-6 * (1 + abs(want)), i


@pytest.mark.parametrize("norm", [True, False])
def test_layer_runs_them_together(norm):
    """nn.DotAttentionConv, positions, norms and attention chained, forward and
    every gradient, against the same chain in 64 bits through autograd."""
    from _heads import turn
    gr = uniform(90, 60, 1500)
    g = gen(59)
    pairs, H, K, F, D = (3, 4), 4, 2, 20, 24
    torch.manual_seed(3)
    layer = nn.DotAttentionConv(D, F, H, kv_heads=K, qk_norm=norm, axis_pairs=pairs).cuda()
    x = torch.randn((gr.n_src, D), generator=g)
    pos = torch.randn((gr.n_src, 2), generator=g) * 10
    b = torch.randn((gr.e, 1, 1), generator=g)
    b[gr.dst % 7 == 1] = -torch.inf
    c = torch.randn((gr.n_dst, H, F), generator=g)
    xd, bd = x.cuda().requires_grad_(True), b.cuda().requires_grad_(True)
    out = layer(gr.g, xd, pos.cuda(), bd)
    (out * c.cuda()).sum().backward()

    theta = (pos.double()[:, [0] * 3 + [1] * 4] * layer.rotary(xd.device).freq.double().cpu()).unsqueeze(1)
    P = {n: p.detach().double().cpu().requires_grad_(True) for n, p in layer.named_parameters()}
    x64, b64 = x.double().requires_grad_(True), b.double().requires_grad_(True)
    q = (x64[: gr.n_dst] @ P["fc_q.weight"].T).view(-1, H, F)
    k, v = ((x64 @ P[f"fc_{s}.weight"].T).view(-1, K, F) for s in "kv")
    if norm:
        f = lambda t, w: t / torch.sqrt((t * t).mean(-1, keepdim=True) + layer.eps) * w
        q, k = f(q, P["norm_q"]), f(k, P["norm_k"])
    q, k = turn(q, theta[: gr.n_dst], False), turn(k, theta, False)
    of = torch.arange(H) // (H // K)
    s = (q[gr.dst] * k[gr.src][:, of]).sum(-1) * F ** -0.5 + b64[:, :, 0]
    s = s.masked_fill(b64[:, :, 0] == -torch.inf, -1e300)  # (finite, so that autograd forms no NaN)
    w = torch.exp(s - s.max()) * (b64[:, :, 0] > -torch.inf)
    total = torch.zeros((gr.n_dst, H), dtype=torch.float64).index_add(0, gr.dst, w)
    a = w / torch.where(total == 0, 1.0, total)[gr.dst]
    want = torch.zeros((gr.n_dst, H, F), dtype=torch.float64).index_add(0, gr.dst, a.unsqueeze(-1) * v[gr.src][:, of])
    (want * c.double()).sum().backward()
    # fp32 products of 24 terms before and after, and the operators' bounds
    # (at most some 100 u): 200 u of the size of each tensor's values
    def near(t, r, what):
        t, r = t.detach().double().cpu(), r.detach()
        assert float((t - r).abs().max()) <= 200 * U32 * float(r.abs().max()) * 4, what
    near(out, want, "out")
    near(xd.grad, x64.grad, "dx")
    near(bd.grad, b64.grad, "dbias")
    for n, p in layer.named_parameters():
        near(p.grad, P[n].grad, n)


def test_layer_in_bf16_keeps_its_frequencies():
    gr = uniform(90, 60, 1500)
    layer = nn.DotAttentionConv(16, 32, 4, axis_pairs=(8, 8)).cuda().bfloat16()
    x = torch.randn(gr.n_src, 16, device="cuda", dtype=BF16)
    pos = torch.randint(0, 1000, (gr.n_src, 2), device="cuda", dtype=torch.int32)
    out = layer(gr.g, x, pos)
    assert out.dtype is BF16 and out.shape == (gr.n_dst, 4, 32) and bool(torch.isfinite(out).all())
    assert layer.rotary(x.device).freq.dtype is F32
    out.float().sum().backward()
    assert all(bool(torch.isfinite(p.grad).all()) for p in layer.parameters())
