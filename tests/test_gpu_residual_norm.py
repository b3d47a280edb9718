"""The residual stream's sum and norm (node_add_norm, its backward) and rows in
8 bits (node_add_norm_i8, node_quantize) against their formulas in 64 bits,
within bounds derived in tests/_rows.py."""
import pytest
import torch

from paper_1909_01315_amd import gnnk
from _heads import U32, close
from _rows import BF16, F32, check_rows8, gen, norm, norm_gradients, normal, spread

pytestmark = pytest.mark.gpu

# rows, columns: one row and one column, every count of lanes, widths that end
# inside a vector, rows of several vectors a lane, of several wavefronts
SHAPES = [(1, 1), (1, 256), (700, 2), (300, 3), (513, 7), (129, 8), (65, 33), (1000, 47), (40, 64), (77, 100), (257, 128),
          (33, 255), (50, 282), (19, 512), (21, 513), (9, 1024), (30, 1500), (6, 2048), (7, 2049), (10, 2600), (5, 4096),
          (3, 4099), (4, 8191), (2, 16384), (9000, 16), (20000, 64), (2, 16383)]


def inputs(n, c, dtype, seed):
    g = gen(seed)
    x, r = normal(g, n, c, dtype=dtype), (3.0 * normal(g, n, c)).to(dtype)
    x[n // 2], r[n // 2] = 0.0, 0.0  # a row of zeros
    w = (1.0 + 0.3 * normal(g, c)).to(dtype)
    return g, x, r, w


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", SHAPES)
def test_norm(n, c, dtype):
    eps = 1e-5
    g, x, r, w = inputs(n, c, dtype, n + c)
    h = x.double() + r.double()
    pads = (0, 5) if c < 9000 else (3,)
    for pad in pads:
        xd, rd, wd = spread(x, pad), spread(r, 2 * pad), w.cuda()
        y, s = gnnk.node_add_norm(xd, rd, wd, eps=eps)
        close(s, h, U32 * h.abs(), "sum")
        close(y, *norm(h, w.double(), eps), "norm")
        close(gnnk.node_add_norm(xd, rd, None, eps=eps)[0], *norm(h, None, eps), "norm without a weight")
        close(gnnk.node_add_norm(xd, None, wd, eps=eps), *norm(x.double(), w.double(), eps), "norm without a residual")
        q, scale, s8 = gnnk.node_add_norm_i8(xd, rd, wd, eps=eps)
        assert torch.equal(s8, s)
        check_rows8(q, scale, *norm(h, w.double(), eps), "norm in 8 bits")
        assert q.shape == (n, c) and (n == 1 or q.stride(0) % 16 == 0)
        q1, s1 = gnnk.node_add_norm_i8(xd, None, None, eps=eps)
        check_rows8(q1, s1, *norm(x.double(), None, eps), "x's norm in 8 bits")
        q2, s2 = gnnk.node_quantize(xd)
        check_rows8(q2, s2, x.double(), 0.0 * x.double(), "x in 8 bits")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", SHAPES)
def test_gradients(n, c, dtype):
    eps = 1e-4
    g, x, r, w = inputs(n, c, dtype, n + 2 * c)
    gy, gs = normal(g, n, c, dtype=dtype), normal(g, n, c, dtype=dtype)
    xd, gyd, gsd, wd = spread(x, 3), spread(gy, 1), spread(gs, 6), w.cuda()
    for with_sum in (True, False):
        dx, dw = gnnk.node_add_norm_backward(xd, wd, gyd, grad_sum=gsd if with_sum else None, eps=eps)
        rx, bx, terms, tb = norm_gradients(x.double(), w.double(), gy.double(), gs.double() if with_sum else None, eps)
        close(dx, rx, bx, "dx")
        assert dw.shape == w.shape
        close(dw, terms.sum(0), tb.sum(0), "dw")
    a, none = gnnk.node_add_norm_backward(xd, wd, gyd, eps=eps, want_weight=False)
    assert none is None and torch.equal(a, dx)
    none, b = gnnk.node_add_norm_backward(xd, wd, gyd, eps=eps, want_x=False)
    assert none is None and torch.equal(b, dw)
    rx, bx, _, _ = norm_gradients(x.double(), None, gy.double(), None, eps)
    plain, none = gnnk.node_add_norm_backward(xd, None, gyd, eps=eps)
    assert none is None
    close(plain, rx, bx, "dx without a weight")


def test_heads_of_a_row_are_normed_together():
    g, x, r, w = inputs(200, 6 * 47, BF16, 3)
    y, s = gnnk.node_add_norm(x.cuda(), r.cuda(), w.cuda())
    heads = lambda t: t.cuda().view(200, 6, 47)
    y3, s3 = gnnk.node_add_norm(heads(x), heads(r), w.cuda().view(6, 47))
    assert y3.shape == s3.shape == (200, 6, 47)
    assert torch.equal(y3.view(200, -1), y) and torch.equal(s3.view(200, -1), s)
    q, sc = gnnk.node_quantize(heads(x))
    assert q.shape == (200, 282) and torch.equal(q, gnnk.node_quantize(x.cuda())[0])
    dx, dw = gnnk.node_add_norm_backward(s3, w.cuda().view(1, 6, 47), heads(r))
    assert dx.shape == (200, 6, 47) and dw.shape == (1, 6, 47)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", [(300, 47), (50, 282), (9, 5000), (400, 16)])
def test_in_place(n, c, dtype):
    g, x, r, w = inputs(n, c, dtype, 5)
    wd = w.cuda()
    y, s = gnnk.node_add_norm(x.cuda(), r.cuda(), wd)
    for pad in (0, 5):
        xd, rd = spread(x, pad), spread(r, pad)
        y1, s1 = gnnk.node_add_norm(xd, rd, wd, out=xd, out_sum=rd)
        assert y1 is xd and s1 is rd and torch.equal(y1, y) and torch.equal(s1, s)
        xd, rd = spread(x, pad), spread(r, pad)
        y1, s1 = gnnk.node_add_norm(xd, rd, wd, out=rd, out_sum=xd)
        assert torch.equal(y1, y) and torch.equal(s1, s)
        xd, rd = spread(x, pad), spread(r, pad)
        q, scale, s1 = gnnk.node_add_norm_i8(xd, rd, wd, out_sum=rd)
        q0, scale0, _ = gnnk.node_add_norm_i8(x.cuda(), r.cuda(), wd)
        assert torch.equal(s1, s) and torch.equal(q, q0) and torch.equal(scale, scale0)
        gs = normal(gen(6), n, c, dtype=dtype)
        dx, _ = gnnk.node_add_norm_backward(x.cuda(), wd, r.cuda(), grad_sum=gs.cuda())
        for which in range(3):
            ts = [spread(t, pad) for t in (x, r, gs)]
            got, _ = gnnk.node_add_norm_backward(ts[0], wd, ts[1], grad_sum=ts[2], grad_x=ts[which])
            assert got is ts[which] and torch.equal(got, dx)


def test_only_the_rows_own_columns_are_written():
    n, c = 70, 45
    g, x, r, w = inputs(n, c, F32, 8)
    outs = [torch.full((n + 2, c + 9), 7.0, device="cuda") for _ in range(3)]
    own = [t[1:n + 1, 3:3 + c] for t in outs]
    gnnk.node_add_norm(x.cuda(), r.cuda(), w.cuda(), out=own[0], out_sum=own[1])
    gnnk.node_add_norm_backward(x.cuda(), w.cuda(), r.cuda(), grad_x=own[2])
    for t in outs:
        t[1:n + 1, 3:3 + c] = 7.0
        assert bool((t == 7.0).all())
    q8 = torch.full((n + 2, c + 9), 77, dtype=torch.int8, device="cuda")
    sc = torch.full((n + 2,), 7.0, device="cuda")
    a, b = gnnk.node_quantize(x.cuda(), out=q8[1:n + 1, 3:3 + c], scale=sc[1:n + 1])
    q0, s0 = gnnk.node_quantize(x.cuda())
    assert torch.equal(a, q0) and torch.equal(b, s0)
    q8[1:n + 1, 3:3 + c] = 77
    assert bool((q8 == 77).all()) and float(sc[0]) == float(sc[-1]) == 7.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("c", [5, 47, 512, 6000])
def test_rows_in_8_bits_at_the_ends_of_the_range(c, dtype):
    """Zeros, the largest and the smallest numbers, infinities and NaN: each in its own row alone."""
    g = gen(21)
    x = normal(g, 12, c, dtype=dtype)
    x[1] = 0.0
    x[2, 3] = float("inf")
    x[3, 0] = float("-inf")
    x[4, c - 1] = float("nan")
    x[5] *= 1e38 / 5
    x[6] *= torch.tensor(1e-38, dtype=dtype)
    x[7] = 0.0
    x[7, 1] = 2.0 ** -133  # one step of bf16's smallest numbers
    x[8, 2] = float("inf")
    x[8, 4] = float("nan")
    q, s = gnnk.node_quantize(x.cuda())
    q, s = q.cpu(), s.cpu()
    bad = torch.zeros(12, dtype=torch.bool)
    bad[[2, 3, 4, 8]] = True
    assert torch.equal(torch.isnan(s), bad) and bool((q[bad] == 0).all())
    assert float(s[1]) == 0.0 and bool((q[1] == 0).all())
    ok = ~bad
    xs = x[ok].double()
    assert bool((s[ok][s[ok] > 0] >= 2.0 ** -126).all())
    # half a step; fp32's product with the scale's inverse and the division's rounding
    tol = s[ok].double().unsqueeze(1) * (0.5 + 127 * 4 * U32)
    assert bool(((q[ok].double() * s[ok].double().unsqueeze(1) - xs).abs() <= tol).all())
    # the norm of a row with an infinity or a NaN is none of the others' business
    y = gnnk.node_add_norm(x.cuda(), None, None, eps=1e-6).cpu()
    y8, s8 = gnnk.node_add_norm_i8(x.cuda(), None, None, eps=1e-6)
    assert torch.equal(torch.isnan(s8.cpu()), ~torch.isfinite(y).all(1))
    assert bool(torch.isfinite(y[[0, 1, 6, 7, 9, 10, 11]]).all())


def test_ties_go_to_the_even_number():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    q, s = gnnk.node_quantize(x)
    assert float(s[0]) == 1.0
    assert q[0].tolist() == [127, 0, 2, 2, 0, -2, -2, 126]


@pytest.mark.parametrize("n,c", [(700, 33), (5000, 376), (200, 2048), (6, 5001)])
def test_halves_of_the_largest_magnitude_go_to_the_even_number(n, c):
    """127 x / max |x| rounded to the nearest, ties to even.  Of values of 8 significant bits it is either a tie or 2^-16 of
    itself away from one, more than the 2^-23 by which the inverse of the step may be off: the numbers are those of the exact
    quotient, which 64 bits round to no tie that it is not.  (Half the largest magnitude is 63.5 steps.)"""
    g = gen(n)
    x = normal(g, n, c, dtype=BF16)
    x[:, 1], x[:, 3] = 0.0, 0.0
    half = x.abs().amax(1) / 2
    x[:, 1], x[n // 2:, 3] = half, -half[n // 2:]
    v = x.double()
    want = torch.round(127.0 * v / v.abs().amax(1, keepdim=True))
    assert bool((want[:, 1] == 64).all()) and bool((want[n // 2:, 3] == -64).all())
    for dtype in (BF16, F32):
        assert torch.equal(gnnk.node_quantize(x.to(dtype).cuda())[0].cpu().double(), want), dtype


@pytest.mark.parametrize("n,c", [(700, 33), (5000, 376), (200, 2048)])
def test_numbers_of_fp32_rows(n, c):
    """The nearest to 127 x / max |x|, but for quotients up to 2^-23 of themselves below halfway, which may go up."""
    x = normal(gen(n + 1), n, c)
    v = x.double()
    v = 127.0 * v / v.abs().amax(1, keepdim=True)
    q = gnnk.node_quantize(x.cuda())[0].cpu().double()
    # (64 bits: the quotient, and what it is compared with, are off by 2^-52 of themselves)
    up = torch.round(v * (1 + 2.0 ** -23 + 2.0 ** -50))
    assert bool(((q == torch.round(v)) | (q == up)).all())


def test_no_rows():
    for dtype in (F32, BF16):
        x, w = torch.empty((0, 40), dtype=dtype, device="cuda"), torch.ones(40, dtype=dtype, device="cuda")
        y, s = gnnk.node_add_norm(x, x, w)
        assert y.shape == s.shape == (0, 40)
        q, sc, s = gnnk.node_add_norm_i8(x, x, w)
        assert q.shape == (0, 40) and sc.shape == (0,)
        assert gnnk.node_quantize(x)[0].shape == (0, 40)
        dx, dw = gnnk.node_add_norm_backward(x, w, x, x)
        assert dx.shape == (0, 40) and bool((dw == 0).all())


def test_weight_gradient_of_many_rows_is_the_same_every_time():
    g = gen(11)
    for n, c, dtype in ((300001, 64, F32), (40000, 513, BF16)):
        x, gy = normal(g, n, c, dtype=dtype), normal(g, n, c, dtype=dtype)
        w = torch.ones(c, dtype=dtype)
        first = gnnk.node_add_norm_backward(x.cuda(), w.cuda(), gy.cuda())
        for _ in range(3):
            again = gnnk.node_add_norm_backward(x.cuda(), w.cuda(), gy.cuda())
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        dx, bx, terms, tb = norm_gradients(x.double(), w.double(), gy.double(), None, 1e-6)
        close(first[1], terms.sum(0), tb.sum(0), "dw")
        close(first[0], dx, bx, "dx")


def test_the_sum_may_be_left_out():
    """The C call takes a residual without keeping the sum."""
    g, x, r, w = inputs(60, 100, F32, 2)
    xd, rd, wd = x.cuda(), r.cuda(), w.cuda()
    y, _ = gnnk.node_add_norm(xd, rd, wd)
    q, s, _ = gnnk.node_add_norm_i8(xd, rd, wd)
    y1, q1, s1 = torch.empty_like(y), torch.empty_like(q), torch.empty_like(s)
    d, lib, stream = gnnk._desc, gnnk.load(), torch.cuda.current_stream().cuda_stream
    assert lib.node_add_norm(d(xd), d(rd), d(wd.view(1, 1, -1)), 1e-6, None, d(y1), stream) == gnnk.OK
    assert lib.node_add_norm_i8(d(xd), d(rd), d(wd.view(1, 1, -1)), 1e-6, None, gnnk._rows8(q1, s1), stream) == gnnk.OK
    assert torch.equal(y1, y) and torch.equal(q1, q) and torch.equal(s1, s)


# rows enough to lie in fewer lanes, of three vectors each
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", [(4096, 141), (4100, 160), (4097, 282), (5000, 380), (4099, 640), (4096, 768), (4110, 769)])
def test_many_rows_in_few_lanes(n, c, dtype):
    test_norm(n, c, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", [(50, 600), (40, 1200), (31, 1501), (12, 2500), (7, 5001), (3, 12000)])
def test_three_vectors_a_lane(n, c, dtype):
    test_norm(n, c, dtype)
    test_gradients(n, c, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", [(4101, 80), (4096, 95), (4100, 191), (4097, 225), (4099, 129), (4105, 401), (4096, 511)])
def test_many_rows_of_any_address(n, c, dtype):
    test_norm(n, c, dtype)
    test_gradients(n, c, dtype)
