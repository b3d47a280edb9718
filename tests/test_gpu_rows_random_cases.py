"""Seeded draws of the operators on whole rows that combine what the
hand-written cases list one at a time, against the same 64-bit forms and
bounds.  GNNK_RANDOM_SEED0 and GNNK_RANDOM_CASES draw others."""
import math
import os
import random

import pytest
import torch

import test_gpu_linear_i8 as linear
from test_gpu_linear_i8 import reset_options  # noqa: F401 (autouse)
from paper_1909_01315_amd import gnnk
from _heads import U32, close
from _rows import BF16, F32, check_rows8, gen, norm, norm_gradients, normal, spread

pytestmark = pytest.mark.gpu

SEED0 = int(os.environ.get("GNNK_RANDOM_SEED0", "0"))
CASES = int(os.environ.get("GNNK_RANDOM_CASES", "40"))


def log_int(r, lo, hi):
    return int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("seed", range(SEED0, SEED0 + CASES))
def test_product(seed):
    r = random.Random(seed)
    n, k, o = log_int(r, 1, 3000), log_int(r, 1, 5000), log_int(r, 1, 2000)
    while n * k * o > 6e8:  # (the 64-bit product is the CPU's)
        n, k = max(1, n // 2), max(1, k // 2)
    if r.random() < 0.5:
        k = (k + 15) // 16 * 16
    pad = r.choice([0, 0, 0, 16, 32, 1, 5, 128])
    lead = r.choice([0, 0, 16, 1, 3]) if pad else None
    lead = min(lead, pad) if pad else None
    tile, dtype, bias, full = r.choice([0, 0, 0, *range(1, 8)]), r.choice([F32, BF16]), r.random() < 0.5, r.random() < 0.3
    print(f"{n} x {k} -> {o}, {dtype}, tile {tile}, pad {pad} lead {lead}, bias {bias}, full {full}", flush=True)
    linear.check(n, k, o, dtype, tile, bias, pad, lead, seed, full)


@pytest.mark.parametrize("seed", range(SEED0, SEED0 + CASES))
def test_norm(seed):
    r = random.Random(1000 + seed)
    c = log_int(r, 1, 16384)
    n = log_int(r, 1, max(1, min(20000, 3000000 // c)))
    dtype, eps, size = r.choice([F32, BF16]), r.choice([1e-6, 1e-3, 1.0]), r.choice([1.0, 1e-3, 100.0])
    pads = [r.choice([0, 0, 1, 2, 3, 8]) for _ in range(3)]
    with_r, with_w, with_gs = (r.random() < 0.6 for _ in range(3))
    print(f"{n} x {c} {dtype} eps {eps} size {size} pads {pads} residual {with_r} weight {with_w} sum's gradient {with_gs}",
          flush=True)
    g = gen(seed)
    x = (size * normal(g, n, c)).to(dtype)
    res = (size * normal(g, n, c)).to(dtype) if with_r else None
    w = (1 + 0.3 * normal(g, c)).to(dtype) if with_w else None
    gy, gs = normal(g, n, c, dtype=dtype), normal(g, n, c, dtype=dtype) if with_gs else None
    wd, w64 = (w.cuda(), w.double()) if with_w else (None, None)
    xd, rd = spread(x, pads[0]), (spread(res, pads[1]) if with_r else None)
    h = x.double() + res.double() if with_r else x.double()
    y, bound = norm(h, w64, eps)
    got = gnnk.node_add_norm(xd, rd, wd, eps=eps)
    if with_r:
        close(got[1], h, U32 * h.abs(), "sum")
    close(got[0] if with_r else got, y, bound, "norm")
    got8 = gnnk.node_add_norm_i8(xd, rd, wd, eps=eps)
    check_rows8(got8[0], got8[1], y, bound, "norm in 8 bits")
    check_rows8(*gnnk.node_quantize(xd), x.double(), 0 * x.double(), "rows in 8 bits")
    dx, dw = gnnk.node_add_norm_backward(xd, wd, spread(gy, pads[2]), grad_sum=gs.cuda() if with_gs else None, eps=eps)
    ex, bx, terms, tb = norm_gradients(x.double(), w64, gy.double(), gs.double() if with_gs else None, eps)
    close(dx, ex, bx, "dx")
    if with_w:
        close(dw, terms.sum(0), tb.sum(0), "dw")
