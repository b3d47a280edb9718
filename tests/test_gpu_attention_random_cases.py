"""Seeded draws of the attention operators that combine what the hand-written
cases list one at a time, against the same 64-bit forms and bounds.
GNNK_RANDOM_SEED0 and GNNK_RANDOM_CASES draw others."""
import os
import random

import pytest
import torch

import test_gpu_dot as dot
import test_gpu_rotary as rot
from test_gpu_dot import reset_options  # noqa: F401 (autouse)
from paper_1909_01315_amd import gnnk
from _heads import TURN_U, U32, angles, close, pair_size, turn

pytestmark = pytest.mark.gpu

SEED0 = int(os.environ.get("GNNK_RANDOM_SEED0", "0"))
CASES = int(os.environ.get("GNNK_RANDOM_CASES", "40"))


def draw_graph(r):
    kind = r.choice(["uniform", "uniform", "hubs", "one", "few"])
    if kind == "hubs":
        return dot.hubs(r.randrange(1000))
    if kind == "one":
        return dot.one(r.choice([1, 2, 63, 64, 65, 700, 5000]), r.randrange(1000))
    n_src, n_dst = r.randint(4, 300), r.randint(6, 300)
    return dot.uniform(n_src, n_dst, r.randint(1, 40) if kind == "few" else r.randint(50, 6000), r.randrange(1000))


@pytest.mark.parametrize("seed", range(SEED0, SEED0 + CASES))
def test_dot(seed):
    r = random.Random(seed)
    for key, values in (("seg_edges", [0, 0, 32, 64, 200]), ("no_fast", [0, 0, 0, 1]), ("no_split", [0, 0, 0, 1]),
                        ("small_deg", [-1, -1, 0, 5, 100]), ("order_edges", [0, 1]), ("neighbour_lists", [-1, 0, 3])):
        gnnk.set_option(key, r.choice(values))
    gr = draw_graph(r)
    K = r.choice([1, 1, 2, 3, 4, 5, 8, 16])
    H = K * r.choice([1, 1, 2, 3, 4, 5, 7, 8, 12, 16])
    F = r.choice([1, 2, 3, 4, 7, 8, 16, 16, 24, 31, 32, 32, 47, 64, 64, 73, 100, 128, 130, 250])
    while gr.e * H * F > 8000000:  # (the 64-bit form holds several values an edge, head and column)
        H, K, F = (H // K, 1, F) if K > 1 else (H, K, max(1, F // 2))
    dtype = r.choice([torch.float32, torch.bfloat16])
    kind = r.choice([None, "heads", "shared", "mask", "lowest"])
    pad, scale, size = r.choice([0, 0, 1, 2, 3, 8]), r.choice([None, None, 1.0, -0.25]), r.choice([1.0, 1.0, 0.01, 4.0])
    print(f"{gr.n_src} x {gr.n_dst}, {gr.e} edges, H {H} K {K} F {F} {dtype} {kind} pad {pad} scale {scale} size {size}")
    dot.check(gr, H, K, F, dtype, kind, pad, seed, scale, size)


@pytest.mark.parametrize("seed", range(SEED0, SEED0 + CASES))
def test_rotary_and_norms(seed):
    r = random.Random(seed)
    n, F = r.choice([1, 2, 7, 64, 300, 3000]), r.choice([2, 3, 5, 8, 16, 23, 32, 47, 64, 80, 128, 200, 512, 700])
    H = r.choice([1, 2, 3, 4, 7, 8, 16, 33])
    while n * H * F > 3000000:
        n = max(1, n // 2)
    dtype, il, pad = r.choice([torch.float32, torch.bfloat16]), r.random() < 0.5, r.choice([0, 1, 4, 5])
    pairs, left = [], r.randint(1, F // 2)
    for _ in range(r.randint(1, 4) - 1):
        pairs.append(r.randint(0, left))
        left -= pairs[-1]
    pairs = tuple(pairs + [left])
    print(f"{n} rows, H {H} F {F} pairs {pairs} interleaved {il} {dtype} pad {pad}")
    g = rot.gen(seed)
    x, z = (rot.normal(g, n, H, F, dtype=dtype) for _ in range(2))
    pos, freq = rot.positions(g, n, len(pairs), r.choice(["i32", "f32"])), rot.frequencies(pairs)
    op, theta, pd = gnnk.Rotary(freq.cuda(), pairs, interleaved=il), angles(pos, freq, pairs), pos.cuda()
    xd, zd = rot.spread(x, pad), rot.spread(z, pad)
    close(gnnk.node_rotary(op, xd, pd), turn(x.double(), theta, il),
          TURN_U * U32 * pair_size(x.double(), sum(pairs), il), "rotary")
    per_head = r.random() < 0.5
    w = (1 + 0.3 * rot.normal(g, 1, H if per_head else 1, F)).to(dtype)
    close(gnnk.node_norm_rotary(xd, w.cuda(), rot=op, pos_q=pd, eps=1e-5), *rot.norm_reference(x, w, theta, il, 1e-5),
          "norm")
    dx, dw = gnnk.node_norm_rotary_backward(xd, w.cuda(), zd, rot=op, pos_q=pd, eps=1e-5)
    want, bound, terms, tb = rot.norm_reference(x, w, theta, il, 1e-5, z)
    close(dx, want, bound, "dx")
    dims = (0,) if per_head else (0, 1)
    close(dw, terms.sum(dims).view(w.shape), tb.sum(dims).view(w.shape), "dw")
