"""What the operators on whole rows refuse (the residual stream's norm, rows
and products in 8 bits), on the host before anything is launched (CPU only: the
tensors' addresses are never used)."""
import ctypes

import pytest
import torch

from paper_1909_01315_amd import gnnk

F32, BF16 = gnnk.F32, gnnk.BF16
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return gnnk.load()


def tensor(at, rows=10, feat=64, dtype=F32, stride=None, heads=1):
    return gnnk._TENSOR.pack(at, rows, heads, feat, heads * feat if stride is None else stride, dtype, 0)


def rows8(at, scale=16 * MB, rows=10, cols=64, stride=None):
    return gnnk._ROWS8.pack(at, scale, rows, cols if stride is None else stride, cols & 0xFFFFFFFF, 0)


def weight8(packed=32 * MB, scale=48 * MB, outs=96, cols=64):
    return gnnk._WEIGHT8.pack(packed, scale, outs & 0xFFFFFFFF, cols & 0xFFFFFFFF)


ROW = 256  # bytes of a row of the tensors above
NORM = dict(x=tensor(MB), r=tensor(2 * MB), w=tensor(3 * MB, rows=1), eps=1e-6, sum=tensor(4 * MB), out=tensor(5 * MB),
            q=rows8(6 * MB))

SHARED = [  # of both forms of the norm
    dict(x=None), dict(x=tensor(0)), dict(x=tensor(MB, stride=63)), dict(x=tensor(MB, rows=-1)),
    dict(x=tensor(MB, feat=0)), dict(x=tensor(MB, dtype=2)),
    dict(r=tensor(2 * MB, rows=9)), dict(r=tensor(2 * MB, feat=32)), dict(r=tensor(2 * MB, dtype=BF16)),
    dict(r=tensor(2 * MB, feat=16, heads=4)),
    dict(w=tensor(3 * MB, rows=2)), dict(w=tensor(3 * MB, rows=1, feat=63)), dict(w=tensor(3 * MB, rows=1, dtype=BF16)),
    dict(r=None),                                                   # a sum of no residual
    dict(sum=tensor(4 * MB, rows=11)), dict(sum=tensor(4 * MB, dtype=BF16)),
    dict(eps=-1e-6), dict(eps=float("nan")),
    dict(x=tensor(MB, feat=16385), r=tensor(2 * MB, feat=16385), w=None, sum=None, out=tensor(5 * MB, feat=16385),
         q=rows8(6 * MB, cols=16385)),
    dict(x=tensor(MB, rows=1 << 31, feat=1), r=None, w=None, sum=None, out=tensor(1 << 50, rows=1 << 31, feat=1),
         q=rows8(1 << 50, rows=1 << 31, cols=1)),
    dict(sum=tensor(MB + 4)), dict(sum=tensor(MB - ROW)), dict(sum=tensor(2 * MB + ROW)), dict(sum=tensor(3 * MB)),
    dict(sum=tensor(MB, stride=80)),                                # x's start in wider rows
]


def refused(lib, status, why=None):
    text = lib.gnnk_last_error()
    return status == gnnk.EINVAL and text and (why is None or why in text)


@pytest.mark.parametrize("change", SHARED + [
    dict(out=None), dict(out=tensor(0)), dict(out=tensor(5 * MB, rows=9)), dict(out=tensor(5 * MB, dtype=BF16)),
    dict(out=tensor(4 * MB)), dict(out=tensor(4 * MB + 8)), dict(out=tensor(MB + 4)), dict(out=tensor(2 * MB - 4)),
    dict(out=tensor(3 * MB - 2000)), dict(out=tensor(MB), sum=tensor(MB)),
])
def test_add_norm(lib, change):
    a = dict(NORM, **change)
    assert refused(lib, lib.node_add_norm(a["x"], a["r"], a["w"], a["eps"], a["sum"], a["out"], None))


@pytest.mark.parametrize("change", SHARED + [
    dict(q=None), dict(q=rows8(0)), dict(q=rows8(6 * MB, scale=0)), dict(q=rows8(6 * MB, rows=9)),
    dict(q=rows8(6 * MB, cols=63)), dict(q=rows8(6 * MB, stride=63)), dict(q=rows8(6 * MB, cols=0)),
    dict(q=rows8(6 * MB, stride=1 << 31)),
    dict(q=rows8(MB)), dict(q=rows8(2 * MB + 100)), dict(q=rows8(3 * MB + 255)), dict(q=rows8(4 * MB)),
    dict(q=rows8(6 * MB, scale=MB)), dict(q=rows8(6 * MB, scale=4 * MB + ROW)), dict(q=rows8(6 * MB, scale=6 * MB + 4)),
])
def test_add_norm_i8(lib, change):
    a = dict(NORM, **change)
    assert refused(lib, lib.node_add_norm_i8(a["x"], a["r"], a["w"], a["eps"], a["sum"], a["q"], None))


@pytest.mark.parametrize("x,q", [
    (None, rows8(6 * MB)), (tensor(MB), None), (tensor(MB), rows8(MB)), (tensor(MB), rows8(6 * MB, scale=MB + 40)),
    (tensor(MB), rows8(6 * MB, rows=11)), (tensor(MB), rows8(6 * MB, cols=65)), (tensor(MB), rows8(6 * MB, 6 * MB)),
    (tensor(MB, feat=16385), rows8(6 * MB, cols=16385)),
])
def test_quantize(lib, x, q):
    assert refused(lib, lib.node_quantize(x, q, None))


BACK = dict(h=tensor(MB), w=tensor(2 * MB, rows=1), g=tensor(3 * MB), gs=tensor(4 * MB), eps=1e-6, dx=tensor(5 * MB),
            dw=tensor(6 * MB, rows=1), work=8 * MB, bytes=MB)


def backward(lib, **change):
    a = dict(BACK, **change)
    return lib.node_add_norm_backward(a["h"], a["w"], a["g"], a["gs"], a["eps"], a["dx"], a["dw"], a["work"],
                                      a["bytes"], None)


@pytest.mark.parametrize("change", [
    dict(h=None), dict(g=None), dict(g=tensor(3 * MB, rows=9)), dict(g=tensor(3 * MB, dtype=BF16)),
    dict(gs=tensor(4 * MB, feat=32)), dict(w=None), dict(w=tensor(2 * MB, rows=2)), dict(dx=tensor(5 * MB, rows=1)),
    dict(dw=tensor(6 * MB, rows=1, feat=32)), dict(dw=tensor(6 * MB, rows=1, dtype=BF16)), dict(eps=-1.0),
    dict(work=8 * MB + 128),
    dict(dx=tensor(MB + 4)), dict(dx=tensor(3 * MB - 4)), dict(dx=tensor(4 * MB + ROW)), dict(dx=tensor(2 * MB)),
    dict(dx=tensor(6 * MB)), dict(dx=tensor(8 * MB)), dict(dw=tensor(MB, rows=1)), dict(dw=tensor(3 * MB, rows=1)),
    dict(dw=tensor(4 * MB, rows=1)), dict(dw=tensor(2 * MB, rows=1)), dict(dw=tensor(8 * MB, rows=1)),
    dict(work=MB), dict(work=3 * MB), dict(work=4 * MB), dict(work=2 * MB),
])
def test_add_norm_backward(lib, change):
    assert refused(lib, backward(lib, **change))


def test_add_norm_backward_asks_for_its_work(lib):
    need = ctypes.c_size_t(0)
    assert lib.node_add_norm_work_bytes(BACK["h"], ctypes.byref(need)) == gnnk.OK and need.value >= 256
    assert backward(lib, work=None) == gnnk.ENOMEM
    assert backward(lib, bytes=need.value - 1) == gnnk.ENOMEM and b"work" in lib.gnnk_last_error()
    sizes = []
    for rows in (0, 1, 100, 10**4, 10**6, 10**8):
        assert lib.node_add_norm_work_bytes(tensor(0, rows=rows, feat=128), ctypes.byref(need)) == gnnk.OK
        sizes.append(need.value)
    assert sizes == sorted(sizes) and sizes[-1] < 10**8 * 128 * 4 // 15  # a row of sums for 16 rows
    assert lib.node_add_norm_work_bytes(None, ctypes.byref(need)) == gnnk.EINVAL
    assert lib.node_add_norm_work_bytes(BACK["h"], None) == gnnk.EINVAL
    assert lib.node_add_norm_work_bytes(tensor(0, feat=16385), ctypes.byref(need)) == gnnk.EINVAL


def test_weight8(lib):
    need = ctypes.c_size_t(0)
    for outs, cols, size in ((1, 1, 8192), (64, 128, 8192), (65, 128, 16384), (64, 129, 16384),
                             (1 << 24, 65536, (1 << 24) * 65536)):
        assert lib.weight8_bytes(outs, cols, ctypes.byref(need)) == gnnk.OK and need.value == size
    for outs, cols in ((0, 1), (1, 0), (-1, 5), ((1 << 24) + 1, 1), (1, 65537)):
        assert lib.weight8_bytes(outs, cols, ctypes.byref(need)) == gnnk.EINVAL and need.value == 0
    assert lib.weight8_bytes(1, 1, None) == gnnk.EINVAL
    w = rows8(MB, scale=0, rows=96, cols=64)
    assert lib.weight8_pack(None, 8 * MB, MB, None) == gnnk.EINVAL
    assert lib.weight8_pack(rows8(MB, rows=0), 8 * MB, MB, None) == gnnk.EINVAL
    assert lib.weight8_pack(w, None, MB, None) == gnnk.ENOMEM
    assert lib.weight8_pack(w, 8 * MB, 2 * 8192 - 1, None) == gnnk.ENOMEM
    assert lib.weight8_pack(w, 8 * MB + 64, MB, None) == gnnk.EINVAL
    assert lib.weight8_pack(w, MB, MB, None) == gnnk.EINVAL and b"overlap" in lib.gnnk_last_error()


LINEAR = dict(x=rows8(MB, 2 * MB), w=weight8(), b=tensor(3 * MB, rows=1, feat=96), out=tensor(4 * MB, feat=96))


@pytest.mark.parametrize("change", [
    dict(x=None), dict(x=rows8(0)), dict(x=rows8(MB, scale=0)), dict(x=rows8(MB, rows=9)), dict(x=rows8(MB, cols=65)),
    dict(x=rows8(MB, stride=63)), dict(x=rows8(MB, cols=65537), w=weight8(cols=65537)),
    dict(w=None), dict(w=weight8(packed=0)), dict(w=weight8(packed=32 * MB + 16)), dict(w=weight8(scale=0)),
    dict(w=weight8(outs=0)), dict(w=weight8(outs=-5)), dict(w=weight8(cols=128)),
    dict(b=tensor(3 * MB, rows=1, feat=95)), dict(b=tensor(3 * MB, rows=1, feat=96, dtype=BF16)),
    dict(b=tensor(3 * MB, rows=2, feat=96)),
    dict(out=None), dict(out=tensor(4 * MB, feat=95)), dict(out=tensor(4 * MB, rows=9, feat=96)),
    dict(out=tensor(4 * MB, feat=96, stride=95)), dict(out=tensor(4 * MB, feat=96, dtype=3)),
    dict(out=tensor(MB, feat=96)), dict(out=tensor(2 * MB + 36, feat=96)), dict(out=tensor(3 * MB - 8, feat=96)),
    dict(out=tensor(32 * MB + 2 * 8192 - 4, feat=96)), dict(out=tensor(48 * MB, feat=96)),
])
def test_linear_i8(lib, change):
    a = dict(LINEAR, **change)
    assert refused(lib, lib.node_linear_i8(a["x"], a["w"], a["b"], a["out"], None))


def test_option(lib):
    assert lib.gnnk_set_option(b"linear8_tile", -1) == gnnk.EINVAL
    assert lib.gnnk_set_option(b"linear8_tile", 100) == gnnk.EINVAL
    assert lib.gnnk_set_option(b"linear8_tile", 0) == gnnk.OK


def test_binding():
    x, w, q, s = torch.zeros(3, 8), torch.ones(8), torch.zeros((3, 8), dtype=torch.int8), torch.zeros(3)
    for call in (lambda: gnnk.node_add_norm(x, x, w), lambda: gnnk.node_add_norm_i8(x, x, w),
                 lambda: gnnk.node_quantize(x), lambda: gnnk.node_add_norm_backward(x, w, x),
                 lambda: gnnk.Weight8(q, s), lambda: gnnk.Weight8.quantize(x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="heads, feat"):
        gnnk.node_quantize(w)
