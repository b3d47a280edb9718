"""What the attention operators refuse, on the host before anything is
launched (CPU only: the tensors' addresses are never used)."""
import ctypes

import pytest
import torch

from paper_1909_01315_amd import gnnk, nn

F32, BF16 = gnnk.F32, gnnk.BF16


@pytest.fixture(scope="module")
def lib():
    return gnnk.load()


def tensor(rows, heads, feat, dtype=F32, stride=None, data=4096):
    return gnnk._TENSOR.pack(data, rows, heads, feat, heads * feat if stride is None else stride, dtype, 0)


def rotary(rows, pairs, axes=None, stride=None, pos=4096, freq=4096, kind=0, interleaved=0):
    axes = len(pairs) if axes is None else axes
    pairs = tuple(pairs) + (0,) * (4 - len(pairs))
    return gnnk._ROTARY.pack(pos, rows, axes if stride is None else stride, freq, kind, axes,
                             *(p & 0xFFFFFFFF for p in pairs), interleaved, 0)


X = dict(rows=10, heads=4, feat=16)


@pytest.mark.parametrize("rot,x,out", [
    (None, tensor(**X), tensor(**X)),
    (rotary(10, (8,)), None, tensor(**X)),
    (rotary(10, (8,)), tensor(**X), None),
    (rotary(9, (8,)), tensor(**X), tensor(**X)),                       # positions of other rows
    (rotary(10, (9,)), tensor(**X), tensor(**X)),                      # more pairs than columns hold
    (rotary(10, (0, 0)), tensor(**X), tensor(**X)),                    # none
    (rotary(10, (-1, 3)), tensor(**X), tensor(**X)),
    (rotary(10, (4, 4), axes=0), tensor(**X), tensor(**X)),
    (rotary(10, (2, 2, 2, 2), axes=5), tensor(**X), tensor(**X)),
    (rotary(10, (4, 4), stride=1), tensor(**X), tensor(**X)),
    (rotary(10, (4, 4), kind=2), tensor(**X), tensor(**X)),
    (rotary(10, (4, 4), pos=0), tensor(**X), tensor(**X)),
    (rotary(10, (4, 4), freq=0), tensor(**X), tensor(**X)),
    (rotary(10, (8,)), tensor(**X), tensor(10, 4, 8)),
    (rotary(10, (8,)), tensor(**X), tensor(**X, dtype=BF16)),
    (rotary(10, (8,)), tensor(**X, stride=63), tensor(**X)),
    (rotary(10, (8,)), tensor(10, 4, 2049), tensor(10, 4, 2049)),
    (rotary(10, (8,)), tensor(10, 1025, 16), tensor(10, 1025, 16)),
    (rotary(1 << 31, (8,)), tensor(1 << 31, 4, 16), tensor(1 << 31, 4, 16)),
])
def test_rotary(lib, rot, x, out):
    assert lib.node_rotary(rot, x, 0, out, None) == gnnk.EINVAL
    assert lib.gnnk_last_error()


NORM = dict(q=tensor(**X), wq=tensor(1, 1, 16), rq=rotary(10, (8,)), oq=tensor(**X), k=tensor(20, 2, 16),
            wk=tensor(1, 2, 16), rk=rotary(20, (8,)), ok=tensor(20, 2, 16), eps=1e-6)


@pytest.mark.parametrize("change", [
    dict(q=None), dict(oq=None), dict(ok=None),
    dict(oq=tensor(10, 4, 8)), dict(ok=tensor(10, 2, 16)), dict(ok=tensor(20, 2, 16, BF16)),
    dict(wq=tensor(1, 2, 16)), dict(wq=tensor(2, 1, 16)), dict(wk=tensor(1, 2, 8)), dict(wq=tensor(1, 1, 16, BF16)),
    dict(k=tensor(20, 2, 8), wk=None, ok=tensor(20, 2, 8)),            # heads of another width
    dict(k=tensor(20, 2, 16, BF16), wk=None, ok=tensor(20, 2, 16, BF16)),
    dict(rq=None), dict(rk=None),                                      # one of them turned
    dict(rk=rotary(20, (4, 4))), dict(rk=rotary(20, (7,))), dict(rk=rotary(20, (8,), interleaved=1)),
    dict(rk=rotary(10, (8,))),
    dict(eps=-1.0), dict(eps=float("nan")),
])
def test_norm_rotary(lib, change):
    a = dict(NORM, **change)
    assert lib.node_norm_rotary(a["q"], a["wq"], a["rq"], a["oq"], a["k"], a["wk"], a["rk"], a["ok"], a["eps"],
                                None) == gnnk.EINVAL
    assert lib.gnnk_last_error()


BACK = dict(NORM, gq=tensor(**X), dq=tensor(**X), dwq=tensor(1, 1, 16), gk=tensor(20, 2, 16), dk=tensor(20, 2, 16),
            dwk=tensor(1, 2, 16), work=4096, bytes=1 << 30)


def backward(lib, **change):
    a = dict(BACK, **change)
    return lib.node_norm_rotary_backward(a["q"], a["wq"], a["rq"], a["gq"], a["dq"], a["dwq"], a["k"], a["wk"],
                                         a["rk"], a["gk"], a["dk"], a["dwk"], a["eps"], a["work"], a["bytes"], None)


@pytest.mark.parametrize("change", [
    dict(gq=None), dict(gk=None), dict(gq=tensor(10, 4, 8)), dict(gk=tensor(20, 2, 16, BF16)),
    dict(dq=tensor(10, 2, 16)), dict(dk=tensor(20, 2, 16, BF16)), dict(dwq=tensor(1, 4, 16)),
    dict(dwk=tensor(1, 1, 16)), dict(wq=None),                         # a gradient of no weight
    dict(work=4097),
])
def test_norm_rotary_backward(lib, change):
    assert backward(lib, **change) == gnnk.EINVAL


def test_norm_rotary_backward_asks_for_its_work(lib):
    need = ctypes.c_size_t(0)
    assert lib.node_norm_rotary_work_bytes(BACK["q"], BACK["wq"], BACK["k"], BACK["wk"], ctypes.byref(need)) == gnnk.OK
    assert need.value > 0
    assert backward(lib, work=None) == gnnk.ENOMEM
    assert backward(lib, bytes=64) == gnnk.ENOMEM and b"work" in lib.gnnk_last_error()
    none = ctypes.c_size_t(7)
    assert lib.node_norm_rotary_work_bytes(BACK["q"], None, BACK["k"], None, ctypes.byref(none)) == gnnk.OK
    assert none.value == 0
    # more rows never need less, and past the blocks that share them no more
    sizes = []
    for rows in (0, 1, 100, 10**4, 10**6, 10**9):
        t = tensor(rows, 8, 128)
        assert lib.node_norm_rotary_work_bytes(t, t, None, None, ctypes.byref(need)) == gnnk.OK
        sizes.append(need.value)
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-3]
    assert lib.node_norm_rotary_work_bytes(None, None, None, None, ctypes.byref(need)) == gnnk.EINVAL
    assert lib.node_norm_rotary_work_bytes(BACK["q"], BACK["wq"], None, None, None) == gnnk.EINVAL
    assert lib.node_norm_rotary_work_bytes(tensor(10, 2000, 16), BACK["wq"], None, None,
                                           ctypes.byref(need)) == gnnk.EINVAL


def test_dot_aggregate_without_a_graph(lib):
    t = tensor(**X)
    assert lib.dot_aggregate(None, t, t, t, None, 1.0, t, None, None) == gnnk.EINVAL
    assert b"NULL graph" in lib.gnnk_last_error()
    assert lib.dot_aggregate_backward(None, t, t, t, None, 1.0, t, t, t, t, t, t, None, None) == gnnk.EINVAL


def test_binding():
    x, w = torch.zeros(3, 2, 8), torch.ones(8)
    with pytest.raises(ValueError, match="GPU"):
        gnnk.node_norm_rotary(x, w)
    with pytest.raises(ValueError, match="GPU"):
        gnnk.Rotary(torch.ones(4), (4,))
    for pairs in ((), (1, 1, 1, 1, 1), (0,), (-1, 2)):
        with pytest.raises(ValueError, match="pairs"):
            gnnk.Rotary(torch.ones(4), pairs)
    pos = torch.zeros(3, 2, requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        nn.norm_rotary(x, w, x, w, None, pos, pos)
    with pytest.raises(ValueError, match="gradient"):
        nn.rotary(None, x, pos)
    with pytest.raises(ValueError, match="divide"):
        nn.DotAttentionConv(8, 8, 4, kv_heads=3)
    with pytest.raises(ValueError, match="pairs"):
        nn.DotAttentionConv(8, 8, 4, axis_pairs=(3, 2))


def test_layer_parameters():
    layer = nn.DotAttentionConv(12, 8, 4, kv_heads=2, axis_pairs=(2, 1))
    shapes = {n: tuple(p.shape) for n, p in layer.named_parameters()}
    assert shapes == {"norm_q": (8,), "norm_k": (8,), "fc_q.weight": (32, 12), "fc_k.weight": (16, 12),
                      "fc_v.weight": (16, 12)}
    assert nn.DotAttentionConv(12, 8, 4, qk_norm=False).norm_q is None
