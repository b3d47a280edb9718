"""Outputs of the operators on queries and keys that overlap what the call
reads or another output are refused on the host (CPU only: the tensors'
addresses are never used); the exact operand is allowed where it is safe
(tests/test_gpu_in_place.py)."""
import pytest

from paper_1909_01315_amd import gnnk

F32, BF16 = gnnk.F32, gnnk.BF16
MB = 1 << 20


def tensor(at, rows=10, heads=4, feat=16, dtype=F32, stride=None):
    return gnnk._TENSOR.pack(at, rows, heads, feat, heads * feat if stride is None else stride, dtype, 0)


def rotary(at, rows=10, pairs=8, freq=64 * MB):
    return gnnk._ROTARY.pack(at, rows, 1, freq, 0, 1, pairs, 0, 0, 0, 0, 0)


@pytest.fixture(scope="module")
def lib():
    return gnnk.load()


ROW = 4 * 16 * 4  # bytes of a row


@pytest.mark.parametrize("x,out,pos,freq", [
    (tensor(MB), tensor(MB + ROW), 32 * MB, 64 * MB),               # a row further
    (tensor(MB), tensor(MB - 4), 32 * MB, 64 * MB),                 # a column before
    (tensor(MB), tensor(MB, stride=80), 32 * MB, 64 * MB),          # the same start in wider rows
    (tensor(MB, stride=100), tensor(MB + 63 * 4, stride=100), 32 * MB, 64 * MB),  # one column shared
    (tensor(MB, stride=100), tensor(MB - 63 * 4, stride=100), 32 * MB, 64 * MB),
    (tensor(MB, stride=100), tensor(MB + 37 * 4, stride=100), 32 * MB, 64 * MB),  # wraps into the next row
    (tensor(MB), tensor(2 * MB), 2 * MB + 4, 64 * MB),              # the positions
    (tensor(MB), tensor(2 * MB), 32 * MB, 2 * MB + 10 * ROW - 4),   # the last frequency's first
])
def test_rotary(lib, x, out, pos, freq):
    assert lib.node_rotary(rotary(pos, freq=freq), x, 0, out, None) == gnnk.EINVAL
    assert b"overlap" in lib.gnnk_last_error()


Q, K = dict(rows=10, heads=4, feat=16), dict(rows=20, heads=2, feat=16)
NORM = dict(q=tensor(MB, **Q), wq=tensor(2 * MB, 1, 1, 16), rq=rotary(3 * MB), oq=tensor(4 * MB, **Q),
            k=tensor(5 * MB, **K), wk=tensor(6 * MB, 1, 2, 16), rk=rotary(7 * MB, 20), ok=tensor(8 * MB, **K))


def wide(at, feat, dtype=F32, rows=3):
    return tensor(at, rows, 1, feat, dtype)


@pytest.mark.parametrize("change", [
    dict(oq=tensor(MB + 4, **Q)), dict(oq=tensor(2 * MB, **Q)), dict(oq=tensor(5 * MB, **Q)),
    dict(oq=tensor(6 * MB, **Q)), dict(oq=tensor(3 * MB, **Q)), dict(oq=tensor(8 * MB + 8, **Q)),
    dict(ok=tensor(MB, **K)), dict(ok=tensor(4 * MB, **K)), dict(ok=tensor(5 * MB - 4, **K)),
    dict(k=tensor(MB, **Q), wk=None, ok=tensor(8 * MB, **Q), rk=rotary(3 * MB), oq=tensor(MB, **Q)),  # k is q
    # in place, in heads that one wavefront does not hold: other blocks still read them
    dict(q=wide(MB, 2048), oq=wide(MB, 2048), wq=None, rq=None, k=None),
    dict(q=wide(MB, 600), oq=wide(MB, 600), wq=None, rq=None, k=None),
    dict(q=wide(MB, 1032, BF16), oq=wide(MB, 1032, BF16), wq=None, rq=None, k=None),
])
def test_norm_rotary(lib, change):
    a = dict(NORM, **change)
    assert lib.node_norm_rotary(a["q"], a["wq"], a["rq"], a["oq"], a["k"], a["wk"], a["rk"], a["ok"], 1e-6,
                                None) == gnnk.EINVAL
    assert b"overlap" in lib.gnnk_last_error()


BACK = dict(NORM, gq=tensor(9 * MB, **Q), dq=tensor(10 * MB, **Q), dwq=tensor(11 * MB, 1, 1, 16),
            gk=tensor(12 * MB, **K), dk=tensor(13 * MB, **K), dwk=tensor(14 * MB, 1, 2, 16))


@pytest.mark.parametrize("change", [
    dict(dq=tensor(9 * MB + 4, **Q)), dict(dq=tensor(12 * MB, **Q)), dict(dq=tensor(13 * MB + 256, **Q)),
    dict(dq=tensor(5 * MB, **Q)), dict(dk=tensor(9 * MB, **K)), dict(dwq=tensor(2 * MB, 1, 1, 16)),
    dict(dwq=tensor(14 * MB + 64, 1, 1, 16)), dict(dwk=tensor(MB, 1, 2, 16)), dict(dwk=tensor(10 * MB, 1, 2, 16)),
    dict(q=wide(MB, 600), gq=wide(9 * MB, 600), dq=wide(9 * MB, 600), wq=None, dwq=None, rq=None, k=None, wk=None,
         dwk=None, dk=None, gk=None),
])
def test_norm_rotary_backward(lib, change):
    a = dict(BACK, **change)
    assert lib.node_norm_rotary_backward(a["q"], a["wq"], a["rq"], a["gq"], a["dq"], a["dwq"], a["k"], a["wk"],
                                         a["rk"], a["gk"], a["dk"], a["dwk"], 1e-6, 128 * MB, 64 * MB,
                                         None) == gnnk.EINVAL
    assert b"overlap" in lib.gnnk_last_error()
