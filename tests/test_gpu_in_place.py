"""Rotations and norms in place: the output is the operand itself, in whole
rows and in wider ones, and the values are those of a call into another
tensor.  (Other overlaps are refused: tests/test_overlap_refusals.py.)"""
import pytest
import torch

from paper_1909_01315_amd import gnnk

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rows(g, n, H, F, dtype, pad=0):
    """(n, H, F) in rows of a stride `pad` columns larger, and the whole buffer"""
    buf = torch.randn((n, H * F + pad), generator=g).to(dtype).cuda()
    return buf[:, pad // 2: pad // 2 + H * F].unflatten(1, (H, F)), buf


def turned(n, pairs, il, g):
    pos = (torch.randn((n, len(pairs)), generator=g) * 20).cuda()
    return gnnk.Rotary.geometric(pairs, interleaved=il), pos


SHAPES = [(1, 1, 2, (1,)), (5000, 8, 32, (6, 5, 5)), (3000, 3, 47, (10, 13)), (300, 2, 256, (64, 64)),
          (700, 5, 23, (3,))]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("n,H,F,pairs", SHAPES + [(40, 2, 1030, (300, 200)), (20, 1, 2048, (1024,))])
def test_rotation(n, H, F, pairs, pad, il, dtype):
    g = torch.Generator().manual_seed(n)
    rot, pos = turned(n, pairs, il, g)
    x, buf = rows(g, n, H, F, dtype, pad)
    want, around = gnnk.node_rotary(rot, x, pos), buf.clone()
    assert gnnk.node_rotary(rot, x, pos, out=x) is x
    assert torch.equal(x, want)
    around[:, pad // 2: pad // 2 + H * F] = want.flatten(1)
    assert torch.equal(buf, around), "nothing beside the columns"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("n,H,F,pairs", SHAPES)
def test_norms_and_gradients(n, H, F, pairs, pad, dtype):
    g = torch.Generator().manual_seed(n)
    rot, pos = turned(n, pairs, False, g)
    q, k, zq, zk = (rows(g, n, h, F, dtype, pad)[0] for h in (H, 2, H, 2))
    w = torch.randn(F, generator=g).to(dtype).cuda()
    args = dict(rot=rot, pos_q=pos, pos_k=pos)
    want = gnnk.node_norm_rotary(q, w, k, w, **args)
    grads = gnnk.node_norm_rotary_backward(q, w, zq, k, w, zk, **args)
    # the gradients into the outputs' gradients, then into the operands
    d, w3, r = gnnk._desc, w.view(1, 1, F), rot._desc(pos)
    work = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    for into in ((zq, zk), (q, k)):
        keep = [t.clone() for t in (q, zq, k, zk)]
        dw = [torch.empty_like(w3) for _ in range(2)]
        gnnk._check(gnnk.load().node_norm_rotary_backward(
            d(q), d(w3), r, d(zq), d(into[0]), d(dw[0]), d(k), d(w3), r, d(zk), d(into[1]), d(dw[1]), 1e-6,
            work.data_ptr(), work.numel(), gnnk._stream()))
        for got, ref in zip((into[0], dw[0].view(F), into[1], dw[1].view(F)), grads):
            assert torch.equal(got, ref)
        for t, old in zip((q, zq, k, zk), keep):
            t.copy_(old)
    oq, ok = gnnk.node_norm_rotary(q, w, k, w, out_q=q, out_k=k, **args)
    assert oq is q and ok is k and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_heads_of_several_blocks_are_refused():
    x = torch.ones(3, 1, 2048, device="cuda")
    with pytest.raises(gnnk.GnnkError) as err:
        gnnk.node_norm_rotary(x, out_q=x)
    assert err.value.status == gnnk.EINVAL
    assert bool((x == 1).all())


def test_parts_of_one_buffer_side_by_side():
    """Operands and outputs in alternate columns of one buffer do not overlap."""
    n, H, F = 500, 4, 16
    g = torch.Generator().manual_seed(3)
    x = torch.randn((n, H, F), generator=g).cuda()
    rot, pos = turned(n, (8,), False, g)
    buf = torch.zeros((n, 3 * H * F), device="cuda")
    q, out_q, out_k = (buf[:, i * H * F: (i + 1) * H * F].unflatten(1, (H, F)) for i in range(3))
    q.copy_(x)
    gnnk.node_norm_rotary(q, None, q, None, rot=rot, pos_q=pos, pos_k=pos, out_q=out_q, out_k=out_k)
    want = gnnk.node_norm_rotary(x, rot=rot, pos_q=pos)
    assert torch.equal(out_q, want) and torch.equal(out_k, want) and torch.equal(q, x)
