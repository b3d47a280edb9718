"""nn.DotAttentionConv is exactly the chain of its operators, each of which is
tested by itself against 64 bits: the forward and what the operators give
backward bit for bit, the dense products around them within the rounding of
fp32 sums; and what the attention's backward refuses."""
import pytest
import torch

from paper_1909_01315_amd import gnnk, nn
from _heads import U32

pytestmark = pytest.mark.gpu

F32 = torch.float32


def graph(n_src, n_dst, e, seed):
    g = torch.Generator().manual_seed(seed)
    src, dst = torch.randint(0, n_src, (e,), generator=g), torch.randint(0, n_dst, (e,), generator=g)
    return gnnk.Graph.from_coo(src.int().cuda(), dst.int().cuda(), n_src, n_dst), dst


def near_product(got, a, b, what):
    """got = a @ b in fp32: at most one rounding a term (and its product's) of the terms' sizes"""
    a, b = a.double().cpu(), b.double().cpu()
    bound = U32 * (a.shape[1] + 1) * (a.abs() @ b.abs())
    assert bool(((got.double().cpu() - a @ b).abs() <= bound).all()), what


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("H,K,F,pairs", [(4, 2, 20, (3, 4)), (8, 8, 16, (8,)), (6, 1, 47, None)])
def test_layer_is_the_chain(H, K, F, pairs, norm):
    gr, dst = graph(90, 60, 1500, 59)
    g = torch.Generator().manual_seed(61)
    torch.manual_seed(3)
    D = 24
    layer = nn.DotAttentionConv(D, F, H, kv_heads=K, qk_norm=norm, axis_pairs=pairs).cuda()
    x = torch.randn((90, D), generator=g).cuda().requires_grad_(True)
    pos = (torch.randn((90, len(pairs)), generator=g) * 10).cuda() if pairs else None
    b = torch.randn((1500, 1, 1), generator=g)
    b[dst % 7 == 1] = -torch.inf
    b = b.cuda().requires_grad_(True)
    c = torch.randn((60, H, F), generator=g).cuda()
    if norm:
        with torch.no_grad():
            layer.norm_q.add_(0.3 * torch.randn(F, generator=g).cuda())
            layer.norm_k.add_(0.3 * torch.randn(F, generator=g).cuda())
    out = layer(gr, x, pos, b)
    (out * c).sum().backward()

    with torch.no_grad():
        q0 = layer.fc_q(x[:60]).view(-1, H, F)
        k0, v = layer.fc_k(x).view(-1, K, F), layer.fc_v(x).view(-1, K, F)
        rot = layer.rotary(x.device)
        pq = pos[:60] if pairs else None
        q, k = q0, k0
        if norm:
            q, k = gnnk.node_norm_rotary(q0, layer.norm_q, k0, layer.norm_k, rot=rot, pos_q=pq, pos_k=pos,
                                         eps=layer.eps)
        elif rot is not None:
            q, k = gnnk.node_rotary(rot, q0, pq), gnnk.node_rotary(rot, k0, pos)
        want, stats = gnnk.dot_aggregate(gr, q, k, v, bias=b, want_stats=True)
        assert torch.equal(out, want)
        dq, dk, dv, db = gnnk.dot_aggregate_backward(gr, q, k, v, want, stats, c, bias=b)
        assert torch.equal(b.grad, db)
        if norm:
            dq, dwq, dk, dwk = gnnk.node_norm_rotary_backward(q0, layer.norm_q, dq, k0, layer.norm_k, dk, rot=rot,
                                                              pos_q=pq, pos_k=pos, eps=layer.eps)
            assert torch.equal(layer.norm_q.grad, dwq) and torch.equal(layer.norm_k.grad, dwk)
        elif rot is not None:
            dq, dk = gnnk.node_rotary(rot, dq, pq, inverse=True), gnnk.node_rotary(rot, dk, pos, inverse=True)
    flat = lambda t: t.flatten(1)
    near_product(q0.flatten(1), x[:60].detach(), layer.fc_q.weight.detach().T, "queries")
    for name, d, rows in (("fc_q", dq, 60), ("fc_k", dk, 90), ("fc_v", dv, 90)):
        near_product(getattr(layer, name).weight.grad, flat(d).T, x[:rows].detach(), name)
    # the three products' sum, those of the queries for the first rows only
    full = torch.cat([torch.nn.functional.pad(flat(dq), (0, 0, 0, 30)), flat(dk), flat(dv)], 1)
    weights = torch.cat([getattr(layer, n).weight.detach() for n in ("fc_q", "fc_k", "fc_v")])
    near_product(x.grad, full, weights, "dx")
    gr.destroy()


def test_backward_refuses_with_a_status():
    gr, _ = graph(70, 60, 900, 1)
    ones = lambda n, h, f, t=F32: torch.ones((n, h, f), dtype=t, device="cuda")
    q, k, v = ones(60, 4, 8), ones(70, 2, 8), ones(70, 2, 8)
    out, stats = gnnk.dot_aggregate(gr, q, k, v, want_stats=True)
    good = dict(out=out, stats=stats, grad_out=q)
    for bad in (dict(grad_out=ones(60, 4, 4)), dict(stats=None), dict(out=ones(60, 2, 8)),
                dict(stats=ones(60, 2, 2)), dict(stats=stats.bfloat16()), dict(grad_out=q.bfloat16()),
                dict(bias=ones(900, 2, 1)), dict(bias=ones(899, 4, 1))):
        with pytest.raises(gnnk.GnnkError) as err:
            gnnk.dot_aggregate_backward(gr, q, k, v, **{**good, **bad})
        assert err.value.status == gnnk.EINVAL, bad
    gr.destroy()
