"""Dot-product attention over edges and its gradients in 64 bits, with bounds
of what the operators' 32-bit arithmetic may differ by (u = 2^-24)."""
import torch

from _heads import U32


class Reference:
    """Everything per edge and head; src and dst are CPU int64 tensors."""

    def __init__(self, src, dst, n_src, n_dst, q, k, v, bias=None, scale=None, dz=None):
        H, F = q.shape[1], q.shape[2]
        K = k.shape[1]
        self.scale = scale = F ** -0.5 if scale is None else scale
        of = torch.arange(H) // (H // K)
        q, k, v = q.double().cpu(), k.double().cpu()[:, of], v.double().cpu()[:, of]
        E = src.numel()
        seg = lambda x, at, n: torch.zeros((n,) + x.shape[1:], dtype=torch.float64).index_add_(0, at, x)
        terms = q[dst] * k[src] * scale
        s, size = terms.sum(-1), terms.abs().sum(-1)
        b = torch.zeros(E, H, dtype=torch.float64)
        if bias is not None:
            b = bias.double().cpu()[:, :, 0].expand(E, H)
            s = torch.where(b == -torch.inf, b, s + b)
        top = torch.full((n_dst, H), -torch.inf, dtype=torch.float64)
        top = top.scatter_reduce(0, dst.view(-1, 1).expand(E, H), s, "amax") if E else top
        self.live = top > -torch.inf
        top = torch.where(self.live, top, 0.0)
        w = torch.exp(s - top[dst])
        total = seg(w, dst, n_dst)
        a = w / torch.where(total == 0, 1.0, total)[dst]
        self.top, self.total = top, total
        gone = (a == 0).unsqueeze(-1)
        kv = torch.where(gone, 0.0, k[src])
        vv = torch.where(gone, 0.0, v[src])
        self.out = seg(a.unsqueeze(-1) * vv, dst, n_dst)
        # a score: 18 u of its terms (the scaled query 2, the products' sum at
        # most 15), 3 u of the bias, 3 u of itself and of its distance to the
        # maximum; an exponential 2 u more.  A row's sums over n edges in fp32:
        # one rounding an edge and one a batch of four where the maximum grew,
        # and 20 for the joins and the division
        n = torch.bincount(dst, minlength=n_dst).double().view(-1, 1)
        finite = lambda x: torch.where(torch.isfinite(x), x, 0.0)
        es = U32 * (18 * finite(size) + 3 * finite(b).abs() + 3 * finite(s).abs() + finite(s - top[dst]).abs() + 2)
        es = torch.where(gone[..., 0], 0.0, es)
        row = U32 * (1.25 * n + 20)
        worst = torch.zeros((n_dst, H), dtype=torch.float64)
        worst = worst.scatter_reduce(0, dst.view(-1, 1).expand(E, H), es, "amax") if E else worst
        ea = worst + row          # relative, of a weight or of a sum of weights
        # a weight below the smallest normal number becomes 0: off by that
        # number at most, whatever its size
        tiny = torch.where(a > 0, torch.finfo(torch.float32).tiny, 0.0)
        self.out_bound = 2 * ea.unsqueeze(-1) * seg(a.unsqueeze(-1) * vv.abs(), dst, n_dst) \
            + seg(tiny.unsqueeze(-1) * vv.abs(), dst, n_dst)
        self.stats_bound = 2 * ea
        if dz is None:
            return
        z = dz.double().cpu()
        da, dsize = (z[dst] * vv).sum(-1), (z[dst] * vv).abs().sum(-1)
        S, Ssize = seg(a * da, dst, n_dst), seg(a * dsize, dst, n_dst)
        ds = a * (da - S[dst])
        # a gradient of a score: its weight off by ea, da by 15 u of its terms,
        # S by both; and the rounding of the sums
        eds = (a * (3 * ea[dst] + 40 * U32) + tiny) * (dsize + Ssize[dst])
        out_n = torch.bincount(src, minlength=n_src).double().view(-1, 1, 1) * (H // K)
        col = U32 * (out_n + 20)
        self.dq = scale * seg(ds.unsqueeze(-1) * kv, dst, n_dst)
        # (the kernel sums a (da - S0) k and delta a k apart: both at most a
        # (|da| + |S|) |k|, one rounding an edge)
        asize = a * (dsize + Ssize[dst])
        self.dq_bound = abs(scale) * (seg(eds.unsqueeze(-1) * kv.abs(), dst, n_dst)
                                 + 2 * row.unsqueeze(-1) * seg(asize.unsqueeze(-1) * kv.abs(), dst, n_dst))
        shared = lambda x: x.view(x.shape[0], K, H // K, F).sum(2)
        gq, gz = torch.where(gone, 0.0, q[dst]), torch.where(gone, 0.0, z[dst])
        self.dk = scale * shared(seg(ds.unsqueeze(-1) * gq, src, n_src))
        self.dk_bound = abs(scale) * shared(seg(eds.unsqueeze(-1) * gq.abs(), src, n_src)) \
            + abs(scale) * col * shared(seg(ds.abs().unsqueeze(-1) * gq.abs(), src, n_src))
        self.dv = shared(seg(a.unsqueeze(-1) * gz, src, n_src))
        sum_v = shared(seg((a * ea[dst] + tiny).unsqueeze(-1) * gz.abs(), src, n_src))
        self.dv_bound = 2 * sum_v + col * shared(seg(a.unsqueeze(-1) * gz.abs(), src, n_src))
        self.dbias = ds.unsqueeze(-1)
        self.dbias_bound = eds.unsqueeze(-1)
        if bias is not None and bias.shape[1] == 1 and H > 1:
            self.dbias = self.dbias.sum(1, keepdim=True)
            self.dbias_bound = self.dbias_bound.sum(1, keepdim=True) \
                + U32 * (H + 8) * ds.abs().sum(1).view(-1, 1, 1)
