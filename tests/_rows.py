"""Plain 64-bit forms of the operators on whole rows (the residual stream's sum
and norm, rows and products in 8 bits) and what 32-bit arithmetic may differ by.

u = 2^-24 is half a step of fp32.
"""
import torch

from _heads import U32

F32, BF16 = torch.float32, torch.bfloat16

# Roundings of 1 / sqrt(mean(h^2) + eps): h is off by 1 (2 of its square), the
# sum of squares takes at most 46 (32 terms a lane, 6 steps across lanes, 8
# wavefronts), the mean and eps 3, all halved by the root; the root and the
# division 1 each
R_U = 28


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g).to(dtype)


def spread(t, pad, lead=None):
    """t (rows, columns) on the GPU in rows of a stride `pad` columns larger, off 16-byte alignment for an odd lead"""
    if pad == 0:
        return t.cuda()
    lead = pad // 2 if lead is None else lead
    n, c = t.shape
    buf = torch.full((n, c + pad), float("nan") if t.dtype.is_floating_point else 101, dtype=t.dtype, device="cuda")
    v = buf[:, lead: lead + c]
    v.copy_(t)
    return v


def norm(h, w, eps):
    """(y, its bound) of 64-bit rows h and weights w (or None): h's own rounding, the root's, the product of
    weight and root, and the last one"""
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    y = h * r if w is None else h * r * w
    return y, (R_U + 4) * U32 * y.abs()


def norm_gradients(h, w, g, gs, eps):
    """(dx, bound, terms of dw, their bound) at rows h, which a call reads as they are"""
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    gw = g * w if w is not None else g
    dx = r * (gw - h * r * r * (gw * h).mean(1, keepdim=True))
    # gw: 1 u, the sum of its products with h 47; r^2, the mean and their product 60; the product with h, the
    # difference and the product with r 31; the sum with gs 1 of both
    m = r * r * (gw * h).abs().mean(1, keepdim=True)
    bound = U32 * r * (34 * gw.abs() + 141 * h.abs() * m)
    if gs is not None:
        dx, bound = dx + gs, bound + U32 * gs.abs()
    # h r: R_U + 1 u; 32 sums in fp32, the product in the first; the tile's rounding and the last one
    return dx, bound, g * h * r, (R_U + 36) * U32 * (g * h * r).abs()


def check_rows8(q, scale, y, bound, what):
    """q and scale stand for rows y, known to within bound"""
    q, s = q.cpu().double(), scale.cpu().double()
    most, off = y.abs().amax(1), bound.amax(1)
    # the scale: the largest magnitude's bound, and the division's rounding
    assert bool(((s - most / 127).abs() <= (off + U32 * most) / 127 + 2.0 ** -126).all()), f"{what}: scale"
    assert bool((q.abs() <= 127).all())
    # half a step, and what the values, the scale, its inverse and the product are off by
    tol = 0.5 * s + 2 * off + 4 * U32 * most
    bad = ((q * s.unsqueeze(1) - y).abs() > tol.unsqueeze(1)).sum()
    assert int(bad) == 0, f"{what}: {int(bad)} values off by more than half a step"
    big = most > 2.0 ** -118
    assert bool((q.abs().amax(1)[big] == 127).all()), f"{what}: a row's largest magnitude is 127 steps"


def product(q, s, wq, ws, bias):
    """(out, bound) of 8-bit rows and weight, on the CPU: the sum in fp32, two products, the bias"""
    v = (q.cpu().double() @ wq.cpu().double().t()) * s.cpu().double().view(-1, 1) * ws.cpu().double().view(1, -1)
    b = 0.0 if bias is None else bias.cpu().double().view(1, -1)
    return v + b, U32 * (4 * v.abs() + torch.as_tensor(b).abs())
