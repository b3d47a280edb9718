"""Plain 64-bit forms of the operators on queries and keys, and the bounds of
what 32-bit arithmetic and one rounding to the output type may differ by.

u = 2^-24 is half a step of fp32.  A result of n roundings, each relative to
the terms it combines, is off by at most n u times the sum of their sizes.
"""
import numpy as np
import torch

U32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def angles(pos, freq, pairs):
    """(rows, 1, P) in 64 bits"""
    axis = np.repeat(np.arange(len(pairs)), pairs)
    return (pos.double().cpu()[:, axis] * freq.double().cpu()).unsqueeze(1)


def split(x, P, interleaved):
    if interleaved:
        return x[..., 0:2 * P:2], x[..., 1:2 * P:2]
    return x[..., :P], x[..., P:2 * P]


def join(a, b, rest, interleaved):
    head = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([head, rest], -1)


def turn(x, theta, interleaved, inverse=False):
    P = theta.shape[-1]
    a, b = split(x, P, interleaved)
    c, s = torch.cos(theta), torch.sin(theta) * (-1.0 if inverse else 1.0)
    return join(a * c - b * s, a * s + b * c, x[..., 2 * P:], interleaved)


def pair_size(x, P, interleaved):
    """|a| + |b| at both columns of a pair, |x| at the others"""
    a, b = split(x.abs(), P, interleaved)
    return join(a + b, a + b, x[..., 2 * P:].abs(), interleaved)


# A turned value: its cosine and sine are off by 2 steps of fp32 (4 u, their
# own rounding) and by the rounding of the angle in half turns, u / 2 * pi <
# 2 u; two products and a sum round once each (3 u).  9 u of |a| + |b|.
TURN_U = 9


def close(got, ref, bound, what):
    """got within bound (of its value in 32 bits) and one rounding to its type
    of ref; the smallest normal number covers what underflows"""
    r = half_step(got.dtype)
    g = got.detach().double().cpu().reshape(ref.shape)
    tol = bound * (1 + r) + r * ref.abs() + torch.finfo(torch.float32).tiny
    same_nan = torch.isnan(g) & torch.isnan(ref)
    bad = ~(((g - ref).abs() <= tol) | same_nan)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst "
                                 f"{float(((g - ref).abs() / tol)[bad].nan_to_num(1e30).max()):.3g} of the bound")
