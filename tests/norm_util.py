"""Plain references in 64 bits, on the CPU, of the operators in include/stem_norm.h, and the bounds that the GPU tests hold them to.

A rounding to a type is off by at most EPS[type] / 2 of the value, EPS = torch.finfo(type).eps; u = 2^-24 is that of fp32."""
import math

import torch

from decode_util import EPS, TINY, U


def halves(rot, layout):
    return (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))


def turned(x, positions, turns, factor, rot, layout, back=False):
    """x [T, H, d], 64 bits, turned by its positions (back: the transposed map), differentiably."""
    a = 2 * math.pi * torch.remainder(positions.double()[:, None] * turns, 1.0)
    c, s = factor * torch.cos(a)[:, None, :], factor * torch.sin(a)[:, None, :] * (-1 if back else 1)
    lo, hi = halves(rot, layout)
    first, second = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
    if layout == "half":
        return torch.cat([first, second, x[..., rot:]], dim=-1)
    return torch.cat([torch.stack([first, second], dim=-1).flatten(-2), x[..., rot:]], dim=-1)


def normed(x, weight, offset, eps):
    n = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + eps)
    return n if weight is None else n * (weight + offset)


def pair_sums(x, rot, layout):
    """|x1| + |x2| in the places of both, |x| behind the rotary part."""
    out = x.abs().clone()
    lo, hi = halves(rot, layout)
    out[..., lo] = out[..., hi] = x[..., lo].abs() + x[..., hi].abs()
    return out


def root_error(d):
    """Relative error of r: the squares' sum of d positive terms (d u), its division by a rounded d, eps, which is rounded, and the sum
    with it (4 u), half of that for the root, which itself is within 1 ulp (2 u)."""
    return ((d + 4) / 2 + 2) * U


def norm_reference(x, weight, offset, eps, positions, turns, factor, rot, layout):
    """(y, bound) of x [T, H, d] (any type, taken to 64 bits).

    n: r's error, that of the weight's sum with the offset (u of it), two products (u each).  c and s are off by 6 u f, two products and a
    sum round (3 u), as decode_util.rotary_reference has it: 9 u f (|n1| + |n2|).  Then the rounding to the type."""
    d = x.shape[-1]
    n = normed(x.double(), None if weight is None else weight.double(), offset, eps)
    y = turned(n, positions, turns, factor, rot, layout)
    rel = root_error(d) + 3 * U
    mags = pair_sums(n, rot, layout)
    fp32 = rel * mags
    fp32[..., :rot] = (rel + 9 * U) * abs(factor) * mags[..., :rot]
    fp32 = 1.01 * fp32
    return y, fp32 + EPS[x.dtype] / 2 * (y.abs() + fp32) + TINY[x.dtype]


def gradients(x, weight, offset, eps, positions, turns, factor, rot, layout, gy):
    """(dx, dweight) by autograd, in 64 bits."""
    x = x.double().requires_grad_()
    leaves = [x]
    if weight is not None:
        leaves.append(weight.double().requires_grad_())
    y = turned(normed(x, leaves[1] if weight is not None else None, offset, eps), positions, turns, factor, rot, layout)
    g = torch.autograd.grad(y, leaves, gy.double())
    return g[0], g[1] if weight is not None else None


def gradient_bounds(x, weight, offset, eps, positions, turns, factor, rot, layout, gy):
    """Bounds of the kernel's (dx, dweight).

    g = R^T dy is off by G = 9 u f (|dy1| + |dy2|) (0 behind the rotary part), u = x r by U1 = e + u relative, e that of r.  h = g w: G |w| and
    two roundings (2 u |h|).  m = mean(h u): mean((G |w| + (2 u + U1) |h|) |u|) and d + 3 roundings of sums of magnitudes.  dx = r (h - u m): the
    errors of h, of u and of m, two more roundings of the terms and one each of the difference and the product, e of the result.
    dweight: per term G |u| + (U1 + u) |g u|; a lane adds up at most 4 H (T / 4096, rounded up) terms in a row, a workgroup 64 lanes' or 4
    waves' sums, the rest is in 64 bits and rounds once."""
    T, H, d = x.shape
    x, gy64 = x.double(), gy.double()
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double() + offset
    r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + eps)
    u, e = x * r, root_error(d)
    g = turned(gy64, positions, turns, factor, rot, layout, back=True)
    G = 9 * U * abs(factor) * pair_sums(gy64, rot, layout)
    G[..., rot:] = 0
    h = g * w
    eh = G * w.abs() + 2 * U * h.abs()
    eu = (e + U) * u.abs()
    m = (h * u).mean(dim=-1, keepdim=True)
    em = (eh * u.abs() + h.abs() * eu + (d + 3) * U * (h * u).abs()).mean(dim=-1, keepdim=True)
    dx = r * (h - u * m)
    fp32 = r * (eh + eu * m.abs() + u.abs() * em + 2 * U * (h.abs() + (u * m).abs())) + (e + 2 * U) * dx.abs()
    fp32 = 1.01 * fp32
    bound = fp32 + EPS[gy.dtype] / 2 * (dx.abs() + fp32) + TINY[gy.dtype]
    terms = (g * u).abs()
    adds = 4 * H * -(-T // 4096) + 70
    bound_w = (G * u.abs() + (e + 2 * U + adds * U) * terms).sum(dim=(0, 1))
    return bound, 1.01 * bound_w + U * (g * u).sum(dim=(0, 1)).abs()
