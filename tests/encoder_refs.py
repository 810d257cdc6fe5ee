"""Plain 64-bit forms of rotary positions, the product in 8-bit integers and group norm, on the CPU."""
import math

import torch


def cells(pos, grid):
    """Grid coordinates [R, axes] of raster indices, those outside the grid taken as the nearest cell."""
    pos = pos.long().clamp(0, math.prod(grid) - 1)
    out = []
    for n in reversed(grid[1:]):
        out.insert(0, pos % n)
        pos = pos // n
    return torch.stack([pos, *out], dim=1).double()


def turned(x, freq, c, layout="halves", sign=1.0):
    """Rows of heads [R, H, dh] (float64), freq [axes, P] or [H, axes, P], c [R, axes]; differentiable."""
    P = freq.shape[-1]
    f = freq if freq.dim() == 3 else freq[None]
    angle = sign * sum(c[:, a, None, None] * f[None, :, a] for a in range(c.shape[1]))
    if layout == "halves":
        i, j = torch.arange(P), torch.arange(P, 2 * P)
    else:
        i, j = torch.arange(0, 2 * P, 2), torch.arange(1, 2 * P, 2)
    a, b = x[..., i], x[..., j]
    out = x.clone()
    out[..., i] = a * torch.cos(angle) - b * torch.sin(angle)
    out[..., j] = a * torch.sin(angle) + b * torch.cos(angle)
    return out


def pair_sizes(x, P, layout):
    """|x_1| + |x_2| of its pair at every channel (zero where channels pass)."""
    s = torch.zeros_like(x)
    i, j = ((torch.arange(P), torch.arange(P, 2 * P)) if layout == "halves" else
            (torch.arange(0, 2 * P, 2), torch.arange(1, 2 * P, 2)))
    s[..., i] = s[..., j] = x[..., i].abs() + x[..., j].abs()
    return s


def steps(x):
    """(q [R, K], scale [R]) of float32 values: float64 holds the quotients' distance to a half exactly enough (it is 0 or
    at least 2^-33 of them)."""
    largest = x.abs().amax(dim=1)
    scale = torch.clamp((largest.double() / 127).float(), min=2.0 ** -126)
    bad = ~torch.isfinite(x).all(dim=1)
    q = torch.round(x.double() / scale.double()[:, None]).clamp(-127, 127)
    q[bad] = 0
    scale[bad] = math.nan
    return q.to(torch.int8), scale


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * torch.special.erfc(-z / math.sqrt(2)) / 2
    return z


def group_norm(x, groups, parts, weight=None, bias=None, activation="none", eps=1e-5):
    """Rows [R, C] (float64), parts: the images' row slices in order; rows of none are left out. Differentiable."""
    C, out = x.shape[1], []
    for rows in parts:
        t = x[rows]
        n = t.shape[0]
        if n == 0:
            continue
        t = t.reshape(n, groups, C // groups).transpose(0, 1).reshape(groups, -1)
        t = t - t.mean(dim=1, keepdim=True)
        t = t / torch.sqrt((t * t).mean(dim=1, keepdim=True) + eps)
        t = t.reshape(groups, n, C // groups).transpose(0, 1).reshape(n, C)
        if weight is not None:
            t = t * weight
        if bias is not None:
            t = t + bias
        out.append(act(t, activation))
    return torch.cat(out)


def gelu_bf16(z):
    """GELU as the kernels form it for bfloat16 results: z / (1 + e^-l), l an odd polynomial."""
    u = z * z
    l = z * (1.59312151 + u * (7.55007635e-2 + u * (-9.3992063e-4 + u * 7.25138e-6)))
    return z / (1 + torch.exp(-l))


def gelu_bf16_bound(z):
    """How far it is from GELU: 0.00105 of l, of which the result for -|z| takes that share, or 10^-4 of it."""
    small = z.abs() * torch.special.erfc(z.abs() / math.sqrt(2)) / 2
    return 0.00105 * small.clamp_min(1e-4)
