"""Plain 64-bit forms of the operators of the blocks, on the CPU, one image and head at a time."""
import math

import torch


def images(off, N, B):
    """Row slices of the images of one side."""
    if off is None:
        return [slice(b * N, (b + 1) * N) for b in range(B)]
    o = off.tolist()
    return [slice(o[b], o[b + 1]) for b in range(B)]


def attention(q, k, v, qs, ks, scale, bias=None, q_pos=None, k_pos=None, grid=None, k_bias=None):
    """(out [R, H, dh], lse [R, H]) of float64 rows; qs, ks the images' row slices; bias [H, W, W]
    float64; differentiable (elementary operations only)."""
    H, Hk = q.shape[1], k.shape[1]
    out, lse = [None] * len(qs), [None] * len(qs)
    order = sorted(range(len(qs)), key=lambda b: qs[b].start)
    for b in order:
        rows = torch.arange(ks[b].start, ks[b].stop)
        if k_bias is not None:
            rows = rows[k_bias[rows] > -math.inf]
        heads, sums = [], []
        n = qs[b].stop - qs[b].start
        for h in range(H):
            j = h // (H // Hk)
            Q, K, V = q[qs[b], h], k[rows, j], v[rows, j]
            if rows.numel() == 0:
                heads.append(torch.zeros((n, q.shape[2]), dtype=torch.float64))
                sums.append(torch.full((n,), -math.inf, dtype=torch.float64))
                continue
            s = Q @ K.T * scale
            if bias is not None:
                span, (gh, gw) = bias.shape[-1] // 2, grid
                kept = rows - ks[b].start
                qp = torch.arange(n) if q_pos is None else q_pos[qs[b]].long()
                kp = kept if k_pos is None else k_pos[rows].long()
                dr = (qp[:, None] // gw - kp[None, :] // gw).clamp(-span, span) + span
                dc = (qp[:, None] % gw - kp[None, :] % gw).clamp(-span, span) + span
                s = s + bias[h][dr, dc]
            if k_bias is not None:
                s = s + k_bias[rows].double()
            m = s.detach().amax(dim=1, keepdim=True)
            m = torch.where(m > -math.inf, m, torch.zeros_like(m))
            e = torch.exp(s - m)
            t = e.sum(dim=1, keepdim=True)
            some = t > 0
            heads.append(torch.where(some, e / torch.where(some, t, torch.ones_like(t)), torch.zeros_like(e)) @ V)
            sums.append((m + torch.log(t))[:, 0])
        out[b], lse[b] = torch.stack(heads, 1), torch.stack(sums, 1)
    return torch.cat([out[b] for b in order]), torch.cat([lse[b] for b in order])


def unit(t, kind, eps):
    if kind == "layer":
        t = t - t.mean(dim=1, keepdim=True)
    return t / torch.sqrt((t * t).mean(dim=1, keepdim=True) + eps)


def residual_norm(x, f, weight=None, bias=None, post_weight=None, post_bias=None, scale=None, gate=None, rows_of=None,
                  norm="layer", eps=1e-6):
    """(y, h) of float64 rows; rows_of: each row's gate row; differentiable."""
    u = f
    if post_weight is not None:
        u = unit(u, norm, eps) * post_weight
        if post_bias is not None:
            u = u + post_bias
    if scale is not None:
        u = u * scale
    if gate is not None:
        u = u * (gate if rows_of is None else gate[rows_of])
    y = x + u
    h = None
    if weight is not None:
        h = unit(y, norm, eps) * weight
        if bias is not None:
            h = h + bias
    return y, h


def rel(got, want):
    """2-norm of the difference over the result's."""
    got, want = got.detach().double().cpu(), want.detach().double()
    n = float(want.norm())
    d = float((got - want).norm())
    return d / n if n else d
