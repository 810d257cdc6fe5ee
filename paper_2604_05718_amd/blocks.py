"""Transformer blocks with a learned relative position bias, trainable, on packed images.

The blocks run attention and everything between their matrix products through the library: packed
attention with the bucketed bias (block_ops.attention), and each norm together with the residual sum,
scale and gate before it (block_ops.residual_norm). Both are differentiable here. The positions that
the bias needs follow the tokens through the merges (merge_local's y_pos), so the same blocks run on
full grids, on images of mixed sizes, and between merges.
"""
from __future__ import annotations

import torch

from . import api, block_ops


class _Once(torch.autograd.Function):
    """The first n tensors as they are, with a history that refuses to be differentiated."""

    @staticmethod
    def forward(ctx, n, *tensors):
        return tuple(t.view_as(t) for t in tensors[:n])

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of the blocks' operators have no gradients of their own: they can be "
                           "differentiated once only")


def _once(grads, *sources):
    """Gradients that the kernels computed from `sources` (None entries pass). Under create_graph they are
    joined to their sources by a node that raises, so that a second differentiation never misses their
    terms in silence (once_differentiable's node hangs on nothing: torch.autograd.grad to given inputs
    would walk past it)."""
    if not torch.is_grad_enabled():
        return tuple(grads)
    some = [g for g in grads if g is not None]
    tied = iter(_Once.apply(len(some), *some, *(t for t in sources if t is not None)))
    return tuple(None if g is None else next(tied) for g in grads)


class _Attention(torch.autograd.Function):
    """attention() of the parts of one projection, and of the bias table by way of its offsets;
    differentiable once."""

    @staticmethod
    def forward(ctx, qkv, table, lut, heads, where):
        H = heads
        q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
        bias = block_ops.bias_expand(table, lut)
        out, lse = block_ops.attention(q, k, v, bias=bias, with_lse=True, **where)
        # (the call's offsets and positions too, so that a buffer written before the backward pass is noticed)
        ctx.tensors = [n for n, t in where.items() if torch.is_tensor(t)]
        ctx.save_for_backward(qkv, table, bias, lut, out, lse, *(where[n] for n in ctx.tensors))
        ctx.rest = {n: t for n, t in where.items() if n not in ctx.tensors}
        ctx.heads, ctx.buckets = H, int(table.shape[0] ** 0.5 + 0.5)
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, table, bias, lut, out, lse, *tensors = ctx.saved_tensors
        H, grad, learned = ctx.heads, torch.empty_like(qkv), ctx.needs_input_grad[1]
        parts = [slice(0, H), slice(H, 2 * H), slice(2 * H, 3 * H)]
        g = block_ops.attention_backward(dout.contiguous(), *(qkv[:, p] for p in parts), out, lse, bias=bias,
                                         dq=grad[:, parts[0]], dk=grad[:, parts[1]], dv=grad[:, parts[2]],
                                         with_dbias=learned, **ctx.rest, **dict(zip(ctx.tensors, tensors)))
        dtable = block_ops.bias_gradient(g.dbias, lut, ctx.buckets, dtype=table.dtype) if learned else None
        return *_once((grad, dtable), dout, qkv, table), None, None, None


class _ResidualNorm(torch.autograd.Function):
    """residual_norm(): (y, h), differentiable in every tensor, once."""

    NAMES = ("weight", "bias", "post_weight", "post_bias", "scale", "gate")

    @staticmethod
    def forward(ctx, x, f, weight, bias, post_weight, post_bias, scale, gate, off, norm, eps):
        given = (weight, bias, post_weight, post_bias, scale, gate)
        y, h, stats = block_ops.residual_norm(x.contiguous(), f.contiguous(), *given, off=off, norm=norm, eps=eps,
                                              with_stats=True)
        ctx.save_for_backward(y, f, stats, off, *given)
        ctx.rest = dict(norm=norm, eps=eps)
        return y, h

    @staticmethod
    def backward(ctx, dy, dh):
        y, f, stats, off, *given = ctx.saved_tensors
        g = block_ops.residual_norm_backward(None if dy is None else dy.contiguous(),
                                             None if dh is None else dh.contiguous(), y, f.contiguous(), stats, *given,
                                             off=off, **ctx.rest)
        grads = (g.dx, g.df, g.dweight, g.dbias, g.dpost_weight, g.dpost_bias, g.dscale, g.dgate)
        return *_once(grads, dy, dh, y, f, *given), None, None, None


class RelativeBlock(torch.nn.Module):
    """Multi-head attention and a 4x MLP, each with a norm on both sides, a residual scale and a gate an
    image. Takes and returns (residual rows, the rows the next projection reads)."""

    def __init__(self, D: int, heads: int, buckets: int, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        kw = dict(device=device, dtype=dtype)

        def weight(*shape, std):
            return torch.nn.Parameter(torch.randn(shape, **kw) * std)

        def rows(value):
            return torch.nn.Parameter(torch.full((D,), value, **kw))

        self.heads = heads
        self.qkv, self.proj = weight(D, 3 * D, std=D ** -0.5), weight(D, D, std=D ** -0.5)
        self.fc1, self.fc2 = weight(D, 4 * D, std=D ** -0.5), weight(4 * D, D, std=(4 * D) ** -0.5)
        self.table = weight(buckets * buckets, heads, std=0.02)
        for side in ("attn", "mlp"):
            setattr(self, side + "_post_weight", rows(1.0))
            setattr(self, side + "_post_bias", rows(0.0))
            setattr(self, side + "_scale", rows(0.5))

    def _join(self, side, x, f, norm, gate, off):
        p = [getattr(self, f"{side}_{n}") for n in ("post_weight", "post_bias", "scale")]
        return _ResidualNorm.apply(x, f, norm.weight, norm.bias, *p, gate, off, "layer", 1e-6)

    def forward(self, x, h, lut, where, mid_norm, next_norm, gate=None, off=None):
        """x, h: rows [R, D]; where: the images, grid and positions as block_ops.attention takes them;
        mid_norm, next_norm: the norms before the MLP and before the next block; gate [B, D] with the
        images' offsets off, for both halves of the block."""
        R, D = x.shape
        qkv = (h @ self.qkv).view(R, 3 * self.heads, D // self.heads)
        a = _Attention.apply(qkv, self.table, lut, self.heads, where).view(R, D)
        x, h = self._join("attn", x, a @ self.proj, mid_norm, gate, off)
        f = torch.nn.functional.gelu(h @ self.fc1) @ self.fc2
        return self._join("mlp", x, f, next_norm, gate, off)


class Norm(torch.nn.Module):
    def __init__(self, D: int, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(D, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(D, device=device, dtype=dtype))


class RelativeEncoder(torch.nn.Module):
    """`depth` RelativeBlocks on a grid, with MPM before the blocks in `merge_before` (inference: the
    merges have no gradient) and the full grid rebuilt at the end."""

    def __init__(self, D: int, heads: int, depth: int, grid: tuple, span: int | None = None, side: int | None = None,
                 merge_before=(), device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.grid, self.merge_before = grid, tuple(merge_before)
        lut, buckets = block_ops.bucket_lut(min(63, max(grid) - 1) if span is None else span, side)
        self.register_buffer("lut", lut.to(device))
        self.blocks = torch.nn.ModuleList(RelativeBlock(D, heads, buckets, device, dtype) for _ in range(depth))
        self.norms = torch.nn.ModuleList(Norm(D, device, dtype) for _ in range(2 * depth + 1))

    def rows(self, x, off, N: int, pos, gate=None):
        """The blocks on packed rows x [R, D] (offsets off [B + 1], at most N an image, positions pos
        [R]): the final norm's rows. Differentiable."""
        where = dict(q_off=off, k_off=off, Nq=N, Nk=N, q_pos=pos, k_pos=pos, grid=self.grid)
        first = self.norms[0]
        h = torch.nn.functional.layer_norm(x, (x.shape[1],), first.weight, first.bias, 1e-6)
        for i, blk in enumerate(self.blocks):
            x, h = blk(x, h, self.lut, where, self.norms[2 * i + 1], self.norms[2 * i + 2], gate, off)
        return h

    @torch.no_grad()
    def forward(self, x, gate=None):
        """Full grids x [B, N, D]: merges in between, the last norm's rows gathered back to the grid."""
        B, N, D = x.shape
        grid_w, window = self.grid[1], max(self.grid)  # a window over the whole grid: every token is a candidate
        off = torch.arange(0, (B + 1) * N, N, dtype=torch.int32, device=x.device)
        pos = torch.arange(N, dtype=torch.int32, device=x.device).repeat(B)
        rows, most, maps = x.reshape(B * N, D), N, []
        first = self.norms[0]
        h = torch.nn.functional.layer_norm(rows, (D,), first.weight, first.bias, 1e-6)
        for i, blk in enumerate(self.blocks):
            if i in self.merge_before:
                m = api.merge_local(rows, grid_w, window, x_off=off, N=N, pos=pos)
                counts = m.y_off.cpu()  # one host read a merge: the rows and the longest image
                total, most = int(counts[-1]), int(torch.diff(counts).max())
                rows, off, pos = m.y[:total], m.y_off, m.y_pos[:total]
                maps.append(m.map)
                n = self.norms[2 * i]
                h = torch.nn.functional.layer_norm(rows, (D,), n.weight, n.bias, 1e-6)
            where = dict(q_off=off, k_off=off, Nq=most, Nk=most, q_pos=pos, k_pos=pos, grid=self.grid)
            rows, h = blk(rows, h, self.lut, where, self.norms[2 * i + 1], self.norms[2 * i + 2], gate, off)
        if not maps:
            return h.view(B, N, D)
        whole = maps[0]
        for m in maps[1:]:
            whole = api.compose(whole, m)
        return api.unmerge(h.contiguous(), off, whole)
