"""Transformer blocks with a learned relative position bias or with rotary positions, trainable, on packed
images, and a decoder head on the rebuilt grid.

The blocks run attention and everything between their matrix products through the library: packed
attention with the bucketed bias or of rotated queries and keys (block_ops.attention, block_ops.rotary), and each
norm together with the residual sum, scale and gate before it (block_ops.residual_norm); the head its group
norm with activation (block_ops.group_norm). All are differentiable here. The positions that
the bias or the rotation needs follow the tokens through the merges (merge_local's y_pos), so the same blocks run on
full grids, on images of mixed sizes, and between merges. For serving, the products of the blocks and of the head
run in 8-bit integers too (quantize(), block_ops.linear_int8).
"""
from __future__ import annotations

import math

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
        # (rows of no image: zeros, since what they hold reaches the weights' gradients, times zero)
        out, lse = block_ops.attention(q, k, v, bias=bias, with_lse=True, clear=True, **where)
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
                                         with_dbias=learned, clear=True, **ctx.rest, **dict(zip(ctx.tensors, tensors)))
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


class _RotaryAttention(torch.autograd.Function):
    """attention() of the parts of one projection, queries and keys turned by their positions (rotary()),
    and of the frequencies [2 heads, axes, pairs] or [axes, pairs]; differentiable once."""

    @staticmethod
    def forward(ctx, qkv, freq, heads, turn, where):
        H = heads
        qk = block_ops.rotary(qkv[:, :2 * H], freq, **turn)
        # (rows of no image are written by no kernel: what they hold would reach the weights' gradients, times zero)
        out = torch.zeros_like(qk[:, :H], memory_format=torch.contiguous_format) if any(ctx.needs_input_grad) else None
        out, lse = block_ops.attention(qk[:, :H], qk[:, H:], qkv[:, 2 * H:], with_lse=True, out=out, **where)
        # (offsets and positions too, so that a buffer written before the backward pass is noticed)
        ctx.tensors = [[n for n, t in d.items() if torch.is_tensor(t)] for d in (turn, where)]
        ctx.save_for_backward(qkv, qk, freq, out, lse, *(turn[n] for n in ctx.tensors[0]),
                              *(where[n] for n in ctx.tensors[1]))
        ctx.rest = [{n: t for n, t in d.items() if not torch.is_tensor(t)} for d in (turn, where)]
        ctx.heads = H
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, qk, freq, out, lse, *tensors = ctx.saved_tensors
        H, grad, learned = ctx.heads, torch.empty_like(qkv), ctx.needs_input_grad[1]
        held = iter(tensors)
        turn, where = ({**rest, **{n: next(held) for n in names}} for rest, names in zip(ctx.rest, ctx.tensors))
        both = grad[:, :2 * H]
        block_ops.attention_backward(dout.contiguous(), qk[:, :H], qk[:, H:], qkv[:, 2 * H:], out, lse, dq=grad[:, :H],
                                     dk=grad[:, H:2 * H], dv=grad[:, 2 * H:], clear=True, **where)
        g = block_ops.rotary_backward(both, qkv[:, :2 * H] if learned else None, freq, dx=both, with_dfreq=learned, **turn)
        return *_once((grad, g.dfreq), dout, qkv, freq), None, None, None


class _GroupNorm(torch.autograd.Function):
    """group_norm(), differentiable in x, weight and bias, once."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups, off, activation, eps):
        x = x.contiguous()
        # (zeros in rows of no image, as in _RotaryAttention)
        out = torch.zeros_like(x) if off is not None and any(ctx.needs_input_grad) else None
        y, stats = block_ops.group_norm(x, groups, weight, bias, off=off, activation=activation, eps=eps, with_stats=True,
                                        out=out)
        ctx.save_for_backward(x, stats, weight, bias, off)
        ctx.rest = dict(groups=groups, activation=activation, eps=eps)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, stats, weight, bias, off = ctx.saved_tensors
        g = block_ops.group_norm_backward(dy.contiguous(), x, stats, weight=weight, bias=bias, off=off, **ctx.rest)
        return *_once((g.dx, g.dweight, g.dbias), dy, x, weight, bias), None, None, None, None


class _Products(torch.nn.Module):
    """A module whose products x @ W can run in 8-bit integers."""

    PRODUCTS = ()  # names of the weights [in, out]

    def __init__(self):
        super().__init__()
        self.quantized = self._stale = False  # (stale: the weights were loaded since)

    def _exact(self):
        """Tensors that stay float32 when the module changes its type, since the kernels take them so."""
        return [getattr(self, n + "_step_scale") for n in self.PRODUCTS] if self.quantized else []

    def _apply(self, fn, recurse=True):
        exact = [t for t in self._exact() if t is not None]

        def convert(t):
            new = fn(t)
            return t.to(new.device) if any(t is e for e in exact) and new.dtype is not t.dtype else new

        return super()._apply(convert, recurse)

    @torch.no_grad()
    def quantize(self):
        """From now on the products run in 8-bit integers, with a scale for each token and output channel, from the
        weights as they are now; without gradients. The steps move with the module; they are no part of its state, and are
        made again from weights that load_state_dict() brings. Returns the module."""
        for n in self.PRODUCTS:
            steps, scale = block_ops.quantize_rows(getattr(self, n).t().contiguous())
            self.register_buffer(n + "_steps", steps, persistent=False)
            self.register_buffer(n + "_step_scale", scale, persistent=False)
        self.quantized, self._stale = True, False
        return self

    def _load_from_state_dict(self, *args, **kwargs):
        super()._load_from_state_dict(*args, **kwargs)
        self._stale = self.quantized

    def product(self, name, x, activation="none"):
        if not self.quantized:
            y = x @ getattr(self, name)
            return torch.nn.functional.gelu(y) if activation == "gelu" else y
        if torch.is_grad_enabled():
            raise RuntimeError("products in 8-bit integers have no gradients: run them under torch.no_grad()")
        if self._stale:
            if x.is_cuda and torch.cuda.is_current_stream_capturing():
                raise RuntimeError("weights were loaded since quantize(): their steps have to be made before a capture")
            self.quantize()
        return block_ops.linear_int8(x, getattr(self, name + "_steps"), getattr(self, name + "_step_scale"),
                                     activation=activation)


class _Block(_Products):
    """Multi-head attention and a 4x MLP, each with a norm on both sides, a residual scale and a gate an
    image. Takes and returns (residual rows, the rows the next projection reads)."""

    PRODUCTS = ("qkv", "proj", "fc1", "fc2")

    def __init__(self, D: int, heads: int, device="cuda", dtype=torch.bfloat16, **positions):
        super().__init__()
        kw = dict(device=device, dtype=dtype)

        def weight(*shape, std):
            return torch.nn.Parameter(torch.randn(shape, **kw) * std)

        def rows(value):
            return torch.nn.Parameter(torch.full((D,), value, **kw))

        self.heads = heads
        self.qkv, self.proj = weight(D, 3 * D, std=D ** -0.5), weight(D, D, std=D ** -0.5)
        self.fc1, self.fc2 = weight(D, 4 * D, std=D ** -0.5), weight(4 * D, D, std=(4 * D) ** -0.5)
        self._positions(weight, **positions)
        for side in ("attn", "mlp"):
            setattr(self, side + "_post_weight", rows(1.0))
            setattr(self, side + "_post_bias", rows(0.0))
            setattr(self, side + "_scale", rows(0.5))

    def _join(self, side, x, f, norm, gate, off):
        p = [getattr(self, f"{side}_{n}") for n in ("post_weight", "post_bias", "scale")]
        return _ResidualNorm.apply(x, f, norm.weight, norm.bias, *p, gate, off, "layer", 1e-6)

    def forward(self, x, h, lut, where, mid_norm, next_norm, gate=None, off=None):
        """x, h: rows [R, D]; lut: the bucket of an axis offset (RelativeBlock); where: the images, grid and positions as
        block_ops.attention takes them; mid_norm, next_norm: the norms before the MLP and before the next block; gate
        [B, D] with the images' offsets off, for both halves of the block."""
        R, D = x.shape
        qkv = self.product("qkv", h).view(R, 3 * self.heads, D // self.heads)
        a = self._attend(qkv, lut, where).view(R, D)
        x, h = self._join("attn", x, self.product("proj", a), mid_norm, gate, off)
        f = self.product("fc2", self.product("fc1", h, "gelu"))
        return self._join("mlp", x, f, next_norm, gate, off)


class RelativeBlock(_Block):
    """A block whose scores have a learned bias by bucket of the grid offset."""

    def __init__(self, D: int, heads: int, buckets: int, device="cuda", dtype=torch.bfloat16):
        super().__init__(D, heads, device, dtype, buckets=buckets)

    def _positions(self, weight, buckets):
        self.table = weight(buckets * buckets, self.heads, std=0.02)

    def _attend(self, qkv, lut, where):
        return _Attention.apply(qkv, self.table, lut, self.heads, where)


class RotaryBlock(_Block):
    """A block whose queries and keys are turned by their places on the grid: by the frequencies [axes, pairs], or,
    learned, by ones of its own for every head that start there."""

    def __init__(self, D: int, heads: int, freq, learned: bool = False, device="cuda", dtype=torch.bfloat16):
        super().__init__(D, heads, device, dtype, freq=freq.to(device, torch.float32), learned=learned)

    def _positions(self, weight, freq, learned):
        self.learned = learned
        if learned:
            self.freq = torch.nn.Parameter(freq.repeat(self.heads, 1, 1))
        else:
            self.register_buffer("freq", freq)

    def _exact(self):
        return [*super()._exact(), self.freq, self.freq.grad]

    def _attend(self, qkv, lut, where):
        freq = torch.cat([self.freq, self.freq]) if self.learned else self.freq  # (queries' heads, then keys')
        turn = dict(pos=where["q_pos"], grid=where["grid"], off=where["q_off"])
        where = {n: where[n] for n in ("q_off", "k_off", "Nq", "Nk")}
        return _RotaryAttention.apply(qkv, freq, self.heads, turn, where)


class Norm(torch.nn.Module):
    def __init__(self, D: int, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(D, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(D, device=device, dtype=dtype))


class _Encoder(torch.nn.Module):
    """Blocks on a grid, with MPM before the blocks in `merge_before` (inference: the
    merges have no gradient) and the full grid rebuilt at the end."""

    def __init__(self, D: int, grid: tuple, blocks, merge_before=(), device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.grid, self.merge_before = grid, tuple(merge_before)
        self.blocks = torch.nn.ModuleList(blocks)
        self.norms = torch.nn.ModuleList(Norm(D, device, dtype) for _ in range(2 * len(self.blocks) + 1))

    def quantize(self):
        """Serves the blocks' products in 8-bit integers from now on (_Products.quantize). Returns the module."""
        for blk in self.blocks:
            blk.quantize()
        return self

    def rows(self, x, off, N: int, pos, gate=None):
        """The blocks on packed rows x [R, D] (offsets off [B + 1], at most N an image, positions pos
        [R]): the final norm's rows. Differentiable. Rows of no image take no part, but have to be finite: a product's gradient
        multiplies them by zero."""
        where = dict(q_off=off, k_off=off, Nq=N, Nk=N, q_pos=pos, k_pos=pos, grid=self.grid)
        first = self.norms[0]
        h = torch.nn.functional.layer_norm(x, (x.shape[1],), first.weight, first.bias, 1e-6)
        for i, blk in enumerate(self.blocks):
            x, h = blk(x, h, self._lut(), where, self.norms[2 * i + 1], self.norms[2 * i + 2], gate, off)
        return h

    def _lut(self):
        return None

    @torch.no_grad()
    def forward(self, x, gate=None):
        """Full grids x [B, N, D]: merges in between, the last norm's rows gathered back to the grid."""
        B, N, D = x.shape
        # (a clip merges as one grid of all its frames' rows)
        grid_w, rows_of_grid = self.grid[-1], math.prod(self.grid[:-1])
        window = max(rows_of_grid, grid_w)  # over the whole grid: every token is a candidate
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
            rows, h = blk(rows, h, self._lut(), where, self.norms[2 * i + 1], self.norms[2 * i + 2], gate, off)
        if not maps:
            return h.view(B, N, D)
        whole = maps[0]
        for m in maps[1:]:
            whole = api.compose(whole, m)
        return api.unmerge(h.contiguous(), off, whole)


class RelativeEncoder(_Encoder):
    """`depth` RelativeBlocks on a grid, with MPM before the blocks in `merge_before` (inference: the
    merges have no gradient) and the full grid rebuilt at the end."""

    def __init__(self, D: int, heads: int, depth: int, grid: tuple, span: int | None = None, side: int | None = None,
                 merge_before=(), device="cuda", dtype=torch.bfloat16):
        lut, buckets = block_ops.bucket_lut(min(63, max(grid) - 1) if span is None else span, side)
        super().__init__(D, grid, (RelativeBlock(D, heads, buckets, device, dtype) for _ in range(depth)), merge_before,
                         device, dtype)
        self.register_buffer("lut", lut.to(device))

    def _lut(self):
        return self.lut


class RotaryEncoder(_Encoder):
    """`depth` RotaryBlocks on a grid, all pairs of a head's channels turned (rotary_frequencies with `theta`, learned by
    every block and head with `learned`), merges and the rebuilt grid as RelativeEncoder's. grid: (rows, columns), or
    (frames, rows, columns) of clips."""

    def __init__(self, D: int, heads: int, depth: int, grid: tuple, theta: float = 100.0, learned: bool = False,
                 merge_before=(), device="cuda", dtype=torch.bfloat16):
        freq = block_ops.rotary_frequencies(D // heads // 2, len(grid), theta)
        super().__init__(D, grid, (RotaryBlock(D, heads, freq, learned, device, dtype) for _ in range(depth)), merge_before,
                         device, dtype)


class GridHead(_Products):
    """A decoder head on rebuilt grids: a product to C channels, group norm with an activation over each grid, a product
    to the classes. Trainable; quantize() serves its products in 8-bit integers."""

    PRODUCTS = ("inner", "classes")

    def __init__(self, D: int, C: int, classes: int, groups: int = 32, activation: str = "silu", device="cuda",
                 dtype=torch.bfloat16):
        super().__init__()
        kw = dict(device=device, dtype=dtype)
        self.groups, self.activation = groups, activation
        self.inner = torch.nn.Parameter(torch.randn((D, C), **kw) * D ** -0.5)
        self.weight, self.bias = torch.nn.Parameter(torch.ones(C, **kw)), torch.nn.Parameter(torch.zeros(C, **kw))
        self.classes = torch.nn.Parameter(torch.randn((C, classes), **kw) * C ** -0.5)

    def forward(self, x, off=None):
        """Grids x [B, N, D] (or packed rows [R, D] by off [B + 1]) to scores of the classes, [B, N, classes]."""
        rows = self.product("inner", x.reshape(-1, x.shape[-1]))
        C, classes = self.classes.shape
        t = _GroupNorm.apply(rows if off is not None else rows.view(*x.shape[:-1], C), self.weight, self.bias, self.groups,
                             off, self.activation, 1e-5)
        return self.product("classes", t.reshape(rows.shape)).view(*x.shape[:-1], classes)
