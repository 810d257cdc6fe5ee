"""Torch-facing binding of the operators of the blocks between the merges: attention over
packed images with a learned relative position bias, and the norms around a block with its
gate and residual scale, each with its gradients.

Argument marshalling only, as in api.py: every step runs in the HIP kernels of libmpm.so on
``torch.cuda.current_stream()``. No autograd history: results of tensors that require gradients are detached
(blocks.py has the differentiable functions).

Rows of heads: queries are [R, H, dh] (packed by q_off, an int32 device tensor [B+1], with at most
Nq rows an image) or [B, N, H, dh] (dense), keys and values likewise with Hk heads; strided views
are taken as they are (the parts of one fused projection, say) as long as a head's channels are
contiguous and rows and heads start at 16-byte multiples.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

import torch

from . import _lib
from .api import _dt

_BYREF = ctypes.byref
_raw_stream = torch._C._cuda_getCurrentRawStream  # the current stream's handle, without its Python object
_NORMS = {"layer": _lib.MPM_NORM_LAYER, "rms": _lib.MPM_NORM_RMS}


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(t):
    """The current stream of a tensor's device."""
    return _raw_stream(t.get_device())


def _device(t, what, dtype, ref, numel=None):
    """Checks an optional contiguous device tensor; returns its address or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != ref.get_device() or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor on {ref.device}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{what} has {t.numel()} entries, expected {numel}")
    return t.data_ptr()


def _heads(t, what, ref, rows=None, heads=None):
    """The mpm_heads of rows of heads [R, H, dh] or [B, N, H, dh]."""
    if t.get_device() != ref.get_device():
        raise ValueError(f"{what} must be on the GPU, on {ref.device}")
    if t.dtype is not ref.dtype:
        raise TypeError(f"{what} must be {ref.dtype}, got {t.dtype}")
    st, sh = t.stride(), t.shape
    dims, dh = len(sh), sh[-1]
    if (dims != 3 and dims != 4) or (st[-1] != 1 and dh > 1):
        raise ValueError(f"{what} must be [R, H, dh] or [B, N, H, dh] with contiguous channels")
    n, row, head = sh[0], st[-3], st[-2]
    if dims == 4:
        if sh[1] == 1:
            row = st[0]  # (one row an image: the images' stride is the rows')
        elif n > 1 and sh[1] > 0 and st[0] != sh[1] * row:
            raise ValueError(f"{what}: dense images must follow each other at the rows' stride")
        n *= sh[1]
    if (rows is not None and n != rows) or dh != ref.shape[-1] or (heads is not None and sh[-2] != heads):
        raise ValueError(f"{what} has shape {tuple(sh)}, expected {rows} rows of {heads} heads of {ref.shape[-1]}")
    # A stride that nothing is reached by may be any number; a tensor without rows has no address and needs none.
    return _lib.Heads(t.data_ptr() if n else ref.data_ptr(), row if n > 1 else 0, head if sh[-2] > 1 else 0)


def _rows_of(t):
    return t.shape[0] if t.dim() == 3 else t.shape[0] * t.shape[1]


def _side(t, off, N, what):
    """(images, most rows an image) of one side of an attention call."""
    if t.dim() == 4:
        if off is not None:
            raise ValueError(f"dense {what} [B, N, H, dh] take no offsets")
        return t.shape[0], t.shape[1]
    if off is None or N is None:
        raise ValueError(f"packed {what} [R, H, dh] need their offsets and the most rows of an image")
    return off.numel() - 1, int(N) or int(t.shape[0] == 0)  # (no rows at all: any N is enough)


def _call(q, k, v, q_off, k_off, Nq, Nk, scale, bias, q_pos, k_pos, grid, k_bias):
    """The mpm_attention_call of these tensors, and the heads of q, k and v."""
    if not q.is_cuda:
        raise ValueError("queries must be on the GPU")
    dt = _dt(q)
    hq, hk = _heads(q, "q", q), _heads(k, "k", q)
    rq, rk, H, Hk = _rows_of(q), _rows_of(k), q.shape[-2], k.shape[-2]
    hv = _heads(v, "v", q, rk, Hk)
    B, nq = _side(q, q_off, Nq, "queries")
    Bk, nk = _side(k, k_off, Nk, "keys")
    if B != Bk:
        raise ValueError(f"queries of {B} images, keys of {Bk}")
    if k_off is None and nk == 0:  # dense images without keys: as packed ones
        k_off, nk = torch.zeros((B + 1,), dtype=torch.int32, device=q.device), 1
    c = _lib.AttentionCall(B, nq, nk, H, Hk, q.shape[-1], dt, q.shape[-1] ** -0.5 if scale is None else scale,
                           _device(q_off, "q_off", torch.int32, q, B + 1), _device(k_off, "k_off", torch.int32, q, B + 1))
    if bias is not None:
        if grid is None:
            raise ValueError("a position bias needs the grid (rows, columns)")
        W = bias.shape[-1]
        if bias.shape != (H, W, W) or W % 2 == 0:
            raise ValueError(f"bias must be [{H}, W, W] with an odd W, got {tuple(bias.shape)}")
        c.bias, c.span = _device(bias, "bias", torch.float32, q), W // 2
        c.grid_h, c.grid_w = grid
        c.q_pos, c.k_pos = _device(q_pos, "q_pos", torch.int32, q, rq), _device(k_pos, "k_pos", torch.int32, q, rk)
    c.k_bias = _device(k_bias, "k_bias", torch.float32, q, rk)
    c.held = k_off  # (until the call)
    return c, hq, hk, hv


def bucket_lut(span: int, side: int | None = None) -> tuple[torch.Tensor, int]:
    """(lut int32 [2 span + 1], buckets an axis): the bucket of each axis offset -span ... span.
    ``side`` None: a bucket for every offset. Otherwise ``side`` buckets a direction besides the
    offset 0: one for each of the first ceil(side / 2) offsets, then logarithmic widths up to span."""
    if side is None:
        return torch.arange(2 * span + 1, dtype=torch.int32), 2 * span + 1
    if not 1 <= side <= max(span, 1):
        raise ValueError("side must be between 1 and span")
    exact = (side + 1) // 2
    dist = []
    for d in range(span + 1):
        if d > exact and span > exact:
            d = min(side, exact + int(math.log(d / exact) / math.log(span / exact) * (side - exact) + 1e-9))
        dist.append(min(d, side))
    return torch.tensor([side - d for d in dist[:0:-1]] + [side + d for d in dist], dtype=torch.int32), 2 * side + 1


def bias_expand(table, lut, out=None):
    """The bias of every offset, float32 [H, W, W], from the learned table [nb * nb, H] and the bucket
    lut [W] of an axis offset (W = 2 span + 1): what attention() takes (mpm_bias_expand)."""
    nb, H, W = math.isqrt(table.shape[0]), table.shape[1], lut.numel()
    if not table.is_cuda or not table.is_contiguous() or nb * nb != table.shape[0] or W % 2 == 0:
        raise ValueError("table must be a contiguous device tensor [nb * nb, H], lut of odd length")
    if out is None:
        out = torch.empty((H, W, W), dtype=torch.float32, device=table.device)
    _lib.check("mpm_bias_expand", _lib.load().mpm_bias_expand(
        table.data_ptr(), _device(lut, "lut", torch.int32, table), nb, W // 2, H, _dt(table),
        _device(out, "out", torch.float32, table, H * W * W), _stream(table)))
    return out


def bias_gradient(dbias, lut, nb: int, dtype=torch.float32, out=None):
    """The table's gradient [nb * nb, H] from attention_backward's dbias [H, W, W] (mpm_bias_gradient)."""
    H, W = dbias.shape[0], lut.numel()
    if not dbias.is_cuda or dbias.shape != (H, W, W) or W % 2 == 0:
        raise ValueError("dbias must be a device tensor [H, W, W], lut of its odd length W")
    if out is None:
        out = torch.empty((nb * nb, H), dtype=dtype, device=dbias.device)
    _lib.check("mpm_bias_gradient", _lib.load().mpm_bias_gradient(
        _device(dbias, "dbias", torch.float32, dbias, H * W * W), _device(lut, "lut", torch.int32, dbias), int(nb),
        W // 2, H, _dt(out), _device(out, "out", out.dtype, dbias, nb * nb * H), _stream(dbias)))
    return out


def attention(q, k, v, q_off=None, k_off=None, Nq=None, Nk=None, scale=None, bias=None, q_pos=None, k_pos=None,
              grid=None, k_bias=None, with_lse=False, out=None):
    """softmax(scale q k^T + bias + k_bias) v of each image (mpm_attention): [R, H, dh] (or q's dense
    shape), and with ``with_lse`` the softmax statistics that attention_backward needs: float32
    [R, H, 2], the maximum taken and the log of the sum, base 2 (their sum times ln 2 is the log-sum-exp).

    ``scale``: default dh ** -0.5. ``bias``: float32 [H, W, W] from bias_expand, with ``grid`` the
    (rows, columns) of the token grid and ``q_pos`` / ``k_pos`` the raster positions, int32 per row
    (None: each row's index in its image). ``k_bias``: float32 per key row, -inf drops a key."""
    c, hq, hk, hv = _call(q, k, v, q_off, k_off, Nq, Nk, scale, bias, q_pos, k_pos, grid, k_bias)
    if out is None:
        out = q.new_empty(q.shape)
    rows = _rows_of(q)
    ho = _heads(out, "out", q, rows, c.H)
    lse = torch.empty((rows, c.H, 2), dtype=torch.float32, device=q.device) if with_lse else None
    if rows == 0:
        return (out, lse) if with_lse else out
    lib = _lib.load()
    need = lib.mpm_attention_workspace_bytes(_BYREF(c))
    ws = torch.empty((need,), dtype=torch.uint8, device=q.device) if need else None
    _lib.check("mpm_attention", lib.mpm_attention(_BYREF(c), _BYREF(hq), _BYREF(hk), _BYREF(hv), _BYREF(ho), _ptr(lse),
                                                  _ptr(ws), need, _stream(q)))
    return (out, lse) if with_lse else out


@dataclass
class AttentionGrads:
    dq: torch.Tensor
    dk: torch.Tensor
    dv: torch.Tensor
    dbias: torch.Tensor | None  # float32 [H, W, W], where the call had a bias


def attention_backward(dout, q, k, v, out, lse, q_off=None, k_off=None, Nq=None, Nk=None, scale=None, bias=None,
                       q_pos=None, k_pos=None, grid=None, k_bias=None, dq=None, dk=None, dv=None,
                       with_dbias=True) -> AttentionGrads:
    """The gradients of attention() (mpm_attention_backward) from dout and the call's own inputs, out
    and lse. ``dq``, ``dk``, ``dv``: where to write them (views of a fused projection's gradient,
    say); ``with_dbias`` False leaves out the bias's gradient."""
    c, hq, hk, hv = _call(q, k, v, q_off, k_off, Nq, Nk, scale, bias, q_pos, k_pos, grid, k_bias)
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) if g is None else g
                  for g, t in ((dq, q), (dk, k), (dv, v)))
    rq, rk = _rows_of(q), _rows_of(k)
    hs = [_heads(dout, "dout", q, rq, c.H), hq, hk, hv, _heads(out, "out", q, rq, c.H)]
    gs = [_heads(dq, "dq", q, rq, c.H), _heads(dk, "dk", q, rk, c.Hk), _heads(dv, "dv", q, rk, c.Hk)]
    dbias = torch.empty_like(bias) if bias is not None and with_dbias else None
    if rq == 0:  # no query: the sums over them are empty
        for t in (dk, dv, dbias):
            if t is not None:
                t.zero_()
        return AttentionGrads(dq, dk, dv, dbias)
    lib = _lib.load()
    if dbias is None:  # (the size without the partial sums of dbias)
        kept, c.bias = c.bias, None
    need = lib.mpm_attention_backward_workspace_bytes(_BYREF(c))
    if dbias is None:
        c.bias = kept
    ws = torch.empty((need,), dtype=torch.uint8, device=q.device)
    _lib.check("mpm_attention_backward", lib.mpm_attention_backward(
        _BYREF(c), *(_BYREF(x) for x in hs), _device(lse, "lse", torch.float32, q, 2 * rq * c.H), *(_BYREF(x) for x in gs),
        _ptr(dbias), _ptr(ws), need, _stream(q)))
    return AttentionGrads(dq, dk, dv, dbias)


def _norm_call(x, weight, bias, post_weight, post_bias, scale, gate, off, norm, eps):
    """The mpm_norm_call of these tensors (x: rows [R, D])."""
    if not x.is_cuda or not x.is_contiguous() or x.dim() != 2:
        raise ValueError("rows must be a contiguous device tensor [R, D]")
    try:
        kind = _NORMS[norm]
    except KeyError:
        raise ValueError(f"unknown norm {norm!r}; expected one of {sorted(_NORMS)}") from None
    R, D = x.shape
    B, per_row, gp, op = 1, 0, None, None
    if gate is not None:
        if gate.dim() != 2 or gate.shape[1] != D:
            raise ValueError(f"gate must be [B, {D}] or [{R}, {D}]")
        B = gate.shape[0]
        if off is not None:
            op = _device(off, "off", torch.int32, x, B + 1)
        elif B == R:
            per_row = 1
        gp = _device(gate, "gate", x.dtype, x)
    p = [_device(t, n, x.dtype, x, D) for t, n in ((weight, "weight"), (bias, "bias"), (post_weight, "post_weight"),
                                                    (post_bias, "post_bias"), (scale, "scale"))]
    return _lib.NormCall(R, D, _dt(x), kind, eps, B, per_row, op, *p, gp)


def residual_norm(x, f, weight=None, bias=None, post_weight=None, post_bias=None, scale=None, gate=None, off=None,
                  norm="layer", eps=1e-6, with_stats=False, out=None):
    """A block's output f into the residual stream x, and the next block's input (mpm_residual_norm):
    y = x + scale * gate * post_norm(f), h = norm(y). Returns (y, h), and with ``with_stats`` the
    float32 [R, 4] statistics that residual_norm_backward needs; h is None without ``weight``.

    x, f: rows [R, D]. ``weight`` / ``bias``: the norm before the next block; ``post_weight`` /
    ``post_bias``: the norm after this one (None: none); ``norm``: "layer" or "rms"; ``scale`` [D];
    ``gate``: [R, D], a row a token, or [B, D], a row an image, image b holding rows off[b] ...
    off[b + 1] (``off`` None: R / B rows each). ``out``: y's tensor (x itself, say)."""
    c = _norm_call(x, weight, bias, post_weight, post_bias, scale, gate, off, norm, eps)
    fp = _device(f, "f", x.dtype, x, x.numel())
    y = torch.empty_like(x) if out is None else out
    h = torch.empty_like(x) if weight is not None else None
    stats = torch.empty((x.shape[0], 4), dtype=torch.float32, device=x.device) if with_stats else None
    if x.shape[0] == 0:
        return (y, h, stats) if with_stats else (y, h)
    _lib.check("mpm_residual_norm", _lib.load().mpm_residual_norm(
        _BYREF(c), _ptr(x), fp, _device(y, "out", x.dtype, x, x.numel()), _ptr(h), _ptr(stats), _stream(x)))
    return (y, h, stats) if with_stats else (y, h)


@dataclass
class NormGradients:
    dx: torch.Tensor
    df: torch.Tensor
    dweight: torch.Tensor | None
    dbias: torch.Tensor | None
    dpost_weight: torch.Tensor | None
    dpost_bias: torch.Tensor | None
    dscale: torch.Tensor | None
    dgate: torch.Tensor | None


def residual_norm_backward(dy, dh, y, f, stats, weight=None, bias=None, post_weight=None, post_bias=None, scale=None,
                           gate=None, off=None, norm="layer", eps=1e-6) -> NormGradients:
    """The gradients of residual_norm() (mpm_residual_norm_backward) from dy (None: zero) and dh (None
    without ``weight``), the stored y, f and stats; the gradient of each parameter that is given."""
    c = _norm_call(y, weight, bias, post_weight, post_bias, scale, gate, off, norm, eps)
    n = y.numel()
    g = NormGradients(torch.empty_like(y), torch.empty_like(y),
                      *(None if t is None else torch.empty_like(t)
                        for t in (weight, bias, post_weight, post_bias, scale, gate)))
    if n == 0:  # no row: the sums over them are empty
        for t in (g.dweight, g.dbias, g.dpost_weight, g.dpost_bias, g.dscale, g.dgate):
            if t is not None:
                t.zero_()
        return g
    lib = _lib.load()
    need = lib.mpm_residual_norm_backward_workspace_bytes(_BYREF(c))
    ws = torch.empty((need,), dtype=torch.uint8, device=y.device)
    grads = _lib.NormGrads(*(_ptr(t) for t in (g.dx, g.df, g.dweight, g.dbias, g.dpost_weight, g.dpost_bias, g.dscale,
                                               g.dgate)))
    _lib.check("mpm_residual_norm_backward", lib.mpm_residual_norm_backward(
        _BYREF(c), _device(dy, "dy", y.dtype, y, n), _device(dh, "dh", y.dtype, y, n), _ptr(y),
        _device(f, "f", y.dtype, y, n), _device(stats, "stats", torch.float32, y, 4 * y.shape[0]), _BYREF(grads),
        _ptr(ws), need, _stream(y)))
    return g
