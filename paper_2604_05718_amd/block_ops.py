"""Torch-facing binding of the operators of the blocks between the merges: attention over
packed images with a learned relative position bias, rotary positions, the norms around a block with its
gate and residual scale, group norm over grids, each with its gradients; and products in 8-bit integers.

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
_LAYOUTS = {"halves": _lib.MPM_ROTARY_HALVES, "pairs": _lib.MPM_ROTARY_PAIRS}
_ACTIVATIONS = {"none": _lib.MPM_ACT_NONE, "relu": _lib.MPM_ACT_RELU, "silu": _lib.MPM_ACT_SILU, "gelu": _lib.MPM_ACT_GELU}
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
              grid=None, k_bias=None, with_lse=False, out=None, clear=False):
    """softmax(scale q k^T + bias + k_bias) v of each image (mpm_attention): [R, H, dh] (or q's dense
    shape), and with ``with_lse`` the softmax statistics that attention_backward needs: float32
    [R, H, 2], the maximum taken and the log of the sum, base 2 (their sum times ln 2 is the log-sum-exp).

    ``scale``: default dh ** -0.5. ``bias``: float32 [H, W, W] from bias_expand, with ``grid`` the
    (rows, columns) of the token grid and ``q_pos`` / ``k_pos`` the raster positions, int32 per row
    (None: each row's index in its image). ``k_bias``: float32 per key row, -inf drops a key. ``clear``: zeros in the rows
    of ``out`` that belong to no image, which are otherwise left as they are."""
    c, hq, hk, hv = _call(q, k, v, q_off, k_off, Nq, Nk, scale, bias, q_pos, k_pos, grid, k_bias)
    if out is None:
        out = q.new_empty(q.shape)
    rows = _rows_of(q)
    ho = _heads(out, "out", q, rows, c.H)
    lse = torch.empty((rows, c.H, 2), dtype=torch.float32, device=q.device) if with_lse else None
    c.q_rows = rows if clear else 0
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
                       with_dbias=True, clear=False) -> AttentionGrads:
    """The gradients of attention() (mpm_attention_backward) from dout and the call's own inputs, out
    and lse. ``dq``, ``dk``, ``dv``: where to write them (views of a fused projection's gradient,
    say); ``with_dbias`` False leaves out the bias's gradient; ``clear``: zeros in the rows of dq, dk and dv that belong
    to no image."""
    c, hq, hk, hv = _call(q, k, v, q_off, k_off, Nq, Nk, scale, bias, q_pos, k_pos, grid, k_bias)
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) if g is None else g
                  for g, t in ((dq, q), (dk, k), (dv, v)))
    rq, rk = _rows_of(q), _rows_of(k)
    hs = [_heads(dout, "dout", q, rq, c.H), hq, hk, hv, _heads(out, "out", q, rq, c.H)]
    gs = [_heads(dq, "dq", q, rq, c.H), _heads(dk, "dk", q, rk, c.Hk), _heads(dv, "dv", q, rk, c.Hk)]
    dbias = torch.empty_like(bias) if bias is not None and with_dbias else None
    c.q_rows, c.k_rows = (rq, rk) if clear else (0, 0)
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
    off[b + 1] (``off`` None: R / B rows each; rows of no image are zeros, in a given ``out`` as they were).
    ``out``: y's tensor (x itself, say)."""
    c = _norm_call(x, weight, bias, post_weight, post_bias, scale, gate, off, norm, eps)
    c.clear = _lib.MPM_CLEAR_ROWS | (_lib.MPM_CLEAR_SUM if out is None else 0)
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
    without ``weight``), the stored y, f and stats; the gradient of each parameter that is given; zeros in rows of no
    image."""
    c = _norm_call(y, weight, bias, post_weight, post_bias, scale, gate, off, norm, eps)
    c.clear = _lib.MPM_CLEAR_ROWS
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


# ---- rotary positions, products in 8-bit integers, group norm ------------------------------


_MOST = 2 ** 31 - 1  # what an int32 of a call holds


def _launch(name, ref, *args):
    """Calls an entry point on the current stream of ref's device, with that device current."""
    device = ref.get_device()
    if device == torch._C._cuda_getDevice():
        status = getattr(_lib.load(), name)(*args, _stream(ref))
    else:
        with torch.cuda.device(device):
            status = getattr(_lib.load(), name)(*args, _stream(ref))
    if status:
        _lib.check(name, status)


def _scratch(need, ref):
    return torch.empty((need,), dtype=torch.uint8, device=ref.device) if need else None


def _one_of(table, key, what):
    try:
        return table[key]
    except KeyError:
        raise ValueError(f"unknown {what} {key!r}; expected one of {sorted(table)}") from None


def rotary_frequencies(pairs: int, axes: int, theta: float = 100.0):
    """float32 [axes, pairs] for rotary(): the pairs dealt to the axes in turns, each axis' ones a geometric range
    of angles a cell from 1 down to about 1 / theta."""
    if pairs < 1 or not 1 <= axes <= 3 or not theta > 0:
        raise ValueError("pairs from 1, axes from 1 to 3 and a theta above zero")
    freq = torch.zeros((axes, pairs), dtype=torch.float64)
    own = -(-pairs // axes)
    for p in range(pairs):
        freq[p % axes, p] = theta ** (-(p // axes) / own)
    return freq.float()


def _rotary_call(x, freq, pos, grid, layout, off):
    """The mpm_rotary_call of these tensors, and the heads of x."""
    if not x.is_cuda:
        raise ValueError("rows of heads must be on the GPU")
    dt, heads = _dt(x), _heads(x, "x", x)
    shape, fs, axes = x.shape, freq.shape, len(grid)
    dense = len(shape) == 4
    rows, H, dh = shape[0] * shape[1] if dense else shape[0], shape[-2], shape[-1]
    if not 1 <= axes <= 3 or math.prod(grid) > _MOST or max(grid) > _MOST or rows > _MOST:
        raise ValueError("grid has one to three axes and, like the rows, at most 2^31 - 1 cells")
    if fs[-2:-1] != (axes,) or len(fs) > 3 or (len(fs) == 3 and fs[0] != H):
        raise ValueError(f"freq must be [{axes}, pairs] or [{H}, {axes}, pairs], got {tuple(fs)}")
    B = shape[0] if dense else 1
    if off is not None:
        if dense:
            raise ValueError("dense rows [B, N, H, dh] take no offsets")
        B = off.numel() - 1
    c = _lib.RotaryCall(rows, H, dh, dt, fs[-1], _one_of(_LAYOUTS, layout, "layout"), axes, (*grid, 1, 1)[:3],
                        len(fs) == 3, _device(freq, "freq", torch.float32, x), _device(pos, "pos", torch.int32, x, rows),
                        B, _device(off, "off", torch.int32, x, B + 1))
    return c, heads


def _like(t, c):
    """A new contiguous tensor like t, rows of heads of a rotary call, and its heads."""
    new = t.new_empty(t.shape)
    return new, _lib.Heads(new.data_ptr(), c.H * c.dh, c.dh)


def _written(t, what, ref, c):
    """The heads of a given tensor that a rotary call writes: every row and head at a place of its own."""
    h = _heads(t, what, ref, c.R, c.H)
    if (h.row == 0 and c.R > 1) or (h.head == 0 and c.H > 1):
        raise ValueError(f"{what} must not be expanded: its rows and heads are written")
    return h


def _share(a, b, c, size):
    """Whether two tensors of a rotary call (their heads, values of `size` bytes) share memory."""
    if c.R == 0:
        return False
    row, head, dh = a.row * size, a.head * size, c.dh * size
    ends = [h.p + ((c.R - 1) * h.row + (c.H - 1) * h.head + c.dh) * size for h in (a, b)]
    if ends[0] <= b.p or ends[1] <= a.p:
        return False
    if (a.row, a.head) != (b.row, b.head):
        return True  # (nested, or in an order of their own)
    # A head of one meets a head of the other where their distance, less whole rows and heads, is under a head.
    for j in range(1 - c.H, c.H):
        off = b.p - a.p - j * head
        i = off // row if row else 0
        if any(abs(off - k * row) < dh for k in (i, i + 1) if abs(k) < c.R):
            return True
    return False


def _in_place_or_apart(what, to, given, c, t):
    """Refuses a tensor that is written and meets another one (`given`: name -> heads) elsewhere than on every value."""
    for name, h in given.items():
        if (to.p, to.row, to.head) != (h.p, h.row, h.head) and _share(to, h, c, t.element_size()):
            raise ValueError(f"{what} overlaps {name}: it must be {name} itself or lie apart")


def rotary(x, freq, pos=None, grid=(1,), layout="halves", off=None, inverse=False, out=None):
    """Rows of heads with every pair of channels turned by its row's place on a grid (mpm_rotary): the shape of x.

    x: [R, H, dh] (packed, with the images' offsets ``off`` [B + 1]: rows of no image are left as they are in
    ``out``; without, every row is turned) or [B, N, H, dh]; strided views as for attention(). ``freq``: float32
    [axes, pairs], or [H, axes, pairs] for frequencies by head, radians a cell (rotary_frequencies); ``grid``: the cells
    of the axes, (rows, columns) or (frames, rows, columns); ``pos``: int32 raster index of each row (None:
    each row's index in its image; without ``off``, packed rows are one image). ``layout``: pair p is channels
    p and p + pairs ("halves") or 2 p and 2 p + 1 ("pairs"); channels from 2 pairs on pass. ``inverse``: by the
    negative angles. ``out``: where to write, x itself or memory apart from it."""
    c, hx = _rotary_call(x, freq, pos, grid, layout, off)
    if out is None:
        out, ho = _like(x, c)
    else:
        ho = _written(out, "out", x, c)
        _in_place_or_apart("out", ho, {"x": hx}, c, x)
    if c.R:
        _launch("mpm_rotary", x, _BYREF(c), _BYREF(hx), _BYREF(ho), int(bool(inverse)))
    return out


@dataclass
class RotaryGrads:
    dx: torch.Tensor
    dfreq: torch.Tensor | None  # float32, as freq


def rotary_backward(dout, x, freq, pos=None, grid=(1,), layout="halves", off=None, dx=None, with_dfreq=True) -> RotaryGrads:
    """The gradients of rotary() (mpm_rotary_backward) from dout and the call's own inputs. ``dx``: where to write it,
    dout itself or memory apart from it, and apart from x; ``with_dfreq`` False leaves out the frequencies' gradient (x
    may be None then)."""
    c, hd = _rotary_call(dout, freq, pos, grid, layout, off)
    given = dx is not None
    if not given:
        dx, hg = _like(dout, c)
    else:
        hg = _written(dx, "dx", dout, c)
        _in_place_or_apart("dx", hg, {"dout": hd}, c, dout)
    hx, dfreq, ws, need = None, None, None, 0
    if with_dfreq:
        hx = _heads(x, "x", dout, c.R, c.H)
        if given and c.R and _share(hg, hx, c, dout.element_size()):
            raise ValueError("dx overlaps x, which the frequencies' gradient still reads")
        hx = _BYREF(hx)
        dfreq = torch.empty_like(freq)
        if c.R == 0:
            dfreq.zero_()
        else:
            need = _lib.load().mpm_rotary_backward_workspace_bytes(_BYREF(c))
            ws = _scratch(need, dout)
    if c.R:
        _launch("mpm_rotary_backward", dout, _BYREF(c), _BYREF(hd), hx, _BYREF(hg), _ptr(dfreq), _ptr(ws), need)
    return RotaryGrads(dx, dfreq)


def _value_rows(x, what):
    """(rows, K, stride of a row in elements) of values [R, K] with contiguous channels, 16 bytes apart at least."""
    if not x.is_cuda or x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] > 1):
        raise ValueError(f"{what} must be a device tensor [R, K] with contiguous channels")
    if max(x.shape) > _MOST:
        raise ValueError(f"{what} has more than 2^31 - 1 rows")
    return x.shape[0], x.shape[1], x.stride(0) if x.shape[0] > 1 else 0


def quantize_rows(x):
    """Rows of values [R, K] as 8-bit steps with a scale each (mpm_quantize_rows): int8 [R, K rounded up to a multiple
    of 16] (zeros past K) and float32 [R]. Of a weight [out, in]: what linear_int8 takes as its weight."""
    R, K, row = _value_rows(x, "x")
    dt = _dt(x)
    q = torch.empty((R, -(-K // 16) * 16), dtype=torch.int8, device=x.device)
    scale = torch.empty((R,), dtype=torch.float32, device=x.device)
    if R:
        _launch("mpm_quantize_rows", x, _ptr(x), R, K, row, dt, _ptr(q), _ptr(scale))
    return q, scale


def _meets(x, K, out, N):
    """Whether rows of K values at x and rows of N at out, as many, share memory."""
    a, b = K * x.element_size(), N * out.element_size()
    row, ahead, rows = x.stride(0) * x.element_size(), out.data_ptr() - x.data_ptr(), x.shape[0] - 1
    if ahead >= rows * row + a or -ahead >= rows * out.stride(0) * out.element_size() + b:
        return False
    between = ahead % row if row else 0  # (columns side by side in rows of one buffer)
    return not (rows and row == out.stride(0) * out.element_size() and a <= between and between + b <= row)


def _meets_rows(t, out, N):
    """Whether a contiguous tensor shares memory with rows of N values at out."""
    row, at = max(1, out.stride(0)) * out.element_size(), t.data_ptr() - out.data_ptr()  # (one row may have any stride)
    first = max(0, (at - N * out.element_size()) // row + 1)  # the first row that ends behind its start
    return t.numel() > 0 and first < out.shape[0] and first * row < at + t.numel() * t.element_size()


def linear_int8(x, weight, weight_scale, x_scale=None, bias=None, activation="none", dtype=None, out=None):
    """act(x weight^T + bias) in 8-bit integers with a scale for each token and output channel (mpm_linear_int8): [R, N].

    x: values [R, K] (float32 or bfloat16, row strides of whole 16 bytes), which are turned into steps on the way, or
    with ``x_scale`` the steps of quantize_rows. ``weight``, ``weight_scale``: quantize_rows of a weight [N, K].
    ``bias`` [N] and the result have ``dtype`` (that of x or of ``out``; bfloat16 for steps). ``activation``: "none", "relu",
    "silu" or "gelu". ``out``: rows [R, N] with contiguous channels and a row stride of its own, apart
    from the inputs."""
    R, K, row = _value_rows(x, "x")
    if x_scale is None:
        x_dt = _dt(x)
    elif x.dtype is torch.int8 and (R <= 1 or row == K) and K % 16 == 0:
        x_dt, row = _lib.MPM_I8, 0
    else:
        raise ValueError("steps must be contiguous int8 rows of a multiple of 16 channels")
    if weight.dim() != 2 or weight.shape[1] != -(-K // 16) * 16:
        raise ValueError(f"weight must be int8 [N, {-(-K // 16) * 16}], got {tuple(weight.shape)}")
    N = weight.shape[0]
    if out is None:
        if dtype is None:
            dtype = x.dtype if x_scale is None else torch.bfloat16
        out = torch.empty((R, N), dtype=dtype, device=x.device)
    elif out.shape != (R, N) or out.get_device() != x.get_device() or dtype not in (None, out.dtype) or (
            out.stride(1) != 1 and N > 1) or (R > 1 and out.stride(0) < N):
        raise ValueError(f"out must be [{R}, {N}] on {x.device} with contiguous channels")
    elif R and N and _meets(x, K, out, N):
        raise ValueError("out must not overlap x: other channels still read it")
    elif R and N and any(t is not None and _meets_rows(t, out, N) for t in (weight, weight_scale, x_scale, bias)):
        raise ValueError("out must not overlap the weight, its shift or a scale: other tokens still read them")
    c = _lib.Linear8Call(R, N, K, x_dt, _dt(out), _one_of(_ACTIVATIONS, activation, "activation"), row,
                         out.stride(0) if R > 1 else N, _device(x_scale, "x_scale", torch.float32, x, R),
                         _device(weight, "weight", torch.int8, x),
                         _device(weight_scale, "weight_scale", torch.float32, x, N),
                         _device(bias, "bias", out.dtype, x, N))
    if R and N:
        # Few results may need no room, which costs more than the call that says so; otherwise at least what it would say.
        if x_scale is not None:
            need = 0
        elif R <= 16 or R * N <= 65536:
            need = _lib.load().mpm_linear_int8_workspace_bytes(_BYREF(c))
        else:
            need = R * weight.shape[1] + 4 * R + 512
        ws = _scratch(need, x)
        _launch("mpm_linear_int8", x, _BYREF(c), _ptr(x), _ptr(out), _ptr(ws), need)
    return out


def _group_call(x, groups, weight, bias, off, activation, eps):
    """The mpm_group_norm_call of these tensors."""
    if not x.is_cuda or not x.is_contiguous() or x.dim() < 2:
        raise ValueError("x must be a contiguous device tensor [R, C] with offsets, or [B, ..., C]")
    C = x.shape[-1]
    if x.dim() == 2:
        if off is None:
            raise ValueError("packed rows [R, C] need their offsets")
        B = off.numel() - 1
    elif off is not None:
        raise ValueError("dense images [B, ..., C] take no offsets")
    else:
        B = x.shape[0]
    R = math.prod(x.shape[:-1])
    if R > _MOST or C < 1 or not 1 <= groups <= C:
        raise ValueError(f"at most 2^31 - 1 rows, and between 1 and {C} groups")
    return _lib.GroupNormCall(R, C, groups, _dt(x), _one_of(_ACTIVATIONS, activation, "activation"), eps, B,
                              _device(off, "off", torch.int32, x, B + 1), _device(weight, "weight", x.dtype, x, C),
                              _device(bias, "bias", x.dtype, x, C))


def _same_or_apart(what, to, given):
    """Refuses a contiguous tensor that is written and meets a part of another one, of as many values."""
    for name, t in given.items():
        if 0 < abs(to.data_ptr() - t.data_ptr()) < t.numel() * t.element_size():
            raise ValueError(f"{what} overlaps {name}: it must be {name} itself or lie apart")


def group_norm(x, groups, weight=None, bias=None, off=None, activation="none", eps=1e-5, with_stats=False, out=None):
    """act(group_norm(x) * weight + bias) over each image's rows and each group of channels, channels last
    (mpm_group_norm): the shape of x, and with ``with_stats`` float32 [B, groups, 2] for group_norm_backward.

    x: dense images [B, ..., C] (a rebuilt grid [B, N, C] or [B, rows, columns, C]) or packed rows [R, C] by ``off``
    [B + 1] (rows of no image are left as they are in ``out``). ``activation``: "none", "relu", "silu" or "gelu".
    ``out``: where to write, x itself or memory apart from it."""
    c = _group_call(x, groups, weight, bias, off, activation, eps)
    y = torch.empty_like(x) if out is None else out
    if y.shape != x.shape:
        raise ValueError(f"out must be {tuple(x.shape)}")
    yp = _device(y, "out", x.dtype, x)
    if out is not None:
        _same_or_apart("out", out, {"x": x})
    stats = torch.empty((c.B, c.groups, 2), dtype=torch.float32, device=x.device) if with_stats else None
    if c.R == 0:
        if with_stats:
            stats.zero_()
        return (y, stats) if with_stats else y
    need = _lib.load().mpm_group_norm_workspace_bytes(_BYREF(c))
    ws = _scratch(need, x)
    _launch("mpm_group_norm", x, _BYREF(c), _ptr(x), yp, _ptr(stats), _ptr(ws), need)
    return (y, stats) if with_stats else y


@dataclass
class GroupNormGrads:
    dx: torch.Tensor
    dweight: torch.Tensor | None
    dbias: torch.Tensor | None


def group_norm_backward(dy, x, stats, groups, weight=None, bias=None, off=None, activation="none", eps=1e-5,
                        dx=None) -> GroupNormGrads:
    """The gradients of group_norm() (mpm_group_norm_backward) from dy, the call's own inputs and its stats; zeros in rows
    of no image. ``dx``: where to write it, dy or x itself or memory apart from them."""
    c = _group_call(x, groups, weight, bias, off, activation, eps)
    g = GroupNormGrads(torch.empty_like(x) if dx is None else dx,
                       *(None if t is None else torch.empty_like(t) for t in (weight, bias)))
    if dy.shape != x.shape or g.dx.shape != x.shape:
        raise ValueError(f"dy and dx must be {tuple(x.shape)}")
    dp, gp = _device(dy, "dy", x.dtype, x), _device(g.dx, "dx", x.dtype, x)
    if dx is not None:
        _same_or_apart("dx", dx, {"dy": dy, "x": x})
    sp = _device(stats, "stats", torch.float32, x, 2 * c.B * c.groups)
    if c.R == 0:
        for t in (g.dweight, g.dbias):
            if t is not None:
                t.zero_()
        return g
    need = _lib.load().mpm_group_norm_backward_workspace_bytes(_BYREF(c))
    ws = _scratch(need, x)
    _launch("mpm_group_norm_backward", x, _BYREF(c), dp, _ptr(x), sp, gp, _ptr(g.dweight), _ptr(g.dbias), _ptr(ws), need)
    return g
