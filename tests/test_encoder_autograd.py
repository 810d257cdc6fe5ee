"""The autograd functions of rotated attention and of group norm, and the modules over them, on the CPU, over stand-ins
that compute what the library's operators promise: what autograd sees of them, not the kernels."""
import pytest
import torch

import block_refs
import encoder_refs as ref
from paper_2604_05718_amd import block_ops, blocks

H, DH, GRID = 2, 8, (3, 4)
OFF = torch.tensor([0, 5, 12], dtype=torch.int32)
POS = torch.cat([torch.arange(5), torch.arange(7)]).to(torch.int32)


class Operators:
    """The stand-ins, and the arguments of the last backward calls."""

    def __init__(self):
        self.calls = {}

    def plain(self, q, k, v, kw):
        imgs = block_refs.images(kw["q_off"], 0, 2)
        return block_refs.attention(q, k, v, imgs, imgs, q.shape[-1] ** -0.5)[0]

    def attention(self, q, k, v, with_lse=True, out=None, **kw):
        assert set(kw) == {"q_off", "k_off", "Nq", "Nk"}  # (no bias, no positions)
        assert out.shape == q.shape and out.is_contiguous() and not out.any()  # (rows of no image stay zero)
        out.copy_(self.plain(q.detach(), k.detach(), v.detach(), kw))
        return out, torch.zeros(out.shape[:2] + (2,))

    def attention_backward(self, dout, q, k, v, out, lse, dq=None, dk=None, dv=None, **kw):
        with torch.enable_grad():
            leaf = [t.detach().requires_grad_() for t in (q, k, v)]
            g = torch.autograd.grad((self.plain(*leaf, kw) * dout).sum(), leaf)
        for to, t in zip((dq, dk, dv), g):
            to.copy_(t)
        return block_ops.AttentionGrads(dq, dk, dv, None)

    def rotary(self, x, freq, pos=None, grid=(1,), layout="halves", off=None):
        return ref.turned(x.detach(), freq.detach(), ref.cells(pos, grid), layout)

    def rotary_backward(self, dout, x, freq, pos=None, grid=(1,), layout="halves", off=None, dx=None, with_dfreq=True):
        self.calls["rotary"] = dict(with_dfreq=with_dfreq, x=x)
        back = ref.turned(dout, freq.detach(), ref.cells(pos, grid), layout, -1.0)
        dfreq = None
        if with_dfreq:
            with torch.enable_grad():
                f = freq.detach().requires_grad_()
                dfreq, = torch.autograd.grad((ref.turned(x.detach(), f, ref.cells(pos, grid), layout) * dout).sum(), f)
        dx.copy_(back)
        return block_ops.RotaryGrads(dx, dfreq)

    def group(self, x, groups, w, b, off, activation, eps):
        rows = x.reshape(-1, x.shape[-1])
        if off is None:
            n = rows.shape[0] // x.shape[0]
            parts = [slice(i * n, (i + 1) * n) for i in range(x.shape[0])]
        else:
            parts = block_refs.images(off, 0, off.numel() - 1)
        return ref.group_norm(rows, groups, parts, w, b, activation, eps).view(x.shape)

    def group_norm(self, x, groups, weight=None, bias=None, off=None, activation="none", eps=1e-5, with_stats=False, out=None):
        assert x.is_contiguous()
        y = self.group(x.detach(), groups, weight.detach(), bias.detach(), off, activation, eps)
        return y, torch.zeros(2, groups, 2)

    def group_norm_backward(self, dy, x, stats, groups, weight=None, bias=None, off=None, activation="none", eps=1e-5):
        assert dy.is_contiguous()
        with torch.enable_grad():
            leaf = [t.detach().requires_grad_() for t in (x, weight, bias)]
            g = torch.autograd.grad((self.group(*leaf[:1], groups, *leaf[1:], off, activation, eps) * dy).sum(), leaf)
        return block_ops.GroupNormGrads(*g)


@pytest.fixture
def operators(monkeypatch):
    ops = Operators()
    for n in ("attention", "attention_backward", "rotary", "rotary_backward", "group_norm", "group_norm_backward"):
        monkeypatch.setattr(block_ops, n, getattr(ops, n))
    return ops


def attention_inputs(per_head=True):
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(12, 3 * H, DH, generator=g, dtype=torch.float64, requires_grad=True)
    freq = torch.randn((2 * H, 2, DH // 2) if per_head else (2, DH // 2), generator=g, dtype=torch.float64)
    off, pos = OFF.clone(), POS.clone()
    return (qkv, freq.requires_grad_(), H, dict(pos=pos, grid=GRID, off=off),
            dict(q_off=off.clone(), k_off=off.clone(), Nq=7, Nk=7))


def group_inputs(dense=False):
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True)
    return [r(2, 6, 8) if dense else r(12, 8), r(8), r(8), 4, None if dense else OFF.clone(), "silu", 1e-5]


@pytest.mark.parametrize("per_head", [True, False])
def test_rotary_attention(operators, per_head):
    """The functions hand the operators' gradients to the right inputs (against differences)."""
    qkv, freq, *rest = attention_inputs(per_head)
    assert torch.autograd.gradcheck(lambda a, f: blocks._RotaryAttention.apply(a, f, *rest), (qkv, freq))


@pytest.mark.parametrize("dense", [True, False])
def test_group_norm(operators, dense):
    *p, groups, off, act, eps = group_inputs(dense)
    assert torch.autograd.gradcheck(lambda *a: blocks._GroupNorm.apply(*a, groups, off, act, eps), p)
    wide = torch.cat([p[0], p[0]], dim=-1).detach().requires_grad_()  # a view is copied
    y = blocks._GroupNorm.apply(wide[..., 8:], *p[1:], groups, off, act, eps)
    assert torch.equal(y, blocks._GroupNorm.apply(*p, groups, off, act, eps))
    y.sum().backward()


def test_fixed_frequencies_cost_no_gradient(operators):
    qkv, freq, *rest = attention_inputs()
    blocks._RotaryAttention.apply(qkv, freq.detach(), *rest).sum().backward()
    assert operators.calls["rotary"] == dict(with_dfreq=False, x=None) and qkv.grad is not None


def test_second_order_raises(operators):
    for case in ("attention", "group"):
        if case == "attention":
            qkv, freq, *rest = attention_inputs()
            out, x = blocks._RotaryAttention.apply(qkv, freq, *rest), qkv
        else:
            *p, groups, off, act, eps = group_inputs()
            out, x = blocks._GroupNorm.apply(*p, groups, off, act, eps), p[0]
        g, = torch.autograd.grad(out.square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad(g.square().sum(), x)


@pytest.mark.parametrize("name", ["pos", "off", "q_off", "k_off"])
def test_written_buffers_are_noticed(operators, name):
    qkv, freq, heads, turn, where = attention_inputs()
    out = blocks._RotaryAttention.apply(qkv, freq, heads, turn, where)
    (turn if name in turn else where)[name].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    *p, groups, off, act, eps = group_inputs()
    y = blocks._GroupNorm.apply(*p, groups, off, act, eps)
    off.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_modules():
    """What the encoders' parameters are, and what products in 8 bits refuse."""
    kw = dict(device="cpu", dtype=torch.float32)
    enc = blocks.RotaryEncoder(32, 2, 2, (4, 5), learned=True, **kw)
    assert enc.blocks[0].freq.shape == (2, 2, 8) and isinstance(enc.blocks[0].freq, torch.nn.Parameter)
    assert torch.equal(enc.blocks[0].freq[1], block_ops.rotary_frequencies(8, 2))
    fixed = blocks.RotaryEncoder(32, 2, 1, (2, 4, 5), theta=50.0, **kw)
    assert fixed.blocks[0].freq.shape == (3, 8) and "freq" not in dict(fixed.blocks[0].named_parameters())
    assert "blocks.0.freq" in fixed.state_dict()
    old = blocks.RelativeEncoder(32, 2, 1, (4, 5), **kw)
    names = [n for n, _ in old.blocks[0].named_parameters()]
    assert names[:6] == ["qkv", "proj", "fc1", "fc2", "table", "attn_post_weight"]
    assert [n for n, _ in old.named_buffers()] == ["lut"]


def test_quantized_products(monkeypatch):
    """quantize() takes the weights [in, out] as rows of out channels; the products then go to linear_int8, the MLP's with its
    activation, and refuse gradients."""
    seen = []

    def quantize_rows(w):
        assert w.is_contiguous()
        return w.clone(), torch.ones(w.shape[0])

    def linear_int8(x, w, scale, activation="none"):
        seen.append((tuple(w.shape), activation))
        return ref.act((x @ w.t()), activation)

    monkeypatch.setattr(block_ops, "quantize_rows", quantize_rows)
    monkeypatch.setattr(block_ops, "linear_int8", linear_int8)
    enc = blocks.RotaryEncoder(16, 2, 1, (4, 5), device="cpu", dtype=torch.float32)
    head = blocks.GridHead(16, 24, 5, groups=4, device="cpu", dtype=torch.float32)
    blk, x = enc.blocks[0], torch.randn(3, 16)
    want = [blk.product("qkv", x), blk.product("fc1", x, "gelu"), head.product("inner", x)]
    assert not seen and enc.quantize() is enc and head.quantize() is head
    with pytest.raises(RuntimeError, match="no_grad"):
        blk.product("qkv", x)
    with torch.no_grad():
        got = [blk.product("qkv", x), blk.product("fc1", x, "gelu"), head.product("inner", x)]
    for a, b in zip(got, want):
        assert torch.allclose(a, b, atol=1e-5)
    assert seen == [((48, 16), "none"), ((64, 16), "gelu"), ((24, 16), "none")]
