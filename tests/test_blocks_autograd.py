"""The autograd functions of the blocks on the CPU, over stand-ins that compute what the library's
operators promise: what autograd sees of them, not the kernels."""
import pytest
import torch

import block_refs as ref
from paper_2604_05718_amd import block_ops, blocks

D, H, GRID = 16, 2, (3, 4)
OFF = torch.tensor([0, 5, 12], dtype=torch.int32)
POS = torch.cat([torch.arange(5), torch.arange(7)]).to(torch.int32)


def bias_expand(table, lut):
    nb, W = int(table.shape[0] ** 0.5 + 0.5), lut.numel()
    l = lut.long()
    return table[(l[:, None] * nb + l[None, :]).reshape(-1)].t().reshape(table.shape[1], W, W)


class Operators:
    """The stand-ins, and the arguments of the last backward call."""

    def __init__(self):
        self.calls = {}

    def plain(self, q, k, v, bias, kw):
        imgs = ref.images(kw["q_off"], 0, 2)
        return ref.attention(q, k, v, imgs, imgs, q.shape[-1] ** -0.5, bias, kw["q_pos"], kw["k_pos"], kw["grid"])[0]

    def attention(self, q, k, v, bias=None, with_lse=True, **kw):
        out = self.plain(q.detach(), k.detach(), v.detach(), bias, kw)
        return out, torch.zeros(out.shape[:2] + (2,))

    def attention_backward(self, dout, q, k, v, out, lse, bias=None, dq=None, dk=None, dv=None, with_dbias=True, **kw):
        self.calls["attention"] = dict(with_dbias=with_dbias)
        with torch.enable_grad():
            leaf = [t.detach().requires_grad_() for t in (q, k, v, bias)]
            g = torch.autograd.grad((self.plain(*leaf, kw) * dout).sum(), leaf)
        for to, t in zip((dq, dk, dv), g):
            to.copy_(t)
        return block_ops.AttentionGrads(dq, dk, dv, g[3] if with_dbias else None)

    def bias_gradient(self, dbias, lut, nb, dtype=torch.float32):
        self.calls["table"] = True
        l = lut.long()
        cells = (l[:, None] * nb + l[None, :]).reshape(-1)
        return torch.zeros(nb * nb, dbias.shape[0], dtype=dtype).index_add_(0, cells, dbias.flatten(1).t().to(dtype))

    def norm(self, x, f, p, off, norm, eps):
        rows = None if off is None else torch.repeat_interleave(torch.arange(2), (off[1:] - off[:-1]).long())
        return ref.residual_norm(x, f, *p, rows_of=rows, norm=norm, eps=eps)

    def residual_norm(self, x, f, *p, off=None, norm="layer", eps=1e-6, with_stats=True):
        self.x = x.detach().clone()
        y, h = self.norm(x.detach(), f.detach(), [None if t is None else t.detach() for t in p], off, norm, eps)
        return y, h, torch.zeros(x.shape[0], 4)

    def residual_norm_backward(self, dy, dh, y, f, stats, *p, off=None, norm="layer", eps=1e-6):
        with torch.enable_grad():
            leaf = [None if t is None else t.detach().requires_grad_() for t in (self.x, f, *p)]
            wy, wh = self.norm(*leaf[:2], leaf[2:], off, norm, eps)
            some = [t for t in leaf if t is not None]
            g = iter(torch.autograd.grad((wy * dy).sum() + (wh * dh).sum(), some))
        return block_ops.NormGradients(*(None if t is None else next(g) for t in leaf))


@pytest.fixture
def operators(monkeypatch):
    ops = Operators()
    for n in ("attention", "attention_backward", "bias_gradient", "residual_norm", "residual_norm_backward"):
        monkeypatch.setattr(block_ops, n, getattr(ops, n))
    monkeypatch.setattr(block_ops, "bias_expand", bias_expand)
    return ops


def attention_inputs():
    g = torch.Generator().manual_seed(1)
    lut, nb = block_ops.bucket_lut(3, 2)
    qkv = torch.randn(12, 3 * H, D // H, generator=g, dtype=torch.float64, requires_grad=True)
    table = torch.randn(nb * nb, H, generator=g, dtype=torch.float64, requires_grad=True)
    off, pos = OFF.clone(), POS.clone()
    return qkv, table, lut, H, dict(q_off=off, k_off=off, Nq=7, Nk=7, q_pos=pos, k_pos=pos, grid=GRID)


def norm_inputs():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True)
    return [r(12, D), r(12, D), r(D), r(D), r(D), r(D), r(D), r(2, D), OFF.clone(), "layer", 1e-6]


def test_first_order(operators):
    """The functions hand the operators' gradients to the right inputs (against differences)."""
    qkv, table, *rest = attention_inputs()
    assert torch.autograd.gradcheck(lambda a, b: blocks._Attention.apply(a, b, *rest), (qkv, table))
    *p, off, norm, eps = norm_inputs()
    assert torch.autograd.gradcheck(lambda *a: blocks._ResidualNorm.apply(*a, off, norm, eps), p)


def test_second_order_raises(operators):
    """The kernels' gradients carry no history: differentiating them again is refused, alone, beside terms
    that have one, and by either way of asking; a graph that is not differentiated is no error."""
    def penalty(case, alone):
        if case == "attention":
            qkv, table, *rest = attention_inputs()
            out, x = blocks._Attention.apply(qkv, table, *rest), qkv
        else:
            *p, off, norm, eps = norm_inputs()
            y, out = blocks._ResidualNorm.apply(*p, off, norm, eps)
            out, x = y * out, p[1]
        g, = torch.autograd.grad(out.square().sum(), x, create_graph=True)
        return g.square().sum() + (0 if alone else out.sum()), x

    for case in ("attention", "norm"):
        for alone in (True, False):
            loss, x = penalty(case, alone)
            with pytest.raises(RuntimeError, match="differentiated once"):
                torch.autograd.grad(loss, x)
            loss, x = penalty(case, alone)
            with pytest.raises(RuntimeError, match="differentiated once"):
                loss.backward()


@pytest.mark.parametrize("name", ["q_off", "k_off", "q_pos", "k_pos"])
def test_written_buffers_of_the_attention_are_noticed(operators, name):
    """A buffer of offsets or positions that is reused before the backward pass is an error, not another
    gradient."""
    qkv, table, lut, heads, where = attention_inputs()
    where = {**where, "k_off": where["k_off"].clone(), "k_pos": where["k_pos"].clone()}
    out = blocks._Attention.apply(qkv, table, lut, heads, where)
    where[name].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_written_offsets_of_the_norms_are_noticed(operators):
    *p, off, norm, eps = norm_inputs()
    y, h = blocks._ResidualNorm.apply(*p, off, norm, eps)
    off.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (y + h).sum().backward()


@pytest.mark.parametrize("learned", [True, False])
def test_a_frozen_table_costs_no_gradient(operators, learned):
    qkv, table, *rest = attention_inputs()
    table.requires_grad_(learned)
    blocks._Attention.apply(qkv, table, *rest).sum().backward()
    assert operators.calls == dict(attention=dict(with_dbias=learned), **(dict(table=True) if learned else {}))
    assert qkv.grad is not None and (table.grad is not None) == learned


def test_strided_rows_of_the_norms(operators, monkeypatch):
    """The operators take contiguous rows; x as a view is copied like f."""
    def contiguous(x, f, *p, **kw):
        assert x.is_contiguous() and f.is_contiguous()
        return operators.residual_norm(x, f, *p, **kw)

    monkeypatch.setattr(block_ops, "residual_norm", contiguous)
    *p, off, norm, eps = norm_inputs()
    wide = [torch.cat([t, t], dim=1).detach().requires_grad_() for t in p[:2]]
    got = blocks._ResidualNorm.apply(wide[0][:, :D], wide[1][:, D:], *p[2:], off, norm, eps)
    want = blocks._ResidualNorm.apply(*p, off, norm, eps)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    (got[0] * got[1]).sum().backward()
    (want[0] * want[1]).sum().backward()
    assert torch.equal(wide[0].grad[:, :D], p[0].grad) and torch.equal(wide[1].grad[:, D:], p[1].grad)
