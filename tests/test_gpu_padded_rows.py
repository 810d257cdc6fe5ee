"""Rows that belong to no image, before the first and behind the last, in training: they reach no gradient, whatever memory
held before, and get zeros."""
import pytest
import torch

import block_refs
import paper_2604_05718_amd as mpm
from paper_2604_05718_amd.blocks import GridHead, RelativeEncoder, RotaryEncoder

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
NAN = float("nan")


def dirt():
    """Leaves NaN in the memory that new tensors get."""
    held = [torch.full((n,), NAN, device=DEV) for n in (*range(1000, 60000, 1000), *([3000000] * 8))]
    del held


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [16, 264, 1000, 4104])
@pytest.mark.parametrize("ns,before,behind", [([5, 0, 9], 3, 6), ([1], 0, 1), ([40, 70], 300, 0), ([0, 0], 2, 5), ([6], 0, 0)])
def test_norms_with_a_gate_by_image(dtype, D, ns, before, behind):
    """residual_norm() and its gradients: the rows of images as without the others, zeros in those, and in a given out
    what was there."""
    g = torch.Generator().manual_seed(D)
    n, R = sum(ns), sum(ns) + before + behind
    rnd = lambda *s: torch.randn(s, generator=g).to(dtype).to(DEV)
    x, f, dy, dh = (rnd(R, D) for _ in range(4))
    inside = slice(before, before + n)
    for t in (x, f, dy, dh):
        t[:before] = NAN
        t[before + n:] = NAN
    w, b, pw, pb, sc, gate = rnd(D), rnd(D), rnd(D), rnd(D), rnd(D), rnd(len(ns), D)
    off = torch.cumsum(torch.tensor([before] + ns), 0).to(torch.int32).to(DEV)
    p = (w, b, pw, pb, sc, gate)
    dirt()
    y, h, stats = mpm.residual_norm(x, f, *p, off=off, with_stats=True)
    d = mpm.residual_norm_backward(dy, dh, y, f, stats, *p, off=off)
    for t in (y, h, d.dx, d.df):
        assert not t[:before].any() and not t[before + n:].any()
    out = torch.full_like(x, 7)
    y2, h2 = mpm.residual_norm(x, f, *p, off=off, out=out)
    assert y2 is out and torch.equal(h2, h) and torch.equal(out[inside], y[inside])
    assert bool((out[:before] == 7).all() and (out[before + n:] == 7).all())
    same = x.clone()
    mpm.residual_norm(same, f, *p, off=off, out=same)
    assert torch.equal(same[inside], y[inside]) and same[:before].isnan().all() and same[before + n:].isnan().all()
    if n:  # (the gradients' rows are dealt to workgroups by the number of all rows: sums in another order)
        y3, h3, st = mpm.residual_norm(x[inside].contiguous(), f[inside].contiguous(), *p, off=off - before, with_stats=True)
        d3 = mpm.residual_norm_backward(dy[inside].contiguous(), dh[inside].contiguous(), y3, f[inside].contiguous(), st, *p,
                                        off=off - before)
        assert torch.equal(y3, y[inside]) and torch.equal(h3, h[inside])
        assert torch.equal(d3.dx, d.dx[inside]) and torch.equal(d3.df, d.df[inside])
        half = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24
        for a, b in ((d3.dweight, d.dweight), (d3.dbias, d.dbias), (d3.dpost_weight, d.dpost_weight),
                     (d3.dpost_bias, d.dpost_bias), (d3.dscale, d.dscale), (d3.dgate, d.dgate)):
            # a rounding of each, and n + 16 sums of each in float32, of terms up to about 8 times the sums
            assert block_refs.rel(a, b.double().cpu()) <= 2 * half + 2 * 8 * (n + 16) * 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(4, 4), (6, 2)])
@pytest.mark.parametrize("ns,before,behind", [([50, 0, 90], 3, 6), ([1], 0, 1), ([2, 3], 1, 0), ([400], 200, 300), ([6], 0, 0)])
def test_attention(dtype, H, Hk, ns, before, behind):
    """attention() and its gradients into columns of wider rows, with and without `clear`; few and many queries."""
    g = torch.Generator().manual_seed(H)
    n, R, dh = sum(ns), sum(ns) + before + behind, 32
    off = torch.cumsum(torch.tensor([before] + ns), 0).to(torch.int32).to(DEV)
    where = dict(q_off=off, k_off=off, Nq=max(ns), Nk=max(ns))
    rows = torch.randn((R, H + 2 * Hk, dh), generator=g).to(dtype).to(DEV)
    dout = torch.randn((R, H, dh), generator=g).to(dtype).to(DEV)
    for t in (rows, dout):
        t[:before] = NAN
        t[before + n:] = NAN
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    inside, res = slice(before, before + n), {}
    for clear in (True, False):
        wide = torch.full((R, H + 1, dh), 7.0, device=DEV, dtype=dtype)
        out, lse = mpm.attention(q, k, v, with_lse=True, out=wide[:, :H], clear=clear, **where)
        grad = torch.full((R, H + 2 * Hk + 1, dh), 7.0, device=DEV, dtype=dtype)
        mpm.attention_backward(dout, q, k, v, out, lse, dq=grad[:, :H], dk=grad[:, H:H + Hk], dv=grad[:, H + Hk:-1],
                               clear=clear, **where)
        assert bool((wide[:, H:] == 7).all() and (grad[:, -1:] == 7).all())  # (the columns beside them)
        for t in (wide[:, :H], grad[:, :-1]):
            assert bool((t[:before] == (0 if clear else 7)).all() and (t[before + n:] == (0 if clear else 7)).all())
        res[clear] = wide[inside], grad[inside]
    for a, b in zip(res[True], res[False]):
        assert a.isfinite().all() and torch.equal(a, b)


ENCODERS = {"rotary": lambda D, grid: RotaryEncoder(D, 2, 2, grid, learned=True, device=DEV, dtype=torch.float32),
            "relative": lambda D, grid: RelativeEncoder(D, 2, 2, grid, device=DEV, dtype=torch.float32)}


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("kind", list(ENCODERS))
def test_gradients_of_a_padded_batch(kind, gated):
    """Encoder and head: rows, their gradient and every parameter's as on the rows of the images alone. Float32: 288 half
    steps of each operator, through eight products in a row 16 times that, as the encoders' own tests have it."""
    torch.manual_seed(4)
    ns, before, behind, D, grid = [30, 17, 33], 5, 9, 48, (8, 9)
    enc = ENCODERS[kind](D, grid)
    head = GridHead(D, 64, 10, groups=8, device=DEV, dtype=torch.float32)
    n, R = sum(ns), sum(ns) + before + behind
    pos = torch.cat([torch.zeros(before, dtype=torch.int64)] + [torch.randperm(72)[:k].sort().values for k in ns]
                    + [torch.zeros(behind, dtype=torch.int64)]).to(torch.int32).to(DEV)
    x, g = torch.randn(R, D), torch.randn(R, 10)
    gate = (torch.rand(len(ns), D) + 0.5).to(DEV).requires_grad_()
    off = torch.cumsum(torch.tensor([before] + ns), 0).to(torch.int32).to(DEV)

    def step(rows, off):
        dirt()
        first = int(off[0])
        xd = x[rows].to(DEV).requires_grad_()
        y = head(enc.rows(xd, off, max(ns), pos[rows], gate if gated else None), off)
        params = {"x": xd, **({"gate": gate} if gated else {}), **{"enc." + k: t for k, t in enc.named_parameters()},
                  **{"head." + k: t for k, t in head.named_parameters()}}
        inside = slice(first, first + n)
        loss = (y[inside] * g[before:before + n].to(DEV)).sum()
        return y[inside].detach(), dict(zip(params, torch.autograd.grad(loss, list(params.values()))))

    y, grads = step(slice(before, before + n), off - before)
    yp, padded = step(slice(0, R), off)
    tol = 16 * 288 * 2.0 ** -24
    assert block_refs.rel(yp, y.double().cpu()) <= tol
    dx = padded["x"]
    assert not dx[:before].any() and not dx[before + n:].any()
    padded["x"] = dx[before:before + n]
    for k, t in grads.items():
        assert block_refs.rel(padded[k], t.double().cpu()) <= tol, k
