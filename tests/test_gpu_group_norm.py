"""Group norm with an activation on the GPU against the plain 64-bit form, and its gradients against the formulas
and against differences."""
import math

import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def inputs(lengths, C, dtype, seed, shift=1.0):
    g = torch.Generator().manual_seed(seed)
    R = sum(lengths)
    x = (torch.randn((R, C), generator=g) * 1.5 + torch.randn(C, generator=g) * shift).to(dtype)
    dy = torch.randn((R, C), generator=g).to(dtype)
    w, b = (1 + 0.2 * torch.randn(C, generator=g)).to(dtype), (0.1 * torch.randn(C, generator=g)).to(dtype)
    off = torch.cumsum(torch.tensor([0] + list(lengths)), 0).to(torch.int32)
    return x, dy, w, b, off


def slices(off, R=None):
    o = off.tolist()
    return [slice(a, b) for a, b in zip(o, o[1:])]


def rel(got, want, size=None):
    """2-norm of the difference over that of the result, or of what it is a sum of where terms cancel."""
    got, want = got.double().cpu(), want.detach().double()
    n = float((want if size is None else size).norm())
    return float((got - want).norm()) / n if n else float((got - want).norm())


# By the 2-norm: float32 values through a dozen operations, each a half step 2^-24 of terms up to 8 times the result (t w + b
# and the activation's argument, rows with a shift): 96 half steps. Bfloat16: its rounding, and that.
TOL = {torch.float32: 96 * 2.0 ** -24, torch.bfloat16: 2.0 ** -8 + 96 * 2.0 ** -24}

SHAPES = [  # lengths, C, groups
    ((1,), 8, 1), ((1, 2, 1), 8, 8), ((5, 0, 17), 16, 2), ((64,), 32, 32), ((118,), 192, 32), ((70, 3, 200, 0), 72, 9),
    ((1024,), 192, 32), ((333, 1024), 768, 32), ((900,), 48, 3), ((50, 60), 264, 11), ((40,), 2056, 8), ((7, 9), 4104, 1),
    ((3,), 16384, 4), ((2500, 100), 24, 1), ((31,) * 20, 40, 5), ((2000, 4096), 64, 4), ((1200, 1), 1024, 32),
    ((1500,), 1024, 1), ((700, 0, 900, 1), 2056, 2), ((2000, 30), 1032, 3),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}x{max(s[0])}-{s[1]}-{s[2]}")
def test_group_norm(dtype, activation, shape):
    lengths, C, G = shape
    x, dy, w, b, off = inputs(lengths, C, dtype, C + G + len(lengths))
    affine = activation != "none" or C % 16 == 0
    kw = dict(weight=w.to(DEV) if affine else None, bias=b.to(DEV) if affine else None, off=off.to(DEV), activation=activation)
    y, stats = mpm.group_norm(x.to(DEV), G, with_stats=True, **kw)
    assert torch.equal(mpm.group_norm(x.to(DEV), G, **kw), y)
    leaf = [t.double().requires_grad_() for t in (x, w, b)]
    want = ref.group_norm(leaf[0], G, slices(off), *(leaf[1:] if affine else ()), activation=activation)
    assert rel(y, want) <= TOL[dtype]
    g = mpm.group_norm_backward(dy.to(DEV), x.to(DEV), stats, G, **kw)
    grads = torch.autograd.grad((want * dy.double()).sum(), leaf[:3 if affine else 1])
    # dx subtracts means from gt: for groups of one or two values it cancels to nothing, so its scale is that of gt rstd.
    scale = torch.ones(G).repeat_interleave(C // G).double() if not affine else w.double()
    rstd = torch.cat([stats[i, :, 1].double().cpu().repeat_interleave(C // G).expand(n, C) for i, n in enumerate(lengths)])
    size = dy.double() * scale * rstd
    assert rel(g.dx, grads[0], size if C // G * min(n for n in lengths if n) < 64 else None) <= 2 * TOL[dtype]
    if affine:
        # sums of R terms: each off as the terms are, and the sum of at most 4096 / 2 a thread and 64 more by their half steps
        terms = (dy.double().square().sum(dim=0) * 2).sqrt()
        tol = HALF[dtype] + (96 + 64) * 2.0 ** -24
        for got, need in ((g.dweight, grads[1]), (g.dbias, grads[2])):
            assert float((got.double().cpu() - need).norm()) <= tol * max(float(need.norm()), float(terms.norm()))
    else:
        assert g.dweight is None and g.dbias is None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_dense_grids(dtype):
    """[B, N, C] and [B, rows, columns, C]: equal to packed images of equal lengths; in place too."""
    x, dy, w, b, off = inputs((60,) * 3, 96, dtype, 1)
    xd, gd, wd, bd = (t.to(DEV) for t in (x, dy, w, b))
    y, stats = mpm.group_norm(xd, 8, wd, bd, off=off.to(DEV), activation="silu", with_stats=True)
    g = mpm.group_norm_backward(gd, xd, stats, 8, wd, bd, off=off.to(DEV), activation="silu")
    for shape in ((3, 60, 96), (3, 10, 6, 96)):
        v, s = mpm.group_norm(xd.view(shape), 8, wd, bd, activation="silu", with_stats=True)
        assert v.shape == shape and torch.equal(v.view(180, 96), y) and torch.equal(s, stats)
        h = mpm.group_norm_backward(gd.view(shape), xd.view(shape), s, 8, wd, bd, activation="silu")
        assert torch.equal(h.dx.view(180, 96), g.dx) and torch.equal(h.dweight, g.dweight) and torch.equal(h.dbias, g.dbias)
    for keep in ("dy", "x"):
        xc, gc = xd.clone(), gd.clone()
        to = gc if keep == "dy" else xc
        h = mpm.group_norm_backward(gc, xc, stats, 8, wd, bd, off=off.to(DEV), activation="silu", dx=to)
        assert torch.equal(to, g.dx) and torch.equal(h.dweight, g.dweight)
    assert torch.equal(mpm.group_norm(xd, 8, wd, bd, off=off.to(DEV), activation="silu", out=xd), y)


def test_rows_of_no_image():
    """Left as they were in the result, zeros in the gradient, whatever they hold."""
    x, dy, w, b, _ = inputs((300,), 40, torch.float32, 2)
    off = torch.tensor([9, 9, 100, 170], dtype=torch.int32)
    x[:9] = math.nan
    x[170:] = math.inf
    dy[170:] = math.nan
    out = torch.full_like(x, 3.0).to(DEV)
    kw = dict(weight=w.to(DEV), bias=b.to(DEV), off=off.to(DEV), activation="relu")
    y, stats = mpm.group_norm(x.to(DEV), 5, with_stats=True, out=out, **kw)
    assert bool((y[:9] == 3).all()) and bool((y[170:] == 3).all()) and not stats[0].any()
    leaf = [t.double().requires_grad_() for t in (x, w, b)]
    want = ref.group_norm(leaf[0], 5, slices(off), *leaf[1:], activation="relu")
    assert rel(y[9:170], want) <= TOL[torch.float32]
    g = mpm.group_norm_backward(dy.to(DEV), x.to(DEV), stats, 5, **kw)
    assert not g.dx[:9].any() and not g.dx[170:].any()
    grads = torch.autograd.grad((want * dy[9:170].double()).sum(), leaf)
    assert rel(g.dx[9:170], grads[0][9:170]) <= 2 * TOL[torch.float32]
    assert rel(g.dweight, grads[1]) <= 2 * TOL[torch.float32] and rel(g.dbias, grads[2]) <= 2 * TOL[torch.float32]


@pytest.mark.parametrize("n", [40, 3000])
def test_values_far_from_zero(n):
    """A mean 2^12 times the deviation: the variance keeps its digits (values a half step of 2^12 apart are inputs, not errors);
    t is off by the mean's half step, 2^-12 of the deviation."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((n, 16), generator=g) + 4096.0
    x[0] = -1e4  # a first value far off is no reference to subtract
    x[0, 8:] = 4096.0
    y, stats = mpm.group_norm(x.to(DEV).view(1, n, 16), 2, with_stats=True)
    want = ref.group_norm(x.double(), 2, [slice(0, n)])
    assert rel(y[0], want) <= 4 * 2.0 ** -12
    v = x[:, 8:].double()
    assert abs(float(stats[0, 1, 1]) * math.sqrt(float(v.var(correction=0)) + 1e-5) - 1) < 64 * 2.0 ** -24
    assert abs(float(stats[0, 1, 0]) - float(v.mean())) <= 4096 * 2.0 ** -23


def test_nan_stays_in_its_group():
    x, dy, w, b, off = inputs((50, 70), 32, torch.bfloat16, 4)
    x[60, 9] = math.nan
    y, stats = mpm.group_norm(x.to(DEV), 4, w.to(DEV), b.to(DEV), off=off.to(DEV), activation="relu", with_stats=True)
    bad = torch.zeros((120, 32), dtype=torch.bool)
    bad[50:, 8:16] = True
    assert torch.equal(y.isnan().cpu(), bad)
    g = mpm.group_norm_backward(dy.to(DEV), x.to(DEV), stats, 4, w.to(DEV), b.to(DEV), off=off.to(DEV), activation="silu")
    assert torch.equal(g.dx.isnan().cpu(), bad)


def test_gradients_against_differences():
    """dx, dw and db against differences of the 64-bit form (a step of 1e-5: off by about 1e-9 of values near 1)."""
    x, dy, w, b, off = inputs((9, 5), 12, torch.float32, 5)
    y, stats = mpm.group_norm(x.to(DEV), 3, w.to(DEV), b.to(DEV), off=off.to(DEV), activation="gelu", with_stats=True)
    g = mpm.group_norm_backward(dy.to(DEV), x.to(DEV), stats, 3, w.to(DEV), b.to(DEV), off=off.to(DEV), activation="gelu")
    loss = lambda *t: float((ref.group_norm(t[0], 3, slices(off), t[1], t[2], "gelu") * dy.double()).sum())
    at = [x.double(), w.double(), b.double()]
    for i, got in enumerate((g.dx, g.dweight, g.dbias)):
        for k in range(0, at[i].numel(), 7):
            e = torch.zeros(at[i].numel(), dtype=torch.float64)
            e[k] = 1e-5
            up, down = (loss(*(t + s * e.view(t.shape) if j == i else t for j, t in enumerate(at))) for s in (1, -1))
            assert abs((up - down) / 2e-5 - float(got.view(-1)[k])) < 1e-4


def test_same_results_every_time_and_under_capture():
    for lengths, C in (((100, 57), 64), ((1500, 2000, 800), 256), ((6000,), 96)):
        x, dy, w, b, off = (t.to(DEV) for t in inputs(lengths, C, torch.bfloat16, 6))

        def step():
            y, stats = mpm.group_norm(x, 8, w, b, off=off, activation="silu", with_stats=True)
            g = mpm.group_norm_backward(dy, x, stats, 8, w, b, off=off, activation="silu")
            return y, stats, g.dx, g.dweight, g.dbias

        want = step()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for k in range(4):
            for t in got:
                t.fill_(k)
            again = step()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, again))
