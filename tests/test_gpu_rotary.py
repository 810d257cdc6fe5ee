"""Rotary positions on the GPU against the plain 64-bit form, and their gradients against the formulas and
against differences."""
import math

import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step of a rounding
# What a sine or cosine is off, and the two products: float32 2^-23.3 (the fraction of a turn rounded) + 2^-22 (the
# functions) + 2^-23; bfloat16 the processor's, 2^-19, likewise.
TRIG = {torch.bfloat16: 2.0 ** -18, torch.float32: 2.0 ** -21}


def frequencies(kind, H, axes, P, g):
    if kind == "fixed":
        return mpm.rotary_frequencies(P, axes)
    return torch.randn((H, axes, P) if kind == "heads" else (axes, P), generator=g) * 0.4


def near(got, want, x, P, layout, dtype, angle=0.0):
    got = got.double().cpu()
    off = (got - want).abs() - HALF[dtype] * want.abs() - (TRIG[dtype] + angle) * ref.pair_sizes(x, P, layout)
    assert float(off.max()) <= 0, float(off.max())


SHAPES = [  # R, H, dh, P, grid
    (1, 1, 8, 4, (5,)), (1, 12, 64, 32, (32, 32)), (3, 5, 40, 13, (7, 9)), (118, 6, 64, 32, (14, 14)),
    (257, 3, 80, 40, (3, 9, 11)), (65, 2, 128, 64, (64, 64)), (30, 130, 64, 32, (8, 8)), (19, 17, 128, 63, (4, 5, 6)),
    (2000, 1, 16, 1, (50, 40)), (77, 4, 24, 12, (9, 9)), (41, 2, 96, 42, (6, 7)),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("kind", ["fixed", "shared", "heads"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotary(dtype, layout, kind, shape):
    R, H, dh, P, grid = shape
    g = torch.Generator().manual_seed(R * 31 + H + dh)
    x = torch.randn((R, H, dh), generator=g).to(dtype)
    d = torch.randn((R, H, dh), generator=g).to(dtype)
    freq = frequencies(kind, H, len(grid), P, g)
    pos = torch.randint(0, math.prod(grid), (R,), generator=g, dtype=torch.int32)
    c = ref.cells(pos, grid)
    where = dict(pos=pos.to(DEV), grid=grid, layout=layout)
    out = mpm.rotary(x.to(DEV), freq.to(DEV), **where)
    f64, x64, d64 = freq.double().requires_grad_(), x.double().requires_grad_(), d.double()
    want = ref.turned(x64, f64, c, layout)
    near(out, want.detach(), x64.detach(), P, layout, dtype)
    back = mpm.rotary(x.to(DEV), freq.to(DEV), inverse=True, **where)
    near(back, ref.turned(x.double(), freq.double(), c, layout, -1.0), x.double(), P, layout, dtype)
    grads = mpm.rotary_backward(d.to(DEV), x.to(DEV), freq.to(DEV), **where)
    dx, df = torch.autograd.grad((want * d64).sum(), [x64, f64])
    near(grads.dx, dx, d64, P, layout, dtype)
    # each term c_a (x_1 dx_2 - x_2 dx_1) is off by TRIG (|x_1| + |x_2|) (|d_1| + |d_2|) and three roundings; a sum of at
    # most 16 rows a thread and 512 threads by 528 more
    i = slice(0, P) if layout == "halves" else slice(0, 2 * P, 2)
    size = ref.pair_sizes(x.double(), P, layout)[..., i] * ref.pair_sizes(d64, P, layout)[..., i]
    size = torch.einsum("ra,rhp->hap", c, size)
    size = size if kind == "heads" else size.sum(dim=0)
    assert grads.dfreq.dtype is torch.float32
    assert bool(((grads.dfreq.double().cpu() - df).abs() <= (TRIG[dtype] + 531 * 2.0 ** -24) * size).all())
    plain = mpm.rotary_backward(d.to(DEV), None, freq.to(DEV), with_dfreq=False, **where)
    assert plain.dfreq is None and torch.equal(plain.dx, grads.dx)


def test_sine_of_bfloat16_calls():
    """The processor's sine and cosine over a whole turn stay below 2^-19."""
    n = 4096
    x = torch.zeros((n, 1, 8), dtype=torch.bfloat16, device=DEV)
    x[:, :, 0] = 1.0
    freq = torch.tensor([[2 * math.pi / n]], dtype=torch.float32, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    # d = (1, 0), x = (1, 0): dx = (cos, -sin), so one row's dfreq (in float32) is c dx_2 = -c sin; with x = (0, 1) it
    # is -c cos
    worst = 0.0
    for k in range(1, n, 37):
        for i, f in ((0, math.sin), (1, math.cos)):
            y = torch.zeros((1, 1, 8), dtype=torch.bfloat16, device=DEV)
            y[..., i] = 1.0
            got = mpm.rotary_backward(x[:1], y, freq, pos=pos[k:k + 1], grid=(n,)).dfreq
            worst = max(worst, abs(-float(got) / k - f(k * float(freq))))
    assert worst < 2.0 ** -19, math.log2(worst)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("side", [2 ** 24, 2 ** 31 - 1])
def test_far_cells(dtype, side):
    """Cells far from the first: the angle's fraction is right where 32 bits hold few digits of it, or none. An angle in
    64 bits, here and in the plain form, is a product and a factor 1 / (2 pi) or a function of it: together at most
    8 half steps 2^-53 of it, 3 side at most."""
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(0, side, (64,), generator=g).to(torch.int32)
    pos[0] = side - 1
    x = torch.randn((64, 2, 16), generator=g).to(dtype)
    freq = torch.rand((1, 8), generator=g) * 3
    out = mpm.rotary(x.to(DEV), freq.to(DEV), pos=pos.to(DEV), grid=(side,))
    near(out, ref.turned(x.double(), freq.double(), ref.cells(pos, (side,))), x.double(), 8, "halves", dtype,
         3 * side * 2.0 ** -50)


def test_views_in_place_and_dense():
    """Queries and keys inside a projection's rows, turned where they stand; dense images count their rows."""
    g = torch.Generator().manual_seed(4)
    B, N, H = 3, 35, 4
    qkv = torch.randn((B, N, 3 * H, 64), generator=g).to(torch.bfloat16).to(DEV)
    before = qkv.clone()
    freq = mpm.rotary_frequencies(20, 2).to(DEV)
    view = qkv[:, :, :2 * H]
    want = mpm.rotary(before[:, :, :2 * H].contiguous(), freq, grid=(5, 7))
    got = mpm.rotary(view, freq, grid=(5, 7), out=view)
    assert got.data_ptr() == qkv.data_ptr() and torch.equal(qkv[:, :, :2 * H], want)
    assert torch.equal(qkv[:, :, 2 * H:], before[:, :, 2 * H:])
    pos = torch.arange(N, dtype=torch.int32, device=DEV).repeat(B)
    rows = before[:, :, :2 * H].reshape(B * N, 2 * H, 64)
    assert torch.equal(mpm.rotary(rows, freq, pos=pos, grid=(5, 7)).view(B, N, 2 * H, 64), want)
    # every second row, heads in another order of strides
    odd = before.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)[0]
    assert torch.equal(mpm.rotary(odd[::2], freq, pos=pos[:N:2].contiguous(), grid=(5, 7))[:, :2 * H], want[0, ::2])
    # back again, in place: the inverse undoes it to two roundings
    mpm.rotary(view, freq, grid=(5, 7), inverse=True, out=view)
    size = ref.pair_sizes(before[:, :, :2 * H].double().cpu(), 20, "halves")
    off = (view.double() - before[:, :, :2 * H].double()).abs().cpu() - (2 * 2.0 ** -8 + 2 * TRIG[torch.bfloat16]) * size
    assert float(off.max()) <= 0


@pytest.mark.parametrize("given", [True, False])
def test_rows_of_no_image(given):
    """A buffer with rows before and behind the images: left as they were, whatever they hold; zeros in the gradient."""
    g = torch.Generator().manual_seed(5)
    R, H, dh, grid = 300, 2, 32, (10, 10)
    off = torch.tensor([7, 7, 60, 61, 61, 140], dtype=torch.int32)
    x = torch.randn((R, H, dh), generator=g)
    x[:7] = math.nan
    x[140:] = math.inf
    pos = torch.full((R,), -5, dtype=torch.int32)
    index = torch.cat([torch.arange(int(b - a)) for a, b in zip(off, off[1:])]).to(torch.int32)
    pos[7:140] = torch.randint(0, 100, (133,), generator=g, dtype=torch.int32) if given else index
    freq = torch.randn((2, 12), generator=g)
    where = dict(pos=pos.to(DEV) if given else None, grid=grid, off=off.to(DEV))
    out = torch.full((R, H, dh), 5.0, device=DEV)
    mpm.rotary(x.to(DEV), freq.to(DEV), out=out, **where)
    assert bool((out[:7] == 5).all()) and bool((out[140:] == 5).all())
    f64, rows = freq.double().requires_grad_(), x[7:140].double()
    want = ref.turned(rows, f64, ref.cells(pos[7:140], grid))
    near(out[7:140], want.detach(), rows, 12, "halves", torch.float32)
    d = torch.randn((R, H, dh), generator=g)
    d[140:] = math.nan
    grads = mpm.rotary_backward(d.to(DEV), x.to(DEV), freq.to(DEV), **where)
    assert not grads.dx[:7].any() and not grads.dx[140:].any()
    df, = torch.autograd.grad((want * d[7:140].double()).sum(), f64)
    assert float((grads.dfreq.double().cpu() - df).norm() / df.norm()) < 528 * 2.0 ** -24
    in_place = d.to(DEV)
    assert torch.equal(mpm.rotary_backward(in_place, x.to(DEV), freq.to(DEV), dx=in_place, **where).dx, grads.dx)


def test_cells_outside_the_grid():
    pos = torch.tensor([-1, -2 ** 31, 12, 2 ** 31 - 1, 5], dtype=torch.int32)
    x = torch.randn((5, 1, 8), generator=torch.Generator().manual_seed(6))
    freq = torch.tensor([[0.3, 0.1], [0.2, 0.7]])
    out = mpm.rotary(x.to(DEV), freq.to(DEV), pos=pos.to(DEV), grid=(3, 4))
    near(out, ref.turned(x.double(), freq.double(), ref.cells(pos, (3, 4))), x.double(), 2, "halves", torch.float32)


def test_gradient_against_differences():
    """dfreq against differences of the 64-bit form: (L(f + h) - L(f - h)) / 2h is off by h^2 / 6 of the third
    derivative, at most c^3 (|x_1| + |x_2|) (|d_1| + |d_2|)."""
    g = torch.Generator().manual_seed(7)
    x, d = torch.randn((23, 3, 16), generator=g), torch.randn((23, 3, 16), generator=g)
    freq = torch.randn((3, 2, 6), generator=g) * 0.5
    pos = torch.randint(0, 20, (23,), generator=g, dtype=torch.int32)
    c = ref.cells(pos, (4, 5))
    got = mpm.rotary_backward(d.to(DEV), x.to(DEV), freq.to(DEV), pos=pos.to(DEV), grid=(4, 5), layout="pairs").dfreq.cpu()
    h = 1e-5
    for k in range(0, freq.numel(), 5):
        e = torch.zeros(freq.numel(), dtype=torch.float64)
        e[k] = h
        up, down = (float((ref.turned(x.double(), freq.double() + s * e.view(freq.shape), c, "pairs") * d.double()).sum())
                    for s in (1, -1))
        assert abs((up - down) / (2 * h) - float(got.view(-1)[k])) < 1e-3


def test_same_results_every_time_and_under_capture():
    """Bit for bit the same on every run, also replayed from a graph with eager work between."""
    g = torch.Generator().manual_seed(8)
    R, H = 3000, 8
    x, d = (torch.randn((R, H, 64), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    freq = (torch.randn((H, 3, 32), generator=g) * 0.3).to(DEV)
    pos = torch.randint(0, 4096, (R,), generator=g, dtype=torch.int32).to(DEV)
    where = dict(pos=pos, grid=(4, 32, 32), layout="pairs")

    def step():
        r = mpm.rotary_backward(d, x, freq, **where)
        return mpm.rotary(x, freq, **where), r.dx, r.dfreq

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
