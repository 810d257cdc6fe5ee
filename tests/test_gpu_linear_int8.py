"""Rows in 8-bit steps and products of them on the GPU, against exact integers."""
import math

import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 8), (5, 24), (3, 200), (130, 512), (67, 768), (9, 836 + 4), (33, 1024), (2, 1032),
                                 (7, 4096), (3, 8200), (2, 65536), (70000, 16)])
def test_quantize(dtype, R, K):
    """Steps and scales equal to the definition, value for value; zeros past K."""
    g = torch.Generator().manual_seed(R + K)
    x = (torch.randn((R, K), generator=g) * torch.exp(torch.randn(K, generator=g))).to(dtype)
    q, scale = mpm.quantize_rows(x.to(DEV))
    want, s = ref.steps(x.float())
    assert q.shape == (R, (K + 15) // 16 * 16)
    assert torch.equal(scale.cpu(), s) and torch.equal(q.cpu()[:, :K], want) and not q[:, K:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_quantize_borders(dtype):
    """Halves (scale 1: ties to even), values next to one, rows of zeros, of the smallest and of the largest numbers,
    and rows that are not finite."""
    tiny = 2.0 ** -133 if dtype is torch.bfloat16 else 2.0 ** -149
    most = torch.finfo(dtype).max
    halves = torch.arange(-126.5, 127.5, 1.0)[:248]
    rows = [torch.cat([halves, torch.tensor([127.0] * 8)]), torch.zeros(256), torch.full((256,), tiny),
            torch.linspace(-1, 1, 256) * most, torch.full((256,), -most), torch.linspace(-3, 3, 256) * 2.0 ** -120,
            torch.linspace(-3, 3, 256) * 2.0 ** -127]
    bad = torch.linspace(-1, 1, 256)
    for v in (math.nan, math.inf, -math.inf):
        b = bad.clone()
        b[200] = v
        rows.append(b)
    x = torch.stack(rows).to(dtype)
    near = (torch.randint(-127, 127, (2000, 256), generator=torch.Generator().manual_seed(1)).float() + 0.5)
    s = torch.rand((2000, 1), generator=torch.Generator().manual_seed(2)) + 0.5
    near = near * s
    near[:, 0] = 127 * s[:, 0]
    x = torch.cat([x, near.to(dtype)])  # products next to a half, on either side by a rounding or on it
    q, scale = mpm.quantize_rows(x.to(DEV))
    want, ws = ref.steps(x.float())
    assert torch.equal(scale.cpu().nan_to_num(-1), ws.nan_to_num(-1)) and torch.equal(q.cpu(), want)
    assert scale[7:10].isnan().all() and not q[7:10].any()
    eye, eye_scale = mpm.quantize_rows(torch.eye(256, device=DEV))
    y = mpm.linear_int8(x[:12].to(DEV), eye, eye_scale)
    assert y[7:10].isnan().all()
    # every other row is finite, but for products of the stored scales that float32 rounds past its largest number
    real = (want[:7].double() * 127 * ws[:7].double()[:, None] * eye_scale.double().cpu()).abs()
    assert bool((y[:7].isfinite().cpu() | (real * (1 + 4 * 2.0 ** -24) > torch.finfo(dtype).max)).all())


def test_quantize_strided_rows():
    x = torch.randn((40, 96), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    for view in (x[:, 16:80], x[::3, :40], x[5:6, 8:]):
        for a, b in zip(mpm.quantize_rows(view), mpm.quantize_rows(view.contiguous())):
            assert torch.equal(a, b)


def expected(q, s, w, ws, bias, activation):
    """(the result in 64 bits, what one half step of float32 may move it): the integer sum rounded, two scales, a shift."""
    sums = (q.double() @ w.double().T)
    z = sums * s.double()[:, None] * ws.double()[None, :]
    size = z.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    return ref.act(z, activation), size


def near(got, q, s, w, ws, bias, activation, dtype):
    want, size = expected(q, s, w, ws, bias, activation)
    # z is off by 4 half steps of its terms; an activation's slope is at most 1.13, and its own error (float32: a few
    # steps of the function; bfloat16: 2^-20 of the sigmoid's exponential) times |z|
    own = {"none": 0.0, "relu": 0.0}.get(activation, 2.0 ** -20) * want.abs().clamp_min(size)
    if activation == "gelu" and dtype is torch.bfloat16:  # the polynomial's own (test_gelu_of_bfloat16_results)
        own = own + ref.gelu_bf16_bound(expected(q, s, w, ws, bias, "none")[0])
    off = (got.double().cpu() - want).abs() - HALF[dtype] * want.abs() - 1.13 * 4 * 2.0 ** -24 * size - own
    assert float(off.max()) <= 0, float(off.max())


KS = [4, 16, 48, 64, 80, 96, 128, 144, 192, 200, 256, 840, 1024]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 63, 64, 65, 129, 333])
@pytest.mark.parametrize("N", [1, 7, 16, 40, 65, 150, 264])
def test_linear(dtype, M, N):
    """Every K of the list by turns with the sizes, values and steps, with and without a shift, all activations."""
    g = torch.Generator().manual_seed(M * 1000 + N)
    for i, K in enumerate(KS):
        K = K if dtype is torch.float32 or K % 8 == 0 else K + 4
        x = torch.randn((M, K), generator=g).to(dtype)
        q, s = ref.steps(x.float())
        w, ws = ref.steps(torch.randn((N, K), generator=g) * 0.1)
        act = ("none", "gelu", "relu", "silu")[i % 4]
        bias = torch.randn(N, generator=g).to(dtype) if i % 3 else None
        pad = (K + 15) // 16 * 16 - K
        wd = torch.nn.functional.pad(w, (0, pad)).to(DEV)
        kw = dict(bias=None if bias is None else bias.to(DEV), activation=act)
        got = mpm.linear_int8(x.to(DEV), wd, ws.to(DEV), **kw)
        assert got.dtype is dtype
        near(got, q, s, w, ws, bias, act, dtype)
        qd = torch.nn.functional.pad(q, (0, pad)).to(DEV)
        assert torch.equal(mpm.linear_int8(qd, wd, ws.to(DEV), x_scale=s.to(DEV), dtype=dtype, **kw), got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(4219, 2048, 272), (2049, 4104, 64), (33000, 264, 144), (40, 70000, 32)])
def test_linear_many(dtype, M, N, K):
    """Sizes of the largest tiles, with ragged ends."""
    g = torch.Generator().manual_seed(M)
    x = torch.randn((M, K), generator=g).to(dtype)
    q, s = ref.steps(x.float())
    w, ws = ref.steps(torch.randn((N, K), generator=g) * 0.1)
    bias = torch.randn(N, generator=g).to(dtype)
    got = mpm.linear_int8(x.to(DEV), w.to(DEV), ws.to(DEV), bias=bias.to(DEV), activation="gelu")
    near(got, q, s, w, ws, bias, "gelu", dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(901, 331), (2201, 603), (5003, 1100)])
@pytest.mark.parametrize("K", [8, 72, 128, 264, 520])
def test_linear_tiles(dtype, M, N, K):
    """Batches of tiles that fill the chip in part, with ragged ends on all three sides."""
    g = torch.Generator().manual_seed(M + K)
    x = torch.randn((M, K), generator=g).to(dtype)
    q, s = ref.steps(x.float())
    w, ws = ref.steps(torch.randn((N, K), generator=g) * 0.1)
    wd = torch.nn.functional.pad(w, (0, (K + 15) // 16 * 16 - K)).to(DEV)
    got = mpm.linear_int8(x.to(DEV), wd, ws.to(DEV), activation="relu")
    near(got, q, s, w, ws, None, "relu", dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 40, 1024), (4, 33, 1032), (2, 24, 8200), (5, 20, 4104), (16, 19, 3008), (16, 18, 3088),
                                   (31, 30, 2056), (200, 120, 2056), (521, 248, 2064), (300, 500, 4360), (250, 200, 16), (333, 100, 2040),
                                   (1200, 16, 5000), (3000, 2901, 1032), (8200, 4100, 1040)])
def test_linear_long(dtype, M, N, K):
    """Long rows, with k split over waves and in the largest tiles."""
    g = torch.Generator().manual_seed(M + K)
    x = torch.randn((M, K), generator=g).to(dtype)
    q, s = ref.steps(x.float())
    w, ws = ref.steps(torch.randn((N, K), generator=g) * 0.1)
    bias = torch.randn(N, generator=g).to(dtype)
    wd = torch.nn.functional.pad(w, (0, (K + 15) // 16 * 16 - K)).to(DEV)
    got = mpm.linear_int8(x.to(DEV), wd, ws.to(DEV), bias=bias.to(DEV), activation="silu")
    near(got, q, s, w, ws, bias, "silu", dtype)


@pytest.mark.parametrize("M", [3, 16, 40, 300])
def test_extreme_steps(M):
    """Sums of the largest products stay whole: 65536 of (-128)^2 in 32 bits; the bytes past K have to be zero on one side."""
    K = 65536
    q = torch.full((M, K), -128, dtype=torch.int8, device=DEV)
    w = torch.full((24, K), -128, dtype=torch.int8, device=DEV)
    w[1] = 127
    one = torch.ones(M, device=DEV)
    y = mpm.linear_int8(q, w, torch.ones(24, device=DEV), x_scale=one, dtype=torch.float32)
    assert bool((y[:, 0] == 2.0 ** 30).all()) and bool((y[:, 1] == -128.0 * 127 * K).all())
    q = torch.ones((M, 32), dtype=torch.int8, device=DEV)
    w = torch.full((8, 32), 7, dtype=torch.int8, device=DEV)
    w[:, 24:] = 0
    assert bool((mpm.linear_int8(q, w, torch.ones(8, device=DEV), x_scale=one, dtype=torch.float32) == 7 * 24).all())


@pytest.mark.parametrize("M", [2, 16, 70, 1100])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rows_of_any_stride(M, dtype):
    """Inputs and results inside wider rows, at odd places: what lies around them stays."""
    g = torch.Generator().manual_seed(M)
    N, K = 72, 64
    x = torch.randn((M, 3 * K), generator=g).to(dtype).to(DEV)[:, K:2 * K]
    w, ws = mpm.quantize_rows(torch.randn((N, K), generator=g).to(DEV))
    want = mpm.linear_int8(x.contiguous(), w, ws, activation="silu")
    for width, at in ((N, 0), (N + 8, 8), (N + 24, 3), (N + 5, 1)):
        whole = torch.full((M + 1, width), 9.0, dtype=dtype, device=DEV)
        view = whole[:M, at:at + N]
        assert mpm.linear_int8(x, w, ws, activation="silu", out=view).data_ptr() == view.data_ptr()
        assert torch.equal(view, want)
        rest = whole.clone()
        rest[:M, at:at + N] = 9.0
        assert bool((rest == 9).all())


def test_streams_and_capture():
    """On a side stream, and replayed from a graph with eager work between: the same bits."""
    g = torch.Generator().manual_seed(9)
    for M in (5, 700):
        x = torch.randn((M, 256), generator=g).to(torch.bfloat16).to(DEV)
        w, ws = mpm.quantize_rows(torch.randn((512, 256), generator=g).to(DEV))
        want = mpm.linear_int8(x, w, ws, activation="gelu")
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            y = mpm.linear_int8(x, w, ws, activation="gelu")
        torch.cuda.current_stream().wait_stream(stream)
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = mpm.linear_int8(x, w, ws, activation="gelu")
        for k in range(4):
            got.fill_(k)
            again = mpm.linear_int8(x, w, ws, activation="gelu")
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(again, want)
