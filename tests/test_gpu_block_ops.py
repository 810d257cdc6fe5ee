"""The operators of the blocks against plain 64-bit forms: packed attention with a bucketed
position bias, and the norms around a block, forward and backward.

Tolerances are relative 2-norms, from the arithmetic: bfloat16 results are rounded once
(2^-9 at most) after products whose probabilities or score gradients were rounded once or twice
more (forward 2, backward 3 such factors): 3 and 4 times 2^-9. Float32 sums of dh products in
exponents of up to about 16: (dh + 16) 2^-24 relative, 2^-24 * 144 for the widest head. Norms:
one rounding of the result and, backward, of the stored y: 2 and 3 times 2^-9, in float32 sums of D
values in a tree 2^-24 * 16."""
import math

import pytest
import torch

import paper_2604_05718_amd as mpm
import block_refs as ref

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
FWD = {torch.bfloat16: 3 * 2.0 ** -9, torch.float32: 144 * 2.0 ** -24}
BWD = {torch.bfloat16: 4 * 2.0 ** -9, torch.float32: 2 * 144 * 2.0 ** -24}
BF, F32 = torch.bfloat16, torch.float32


def offsets(ns):
    return torch.cumsum(torch.tensor([0] + list(ns)), 0).to(torch.int32)


def positions(ns, cells, gen, how):
    """Grid cells of packed rows: sorted and distinct, in any order, or all the same."""
    out = []
    for n in ns:
        if how == "sorted":
            p = torch.randperm(cells, generator=gen)[:n].sort().values
        elif how == "shuffled":
            p = torch.randperm(cells, generator=gen)[:n]
        else:
            p = torch.full((n,), cells // 3)
        out.append(p)
    return torch.cat(out).to(torch.int32)


class Case:
    """One attention call: CPU tensors of the storage type, and the keyword arguments on the GPU."""

    def __init__(self, dtype, nq, nk, H, Hk, dh, grid=None, span=None, how="sorted", kbias=False, seed=0, inf_bias=False):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.H, self.Hk, self.dh, self.grid = dtype, H, Hk, dh, grid
        nk = nq if nk is None else nk
        self.q = torch.randn(sum(nq), H, dh, generator=g).to(dtype)
        self.k, self.v = (torch.randn(sum(nk), Hk, dh, generator=g).to(dtype) for _ in range(2))
        self.dout = torch.randn(sum(nq), H, dh, generator=g).to(dtype)
        self.q_off, self.k_off = offsets(nq), offsets(nk)
        self.Nq, self.Nk, self.B = max(max(nq), 1), max(max(nk), 1), len(nq)
        self.bias = self.q_pos = self.k_pos = self.k_bias = None
        if span is not None:
            W, cells = 2 * span + 1, grid[0] * grid[1]
            self.bias = 0.7 * torch.randn(H, W, W, generator=g)
            if inf_bias:
                self.bias[torch.rand(H, W, W, generator=g) < 0.2] = -math.inf
            self.k_pos = positions(nk, cells, g, how)
            self.q_pos = self.k_pos if list(nq) == list(nk) else torch.randint(0, cells, (sum(nq),), generator=g).to(torch.int32)
        if kbias:
            size = torch.randint(0, 5, (sum(nk),), generator=g)
            self.k_bias = size.float().log()
        self.scale = dh ** -0.5

    def kw(self):
        dev = lambda t: None if t is None else t.to(DEV)
        d = dict(q_off=dev(self.q_off), k_off=dev(self.k_off), Nq=self.Nq, Nk=self.Nk, k_bias=dev(self.k_bias))
        if self.bias is not None:
            d.update(bias=dev(self.bias), q_pos=dev(self.q_pos), k_pos=dev(self.k_pos), grid=self.grid)
        return d

    def plain(self, grads=False):
        """out, lse (and the gradients of q, k, v and the bias) in 64 bits."""
        leaf = [t.double().requires_grad_(grads) for t in (self.q, self.k, self.v)]
        bias = None if self.bias is None else self.bias.double().requires_grad_(grads)
        out, lse = ref.attention(*leaf, ref.images(self.q_off, 0, self.B), ref.images(self.k_off, 0, self.B), self.scale,
                                 bias, self.q_pos, self.k_pos, self.grid, self.k_bias)
        if not grads:
            return out.detach(), lse.detach()
        want = leaf + ([bias] if bias is not None else [])
        g = torch.autograd.grad((out * self.dout.double()).sum(), want, allow_unused=True)
        g = [torch.zeros_like(w) if x is None else x for x, w in zip(g, want)]
        return out.detach(), lse.detach(), g

    def dev(self):
        return self.q.to(DEV), self.k.to(DEV), self.v.to(DEV)


RAGGED = [1, 33, 0, 128, 129, 64, 7, 200]
SHAPES = [
    # nq, nk, H, Hk, dh, grid, span, how, k_bias
    (RAGGED, None, 3, 3, 64, (15, 14), 14, "sorted", False),
    (RAGGED, None, 3, 3, 64, None, None, "sorted", False),
    (RAGGED, None, 4, 2, 32, (15, 14), 5, "sorted", True),
    ([70, 40], None, 6, 2, 40, (11, 13), 12, "shuffled", True),
    ([65], None, 2, 1, 128, (9, 9), 8, "sorted", False),
    ([31, 90], None, 2, 2, 80, (10, 9), 2, "same", False),
    ([5, 5, 5], [300, 0, 17], 3, 1, 64, (20, 20), 19, "sorted", True),
    ([1, 1], [500, 1], 4, 4, 64, (32, 32), 31, "sorted", False),
    ([130], None, 1, 1, 8, (12, 12), 0, "sorted", False),
    ([300], None, 1, 1, 16, (64, 64), 63, "sorted", False),
    ([40, 1], None, 2, 2, 24, (200, 3), 63, "shuffled", False),
    # the widest heads with the largest table, tables of the middle size, long images in wide blocks
    ([300, 5], None, 2, 1, 128, (64, 64), 63, "sorted", True),
    ([90, 270], None, 2, 2, 64, (36, 30), 35, "sorted", False),
    ([600], None, 4, 2, 64, (64, 50), 63, "shuffled", True),
    ([1800, 100], None, 2, 2, 64, None, None, "sorted", False),
    ([1900], None, 1, 1, 64, (64, 64), 20, "sorted", False),
    ([1850], None, 1, 1, 64, (64, 64), 63, "sorted", True),
    ([200] * 50, None, 6, 6, 32, (16, 16), 15, "sorted", False),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_attention(dtype, i):
    nq, nk, H, Hk, dh, grid, span, how, kb = SHAPES[i]
    c = Case(dtype, nq, nk, H, Hk, dh, grid, span, how, kb, seed=i)
    print(f"attention shape {i} {dtype}", flush=True)
    out, lse = mpm.attention(*c.dev(), with_lse=True, **c.kw())
    torch.cuda.synchronize()
    want, wl = c.plain()
    assert ref.rel(out, want) <= FWD[dtype]
    empty = torch.isinf(wl)
    lse = lse.cpu().double().sum(-1) * math.log(2.0)
    assert torch.equal(torch.isinf(lse), empty) and torch.all(out.cpu()[empty] == 0)
    assert ref.rel(lse[~empty], wl[~empty]) <= 144 * 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_attention_backward(dtype, i):
    nq, nk, H, Hk, dh, grid, span, how, kb = SHAPES[i]
    c = Case(dtype, nq, nk, H, Hk, dh, grid, span, how, kb, seed=100 + i)
    print(f"attention backward shape {i} {dtype}", flush=True)
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    torch.cuda.synchronize()
    _, _, want = c.plain(grads=True)
    for name, got, w in zip(("dq", "dk", "dv"), (g.dq, g.dk, g.dv), want):
        assert ref.rel(got, w) <= BWD[dtype], name
    if c.bias is None:
        assert g.dbias is None
    elif i != 5 and i != 8:  # one bucket alone holds the sum of whole rows, which is zero
        assert ref.rel(g.dbias, want[3]) <= BWD[dtype]
    again = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    for a, b in ((g.dq, again.dq), (g.dk, again.dk), (g.dv, again.dv), (g.dbias, again.dbias)):
        assert a is None or torch.equal(a, b)


FEW = [
    # nq, nk, H, Hk, dh, grid, span, k_bias: at most 32 columns of queries a key head
    ([1, 1, 1], [5000, 31, 900], 4, 4, 64, (80, 70), 63, True),
    ([1] * 5, [600] * 5, 3, 3, 64, (25, 25), 24, False),
    ([2, 0, 1], [700, 33, 0], 6, 2, 40, (30, 30), 29, False),
    ([7], [16384], 2, 2, 64, (128, 128), 63, True),
    ([4, 3], [2000, 1999], 8, 1, 128, None, None, True),
    ([20], [333], 1, 1, 8, (20, 20), 3, False),
    ([16], [1], 4, 2, 64, (9, 9), 8, False),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(FEW)))
def test_attention_of_few_queries(dtype, i):
    nq, nk, H, Hk, dh, grid, span, kb = FEW[i]
    c = Case(dtype, nq, nk, H, Hk, dh, grid, span, "sorted", kb, seed=200 + i)
    print(f"few queries {i} {dtype}", flush=True)
    if kb:
        c.k_bias[-20:] = -math.inf
    k, v = c.k.to(DEV), c.v.to(DEV)
    if kb:
        k[torch.isinf(c.k_bias).to(DEV)] = math.nan
        v[torch.isinf(c.k_bias).to(DEV)] = math.nan
    out, lse = mpm.attention(c.q.to(DEV), k, v, with_lse=True, **c.kw())
    torch.cuda.synchronize()
    want, wl = c.plain()
    assert ref.rel(out, want) <= FWD[dtype]
    empty = torch.isinf(wl)
    lse = lse.cpu().double().sum(-1) * math.log(2.0)
    assert torch.equal(torch.isinf(lse), empty) and torch.all(out.cpu()[empty] == 0)
    assert ref.rel(lse[~empty], wl[~empty]) <= 144 * 2.0 ** -24


def test_attention_gradients_against_differences():
    """Float32 gradients against central differences of the 64-bit form along random directions
    (error: the gradient's own tolerance of the directional derivative's scale, and step^2)."""
    c = Case(F32, [37, 20], None, 4, 2, 16, (9, 8), 4, "sorted", True, seed=5)
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    qs, ks = ref.images(c.q_off, 0, 2), ref.images(c.k_off, 0, 2)

    def loss(x):
        o, _ = ref.attention(*x[:3], qs, ks, c.scale, x[3], c.q_pos, c.k_pos, c.grid, c.k_bias)
        return float((o * c.dout.double()).sum())

    at = [c.q.double(), c.k.double(), c.v.double(), c.bias.double()]
    gen = torch.Generator().manual_seed(6)
    for j, got in enumerate((g.dq, g.dk, g.dv, g.dbias)):
        d = torch.randn(at[j].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        plus, minus = list(at), list(at)
        plus[j], minus[j] = at[j] + h * d, at[j] - h * d
        diff = (loss(plus) - loss(minus)) / (2 * h)
        got = got.double().cpu()
        assert abs(float((got * d).sum()) - diff) <= 1e-4 * float(got.norm() * d.norm()) / math.sqrt(d.numel()) + 1e-6


@pytest.mark.parametrize("lowest", [torch.finfo(F32).min, -1e9])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_dropped_keys_are_not_read(dtype, lowest):
    """NaN and infinities in the rows of dropped keys reach neither results nor gradients; keys at a
    finite mask value stay keys, of equal weight where every key of an image has it (the value hides
    their scores, in 64 bits too where it is the type's lowest)."""
    c = Case(dtype, [70, 33, 4], None, 2, 2, 64, (10, 9), 9, "sorted", True, seed=7)
    c.k_bias[70:74] = -math.inf
    low = torch.arange(103, 107)
    c.k_bias[low] = lowest  # the last image: every key
    if lowest == -1e9:
        c.q[low] = c.k[low] = 0  # 64 bits would still tell the scores apart
        c.k_pos[low] = 9  # (the queries' too)
    want, _, wg = c.plain(grads=True)
    drop = torch.isinf(c.k_bias)
    assert drop.any()
    q, k, v = c.dev()
    k[drop.to(DEV)], v[drop.to(DEV)] = math.nan, math.inf
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    torch.cuda.synchronize()
    assert torch.isfinite(out).all() and ref.rel(out, want) <= FWD[dtype]
    for got, w in zip((g.dq, g.dk, g.dv), wg):
        assert torch.isfinite(got).all() and ref.rel(got, w) <= BWD[dtype]
        assert ref.rel(got[low], w[low]) <= BWD[dtype]
    assert torch.all(g.dk.cpu()[drop] == 0) and torch.all(g.dv.cpu()[drop] == 0)


@pytest.mark.parametrize("low", [torch.finfo(F32).min, -1e9, -1e4, -200.0])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_masks_before_real_keys(dtype, low):
    """Finite mask values on the first keys, several tiles of them, and none on later ones: only the later
    keys count, in the few-query form too (the masked weights are below 2^-100)."""
    c = Case(dtype, [150, 40, 3], [400, 90, 700], 2, 2, 64, (30, 30), 29, "sorted", True, seed=9)
    c.k_bias = torch.zeros(1190)
    for a, b in ((0, 300), (400, 489), (490, 1100)):
        c.k_bias[a:b] = low
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    few = dict(c.kw(), q_off=offsets([5, 0, 3]).to(DEV), Nq=5, q_pos=c.q_pos[:8].contiguous().to(DEV))
    some = mpm.attention(q[:8], k, v, **few)
    torch.cuda.synchronize()
    want, _, wg = c.plain(grads=True)
    assert ref.rel(out, want) <= FWD[dtype]
    for got, w in zip((g.dq, g.dk, g.dv, g.dbias), wg):
        assert ref.rel(got, w) <= BWD[dtype]
    assert ref.rel(some[:5], want[:5]) <= FWD[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [30.0, 300.0])
def test_large_scores(dtype, size):
    """Scores of either sign far from zero, rising along the keys: what is taken from them follows. The
    exponent's error is 2^-24 of the scores (times the products' depth), which bounds float32."""
    c = Case(dtype, [70], [300], 2, 2, 32, (18, 18), 17, "sorted", True, seed=10)
    c.k_bias = torch.linspace(-size, size, 300) - size * 0.5
    out, lse = mpm.attention(*c.dev(), with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), *c.dev(), out, lse, **c.kw())
    torch.cuda.synchronize()
    want, wl, wg = c.plain(grads=True)
    tol = {BF: BWD[BF], F32: 2 * (144 + 4 * size) * 2.0 ** -24}[dtype]
    assert ref.rel(out, want) <= tol
    assert ref.rel(lse.cpu().double().sum(-1) * math.log(2.0), wl) <= 144 * 2.0 ** -24
    for got, w in zip((g.dq, g.dk, g.dv), wg):
        assert ref.rel(got, w) <= tol


def test_bias_of_minus_infinity_masks():
    """Offsets whose bias is -inf take no part, and a query all of whose keys are masked gets zeros."""
    c = Case(F32, [50, 3], None, 2, 2, 32, (8, 8), 7, "sorted", False, seed=8, inf_bias=True)
    c.bias[:, 7, 7] = -math.inf  # a token alone would see itself only
    c.q_pos[50:] = c.k_pos[50:] = 9
    out, lse = mpm.attention(*c.dev(), with_lse=True, **c.kw())
    q, k, v = c.dev()
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    torch.cuda.synchronize()
    want, wl = c.plain()
    assert ref.rel(out, want) <= FWD[F32]
    assert torch.all(out[50:] == 0) and torch.all(torch.isinf(lse[50:].sum(-1)))
    for t in (g.dq[50:], g.dk[50:], g.dv[50:]):
        assert torch.all(t == 0)
    assert torch.isfinite(g.dbias).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_dense_and_streams(dtype):
    """Views of one fused projection, dense images, gradients into views, and another stream: the
    results of contiguous packed rows, bit for bit."""
    B, N, H, dh = 3, 50, 4, 32
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn(B, N, 3, H, dh, generator=g).to(dtype).to(DEV)
    dout = torch.randn(B, N, H, dh, generator=g).to(dtype).to(DEV)
    bias = torch.randn(H, 15, 15, generator=g).to(DEV)
    kw = dict(bias=bias, grid=(8, 7))
    q, k, v = qkv.unbind(2)
    out, lse = mpm.attention(q, k, v, with_lse=True, **kw)
    dqkv = torch.empty_like(qkv)
    got = mpm.attention_backward(dout, q, k, v, out, lse, dq=dqkv[:, :, 0], dk=dqkv[:, :, 1], dv=dqkv[:, :, 2], **kw)
    off = offsets([N] * B).to(DEV)
    flat = [t.reshape(B * N, H, dh).contiguous() for t in (q, k, v, dout)]
    pos = torch.arange(N).repeat(B).to(torch.int32).to(DEV)
    pk = dict(q_off=off, k_off=off, Nq=N, Nk=N, q_pos=pos, k_pos=pos, **kw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out2, lse2 = mpm.attention(*flat[:3], with_lse=True, **pk)
        got2 = mpm.attention_backward(flat[3], *flat[:3], out2, lse2, **pk)
    torch.cuda.synchronize()
    assert torch.equal(out.reshape(B * N, H, dh), out2) and torch.equal(lse, lse2)
    for a, b in ((dqkv[:, :, 0], got2.dq), (dqkv[:, :, 1], got2.dk), (dqkv[:, :, 2], got2.dv)):
        assert torch.equal(a.reshape(B * N, H, dh), b)
    assert torch.equal(got.dbias, got2.dbias)


def test_rows_past_32_bit_offsets():
    """Rows whose byte offsets pass 32 bits (a stride of 2^30 elements)."""
    H, dh, n, stride = 1, 8, 5, 1 << 30
    store = torch.zeros((n - 1) * stride + 64, dtype=BF, device=DEV)
    k = torch.as_strided(store, (n, H, dh), (stride, dh, 1))
    v = torch.as_strided(store, (n, H, dh), (stride, dh, 1), storage_offset=16)
    g = torch.Generator().manual_seed(10)
    kc, vc, qc = (torch.randn(m, H, dh, generator=g).to(BF) for m in (n, n, 40))
    k.copy_(kc.to(DEV))
    v.copy_(vc.to(DEV))
    off = dict(q_off=offsets([40]).to(DEV), k_off=offsets([n]).to(DEV), Nq=40, Nk=n)
    out, lse = mpm.attention(qc.to(DEV), k, v, with_lse=True, **off)
    same, lse2 = mpm.attention(qc.to(DEV), kc.to(DEV), vc.to(DEV), with_lse=True, **off)
    torch.cuda.synchronize()
    assert torch.equal(out, same) and torch.equal(lse, lse2)


def test_attention_in_a_graph():
    """Forward, backward and the table's gradient captured once and replayed on new inputs, with eager
    work between the replays."""
    c = Case(BF, [60, 90], None, 3, 3, 64, (10, 10), 9, "sorted", False, seed=11)
    lut, nb = mpm.bucket_lut(9, 4)
    lut = lut.to(DEV)
    table = torch.randn(nb * nb, 3, device=DEV).to(BF)
    q, k, v = c.dev()
    dout, kw = c.dout.to(DEV), c.kw()

    def step():
        kw["bias"] = mpm.bias_expand(table, lut)
        out, lse = mpm.attention(q, k, v, with_lse=True, **kw)
        g = mpm.attention_backward(dout, q, k, v, out, lse, **kw)
        return out, g.dq, g.dk, g.dv, mpm.bias_gradient(g.dbias, lut, nb, dtype=BF)

    step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step()
    for i in range(4):
        q.normal_()
        table.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in res]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("span,side,H", [(0, None, 1), (4, None, 3), (31, None, 12), (63, 15, 16), (63, None, 5), (9, 1, 2)])
def test_bias_table(dtype, span, side, H):
    lut, nb = mpm.bucket_lut(span, side)
    assert lut.numel() == 2 * span + 1 and int(lut.min()) >= 0 and int(lut.max()) == nb - 1 and lut[span] == nb // 2
    W = 2 * span + 1
    g = torch.Generator().manual_seed(span)
    table = torch.randn(nb * nb, H, generator=g).to(dtype)
    cell = (lut.long()[:, None] * nb + lut.long()[None, :]).reshape(-1)
    bias = mpm.bias_expand(table.to(DEV), lut.to(DEV))
    assert torch.equal(bias.cpu(), table.float()[cell].t().reshape(H, W, W))
    dbias = torch.randn(H, W, W, generator=g)
    got = mpm.bias_gradient(dbias.to(DEV), lut.to(DEV), nb, dtype=dtype)
    want = torch.zeros(nb * nb, H, dtype=torch.float64).index_add_(0, cell, dbias.double().reshape(H, -1).t().contiguous())
    # one rounding, and a sum of up to W^2 terms in runs of at most W: (W / 64 + 8) additions deep a row
    assert ref.rel(got, want) <= (2.0 ** -9 if dtype == BF else 256 * 2.0 ** -24)
    assert torch.equal(got, mpm.bias_gradient(dbias.to(DEV), lut.to(DEV), nb, dtype=dtype))


NORMS = [
    # lengths, D, norm, pre, shifts, post, scale, gate
    ([118], 192, "layer", True, True, False, True, "none"),
    ([5, 0, 77, 1, 300], 768, "layer", True, True, True, True, "image"),
    ([700, 20], 1024, "layer", True, True, True, False, "row"),
    ([33, 4], 8, "rms", True, False, True, True, "row"),
    ([3, 9], 2048, "rms", True, True, False, False, "image"),
    ([10], 5000, "layer", True, False, True, True, "none"),
    ([6], 16384, "layer", True, True, True, True, "image"),
    ([64, 65], 72, "layer", False, False, True, True, "none"),
    ([17], 520, "layer", False, False, False, True, "image"),
]
NORM_FWD = {BF: 2 * 2.0 ** -9, F32: 16 * 2.0 ** -24}
NORM_BWD = {BF: 3 * 2.0 ** -9, F32: 2 * 16 * 2.0 ** -24}


def norm_case(dtype, i):
    ns, D, norm, pre, shifts, post, scale, gate = NORMS[i]
    g = torch.Generator().manual_seed(40 + i)
    R = sum(ns)
    rn = lambda *s, m=0.0, sd=1.0: (torch.randn(s, generator=g) * sd + m).to(dtype)
    x, f, dy, dh = rn(R, D, m=0.3, sd=2.0), rn(R, D, m=-0.5), rn(R, D), rn(R, D)
    p = dict(weight=rn(D, m=1.0, sd=0.3) if pre else None, bias=rn(D) if pre and shifts else None,
             post_weight=rn(D, m=1.0, sd=0.3) if post else None, post_bias=rn(D) if post and shifts else None,
             scale=rn(D, sd=0.5) if scale else None, gate=None)
    off = rows_of = None
    if gate == "image":
        p["gate"] = rn(len(ns), D, m=0.5)
        off, rows_of = offsets(ns), torch.repeat_interleave(torch.arange(len(ns)), torch.tensor(ns))
    elif gate == "row":
        p["gate"] = rn(R, D, m=0.5)
    return x, f, dy, dh, p, off, rows_of, norm


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(NORMS)))
def test_residual_norm(dtype, i):
    x, f, dy, dh, p, off, rows_of, norm = norm_case(dtype, i)
    dev = lambda t: None if t is None else t.to(DEV)
    kw = dict({k: dev(t) for k, t in p.items()}, off=dev(off), norm=norm)
    print(f"residual_norm {i} {dtype}", flush=True)
    xd, fd = x.to(DEV), f.to(DEV)
    y, h, stats = mpm.residual_norm(xd, fd, with_stats=True, **kw)
    g = mpm.residual_norm_backward(dy.to(DEV), dh.to(DEV) if h is not None else None, y, fd, stats, **kw)
    torch.cuda.synchronize()
    leaf = {"x": x.double().requires_grad_(), "f": f.double().requires_grad_()}
    leaf.update({k: t.double().requires_grad_() for k, t in p.items() if t is not None})
    wy, wh = ref.residual_norm(leaf["x"], leaf["f"], **{k: leaf.get(k) for k in p}, rows_of=rows_of, norm=norm)
    assert ref.rel(y, wy) <= NORM_FWD[dtype]
    loss = (wy * dy.double()).sum()
    if h is not None:
        assert ref.rel(h, wh) <= NORM_FWD[dtype]
        loss = loss + (wh * dh.double()).sum()
    want = dict(zip(leaf, torch.autograd.grad(loss, list(leaf.values()))))
    got = {"x": g.dx, "f": g.df, "weight": g.dweight, "bias": g.dbias, "post_weight": g.dpost_weight,
           "post_bias": g.dpost_bias, "scale": g.dscale, "gate": g.dgate}
    for k, t in got.items():
        assert (t is None) == (k not in want), k
        if t is not None:
            assert ref.rel(t, want[k]) <= NORM_BWD[dtype], k
    again = mpm.residual_norm_backward(dy.to(DEV), dh.to(DEV) if h is not None else None, y, fd, stats, **kw)
    for k, t in vars(g).items():
        assert t is None or torch.equal(t, getattr(again, k)), k
    # y into x's own memory, and without the gradient from past the block
    y2, h2 = mpm.residual_norm(xd, fd, out=xd, **kw)
    assert y2.data_ptr() == xd.data_ptr() and torch.equal(y2, y) and (h is None or torch.equal(h2, h))
    if h is not None:
        zero = mpm.residual_norm_backward(torch.zeros_like(y), dh.to(DEV), y, fd, stats, **kw)
        none = mpm.residual_norm_backward(None, dh.to(DEV), y, fd, stats, **kw)
        assert torch.equal(zero.dx, none.dx) and torch.equal(zero.df, none.df)


def test_norm_gradients_against_differences():
    x, f, dy, dh, p, off, rows_of, norm = norm_case(F32, 1)
    dev = lambda t: None if t is None else t.to(DEV)
    kw = dict({k: dev(t) for k, t in p.items()}, off=dev(off), norm=norm)
    y, h, stats = mpm.residual_norm(x.to(DEV), f.to(DEV), with_stats=True, **kw)
    g = mpm.residual_norm_backward(dy.to(DEV), dh.to(DEV), y, f.to(DEV), stats, **kw)
    at = {"x": x.double(), "f": f.double(), **{k: t.double() for k, t in p.items()}}

    def loss(a):
        wy, wh = ref.residual_norm(a["x"], a["f"], **{k: a[k] for k in p}, rows_of=rows_of, norm=norm)
        return float((wy * dy.double()).sum() + (wh * dh.double()).sum())

    gen = torch.Generator().manual_seed(12)
    got = {"x": g.dx, "f": g.df, "weight": g.dweight, "bias": g.dbias, "post_weight": g.dpost_weight,
           "post_bias": g.dpost_bias, "scale": g.dscale, "gate": g.dgate}
    for k, t in got.items():
        d, s = torch.randn(at[k].shape, generator=gen, dtype=torch.float64), 1e-5
        diff = (loss({**at, k: at[k] + s * d}) - loss({**at, k: at[k] - s * d})) / (2 * s)
        t = t.double().cpu()
        assert abs(float((t * d).sum()) - diff) <= 1e-4 * float(t.norm() * d.norm()) / math.sqrt(d.numel()) + 1e-5, k


def test_norm_of_constant_rows():
    """Rows without variance: the normed row is the shift, and nothing is infinite."""
    x = torch.full((4, 64), 3.0, dtype=F32, device=DEV)
    w, b = torch.ones(64, device=DEV), torch.full((64,), 0.25, device=DEV)
    y, h, stats = mpm.residual_norm(x, torch.zeros_like(x), weight=w, bias=b, with_stats=True)
    assert torch.equal(y, x) and torch.all(h == 0.25)
    g = mpm.residual_norm_backward(None, torch.ones_like(x), y, torch.zeros_like(x), stats, weight=w, bias=b)
    assert torch.isfinite(g.dx).all() and torch.all(g.dbias == 4)
