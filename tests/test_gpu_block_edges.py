"""The operators of the blocks at the edges of what they take: images out of the middle of a packed
tensor. Tolerances as in test_gpu_block_ops.py."""
import pytest
import torch

import block_refs as ref
import paper_2604_05718_amd as mpm
from test_gpu_block_ops import BF, BWD, DEV, F32, FWD, Case, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("biased", [True, False])
@pytest.mark.parametrize("first", [1, 3])
def test_images_in_the_middle_of_a_packed_tensor(dtype, biased, first):
    """Offsets that start past zero (some images of a larger tensor): the results and gradients of the same
    images packed from zero, bit for bit, and nothing written outside them."""
    ns = [300, 40, 129, 7]
    c = Case(dtype, ns, None, 4, 2, 32, *(((20, 20), 19, "sorted", True) if biased else (None, None)), seed=300)
    a, b = int(c.q_off[first]), int(c.q_off[-1])
    print(f"images {first} to 3, {dtype}, biased {biased}", flush=True)
    most, part = max(ns[first:]), c.q_off[first:].to(DEV)
    kw = dict(c.kw(), q_off=part, k_off=part, Nq=most, Nk=most)
    q, k, v, dout = *c.dev(), c.dout.to(DEV)
    seven = [torch.full_like(t, 7) for t in (q, q, k, v)]
    out, lse = mpm.attention(q, k, v, with_lse=True, out=seven[0], **kw)
    g = mpm.attention_backward(dout, q, k, v, out, lse, dq=seven[1], dk=seven[2], dv=seven[3], **kw)
    torch.cuda.synchronize()
    own = offsets(ns[first:]).to(DEV)
    kw.update(q_off=own, k_off=own, **{n: kw[n][a:b].contiguous() for n in ("q_pos", "k_pos", "k_bias") if kw.get(n) is not None})
    q, k, v, dout = (t[a:b].contiguous() for t in (q, k, v, dout))
    want, wl = mpm.attention(q, k, v, with_lse=True, **kw)
    w = mpm.attention_backward(dout, q, k, v, want, wl, **kw)
    torch.cuda.synchronize()
    for got, t in zip(seven, (want, w.dq, w.dk, w.dv)):
        assert torch.equal(got[a:b], t)
        assert torch.all(got[:a] == 7) and torch.all(got[b:] == 7)
    assert torch.equal(lse[a:b], wl)
    assert g.dbias is None if not biased else torch.equal(g.dbias, w.dbias)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradients_without_the_bias_gradient(dtype):
    """with_dbias=False: no dbias, in the smaller workspace, and the other gradients of the formulas."""
    c = Case(dtype, [200, 33], None, 4, 2, 64, (16, 15), 15, "sorted", True, seed=310)
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, with_dbias=False, **c.kw())
    torch.cuda.synchronize()
    _, _, want = c.plain(grads=True)
    assert g.dbias is None
    for got, w in zip((g.dq, g.dk, g.dv), want):
        assert ref.rel(got, w) <= BWD[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [2.0 ** 93, 1e21, 1e-20, 2.0 ** -80])
@pytest.mark.parametrize("shift", [-41.0, -11.0, 11.0, 41.0])
def test_values_of_any_size(dtype, size, shift):
    """Values far from one under scores far from zero (shift: every score's, in nats): the sums before the
    division neither overflow nor sink into denormals, in the form for few queries too. The exponent's error
    is 2^-24 of the scores, as in test_large_scores."""
    c = Case(dtype, [70, 3], [300, 2000], 2, 2, 32, (50, 50), 49, "sorted", True, seed=320)
    c.k_bias = torch.full((2300,), shift)
    c.v = (c.v.float() * size).to(dtype)
    print(f"values of {size} at {shift}, {dtype}", flush=True)
    q, k, v = c.dev()
    out = mpm.attention(q, k, v, **c.kw())
    few = dict(c.kw(), q_off=offsets([5, 0]).to(DEV), Nq=5, q_pos=c.q_pos[:5].contiguous().to(DEV))
    some = mpm.attention(q[:5], k, v, **few)
    torch.cuda.synchronize()
    want, _ = c.plain()
    tol = FWD[BF] if dtype == BF else (144 + 4 * abs(shift)) * 2.0 ** -24
    assert torch.isfinite(out).all() and ref.rel(out, want) <= tol
    assert torch.isfinite(some).all() and ref.rel(some, want[:5]) <= tol


ORDERS = [(F32, 63, (64, 64)), (F32, 55, (64, 64)), (F32, 53, (200, 50)), (F32, 23, (24, 24)), (F32, 9, (24, 24)),
          (BF, 55, (64, 64)), (BF, 53, (200, 50)), (BF, 9, (24, 24)), (BF, 63, (64, 64)), (BF, 35, (36, 36)),
          (BF, 23, (24, 24))]


@pytest.mark.parametrize("dtype,span,grid", ORDERS)
def test_bias_gradient_does_not_depend_on_the_order_of_keys(dtype, span, grid):
    """The same keys in another order, with the call's own output and statistics: every score gradient is the
    same number, and so has to be their sum at every offset, bit for bit."""
    c = Case(dtype, [60], [500], 2, 1, 64, grid, span, "sorted", False, seed=330)
    print(f"order of keys, span {span}, grid {grid}, {dtype}", flush=True)
    q, k, v = c.dev()
    kw = c.kw()
    out, lse = mpm.attention(q, k, v, with_lse=True, **kw)
    order = torch.randperm(500, generator=torch.Generator().manual_seed(1)).to(DEV)
    a = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **kw)
    kw["k_pos"] = kw["k_pos"][order].contiguous()
    b = mpm.attention_backward(c.dout.to(DEV), q, k[order], v[order], out, lse, **kw)
    torch.cuda.synchronize()
    assert torch.equal(a.dk[order], b.dk) and torch.equal(a.dv[order], b.dv)
    _, _, want = c.plain(grads=True)
    assert ref.rel(a.dbias, want[3]) <= BWD[dtype]
    assert torch.equal(a.dbias, b.dbias)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("how", ["sorted", "shuffled"])
@pytest.mark.parametrize("span", [19, 7])
def test_bias_gradient_beside_keys_of_no_weight(dtype, how, span):
    """Keys at a finite mask value, whose values are large: their probability is zero and so is their part
    of every gradient; the others keep theirs."""
    c = Case(dtype, [300, 90], None, 2, 2, 64, (20, 20), span, how, True, seed=340)
    c.k_bias = torch.zeros(390)
    low = torch.arange(0, 390, 13)
    c.k_bias[low] = -1e9
    c.v[low] = (c.v[low].float() * (1e6 if dtype == BF else 1e12)).to(dtype)
    print(f"keys of no weight, {dtype}, {how}, span {span}", flush=True)
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    torch.cuda.synchronize()
    _, _, want = c.plain(grads=True)
    for got, w in zip((g.dq, g.dk, g.dv, g.dbias), want):
        assert ref.rel(got, w) <= BWD[dtype]


@pytest.mark.parametrize("dtype,far", [(BF, -20.8), (F32, -13.9), (BF, -10.0)])
@pytest.mark.parametrize("span", [23, 63])
def test_bias_gradient_of_far_offsets(dtype, far, span):
    """Attention that a table has made sharp: the far offsets' score gradients are 2^-30 (2^-20 in float32) of the
    near ones', and stay exact on their own."""
    grid = (span + 1, span + 1)
    c = Case(dtype, [250], None, 2, 2, 64, grid, span, "sorted", False, seed=350)
    near = torch.zeros(2 * span + 1, 2 * span + 1, dtype=torch.bool)
    reach = 2 if span == 23 else 6
    near[span - reach:span + reach + 1, span - reach:span + reach + 1] = True
    c.bias = torch.where(near, c.bias, c.bias + far)
    print(f"far offsets, {dtype}, {far}, span {span}", flush=True)
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    torch.cuda.synchronize()
    _, _, want = c.plain(grads=True)
    assert ref.rel(g.dbias[:, near.to(DEV)], want[3][:, near]) <= BWD[dtype]
    assert ref.rel(g.dbias[:, ~near.to(DEV)], want[3][:, ~near]) <= BWD[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_key_bias_that_is_no_number(dtype):
    """A NaN among the key biases is not a dropped key: every query of its image gets NaN, forward (the form
    for few queries too) and in the gradients; other images are as without it."""
    c = Case(dtype, [70, 40], None, 2, 2, 64, (10, 9), 9, "sorted", True, seed=360)
    c.k_bias = torch.zeros(110)
    clean = c.kw()
    c.k_bias[33] = float("nan")
    q, k, v = c.dev()

    def results(kw):
        out, lse = mpm.attention(q, k, v, with_lse=True, **kw)
        g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **kw)
        few = dict(kw, q_off=offsets([3, 2]).to(DEV), Nq=3, q_pos=kw["q_pos"][:5].contiguous())
        return out, lse, g.dq, g.dk, g.dv, mpm.attention(q[:5], k, v, **few)

    want, got = results(clean), results(c.kw())
    torch.cuda.synchronize()
    for w, t in zip(want[:5], got[:5]):
        assert torch.equal(w[70:], t[70:])
    assert torch.equal(want[5][3:], got[5][3:]) and torch.isnan(got[5][:3]).all()
    assert torch.isnan(got[0][:70]).all() and torch.isnan(got[1][:70].sum(-1)).all()
    for t in got[2:5]:
        assert torch.isnan(t[:70]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("span", [9, 4])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("masked", [False, True])
def test_table_entries_that_no_pair_meets(dtype, span, value, masked):
    """What the table holds at offsets that only dropped keys, or no rows at all, would have reaches neither
    results nor gradients: every token lies in the grid's rows 6 to 9, and offsets of four and more rows, which a
    dropped key in row 0 has, are NaN or infinite."""
    ns = [37, 5, 20]
    c = Case(dtype, ns, None, 2, 2, 64, (10, 10), span, "sorted", masked, seed=370)
    g = torch.Generator().manual_seed(1)
    c.k_pos = torch.cat([60 + torch.randperm(40, generator=g)[:n].sort().values for n in ns]).to(torch.int32)
    c.q_pos = c.k_pos.clone()
    if masked:
        c.k_bias = torch.zeros(sum(ns))
        for i in (0, 11, 40, 50):
            c.k_bias[i], c.k_pos[i] = -float("inf"), 3
    want, _, wg = c.plain(grads=True)
    c.bias[:, :span - 3], c.bias[:, span + 4:] = value, value
    print(f"entries of {value}, {dtype}, span {span}, masked {masked}", flush=True)
    q, k, v = c.dev()
    kw = c.kw()
    out, lse = mpm.attention(q, k, v, with_lse=True, **kw)
    r = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **kw)
    few = dict(kw, q_off=offsets([3, 0, 2]).to(DEV), Nq=3, q_pos=kw["q_pos"][:5].contiguous())
    some = mpm.attention(q[:5], k, v, **few)
    torch.cuda.synchronize()
    assert ref.rel(out, want) <= FWD[dtype] and ref.rel(some[:3], want[:3]) <= FWD[dtype]
    for got, w in zip((r.dq, r.dk, r.dv, r.dbias), wg):
        assert ref.rel(got, w) <= BWD[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("where", ["k_bias", "bias"])
def test_the_largest_finite_scores(dtype, where):
    """A term of 3e38, which passes the type's range in base 2, wins its rows; the type's lowest value beside it
    takes no part."""
    c = Case(dtype, [70, 5], [90, 40], 2, 2, 64, (10, 10), 9, "sorted", True, seed=380)
    c.k_bias = torch.zeros(130)
    if where == "k_bias":
        c.k_bias[17], c.k_bias[100] = 3e38, torch.finfo(F32).max
        c.k_bias[18] = torch.finfo(F32).min
    else:
        c.bias[:, 9, 12] = 3e38
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    few = dict(c.kw(), q_off=offsets([3, 0]).to(DEV), Nq=3, q_pos=c.q_pos[:3].contiguous().to(DEV))
    some = mpm.attention(q[:3], k, v, **few)
    torch.cuda.synchronize()
    want, _, wg = c.plain(grads=True)
    assert ref.rel(out, want) <= FWD[dtype] and ref.rel(some, want[:3]) <= FWD[dtype]
    assert ref.rel(g.dv, wg[2]) <= BWD[dtype]
    for got, w in zip((g.dq, g.dk, g.dbias), (wg[0], wg[1], wg[3])):  # zero where one key has all of a row
        assert float((got.double().cpu() - w).norm()) <= BWD[dtype] * max(float(w.norm()), float(c.dout.double().norm()))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_first_rows_of_dense_images(dtype):
    """One row a dense image, a view into the batch, results and gradients written into views as well: those
    of the copied rows, bit for bit."""
    g = torch.Generator().manual_seed(390)
    x, kv, d = (torch.randn(3, 50, 4, 32, generator=g).to(dtype).to(DEV) for _ in range(3))
    into = [torch.full_like(x, 7) for _ in range(2)]
    out, lse = mpm.attention(x[:, :1], kv, kv, with_lse=True, out=into[0][:, :1])
    a = mpm.attention_backward(d[:, :1], x[:, :1], kv, kv, out, lse, dq=into[1][:, :1])
    q = x[:, :1].contiguous()
    want, wl = mpm.attention(q, kv, kv, with_lse=True)
    b = mpm.attention_backward(d[:, :1].contiguous(), q, kv, kv, want, wl)
    torch.cuda.synchronize()
    assert torch.equal(lse, wl)
    for got, w in ((into[0], want), (into[1], b.dq)):
        assert torch.equal(got[:, :1], w) and torch.all(got[:, 1:] == 7)
    assert torch.equal(a.dk, b.dk) and torch.equal(a.dv, b.dv)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Nq", [3, 40])
@pytest.mark.parametrize("dense", [False, True])
def test_no_keys_at_all(dtype, Nq, dense):
    """Queries of images none of which has a key: zeros, statistics of an empty sum, and zero gradients."""
    g = torch.Generator().manual_seed(400)
    q, d = (torch.randn(2 * Nq, 4, 32, generator=g).to(dtype).to(DEV) for _ in range(2))
    k = torch.zeros(0, 2, 32, dtype=dtype, device=DEV)
    kw = dict(bias=torch.randn(4, 9, 9, generator=g).to(DEV), grid=(9, 5))
    if dense:
        q, d, k = q.view(2, Nq, 4, 32), d.view(2, Nq, 4, 32), k.view(2, 0, 2, 32)
    else:
        none = torch.zeros(0, device=DEV)
        kw.update(q_off=offsets([Nq, Nq]).to(DEV), k_off=offsets([0, 0]).to(DEV), Nq=Nq, Nk=0, k_bias=none,
                  q_pos=torch.zeros(2 * Nq, dtype=torch.int32, device=DEV), k_pos=none.int())
    out, lse = mpm.attention(q, k, k, with_lse=True, **kw)
    r = mpm.attention_backward(d, q, k, k, out, lse, **kw)
    torch.cuda.synchronize()
    assert out.shape == q.shape and not out.any() and torch.isinf(lse.sum(-1)).all()
    assert not r.dq.any() and not r.dbias.any() and r.dk.shape == k.shape == r.dv.shape


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("R,D", [(5000, 64), (3000, 768), (700, 2048), (300, 5000), (40, 16384)])
def test_residual_norm_in_place(dtype, R, D):
    """y into x's own memory, many rows a workgroup, for every width of a row group: the results of a call with
    a y of its own, bit for bit, time after time."""
    g = torch.Generator().manual_seed(410)
    x, f = (torch.randn(R, D, generator=g).to(dtype).to(DEV) for _ in range(2))
    w, gate = torch.ones(D, dtype=dtype, device=DEV), torch.randn(R, D, generator=g).to(dtype).to(DEV)
    for kw in (dict(weight=w), dict(weight=w, post_weight=w, gate=gate), dict(scale=w)):
        want = mpm.residual_norm(x, f, **kw)
        for _ in range(3):
            y = x.clone()
            got = mpm.residual_norm(y, f, out=y, **kw)
            torch.cuda.synchronize()
            assert got[0].data_ptr() == y.data_ptr() and torch.equal(y, want[0])
            assert want[1] is None or torch.equal(got[1], want[1])


@pytest.mark.parametrize("B", [65535, 65531, 65530])
def test_gates_of_the_most_images(B):
    """A gate an image for as many images as a call takes, two rows each: every image's gradient is there."""
    g = torch.Generator().manual_seed(420)
    D = 8
    f, dy, gate = (torch.randn(n, D, generator=g) for n in (2 * B, 2 * B, B))
    x = torch.zeros(2 * B, D)
    y, h, stats = mpm.residual_norm(x.to(DEV), f.to(DEV), gate=gate.to(DEV), with_stats=True)
    r = mpm.residual_norm_backward(dy.to(DEV), None, y, f.to(DEV), stats, gate=gate.to(DEV))
    torch.cuda.synchronize()
    want = (dy.double() * f.double()).view(B, 2, D).sum(1)
    assert ref.rel(r.dgate, want) <= 2 * 16 * 2.0 ** -24
    assert ref.rel(r.dgate[-6:], want[-6:]) <= 2 * 16 * 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("score,value", [(41.0, 1e21), (41.0, 2.0 ** 95), (-41.0, 1e-20), (11.0, 2.0 ** 95)])
def test_one_key_of_a_large_value(dtype, score, value):
    """One key with a score far from zero and a value far from one, alone or beside a key of no weight."""
    q = torch.zeros(2, 1, 32, dtype=dtype, device=DEV)
    k = torch.zeros(3, 1, 32, dtype=dtype, device=DEV)
    v = torch.full((3, 1, 32), value, dtype=dtype, device=DEV)
    v[1:] = 1.0
    kw = dict(q_off=offsets([1, 1]).to(DEV), k_off=offsets([1, 2]).to(DEV), Nq=1, Nk=2,
              k_bias=torch.tensor([score, score - 200.0, score], device=DEV))
    for n in (1, 40):  # the form for few queries, and the other
        rows = q.repeat_interleave(n, 0)
        kw.update(q_off=offsets([n, n]).to(DEV), Nq=n)
        out = mpm.attention(rows, k, v, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out[:n], v[:1].expand(n, 1, 32)) and torch.all(out[n:] == 1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-5, 3.0])
def test_scales(dtype, scale):
    """Factors of the scores of either sign, none, and ones outside the range in which the products start from the
    statistics. Scores of up to 3 * 30: the exponent's error is 2^-24 of them, as in test_large_scores."""
    c = Case(dtype, [90, 33], None, 2, 2, 32, (12, 10), 11, "sorted", True, seed=430)
    c.scale = scale
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, scale=scale, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, scale=scale, **c.kw())
    torch.cuda.synchronize()
    want, _, wg = c.plain(grads=True)
    slack = 1 if dtype == BF else 1 + 4 * 90 / 144
    assert ref.rel(out, want) <= FWD[dtype] * slack
    for got, w in zip((g.dq, g.dk, g.dv, g.dbias), wg):
        assert ref.rel(got, w) <= BWD[dtype] * slack


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("score", [0.0, 0.3, -7.7, 30.0])
@pytest.mark.parametrize("nq", [3, 200])
def test_rows_that_one_key_has_all_of(dtype, score, nq):
    """One key an image, or one that outweighs the others by 2^40: its values come out as they are (in float32
    up to the roundings of p v, 1 / p and their product, below 2^-22), and the score gradients, zero by the formula, are what float32 sums of dh products of a row leave (2^-24 times dh of its
    largest, the norm of dout.v), through scale k into dq."""
    g = torch.Generator().manual_seed(440)
    q, d = (torch.randn(2 * nq, 2, 64, generator=g).to(dtype) for _ in range(2))
    k, v = (torch.randn(301, 2, 64, generator=g).to(dtype) for _ in range(2))
    k_bias = torch.full((301,), score)
    k_bias[2:] -= 60.0
    dev = lambda t: t.to(DEV)
    kw = dict(q_off=dev(offsets([nq, nq])), k_off=dev(offsets([1, 300])), Nq=nq, Nk=300, k_bias=dev(k_bias),
              bias=torch.zeros(2, 9, 9, device=DEV), grid=(20, 20))
    out, lse = mpm.attention(dev(q), dev(k), dev(v), with_lse=True, **kw)
    r = mpm.attention_backward(dev(d), dev(q), dev(k), dev(v), out, lse, **kw)
    torch.cuda.synchronize()
    one = v[[0] * nq + [1] * nq].double()
    assert torch.all((out.cpu().double() - one).abs() <= (0 if dtype == BF else 2.0 ** -22) * one.abs())
    ds = 64 * 2.0 ** -24 * (d.double().norm(dim=-1) * one.norm(dim=-1)).max()
    assert float(r.dbias.abs().max()) <= ds * nq * 2
    assert float(r.dq.float().abs().max()) <= 0.125 * ds * float(k.float().abs().max()) * 2
    want = torch.zeros(301, 2, 64, dtype=torch.float64)
    want[0], want[1] = d[:nq].double().sum(0), d[nq:].double().sum(0)
    assert ref.rel(r.dv[:2], want[:2]) <= BWD[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -60, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("span", [11, 63])
def test_gradients_of_any_size(dtype, size, span):
    """Gradients scale with dout over the type's range, the bias's too."""
    c = Case(dtype, [60, 90], None, 2, 2, 32, (12, 12) if span == 11 else (64, 64), span, "sorted", False, seed=450)
    c.dout = (c.dout.float() * size).to(dtype)
    q, k, v = c.dev()
    out, lse = mpm.attention(q, k, v, with_lse=True, **c.kw())
    g = mpm.attention_backward(c.dout.to(DEV), q, k, v, out, lse, **c.kw())
    torch.cuda.synchronize()
    _, _, want = c.plain(grads=True)
    for got, w in zip((g.dq, g.dk, g.dv, g.dbias), want):
        assert ref.rel(got, w) <= BWD[dtype]
