"""Refusals of rotary positions, products in 8-bit integers and group norm, and their bindings without a GPU:
every check runs on the host, before any launch."""
import ctypes
import json
import os
import subprocess
import sys

import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm
from paper_2604_05718_amd import _lib, block_ops
from test_block_bindings import Recorder, device

P = 0x10000  # a stand-in device pointer: never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = _lib.MPM_ERR_INVALID_ARG, _lib.MPM_ERR_UNSUPPORTED, _lib.MPM_ERR_WORKSPACE
R = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def ptr(at=P):
    return ctypes.c_void_p(at)


def heads(p=P, row=64, head=64):
    return _lib.Heads(p, row, head)


def rotary(grid=(8, 8, 1), **kw):
    c = dict(R=10, H=4, dh=64, dt=1, pairs=32, layout=0, axes=2, freq=P, pos=P, B=1)
    c.update(kw)
    return _lib.RotaryCall(grid=(ctypes.c_int32 * 3)(*grid), **c)


@pytest.mark.parametrize("kw,status", [
    (dict(R=0), INVALID), (dict(H=0), INVALID), (dict(dh=0), INVALID), (dict(dh=60), INVALID), (dict(dt=2), INVALID),
    (dict(pairs=0), INVALID), (dict(pairs=33), INVALID), (dict(layout=2), INVALID), (dict(layout=-1), INVALID),
    (dict(axes=0), INVALID), (dict(axes=4), INVALID), (dict(grid=(0, 8, 1)), INVALID), (dict(grid=(8, -1, 1)), INVALID),
    (dict(grid=(1 << 16, 1 << 15, 1)), INVALID), (dict(grid=(1 << 30, 1 << 30, 1 << 30), axes=3), INVALID),
    (dict(freq=None), INVALID), (dict(freq=P + 2), INVALID), (dict(pos=P + 1), INVALID), (dict(off=P + 2), INVALID),
    (dict(B=0), INVALID), (dict(B=3), INVALID), (dict(H=1025), UNSUPPORTED), (dict(dh=136), UNSUPPORTED),
    (dict(B=65536, off=P), UNSUPPORTED),
])
def test_rotary_refuses_calls(lib, kw, status):
    c = rotary(**kw)
    assert lib.mpm_rotary(R(c), R(heads()), R(heads()), 0, None) == status
    assert lib.mpm_rotary_backward(R(c), R(heads()), None, R(heads()), None, None, 0, None) == status
    assert lib.mpm_rotary_backward_workspace_bytes(R(c)) == 0


def test_rotary_refuses_rows(lib):
    c = rotary()
    assert lib.mpm_rotary(None, R(heads()), R(heads()), 0, None) == INVALID
    for bad in (heads(p=None), heads(p=P + 8), heads(row=60), heads(head=-8)):
        assert lib.mpm_rotary(R(c), R(bad), R(heads()), 0, None) == INVALID
        assert lib.mpm_rotary(R(c), R(heads()), R(bad), 0, None) == INVALID
        for at in (0, 1, 2):
            h = [bad if i == at else heads() for i in range(3)]
            assert lib.mpm_rotary_backward(R(c), *(R(x) for x in h), ptr(), ptr(), 1 << 40, None) == INVALID
    back = lambda x, df, ws=ptr(), n=1 << 40: lib.mpm_rotary_backward(R(c), R(heads()), x, R(heads()), df, ws, n, None)
    assert back(None, ptr()) == INVALID and back(R(heads()), None) == INVALID
    assert back(R(heads()), ptr(P + 2)) == INVALID and back(R(heads()), ptr(), ws=None) == INVALID
    need = lib.mpm_rotary_backward_workspace_bytes(R(c))
    assert need > 0 and back(R(heads()), ptr(), n=need - 1) == WORKSPACE
    assert back(R(heads()), ptr(), ws=ptr(P + 16)) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(x=ptr(P + 8)), INVALID), (dict(R=0), INVALID), (dict(K=0), INVALID),
    (dict(K=60), INVALID), (dict(row=60), INVALID), (dict(row=-64), INVALID), (dict(dt=2), INVALID),
    (dict(q=None), INVALID), (dict(q=ptr(P + 4)), INVALID), (dict(scale=None), INVALID), (dict(scale=ptr(P + 2)), INVALID),
    (dict(K=65544, row=65544), UNSUPPORTED),
])
def test_quantize_refuses(lib, kw, status):
    a = dict(x=ptr(), R=4, K=64, row=64, dt=1, q=ptr(), scale=ptr())
    a.update(kw)
    assert lib.mpm_quantize_rows(*a.values(), None) == status


def linear(**kw):
    c = dict(M=100, N=64, K=64, x_dt=1, dt=1, act=0, x_row=64, out_row=64, w=P, w_scale=P)
    c.update(kw)
    return _lib.Linear8Call(**c)


@pytest.mark.parametrize("kw,status", [
    (dict(M=0), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(K=60), INVALID), (dict(x_dt=3), INVALID),
    (dict(dt=2), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(x_row=60), INVALID),
    (dict(x_row=-64), INVALID), (dict(out_row=63), INVALID), (dict(x_scale=P), INVALID), (dict(x_dt=2), INVALID),
    (dict(x_dt=2, x_scale=P + 2), INVALID), (dict(w=None), INVALID), (dict(w=P + 8), INVALID), (dict(w_scale=None), INVALID),
    (dict(w_scale=P + 1), INVALID), (dict(bias=P + 1), INVALID), (dict(dt=0, bias=P + 2), INVALID),
    (dict(K=65552, x_dt=2, x_scale=P), UNSUPPORTED), (dict(N=1048577, out_row=1048577), UNSUPPORTED),
])
def test_linear_refuses_calls(lib, kw, status):
    c = linear(**kw)
    assert lib.mpm_linear_int8(R(c), ptr(), ptr(), ptr(), 1 << 40, None) == status
    assert lib.mpm_linear_int8_workspace_bytes(R(c)) == 0


def test_linear_refuses_pointers(lib):
    c = linear()
    go = lambda x=ptr(), out=ptr(), ws=ptr(), n=1 << 40: lib.mpm_linear_int8(R(c), x, out, ws, n, None)
    assert lib.mpm_linear_int8(None, ptr(), ptr(), None, 0, None) == INVALID
    assert go(x=None) == INVALID and go(x=ptr(P + 8)) == INVALID and go(out=None) == INVALID and go(out=ptr(P + 1)) == INVALID
    assert lib.mpm_linear_int8_workspace_bytes(R(c)) == 0  # (few results)
    c = linear(M=5000)
    need = lib.mpm_linear_int8_workspace_bytes(R(c))
    assert need >= 5000 * 64 + 20000 and go(n=need - 1) == WORKSPACE and go(ws=None) == INVALID and go(ws=ptr(P + 64)) == INVALID
    assert lib.mpm_linear_int8_workspace_bytes(R(linear(x_dt=2, x_scale=P))) == 0


def group(**kw):
    c = dict(R=12, C=64, groups=8, dt=1, act=0, eps=1e-5, B=2)
    c.update(kw)
    return _lib.GroupNormCall(**c)


@pytest.mark.parametrize("kw,status", [
    (dict(R=0), INVALID), (dict(C=0), INVALID), (dict(C=60, groups=6), INVALID), (dict(groups=0), INVALID),
    (dict(groups=7), INVALID), (dict(dt=2), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID),
    (dict(eps=-1e-5), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(B=0), INVALID),
    (dict(B=5), INVALID), (dict(off=P + 2), INVALID), (dict(b=P), INVALID), (dict(w=P + 8), INVALID),
    (dict(w=P, b=P + 4), INVALID), (dict(C=16392), UNSUPPORTED), (dict(B=65536, off=P), UNSUPPORTED),
])
def test_group_norm_refuses_calls(lib, kw, status):
    c = group(**kw)
    dw, db = (ptr() if getattr(c, n) else None for n in "wb")
    assert lib.mpm_group_norm(R(c), ptr(), ptr(), None, ptr(), 1 << 40, None) == status
    assert lib.mpm_group_norm_backward(R(c), ptr(), ptr(), ptr(), ptr(), dw, db, ptr(), 1 << 40, None) == status
    assert lib.mpm_group_norm_workspace_bytes(R(c)) == lib.mpm_group_norm_backward_workspace_bytes(R(c)) == 0


def test_group_norm_refuses_pointers(lib):
    big = 1 << 40
    assert lib.mpm_group_norm(None, ptr(), ptr(), None, ptr(), big, None) == INVALID
    for args in ((None, ptr(), None), (ptr(), None, None), (ptr(P + 8), ptr(), None), (ptr(), ptr(P + 4), None),
                 (ptr(), ptr(), ptr(P + 4))):
        assert lib.mpm_group_norm(R(group()), *args, ptr(), big, None) == INVALID
    back = lambda c, *a, ws=ptr(), n=big: lib.mpm_group_norm_backward(R(c), *a, ws, n, None)
    ok = [ptr()] * 4
    for i in range(4):
        for bad in (None, ptr(P + 4)):
            assert back(group(), *(bad if j == i else p for j, p in enumerate(ok)), None, None) == INVALID
    assert back(group(), *ok, ptr(), None) == INVALID and back(group(w=P), *ok, None, None) == INVALID
    assert back(group(w=P), *ok, ptr(), ptr()) == INVALID and back(group(w=P, b=P), *ok, ptr(), None) == INVALID
    assert back(group(w=P), *ok, ptr(P + 8), None) == INVALID
    need = lib.mpm_group_norm_backward_workspace_bytes(R(group(R=400000)))
    assert need > 0 and back(group(R=400000), *ok, None, None, n=need - 1) == WORKSPACE
    assert back(group(R=400000), *ok, None, None, ws=ptr(P + 16)) == INVALID


INJECT = r"""
import ctypes, json
from paper_2604_05718_amd import _lib
lib, r, p, big = _lib.load(), ctypes.byref, ctypes.c_void_p(0x10000), 1 << 40
h = r(_lib.Heads(0x10000, 64, 64))
c = _lib.RotaryCall(R=4, H=1, dh=64, dt=1, pairs=32, axes=1, grid=(ctypes.c_int32 * 3)(4, 1, 1), freq=0x10000, B=1)
l = _lib.Linear8Call(M=4, N=8, K=64, x_dt=1, dt=1, x_row=64, out_row=8, w=0x10000, w_scale=0x10000)
g = _lib.GroupNormCall(R=4, C=64, groups=8, dt=1, eps=1e-5, B=1)
print(json.dumps([
    lib.mpm_rotary(r(c), h, h, 0, None), lib.mpm_rotary_backward(r(c), h, h, h, p, p, big, None),
    lib.mpm_quantize_rows(p, 4, 64, 64, 1, p, p, None), lib.mpm_linear_int8(r(l), p, p, p, big, None),
    lib.mpm_group_norm(r(g), p, p, None, p, big, None),
    lib.mpm_group_norm_backward(r(g), p, p, p, p, None, None, p, big, None),
    lib.mpm_quantize_rows(p, 0, 64, 64, 1, p, p, None)]))
"""


def test_injected_launch_failures():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, MPM_FAULT_INJECT="launch", PYTHONPATH=root)
    env.pop("MPM_CHECKED", None)
    p = subprocess.run([sys.executable, "-c", INJECT], capture_output=True, text=True, cwd=root, env=env, timeout=100)
    assert p.returncode == 0, p.stderr[-2000:]
    assert json.loads(p.stdout) == [4] * 6 + [1]  # MPM_ERR_HIP; argument errors come first


def test_gelu_of_bfloat16_results():
    """The polynomial form against GELU over |z| <= 40, in 64 bits (float32 adds 2^-20)."""
    z = torch.linspace(-40, 40, 400001, dtype=torch.float64)
    off = (ref.gelu_bf16(z) - ref.act(z, "gelu")).abs()
    assert bool((off <= ref.gelu_bf16_bound(z)).all())
    assert float((off / ref.act(z, "gelu").abs().clamp_min(1e-4)).max()) < 2.0 ** -8 / 3


# ---- the bindings ------------------------------------------------------------------------


@pytest.fixture
def recorded(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(block_ops._lib, "load", lambda: lib)
    monkeypatch.setattr(block_ops, "_stream", lambda t: "stream")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return lib


def test_bindings_refuse_host_tensors():
    t = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError, match="GPU"):
        mpm.rotary(t, torch.zeros(1, 4), grid=(4,))
    for call in (lambda: mpm.quantize_rows(t[0]), lambda: mpm.linear_int8(t[0], t[0].to(torch.int8), t[0, 0]),
                 lambda: mpm.group_norm(t, 2)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_rotary_binding(recorded):
    x, f = device(torch.zeros(6, 4, 16)), device(torch.zeros(2, 8))
    off, pos = device(torch.zeros(3, dtype=torch.int32)), device(torch.zeros(6, dtype=torch.int32))
    out = mpm.rotary(x, f, pos=pos, grid=(3, 5), layout="pairs", off=off, inverse=True)
    name, (c, hx, ho, inverse, stream) = recorded.calls[0]
    assert name == "mpm_rotary" and out.shape == x.shape and inverse == 1 and stream == "stream"
    assert (c.R, c.H, c.dh, c.dt, c.pairs, c.layout, c.axes, list(c.grid)) == (6, 4, 16, 0, 8, 1, 2, [3, 5, 1])
    assert (c.freq_per_head, c.pos, c.B, c.off) == (0, pos.data_ptr(), 2, off.data_ptr())
    assert (hx.p, hx.row, hx.head) == (x.data_ptr(), 64, 16)
    whole = device(torch.zeros(3, 5, 12, 16))
    mpm.rotary(whole[:, :, :8], device(torch.zeros(8, 1, 8)), grid=(5,), out=whole[:, :, :8])
    c, hx, ho = recorded.calls[1][1][:3]
    assert (c.R, c.H, c.B, c.freq_per_head, c.pos) == (15, 8, 3, 1, None) and (hx.row, hx.p) == (192, whole.data_ptr())
    assert (ho.p, ho.row) == (hx.p, hx.row)
    bad = [dict(freq=device(torch.zeros(3, 8))), dict(freq=device(torch.zeros(5, 2, 8))), dict(grid=(3,)), dict(grid=()),
           dict(layout="whole"), dict(pos=device(torch.zeros(5, dtype=torch.int32))), dict(pos=device(torch.zeros(6))),
           dict(freq=device(torch.zeros(2, 8, dtype=torch.float64))), dict(out=device(torch.zeros(6, 4, 8))),
           dict(out=device(torch.zeros(5, 4, 16))), dict(out=device(torch.zeros(6, 1, 16)).expand(6, 4, 16)),
           dict(out=device(torch.zeros(1, 4, 16)).expand(6, 4, 16)), dict(grid=(1 << 20, 1 << 20)), dict(grid=(2 ** 32 + 3, 5))]
    for kw in bad:
        with pytest.raises(ValueError):
            mpm.rotary(**{**dict(x=x, freq=f, grid=(3, 5)), **kw})
    with pytest.raises(ValueError, match="offsets"):
        mpm.rotary(whole, f, grid=(3, 5), off=off)
    with pytest.raises(TypeError):
        mpm.rotary(device(torch.zeros(6, 4, 16, dtype=torch.float16)), f, grid=(3, 5))
    assert len(recorded.calls) == 2


def test_rotary_backward_binding(recorded):
    x, f = device(torch.zeros(6, 4, 16)), device(torch.zeros(2, 8))
    g = mpm.rotary_backward(x, x, f, grid=(3, 5))
    assert g.dfreq.shape == f.shape and recorded.calls[0][1][2].p == x.data_ptr()
    g = mpm.rotary_backward(x, None, f, grid=(3, 5), with_dfreq=False, dx=x)
    name, (c, hd, hx, hg, dfreq, ws, need, stream) = recorded.calls[1]
    assert g.dx is x and g.dfreq is None and hx is None and dfreq is None and need == 0 and hg.p == x.data_ptr()
    empty = device(torch.zeros(0, 4, 16))
    assert mpm.rotary(empty, f, grid=(3, 5)).shape == empty.shape
    g = mpm.rotary_backward(empty, empty, f, grid=(3, 5))
    assert g.dx.shape == empty.shape and not g.dfreq.any() and len(recorded.calls) == 2


def test_rotary_frequencies():
    f = mpm.rotary_frequencies(5, 2, theta=16.0)
    assert f.shape == (2, 5) and f.dtype is torch.float32
    assert torch.allclose(f[0, ::2], 16.0 ** -(torch.arange(3) / 3)) and torch.allclose(f[1, 1::2], f[0, :4:2])
    assert not f[0, 1::2].any() and not f[1, ::2].any()
    for bad in ((0, 2), (4, 0), (4, 4), (4, 2, 0.0)):
        with pytest.raises(ValueError):
            mpm.rotary_frequencies(*bad)


def test_linear_binding(recorded):
    bf = torch.bfloat16
    x, w = device(torch.zeros(5, 40, dtype=bf)), device(torch.zeros(6, 48, dtype=torch.int8))
    ws, b = device(torch.zeros(6)), device(torch.zeros(6, dtype=bf))
    y = mpm.linear_int8(x, w, ws, bias=b, activation="gelu")
    name, (c, xp, yp, wp, need, stream) = recorded.calls[0]
    assert name == "mpm_linear_int8" and y.shape == (5, 6) and y.dtype is bf and xp == x.data_ptr()
    assert (c.M, c.N, c.K, c.x_dt, c.dt, c.act, c.x_row, c.out_row, c.x_scale) == (5, 6, 40, 1, 1, 3, 40, 6, None)
    q, s = device(torch.zeros(5, 48, dtype=torch.int8)), device(torch.zeros(5))
    wide = device(torch.zeros(5, 20))
    assert mpm.linear_int8(q, w, ws, x_scale=s, out=wide[:, 3:9]).dtype is torch.float32
    c = recorded.calls[1][1][0]
    assert (c.x_dt, c.dt, c.x_scale, c.out_row) == (2, 0, s.data_ptr(), 20)
    assert mpm.linear_int8(q, w, ws, x_scale=s).dtype is bf
    assert mpm.linear_int8(x[:0], w, ws).shape == (0, 6) and len(recorded.calls) == 3
    bad = [dict(weight=device(torch.zeros(6, 40, dtype=torch.int8))), dict(weight=device(torch.zeros(6, 48))),
           dict(weight_scale=device(torch.zeros(5))), dict(bias=ws), dict(bias=device(torch.zeros(5, dtype=bf))),
           dict(activation="tanh"), dict(x_scale=s), dict(x=q[:, :40], x_scale=s), dict(x=q, x_scale=device(torch.zeros(4))),
           dict(x=device(torch.zeros(40, 5, dtype=bf)).t()), dict(x=device(torch.zeros(40, dtype=bf))),
           dict(out=device(torch.zeros(5, 7, dtype=bf))), dict(out=device(torch.zeros(6, 5, dtype=bf)).t()),
           dict(out=device(torch.zeros(5, 6, dtype=bf)), dtype=torch.float32),
           dict(out=device(torch.zeros(1, 6, dtype=bf)).expand(5, 6))]
    for kw in bad:
        with pytest.raises(ValueError):
            mpm.linear_int8(**{**dict(x=x, weight=w, weight_scale=ws), **kw})
    with pytest.raises(TypeError):
        mpm.linear_int8(x.to(torch.float16), w, ws)
    q, scale = mpm.quantize_rows(device(torch.zeros(5, 40)))
    assert q.shape == (5, 48) and q.dtype is torch.int8 and scale.shape == (5,)
    assert recorded.calls[3][0] == "mpm_quantize_rows" and mpm.quantize_rows(x[:0])[0].shape == (0, 48)


@pytest.mark.parametrize("at,ok", [((0, 0), False), ((0, 34), False), ((0, 40), True), ((0, 58), True), ((4, 0), False),
                                   ((4, 40), True), ((5, 0), True), ((5, 40), True)])
def test_linear_out_beside_x(recorded, at, ok):
    """out in the buffer of x: beside its columns or behind its rows, not on them."""
    buffer = device(torch.zeros(10, 64, dtype=torch.bfloat16))
    w, ws = device(torch.zeros(6, 48, dtype=torch.int8)), device(torch.zeros(6))
    x, out = buffer[:5, :40], buffer[at[0]:at[0] + 5, at[1]:at[1] + 6]
    if ok:
        assert mpm.linear_int8(x, w, ws, out=out) is out and len(recorded.calls) == 1
        return
    with pytest.raises(ValueError, match="overlap"):
        mpm.linear_int8(x, w, ws, out=out)


def test_group_norm_binding(recorded):
    x, w = device(torch.zeros(2, 3, 5, 16)), device(torch.ones(16))
    y, stats = mpm.group_norm(x, 4, w, w, activation="silu", with_stats=True)
    name, (c, xp, yp, sp, ws, need, stream) = recorded.calls[0]
    assert name == "mpm_group_norm" and y.shape == x.shape and stats.shape == (2, 4, 2)
    assert (c.R, c.C, c.groups, c.dt, c.act, c.B, c.off) == (30, 16, 4, 0, 2, 2, None)
    stats = device(stats)  # (made on the host, as nothing of this is on a GPU)
    g = mpm.group_norm_backward(x, x, stats, 4, w, w, activation="silu", dx=x)
    assert g.dx is x and g.dweight.shape == g.dbias.shape == (16,)
    rows, off = x.view(30, 16), device(torch.zeros(4, dtype=torch.int32))
    mpm.group_norm(rows, 4, off=off, out=rows)
    c = recorded.calls[2][1][0]
    assert (c.R, c.B, c.off) == (30, 3, off.data_ptr())
    for kw in (dict(x=rows), dict(off=off), dict(weight=device(torch.ones(15))), dict(activation="tanh"),
               dict(x=x.transpose(1, 2)), dict(weight=device(torch.ones(16, dtype=torch.bfloat16))),
               dict(out=device(torch.zeros(30, 16))), dict(x=w)):
        with pytest.raises(ValueError):
            mpm.group_norm(**{**dict(x=x, groups=4), **kw})
    for kw in (dict(dy=rows), dict(stats=device(torch.zeros(2, 4))), dict(dx=rows)):
        with pytest.raises(ValueError):
            mpm.group_norm_backward(**{**dict(dy=x, x=x, stats=stats, groups=4), **kw})
    empty = device(torch.zeros(0, 16))
    y, stats = mpm.group_norm(empty, 4, w, w, off=off, with_stats=True)
    g = mpm.group_norm_backward(empty, empty, device(stats), 4, w, w, off=off)
    assert not stats.any() and not g.dweight.any() and not g.dbias.any() and len(recorded.calls) == 3


def test_the_device_of_the_tensor_is_current_for_the_launch(recorded, monkeypatch):
    """A tensor on another device than the current one: the call runs with its device current."""
    entered = []

    class On:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            entered.append(self.d)

        def __exit__(self, *a):
            entered.append("left")

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(torch.cuda, "device", On)
    mpm.quantize_rows(device(torch.zeros(5, 40)))
    assert entered == [0, "left"]
