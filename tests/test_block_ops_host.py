"""Refusals of the operators of the blocks: every check runs on the host, before any launch."""
import ctypes

import pytest
import torch

import paper_2604_05718_amd as mpm
from paper_2604_05718_amd import _lib

P = 0x10000  # a stand-in device pointer: never dereferenced


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def heads(p=P, row=64, head=64):
    return _lib.Heads(p, row, head)


def call(**kw):
    c = dict(B=2, Nq=8, Nk=8, H=4, Hk=2, dh=64, dt=_lib.MPM_BF16, scale=0.125)
    c.update(kw)
    return _lib.AttentionCall(**c)


def attend(lib, c, q=None, k=None, v=None, out=None, lse=None):
    r = ctypes.byref
    hs = [heads() if x is None else x for x in (q, k, v, out)]
    return lib.mpm_attention(None if c is None else r(c), *(r(x) for x in hs), lse, None, 0, None)


INVALID, UNSUPPORTED, WORKSPACE = _lib.MPM_ERR_INVALID_ARG, _lib.MPM_ERR_UNSUPPORTED, _lib.MPM_ERR_WORKSPACE
BIAS = dict(bias=P, span=7, grid_h=8, grid_w=8)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(Nq=0), INVALID), (dict(Nk=0), INVALID), (dict(H=0), INVALID), (dict(Hk=0), INVALID),
    (dict(H=3), INVALID), (dict(dh=0), INVALID), (dict(dh=4), INVALID), (dict(dh=66), INVALID), (dict(dt=2), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(q_off=P + 2), INVALID),
    (dict(k_off=P + 1), INVALID), (dict(k_bias=P + 2), INVALID), (dict(BIAS, span=-1), INVALID),
    (dict(BIAS, span=64), INVALID), (dict(BIAS, grid_h=0), INVALID), (dict(BIAS, grid_w=16385), INVALID),
    (dict(BIAS, q_pos=P + 2), INVALID), (dict(BIAS, bias=P + 2), INVALID), (dict(B=65536), UNSUPPORTED),
    (dict(Nq=16385), UNSUPPORTED), (dict(Nk=16385), UNSUPPORTED), (dict(H=2048), UNSUPPORTED), (dict(dh=136), UNSUPPORTED),
])
def test_attention_refuses_calls(lib, kw, status):
    assert attend(lib, call(**kw)) == status
    assert lib.mpm_attention_workspace_bytes(ctypes.byref(call(**kw))) == 0
    assert lib.mpm_attention_backward_workspace_bytes(ctypes.byref(call(**kw))) == 0


@pytest.mark.parametrize("bad", [heads(p=None), heads(p=P + 8), heads(row=60), heads(head=-8), heads(row=-64)])
@pytest.mark.parametrize("which", ["q", "k", "v", "out"])
def test_attention_refuses_rows(lib, bad, which):
    assert attend(lib, call(), **{which: bad}) == INVALID


def test_attention_refuses_null_call_and_lse(lib):
    assert attend(lib, None) == INVALID
    assert attend(lib, call(), lse=ctypes.c_void_p(P + 2)) == INVALID


def test_backward_refuses(lib):
    r = ctypes.byref
    h = [r(heads()) for _ in range(8)]
    p = ctypes.c_void_p(P)
    back = lambda c, lse=p, dbias=None, ws=p, n=1 << 40: lib.mpm_attention_backward(
        r(c), *h[:5], lse, *h[5:], dbias, ws, n, None)
    assert back(call(), lse=None) == INVALID
    assert back(call(), dbias=p) == INVALID  # no bias
    assert back(call(), ws=None) == INVALID
    assert back(call(), ws=ctypes.c_void_p(P + 16)) == INVALID
    c = call(**BIAS)
    need = lib.mpm_attention_backward_workspace_bytes(r(c))
    assert need > lib.mpm_attention_backward_workspace_bytes(r(call())) > 0
    assert back(c, dbias=p, n=need - 1) == WORKSPACE


def test_bias_refuses(lib):
    p = ctypes.c_void_p(P)
    ok = dict(table=p, lut=p, nb=5, span=7, H=3, dt=1, out=p)
    for kw, status in ((dict(table=None), INVALID), (dict(lut=None), INVALID), (dict(out=None), INVALID),
                       (dict(nb=0), INVALID), (dict(span=-1), INVALID), (dict(H=0), INVALID), (dict(dt=7), INVALID),
                       (dict(lut=ctypes.c_void_p(P + 2)), INVALID), (dict(span=64), UNSUPPORTED),
                       (dict(nb=128), UNSUPPORTED), (dict(H=1025), UNSUPPORTED)):
        a = {**ok, **kw}
        args = (a["nb"], a["span"], a["H"], a["dt"])
        assert lib.mpm_bias_expand(a["table"], a["lut"], *args, a["out"], None) == status
        assert lib.mpm_bias_gradient(a["out"], a["lut"], *args, a["table"], None) == status


def norm(**kw):
    c = dict(R=6, D=64, dt=_lib.MPM_BF16, kind=0, eps=1e-6, B=1)
    c.update(kw)
    return _lib.NormCall(**c)


@pytest.mark.parametrize("kw,status", [
    (dict(R=0), INVALID), (dict(D=0), INVALID), (dict(D=60), INVALID), (dict(dt=5), INVALID), (dict(kind=2), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(b=P), INVALID), (dict(post_b=P), INVALID),
    (dict(post_w=P + 8), INVALID), (dict(scale=P + 2), INVALID), (dict(gate=P, B=0), INVALID), (dict(gate=P, B=4), INVALID),
    (dict(gate=P, B=2, off=P + 2), INVALID), (dict(gate=P, B=65536, off=P), UNSUPPORTED), (dict(D=16392), UNSUPPORTED),
])
def test_norm_refuses_calls(lib, kw, status):
    p = ctypes.c_void_p(P)
    r = ctypes.byref
    c = norm(**kw)
    assert lib.mpm_residual_norm(r(c), p, p, p, None, None, None) == status
    g = _lib.NormGrads(P, P)
    assert lib.mpm_residual_norm_backward(r(c), p, None, p, p, p, r(g), p, 1 << 40, None) == status
    assert lib.mpm_residual_norm_backward_workspace_bytes(r(c)) == 0


def test_norm_refuses_pointers(lib):
    p, odd, r = ctypes.c_void_p(P), ctypes.c_void_p(P + 8), ctypes.byref
    assert lib.mpm_residual_norm(None, p, p, p, None, None, None) == INVALID
    for args in ((None, p, p, None, None), (p, None, p, None, None), (p, p, None, None, None), (odd, p, p, None, None),
                 (p, p, p, p, None), (p, p, p, None, odd)):  # h without a weight; odd stats
        assert lib.mpm_residual_norm(r(norm()), *args, None) == INVALID
    assert lib.mpm_residual_norm(r(norm(w=P)), p, p, p, None, None, None) == INVALID  # a weight without h
    back = lambda c, g, dh=None, ws=p, n=1 << 40: lib.mpm_residual_norm_backward(r(c), p, dh, p, p, p, r(g), ws, n, None)
    full = _lib.NormGrads(P, P)
    assert back(norm(), _lib.NormGrads(None, P)) == INVALID
    assert back(norm(scale=P), full) == INVALID       # no dscale
    assert back(norm(), _lib.NormGrads(P, P, P)) == INVALID  # dw without w
    assert back(norm(w=P), _lib.NormGrads(P, P, P)) == INVALID  # no dh
    need = lib.mpm_residual_norm_backward_workspace_bytes(r(norm()))
    assert need > 0 and back(norm(), full, n=need - 1) == WORKSPACE
    assert back(norm(), full, ws=None) == INVALID


def test_bindings_refuse_host_tensors():
    t = torch.zeros(4, 2, 8)
    off = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        mpm.attention(t, t, t, q_off=off, k_off=off, Nq=4, Nk=4)
    with pytest.raises(ValueError, match="device"):
        mpm.residual_norm(t.view(4, 16), t.view(4, 16))
    with pytest.raises(ValueError, match="device"):
        mpm.bias_expand(torch.zeros(9, 2), torch.arange(3, dtype=torch.int32))


def test_bucket_lut():
    lut, nb = mpm.bucket_lut(5)
    assert nb == 11 and lut.tolist() == list(range(11))
    lut, nb = mpm.bucket_lut(20, 5)
    assert nb == 11 and len(lut) == 41 and lut.tolist() == sorted(lut.tolist())
    assert lut[20] == 5 and lut[21:24].tolist() == [6, 7, 8] and lut[40] == 10 and lut[0] == 0
    assert (lut + lut.flip(0) == 10).all()
    assert mpm.bucket_lut(0)[1] == 1
    with pytest.raises(ValueError):
        mpm.bucket_lut(4, 5)
