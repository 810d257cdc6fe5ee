"""What the norms around a block and attention do with rows of no image, without a GPU: which calls are refused and what the
bindings ask for."""
import ctypes

import pytest
import torch

import paper_2604_05718_amd as mpm
from paper_2604_05718_amd import _lib, block_ops
from test_block_bindings import Recorder, device

P = 0x10000
INVALID = 1


def test_refusals():
    lib, r, p, q = _lib.load(), ctypes.byref, ctypes.c_void_p(P), ctypes.c_void_p(2 * P)
    call = lambda clear: r(_lib.NormCall(R=6, D=64, dt=_lib.MPM_BF16, eps=1e-6, B=2, off=P, gate=P, clear=clear))
    for clear in (4, -1, 7):
        assert lib.mpm_residual_norm(call(clear), p, p, q, None, None, None) == INVALID
        g = _lib.NormGrads(P, P, None, None, None, None, None, P)
        assert lib.mpm_residual_norm_backward(call(clear), p, None, p, p, p, r(g), p, 1 << 40, None) == INVALID
        assert lib.mpm_residual_norm_backward_workspace_bytes(call(clear)) == 0
    for clear in (_lib.MPM_CLEAR_SUM, _lib.MPM_CLEAR_SUM | _lib.MPM_CLEAR_ROWS):  # y at x keeps its rows
        assert lib.mpm_residual_norm(call(clear), p, p, p, None, None, None) == INVALID


def test_attention_refusals():
    lib, r = _lib.load(), ctypes.byref
    h = [r(_lib.Heads(P, 64, 64)) for _ in range(8)]
    for kw in (dict(q_rows=-1), dict(k_rows=-1)):
        c = r(_lib.AttentionCall(B=1, Nq=40, Nk=40, H=1, Hk=1, dh=64, dt=1, scale=0.1, q_off=P, k_off=P, **kw))
        assert lib.mpm_attention(c, *h[:4], None, None, 0, None) == INVALID
        assert lib.mpm_attention_backward(c, *h[:5], P, *h[5:], None, P, 1 << 40, None) == INVALID


def test_bindings(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(block_ops._lib, "load", lambda: lib)
    monkeypatch.setattr(block_ops, "_stream", lambda t: None)
    x, gate, off = device(torch.zeros(6, 16)), device(torch.zeros(2, 16)), device(torch.zeros(3, dtype=torch.int32))
    mpm.residual_norm(x, x, gate=gate, off=off)
    mpm.residual_norm(x, x, gate=gate, off=off, out=x)
    asked = lambda i: lib.calls[i][1][0].clear
    assert asked(0) == _lib.MPM_CLEAR_ROWS | _lib.MPM_CLEAR_SUM and asked(1) == _lib.MPM_CLEAR_ROWS
    mpm.residual_norm_backward(x, None, x, x, device(torch.zeros(6, 4)), gate=gate, off=off)
    assert lib.calls[-1][0] == "mpm_residual_norm_backward" and asked(-1) == _lib.MPM_CLEAR_ROWS
    qkv = device(torch.zeros(6, 4, 8))
    at = dict(q_off=off, k_off=off, Nq=3, Nk=3)
    for clear in (True, False):
        mpm.attention(qkv[:, :2], qkv[:, 2:3], qkv[:, 3:], clear=clear, **at)
        assert (lib.calls[-1][1][0].q_rows, lib.calls[-1][1][0].k_rows) == (6 * clear, 0)
        grads = dict(dq=qkv[:, :2], dk=qkv[:, 2:3], dv=qkv[:, 3:])
        mpm.attention_backward(qkv[:, :2], qkv[:, :2], qkv[:, 2:3], qkv[:, 3:], qkv[:, :2], device(torch.zeros(6, 2, 2)),
                               clear=clear, **grads, **at)
        assert (lib.calls[-1][1][0].q_rows, lib.calls[-1][1][0].k_rows) == (6 * clear, 6 * clear)
