"""The bindings of the operators of the blocks without a GPU: what they refuse and what they hand on."""
import pytest
import torch

from paper_2604_05718_amd import block_ops


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a GPU: the checks before a launch can be reached without one."""

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return 0


def device(t):
    return t.as_subclass(OnDevice)


@pytest.fixture
def no_launch(monkeypatch):
    """Anything that gets past the bindings' checks fails."""
    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was reached")

    monkeypatch.setattr(block_ops._lib, "load", Library)


def test_bias_gradient_refuses(no_launch):
    """A lut of even length would make the kernel read past it, and past dbias."""
    lut = lambda n: device(torch.zeros(n, dtype=torch.int32))
    dbias = lambda *s: device(torch.zeros(s))
    with pytest.raises(ValueError, match="odd"):
        block_ops.bias_gradient(dbias(2, 4, 4), lut(4), 3)
    for bad in (dbias(2, 25), dbias(2, 5, 3), dbias(2, 5, 5, 1), dbias(50)):
        with pytest.raises(ValueError, match="dbias"):
            block_ops.bias_gradient(bad, lut(5), 3)
    with pytest.raises(ValueError, match="device"):
        block_ops.bias_gradient(torch.zeros(2, 5, 5), torch.zeros(5, dtype=torch.int32), 3)


def test_workspace_without_the_bias_gradient():
    """A call that asks for no dbias needs no room for its partial sums (host checks of the library: the
    launch is refused for a workspace one byte short, and injected to fail after the checks)."""
    import json
    import os
    import subprocess
    import sys

    code = r"""
import ctypes, json
from paper_2604_05718_amd import _lib
lib, r, p = _lib.load(), ctypes.byref, ctypes.c_void_p(0x10000)
h = [r(_lib.Heads(0x10000, 64, 64)) for _ in range(8)]
kw = dict(B=3, Nq=400, Nk=400, H=2, Hk=2, dh=64, dt=1, scale=0.1)
c = _lib.AttentionCall(**kw, bias=0x10000, span=20, grid_h=20, grid_w=20)
full, less = (lib.mpm_attention_backward_workspace_bytes(r(x)) for x in (c, _lib.AttentionCall(**kw)))
back = lambda dbias, n: lib.mpm_attention_backward(r(c), *h[:5], p, *h[5:], dbias, p, n, None)
print(json.dumps([less < full, back(None, less), back(None, less - 1), back(p, less), back(p, full), back(p, full - 1)]))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, MPM_FAULT_INJECT="launch", PYTHONPATH=root)
    env.pop("MPM_CHECKED", None)
    p = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=root, env=env, timeout=100)
    assert p.returncode == 0, p.stderr[-2000:]
    assert json.loads(p.stdout) == [True, 4, 3, 3, 4, 3]


class Recorder:
    """A library whose calls succeed and are remembered."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace_bytes"):
                return 0
            self.calls.append((name, [getattr(a, "_obj", a) for a in args]))
            return 0
        return call


@pytest.fixture
def recorded(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(block_ops._lib, "load", lambda: lib)
    monkeypatch.setattr(block_ops, "_stream", lambda t: None)
    return lib


def test_one_row_of_dense_images(recorded):
    """A slice of one row of every image, the first tokens of a batch say: the images' stride is the rows'."""
    whole = torch.zeros(3, 20, 4, 16)
    q, kv = device(whole[:, :1]), device(torch.zeros(3, 20, 4, 16))
    block_ops.attention(q, kv, kv)
    (name, (call, hq, hk, hv, ho, *_)), = recorded.calls
    assert name == "mpm_attention" and (call.B, call.Nq, call.Nk) == (3, 1, 20)
    assert (hq.p, hq.row, hq.head) == (whole.data_ptr(), 20 * 64, 16)
    assert (ho.row, ho.head) == (64, 16) and (hk.row, hk.head) == (64, 16)
    block_ops.attention_backward(q, q, kv, kv, q, device(torch.zeros(3, 4, 2)), dq=q, dk=kv, dv=kv)
    args = recorded.calls[1][1]
    assert [h.row for h in args[1:6] + args[7:10]] == [1280, 1280, 64, 64, 1280, 1280, 64, 64]
    with pytest.raises(ValueError, match="dense images"):
        block_ops.attention(device(whole[:, :2]), kv, kv)


def test_strides_that_nothing_is_reached_by(recorded):
    """Of a single row or a single head any stride is right."""
    odd = device(torch.as_strided(torch.zeros(64), (1, 1, 16), (7, 5, 1)))
    off = device(torch.tensor([0, 1], dtype=torch.int32))
    block_ops.attention(odd, odd, odd, q_off=off, k_off=off, Nq=1, Nk=1)
    assert [(h.row, h.head) for h in recorded.calls[0][1][1:4]] == [(0, 0)] * 3


def test_calls_without_rows(no_launch):
    """No query, or no row of a norm: empty results, and gradients that are sums over nothing."""
    q, k = device(torch.zeros(0, 2, 8)), device(torch.ones(5, 2, 8))
    off, k_off = (device(torch.tensor(o, dtype=torch.int32)) for o in ([0, 0, 0], [0, 3, 5]))
    where = dict(q_off=off, k_off=k_off, Nq=0, Nk=3, bias=device(torch.ones(2, 5, 5)), grid=(3, 3))
    out, lse = block_ops.attention(q, k, k, with_lse=True, out=q, **where)
    assert out.shape == (0, 2, 8) and lse.shape == (0, 2, 2)
    g = block_ops.attention_backward(q, q, k, k, out, lse, dq=q, dk=device(torch.ones(5, 2, 8)),
                                     dv=device(torch.ones(5, 2, 8)), **where)
    assert g.dq.shape == q.shape and not g.dk.any() and not g.dv.any() and not g.dbias.any()
    x, w = device(torch.zeros(0, 16)), device(torch.ones(16))
    y, h, stats = block_ops.residual_norm(x, x, weight=w, scale=w, gate=device(torch.ones(3, 16)),
                                          off=device(torch.zeros(4, dtype=torch.int32)), with_stats=True)
    assert y.shape == h.shape == (0, 16) and stats.shape == (0, 4)
    n = block_ops.residual_norm_backward(None, x, x, x, stats, weight=w, scale=w, gate=device(torch.ones(3, 16)),
                                         off=device(torch.zeros(4, dtype=torch.int32)))
    assert n.dx.shape == (0, 16) and n.dgate.shape == (3, 16)
    assert not n.dweight.any() and not n.dscale.any() and not n.dgate.any() and n.dbias is None
