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
