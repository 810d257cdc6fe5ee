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
