"""The encoder's modules after a change of type, device or weights, on the GPU."""
import pytest
import torch

from paper_2604_05718_amd.blocks import GridHead, RelativeEncoder, RotaryEncoder

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
GRID, NS, D = (8, 9), [40, 23], 32


def batch(dtype):
    g = torch.Generator().manual_seed(3)
    pos = torch.cat([torch.randperm(72, generator=g)[:n].sort().values for n in NS]).to(torch.int32).to(DEV)
    off = torch.tensor([0, 40, 63], dtype=torch.int32, device=DEV)
    return torch.randn((63, D), generator=g).to(dtype).to(DEV), off, max(NS), pos


@pytest.mark.parametrize("learned", [True, False])
def test_converted(learned):
    """A float32 encoder turned into bfloat16 computes what a bfloat16 one with its parameters does, gradients too."""
    torch.manual_seed(1)
    enc = RotaryEncoder(D, 4, 2, GRID, learned=learned, device=DEV, dtype=torch.float32)
    other = RotaryEncoder(D, 4, 2, GRID, learned=learned, device=DEV)
    enc.to(torch.bfloat16)
    other.load_state_dict(enc.state_dict())
    res = []
    for m in (enc, other):
        y = m.rows(*batch(torch.bfloat16))
        y.float().square().mean().backward()
        res.append([y.detach(), *(t.grad for t in m.parameters())])
    assert len(res[0]) > 20 and all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(*res))


def test_served_after_a_change():
    """The products in 8 bits of a module that moved to the host and back, and of one that loaded other weights."""
    torch.manual_seed(2)
    enc, other = (RotaryEncoder(D, 4, 2, GRID, device=DEV) for _ in range(2))
    at = batch(torch.bfloat16)
    with torch.no_grad():
        want = [m.rows(*at) for m in (enc.quantize(), other.quantize())]
        assert not torch.equal(*want)
        assert torch.equal(enc.cpu().to(DEV).rows(*at), want[0])
        enc.load_state_dict(other.state_dict())
        with pytest.raises(RuntimeError, match="before a capture"), torch.cuda.graph(torch.cuda.CUDAGraph()):
            enc.blocks[0].product("qkv", at[0])
        assert torch.equal(enc.rows(*at), want[1])


@pytest.mark.parametrize("kind", [RotaryEncoder, RelativeEncoder])
def test_without_images(kind):
    """No grid at all: through encoder and head, trained and served."""
    enc, head = kind(D, 4, 2, GRID, device=DEV), GridHead(D, 24, 5, groups=4, device=DEV)
    x = torch.zeros((0, 72, D), device=DEV, dtype=torch.bfloat16)
    assert head(enc(x)).shape == (0, 72, 5)
    off = torch.zeros(1, dtype=torch.int32, device=DEV)
    rows = x.view(0, D).requires_grad_()
    head(enc.rows(rows, off, 0, torch.zeros(0, dtype=torch.int32, device=DEV)), off).sum().backward()
    assert all(p.grad is not None and not p.grad.any() for p in [*enc.parameters(), *head.parameters()])
    enc.quantize()
    head.quantize()
    with torch.no_grad():
        assert head(enc(x)).shape == (0, 72, 5)
