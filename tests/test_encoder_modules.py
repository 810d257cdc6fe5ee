"""What the encoder's modules keep when their type, device or weights change."""
import copy

import pytest
import torch

from paper_2604_05718_amd import block_ops, blocks

CONVERSIONS = {"to": lambda m: m.to(torch.bfloat16), "bfloat16": lambda m: m.bfloat16(), "half": lambda m: m.half(),
               "double": lambda m: m.double(), "and_back": lambda m: m.bfloat16().float()}


@pytest.mark.parametrize("learned", [True, False])
@pytest.mark.parametrize("name", list(CONVERSIONS))
def test_frequencies_stay_float32(name, learned):
    """The rotation takes its frequencies in float32, whatever the blocks' type; they lose no digits on the way."""
    enc = blocks.RotaryEncoder(32, 2, 2, (4, 5), learned=learned, device="cpu", dtype=torch.float32)
    before = copy.deepcopy(enc)
    if learned:
        for b in enc.blocks:
            b.freq.grad = torch.rand_like(b.freq)
            before.blocks[0].freq.grad = enc.blocks[0].freq.grad.clone()
    held = [b.freq for b in enc.blocks]
    assert CONVERSIONS[name](enc) is enc
    want = next(iter(CONVERSIONS[name](torch.nn.Linear(1, 1)).parameters())).dtype
    for b, old, was in zip(enc.blocks, held, before.blocks):
        assert b.freq.dtype is torch.float32 and torch.equal(b.freq, was.freq)
        assert isinstance(b.freq, torch.nn.Parameter) == learned and (not learned or b.freq is old)
        assert b.qkv.dtype is want and b.attn_scale.dtype is want
    if learned:
        assert torch.equal(enc.blocks[0].freq.grad, before.blocks[0].freq.grad)
    enc.to("meta")
    assert enc.blocks[0].freq.is_meta and enc.blocks[0].freq.dtype is torch.float32


def test_frequencies_of_another_type():
    b = blocks.RotaryBlock(32, 2, torch.rand(2, 8, dtype=torch.float64), device="cpu")
    assert b.freq.dtype is torch.float32


@pytest.fixture
def served(monkeypatch):
    """Stand-ins of the 8-bit operators: the weights' rows as steps, by twos."""
    monkeypatch.setattr(block_ops, "quantize_rows", lambda w: ((w * 2).to(torch.int8), torch.full((w.shape[0],), 0.5)))
    monkeypatch.setattr(block_ops, "linear_int8", lambda x, w, s, activation="none": (x.float() @ w.float().t()) * s)


def modules(dtype=torch.float32):
    torch.manual_seed(1)
    enc = blocks.RotaryEncoder(16, 2, 1, (4, 5), device="cpu", dtype=dtype)
    return enc, enc.blocks[0], blocks.GridHead(16, 24, 5, groups=4, device="cpu", dtype=dtype)


def test_steps_follow_the_module(served):
    """To another device and through another type: the steps and their float32 scales as they were."""
    enc, blk, head = modules()
    keys = [list(m.state_dict()) for m in (blk, head)]
    for m in (enc.quantize(), head.quantize()):
        m.bfloat16()
    assert [list(m.state_dict()) for m in (blk, head)] == keys
    for m in (blk, head):
        for n in m.PRODUCTS:
            steps, scale = getattr(m, n + "_steps"), getattr(m, n + "_step_scale")
            assert steps.dtype is torch.int8 and scale.dtype is torch.float32 and bool((scale == 0.5).all())
            assert steps.shape == getattr(m, n).t().shape
    copied = copy.deepcopy(blk)
    assert torch.equal(copied.qkv_steps, blk.qkv_steps) and copied.quantized
    for m in (enc, head):
        m.to("meta")
    assert blk.fc1_steps.is_meta and blk.fc1_step_scale.is_meta and head.inner_steps.is_meta


def test_steps_of_loaded_weights(served):
    """Weights that are loaded after quantize(), into the module or into one around it, are the ones that are served."""
    enc, blk, head = modules()
    enc.quantize()
    x = torch.randn(3, 16)
    state = {n: t.round() + 3 if t.dim() == 2 else t for n, t in enc.state_dict().items()}
    with torch.no_grad():
        old = blk.product("qkv", x)
        enc.load_state_dict(state)
        new = blk.product("qkv", x)
        assert torch.allclose(new, x @ state["blocks.0.qkv"]) and not torch.allclose(new, old)
        steps = blk.qkv_steps
        blk.product("qkv", x)
        assert blk.qkv_steps is steps  # (made once)
        plain = modules()[1]
        plain.load_state_dict(blk.state_dict())
        assert not plain.quantized and torch.equal(plain.product("qkv", x), x @ blk.qkv)


@pytest.mark.parametrize("shape", [(0, 20, 16), (3, 0, 16), (0, 4, 5, 16)])
def test_a_head_without_rows(monkeypatch, shape):
    """No grids, or grids without cells: no scores, and gradients of zeros."""
    def group_norm(x, groups, *args, **kw):
        return torch.empty_like(x), torch.zeros(shape[0], groups, 2)

    def group_norm_backward(dy, x, stats, groups, weight, bias, **kw):
        return block_ops.GroupNormGrads(*(torch.zeros_like(t) for t in (x, weight, bias)))

    monkeypatch.setattr(block_ops, "group_norm", group_norm)
    monkeypatch.setattr(block_ops, "group_norm_backward", group_norm_backward)
    head, x = modules()[2], torch.zeros(shape, requires_grad=True)
    y = head(x)
    assert y.shape == (*shape[:-1], 5)
    y.sum().backward()
    assert x.grad.shape == x.shape and all(not p.grad.any() for p in head.parameters())
    off = torch.zeros(1, dtype=torch.int32)
    assert head(torch.zeros(0, 16), off).shape == (0, 5)
