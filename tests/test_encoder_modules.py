"""What the encoder's modules keep when their type, device or weights change."""
import copy

import pytest
import torch

from paper_2604_05718_amd import blocks

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
