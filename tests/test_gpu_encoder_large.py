"""Rotary positions, 8-bit products and group norm on tensors whose last rows lie past 2^32 bytes and 2^31 elements,
against the same rows alone (the operators give a row the same result wherever it stands)."""
import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
LAST = 300


def rows(R, C, dtype=torch.bfloat16):
    """[R, C] of zeros but for ones in between and random last rows (more than 2^31 values)."""
    assert R * C > 2 ** 31 + LAST * C
    x = torch.zeros((R, C), dtype=dtype, device=DEV)
    x[::1000] = 1
    x[-LAST:] = torch.randn((LAST, C), generator=torch.Generator().manual_seed(C)).to(dtype).to(DEV)
    return x


def test_rotary():
    R, H, dh = 1_060_000, 16, 128
    x = rows(R, H * dh).view(R, H, dh)
    freq = mpm.rotary_frequencies(dh // 2, 2).to(DEV)
    pos = torch.arange(R, device=DEV, dtype=torch.int32) % (32 * 40)
    last = slice(R - LAST, R)
    got = mpm.rotary(x, freq, pos=pos, grid=(32, 40))
    assert torch.equal(got[last], mpm.rotary(x[last], freq, pos=pos[last].contiguous(), grid=(32, 40)))
    got = mpm.rotary_backward(x, x, freq, pos=pos, grid=(32, 40), dx=got, with_dfreq=False).dx
    assert torch.equal(got[last], mpm.rotary(x[last], freq, pos=pos[last].contiguous(), grid=(32, 40), inverse=True))


def test_quantized_rows_and_products():
    R, K, N = 530_000, 4096, 40
    x = rows(R, K)
    w, ws = mpm.quantize_rows(torch.randn((N, K), generator=torch.Generator().manual_seed(1)).to(DEV))
    q, s = mpm.quantize_rows(x)
    ql, sl = mpm.quantize_rows(x[-LAST:])
    assert torch.equal(q[-LAST:], ql) and torch.equal(s[-LAST:], sl)
    y = mpm.linear_int8(x, w, ws)
    assert torch.equal(y[-LAST:], mpm.linear_int8(x[-LAST:], w, ws))
    assert torch.equal(mpm.linear_int8(q, w, ws, x_scale=s), y)


def test_products_of_many_channels():
    M, N, K = 66_000, 32800, 32
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    w, ws = mpm.quantize_rows(torch.randn((N, K), generator=torch.Generator().manual_seed(3)).to(DEV))
    y = mpm.linear_int8(x, w, ws)
    assert y.numel() > 2 ** 31
    assert torch.equal(y[-LAST:], mpm.linear_int8(x[-LAST:], w, ws))


@pytest.mark.parametrize("images", [1, 5])
def test_group_norm(images):
    """The last image against 64 bits (its tolerances: those of the operator's small tests), with the rest of the rows in one
    image or in five."""
    R, C, G = 1_060_000, 2048, 32
    x = rows(R, C)
    off = torch.linspace(0, R - LAST, images + 1).to(torch.int32)
    off = torch.cat([off, torch.tensor([R], dtype=torch.int32)]).to(DEV)
    y, stats = mpm.group_norm(x, G, off=off, activation="silu", with_stats=True)
    dx = mpm.group_norm_backward(x, x, stats, G, off=off, activation="silu").dx
    leaf = x[-LAST:].double().cpu().requires_grad_()
    want = ref.group_norm(leaf, G, [slice(0, LAST)], activation="silu")
    need, = torch.autograd.grad((want * leaf.detach()).sum(), leaf)
    tol = 2.0 ** -8 + 96 * 2.0 ** -24
    for got, w, t in ((y, want.detach(), tol), (dx, need, 2 * tol)):
        assert float((got[-LAST:].double().cpu() - w).norm()) <= t * float(w.norm())
