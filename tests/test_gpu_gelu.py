"""GELU of bfloat16 results and its slope on the GPU: every bfloat16 number as the argument.

Of the normal distribution's integral the kernels have, down to -11, a fit of 2^-17, 4 z^2 2^-24 for the roundings of the
exponent (its partial sums, times the powers of z that they meet, add up to 3.6 z^2 or 4), and 2^-20 for the exponential's
own and the products'. Below, 2^-100 of the result: the fit is within 2^-106 of it in 64 bits and what is below 2^-126 may
become zero."""
import math

import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
BF16 = torch.bfloat16


def arguments():
    """All finite bfloat16 numbers."""
    z = torch.arange(-2 ** 15, 2 ** 15).to(torch.int16).view(BF16)
    return z[z.isfinite()]


def relative(z):
    return 2.0 ** -17 + 2.0 ** -20 + 4 * z * z * 2.0 ** -24


def assert_rounded(got, want, off):
    """got is the rounding to bfloat16 of a value within `off` of want."""
    lo, hi = ((want + s * off).to(torch.float32).to(BF16) for s in (-1, 1))  # (twice rounded: as much as 2^-24 of it)
    bad = ~((lo <= got) & (got <= hi))
    assert not bad.any(), (int(bad.sum()), want[bad][:4], got[bad][:4])


def size(z):
    return (ref.act(z, "gelu").abs() * relative(z).clamp_max(1.0) + 2.0 ** -100)


@pytest.mark.parametrize("M", [1, 300])
def test_of_a_product(M):
    """Rows of zeros, so that the shift is the argument, by few tokens' kernel and by tiles."""
    z = arguments()
    w, ws = torch.zeros((z.numel(), 16), dtype=torch.int8, device=DEV), torch.ones(z.numel(), device=DEV)
    y = mpm.linear_int8(torch.zeros((M, 16), dtype=BF16, device=DEV), w, ws, bias=z.to(DEV), activation="gelu").cpu()
    assert torch.equal(y, y[:1].expand_as(y))
    assert_rounded(y[0], ref.act(z.double(), "gelu"), size(z.double()))
    z = torch.tensor([math.inf, -math.inf, math.nan], dtype=BF16)
    y = mpm.linear_int8(torch.zeros((M, 16), dtype=BF16, device=DEV), w[:3], ws[:3], bias=z.to(DEV), activation="gelu")
    assert torch.equal(y.cpu()[M - 1].isnan(), torch.tensor([False, True, True])) and bool((y[:, 0] == math.inf).all())


def test_of_a_norm_and_its_slope():
    """One row with weights of zero, so that the shift is the argument, and its gradient the slope."""
    z = arguments()
    z = torch.cat([z, torch.zeros(2 ** 16 - z.numel(), dtype=BF16)])
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn((1, 1, 2 ** 14), generator=g).to(BF16).to(DEV), torch.zeros(2 ** 14, dtype=BF16, device=DEV)
    for part in z.split(2 ** 14):
        b = part.to(DEV)
        y, stats = mpm.group_norm(x, 1, w, b, activation="gelu", with_stats=True)
        d = mpm.group_norm_backward(torch.ones_like(x), x, stats, 1, w, b, activation="gelu")
        p = part.double()
        assert_rounded(y.cpu().view(-1), ref.act(p, "gelu"), size(p))
        cdf = torch.special.erfc(-p / math.sqrt(2)) / 2
        pdf = p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)
        assert_rounded(d.dbias.cpu(), cdf + pdf, (cdf + pdf.abs()) * relative(p).clamp_max(1.0) + 2.0 ** -100)
