"""Group norm of values that are not finite, or far from the others, in every form that a call may take: by slabs (groups of
whole vectors and of parts of them) and, for groups too wide for those, by passes whose parts are joined in the second one,
by a launch between, and by channels first."""
import math

import pytest
import torch

import encoder_refs as ref
import paper_2604_05718_amd as mpm

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16

FORMS = [  # dtype, rows, C, groups
    (BF16, 120, 64, 4), (F32, 300, 48, 8), (BF16, 3000, 24, 2), (F32, 1, 16, 2), (F32, 20, 1032, 1), (F32, 100, 2064, 2),
    (BF16, 100, 4128, 2), (F32, 1000, 1032, 1), (BF16, 1000, 4096, 1), (BF16, 9216, 768, 32),
]


@pytest.mark.parametrize("activation", ["none", "relu"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: f"{'bf16' if f[0] is BF16 else 'f32'}-{f[1]}x{f[2]}-{f[3]}")
def test_not_finite(form, value, activation):
    """One value of the second image, in the first row and in late ones: NaN in its group, statistics and gradient, and the other
    groups as without it."""
    dtype, rows, C, G = form
    g = torch.Generator().manual_seed(rows + C)
    x = torch.randn((2, rows, C), generator=g).to(dtype).to(DEV)
    dy = torch.randn((2, rows, C), generator=g).to(dtype).to(DEV)
    w, b = ((1 + 0.2 * torch.randn(C, generator=g)).to(dtype).to(DEV), torch.randn(C, generator=g).to(dtype).to(DEV))
    kw = dict(weight=w, bias=b, activation=activation)
    y, stats = mpm.group_norm(x, G, with_stats=True, **kw)
    d = mpm.group_norm_backward(dy, x, stats, G, **kw)
    for row in sorted({0, rows // 2, rows - 1}):
        c = (row * 7) % C
        i = c // (C // G)
        bad = torch.zeros((2, 1, C), dtype=torch.bool, device=DEV)
        bad[1, 0, i * (C // G):(i + 1) * (C // G)] = True
        z = x.clone()
        z[1, row, c] = value
        got, st = mpm.group_norm(z, G, with_stats=True, **kw)
        assert torch.equal(got.isnan(), bad.expand_as(got)), (row, c)
        assert torch.equal(got.masked_fill(bad, 0), y.masked_fill(bad, 0))
        assert st[1, i].isnan()[1] and not st[1, i].isfinite()[0]  # (the mean is the infinity, or NaN)
        st[1, i] = stats[1, i]
        assert torch.equal(st, stats)
        st[1, i] = math.nan
        e = mpm.group_norm_backward(dy, z, st, G, **kw)
        assert torch.equal(e.dx.isnan(), bad.expand_as(got)) and torch.equal(e.dx.masked_fill(bad, 0), d.dx.masked_fill(bad, 0))


@pytest.mark.parametrize("form", [(300, 48, 8), (670, 836, 11), (4000, 64, 1), (9216, 64, 2), (2000, 12, 1), (1000, 1032, 1),
                                  (20, 1032, 1), (9216, 768, 32)], ids=lambda f: f"{f[0]}x{f[1]}-{f[2]}")
def test_first_value_far_off(form):
    """Float32: the first value of each group is no reference that costs the mean its digits, however far off. The mean is off
    by its own half step and, as the sum of the N deviations in float32, by at most 96 half steps of their mean magnitude (sums
    of up to 64 values in a thread and of threads by 64 lanes); the deviation, a sum of squares, by 96 half steps and eps' one."""
    rows, C, G = form
    g = torch.Generator().manual_seed(rows + C)
    for k in range(6):
        x = torch.randn((1, rows, C), generator=g)
        x[0, 0, ::C // G] = math.sqrt(rows * C / G) * (0.3 + k * torch.rand(G, generator=g))
        y, stats = mpm.group_norm(x.to(DEV), G, with_stats=True)
        v = x[0].double().view(rows, G, C // G)
        mean, var = v.mean(dim=(0, 2)), v.var(dim=(0, 2), correction=0)
        size = (v - mean[None, :, None]).abs().mean(dim=(0, 2))
        off = (stats[0, :, 0].double().cpu() - mean).abs() - 2.0 ** -24 * (mean.abs() + 96 * size)
        assert float(off.max()) <= 0, (k, float(off.max()))
        assert float((stats[0, :, 1].double().cpu() * torch.sqrt(var + 1e-5) - 1).abs().max()) <= 96 * 2.0 ** -24


def test_the_plain_form_agrees():
    """What the formula gives for an infinity (on the CPU in 64 bits)."""
    x = torch.randn((9, 4), generator=torch.Generator().manual_seed(1)).double()
    x[8, 1] = math.inf
    for act in ("none", "relu"):
        y = ref.group_norm(x, 2, [slice(0, 9)], activation=act)
        assert y[:, :2].isnan().all() and y[:, 2:].isfinite().all()
