"""Outputs that meet an input: the rotary, group norm and 8-bit bindings take the input itself and memory apart from it, and
refuse the rest. What a refusal has to say is found by marking every value's place (no GPU)."""
import pytest
import torch

import paper_2604_05718_amd as mpm
from paper_2604_05718_amd import block_ops
from test_block_bindings import Recorder, device


@pytest.fixture
def recorded(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(block_ops._lib, "load", lambda: lib)
    monkeypatch.setattr(block_ops, "_stream", lambda t: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return lib


BUFFER = 40 * 96  # values


def places(shape, strides, at):
    return set(torch.arange(BUFFER).as_strided(shape, strides, at).flatten().tolist())


# (strides of x, of out) of 6 rows of 3 heads of 8, and where out starts beside x (in values, multiples of 16 bytes)
VIEWS = [
    ((96, 8, 1), (96, 8, 1)), ((96, 16, 1), (96, 16, 1)), ((24, 8, 1), (24, 8, 1)), ((8, 48, 1), (8, 48, 1)),
    ((16, 96, 1), (16, 96, 1)), ((96, 8, 1), (48, 8, 1)), ((48, 16, 1), (96, 16, 1)), ((0, 8, 1), (24, 8, 1)),
]


@pytest.mark.parametrize("views", VIEWS, ids=str)
def test_rotary(recorded, views):
    """Every start of out around x: refused where it shares values with x and is not x. Views with other strides than x's, whose
    rows may lie in one another's gaps, are refused where their ranges meet."""
    buffer = device(torch.zeros(BUFFER))
    freq, shape, at = device(torch.zeros(1, 4)), (6, 3, 8), 1600
    x = buffer.as_strided(shape, views[0], at)
    mine = places(shape, views[0], at)
    refused = 0
    for start in range(at - 700, at + 700, 4):
        out = buffer.as_strided(shape, views[1], start)
        theirs = places(shape, views[1], start)
        shared = bool(mine & theirs) if views[0] == views[1] else min(mine) <= max(theirs) and min(theirs) <= max(mine)
        same = start == at and views[0] == views[1]
        calls = [(lambda: mpm.rotary(x, freq, grid=(6,), out=out), shared and not same)]
        if views[0][0]:
            calls.append((lambda: mpm.rotary_backward(x, None, freq, grid=(6,), dx=out, with_dfreq=False), shared and not same))
            calls.append((lambda: mpm.rotary_backward(device(torch.zeros(shape)), x, freq, grid=(6,), dx=out), shared))
        for call, bad in calls:
            if bad:
                refused += 1
                with pytest.raises(ValueError, match="overlaps"):
                    call()
            else:
                call()
    assert refused


def test_rotary_of_one_row_or_head(recorded):
    buffer, freq = device(torch.zeros(BUFFER)), device(torch.zeros(1, 4))
    for shape, strides in (((1, 3, 8), (7, 8, 1)), ((6, 1, 8), (24, 5, 1)), ((1, 1, 8), (3, 3, 1))):
        x = buffer.as_strided(shape, strides, 400)
        for start in range(300, 500, 4):
            out = buffer.as_strided(shape, strides, start)
            if start != 400 and places(shape, strides, 400) & places(shape, strides, start):
                with pytest.raises(ValueError, match="overlaps"):
                    mpm.rotary(x, freq, grid=(6,), out=out)
            else:
                mpm.rotary(x, freq, grid=(6,), out=out)


def test_group_norm(recorded):
    buffer, n = device(torch.zeros(2000)), 160
    x, other, stats = buffer[800:800 + n].view(2, 5, 16), device(torch.zeros(2, 5, 16)), device(torch.zeros(2, 4, 2))
    for start in (600, 636, 640, 644, 796, 800, 804, 956, 960, 1000):
        out = buffer[start:start + n].view(2, 5, 16)
        calls = [lambda: mpm.group_norm(x, 4, out=out), lambda: mpm.group_norm_backward(x, other, stats, 4, dx=out),
                 lambda: mpm.group_norm_backward(other, x, stats, 4, dx=out)]
        for call in calls:
            if 640 < start < 960 and start != 800:
                with pytest.raises(ValueError, match="overlaps"):
                    call()
            else:
                call()


def test_no_rows_meet_nothing(recorded):
    x, freq = device(torch.zeros(0, 3, 8)), device(torch.zeros(1, 4))
    assert mpm.rotary(x, freq, grid=(6,), out=device(torch.zeros(0, 3, 16))[:, :, :8]).shape == x.shape


@pytest.mark.parametrize("stride", [6, 8, 40])
@pytest.mark.parametrize("name", ["weight", "weight_scale", "x_scale", "bias"])
def test_linear(recorded, name, stride):
    """out anywhere around each input beside x: rows of 6 results."""
    buffer = torch.zeros(8000, dtype=torch.uint8)
    sizes = dict(weight=(torch.int8, (6, 48)), weight_scale=(torch.float32, (6,)), x_scale=(torch.float32, (5,)),
                 bias=(torch.float32, (6,)))
    given = {n: torch.zeros(s, dtype=t) for n, (t, s) in sizes.items()}
    dtype, shape = sizes[name]
    at, many = 4000, torch.zeros(shape, dtype=dtype).numel() * torch.zeros((), dtype=dtype).element_size()
    given[name] = buffer[at:at + many].view(dtype).view(shape)
    given = {n: device(t) for n, t in given.items()}
    x = device(torch.zeros(5, 48, dtype=torch.int8))
    floats, seen = buffer.view(torch.float32), set()
    for start in range(700, 1150):
        out = device(floats.as_strided((5, 6), (stride, 1), start))
        bad = any(4 * (start + r * stride) < at + many and at < 4 * (start + r * stride + 6) for r in range(5))
        seen.add(bad)
        if bad:
            with pytest.raises(ValueError, match="overlap"):
                mpm.linear_int8(x, out=out, **given)
        else:
            mpm.linear_int8(x, out=out, **given)
    assert seen == {True, False}
