"""The trainable blocks with a relative position bias: their gradients through the library's operators
against the same blocks in plain 64-bit torch, a few steps of training, and inference between merges."""
import pytest
import torch

import block_refs as ref
import paper_2604_05718_amd as mpm
from paper_2604_05718_amd.blocks import RelativeEncoder

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def plain(enc, x, ns, pos, gate, grid):
    """enc.rows() in float64 on the CPU from copies of its parameters; returns (rows, parameters)."""
    p = {n: t.detach().double().cpu().requires_grad_() for n, t in enc.named_parameters()}
    rows_of = torch.repeat_interleave(torch.arange(len(ns)), torch.tensor(ns))
    off = torch.cumsum(torch.tensor([0] + ns), 0)
    imgs = ref.images(off, 0, len(ns))
    lut = enc.lut.cpu().long()
    h = ref.unit(x, "layer", 1e-6) * p["norms.0.weight"] + p["norms.0.bias"]
    R, D = x.shape
    for i, blk in enumerate(enc.blocks):
        b = f"blocks.{i}."
        H, W = blk.heads, lut.numel()
        nb = int(p[b + "table"].shape[0] ** 0.5 + 0.5)
        bias = p[b + "table"][(lut[:, None] * nb + lut[None, :]).reshape(-1)].t().reshape(H, W, W)
        q, k, v = (h @ p[b + "qkv"]).view(R, 3, H, D // H).unbind(1)
        a, _ = ref.attention(q, k, v, imgs, imgs, (D // H) ** -0.5, bias, pos, pos, grid)
        for side, f, n in (("attn", lambda: a.reshape(R, D) @ p[b + "proj"], 2 * i + 1),
                           ("mlp", lambda: torch.nn.functional.gelu(h @ p[b + "fc1"]) @ p[b + "fc2"], 2 * i + 2)):
            x, h = ref.residual_norm(x, f(), p[f"norms.{n}.weight"], p[f"norms.{n}.bias"], p[b + side + "_post_weight"],
                                     p[b + side + "_post_bias"], p[b + side + "_scale"], gate, rows_of)
    return h, p


def test_gradients_of_the_blocks():
    """Float32, two blocks on ragged images: rows and every parameter's gradient. Errors grow from the
    operators' own (144 and 288 times 2^-24) through eight products in a row: 16 times that."""
    torch.manual_seed(1)
    ns, grid, D = [40, 1, 23], (8, 9), 32
    enc = RelativeEncoder(D, 4, 2, grid, side=3, device=DEV, dtype=torch.float32)
    pos = torch.cat([torch.randperm(72)[:n].sort().values for n in ns]).to(torch.int32)
    x, gate, g = torch.randn(sum(ns), D), torch.rand(len(ns), D) + 0.5, torch.randn(sum(ns), D)
    off = torch.cumsum(torch.tensor([0] + ns), 0).to(torch.int32)
    xd, gd = x.to(DEV).requires_grad_(), gate.to(DEV).requires_grad_()
    out = enc.rows(xd, off.to(DEV), max(ns), pos.to(DEV), gd)
    (out * g.to(DEV)).sum().backward()
    x64, g64 = x.double().requires_grad_(), gate.double().requires_grad_()
    want, p = plain(enc, x64, ns, pos, g64, grid)
    (want * g.double()).sum().backward()
    tol = 16 * 288 * 2.0 ** -24
    assert ref.rel(out, want) <= tol
    assert ref.rel(xd.grad, x64.grad) <= tol and ref.rel(gd.grad, g64.grad) <= tol
    for n, t in enc.named_parameters():
        assert ref.rel(t.grad, p[n].grad) <= tol, n


def test_training_lowers_the_loss():
    """bfloat16 blocks on tokens merged once: a few steps of gradient descent towards given rows."""
    torch.manual_seed(2)
    B, grid, D = 3, (16, 16), 128
    x = torch.randn(B, 256, D, device=DEV).to(torch.bfloat16)
    m = mpm.merge_local(x, 16, 16)
    total = int(m.y_off[-1])
    rows, pos, most = m.y[:total], m.y_pos[:total], int(torch.diff(m.y_off.cpu()).max())
    enc = RelativeEncoder(D, 2, 2, grid, device=DEV)
    target = torch.randn(total, D, device=DEV)
    losses = []
    for _ in range(8):
        loss = (enc.rows(rows, m.y_off, most, pos).float() - target).square().mean()
        enc.zero_grad()
        loss.backward()
        with torch.no_grad():
            for t in enc.parameters():
                t -= (2.0 * t.grad).to(t.dtype)
        losses.append(loss.item())
    assert all(b < a for a, b in zip(losses, losses[1:])), losses


def test_inference_between_merges():
    """Merges before blocks 1 and 2: tokens of one cluster leave with one value, and without merges the
    packed path equals the grid's."""
    torch.manual_seed(3)
    B, grid, D = 2, (12, 20), 64
    enc = RelativeEncoder(D, 2, 3, grid, side=4, merge_before=(1, 2), device=DEV)
    x = torch.randn(B, 240, D, device=DEV).to(torch.bfloat16)
    out = enc(x)
    torch.cuda.synchronize()
    assert out.shape == (B, 240, D) and torch.isfinite(out).all()
    for b in range(B):
        assert len(torch.unique(out[b].float(), dim=0)) < 240
    enc.merge_before = ()
    off = torch.arange(0, 481, 240, dtype=torch.int32, device=DEV)
    pos = torch.arange(240, dtype=torch.int32, device=DEV).repeat(B)
    assert torch.equal(enc(x).reshape(-1, D), enc.rows(x.reshape(-1, D), off, 240, pos).detach())
