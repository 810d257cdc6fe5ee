"""The operators of the blocks under the library's two modes, each read once per process and so tested in
a child: MPM_FAULT_INJECT=launch (no GPU) fails every launching entry point after its checks;
MPM_CHECKED=1 validates packed offsets on the device first and launches nothing on bad ones."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

INJECT = r"""
import ctypes, json
from paper_2604_05718_amd import _lib
lib, r, p = _lib.load(), ctypes.byref, ctypes.c_void_p(0x10000)
h = [r(_lib.Heads(0x10000, 64, 64)) for _ in range(8)]
c = _lib.AttentionCall(B=1, Nq=40, Nk=40, H=1, Hk=1, dh=64, dt=1, scale=0.1)
n = _lib.NormCall(R=4, D=64, dt=1, eps=1e-6, B=1)
bad = _lib.NormCall(R=0, D=64, dt=1, eps=1e-6, B=1)
big = 1 << 40
print(json.dumps([
    lib.mpm_attention(r(c), *h[:4], None, None, 0, None),
    lib.mpm_attention_backward(r(c), *h[:5], p, *h[5:], None, p, big, None),
    lib.mpm_bias_expand(p, p, 3, 4, 2, 1, p, None), lib.mpm_bias_gradient(p, p, 3, 4, 2, 1, p, None),
    lib.mpm_residual_norm(r(n), p, p, p, None, None, None),
    lib.mpm_residual_norm_backward(r(n), p, None, p, p, p, r(_lib.NormGrads(0x10000, 0x10000)), p, big, None),
    lib.mpm_residual_norm(r(bad), p, p, p, None, None, None)]))
"""

CHECKED = r"""
import json, sys
import torch
import paper_2604_05718_amd as mpm
d = torch.device("cuda:0")
q = torch.load(sys.argv[1], weights_only=True)
off = lambda *v: torch.tensor(v, dtype=torch.int32, device=d)
res = {}
x = [t.to(d) for t in q]
def attend(qo, ko, **kw):
    out = torch.full_like(x[0], 7)
    try:
        mpm.attention(*x[:3], q_off=qo, k_off=ko, Nq=30, Nk=30, out=out, **kw)
        return 0, out
    except mpm.MPMError as e:
        return e.status, out
good = off(0, 30, 50)
s, out = attend(good, good)
res["valid"] = s
torch.save(out.cpu(), sys.argv[2])
for name, qo, ko in (("queries_too_many", off(0, 31, 50), good), ("keys_decrease", good, off(0, 30, 20)),
                     ("keys_negative", good, off(-1, 20, 50))):
    s, out = attend(qo, ko)
    torch.cuda.synchronize()
    res[name] = [s, bool((out == 7).all())]
rows = x[3]
gate = torch.ones(2, rows.shape[1], device=d, dtype=rows.dtype)
for name, o in (("norm_valid", good), ("norm_past_the_rows", off(0, 30, 51)), ("norm_decrease", off(0, 30, 20))):
    y = torch.full_like(rows, 7)
    try:
        mpm.residual_norm(rows, rows, gate=gate, off=o, out=y)
        s = 0
    except mpm.MPMError as e:
        s = e.status
    torch.cuda.synchronize()
    res[name] = [s, bool((y == 7).all())]
print(json.dumps(res))
"""


def child(code, *args, **env):
    e = {k: v for k, v in os.environ.items() if k not in ("MPM_FAULT_INJECT", "MPM_CHECKED")}
    e.update(env, PYTHONPATH=ROOT)
    p = subprocess.run([sys.executable, "-c", code, *args], capture_output=True, text=True, cwd=ROOT, env=e, timeout=100)
    assert p.returncode == 0, p.stderr[-2000:]
    return json.loads(p.stdout.strip().splitlines()[-1])


def test_injected_launch_failures():
    assert child(INJECT, MPM_FAULT_INJECT="launch") == [4] * 6 + [1]  # MPM_ERR_HIP; argument errors come first


@pytest.mark.gpu
def test_checked_offsets(tmp_path):
    import torch

    import paper_2604_05718_amd as mpm

    g = torch.Generator().manual_seed(1)
    q = [torch.randn(50, 2, 32, generator=g).to(torch.bfloat16) for _ in range(3)] + [torch.randn(50, 64, generator=g)]
    torch.save(q, tmp_path / "in.pt")
    res = child(CHECKED, str(tmp_path / "in.pt"), str(tmp_path / "out.pt"), MPM_CHECKED="1")
    assert res["valid"] == 0 and res["norm_valid"] == [0, False]
    for name in ("queries_too_many", "keys_decrease", "keys_negative", "norm_past_the_rows", "norm_decrease"):
        assert res[name] == [1, True], name
    off = torch.tensor([0, 30, 50], dtype=torch.int32, device="cuda")
    want = mpm.attention(*(t.to("cuda") for t in q[:3]), q_off=off, k_off=off, Nq=30, Nk=30)
    assert torch.equal(want.cpu(), torch.load(tmp_path / "out.pt", weights_only=True))
