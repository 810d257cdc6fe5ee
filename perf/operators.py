"""The operators of the blocks between the merges, as timed cases.

Attention over packed images whose tokens keep their grid positions, with a learned
relative position bias by buckets (score = scale q.k + table[bucket of the grid offset] +
an optional bias per key), forward and with its gradients; and the norm after a block and
the norm before the next one, fused with the block's gate, its residual scale and the
residual sum, forward and with its gradients.

`run` computes them in plain torch in 32 bits, rounded once at the end, or, where `own` is
set, with the library's calls. Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_INF = float("inf")


def listed():
    return [
        # One 224x224 image (14x14 patches) at ViT-Ti width after a merge: one block's attention
        # in interactive use, nothing but latency.
        dict(name="attend_ti_224", kind="attend", dtype="bf16", B=1, gh=14, gw=14, keep=0.6, H=3, Hk=3, dh=64,
             nq=0, span=13, side=0, kbias=False),
        # ViT-B/16 at 512x512, the benchmark's batch after its merges: packed ragged images, a
        # table entry for every offset of the grid.
        dict(name="attend_b_512", kind="attend", dtype="bf16", B=64, gh=32, gw=32, keep=0.7, H=12, Hk=12, dh=64,
             nq=0, span=31, side=0, kbias=False),
        # ViT-L/16 at 1024x1024, full grids of 4096 tokens, logarithmic buckets: the longest rows
        # of the benchmark's workloads.
        dict(name="attend_l_1024", kind="attend", dtype="bf16", B=8, gh=64, gw=64, keep=1.0, H=16, Hk=16, dh=64,
             nq=0, span=63, side=15, kbias=False),
        # One query (a clicked point) an image against the largest grid the library takes, keys
        # weighted by the tokens they stand for, some dropped.
        dict(name="attend_point", kind="attend", dtype="bf16", B=4, gh=128, gw=128, keep=1.0, H=16, Hk=16, dh=64,
             nq=1, span=63, side=15, kbias=True),
        # float32, shared key heads, odd grid and head width, dropped keys.
        dict(name="attend_odd_f32", kind="attend", dtype="f32", B=5, gh=27, gw=31, keep=0.7, H=6, Hk=2, dh=40,
             nq=0, span=30, side=7, kbias=True),
        # A training step of ViT-B/16 at 512x512 on merged images.
        dict(name="step_b_512", kind="attend_step", dtype="bf16", B=32, gh=32, gw=32, keep=0.7, H=12, Hk=12, dh=64,
             nq=0, span=31, side=0, kbias=False),
        # A training step of ViT-L/16 at 1024x1024 on full grids.
        dict(name="step_l_1024", kind="attend_step", dtype="bf16", B=3, gh=64, gw=64, keep=1.0, H=16, Hk=16, dh=64,
             nq=0, span=63, side=15, kbias=False),
        # A float32 training step of ViT-S/16 at 384x384 (24x24 patches), weighted keys.
        dict(name="step_s_384_f32", kind="attend_step", dtype="f32", B=4, gh=24, gw=24, keep=0.8, H=6, Hk=6, dh=64,
             nq=0, span=23, side=8, kbias=True),
        # The norms around a block of one merged 224x224 image at ViT-Ti width: latency.
        dict(name="norm_ti_224", kind="norm", dtype="bf16", B=1, N=196, keep=0.6, D=192, norm="layer", post=False,
             scale=True, gate="none"),
        # ViT-B/16 at 512x512, merged, a norm on both sides and a gate per image.
        dict(name="norm_b_512", kind="norm", dtype="bf16", B=64, N=1024, keep=0.7, D=768, norm="layer", post=True,
             scale=True, gate="image"),
        # A training step at ViT-L/16 1024x1024.
        dict(name="norm_step_l_1024", kind="norm_step", dtype="bf16", B=16, N=4096, keep=0.7, D=1024, norm="layer",
             post=True, scale=True, gate="image"),
        # float32 root-mean-square norms, a gate per token, odd sizes.
        dict(name="norm_step_odd_f32", kind="norm_step", dtype="f32", B=7, N=837, keep=0.8, D=836, norm="rms",
             post=True, scale=True, gate="row"),
    ]


def _cost(case):
    """A case's weight (float32 products cost sixteen times as much)."""
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] * (16 if case["dtype"] == "f32" else 1) / 1e15


def _largest(kind):
    return max((c for c in listed() if c["kind"] == kind), key=_cost)


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["attend", "attend", "attend_step", "attend_step", "norm", "norm_step"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        keep = rng.choice([1.0, round(rng.uniform(0.4, 0.9), 2)])
        if kind.startswith("norm"):
            case = dict(kind=kind, dtype=dtype, B=log_int(1, 64), N=log_int(49, 4096), keep=keep,
                        D=rng.choice([192, 384, 768, 1024]) if rng.random() < 0.5 else 8 * log_int(6, 256),
                        norm=rng.choice(["layer", "layer", "rms"]), post=rng.random() < 0.6, scale=rng.random() < 0.7,
                        gate=rng.choice(["none", "image", "row"]))
        else:
            gh = log_int(5, 64)
            gw = max(4, min(64, gh + rng.randint(-5, 5)))
            H = rng.choice([3, 4, 6, 8, 12, 16])
            shared = rng.choice([1, 1, 1, 2, 3])
            point = kind == "attend" and rng.random() < 0.25
            if point and rng.random() < 0.5:
                gh, gw = log_int(65, 128), log_int(65, 128)
            most = max(gh, gw) - 1
            span = min(63, most) if rng.random() < 0.6 else rng.randint(3, min(63, max(4, most)))
            side = 0 if rng.random() < 0.5 else rng.randint(2, span)
            case = dict(kind=kind, dtype=dtype, B=log_int(1, 64), gh=gh, gw=gw, keep=keep, H=H,
                        Hk=H // shared if H % shared == 0 else H, dh=rng.choice([64, 64, 64, 32, 40, 80, 128]),
                        nq=rng.choice([1, 1, 2, 7, 20]) if point else 0, span=span, side=side,
                        kbias=rng.random() < 0.4)
            if rng.random() < 0.2:
                case.update(span=0)  # no position bias
            # the plain form holds every score of the batch at once
            if case["B"] * H * (case["nq"] or gh * gw) * gh * gw > 2.2e9:
                continue
            # ... and adds every score's gradient into the table
            if kind == "attend_step" and case["span"] and case["B"] * H * (gh * gw) ** 2 > 8.5e8:
                continue
        if _cost(case) <= _cost(_largest(kind)):
            return case


# ---- inputs ------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _lengths(case, N, seed):
    """Tokens an image, as merges leave them: the same spread around the kept share for every
    seed, dealt to the images in another order."""
    B = case["B"]
    if case["keep"] >= 1.0:
        return torch.full((B,), N, dtype=torch.long)
    g = torch.Generator().manual_seed(int(seed) * 104729 + 11)
    lo, hi = max(0.02, case["keep"] - 0.15), min(1.0, case["keep"] + 0.15)
    n = (torch.linspace(lo, hi, B) * N if B > 1 else torch.tensor([case["keep"] * N])).long().clamp(1, N)
    return n[torch.randperm(B, generator=g)]


def _offsets(n):
    off = torch.zeros((n.numel() + 1,), dtype=torch.int32)
    off[1:] = torch.cumsum(n, 0)
    return off.to(DEV)


def _positions(n, N, g):
    """Sorted grid cells of the tokens each image kept, packed."""
    B = n.numel()
    order = torch.rand((B, N), generator=g, device=DEV).argsort(dim=1)
    kept = torch.arange(N, device=DEV)[None, :] < n.to(DEV)[:, None]
    cells = torch.zeros((B, N), dtype=torch.bool, device=DEV).scatter_(1, order, kept)
    return cells.nonzero()[:, 1].to(torch.int32)


def _lut(span, side):
    """Bucket of a clamped axis offset -span ... span: one each (side 0), or `side` buckets a
    direction, single offsets first and logarithmic widths after them."""
    if side == 0:
        return torch.arange(2 * span + 1, dtype=torch.int32), 2 * span + 1
    exact = max(1, (side + 1) // 2)
    out = []
    for d in range(-span, span + 1):
        a = abs(d)
        if a > exact and span > exact:
            a = min(side, exact + int(math.log(a / exact) / math.log(span / exact) * (side - exact) + 1e-9))
        a = min(a, side)
        out.append(side + (a if d >= 0 else -a))
    return torch.tensor(out, dtype=torch.int32), 2 * side + 1


def _prepare_attend(case, seed):
    g, dt = _generator(seed), _DT[case["dtype"]]
    N, H, Hk, dh = case["gh"] * case["gw"], case["H"], case["Hk"], case["dh"]

    def randn(*shape, s=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * s).to(dt)

    n = _lengths(case, N, seed)
    R = int(n.sum())
    st = dict(case=case, k_off=_offsets(n), Nk=int(n.max()), k_pos=_positions(n, N, g))
    if case["nq"]:  # a few queries an image, at points of the grid
        B, nq = case["B"], case["nq"]
        st.update(q=randn(B * nq, H, dh), kv=randn(R, 2, Hk, dh), Nq=nq,
                  q_off=torch.arange(0, (B + 1) * nq, nq, dtype=torch.int32, device=DEV),
                  q_pos=torch.randint(0, N, (B * nq,), generator=g, device=DEV, dtype=torch.int32))
        st["q"], (st["k"], st["v"]) = st["q"], st["kv"].unbind(1)
    else:  # the rows of one projection, as a block's product leaves them: all of q, k, v in a row
        st["qkv"] = randn(R, (H + 2 * Hk), dh)
        st.update(q=st["qkv"][:, :H], k=st["qkv"][:, H:H + Hk], v=st["qkv"][:, H + Hk:], Nq=st["Nk"], q_off=st["k_off"],
                  q_pos=st["k_pos"])
    st["lut"], st["nb"] = None, 0
    if case["span"]:
        lut, nb = _lut(case["span"], case["side"])
        st.update(lut=lut.to(DEV), nb=nb, table=randn(nb * nb, H, s=0.5))
    st["k_bias"] = None
    if case["kbias"]:  # log of the tokens a key stands for (one to four), -inf where it was dropped
        size = torch.randint(0, 20, (R,), generator=g, device=DEV)
        size = torch.where(size > 16, size - 15, (size > 0).long())
        st["k_bias"] = size.float().log()
    if case["kind"] == "attend_step":
        st["dout"] = randn(st["q"].shape[0], H, dh)
    return st


def _prepare_norm(case, seed):
    g, dt, D = _generator(seed), _DT[case["dtype"]], case["D"]

    def randn(*shape, s=1.0, m=0.0):
        return (torch.randn(shape, generator=g, device=DEV) * s + m).to(dt)

    n = _lengths(case, case["N"], seed)
    R = int(n.sum())
    st = dict(case=case, off=_offsets(n), x=randn(R, D, s=2.0, m=0.1), f=randn(R, D, s=1.5, m=-0.2),
              w=randn(D, s=0.2, m=1.0), b=randn(D, s=0.1) if case["norm"] == "layer" else None, post_w=None, post_b=None,
              scale=randn(D, s=0.05, m=0.3) if case["scale"] else None, gate=None)
    if case["post"]:
        st["post_w"] = randn(D, s=0.2, m=1.0)
        st["post_b"] = randn(D, s=0.1) if case["norm"] == "layer" else None
    if case["gate"] != "none":
        st["gate"] = randn(case["B"] if case["gate"] == "image" else R, D, s=0.3, m=0.8)
    if case["kind"] == "norm_step":
        st.update(dy=randn(R, D), dh=randn(R, D))
    return st


def prepare(case, seed):
    return _prepare_norm(case, seed) if case["kind"].startswith("norm") else _prepare_attend(case, seed)


# ---- the plain form ----------------------------------------------------------------------


def _padded(off, N, rows):
    """Row numbers [B, N] of the images' slots (slots past an image's end: row 0) and which exist."""
    i = torch.arange(N, device=DEV)
    valid = i[None, :] < (off[1:] - off[:-1])[:, None]
    return torch.where(valid, off[:-1, None].long() + i[None, :], 0).clamp_(max=rows - 1), valid


def _plain_attend(st):
    case = st["case"]
    H, Hk, dh, B = case["H"], case["Hk"], case["dh"], case["B"]
    Nq, Nk = st["Nq"], st["Nk"]
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    qi, qv = _padded(st["q_off"], Nq, q.shape[0])
    ki, kv = _padded(st["k_off"], Nk, k.shape[0])
    kb = None if st["k_bias"] is None else st["k_bias"][ki]
    if kb is not None:
        kv = kv & (kb > -_INF)
    q = q[qi].permute(0, 2, 1, 3).reshape(B, Hk, H // Hk * Nq, dh)  # the queries that share a key head in a row
    k = k[ki].masked_fill(~kv[:, :, None, None], 0).permute(0, 2, 1, 3).contiguous()  # [B, Hk, Nk, dh]
    v = v[ki].masked_fill(~kv[:, :, None, None], 0).permute(0, 2, 1, 3).contiguous()
    scale = dh ** -0.5
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(B, H, Nq, Nk) * scale
    bucket = None
    if st["lut"] is not None:
        gw, span = case["gw"], case["span"]
        qp, kp = st["q_pos"][qi].long(), st["k_pos"][ki].long()
        dr = (qp[:, :, None] // gw - kp[:, None, :] // gw).clamp(-span, span) + span
        dc = (qp[:, :, None] % gw - kp[:, None, :] % gw).clamp(-span, span) + span
        bucket = st["lut"][dr].long() * st["nb"] + st["lut"][dc].long()  # [B, Nq, Nk]
        s += st["table"].float().t().contiguous()[:, bucket].transpose(0, 1)
    if kb is not None:
        s += torch.where(kv, kb, 0.0)[:, None, None, :]
    s.masked_fill_(~kv[:, None, None, :], -_INF)
    m = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -_INF, m, 0.0))
    total = p.sum(dim=-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    del s
    o = torch.matmul(p.view(B, Hk, H // Hk * Nq, Nk), v)  # [B, Hk, H/Hk*Nq, dh]

    def packed(t, heads, valid):  # [B, heads, n, dh] -> the existing rows
        return t.reshape(B, heads, -1, dh).permute(0, 2, 1, 3)[valid].to(_DT[case["dtype"]])

    out = packed(o, H, qv)
    if case["kind"] == "attend":
        return {"out": out}
    # the gradients, by the formula: dS = P (dP - sum_j P dP)
    do = st["dout"].float()[qi].masked_fill(~qv[:, :, None, None], 0).permute(0, 2, 1, 3).reshape(B, Hk, H // Hk * Nq, dh)
    p = p.view(B, Hk, H // Hk * Nq, Nk)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = p * (dp - (p * dp).sum(dim=-1, keepdim=True))
    del dp, p
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q) * scale
    _, kreal = _padded(st["k_off"], Nk, st["k"].shape[0])
    dqkv = torch.cat([packed(dq, H, qv), packed(dk, Hk, kreal), packed(dv, Hk, kreal)], dim=1)
    res = {"out": out, "dqkv": dqkv}
    if bucket is not None:
        ds = ds.view(B, H, Nq, Nk).permute(0, 2, 3, 1).reshape(-1, H)
        dt = torch.zeros((st["nb"] ** 2, H), device=DEV).index_add_(0, bucket.reshape(-1), ds)
        res["dtable"] = dt.to(_DT[case["dtype"]])
    return res


def _plain_unit(u, kind, eps):
    """Rows to unit variance (layer) or unit mean square (rms), and the reciprocal they took."""
    if kind == "layer":
        u = u - u.mean(dim=1, keepdim=True)
    r = torch.rsqrt((u * u).mean(dim=1, keepdim=True) + eps)
    return u * r, r


def _plain_unit_grad(d, unit, r, kind):
    g = d - unit * (d * unit).mean(dim=1, keepdim=True)
    if kind == "layer":
        g = g - d.mean(dim=1, keepdim=True)
    return g * r


EPS = 1e-6


def _plain_norm(st):
    case, kind, dt = st["case"], st["case"]["norm"], _DT[st["case"]["dtype"]]
    f32 = {k: (v.float() if torch.is_tensor(v) and v.is_floating_point() else v) for k, v in st.items()}
    u, pu, pr = f32["f"], None, None
    if case["post"]:
        pu, pr = _plain_unit(u, kind, EPS)
        u = pu * f32["post_w"] + (f32["post_b"] if f32["post_b"] is not None else 0.0)
    image = None
    factor = f32["scale"] if case["scale"] else torch.ones((), device=DEV)
    if case["gate"] == "image":
        image = torch.repeat_interleave(torch.arange(case["B"], device=DEV), (st["off"][1:] - st["off"][:-1]).long(),
                                        output_size=st["x"].shape[0])
    gate = None if case["gate"] == "none" else (f32["gate"][image] if image is not None else f32["gate"])
    both = factor if gate is None else factor * gate
    y = f32["x"] + both * u
    unit, r = _plain_unit(y, kind, EPS)
    h = unit * f32["w"] + (f32["b"] if f32["b"] is not None else 0.0)
    res = {"y": y.to(dt), "h": h.to(dt)}
    if case["kind"] == "norm":
        return res
    dh = f32["dh"]
    dx = f32["dy"] + _plain_unit_grad(dh * f32["w"], unit, r, kind)
    du = dx * both
    res["dx"], res["dw"] = dx, (dh * unit).sum(dim=0)
    if f32["b"] is not None:
        res["db"] = dh.sum(dim=0)
    if case["scale"]:
        res["dscale"] = (dx * u * (gate if gate is not None else 1.0)).sum(dim=0)
    if gate is not None:
        dg = dx * u * factor
        res["dgate"] = dg if image is None else torch.zeros_like(f32["gate"]).index_add_(0, image, dg)
    if case["post"]:
        res["df"], res["dpost_w"] = _plain_unit_grad(du * f32["post_w"], pu, pr, kind), (du * pu).sum(dim=0)
        if f32["post_b"] is not None:
            res["dpost_b"] = du.sum(dim=0)
    else:
        res["df"] = du
    return {k: v.to(dt) for k, v in res.items()}


# ---- the library's calls -----------------------------------------------------------------


def _own_attend(st):
    import paper_2604_05718_amd as mpm

    case = st["case"]
    where = dict(q_off=st["q_off"], k_off=st["k_off"], Nq=st["Nq"], Nk=st["Nk"], k_bias=st["k_bias"])
    if st["lut"] is not None:
        where.update(bias=mpm.bias_expand(st["table"], st["lut"]), q_pos=st["q_pos"], k_pos=st["k_pos"],
                     grid=(case["gh"], case["gw"]))
    if case["kind"] == "attend":
        return {"out": mpm.attention(st["q"], st["k"], st["v"], **where)}
    out, lse = mpm.attention(st["q"], st["k"], st["v"], with_lse=True, **where)
    dqkv = torch.empty_like(st["qkv"])
    H, Hk = case["H"], case["Hk"]
    grads = mpm.attention_backward(st["dout"], st["q"], st["k"], st["v"], out, lse, dq=dqkv[:, :H], dk=dqkv[:, H:H + Hk],
                                   dv=dqkv[:, H + Hk:], **where)
    res = {"out": out, "dqkv": dqkv}
    if st["lut"] is not None:
        res["dtable"] = mpm.bias_gradient(grads.dbias, st["lut"], st["nb"], dtype=st["table"].dtype)
    return res


def _own_norm(st):
    import paper_2604_05718_amd as mpm

    case = st["case"]
    kw = dict(weight=st["w"], bias=st["b"], post_weight=st["post_w"], post_bias=st["post_b"], scale=st["scale"],
              gate=st["gate"], off=st["off"] if case["gate"] == "image" else None, norm=case["norm"], eps=EPS)
    if case["kind"] == "norm":
        y, h = mpm.residual_norm(st["x"], st["f"], **kw)
        return {"y": y, "h": h}
    y, h, stats = mpm.residual_norm(st["x"], st["f"], with_stats=True, **kw)
    g = mpm.residual_norm_backward(st["dy"], st["dh"], y, st["f"], stats, **kw)
    res = {"y": y, "h": h, "dx": g.dx, "dw": g.dweight, "db": g.dbias, "dscale": g.dscale, "dgate": g.dgate, "df": g.df,
           "dpost_w": g.dpost_weight, "dpost_b": g.dpost_bias}
    return {k: v for k, v in res.items() if v is not None}


def run(state):
    norm = state["case"]["kind"].startswith("norm")
    if own:
        return _own_norm(state) if norm else _own_attend(state)
    return _plain_norm(state) if norm else _plain_attend(state)


# ---- what a pass cannot do without -------------------------------------------------------


def work(case):
    s, B = _BYTES[case["dtype"]], case["B"]
    if case["kind"].startswith("norm"):
        n = _lengths(case, case["N"], 0)
        R, D = int(n.sum()), case["D"]
        gate = {"none": 0, "image": B * D, "row": R * D}[case["gate"]]
        if case["kind"] == "norm":  # x, f in; y, h out
            return {"bytes": float(s * (4 * R * D + gate)), "flops": 14.0 * R * D}
        return {"bytes": float(s * (8 * R * D + 2 * gate)), "flops": 40.0 * R * D}
    n = _lengths(case, case["gh"] * case["gw"], 0).double()
    nq = torch.full_like(n, case["nq"]) if case["nq"] else n
    H, Hk, dh = case["H"], case["Hk"], case["dh"]
    q, kv = float(nq.sum()) * H * dh * s, float(n.sum()) * Hk * dh * s * 2
    pairs = float((nq * n).sum()) * H
    table = 0
    if case["span"]:
        table = (2 * case["side"] + 1 if case["side"] else 2 * case["span"] + 1) ** 2 * H * s
    ints = 4.0 * float(nq.sum() + n.sum()) * (1 if case["span"] else 0) + (4.0 * float(n.sum()) if case["kbias"] else 0)
    if case["kind"] == "attend":  # two products
        return {"bytes": 2 * q + kv + table + ints, "flops": 4.0 * pairs * dh}
    # out, and the gradients of all: seven products
    return {"bytes": 4 * q + 2 * kv + 2 * table + ints, "flops": 14.0 * pairs * dh}


# ---- the definition in 64 bits -----------------------------------------------------------


def _exact_attend(case, seed):
    st = _prepare_attend(case, seed)
    H, Hk, dh, gw, span = case["H"], case["Hk"], case["dh"], case["gw"], case["span"]
    qo, ko = st["q_off"].tolist(), st["k_off"].tolist()
    step = case["kind"] == "attend_step"
    out = torch.zeros((st["q"].shape[0], H, dh), dtype=torch.float64, device=DEV)
    if step:
        dq, dk, dv = (torch.zeros(st[x].shape, dtype=torch.float64, device=DEV) for x in "qkv")
        dt = torch.zeros((st["nb"] ** 2, H), dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        rq, rk = slice(qo[b], qo[b + 1]), torch.arange(ko[b], ko[b + 1], device=DEV)
        kb = None
        if st["k_bias"] is not None:  # dropped keys take no part
            rk = rk[st["k_bias"][rk] > -_INF]
            kb = st["k_bias"][rk].double()
        if rk.numel() == 0:
            continue
        cell = None
        if span:
            qp, kp = st["q_pos"][rq].long(), st["k_pos"][rk].long()
            row = torch.div(qp, gw, rounding_mode="floor")[:, None] - torch.div(kp, gw, rounding_mode="floor")[None, :]
            col = torch.remainder(qp, gw)[:, None] - torch.remainder(kp, gw)[None, :]
            axis = st["lut"].long()
            cell = axis[torch.clamp(row, -span, span) + span] * st["nb"] + axis[torch.clamp(col, -span, span) + span]
        for h in range(H):
            j = h // (H // Hk)
            Q, K, V = st["q"][rq, h].double(), st["k"][rk, j].double(), st["v"][rk, j].double()
            S = (Q @ K.T.contiguous()) / math.sqrt(dh)
            if cell is not None:
                S = S + st["table"][:, h].double()[cell]
            if kb is not None:
                S = S + kb
            P = torch.softmax(S, dim=1)
            O = P @ V
            out[rq, h] = O
            if step:
                G = st["dout"][rq, h].double()
                dS = P * (G @ V.T.contiguous() - (G * O).sum(dim=1, keepdim=True))
                dq[rq, h] = dS @ K / math.sqrt(dh)
                dk[rk, j] += dS.T.contiguous() @ Q / math.sqrt(dh)
                dv[rk, j] += P.T.contiguous() @ G
                if cell is not None:
                    dt[:, h] += torch.bincount(cell.reshape(-1), weights=dS.reshape(-1), minlength=st["nb"] ** 2)
    if not step:
        return {"out": out}
    res = {"out": out, "dqkv": torch.cat([dq, dk, dv], dim=1)}
    if span:
        res["dtable"] = dt
    return res


def _exact_norm(case, seed):
    st = _prepare_norm(case, seed)
    leaf = {k: st[k].double().requires_grad_() for k in ("x", "f", "w", "b", "post_w", "post_b", "scale", "gate")
            if st[k] is not None}

    def normed(t, w, b):
        if case["norm"] == "layer":
            var, mean = torch.var_mean(t, dim=1, correction=0, keepdim=True)
            t = (t - mean) / torch.sqrt(var + EPS)
        else:
            t = t / torch.sqrt(t.square().mean(dim=1, keepdim=True) + EPS)
        t = t * w
        return t if b is None else t + b

    u = normed(leaf["f"], leaf["post_w"], leaf.get("post_b")) if case["post"] else leaf["f"]
    if case["scale"]:
        u = u * leaf["scale"]
    if case["gate"] == "image":
        n = (st["off"][1:] - st["off"][:-1]).tolist()
        u = torch.cat([part * leaf["gate"][i] for i, part in enumerate(u.split(n))])
    elif case["gate"] == "row":
        u = u * leaf["gate"]
    y = leaf["x"] + u
    h = normed(y, leaf["w"], leaf.get("b"))
    res = {"y": y.detach(), "h": h.detach()}
    if case["kind"] == "norm_step":
        names = {"x": "dx", "f": "df", "w": "dw", "b": "db", "post_w": "dpost_w", "post_b": "dpost_b", "scale": "dscale",
                 "gate": "dgate"}
        total = (y * st["dy"].double()).sum() + (h * st["dh"].double()).sum()
        got = torch.autograd.grad(total, list(leaf.values()))
        res.update({names[k]: v for k, v in zip(leaf, got)})
    return res


def exact(case, seed):
    return _exact_norm(case, seed) if case["kind"].startswith("norm") else _exact_attend(case, seed)
