"""The operators of an encoder with rotated positions, served in 8 bits, and of its decoder head, as
timed cases.

Rotary positions: queries and keys turned by the grid coordinates (time, row, column) that their tokens
carry through the merges, by given or learned frequencies, forward and with the gradients. The product
of a block in 8-bit integers, tokens quantised on the way in, with a scale for each token and channel.
Group norm with an activation over the rebuilt grids, channels last, forward and with its gradients.

`run` computes them in plain torch in 32 bits (angles and rounding borders in 64), rounded once at the
end, or, where `own` is set, with the library's calls. Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
EPS = 1e-5


def listed():
    return [
        # Queries and keys of one 224x224 image (14x14 patches) at ViT-Ti width after a merge: one block of
        # interactive use, nothing but latency.
        dict(name="rotary_ti_224", kind="rotary", dtype="bf16", B=1, gt=0, gh=14, gw=14, keep=0.6, H=3, Hk=3, dh=64, pairs=32,
             layout="halves", freq="fixed"),
        # ViT-B/16 at 512x512, the benchmark's batch after its merges: the query and key heads of one
        # projection's rows, in place of the position table.
        dict(name="rotary_b_512", kind="rotary", dtype="bf16", B=64, gt=0, gh=32, gw=32, keep=0.7, H=12, Hk=12, dh=64, pairs=32,
             layout="halves", freq="fixed"),
        # A training step on clips of 8 frames of 32x32 patches, frequencies of all three axes learned by
        # every head.
        dict(name="rotary_step_clip", kind="rotary_step", dtype="bf16", B=8, gt=8, gh=32, gw=32, keep=0.7, H=16, Hk=16, dh=64,
             pairs=32, layout="pairs", freq="heads"),
        # float32, shared key heads, odd grid, a head of which a part is turned, learned frequencies.
        dict(name="rotary_step_odd_f32", kind="rotary_step", dtype="f32", B=5, gt=0, gh=27, gw=31, keep=0.7, H=6, Hk=2, dh=40,
             pairs=13, layout="halves", freq="shared"),
        # One token (a class or a point token) through the widest layer of ViT-L.
        dict(name="linear8_token", kind="linear8", dtype="bf16", M=1, K=1024, N=4096, bias=True, act="gelu"),
        # The query, key and value projection of ViT-B/16 at 512x512 on the merged batch.
        dict(name="linear8_b_512", kind="linear8", dtype="bf16", M=45888, K=768, N=2304, bias=True, act="none"),
        # The first product of ViT-L's MLP at 1024x1024, merged, with its activation.
        dict(name="linear8_l_1024", kind="linear8", dtype="bf16", M=45920, K=1024, N=4096, bias=True, act="gelu"),
        # float32 tokens of odd numbers into a head of 150 classes.
        dict(name="linear8_odd_f32", kind="linear8", dtype="f32", M=4103, K=836, N=150, bias=False, act="none"),
        # One rebuilt 32x32 grid at ViT-Ti width: latency.
        dict(name="group_ti_512", kind="group", dtype="bf16", B=1, N=1024, keep=1.0, C=192, G=32, act="silu", affine=True),
        # ViT-B/16 at 512x512: the benchmark's rebuilt grids.
        dict(name="group_b_512", kind="group", dtype="bf16", B=64, N=1024, keep=1.0, C=768, G=32, act="silu", affine=True),
        # A training step at ViT-L/16 1024x1024.
        dict(name="group_step_l_1024", kind="group_step", dtype="bf16", B=16, N=4096, keep=1.0, C=1024, G=32, act="silu",
             affine=True),
        # float32, packed images of odd lengths, groups that are no whole number of vectors.
        dict(name="group_step_odd_f32", kind="group_step", dtype="f32", B=7, N=837, keep=0.8, C=836, G=11, act="relu",
             affine=True),
    ]


def _cost(case):
    """A case's weight (products count by the rate of 8-bit ones)."""
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (2e15 if case["kind"] == "linear8" else 1e14)


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rotary", "rotary_step", "linear8", "linear8", "group", "group_step"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        keep = rng.choice([1.0, round(rng.uniform(0.4, 0.9), 2)])
        if kind.startswith("rotary"):
            gh = log_int(5, 64)
            gw = max(4, min(64, gh + rng.randint(-5, 5)))
            H = rng.choice([3, 4, 6, 8, 12, 16])
            shared = rng.choice([1, 1, 1, 2, 3])
            dh = rng.choice([64, 64, 64, 32, 40, 80, 128])
            case = dict(kind=kind, dtype=dtype, B=log_int(1, 64), gt=0 if rng.random() < 0.6 else log_int(2, 16), gh=gh, gw=gw,
                        keep=keep, H=H, Hk=H // shared if H % shared == 0 else H, dh=dh,
                        pairs=dh // 2 if rng.random() < 0.6 else rng.randint(dh // 8, dh // 2),
                        layout=rng.choice(["halves", "halves", "pairs"]),
                        freq=rng.choice(["fixed", "fixed", "shared", "heads"]))
        elif kind == "linear8":
            K = rng.choice([192, 384, 768, 1024]) if rng.random() < 0.4 else 8 * log_int(6, 512)
            N = rng.choice([192, 384, 576, 768, 1024, 2304, 4096]) if rng.random() < 0.4 else log_int(19, 4096)
            case = dict(kind=kind, dtype=dtype, M=log_int(1, 46000), K=K, N=N, bias=rng.random() < 0.7,
                        act=rng.choice(["none", "none", "gelu"]))
        else:
            G = rng.choice([1, 4, 8, 16, 32, 32, 32])
            C = G * rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48])
            C += -C % 8 if G == 1 else 0
            if C % 8 or not 32 <= C <= 1024:
                continue
            case = dict(kind=kind, dtype=dtype, B=log_int(1, 64), N=log_int(49, 9216), keep=keep, C=C, G=G,
                        act=rng.choice(["none", "relu", "silu", "silu"]), affine=rng.random() < 0.9)
        if _cost(case) <= most:
            return case


def _grid(case):
    """(rows, columns), or (frames, rows, columns) of a clip."""
    return (case["gt"], case["gh"], case["gw"]) if case["gt"] else (case["gh"], case["gw"])


# ---- inputs ------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 31)
    return g


def _lengths(case, N, seed):
    """Tokens an image, as merges leave them: the same spread around the kept share for every
    seed, dealt to the images in another order."""
    B = case["B"]
    if case["keep"] >= 1.0:
        return torch.full((B,), N, dtype=torch.long)
    g = torch.Generator().manual_seed(int(seed) * 104729 + 13)
    lo, hi = max(0.02, case["keep"] - 0.15), min(1.0, case["keep"] + 0.15)
    n = (torch.linspace(lo, hi, B) * N if B > 1 else torch.tensor([case["keep"] * N])).long().clamp(1, N)
    return n[torch.randperm(B, generator=g)]


def _offsets(n):
    off = torch.zeros((n.numel() + 1,), dtype=torch.int32)
    off[1:] = torch.cumsum(n, 0)
    return off.to(DEV)


def _positions(n, N, g):
    """Sorted grid cells of the tokens each image kept, packed."""
    order = torch.rand((n.numel(), N), generator=g, device=DEV).argsort(dim=1)
    kept = torch.arange(N, device=DEV)[None, :] < n.to(DEV)[:, None]
    cells = torch.zeros((n.numel(), N), dtype=torch.bool, device=DEV).scatter_(1, order, kept)
    return cells.nonzero()[:, 1].to(torch.int32)


def _prepare_rotary(case, seed):
    g, dt, grid = _generator(seed), _DT[case["dtype"]], _grid(case)
    N, heads, P, A = math.prod(grid), case["H"] + case["Hk"], case["pairs"], len(grid)
    n = _lengths(case, N, seed)
    R = int(n.sum())
    # the rows of one projection, as a block's product leaves them: all of q, k, v in a row
    qkv = torch.randn((R, heads + case["Hk"], case["dh"]), generator=g, device=DEV).to(dt)
    if case["freq"] == "fixed":  # the pairs dealt to the axes in turns, a geometric range of wavelengths each
        p = torch.arange(P, device=DEV)
        each = 100.0 ** (-(p // A).float() / max(1, (P + A - 1) // A))
        freq = torch.where(p % A == torch.arange(A, device=DEV)[:, None], each, 0.0)
    else:  # learned: every axis turns every pair
        shape = (heads, A, P) if case["freq"] == "heads" else (A, P)
        freq = torch.randn(shape, generator=g, device=DEV) * 0.3
    st = dict(case=case, qkv=qkv, x=qkv[:, :heads], freq=freq.contiguous(), pos=_positions(n, N, g))
    if case["kind"] == "rotary_step":
        st["dout"] = torch.randn((R, heads, case["dh"]), generator=g, device=DEV).to(dt)
    return st


def _steps8(t):
    """Rows of 8-bit steps and their scales: max |t| / 127 rounded to float32 (by way of 64 bits: torch divides by a
    number by way of its reciprocal), the quotient rounded to even."""
    scale = (t.float().abs().amax(dim=1, keepdim=True).double() / 127.0).float().clamp_min(2.0 ** -126)
    return torch.round(t.double() / scale.double()).clamp_(-127, 127), scale


def _prepare_linear8(case, seed):
    g, dt, K, N = _generator(seed), _DT[case["dtype"]], case["K"], case["N"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    # rows of a norm: channels of unequal size, a few of them large
    x = (randn(case["M"], K) * torch.exp(randn(K) * 0.5)).to(dt)
    q, scale = _steps8(randn(N, K) * K ** -0.5)
    w = torch.zeros((N, (K + 15) // 16 * 16), dtype=torch.int8, device=DEV)  # rows of whole 16 bytes, as the library keeps them
    w[:, :K] = q.to(torch.int8)
    return dict(case=case, x=x, w=w, w_scale=scale[:, 0].contiguous(), bias=(randn(N) * 0.1).to(dt) if case["bias"] else None)


def _prepare_group(case, seed):
    g, dt, C, B = _generator(seed), _DT[case["dtype"]], case["C"], case["B"]

    def randn(*shape, s=1.0, m=0.0):
        return (torch.randn(shape, generator=g, device=DEV) * s + m).to(dt)

    n = _lengths(case, case["N"], seed)
    R = int(n.sum())
    x = (torch.randn((R, C), generator=g, device=DEV) * 1.5 + torch.randn((C,), generator=g, device=DEV)).to(dt)
    st = dict(case=case, x=x, off=None, n=n.to(DEV), w=randn(C, s=0.2, m=1.0) if case["affine"] else None,
              b=randn(C, s=0.1) if case["affine"] else None)
    if case["keep"] >= 1.0:
        st["x"] = x.view(B, case["N"], C)
    else:
        st["off"] = _offsets(n)
    if case["kind"] == "group_step":
        st["dy"] = randn(R, C).view(st["x"].shape)
    return st


def _family(case):
    return case["kind"].split("_")[0]


def prepare(case, seed):
    return {"rotary": _prepare_rotary, "linear8": _prepare_linear8, "group": _prepare_group}[_family(case)](case, seed)


# ---- the plain form ----------------------------------------------------------------------


def _coordinates(pos, grid):
    """Grid coordinates [R, A] of raster indices."""
    strides = [math.prod(grid[a + 1:]) for a in range(len(grid))]
    return torch.stack([pos.long() // s % n for s, n in zip(strides, grid)], dim=1)


def _parts(t, P, layout):
    """The two channels of every pair, and the channels that are left."""
    if layout == "halves":
        return t[..., :P], t[..., P:2 * P], t[..., 2 * P:]
    return t[..., 0:2 * P:2], t[..., 1:2 * P:2], t[..., 2 * P:]


def _whole(a, b, rest, layout):
    turned = torch.cat([a, b], dim=-1) if layout == "halves" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([turned, rest], dim=-1)


def _plain_rotary(st):
    case, dt = st["case"], _DT[st["case"]["dtype"]]
    P, layout = case["pairs"], case["layout"]
    c = _coordinates(st["pos"], _grid(case)).double()
    f = st["freq"].double().reshape(-1, len(_grid(case)), P)
    angle = torch.matmul(c, f.permute(1, 0, 2).reshape(len(_grid(case)), -1)).view(c.shape[0], -1, P)  # [R, 1 or heads, P]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    x1, x2, rest = _parts(st["x"].float(), P, layout)
    res = {"out": _whole(x1 * cos - x2 * sin, x1 * sin + x2 * cos, rest, layout).to(dt)}
    if case["kind"] == "rotary":
        return res
    d1, d2, rest = _parts(st["dout"].float(), P, layout)
    g1, g2 = d1 * cos + d2 * sin, d2 * cos - d1 * sin
    res["dx"] = _whole(g1, g2, rest, layout).to(dt)
    if case["freq"] != "fixed":
        turn = (x1 * g2 - x2 * g1).double()
        if f.shape[0] == 1:
            turn = turn.sum(dim=1, keepdim=True)
        d = torch.matmul(c.t().contiguous(), turn.reshape(c.shape[0], -1))  # [A, (1 or heads) P]
        res["dfreq"] = d.view(len(_grid(case)), -1, P).permute(1, 0, 2).reshape(st["freq"].shape).float()
    return res


def _gelu(t):
    return 0.5 * t * (1.0 + torch.erf(t * 0.5 ** 0.5))


def _plain_linear8(st):
    case = st["case"]
    q, scale = _steps8(st["x"])
    y = torch.matmul(q.float(), st["w"][:, :case["K"]].float().t().contiguous()) * scale * st["w_scale"]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    return {"out": (_gelu(y) if case["act"] == "gelu" else y).to(_DT[case["dtype"]])}


def _padded(n, N):
    """Row numbers [B, N] of the images' slots (slots past an image's end: row 0) and which exist."""
    i = torch.arange(N, device=DEV)
    valid = i[None, :] < n[:, None]
    return torch.where(valid, (torch.cumsum(n, 0) - n)[:, None] + i[None, :], 0), valid


def _plain_group(st):
    case, dt, C, G = st["case"], _DT[st["case"]["dtype"]], st["case"]["C"], st["case"]["G"]
    shape, rows, valid = st["x"].shape, None, None
    if st["off"] is not None:
        rows, valid = _padded(st["n"], int(case["N"]))

    def images(t):  # [B, N, G, C / G]
        t = t.float()
        if rows is not None:
            t = t[rows].masked_fill(~valid[:, :, None], 0.0)
        return t.reshape(case["B"], -1, G, C // G)

    def packed(t):
        t = t.reshape(case["B"], -1, C)
        return (t if valid is None else t[valid]).reshape(shape).to(dt)

    def mean(t):
        return t.sum(dim=(1, 3), keepdim=True) / count

    real = None if valid is None else valid[:, :, None, None]
    count = (st["n"].float() * (C // G)).view(-1, 1, 1, 1)
    x = images(st["x"])
    t = x - mean(x)
    if real is not None:
        t = torch.where(real, t, 0.0)
    rstd = torch.rsqrt(mean(t * t) + EPS)
    t = t * rstd
    w = st["w"].float().view(G, -1) if case["affine"] else torch.ones((), device=DEV)
    z = t * w + (st["b"].float().view(G, -1) if case["affine"] else 0.0)
    s = torch.sigmoid(z)
    y = {"none": z, "relu": z.clamp_min(0.0), "silu": z * s}[case["act"]]
    res = {"y": packed(y)}
    if case["kind"] == "group":
        return res
    slope = {"none": torch.ones_like(z), "relu": (z > 0).float(), "silu": s * (1.0 + z * (1.0 - s))}[case["act"]]
    gz = images(st["dy"]) * slope
    gt = gz * w
    res["dx"] = packed(rstd * (gt - mean(gt) - t * mean(gt * t)))
    if case["affine"]:
        res["dw"], res["db"] = (v.double().sum(dim=(0, 1)).reshape(C).to(dt) for v in (gz * t, gz))
    return res


# ---- the library's calls -----------------------------------------------------------------


def _own_rotary(st):
    import paper_2604_05718_amd as mpm

    case = st["case"]
    where = dict(pos=st["pos"], grid=_grid(case), layout=case["layout"])
    res = {"out": mpm.rotary(st["x"], st["freq"], **where)}
    if case["kind"] == "rotary_step":
        learned = case["freq"] != "fixed"
        g = mpm.rotary_backward(st["dout"], st["x"], st["freq"], with_dfreq=learned, **where)
        res["dx"] = g.dx
        if learned:
            res["dfreq"] = g.dfreq
    return res


def _own_linear8(st):
    import paper_2604_05718_amd as mpm

    return {"out": mpm.linear_int8(st["x"], st["w"], st["w_scale"], bias=st["bias"], activation=st["case"]["act"])}


def _own_group(st):
    import paper_2604_05718_amd as mpm

    case = st["case"]
    kw = dict(weight=st["w"], bias=st["b"], off=st["off"], activation=case["act"], eps=EPS)
    if case["kind"] == "group":
        return {"y": mpm.group_norm(st["x"], case["G"], **kw)}
    y, stats = mpm.group_norm(st["x"], case["G"], with_stats=True, **kw)
    g = mpm.group_norm_backward(st["dy"], st["x"], stats, case["G"], **kw)
    res = {"y": y, "dx": g.dx}
    if case["affine"]:
        res.update(dw=g.dweight, db=g.dbias)
    return res


def run(state):
    family = _family(state["case"])
    if own:
        return {"rotary": _own_rotary, "linear8": _own_linear8, "group": _own_group}[family](state)
    return {"rotary": _plain_rotary, "linear8": _plain_linear8, "group": _plain_group}[family](state)


# ---- what a pass cannot do without -------------------------------------------------------


def work(case):
    s = _BYTES[case["dtype"]]
    if _family(case) == "linear8":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": float(s * (M * K + M * N) + N * K + 4 * N + (s * N if case["bias"] else 0)),
                "flops": 2.0 * M * K * N}
    if _family(case) == "rotary":
        R = int(_lengths(case, math.prod(_grid(case)), 0).sum())
        values = float(R * (case["H"] + case["Hk"]) * case["dh"])
        if case["kind"] == "rotary":  # x in, out out
            return {"bytes": 2 * s * values + 4 * R, "flops": 3 * values}
        return {"bytes": 4 * s * values + 4 * R, "flops": 9 * values}  # and dout in, dx out
    values = float(int(_lengths(case, case["N"], 0).sum()) * case["C"])
    if case["kind"] == "group":  # x in, y out
        return {"bytes": 2 * s * values, "flops": 10 * values}
    return {"bytes": 4 * s * values, "flops": 30 * values}  # and dy in, dx out


# ---- the definition in 64 bits -----------------------------------------------------------


def _exact_rotary(case, seed):
    st = _prepare_rotary(case, seed)
    P, grid = case["pairs"], _grid(case)
    cell, where = st["pos"].double(), []
    for side in reversed(grid):  # column first
        rest = torch.floor(cell / side)
        where.insert(0, cell - rest * side)
        cell = rest
    freq = st["freq"].double() if st["freq"].dim() == 3 else st["freq"].double()[None]
    angle = sum(where[a][:, None, None] * freq[None, :, a, :] for a in range(len(grid)))
    turn = torch.polar(torch.ones_like(angle), angle)
    index = torch.arange(2 * P, device=DEV)
    index = index.view(2, P) if case["layout"] == "halves" else index.view(P, 2).t()

    def numbers(t):
        t = t.double()
        return torch.complex(t[:, :, index[0]], t[:, :, index[1]])

    def rows(z, like):
        out = like.double().clone()
        out[:, :, index[0]], out[:, :, index[1]] = z.real, z.imag
        return out

    x = numbers(st["x"])
    res = {"out": rows(x * turn, st["x"])}
    if case["kind"] == "rotary_step":
        back = numbers(st["dout"]) * turn.conj()
        res["dx"] = rows(back, st["dout"])
        if case["freq"] != "fixed":
            d = (x.conj() * back).imag  # the gradient of every angle
            if freq.shape[0] == 1:
                d = d.sum(dim=1, keepdim=True)
            d = torch.stack([(where[a][:, None, None] * d).sum(dim=0) for a in range(len(grid))], dim=1)
            res["dfreq"] = d.view(st["freq"].shape)
    return res


def _exact_linear8(case, seed):
    st = _prepare_linear8(case, seed)
    x, K = st["x"].double(), case["K"]
    step = (x.abs().max(dim=1).values.float() / torch.tensor(127.0, device=DEV)).double()
    step = torch.clamp(step, min=2.0 ** -126)
    part = x / step[:, None]
    low = torch.floor(part)
    over = part - low
    up = (over > 0.5) | ((over == 0.5) & (low % 2 != 0))
    whole = torch.clamp(low + up, -127.0, 127.0)
    y = torch.mm(whole, st["w"][:, :K].double().T.contiguous())
    y = y * step[:, None] * st["w_scale"].double()[None, :]
    if case["bias"]:
        y = y + st["bias"].double()
    if case["act"] == "gelu":
        y = y * torch.special.erfc(-y / math.sqrt(2.0)) / 2.0
    return {"out": y}


def _exact_group(case, seed):
    st = _prepare_group(case, seed)
    C, G = case["C"], case["G"]
    x = st["x"].double().reshape(-1, C).requires_grad_()
    w = st["w"].double().requires_grad_() if case["affine"] else torch.ones(C, dtype=torch.float64, device=DEV)
    b = st["b"].double().requires_grad_() if case["affine"] else torch.zeros(C, dtype=torch.float64, device=DEV)
    parts = []
    for image in x.split(st["n"].tolist()):
        grouped = image.view(image.shape[0], G, C // G).transpose(0, 1).reshape(G, -1)
        var, mean = torch.var_mean(grouped, dim=1, correction=0, keepdim=True)
        unit = ((grouped - mean) / torch.sqrt(var + EPS)).view(G, image.shape[0], C // G).transpose(0, 1).reshape(-1, C)
        z = unit * w + b
        parts.append(z if case["act"] == "none" else torch.relu(z) if case["act"] == "relu" else z / (1.0 + torch.exp(-z)))
    y = torch.cat(parts)
    res = {"y": y.detach().view(st["x"].shape)}
    if case["kind"] == "group_step":
        leaves = [x, w, b] if case["affine"] else [x]
        got = torch.autograd.grad((y * st["dy"].double().view(-1, C)).sum(), leaves)
        res["dx"] = got[0].view(st["x"].shape)
        if case["affine"]:
            res.update(dw=got[1], db=got[2])
    return res


def exact(case, seed):
    return {"rotary": _exact_rotary, "linear8": _exact_linear8, "group": _exact_group}[_family(case)](case, seed)
