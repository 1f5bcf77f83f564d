"""What the 8-bit transformer operators are measured on: residual + root-mean-square norm with 8-bit codes,
the sliced linear layer on 8-bit codes, and rotary positions with several axes.

Every case is a batch of B samples of R rows (tokens); sample i runs one of T paths, path t uses the leading
widths of the full extents, and the batch is grouped by path as dsn_route does it.
"""
import math

import torch

own = False
_contexts = {}
DEV = "cuda"


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # norm: one new token of a ViT-B-wide stream; latency of one call
        dict(name="norm 1 token", op="norm", B=1, R=1, C=768, T=1, g=8, dtype="bf16", residual=True, grouped=False, raw=False),
        # norm: the pre-norm of a slimmable ViT-S block, the gather to grouped order fused
        dict(name="norm vit-s", op="norm", B=256, R=197, C=384, T=4, g=8, dtype="bf16", residual=True, grouped=True, raw=False),
        # norm: widths that are no multiple of anything, fp32 stream, no residual, small images
        dict(name="norm odd f32", op="norm", B=37, R=121, C=1000, T=3, g=1, dtype="f32", residual=False, grouped=True, raw=False),
        # norm: a long prompt at a wide stream, one path
        dict(name="norm 16k x 4096", op="norm", B=4, R=4096, C=4096, T=1, g=8, dtype="bf16", residual=True, grouped=False, raw=False),
        # linear: one new token, all weights read for one row
        dict(name="linear 1 token", op="linear", B=1, R=1, C=4096, N=4096, T=1, g=8, y="bf16", act="none", bias=False, residual=False,
             order="input"),
        # linear: a batch of single tokens on mixed paths, straight from input order
        dict(name="linear 24 tokens", op="linear", B=24, R=1, C=768, N=2304, T=4, g=8, y="bf16", act="none", bias=True, residual=False,
             order="input"),
        # linear: odd widths and rows, fp32 output with skip features, activation
        dict(name="linear odd f32", op="linear", B=9, R=61, C=1000, N=777, T=3, g=1, y="f32", act="gelu", bias=True, residual=True,
             order="input"),
        # linear: QKV of the slimmable ViT-B-wide block, eight paths, grouped rows
        dict(name="linear vit-b qkv", op="linear", B=128, R=197, C=768, N=2304, T=8, g=8, y="bf16", act="none", bias=True, residual=False,
             order="grouped"),
        # linear: a long prompt through a wide square layer
        dict(name="linear 16k x 4096", op="linear", B=4, R=4096, C=4096, N=4096, T=1, g=8, y="bf16", act="none", bias=False,
             residual=False, order="grouped"),
        # rotary: one new token, 32 plain heads, temporal axis only
        dict(name="rotary 1 token", op="rotary", B=1, R=1, H=32, D=128, T=1, qkv=False, dtype="bf16", axes=1, pairs=64, ladder="shared",
             pairing="halves", shared=False, top=100000),
        # rotary: q and k of the slimmable ViT-B-wide block, two axes of a 14 x 14 grid and a class token at the origin
        dict(name="rotary vit-b", op="rotary", B=128, R=197, H=12, D=64, T=8, qkv=True, dtype="bf16", axes=2, pairs=32, ladder="per_axis",
             pairing="halves", shared=True, top=14),
        # rotary: video tokens, three axes, fp32, neighbouring pairs, part of the head turned
        dict(name="rotary video", op="rotary", B=2, R=16383, H=16, D=80, T=1, qkv=False, dtype="f32", axes=3, pairs=36, ladder="shared",
             pairing="interleaved", shared=False, top=5000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "rotary"])
    T = rng.choice([1, 1, 2, 3, 4, 8, 14])
    R = rng.choice([1, 1, 7, 49, 196, 197, 256, _log(rng, 1, 4096)])
    if op == "norm":
        C = _log(rng, 32, 8192)
        B = max(1, min(1024, _log(rng, 1, 16384) // R, 4 * 4096 * 4096 // (R * C)))
        return dict(op=op, B=B, R=R, C=C, T=T, g=rng.choice([1, 8]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    residual=rng.random() < 0.6, grouped=rng.random() < 0.5, raw=rng.random() < 0.2)
    if op == "linear":
        C, N = _log(rng, 32, 8192), _log(rng, 32, 8192)
        B = max(1, min(1024, _log(rng, 1, 16384) // R, 4096 * 4096 * 16384 // (R * C * N)))
        return dict(op=op, B=B, R=R, C=C, N=N, T=T, g=rng.choice([1, 8]), y=rng.choice(["bf16", "bf16", "f32"]),
                    act=rng.choice(["none", "relu", "gelu"]), bias=rng.random() < 0.5, residual=rng.random() < 0.3,
                    order=rng.choice(["input", "grouped"]))
    D = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
    H = rng.randint(1, 32)
    qkv = rng.random() < 0.5
    axes = rng.choice([1, 2, 3])
    pairs = rng.choice([D // 2, D // 2, rng.randint(axes, D // 2)])
    B = max(1, min(1024, _log(rng, 1, 32768) // R, 32768 * 16 * 80 // (R * H * D * (3 if qkv else 1))))
    return dict(op=op, B=B, R=R, H=H, D=D, T=T, qkv=qkv, dtype=rng.choice(["bf16", "bf16", "f32"]), axes=axes, pairs=pairs,
                ladder=rng.choice(["shared", "per_axis"]), pairing=rng.choice(["halves", "interleaved"]), shared=rng.random() < 0.5,
                top=_log(rng, 10, 1000000))


def _widths(C, T, g):
    """Path t of T uses the leading half .. whole of C, in granules of g."""
    return [min(C, max(1, (C * (T + t + 1) // (2 * T)) // g * g)) if t + 1 < T else C for t in range(T)]


def _counts(B, T):
    return [len(range(t, B, T)) for t in range(T)]


def _sections(case):
    """Pairs of each axis: as even as they go, the last axis takes what is left."""
    a, p = case["axes"], case["pairs"]
    return [p // a] * (a - 1) + [p - p // a * (a - 1)]


def work(case):
    B, R, T = case["B"], case["R"], case["T"]
    n = _counts(B, T)
    if case["op"] == "norm":
        e = 2 if case["dtype"] == "bf16" else 4
        live = sum(n[t] * R * k for t, k in enumerate(_widths(case["C"], T, case["g"])))
        per = e * (3 if case["residual"] else 1) + e + (0 if case["raw"] else 1)
        return {"bytes": live * per + (0 if case["raw"] else 4 * B * R) + 4 * case["C"], "flops": 10 * live}
    if case["op"] == "linear":
        e = 2 if case["y"] == "bf16" else 4
        ki, ko = _widths(case["C"], T, case["g"]), _widths(case["N"], T, case["g"])
        used = [t for t in range(T) if n[t]]
        rows_in = sum(n[t] * R * (ki[t] + 4) for t in used)
        rows_out = sum(n[t] * R * ko[t] * e * (2 if case["residual"] else 1) for t in used)
        w = max(ki[t] for t in used) * max(ko[t] for t in used) + 4 * max(ko[t] for t in used) * (2 if case["bias"] else 1)
        return {"bytes": rows_in + rows_out + w, "flops": sum(2 * n[t] * R * ki[t] * ko[t] for t in used)}
    e = 2 if case["dtype"] == "bf16" else 4
    v = 3 if case["qkv"] else 1
    live = sum(n[t] * R * h for t, h in enumerate(_widths(case["H"], T, 1))) * v * case["D"]
    return {"bytes": 2 * e * live + 4 * case["axes"] * (R if case["shared"] else B * R), "flops": 3 * live * (2 / 3 if case["qkv"] else 1)}


# ------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, R, T = case["B"], case["R"], case["T"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def uniform(lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(*shape, generator=g, device=DEV)

    s = {"case": case}
    s["idx"] = (torch.arange(B, device=DEV) % T)[torch.randperm(B, generator=g, device=DEV)]   # path of every sample
    order = torch.sort(s["idx"], stable=True).indices
    counts = torch.bincount(s["idx"], minlength=T)
    s["perm"] = order.to(torch.int32)
    s["inv"] = torch.argsort(order).to(torch.int32)
    s["counts"] = counts.to(torch.int32)
    s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    dt = torch.float32 if case.get("dtype", case.get("y")) == "f32" else torch.bfloat16
    if case["op"] == "norm":
        C = case["C"]
        ld = -(-C // 16) * 16                     # rows start on 16-byte boundaries in every type
        s["ld"], s["k"] = ld, _widths(C, T, case["g"])
        # a residual stream: channels of different sizes, a few large ones
        size = torch.exp(0.7 * normal(ld))
        s["x"] = (normal(B, R, ld) * size).to(dt)
        s["res"] = (normal(B, R, ld) * size).to(dt) if case["residual"] else None
        s["w"] = uniform(0.2, 1.8, C)
        s["sum"] = torch.zeros(B, R, ld, dtype=dt, device=DEV) if case["residual"] else None
        s["q"] = None if case["raw"] else torch.zeros(B, R, ld, dtype=torch.int8, device=DEV)
        s["scale"] = None if case["raw"] else torch.zeros(B, R, device=DEV)
        s["out"] = torch.zeros(B, R, ld, dtype=dt, device=DEV)
    elif case["op"] == "linear":
        C, N = case["C"], case["N"]
        ldx, ldy = -(-C // 16) * 16, -(-N // 8) * 8
        s["ldx"], s["ldy"], s["ki"], s["ko"] = ldx, ldy, _widths(C, T, case["g"]), _widths(N, T, case["g"])
        # rows as the norm writes them (their largest value at 127), weights rounded per channel
        s["x"] = (normal(B, R, ldx) * 38).round().clamp(-127, 127).to(torch.int8)
        s["sx"] = uniform(0.01, 0.05, B, R)
        s["w"] = (normal(N, ldx) * 36).round().clamp(-127, 127).to(torch.int8)
        s["sw"] = uniform(0.5, 1.5, N) * 0.02 / math.sqrt(C)
        s["bias"] = normal(N) * 0.1 if case["bias"] else None
        s["res"] = normal(B, R, ldy).to(dt) if case["residual"] else None
        s["out"] = torch.zeros(B, R, ldy, dtype=dt, device=DEV)
    else:
        H, D = case["H"], case["D"]
        ld = H * D * (3 if case["qkv"] else 1)
        s["h"] = _widths(H, T, 1)
        s["x"] = normal(B, R, ld).to(dt)
        s["pos"] = torch.randint(0, case["top"], (case["axes"], R if case["shared"] else B * R), generator=g, device=DEV).to(torch.int32)
        s["out"] = torch.zeros(B, R, ld, dtype=dt, device=DEV)
    if own:
        _keep_descriptor(s)
    return s


def _keep_descriptor(s):
    """What a user's program keeps beside its weights: the context, the routing and the layer's descriptor."""
    import paper_2109_10060_b200 as dsn
    dev = torch.cuda.current_device()
    if dev not in _contexts:
        _contexts[dev] = dsn.Context(dev)
    s["ctx"] = _contexts[dev]
    case = s["case"]
    s["r"] = dsn.make_routing(case["B"], case["T"], s["counts"], s["offsets"], s["perm"], s["inv"])
    if case["op"] == "norm":
        s["d"] = dsn.make_norm_desc(dsn.F32 if case["dtype"] == "f32" else dsn.BF16, case["R"], case["C"], s["k"], s["w"], eps=1e-6,
                                    ldx=s["ld"], ld_res=s["ld"], ld_sum=s["ld"], ldq=s["ld"], ldy=s["ld"], in_order=dsn.INPUT_ORDER,
                                    out_order=dsn.GROUPED if case["grouped"] else dsn.INPUT_ORDER)
    elif case["op"] == "linear":
        order = dsn.INPUT_ORDER if case["order"] == "input" else dsn.GROUPED
        s["d"] = dsn.make_linear_i8_desc(case["R"], case["C"], case["N"], s["ki"], s["ko"], s["w"], s["sw"], bias=s["bias"],
                                         act={"none": dsn.ACT_NONE, "relu": dsn.ACT_RELU, "gelu": dsn.ACT_GELU}[case["act"]],
                                         residual=s["res"], y_dtype=dsn.F32 if case["y"] == "f32" else dsn.BF16, ldx=s["ldx"],
                                         ldw=s["ldx"], ldy=s["ldy"], in_order=order, out_order=order)
        n = dsn.dsn_linear_i8_workspace_bytes(s["d"], case["B"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    else:
        s["d"] = dsn.make_rotary_desc(dsn.F32 if case["dtype"] == "f32" else dsn.BF16, case["R"], case["H"], case["D"], s["h"],
                                      _sections(case), vectors=3 if case["qkv"] else 1, rotated=2 if case["qkv"] else 1, base=10000.0,
                                      ladder=dsn.ROTARY_SHARED if case["ladder"] == "shared" else dsn.ROTARY_PER_AXIS,
                                      pairing=dsn.ROTARY_HALVES if case["pairing"] == "halves" else dsn.ROTARY_INTERLEAVED,
                                      shared_positions=case["shared"], order=dsn.GROUPED)


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2109_10060_b200 as dsn
        if op == "norm":
            dsn.dsn_rmsnorm_quant(s["ctx"], s["d"], s["r"], s["x"], q=s["q"], scale=s["scale"], y=s["out"], residual=s["res"], sum_out=s["sum"])
            return {k: s[k] for k in ("out", "scale", "sum") if s[k] is not None}
        if op == "linear":
            dsn.dsn_sliced_linear_i8(s["ctx"], s["d"], s["r"], s["x"], s["sx"], s["out"], s["ws"])
        else:
            dsn.dsn_rotary_axes(s["ctx"], s["d"], s["r"], s["pos"], s["x"], s["out"])
        return {"out": s["out"]}
    return {"norm": _norm, "linear": _linear, "rotary": _rotary}[op](s)


def _paths(s, grouped):
    """Path of every sample as the rows lie, [B, 1, 1]."""
    idx = s["idx"][s["perm"].long()] if grouped else s["idx"]
    return idx.view(-1, 1, 1)


def _live(s, widths, ld, grouped):
    """Which columns of which samples exist, [B, 1, ld]."""
    return torch.arange(ld, device=DEV) < torch.tensor(widths, device=DEV)[_paths(s, grouped)]


def _norm(s):
    case, C = s["case"], s["case"]["C"]
    live = _live(s, s["k"], s["ld"], False)
    w = torch.zeros(s["ld"], device=DEV)
    w[:C] = s["w"]
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    h = torch.where(live, h, 0.0)
    k = torch.tensor(s["k"], device=DEV, dtype=torch.float32)[_paths(s, False)]
    r = torch.rsqrt((h * h).sum(-1, keepdim=True) / k + 1e-6)
    hw = h * w
    out = {}
    if case["raw"]:
        y = hw * r
    else:
        top = hw.abs().amax(-1, keepdim=True)
        scale = top * r / 127
        # the code does not depend on the row's norm; written so that ties fall the same way whatever the sum of squares
        y = torch.round(hw * torch.where(top > 0, 127 / top, 0.0)) * scale
        out["scale"] = scale.squeeze(-1)
    out["out"] = y.to(s["x"].dtype)
    if case["grouped"]:
        out = {n: v[s["perm"].long()] for n, v in out.items()}
    if s["res"] is not None:
        out["sum"] = h.to(s["x"].dtype)
    return out


def _linear(s):
    case, N, grouped = s["case"], s["case"]["N"], s["case"]["order"] == "grouped"
    x = torch.where(_live(s, s["ki"], s["ldx"], grouped), s["x"].float(), 0.0)
    y = (x.view(-1, s["ldx"]) @ s["w"].float().t()).view(case["B"], case["R"], N)
    y = y * s["sx"].unsqueeze(-1) * s["sw"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["res"] is not None:
        y = y + s["res"][..., :N].float()
    if case["act"] == "relu":
        y = y.clamp_min(0)
    elif case["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    out = torch.zeros(case["B"], case["R"], s["ldy"], dtype=s["out"].dtype, device=DEV)
    out[..., :N] = torch.where(_live(s, s["ko"], N, grouped), y, 0.0)
    return {"out": out}


def _frequencies(case):
    """Axis and angle per unit of position of every pair."""
    sec = _sections(case)
    axis = torch.repeat_interleave(torch.arange(len(sec)), torch.tensor(sec))
    if case["ladder"] == "shared":
        e = torch.arange(sum(sec), dtype=torch.float64) / sum(sec)
    else:
        e = torch.cat([torch.arange(n, dtype=torch.float64) / n for n in sec])
    return axis.to(DEV), (10000.0 ** -e).to(DEV)


def _rotary(s):
    case = s["case"]
    B, R, H, D, P = case["B"], case["R"], case["H"], case["D"], case["pairs"]
    V = 3 if case["qkv"] else 1
    axis, freq = _frequencies(case)
    a = s["pos"].double()[axis].t() * freq                     # [rows, P]: angles of far positions, in 64 bits
    a = a.view(1 if case["shared"] else B, R, 1, 1, P)
    cos, sin = torch.cos(a).float(), torch.sin(a).float()
    x = s["x"].float().view(B, R, H, V, D)
    turn = x[..., : 2 if case["qkv"] else 1, : 2 * P]
    if case["pairing"] == "halves":
        u, v = turn[..., :P], turn[..., P:]
        t = torch.cat([u * cos - v * sin, u * sin + v * cos], -1)
    else:
        u, v = turn[..., 0::2], turn[..., 1::2]
        t = torch.stack([u * cos - v * sin, u * sin + v * cos], -1).flatten(-2)
    y = x.clone()
    y[..., : 2 if case["qkv"] else 1, : 2 * P] = t
    live = torch.arange(H, device=DEV).view(1, 1, H, 1, 1) < torch.tensor(s["h"], device=DEV)[_paths(s, True)].view(B, 1, 1, 1, 1)
    return {"out": torch.where(live, y, 0.0).to(s["x"].dtype).view(B, R, H * V * D)}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "linear" and 2 * case["B"] * case["R"] * case["C"] * case["N"] > 2e12:
        return None
    s = prepare(case, seed)
    path = s["idx"].tolist()
    perm = s["perm"].tolist()
    if case["op"] == "norm":
        out = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV)
        scale = torch.zeros(case["B"], case["R"], dtype=torch.float64, device=DEV)
        total = torch.zeros_like(out)
        for t, k in enumerate(s["k"]):
            at = [i for i in range(case["B"]) if path[i] == t]
            if not at:
                continue
            h = s["x"][at, :, :k].double()
            if s["res"] is not None:
                h = h + s["res"][at, :, :k].double()
            total[at, :, :k] = h
            n = h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * s["w"][:k].double()
            if not case["raw"]:
                step = n.abs().amax(-1, keepdim=True) / 127
                scale[at] = step.squeeze(-1)
                n = torch.where(step > 0, torch.round(n / step) * step, 0.0)
            out[at, :, :k] = n
        if case["grouped"]:
            out, scale = out[perm], scale[perm]
        got = {"out": out}
        if not case["raw"]:
            got["scale"] = scale
        if s["res"] is not None:
            got["sum"] = total
        return got
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    grouped = case["op"] == "rotary" or case["order"] == "grouped"
    rows = [path[i] for i in perm] if grouped else path         # path of every sample as the rows lie
    if case["op"] == "linear":
        for t in range(case["T"]):
            at = [i for i in range(case["B"]) if rows[i] == t]
            if not at:
                continue
            ki, ko = s["ki"][t], s["ko"][t]
            y = torch.einsum("brc,oc->bro", s["x"][at, :, :ki].double(), s["w"][:ko, :ki].double())
            y = y * s["sx"][at].double()[..., None] * s["sw"][:ko].double()
            if s["bias"] is not None:
                y = y + s["bias"][:ko].double()
            if s["res"] is not None:
                y = y + s["res"][at, :, :ko].double()
            if case["act"] == "relu":
                y = torch.relu(y)
            elif case["act"] == "gelu":
                y = y * torch.special.ndtr(y)
            out[at, :, :ko] = y
        return {"out": out}
    D, P = case["D"], case["pairs"]
    sec = _sections(case)
    first = 0
    turns = []                                                   # one complex factor per pair and row
    for a, n in enumerate(sec):
        for j in range(n):
            e = (first + j) / P if case["ladder"] == "shared" else j / n
            angle = s["pos"][a].double() * (10000.0 ** -e)
            turns.append(torch.polar(torch.ones_like(angle), angle))
        first += n
    z = torch.stack(turns, -1).view(1 if case["shared"] else case["B"], case["R"], P)
    V = 3 if case["qkv"] else 1
    i0 = torch.arange(P, device=DEV) * (1 if case["pairing"] == "halves" else 2)
    i1 = i0 + (P if case["pairing"] == "halves" else 1)
    for h in range(case["H"]):
        at = [i for i in range(case["B"]) if h < s["h"][rows[i]]]
        for v in range(V):
            c0 = (h * V + v) * D
            if not at:
                continue
            vec = s["x"][at, :, c0:c0 + D].double()
            if v < 2:
                c = torch.complex(vec[..., i0], vec[..., i1]) * (z if case["shared"] else z[at])
                vec[..., i0], vec[..., i1] = c.real, c.imag
            out[at, :, c0:c0 + D] = vec
    return {"out": out}
