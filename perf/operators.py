"""The operators of an attention layer around the quantized attention, measured: what a video-DiT block calls
next to `vc_attn`.

    qk      vc_qk_norm_rope   RMS norm of queries and keys and the position rotation, in one pass
    cross   vc_cross_attn     attention to an encoder's states (text, image tokens) of another length
    quant   vc_quant_fp8      activations (or weights) to E4M3 with a scale for each block of 128
    linear  vc_linear_fp8     product of two such matrices: the projections in front of and behind attention

Sizes are those of the Wan- and HunyuanVideo-shaped workloads and of the tests' odd grids.  With `own` false, `run`
computes the same in elementary torch operations in 32 bits (rotation angles in 64), rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
THETA = 10000.0
YARN_FAST, YARN_SLOW = 32.0, 1.0


# ----------------------------------------------------------------------------- cases
def _qk(B, Hq, Hk, grid, d, dtype="bf16", norm="head", rotary="interleaved", dims=None, scaling="none", factor=1.0,
        original=0, start=0, positions=False, token_major=True, name=None):
    if dims is None:
        side = 2 * (d // 6)
        dims = (d - 2 * side, side, side)
    c = {"op": "qk", "B": B, "Hq": Hq, "Hk": Hk, "t": grid[0], "y": grid[1], "x": grid[2], "d": d, "dtype": dtype, "norm": norm,
         "rotary": rotary, "dt": dims[0], "dy": dims[1], "dx": dims[2], "scaling": scaling, "factor": float(factor),
         "original": original, "start": start, "positions": positions, "token_major": token_major}
    return dict(c, name=name) if name else c


def _cross(B, H, Hkv, Nq, Nkv, d, dtype="bf16", lengths="full", mask=False, lse=False, token_major=True, name=None):
    c = {"op": "cross", "B": B, "H": H, "Hkv": Hkv, "Nq": Nq, "Nkv": Nkv, "d": d, "dtype": dtype, "lengths": lengths,
         "mask": mask, "lse": lse, "token_major": token_major}
    return dict(c, name=name) if name else c


def _quant(B, H, N, d, dtype="bf16", block_rows=1, token_major=False, name=None):
    c = {"op": "quant", "B": B, "H": H, "N": N, "d": d, "dtype": dtype, "block_rows": block_rows, "token_major": token_major}
    return dict(c, name=name) if name else c


def _linear(M, N, K, dtype="bf16", bias=True, name=None):
    c = {"op": "linear", "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias}
    return dict(c, name=name) if name else c


def listed():
    wan = (21, 30, 52)
    return [
        # two heads of a short clip: the smallest call, where the launch counts
        _qk(1, 2, 2, (4, 16, 16), 128, name="qk tiny"),
        # grouped narrow heads of an odd grid in half precision, part of the head rotated in halves, positions of a
        # sequence longer than the trained one
        _qk(2, 6, 2, (1955, 1, 1), 64, dtype="fp16", rotary="half", dims=(48, 0, 0), scaling="yarn", factor=4.0, original=512,
            positions=True, name="qk odd fp16 half yarn"),
        # Wan-14B layer: one norm over all heads of a token, three-axis rotation, as the projection leaves Q and K
        _qk(1, 40, 40, wan, 128, norm="token", name="qk wan14b"),
        # a single query token against a long encoder sequence: keys and values are read once and that is all
        _cross(2, 16, 16, 1, 16384, 128, name="cross one token"),
        # odd clip with grouped narrow heads, image tokens with holes in their mask, one batch without any
        _cross(3, 6, 2, 1955, 257, 64, dtype="fp16", lengths="empty", mask=True, lse=True, name="cross odd fp16 d64"),
        # Wan-1.3B layer, prompt shorter than the padded text
        _cross(1, 12, 12, 32760, 512, 128, lengths="ragged", name="cross wan1.3b"),
        # Wan-14B layer, all 512 text tokens
        _cross(1, 40, 40, 32760, 512, 128, name="cross wan14b"),
        # the prompt's states on their way to K and V
        _quant(1, 1, 512, 4096, dtype="fp32", token_major=True, name="quant text fp32"),
        # the output of a Wan-14B attention, heads outermost, on its way to the output projection
        _quant(1, 40, 32760, 128, name="quant wan14b"),
        # a conditioning vector: one row, the weights are read once
        _linear(1, 5120, 5120, name="linear one row"),
        # an odd number of prompt tokens, a width that ends inside a block, single-precision output
        _linear(1955, 1000, 1536 - 48, dtype="fp32", bias=False, name="linear odd fp32"),
        # Wan-14B projection
        _linear(32760, 5120, 5120, name="linear wan14b"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any operator, type and layout; one to 32760 rows, one to 16384 keys, widths up to 5120."""
    op = rng.choice(["qk", "cross", "quant", "linear"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    B = rng.choice([1, 1, 2, 3])
    d = rng.choice([128, 128, 64])
    while True:
        if op == "qk":
            n = _log(rng, 1, 32760)
            t = rng.randint(1, min(n, 21))
            x = max(1, round(math.sqrt(n / t) * rng.uniform(0.8, 1.6)))
            y = max(1, round(n / t / x))
            Hq = rng.choice([1, 2, 5, 6, 12, 16, 24, 40])
            Hk = rng.choice([Hq, Hq, 1, max(1, Hq // 2)])
            scaling = rng.choice(["none", "none", "linear", "ntk", "yarn"])
            rotary = rng.choice(["interleaved", "half", "none"])
            norm = rng.choice(["head", "token", "none"]) if rotary != "none" else rng.choice(["head", "token"])
            dims = rng.choice([None, None, (d, 0, 0), (d // 2, 0, 0), (16, 24, 24), (d // 4, d // 8, d // 4)])
            if B * t * y * x * (Hq + Hk) * d <= 2 * 32760 * 40 * 128:
                return _qk(B, Hq, Hk, (t, y, x), d, dtype, norm, rotary, dims, scaling, 1.0 if scaling == "none" else rng.uniform(1.2, 8.0),
                           rng.randint(64, 4096) if scaling == "yarn" else 0, rng.choice([0, 0, rng.randint(1, 100000)]), rng.random() < 0.3, rng.random() < 0.6)
        elif op == "cross":
            dtype = "fp16" if dtype == "fp32" else dtype
            Nq, Nkv = _log(rng, 1, 32760), _log(rng, 1, 16384)
            Hkv = rng.choice([1, 2, 3, 6, 12, 20])
            H = Hkv * rng.choice([1, 1, 2, 4])
            if B * H * Nq * Nkv <= 40 * 32760 * 512 // 2:
                return _cross(B, H, Hkv, Nq, Nkv, d, dtype, rng.choice(["full", "ragged", "empty"]), rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.6)
        elif op == "quant":
            N, H = _log(rng, 1, 32760), rng.choice([1, 2, 6, 12, 24, 40])
            if H == 1:
                d = 16 * rng.randint(1, 320)
            if B * N * H * d <= 32760 * 5120:
                return _quant(B, H, N, d, dtype, rng.choice([1, 1, 128]), rng.random() < 0.5)
        else:
            M, N, K = _log(rng, 1, 32760), _log(rng, 8, 5120), 16 * _log(rng, 1, 320)
            return _linear(M, N, K, dtype, rng.random() < 0.5)


# ----------------------------------------------------------------------------- inputs
def _heads(case, H, N, g, token_major, scale=1.0):
    """[B, H, N, d] in the case's type: a view of [B, N, H, d] memory where a projection wrote it."""
    x = torch.randn((case["B"], N, H, case["d"]) if token_major else (case["B"], H, N, case["d"]), generator=g, device="cuda")
    x = x.mul_(scale).to(DTYPES[case["dtype"]])
    return x.transpose(1, 2) if token_major else x


def _codes(rows, K, block_rows, g):
    """E4M3 codes [rows, K] of normal values with a few large channels, and their scales."""
    w = torch.randn(rows, K, generator=g, device="cuda")
    w *= torch.rand(1, K, generator=g, device="cuda").pow_(-0.25)
    nb = (K + 127) // 128
    nr = (rows + block_rows - 1) // block_rows
    pad = torch.zeros(nr * block_rows, nb * 128, device="cuda")
    pad[:rows, :K] = w
    scale = pad.view(nr, block_rows, nb, 128).abs().amax(dim=(1, 3)).clamp_min(1e-30) / 448.0
    full = scale.repeat_interleave(block_rows, dim=0)[:rows].repeat_interleave(128, dim=1)[:, :K]
    return (w / full).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    dt = DTYPES[case["dtype"]]
    op, tm = case["op"], case.get("token_major", False)
    if op == "qk":
        B, N, d = case["B"], case["t"] * case["y"] * case["x"], case["d"]
        s["q"], s["k"] = (_heads(case, H, N, g, tm, 1.5) for H in (case["Hq"], case["Hk"]))
        s["wq"] = s["wk"] = s["pos"] = None
        if case["norm"] != "none":
            s["wq"], s["wk"] = ((1.0 + 0.2 * torch.randn(d * (H if case["norm"] == "token" else 1), generator=g, device="cuda")).to(dt)
                                for H in (case["Hq"], case["Hk"]))
        if case["positions"]:   # several clips packed into one sequence: positions start again
            s["pos"] = torch.randint(0, 8192, (B, N, 3), generator=g, device="cuda", dtype=torch.int32)
    elif op == "cross":
        B, Nq, Nkv = case["B"], case["Nq"], case["Nkv"]
        s["q"] = _heads(case, case["H"], Nq, g, tm, 2.0)
        s["k"] = _heads(case, case["Hkv"], Nkv, g, tm)
        s["v"] = _heads(case, case["Hkv"], Nkv, g, tm)
        s["len"] = s["mask"] = None
        if case["lengths"] != "full":
            s["len"] = torch.randint((Nkv + 3) // 4, Nkv + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            if case["lengths"] == "empty" and B > 1:
                s["len"][B - 1] = 0
        if case["mask"]:
            s["mask"] = torch.rand(B, Nkv, generator=g, device="cuda") < 0.8
    elif op == "quant":
        s["x"] = _heads(case, case["H"], case["N"], g, tm)
        s["x"].mul_(torch.rand(1, case["H"], 1, case["d"], generator=g, device="cuda").pow_(-0.25).to(dt))
    else:
        s["x"], xs = _codes(case["M"], case["K"], 1, g)
        s["xs"] = xs.t().contiguous()                      # [blocks of K][M]
        s["w"], s["ws"] = _codes(case["N"], case["K"], 128, g)
        s["bias"] = torch.randn(case["N"], generator=g, device="cuda").to(dt) if case["bias"] else None
    if own:
        _plan(s, dt)
    return s


def _plan(s, dt):
    """Outputs, workspaces and parameter blocks, as a program that calls the library in a loop holds them."""
    import paper_2609_15810_b200 as vc
    s["vc"] = vc
    if s["op"] == "qk":
        s["qo"], s["ko"] = (torch.empty(t.shape, dtype=dt, device="cuda") for t in (s["q"], s["k"]))
        s["p"] = vc.QkParams.of(
            s["q"], s["k"], s["qo"], s["ko"], grid=(s["t"], s["y"], s["x"]), weight=s["wq"],
            norm={"none": vc.VC_NORM_NONE, "head": vc.VC_NORM_HEAD, "token": vc.VC_NORM_TOKEN}[s["norm"]], eps=EPS,
            rotary={"none": vc.VC_ROTARY_NONE, "interleaved": vc.VC_ROTARY_INTERLEAVED, "half": vc.VC_ROTARY_HALF}[s["rotary"]],
            rope_dims=(s["dt"], s["dy"], s["dx"]), rope_theta=THETA, start=(s["start"], 0, 0),
            rope_scaling={"none": vc.VC_ROPE_SCALING_NONE, "linear": vc.VC_ROPE_SCALING_LINEAR, "ntk": vc.VC_ROPE_SCALING_NTK,
                          "yarn": vc.VC_ROPE_SCALING_YARN}[s["scaling"]],
            rope_factor=(s["factor"], 1.0, 1.0), rope_original=(s["original"], s["original"], s["original"]))
    elif s["op"] == "cross":
        B, H, Nq, d = s["q"].shape
        s["o"] = torch.empty((B, Nq, H, d) if s["token_major"] else (B, H, Nq, d), dtype=dt, device="cuda")
        s["o"] = s["o"].transpose(1, 2) if s["token_major"] else s["o"]
        s["lse_out"] = torch.empty(B, H, Nq, dtype=torch.float32, device="cuda") if s["lse"] else None
        s["p"] = vc.CrossParams.of(s["q"], s["k"], s["v"], s["o"])
        s["work"] = torch.empty(vc.vc_cross_workspace_bytes(s["p"]), dtype=torch.uint8, device="cuda")
    elif s["op"] == "quant":
        s["p"] = vc.QuantParams.of(s["x"], block_rows=s["block_rows"])
        rows, cols = s["B"] * s["N"], s["H"] * s["d"]
        nb = (cols + 127) // 128
        s["codes"] = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda")
        s["scale"] = torch.empty((nb, rows) if s["block_rows"] == 1 else ((rows + 127) // 128, nb), dtype=torch.float32, device="cuda")
    else:
        s["out"] = torch.empty(s["M"], s["N"], dtype=dt, device="cuda")
        s["p"] = vc.LinearParams.of(s["x"], s["w"], s["out"], bias=s["bias"])
        s["work"] = torch.empty(vc.vc_linear_workspace_bytes(s["p"]), dtype=torch.uint8, device="cuda")


# ----------------------------------------------------------------------------- plain forms
def _frequencies(s, axis, n):
    """Radians per position of the axis's pairs, 64 bits, and the factor of cos and sin."""
    i = torch.arange(n // 2, device="cuda", dtype=torch.float64)
    factor = s["factor"] if axis == 0 else 1.0
    theta = THETA
    if s["scaling"] == "ntk" and n > 2:
        theta = THETA * factor ** (n / (n - 2))
    f = theta ** (-2.0 * i / n)
    if s["scaling"] == "linear":
        f = f / factor
    if s["scaling"] == "yarn":
        lo, hi = (n * math.log(s["original"] / (b * 2.0 * math.pi)) / (2.0 * math.log(THETA)) for b in (YARN_FAST, YARN_SLOW))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), n - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        f = f / factor * ramp + f * (1.0 - ramp)
    return f


def _turn(x, cos, sin, start, n, half):
    """The n channels from `start` of x rotated by their pairs' angles, in place."""
    a = slice(start, start + n // 2) if half else slice(start, start + n, 2)
    b = slice(start + n // 2, start + n) if half else slice(start + 1, start + n, 2)
    x0, x1 = x[..., a], x[..., b]
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    x[..., a] = y0
    x[..., b] = y1


def _plain_qk(s):
    B, N, Y, X = s["B"], s["t"] * s["y"] * s["x"], s["y"], s["x"]
    token = torch.arange(N, device="cuda")
    grid = torch.stack([token // (Y * X) + s["start"], token // X % Y, token % X], dim=1)[None]        # [1, N, 3]
    pos = (grid if s["pos"] is None else s["pos"]).double()[:, None]                                  # [1 or B, 1, N, 3]
    dims = [s["dt"], s["dy"], s["dx"]] if s["rotary"] != "none" else []
    mult = 0.1 * math.log(s["factor"]) + 1.0 if s["scaling"] == "yarn" else 1.0
    angles = [pos[..., a:a + 1] * _frequencies(s, a, n) for a, n in enumerate(dims) if n]
    tables = [((a.cos() * mult).float(), (a.sin() * mult).float()) for a in angles]
    starts = [sum(dims[:a]) for a, n in enumerate(dims) if n]
    sizes = [n for n in dims if n]
    return {name: _plain_qk_one(s, s[name], s["w" + name], tables, starts, sizes) for name in ("q", "k")}


def _plain_qk_one(s, x, w, tables, starts, sizes):
    B, H, N, d = x.shape
    y = x.float()
    if s["norm"] == "head":
        y = y * torch.rsqrt((y * y).mean(dim=3, keepdim=True) + EPS) * w.float()
    elif s["norm"] == "token":
        y = y * torch.rsqrt((y * y).mean(dim=(1, 3), keepdim=True) + EPS) * w.float().view(1, H, 1, d)
    else:
        y = y.clone()
    [_turn(y, c, sn, a, n, s["rotary"] == "half") for (c, sn), a, n in zip(tables, starts, sizes)]
    return y.to(x.dtype).contiguous()


def _plain_cross(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    B, H, Nq, d = q.shape
    Hkv, Nkv = k.shape[1], k.shape[2]
    scores = q.reshape(B, Hkv, -1, d) @ k.transpose(2, 3) * d ** -0.5       # rows of the heads that share keys, together
    keep = torch.ones(B, Nkv, dtype=torch.bool, device="cuda")
    if s["len"] is not None:
        keep = torch.arange(Nkv, device="cuda")[None] < s["len"][:, None]
    if s["mask"] is not None:
        keep = keep & s["mask"]
    scores.masked_fill_(~keep[:, None, None], -math.inf)
    top = scores.amax(dim=3, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(dim=3, keepdim=True)
    o = p @ v / torch.where(total == 0.0, 1.0, total)
    out = {"o": o.view(B, H, Nq, d).to(s["q"].dtype)}
    if s["lse"]:
        out["lse"] = (top + total.log()).view(B, H, Nq)
    return out


def _plain_quant(s):
    B, H, N, d = s["x"].shape
    rows, cols, br = B * N, H * d, s["block_rows"]
    nb, nr = (cols + 127) // 128, (rows + br - 1) // br
    x = s["x"].transpose(1, 2).reshape(rows, cols).float()
    x = torch.nn.functional.pad(x, (0, nb * 128 - cols, 0, nr * br - rows)).view(nr, br, nb, 128)
    top = x.abs().amax(dim=(1, 3), keepdim=True).clamp_min(448.0 * 2.0 ** -100)
    codes = (x * (448.0 / top)).to(torch.float8_e4m3fn).view(nr * br, nb * 128)[:rows, :cols].contiguous()
    scale = (top / 448.0).view(nr, nb)
    return {"codes": codes, "scale": scale.t().contiguous() if br == 1 else scale}


def _plain_linear(s):
    x = s["x"].float() * s["xs"].t().repeat_interleave(128, dim=1)[:, :s["K"]]
    w = s["w"].float() * s["ws"].repeat_interleave(128, dim=0)[:s["N"]].repeat_interleave(128, dim=1)[:, :s["K"]]
    y = x @ w.t()
    if s["bias"] is not None:
        y += s["bias"].float()
    return y.to(DTYPES[s["dtype"]])


# ----------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return {"qk": _plain_qk, "cross": _plain_cross, "quant": _plain_quant, "linear": _plain_linear}[s["op"]](s)
    vc = s["vc"]
    if s["op"] == "qk":
        vc.vc_qk_norm_rope(s["p"], s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["qo"], s["ko"])
        return {"q": s["qo"], "k": s["ko"]}
    if s["op"] == "cross":
        vc.vc_cross_attn(s["p"], s["q"], s["k"], s["v"], s["len"], s["mask"], s["o"], s["lse_out"], s["work"])
        return {"o": s["o"], "lse": s["lse_out"]} if s["lse"] else {"o": s["o"]}
    if s["op"] == "quant":
        vc.vc_quant_fp8(s["p"], s["x"], s["codes"], s["scale"])
        return {"codes": s["codes"], "scale": s["scale"]}
    vc.vc_linear_fp8(s["p"], s["x"], s["xs"], s["w"], s["ws"], s["bias"], s["out"], s["work"])
    return s["out"]


def work(case):
    """Inputs read once, outputs written once; the products of the operator."""
    size = {"bf16": 2.0, "fp16": 2.0, "fp32": 4.0}[case["dtype"]]
    if case["op"] == "qk":
        rows = float(case["B"] * case["t"] * case["y"] * case["x"] * (case["Hq"] + case["Hk"]))
        return {"bytes": 2 * size * rows * case["d"], "flops": rows * case["d"] * 7.0}
    if case["op"] == "cross":
        B, d = case["B"], case["d"]
        kept = case["Nkv"] * (1.0 if case["lengths"] == "full" else 0.625)
        return {"bytes": size * B * d * (2.0 * case["H"] * case["Nq"] + 2.0 * case["Hkv"] * kept), "flops": 4.0 * B * case["H"] * case["Nq"] * kept * d}
    if case["op"] == "quant":
        n = float(case["B"] * case["N"] * case["H"] * case["d"])
        return {"bytes": n * (size + 1.0) + n / 32.0 / case["block_rows"], "flops": 3.0 * n}
    M, N, K = float(case["M"]), float(case["N"]), float(case["K"])
    return {"bytes": M * K + N * K + M * K / 32.0 + M * N * size, "flops": 2.0 * M * N * K}


# ----------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"qk": _exact_qk, "cross": _exact_cross, "quant": _exact_quant, "linear": _exact_linear}[case["op"]](s)


def _exact_qk(s):
    """Pair by pair as complex numbers."""
    N = s["t"] * s["y"] * s["x"]
    at = s["pos"]
    if at is None:
        t, y, x = torch.meshgrid(*(torch.arange(n, device="cuda") for n in (s["t"], s["y"], s["x"])), indexing="ij")
        at = torch.stack([t + s["start"], y, x], dim=3).reshape(1, N, 3).expand(s["B"], N, 3)
    out = {}
    for name in ("q", "k"):
        x, w = s[name].double(), s["w" + name]
        B, H, _, d = x.shape
        if w is not None:
            w = w.double().view(-1, 1, d)
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        for b in range(B):
            v = x[b]
            if s["norm"] != "none":
                power = torch.linalg.vector_norm(v, dim=2 if s["norm"] == "head" else (0, 2), keepdim=True) ** 2
                v = v / torch.sqrt(power / (d if s["norm"] == "head" else H * d) + EPS) * w
            y[b] = v
            c0 = 0
            for axis, n in enumerate((s["dt"], s["dy"], s["dx"]) if s["rotary"] != "none" else ()):
                for p in range(n // 2):
                    f = _exact_frequency(s, axis, n, p)
                    angle = at[b, :, axis].double() * f
                    one = torch.polar(torch.full_like(angle, 0.1 * math.log(s["factor"]) + 1.0 if s["scaling"] == "yarn" else 1.0), angle)
                    i, j = (c0 + p, c0 + p + n // 2) if s["rotary"] == "half" else (c0 + 2 * p, c0 + 2 * p + 1)
                    z = torch.complex(v[:, :, i].contiguous(), v[:, :, j].contiguous()) * one
                    y[b, :, :, i], y[b, :, :, j] = z.real, z.imag
                c0 += n
        out[name] = y
    return out


def _exact_frequency(s, axis, n, p):
    factor = s["factor"] if axis == 0 else 1.0
    base = 1.0 / THETA ** (2.0 * p / n)
    if s["scaling"] == "linear":
        return base / factor
    if s["scaling"] == "ntk":
        return base if n <= 2 else (THETA * factor ** (n / (n - 2))) ** (-2.0 * p / n)
    if s["scaling"] == "yarn":
        edge = [n * math.log(s["original"] / (2.0 * math.pi * turns)) / (2.0 * math.log(THETA)) for turns in (YARN_FAST, YARN_SLOW)]
        first, last = max(int(math.floor(edge[0])), 0), min(int(math.ceil(edge[1])), n - 1)
        share = min(1.0, max(0.0, (p - first) / max(last - first, 0.001)))
        return base * (1.0 - share) + base / factor * share
    return base


def _exact_cross(s):
    """Head by head, the kept keys alone."""
    B, H, Nq, d = s["q"].shape
    Hkv, Nkv = s["k"].shape[1:3]
    if float(B) * H * Nq * Nkv > 1e9:
        return None
    o = torch.zeros(B, H, Nq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, Nq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        kept = [j for j in range(Nkv if s["len"] is None else int(s["len"][b]))]
        kept = torch.tensor(kept, device="cuda", dtype=torch.long)
        if s["mask"] is not None:
            kept = kept[s["mask"][b, kept]]
        if kept.numel() == 0:
            continue
        for h in range(H):
            k, v = (s[t][b, h // (H // Hkv), kept].double() for t in ("k", "v"))
            x = torch.mm(s["q"][b, h].double(), k.t()) / math.sqrt(d)
            lse[b, h] = torch.logsumexp(x, dim=1)
            o[b, h] = torch.mm(torch.exp(x - lse[b, h][:, None]), v)
    return {"o": o, "lse": lse} if s["lse"] else {"o": o}


def _exact_quant(s):
    """The scales; a code is a rounding of what 32 bits say."""
    B, H, N, d = s["x"].shape
    x = s["x"].double().abs().permute(0, 2, 1, 3).reshape(B * N, H * d)
    step = s["block_rows"]
    cols = torch.stack([x[:, c:c + 128].amax(dim=1) for c in range(0, H * d, 128)], dim=1)
    rows = cols if step == 1 else torch.stack([cols[r:r + step].amax(dim=0) for r in range(0, B * N, step)])
    scale = torch.clamp_min(rows, 448.0 * 2.0 ** -100) / 448.0
    return {"codes": None, "scale": scale.t().contiguous() if step == 1 else scale}


def _exact_linear(s):
    """Block by block of the common width."""
    M, N, K = s["M"], s["N"], s["K"]
    y = torch.zeros(M, N, dtype=torch.float64, device="cuda") if s["bias"] is None else s["bias"].double()[None].repeat(M, 1)
    for b in range((K + 127) // 128):
        part = slice(128 * b, min(K, 128 * b + 128))
        ws = s["ws"][:, b].double().repeat_interleave(128)[:N, None]
        y.addmm_(s["x"][:, part].double() * s["xs"][b].double()[:, None], (s["w"][:, part].double() * ws).t())
    return y
