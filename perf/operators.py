"""Performance cases of the operators around the FP4 linears: the
root-mean-square norm with the residual's addition (and its backward pass),
rotary positions, and products of few tokens with 4-bit weights.

``own`` false computes each operator in its plain form (elementary torch
operations in FP32); true calls the library.  Sizes are those of the
synthetic denoisers in ``workloads`` plus generic ragged ones; ``draw`` gives
further cases over the same ranges: 1 to 26574 rows, 1 to 12288 columns, heads
of 32 to 256, 1 to 64 tokens against 4-bit weights of up to 18432 x 3072.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # one token's residual add and norm, written in 8 bits: latency
        dict(name="norm8-1", op="norm", rows=1, width=1152, type="bf16", out="mxfp8",
             residual=True, gain=True, groups=1),
        # 8 SANA-like rollouts of 1024 tokens, the gain modulated per rollout
        dict(name="norm-sana", op="norm", rows=8192, width=2240, type="bf16", out="same",
             residual=True, gain=True, groups=8),
        # the FLUX.1-like hidden state (4 rollouts, 18432 tokens), in 8 bits
        dict(name="norm8-flux", op="norm", rows=18432, width=3072, type="bf16", out="mxfp8",
             residual=True, gain=True, groups=4),
        # a training step in FP32 at sizes that are no multiple of anything
        dict(name="norm-back-ragged", op="norm_back", rows=777, width=1235, type="f32",
             residual=True, gain=True, groups=1),
        # the largest: gradients through 6 SD3.5-like images (26574 tokens)
        dict(name="norm-back-sd35", op="norm_back", rows=26574, width=2432, type="bf16",
             residual=True, gain=True, groups=6),
        # one new token's q (24 heads) and k (8 heads) at its position
        dict(name="rotary-1", op="rotary", tokens=1, q_heads=24, k_heads=8, dim=128, rotated=128,
             layout="half", type="bf16", table=4608, positions="int64", inverse=False),
        # q and k of the packed QKV output of 4 FLUX.1-like rollouts, every
        # rollout at positions 0 to 4607
        dict(name="rotary-flux", op="rotary", tokens=18432, q_heads=24, k_heads=24, dim=128,
             rotated=128, layout="interleaved", type="bf16", table=4608, positions="none",
             inverse=False),
        # gradients of q and k of 6 x 333 text tokens, 80 of 128 elements of a
        # head rotated, positions given
        dict(name="rotary-back-text", op="rotary", tokens=1998, q_heads=19, k_heads=19, dim=128,
             rotated=80, layout="half", type="f16", table=8192, positions="int32", inverse=True),
        # one conditioning vector through the smallest layer: latency
        dict(name="w4-1", op="product", M=1, N=1152, K=1152, fmt="nvfp4", x="bf16", bias=True),
        # four rollouts' conditioning vectors to six modulation vectors each
        dict(name="w4-modulation", op="product", M=4, N=18432, K=3072, fmt="nvfp4", x="bf16",
             bias=True),
        # odd token count and width, K a multiple of the 32-element group only
        dict(name="w4-ragged", op="product", M=13, N=1235, K=1056, fmt="mxfp4", x="bf16",
             bias=False),
        # 64 tokens in 8 bits through the SD3.5-like MLP-up layer
        dict(name="w4a8-up", op="product", M=64, N=9728, K=2432, fmt="mxfp4", x="mxfp8", bias=True),
    ]


#: bytes of the largest listed norm and rotary cases; weight elements of the largest product
MOST_BYTES = 4.5e8
MOST_WEIGHT = 18432 * 3072
WIDTHS = (1152, 2240, 2432, 3072, 5600, 9728, 12288)


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm_back", "rotary", "product", "product"))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "product":
        fmt, x = rng.choice((("nvfp4", "bf16"), ("mxfp4", "bf16"), ("mxfp4", "mxfp8")))
        block = 16 if fmt == "nvfp4" else 32
        K = rng.choice(WIDTHS) if rng.random() < 0.5 else block * _log_uniform(rng, 1, 12288 // block)
        N = rng.choice(WIDTHS) if rng.random() < 0.4 else _log_uniform(rng, 1, 18432)
        return dict(op=op, M=_log_uniform(rng, 1, 64), N=max(1, min(N, MOST_WEIGHT // K)), K=K,
                    fmt=fmt, x=x, bias=rng.random() < 0.75)
    if op == "rotary":
        dim = rng.choice((32, 64, 80, 96, 128, 128, 192, 256))
        rotated = dim if rng.random() < 0.5 else 2 * rng.randint(1, dim // 2)
        k_heads = rng.randint(0, 32)
        q_heads = k_heads * rng.choice((1, 1, 2, 4)) if k_heads else rng.randint(1, 64)
        tokens = _log_uniform(rng, 1, 18432)
        tokens = max(1, min(tokens, int(MOST_BYTES / (2 * BYTES[kind] * dim * (q_heads + k_heads)))))
        return dict(op=op, tokens=tokens, q_heads=q_heads, k_heads=k_heads, dim=dim, rotated=rotated,
                    layout=rng.choice(("half", "interleaved")), type=kind,
                    table=_log_uniform(rng, 16, 32768), positions=rng.choice(("none", "int32", "int64")),
                    inverse=rng.random() < 0.5)
    out = "same"
    if op == "norm":
        out = rng.choice(("same", "same", "mxfp8"))
    width = rng.choice(WIDTHS) if rng.random() < 0.4 else _log_uniform(rng, 1, 12288)
    if out == "mxfp8":
        width = max(32, width // 32 * 32)
    rows = _log_uniform(rng, 1, 26574)
    rows = max(1, min(rows, int(MOST_BYTES / (4 * BYTES[kind] * width))))
    gain = rng.random() < 0.8
    groups = rng.choice((1, 1, 2, 4, 6, 8)) if gain else 1
    rows = max(groups, rows // groups * groups)
    case = dict(op=op, rows=rows, width=width, type=kind, residual=rng.random() < 0.75, gain=gain,
                groups=groups)
    return dict(case, out=out) if op == "norm" else case


# ---- inputs ---------------------------------------------------------------

def _normal(seed, role, *shape):
    g = torch.Generator(device=DEV).manual_seed(1000 * int(seed) + role)
    return torch.randn(*shape, device=DEV, generator=g)


def _hidden(seed, role, rows, width, kind):
    """A hidden state: N(0, 1) with a scale 10^U(-1, 1) per token."""
    g = torch.Generator(device=DEV).manual_seed(1000 * int(seed) + role + 500)
    scale = 10.0 ** (2.0 * torch.rand(rows, 1, device=DEV, generator=g) - 1.0)
    return (_normal(seed, role, rows, width) * scale).to(TYPES[kind])


def _mx_scale_exponent(amax, largest):
    """Exponent of the power-of-two scale of a block with this largest
    magnitude, for elements whose largest exponent is `largest`."""
    e = torch.frexp(amax)[1] - 1 - largest
    return torch.where(amax > 0, e, -127).clamp(-127, 127)


def _e2m1_codes(y):
    """Codes of the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to even), sign in bit 3."""
    a = y.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return c + 8 * torch.signbit(y).to(torch.uint8)


def _weight(seed, N, K, fmt):
    """A quantized N(0, 0.02^2) weight: packed codes, group scales, and NVFP4's tensor scale."""
    w = 0.02 * _normal(seed, 11, N, K)
    block = 16 if fmt == "nvfp4" else 32
    b = w.view(N, K // block, block)
    amax = b.abs().amax(-1)
    if fmt == "nvfp4":
        alpha = (amax.max() / 2688.0).view(1)
        s = (amax / (6.0 * alpha)).clamp(max=448.0).to(torch.float8_e4m3fn)
        step = s.float() * alpha
    else:
        e = _mx_scale_exponent(amax, 2)
        s, step = e + 127, torch.exp2(e.float())
    c = _e2m1_codes((b / step.clamp(min=1e-30).unsqueeze(-1)).view(N, K))
    packed = c[:, 0::2] | (c[:, 1::2] << 4)
    if fmt == "nvfp4":
        return packed.contiguous(), s.view(torch.uint8).contiguous(), alpha
    return packed.contiguous(), s.to(torch.uint8).contiguous()


def _table(case):
    """cos and sin of position x frequency, [positions, rotated] FP32 (cos of
    every pair, then sin): what a program keeps for all its calls."""
    i = torch.arange(case["rotated"] // 2, device=DEV, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * i / case["rotated"])
    a = torch.arange(case["table"], device=DEV, dtype=torch.float64).unsqueeze(1) * f
    return torch.cat((a.cos(), a.sin()), 1).float()


def _mxfp8(y):
    """E4M3 codes and E8M0 scales of rows of 32-element groups, each as values."""
    b = y.view(y.shape[0], -1, 32)
    e = _mx_scale_exponent(b.abs().amax(-1), 8)
    # two factors, each a normal number at every exponent
    half = torch.div(e, 2, rounding_mode="floor")
    q = b * torch.exp2(-half.float()).unsqueeze(-1) * torch.exp2((half - e).float()).unsqueeze(-1)
    codes = q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(y.shape)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    op = case["op"]
    s = dict(case=case)
    if op in ("norm", "norm_back"):
        rows, width, kind = case["rows"], case["width"], case["type"]
        s["x"] = _hidden(seed, 1, rows, width, kind)
        s["r"] = _hidden(seed, 2, rows, width, kind) if case["residual"] else None
        s["gain"] = None
        if case["gain"]:
            s["gain"] = (1 + 0.2 * _normal(seed, 3, case["groups"], width)).to(TYPES[kind])
        if op == "norm_back":
            s["dy"] = (1e-2 * _normal(seed, 4, rows, width)).to(TYPES[kind])
            # the gradient that reaches the sum past the norm
            if case["residual"]:
                s["r"] = (1e-2 * _normal(seed, 5, rows, width)).to(TYPES[kind])
    elif op == "rotary":
        T, H, G = case["tokens"], case["q_heads"], case["k_heads"]
        # q, k and v side by side in one buffer, as the QKV linear leaves them
        qkv = _normal(seed, 1, T, H + 2 * G, case["dim"]).to(TYPES[case["type"]])
        s["q"], s["k"] = qkv[:, :H], (qkv[:, H:H + G] if G else None)
        s["table"], s["positions"] = _table(case), None
        if case["positions"] != "none":
            g = torch.Generator(device=DEV).manual_seed(1000 * int(seed) + 2)
            s["positions"] = torch.randint(case["table"], (T,), device=DEV, generator=g,
                                           dtype=getattr(torch, case["positions"]))
    else:
        M, N, K = case["M"], case["N"], case["K"]
        s["w"] = _weight(seed, N, K, case["fmt"])
        x = _normal(seed, 1, M, K)
        if case["x"] == "mxfp8":
            codes, scales = _mxfp8(x)
            s["x"] = (codes.view(torch.uint8), scales.view(torch.uint8))
        else:
            s["x"] = (x.to(torch.bfloat16),)
        s["bias"] = (0.02 * _normal(seed, 3, N)).to(torch.bfloat16) if case["bias"] else None
    return s


# ---- the plain forms, in FP32 ---------------------------------------------

def _per_row(gain, rows):
    return gain.float().repeat_interleave(rows // gain.shape[0], 0)


def _plain_norm(s, case):
    v = s["x"].float()
    if s["r"] is not None:
        v = v + s["r"].float()
    y = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
    if s["gain"] is not None:
        y = y * _per_row(s["gain"], case["rows"])
    out = {"sum": v.to(s["x"].dtype)} if s["r"] is not None else {}
    if case["out"] == "mxfp8":
        out["codes"], out["scales"] = _mxfp8(y)
    else:
        out["out"] = y.to(s["x"].dtype)
    return out


def _plain_norm_back(s, case):
    v, dy = s["x"].float(), s["dy"].float()
    rho = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
    n = v * rho
    g = dy if s["gain"] is None else dy * _per_row(s["gain"], case["rows"])
    dx = rho * (g - n * (g * n).mean(-1, keepdim=True))
    if s["r"] is not None:
        dx = dx + s["r"].float()
    out = {"dx": dx.to(s["x"].dtype)}
    if s["gain"] is not None:
        out["dgain"] = (dy * n).view(case["groups"], -1, case["width"]).sum(1)
    return out


def _plain_rotated(t, cs, case):
    R = case["rotated"]
    c, sn = cs[:, None, :R // 2], cs[:, None, R // 2:]
    if case["inverse"]:
        sn = -sn
    f = t.float()
    if case["layout"] == "half":
        u, v = f[..., :R // 2], f[..., R // 2:R]
        r = torch.cat((u * c - v * sn, u * sn + v * c), -1)
    else:
        u, v = f[..., 0:R:2], f[..., 1:R:2]
        r = torch.stack((u * c - v * sn, u * sn + v * c), -1).flatten(-2)
    return torch.cat((r, f[..., R:]), -1).to(t.dtype)


def _plain_rotary(s, case):
    at = s["positions"]
    if at is None:
        at = torch.arange(case["tokens"], device=DEV) % case["table"]
    cs = s["table"][at.long()]
    out = {"q": _plain_rotated(s["q"], cs, case)}
    if s["k"] is not None:
        out["k"] = _plain_rotated(s["k"], cs, case)
    return out


def _e2m1_values(packed):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    return table[torch.stack((packed & 15, packed >> 4), -1).flatten(-2).int()]


def _e8m0_values(scales):
    return torch.exp2(scales.float() - 127.0)


def _plain_product(s, case):
    N, K = case["N"], case["K"]
    w = _e2m1_values(s["w"][0])
    if case["fmt"] == "nvfp4":
        w = w.view(N, -1, 16) * (s["w"][1].view(torch.float8_e4m3fn).float() * s["w"][2]).unsqueeze(-1)
    else:
        w = w.view(N, -1, 32) * _e8m0_values(s["w"][1]).unsqueeze(-1)
    x = s["x"][0]
    if case["x"] == "mxfp8":
        x = x.view(torch.float8_e4m3fn).float().view(case["M"], -1, 32) * _e8m0_values(s["x"][1]).unsqueeze(-1)
    y = x.float().view(case["M"], K) @ w.view(N, K).t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return {"out": y.to(torch.bfloat16)}


# ---- one pass -------------------------------------------------------------

def _call(s, case):
    import paper_2604_06916_amd as sol
    op = case["op"]
    if op == "norm":
        if case["out"] == "mxfp8":
            codes, scales, total = sol.mxfp8_add_rmsnorm(s["x"], s["r"], s["gain"], EPS)
            out = {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}
        else:
            y, total = sol.add_rmsnorm(s["x"], s["r"], s["gain"], EPS)
            out = {"out": y}
        return dict(out, sum=total) if s["r"] is not None else out
    if op == "norm_back":
        dx, dgain = sol.rmsnorm_backward(s["dy"], s["x"], s["gain"], s["r"], EPS)
        return {"dx": dx, "dgain": dgain} if dgain is not None else {"dx": dx}
    if op == "rotary":
        q, k = sol.rotary(s["q"], s["k"], s["table"], s["positions"], layout=case["layout"],
                          inverse=case["inverse"])
        return {"q": q, "k": k} if k is not None else {"q": q}
    if case["x"] == "mxfp8":
        return {"out": sol.mxfp8_linear(*s["x"], *s["w"], s["bias"])}
    f = sol.nvfp4_weight_linear if case["fmt"] == "nvfp4" else sol.mxfp4_weight_linear
    return {"out": f(*s["x"], *s["w"], s["bias"])}


def run(state):
    case = state["case"]
    if own:
        return _call(state, case)
    return {"norm": _plain_norm, "norm_back": _plain_norm_back, "rotary": _plain_rotary,
            "product": _plain_product}[case["op"]](state, case)


def work(case):
    op = case["op"]
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        w = N * K * (0.5 + (1 / 16 if case["fmt"] == "nvfp4" else 1 / 32))
        x = M * K * (2 if case["x"] == "bf16" else 1 + 1 / 32)
        return {"bytes": w + x + 2 * M * N + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    b = BYTES[case["type"]]
    if op == "rotary":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"])
        cs = 4 * case["rotated"] * min(case["tokens"], case["table"])
        at = case["tokens"] * {"none": 0, "int32": 4, "int64": 8}[case["positions"]]
        return {"bytes": 2 * b * n * case["dim"] + cs + at, "flops": 3 * n * case["rotated"]}
    n, g = case["rows"] * case["width"], case["groups"] * case["width"] if case["gain"] else 0
    if op == "norm":
        out = b if case["out"] == "same" else 1 + 1 / 32
        return {"bytes": n * (b + (2 * b if case["residual"] else 0) + out) + b * g, "flops": 5 * n}
    return {"bytes": n * b * (4 if case["residual"] else 3) + (b + 4) * g, "flops": 10 * n}


# ---- the definitions, in 64 bits ------------------------------------------

def _exact_norm(s, case):
    rows, width = case["rows"], case["width"]
    v = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
    y = v / (v.pow(2).sum(1, keepdim=True) / width + EPS).sqrt()
    if s["gain"] is not None:
        y = (y.view(case["groups"], -1, width) * s["gain"].double().view(case["groups"], 1, width)).view(rows, width)
    out = {} if s["r"] is None else {"sum": v}
    if case["out"] == "same":
        return dict(out, out=y)
    b = y.view(rows, width // 32, 32)
    scale = torch.ldexp(torch.ones_like(b[..., 0]), (torch.frexp(b.abs().max(-1)[0])[1] - 9).clamp(-127, 127))
    return dict(out, codes=(b / scale.unsqueeze(-1)).clamp(-448, 448).view(rows, width), scales=scale)


def _exact_norm_back(s, case):
    """The gradients, with s = x, q = mean(s^2) + eps: y = s q^-1/2 g has
    dy_j / ds_i = g_j (delta_ij q^-1/2 - s_i s_j q^-3/2 / width)."""
    rows, width = case["rows"], case["width"]
    v, dy = s["x"].double(), s["dy"].double()
    q = v.pow(2).sum(1, keepdim=True) / width + EPS
    g = dy
    if s["gain"] is not None:
        g = (dy.view(case["groups"], -1, width) * s["gain"].double().view(case["groups"], 1, width)).view(rows, width)
    dx = g / q.sqrt() - v * (g * v).sum(1, keepdim=True) / (width * q * q.sqrt())
    if s["r"] is not None:
        dx += s["r"].double()
    out = {"dx": dx}
    if s["gain"] is not None:
        out["dgain"] = (dy * v / q.sqrt()).view(case["groups"], rows // case["groups"], width).sum(1)
    return out


def _exact_rotary(s, case):
    R, T = case["rotated"], case["tokens"]
    at = torch.arange(T, device=DEV).remainder(case["table"]) if s["positions"] is None else s["positions"].long()
    turn = torch.complex(s["table"][at, :R // 2].double(), s["table"][at, R // 2:].double())[:, None]
    if case["inverse"]:
        turn = turn.conj()
    out = {}
    for name in ("q", "k"):
        if s[name] is None:
            continue
        t = s[name].double().clone()
        first, second = (slice(0, R // 2), slice(R // 2, R)) if case["layout"] == "half" else \
            (slice(0, R, 2), slice(1, R, 2))
        z = torch.complex(t[..., first], t[..., second]) * turn
        t[..., first], t[..., second] = z.real, z.imag
        out[name] = t
    return out


def _exact_product(s, case):
    M, N, K = case["M"], case["N"], case["K"]
    codes, scales = s["w"][0], s["w"][1].long()
    mag = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], device=DEV, dtype=torch.float64) / 2
    w = torch.empty(N, K, device=DEV, dtype=torch.float64)
    for half, nibble in ((0, codes.long() & 15), (1, codes.long() >> 4)):
        w[:, half::2] = mag[nibble & 7] * (1 - 2 * (nibble >> 3))
    if case["fmt"] == "nvfp4":
        m, e = scales & 7, scales >> 3                      # E4M3, bias 7, subnormals below 2^-6
        value = torch.where(e > 0, (8 + m) * 2.0 ** (e.double() - 10), m * 2.0 ** -9)
        w = w.view(N, -1, 16) * (value * s["w"][2].double()).unsqueeze(-1)
    else:
        w = w.view(N, -1, 32) * 2.0 ** (scales.double() - 127).unsqueeze(-1)
    x = s["x"][0]
    if case["x"] == "mxfp8":
        c = x.long()
        m, e = c & 7, (c >> 3) & 15
        x = torch.where(e > 0, (8 + m) * 2.0 ** (e.double() - 10), m * 2.0 ** -9) * (1 - 2 * (c >> 7))
        x = x.view(M, -1, 32) * 2.0 ** (s["x"][1].double() - 127).unsqueeze(-1)
    y = x.double().reshape(M, K) @ w.view(N, K).t().contiguous()
    return {"out": y if s["bias"] is None else y + s["bias"].double()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_back": _exact_norm_back, "rotary": _exact_rotary,
            "product": _exact_product}[case["op"]](s, case)
