"""Performance cases of the layer norm around the FP4 linears (with the
residual's addition, a gain and a shift, and its backward pass) and of
low-rank adapters beside a shared linear (with their gradients).

``own`` false computes each operator in its plain form (elementary torch
operations in FP32); true calls the library.  Sizes are those of the
synthetic denoisers in ``workloads`` plus generic ragged ones; ``draw`` gives
further cases over the same ranges: 1 to 26574 rows or tokens, 1 to 12288
columns of the norm and 1 to 9728 features of a linear, 1 to 64 adapters of
rank 1 to 128.
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
        dict(name="ln8-1", op="norm", rows=1, width=1152, type="bf16", out="mxfp8",
             residual=True, gain=True, shift=True, groups=1),
        # 8 SANA-like rollouts of 1024 tokens, gain and shift of every rollout
        dict(name="ln-sana", op="norm", rows=8192, width=2240, type="bf16", out="same",
             residual=True, gain=True, shift=True, groups=8),
        # 6 SD3.5-like rollouts (26574 tokens), in the 8 bits that a linear reads
        dict(name="ln8-sd35", op="norm", rows=26574, width=2432, type="bf16", out="mxfp8",
             residual=True, gain=True, shift=True, groups=6),
        # a training step in FP32 at sizes that are no multiple of anything
        dict(name="ln-back-ragged", op="norm_back", rows=1009, width=1283, type="f32",
             residual=True, gain=True, shift=True, groups=1),
        # gradients through the SD3.5-like rollouts
        dict(name="ln-back-sd35", op="norm_back", rows=26574, width=2432, type="bf16",
             residual=True, gain=True, shift=True, groups=6),
        # one token and the one adapter of a policy on the smallest layer: latency
        dict(name="adapter-1", op="adapters", tokens=1, K=1152, N=1152, rank=16, adapters=1,
             requests=1, order="one", none=0.0, hidden=False),
        # one token each of 64 requests, 48 adapters, on the SD3.5-like QKV layer
        dict(name="adapter-64", op="adapters", tokens=64, K=2432, N=7296, rank=32, adapters=48,
             requests=64, order="mixed", none=0.0, hidden=False),
        # requests of odd lengths through odd sizes, tokens in no order, a tenth without an adapter
        dict(name="adapter-ragged", op="adapters", tokens=1371, K=1235, N=1111, rank=24, adapters=5,
             requests=1371, order="mixed", none=0.1, hidden=False),
        # the training forward of the SD3.5-like QKV layer, the old and the new policy's rollouts
        dict(name="adapter-sd35", op="adapters", tokens=26574, K=2432, N=7296, rank=32, adapters=2,
             requests=6, order="blocks", none=0.0, hidden=True),
        # gradients at odd sizes, several requests an adapter
        dict(name="adapter-back-ragged", op="adapters_back", tokens=777, K=1235, N=1056, rank=8,
             adapters=5, requests=13, order="blocks", none=0.1, past=False),
        # gradients of the one adapter on the SANA-like QKV layer
        dict(name="adapter-back-sana", op="adapters_back", tokens=8192, K=2240, N=6720, rank=32,
             adapters=1, requests=8, order="one", none=0.0, past=True),
        # the largest: gradients of the SD3.5-like QKV layer's adapters
        dict(name="adapter-back-sd35", op="adapters_back", tokens=26574, K=2432, N=7296, rank=32,
             adapters=2, requests=6, order="blocks", none=0.0, past=True),
    ]


#: bytes of the largest listed norm case; elements and products of the largest adapter case
MOST_NORM = 5.1e8
MOST_ELEMENTS = 26574 * (3 * 2432 + 7296)
MOST_PRODUCTS = 26574 * (2432 + 7296) * 32
MOST_WEIGHTS = 48 * (2432 + 7296) * 32
WIDTHS = (1152, 2240, 2432, 5600, 7296, 9728)


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm_back", "adapters", "adapters", "adapters_back", "adapters_back"))
    if op in ("norm", "norm_back"):
        kind = rng.choice(("bf16", "bf16", "f16", "f32"))
        out = rng.choice(("same", "same", "mxfp8")) if op == "norm" else "same"
        width = rng.choice(WIDTHS) if rng.random() < 0.4 else _log_uniform(rng, 1, 12288)
        if out == "mxfp8":
            width = max(32, width // 32 * 32)
        rows = _log_uniform(rng, 1, 26574)
        rows = max(1, min(rows, int(MOST_NORM / (4 * BYTES[kind] * width))))
        gain, shift = rng.random() < 0.8, rng.random() < 0.7
        groups = rng.choice((1, 1, 2, 4, 6, 8)) if gain or shift else 1
        rows = max(groups, rows // groups * groups)
        case = dict(op=op, rows=rows, width=width, type=kind, residual=rng.random() < 0.75, gain=gain, shift=shift,
                    groups=groups)
        return dict(case, out=out) if op == "norm" else case
    K = rng.choice(WIDTHS) if rng.random() < 0.5 else _log_uniform(rng, 1, 9728)
    N = rng.choice(WIDTHS) if rng.random() < 0.5 else _log_uniform(rng, 1, 9728)
    rank = rng.choice((8, 16, 32, 64, 128)) if rng.random() < 0.75 else rng.randint(1, 128)
    adapters = 1 if rng.random() < 0.25 else _log_uniform(rng, 2, 64)
    adapters = max(1, min(adapters, int(MOST_WEIGHTS / ((K + N) * rank))))
    tokens = _log_uniform(rng, 1, 26574)
    tokens = max(1, min(tokens, MOST_ELEMENTS // (3 * K + 2 * N), MOST_PRODUCTS // ((K + N) * rank)))
    order = rng.choice(("blocks", "blocks", "mixed"))
    if adapters == 1 and rng.random() < 0.7:
        order = "one"
    requests = tokens if order == "mixed" else min(tokens, _log_uniform(rng, 1, 96))
    none = 0.0 if order == "one" else rng.choice((0.0, 0.0, 0.1, 0.5))
    case = dict(op=op, tokens=tokens, K=K, N=N, rank=rank, adapters=adapters, requests=requests, order=order, none=none)
    if op == "adapters":
        return dict(case, hidden=rng.random() < 0.4)
    return dict(case, past=rng.random() < 0.75)


# ---- inputs ---------------------------------------------------------------

def _normal(seed, role, *shape):
    g = torch.Generator(device=DEV).manual_seed(1000 * int(seed) + role)
    return torch.randn(*shape, device=DEV, generator=g)


def _hidden_state(seed, role, rows, width, kind):
    """A hidden state: N(0, 1) with a scale 10^U(-1, 1) per token."""
    g = torch.Generator(device=DEV).manual_seed(1000 * int(seed) + role + 500)
    scale = 10.0 ** (2.0 * torch.rand(rows, 1, device=DEV, generator=g) - 1.0)
    return (_normal(seed, role, rows, width) * scale).to(TYPES[kind])


def _mx_scale_exponent(amax, largest):
    """Exponent of the power-of-two scale of a block with this largest
    magnitude, for elements whose largest exponent is `largest`."""
    e = torch.frexp(amax)[1] - 1 - largest
    return torch.where(amax > 0, e, -127).clamp(-127, 127)


def _mxfp8(y):
    """E4M3 codes and E8M0 scales of rows of 32-element groups, each as values."""
    b = y.view(y.shape[0], -1, 32)
    e = _mx_scale_exponent(b.abs().amax(-1), 8)
    # two factors, each a normal number at every exponent
    half = torch.div(e, 2, rounding_mode="floor")
    q = b * torch.exp2(-half.float()).unsqueeze(-1) * torch.exp2((half - e).float()).unsqueeze(-1)
    codes = q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(y.shape)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _index(case, seed):
    """The adapter of every token, -1 for none: requests take the adapters in
    a shuffled order over and over, a share of the requests none."""
    T, R, E = case["tokens"], case["requests"], case["adapters"]
    g = torch.Generator().manual_seed(1000 * int(seed) + 77)
    of = torch.randperm(E, generator=g).repeat(-(-R // E))[:R]
    of[torch.rand(R, generator=g) < case["none"]] = -1
    if case["order"] == "mixed":
        return of[torch.randperm(T, generator=g)].to(torch.int32)
    cuts = torch.cat((torch.tensor([0]), torch.randperm(T - 1, generator=g)[:R - 1].sort()[0] + 1, torch.tensor([T])))
    return of.repeat_interleave(cuts.diff()).to(torch.int32)


def prepare(case, seed):
    op = case["op"]
    s = dict(case=case)
    if op in ("norm", "norm_back"):
        rows, width, kind, groups = case["rows"], case["width"], case["type"], case["groups"]
        s["x"] = _hidden_state(seed, 1, rows, width, kind)
        s["r"] = _hidden_state(seed, 2, rows, width, kind) if case["residual"] else None
        s["gain"] = s["shift"] = None
        if case["gain"]:
            s["gain"] = (1 + 0.2 * _normal(seed, 3, groups, width)).to(TYPES[kind])
        if case["shift"]:
            s["shift"] = (0.2 * _normal(seed, 6, groups, width)).to(TYPES[kind])
        if op == "norm_back":
            s["dy"] = (1e-2 * _normal(seed, 4, rows, width)).to(TYPES[kind])
            # the gradient that reaches the sum past the norm
            if case["residual"]:
                s["r"] = (1e-2 * _normal(seed, 5, rows, width)).to(TYPES[kind])
        return s
    T, K, N, r, E = (case[k] for k in ("tokens", "K", "N", "rank", "adapters"))
    bf16 = torch.bfloat16
    s["x"] = _normal(seed, 1, T, K).to(bf16)
    s["a"] = (_normal(seed, 2, E, r, K) / math.sqrt(K)).to(bf16)
    s["b"] = (0.1 * _normal(seed, 3, E, N, r)).to(bf16)
    # alpha / rank of every adapter
    s["scales"] = torch.tensor([(0.5, 1.0, 2.0)[(e + 2) % 3] for e in range(E)], device=DEV)
    index = None if case["order"] == "one" else _index(case, seed)
    s["rows"] = [None] if index is None else [(index == e).nonzero()[:, 0].to(DEV) for e in range(E)]
    s["index"] = None if index is None else index.to(DEV)
    s["plan"] = None
    if own and index is not None:
        import paper_2604_06916_amd as sol
        s["plan"] = sol.adapter_plan(s["index"], E)
    if op == "adapters":
        s["y"] = _normal(seed, 4, T, N).to(bf16)
    else:
        s["dy"] = (1e-2 * _normal(seed, 5, T, N)).to(bf16)
        s["past"] = (1e-2 * _normal(seed, 6, T, K)).to(bf16) if case["past"] else None
        # what the forward pass kept
        s["hidden"] = torch.zeros(T, r, device=DEV)
        for e, rows in enumerate(s["rows"]):
            rows = slice(None) if rows is None else rows
            s["hidden"][rows] = s["x"][rows].float() @ s["a"][e].float().t()
    return s


# ---- the plain forms, in FP32 ---------------------------------------------

def _per_row(gain, rows):
    return gain.float().repeat_interleave(rows // gain.shape[0], 0)


def _plain_norm(s, case):
    v = s["x"].float()
    if s["r"] is not None:
        v = v + s["r"].float()
    d = v - v.mean(-1, keepdim=True)
    y = d * torch.rsqrt(d.square().mean(-1, keepdim=True) + EPS)
    if s["gain"] is not None:
        y = y * _per_row(s["gain"], case["rows"])
    if s["shift"] is not None:
        y = y + _per_row(s["shift"], case["rows"])
    out = {"sum": v.to(s["x"].dtype)} if s["r"] is not None else {}
    if case["out"] == "mxfp8":
        out["codes"], out["scales"] = _mxfp8(y)
    else:
        out["out"] = y.to(s["x"].dtype)
    return out


def _plain_norm_back(s, case):
    v, dy = s["x"].float(), s["dy"].float()
    d = v - v.mean(-1, keepdim=True)
    rho = torch.rsqrt(d.square().mean(-1, keepdim=True) + EPS)
    n = d * rho
    g = dy if s["gain"] is None else dy * _per_row(s["gain"], case["rows"])
    dx = rho * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    if s["r"] is not None:
        dx = dx + s["r"].float()
    out = {"dx": dx.to(s["x"].dtype)}
    if s["gain"] is not None:
        out["dgain"] = (dy * n).view(case["groups"], -1, case["width"]).sum(1)
    if s["shift"] is not None:
        out["dshift"] = dy.view(case["groups"], -1, case["width"]).sum(1)
    return out


def _plain_adapters(s, case):
    out = s["y"].float()
    hidden = torch.zeros(case["tokens"], case["rank"], device=DEV)
    for e, rows in enumerate(s["rows"]):
        rows = slice(None) if rows is None else rows
        h = s["x"][rows].float() @ s["a"][e].float().t()
        hidden[rows] = h
        out[rows] += s["scales"][e] * (h @ s["b"][e].float().t())
    out = {"out": out.to(torch.bfloat16)}
    return dict(out, hidden=hidden) if case["hidden"] else out


def _plain_adapters_back(s, case):
    past = s["past"]
    dx = torch.zeros(case["tokens"], case["K"], device=DEV) if past is None else past.float()
    da, db = torch.zeros(s["a"].shape, device=DEV), torch.zeros(s["b"].shape, device=DEV)
    for e, rows in enumerate(s["rows"]):
        rows = slice(None) if rows is None else rows
        dy = s["dy"][rows].float() * s["scales"][e]
        g = dy @ s["b"][e].float()
        dx[rows] += g @ s["a"][e].float()
        da[e] = g.t() @ s["x"][rows].float()
        db[e] = dy.t() @ s["hidden"][rows]
    return {"dx": dx.to(torch.bfloat16), "da": da, "db": db}


# ---- one pass -------------------------------------------------------------

def _call(s, case):
    import paper_2604_06916_amd as sol
    op = case["op"]
    if op == "norm":
        if case["out"] == "mxfp8":
            codes, scales, total = sol.mxfp8_add_layernorm(s["x"], s["r"], s["gain"], s["shift"], EPS)
            out = {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}
        else:
            y, total = sol.add_layernorm(s["x"], s["r"], s["gain"], s["shift"], EPS)
            out = {"out": y}
        return dict(out, sum=total) if s["r"] is not None else out
    if op == "norm_back":
        dx, dgain, dshift = sol.layernorm_backward(s["dy"], s["x"], s["gain"], s["shift"], s["r"], EPS)
        out = {"dx": dx}
        if dgain is not None:
            out["dgain"] = dgain
        return out if dshift is None else dict(out, dshift=dshift)
    if op == "adapters":
        out, hidden = sol.add_adapters(s["y"], s["x"], s["a"], s["b"], s["scales"], s["plan"], hidden=case["hidden"])
        return {"out": out} if hidden is None else {"out": out, "hidden": hidden}
    dx, da, db = sol.adapters_backward(s["dy"], s["x"], s["hidden"], s["a"], s["b"], s["scales"], s["plan"], s["past"])
    return {"dx": dx, "da": da, "db": db}


def run(state):
    case = state["case"]
    if own:
        return _call(state, case)
    return {"norm": _plain_norm, "norm_back": _plain_norm_back, "adapters": _plain_adapters,
            "adapters_back": _plain_adapters_back}[case["op"]](state, case)


def work(case):
    op = case["op"]
    if op in ("adapters", "adapters_back"):
        T, K, N, r, E = (case[k] for k in ("tokens", "K", "N", "rank", "adapters"))
        used = min(E, case["requests"])
        at = 0 if case["order"] == "one" else 4 * T
        weights = 2 * used * (K + N) * r + at
        if op == "adapters":
            return {"bytes": 2 * T * (K + 2 * N) + weights + (4 * T * r if case["hidden"] else 0),
                    "flops": 2 * T * r * (K + N)}
        return {"bytes": 2 * T * (N + K * (3 if case["past"] else 2)) + 4 * T * r + weights + 4 * E * (K + N) * r,
                "flops": 4 * T * r * (K + N)}
    b = BYTES[case["type"]]
    n, g = case["rows"] * case["width"], case["groups"] * case["width"]
    rows = (1 if case["gain"] else 0) + (1 if case["shift"] else 0)
    if op == "norm":
        out = b if case["out"] == "same" else 1 + 1 / 32
        return {"bytes": n * (b + (2 * b if case["residual"] else 0) + out) + b * g * rows, "flops": 8 * n}
    return {"bytes": n * b * (4 if case["residual"] else 3) + (b if case["gain"] else 0) * g + 4 * g * rows,
            "flops": 14 * n}


# ---- the definitions, in 64 bits ------------------------------------------

def _grouped(t, rows, gain, width):
    return t.view(gain.shape[0], rows // gain.shape[0], width), gain.double().view(gain.shape[0], 1, width)


def _exact_norm(s, case):
    rows, width = case["rows"], case["width"]
    v = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
    mean = v.sum(1, keepdim=True) / width
    y = (v - mean) / ((v - mean).pow(2).sum(1, keepdim=True) / width + EPS).sqrt()
    if s["gain"] is not None:
        y, g = _grouped(y, rows, s["gain"], width)
        y = (y * g).view(rows, width)
    if s["shift"] is not None:
        y, t = _grouped(y, rows, s["shift"], width)
        y = (y + t).view(rows, width)
    out = {} if s["r"] is None else {"sum": v}
    if case["out"] == "same":
        return dict(out, out=y)
    b = y.view(rows, width // 32, 32)
    scale = torch.ldexp(torch.ones_like(b[..., 0]), (torch.frexp(b.abs().max(-1)[0])[1] - 9).clamp(-127, 127))
    return dict(out, codes=(b / scale.unsqueeze(-1)).clamp(-448, 448).view(rows, width), scales=scale)


def _exact_norm_back(s, case):
    """The gradients, with c = s - mean(s), q = mean(c^2) + eps, y = c q^-1/2 g:
    dL/dc_i = G_i q^-1/2 - c_i q^-3/2 sum(G c) / width, and ds = dc - mean(dc)."""
    rows, width = case["rows"], case["width"]
    v, dy = s["x"].double(), s["dy"].double()
    c = v - v.sum(1, keepdim=True) / width
    q = c.pow(2).sum(1, keepdim=True) / width + EPS
    G = dy
    if s["gain"] is not None:
        G, g = _grouped(dy, rows, s["gain"], width)
        G = (G * g).view(rows, width)
    dc = G / q.sqrt() - c * (G * c).sum(1, keepdim=True) / (width * q * q.sqrt())
    dx = dc - dc.sum(1, keepdim=True) / width
    if s["r"] is not None:
        dx += s["r"].double()
    out = {"dx": dx}
    if s["gain"] is not None:
        out["dgain"] = (dy * c / q.sqrt()).view(case["groups"], rows // case["groups"], width).sum(1)
    if s["shift"] is not None:
        out["dshift"] = dy.view(case["groups"], rows // case["groups"], width).sum(1)
    return out


def _segments(s, case):
    """(adapter, its tokens) from the sorted index."""
    if s["index"] is None:
        return [(0, torch.arange(case["tokens"], device=DEV))]
    of, order = s["index"].long().sort(stable=True)
    ends = torch.searchsorted(of, torch.arange(case["adapters"] + 1, device=DEV)).tolist()
    return [(e, order[ends[e]:ends[e + 1]]) for e in range(case["adapters"]) if ends[e + 1] > ends[e]]


def _exact_adapters(s, case):
    out = s["y"].double()
    hidden = out.new_zeros(case["tokens"], case["rank"])
    for e, at in _segments(s, case):
        h = torch.mm(s["x"].double()[at], s["a"][e].double().t())
        hidden.index_copy_(0, at, h)
        out.index_add_(0, at, torch.mm(h * s["scales"][e].double(), s["b"][e].double().t()))
    return {"out": out, "hidden": hidden} if case["hidden"] else {"out": out}


def _exact_adapters_back(s, case):
    x, dy, h = s["x"].double(), s["dy"].double(), s["hidden"].double()
    dx = torch.zeros_like(x) if s["past"] is None else s["past"].double()
    da, db = (torch.zeros(s[k].shape, device=DEV, dtype=torch.float64) for k in ("a", "b"))
    for e, at in _segments(s, case):
        c = s["scales"][e].double()
        g = torch.mm(dy[at], s["b"][e].double()) * c
        dx.index_add_(0, at, torch.mm(g, s["a"][e].double()))
        da[e] = torch.mm(g.t().contiguous(), x[at])
        db[e] = torch.mm(dy[at].t().contiguous(), h[at]) * c
    return {"dx": dx, "da": da, "db": db}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_back": _exact_norm_back, "adapters": _exact_adapters,
            "adapters_back": _exact_adapters_back}[case["op"]](s, case)
