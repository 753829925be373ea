"""The conditioned Stage-1 blocks (norms modulated by a few-token linear of
the condition, residuals added in the norms, rotary positions in the packed
QKV), stage by stage against float64 from the GPU's own input to each stage;
and a captured step replayed with each step's condition against eager steps.

Tolerances: linears 2e-3 (the GEMM bar), BF16 stages one rounding (2^-7
relative), MXFP4 and MXFP8 encodings compared as what the linears make of
them (their codes are pinned in test_gpu_norm.py)."""
import numpy as np
import pytest
import torch

import oracle.nvfp4 as O
import oracle.operators as R
from gpu_util import bf16_from_dev, device, say, u8_from_dev
from oracle import stage1 as S

pytestmark = pytest.mark.gpu


def config(steps=2, blocks=2):
    from paper_2604_06916_amd.stage1 import Stage1Config
    return Stage1Config(blocks=blocks, hidden=256, heads=2, mlp=512, rollouts=4, tokens=64, steps=steps, keep=2,
                        w_sigma=0.05, seed=6100, conditioned=True)


def f64(t):
    return O.bf16_bits_to_f32(bf16_from_dev(t)).astype(np.float64)


def rel(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


@pytest.mark.parametrize("backend", ["bf16", "nvfp4", "mxfp4"])
def test_stages(backend):
    from paper_2604_06916_amd import stage1 as G
    cfg, dev = config(), device()
    H, hd, T = cfg.hidden, cfg.head_dim, cfg.tokens
    model = G.make_weights(cfg, dev)
    runner = G.Runner(cfg, model, backend, dev)
    runner.trace = []
    x0 = G.initial_latents(cfg, dev)
    keep = x0.clone()
    runner.set_step(1)
    runner.blocks(x0)
    torch.cuda.synchronize()
    assert torch.equal(x0, keep)
    time, text = (f64(t) for t in G.make_condition(cfg, dev))
    c = R.add_rmsnorm(np.repeat(time[1:2], cfg.rollouts, 0), text, None, G.EPS)[1]
    if backend == "mxfp4":
        got = R.mxfp8_values(*(u8_from_dev(t) for t in runner.c))
        assert rel(got, c) <= 2.0 ** -4
        c = got
    else:
        assert rel(f64(runner.c[0]), c) <= 2.0 ** -8
        c = f64(runner.c[0])
    ang = np.arange(T)[:, None] * 10000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    table = np.concatenate((np.cos(ang), np.sin(ang)), 1)
    x3 = f64(runner.trace.pop()[1])
    per = len(runner.trace) // cfg.blocks
    assert per * cfg.blocks == len(runner.trace)
    last = None
    for b in range(cfg.blocks):
        names = dict(runner.trace[b * per: (b + 1) * per])
        t = {n: f64(v) if v.dtype == torch.bfloat16 else u8_from_dev(v) for n, v in names.items()}
        blk = {n: (bf16_from_dev(w), bf16_from_dev(bias)) for n, (w, bias) in model[b].items()}
        L = {n: (S.prepare(backend, w), bias) for n, (w, bias) in blk.items()}
        bias = O.bf16_bits_to_f32(blk["mod"][1]).astype(np.float64)
        w = L["mod"][0]
        w = w if backend == "bf16" else O.nvfp4_dequantize_ref(*w) if backend == "nvfp4" else O.mxfp4_unscaled_ref(*w)
        gains = c @ w.T + bias
        assert rel(t["gains"], gains) <= 2e-3

        def linear(h, name):
            if backend == "mxfp4":
                return O.mxfp4_gemm_ref(t[h], t[h + " scales"], *L[name][0], L[name][1])
            return S.linear(backend, t[h], *L[name])

        def norm_check(x, r, gain, total, h):
            s, y = R.add_rmsnorm(x, r, gain, G.EPS)
            assert rel(total, S.bf16_round(s)) <= 2.0 ** -9
            if backend == "mxfp4":
                # E2M1 rounds within a quarter of the value and clips 8 to 6
                assert rel(O.mxfp4_unscaled_ref(t[h], t[h + " scales"]), y) <= 0.25, h
            else:
                assert rel(t[h], y) <= 2.0 ** -8, h
        g = t["gains"]
        x_in = (f64(x0), None) if last is None else last
        norm_check(*x_in, g[:, :H], t["x"], "h1")
        assert rel(t["qkv"], linear("h1", "qkv")) <= 2e-3
        qkv = t["qkv"].reshape(-1, 3, cfg.heads, hd).copy()
        at = np.arange(qkv.shape[0]) % T
        for i in (0, 1):
            qkv[:, i] = R.rotate(qkv[:, i], table, at, "interleaved")[0]
        assert rel(t["rotated"], qkv.reshape(t["rotated"].shape)) <= 2.0 ** -8
        assert np.array_equal(t["rotated"][:, 2 * H:], t["qkv"][:, 2 * H:])
        a = S.attention(t["rotated"], cfg.rollouts, T, cfg.heads, hd)
        assert rel(t["a"], a) <= 2.0 ** -7
        assert rel(t["o"], S.linear(backend, t["a"], *L["out"])) <= 2e-3
        norm_check(t["o"], t["x"], g[:, H:], t["x2"], "h2")
        assert rel(t["up"], linear("h2", "up")) <= 2e-3
        # a GELU result rounded the other way flips FP4 codes of the down layer
        assert rel(t["d"], S.linear(backend, S.bf16_round(S.gelu_tanh(t["up"])), *L["down"])) <= (
            2e-3 if backend == "bf16" else 5e-2)
        last = (t["d"], t["x2"])
        say(f"{backend} block {b}: stages agree")
    assert rel(x3, t["x2"] + t["d"]) <= 2.0 ** -8


@pytest.mark.parametrize("backend", ["nvfp4", "mxfp4"])
def test_captured_steps(backend):
    from paper_2604_06916_amd import stage1 as G
    cfg, dev = config(steps=3), device()
    runner = G.Runner(cfg, G.make_weights(cfg, dev), backend, dev)
    x0 = G.initial_latents(cfg, dev)
    want = runner.rollout(x0)
    static = x0.clone()
    graph = runner.capture_step(static)
    for _ in range(2):
        static.copy_(x0)
        for t in range(cfg.steps):
            runner.set_step(t)
            graph.replay()
            torch.cuda.synchronize()
        assert torch.equal(static, want)


def test_the_condition_matters_and_the_plain_loop_is_as_it_was():
    from dataclasses import replace

    from paper_2604_06916_amd import stage1 as G
    cfg, dev = config(), device()
    x0 = G.initial_latents(cfg, dev)
    runner = G.Runner(cfg, G.make_weights(cfg, dev), "mxfp4", dev)
    a = runner.blocks(x0)
    runner.set_step(1)
    assert not torch.equal(a, runner.blocks(x0))
    plain = replace(cfg, conditioned=False)
    model = G.make_weights(plain, dev)
    assert all(torch.equal(p, q) for m, n in zip(model, G.make_weights(cfg, dev)) for k in m for p, q in zip(m[k], n[k]))
    assert "mod" not in model[0] and not hasattr(G.Runner(plain, model, "mxfp4", dev), "gains")
