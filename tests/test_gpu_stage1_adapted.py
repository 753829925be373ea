"""The conditioned Stage-1 blocks with layer norms and with the adapters of
several policies, stage by stage against float64 from the GPU's own input to
each stage; a captured step against eager ones; and one block's pieces run
forward and backward together, their gradients against float64 autograd.

Tolerances as for the conditioned blocks: linears 2e-3, BF16 stages one rounding
(2^-8 in the norm), MXFP4 codes a quarter of the value."""
import numpy as np
import pytest
import torch

import oracle.nvfp4 as O
import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import bf16_from_dev, device, u8_from_dev
from oracle import stage1 as S
from test_gpu_stage1_conditioned import f64, rel

pytestmark = pytest.mark.gpu


def config(layer_norm, adapters, steps=2):
    from paper_2604_06916_amd.stage1 import Stage1Config
    return Stage1Config(blocks=2, hidden=256, heads=2, mlp=512, rollouts=4, tokens=72, steps=steps, keep=2,
                        w_sigma=0.05, seed=6200, conditioned=True, layer_norm=layer_norm, adapters=adapters, rank=24)


@pytest.mark.parametrize("layer_norm,adapters", [(True, 0), (False, 3), (True, 2)])
@pytest.mark.parametrize("backend", ["bf16", "nvfp4", "mxfp4"])
def test_stages(backend, layer_norm, adapters):
    from paper_2604_06916_amd import stage1 as G
    cfg, dev = config(layer_norm, adapters), device()
    H = cfg.hidden
    model = G.make_weights(cfg, dev)
    runner = G.Runner(cfg, model, backend, dev)
    runner.trace = []
    x0 = G.initial_latents(cfg, dev)
    runner.blocks(x0)
    torch.cuda.synchronize()
    runner.trace.pop()
    per = len(runner.trace) // cfg.blocks
    policy = np.repeat(np.arange(cfg.rollouts) % max(adapters, 1), cfg.tokens)
    last = None
    for b in range(cfg.blocks):
        names = dict(runner.trace[b * per: (b + 1) * per])
        t = {n: f64(v) if v.dtype == torch.bfloat16 else u8_from_dev(v) for n, v in names.items()}
        L = {n: (S.prepare(backend, bf16_from_dev(w)), bf16_from_dev(bias)) for n, (w, bias) in model[b].items()
             if not n.endswith(" adapters")}
        g = t["gains"]
        assert g.shape == (cfg.rollouts, (4 if layer_norm else 2) * H)

        def norm_check(x, r, i, total, h):
            if layer_norm:
                s, y, _ = R.add_layernorm(x, r, g[:, i * H: (i + 1) * H], g[:, (i + 2) * H: (i + 3) * H], G.EPS)
            else:
                s, y = R.add_rmsnorm(x, r, g[:, i * H: (i + 1) * H], G.EPS)
            assert rel(total, S.bf16_round(s)) <= 2.0 ** -9
            if h + " scales" in t:
                assert rel(O.mxfp4_unscaled_ref(t[h], t[h + " scales"]), y) <= 0.25
            else:
                assert rel(t[h], y) <= 2.0 ** -8

        def linear_check(h, name, got):
            if h + " scales" in t:
                want = O.mxfp4_gemm_ref(t[h], t[h + " scales"], *L[name][0], L[name][1])
            else:
                want = S.linear(backend, t[h], *L[name])
            if adapters:
                assert rel(t[name + " linear"], want) <= 2e-3
                a, up = (f64(w) for w in model[b][name + " adapters"])
                c = np.full(adapters, G.ADAPTER_ALPHA / cfg.rank)
                want = R.add_adapters(t[name + " linear"], t[h], a, up, c, policy)[0]
                assert rel(want, t[name + " linear"]) > 0.05          # the adapters matter
                assert rel(t[got], want) <= 2.0 ** -8
            else:
                assert rel(t[got], want) <= 2e-3
        assert ("h1 scales" in t) == (backend == "mxfp4" and not adapters)
        norm_check(*((f64(x0), None) if last is None else last), 0, t["x"], "h1")
        linear_check("h1", "qkv", "qkv")
        linear_check("a", "out", "o")
        norm_check(t["o"], t["x"], 1, t["x2"], "h2")
        last = (t["d"], t["x2"])


@pytest.mark.parametrize("backend", ["nvfp4", "mxfp4"])
def test_captured_steps(backend):
    from paper_2604_06916_amd import stage1 as G
    cfg, dev = config(True, 2, steps=3), device()
    runner = G.Runner(cfg, G.make_weights(cfg, dev), backend, dev)
    x0 = G.initial_latents(cfg, dev)
    want = runner.rollout(x0)
    static = x0.clone()
    graph = runner.capture_step(static)
    for _ in range(3):
        static.copy_(x0)
        for t in range(cfg.steps):
            runner.set_step(t)
            graph.replay()
            torch.cuda.synchronize()
        assert torch.equal(static, want)


def test_rollouts_of_one_policy_do_not_see_another():
    """The same latents and prompts under two policies; changing the second's
    adapters changes its rollouts alone."""
    from paper_2604_06916_amd import stage1 as G
    cfg, dev = config(True, 2), device()
    model = G.make_weights(cfg, dev)
    runner = G.Runner(cfg, model, "mxfp4", dev)
    x0 = G.initial_latents(cfg, dev)
    a = runner.blocks(x0).view(cfg.rollouts, -1).clone()
    for blk in model:
        for name in ("qkv adapters", "out adapters"):
            blk[name][1][1] = -blk[name][1][1]
    b = G.Runner(cfg, model, "mxfp4", dev).blocks(x0).view(cfg.rollouts, -1)
    assert torch.equal(a[::2], b[::2]) and not torch.equal(a[1], b[1]) and not torch.equal(a[3], b[3])


def test_a_norm_a_linear_and_adapters_forward_and_backward():
    """out = adapters(linear(layernorm(x + r))): the calls' gradients, the base
    weight frozen, against float64 autograd of the same chain.  The chain's own
    BF16 values are what the calls are given (sum, h, dh), so each gradient is
    off by the BF16 roundings of dh (2^-8 of it) and its own: 2^-6 of its norm."""
    dev, f32 = device(), torch.float64
    g = torch.Generator().manual_seed(9)
    rows, H, N, rank, E = 150, 96, 160, 8, 3

    def draw(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g)).to(torch.bfloat16).to(dev)
    x, r, w = draw(rows, H), draw(rows, H), draw(N, H, scale=H ** -0.5)
    gain, shift = 1 + draw(3, H, scale=0.3), draw(3, H, scale=0.3)
    a, b = draw(E, rank, H, scale=H ** -0.5), draw(E, N, rank, scale=0.3)
    c = torch.tensor([2.0, 0.5, 1.0], device=dev)
    index = torch.randint(-1, E, (rows,), generator=g).to(dev)
    dy = draw(rows, N, scale=0.1)
    plan = sol.adapter_plan(index, E)
    h, total = sol.add_layernorm(x, r, gain, shift)
    y = (h.float() @ w.float().t()).to(torch.bfloat16)
    out, hidden = sol.add_adapters(y, h, a, b, c, plan, hidden=True)
    past = (dy.float() @ w.float()).to(torch.bfloat16)
    dh, da, db = sol.adapters_backward(dy, h, hidden, a, b, c, plan, past)
    dx, dgain, dshift = sol.layernorm_backward(dh, total, gain, shift)
    leaves = [t.cpu().to(f32).requires_grad_() for t in (x, gain, shift, a, b)]
    n = torch.nn.functional.layer_norm(leaves[0] + r.cpu().to(f32), (H,), eps=1e-6)
    h64 = n * leaves[1].repeat_interleave(50, 0) + leaves[2].repeat_interleave(50, 0)
    at = index.cpu()
    e = at.clamp(min=0)
    add = torch.einsum("tnr,trk,tk->tn", leaves[4][e], leaves[3][e], h64) * (c.cpu().to(f32)[e] * (at >= 0))[:, None]
    out64 = h64 @ w.cpu().to(f32).t() + add
    assert rel(f64(out), out64.detach().numpy()) <= 2.0 ** -6
    grads = torch.autograd.grad((out64 * dy.cpu().to(f32)).sum(), leaves)
    for got, want in zip((dx, dgain, dshift, da, db), grads):
        got = got.detach().cpu().double().numpy()
        assert rel(got, want.numpy()) <= 2.0 ** -6
