"""The events that time a Stage-1 rollout cover every op of its blocks,
conditioned or not: four linears a block and step, the other ops by kind."""
import pytest
import torch

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("backend", ["bf16", "nvfp4", "mxfp4"])
@pytest.mark.parametrize("conditioned", [False, True])
def test_every_op_is_timed(backend, conditioned):
    from paper_2604_06916_amd import stage1 as G
    cfg = G.Stage1Config(blocks=2, hidden=256, heads=2, mlp=512, rollouts=4, tokens=64, steps=3, keep=2, w_sigma=0.05,
                         seed=6100, conditioned=conditioned)
    dev = device()
    runner = G.Runner(cfg, G.make_weights(cfg, dev), backend, dev)
    x0 = G.initial_latents(cfg, dev)
    want = runner.rollout(x0)
    runner.linear_events, runner.op_events = [], {}
    got = runner.rollout(x0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    n = cfg.blocks * cfg.steps
    assert len(runner.linear_events) == 4 * n
    counts = {kind: len(events) for kind, events in runner.op_events.items()}
    gelu = "gelu+amax" if backend == "nvfp4" else "gelu"
    kinds = {"norm": 2 * n, "attention": n, "copy": n, gelu: n, "euler": cfg.steps}
    if conditioned:
        # the last block's residual has no norm after it
        assert counts == {**kinds, "condition": cfg.steps, "modulation": n, "rotary": n, "residual": cfg.steps}
    else:
        assert counts == {**kinds, "residual": 2 * n}
    assert all(a.elapsed_time(b) >= 0 for events in (runner.linear_events, *runner.op_events.values()) for a, b in events)
