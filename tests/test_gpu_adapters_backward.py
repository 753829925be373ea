"""Gradients of the low-rank adapters against float64, element by element, and
against differences of the definition.

Bounds, in units of E = 2^-24 of the magnitudes that a value is formed from: g is
an FP32 sum of N exact products, shared by up to N / 128 workgroups, and a product
with the scale: N + 64 roundings at most.  For dx it is cut to two BF16 pieces,
2^-18, and summed over 2 rank products; for da it keeps 24 bits in three, each of
whose products with a token's x is added: 3 tokens + 64.  db the same with h,
which comes in FP32.  dx is rounded to BF16 once (2^-8 as in the forward pass)."""
import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device
from test_gpu_adapters import E, close, draw, f64, index_of, weights

pytestmark = pytest.mark.gpu


def case(seed, tokens, K, N, rank, adapters, kind, dtype=torch.int32):
    a, b, c = weights(seed, adapters, rank, K, N)
    x, dy, past = draw(seed + 2, tokens, K), draw(seed + 3, tokens, N, scale=0.1), draw(seed + 4, tokens, K, scale=0.1)
    if kind == "one":
        index, plan = None, None
    else:
        index = index_of(seed, tokens, adapters, kind, dtype)
        plan = sol.adapter_plan(index, adapters)
    _, hidden = sol.add_adapters(dy, x, a, b, c, plan, hidden=True)
    return dy, x, hidden, a, b, c, plan, past, index


def check(dy, x, hidden, a, b, c, plan, past, index, **kw):
    tokens, (_, rank, K), N = x.shape[0], a.shape, b.shape[1]
    at = np.zeros(tokens, np.int64) if index is None else index.cpu().numpy()
    h = np.nan_to_num(f64(hidden))
    dx, da, db, sx, sa, sb = R.adapters_backward(f64(dy), f64(x), h, f64(a), f64(b), np.ones(a.shape[0]) if c is None else
                                                 f64(c), at, None if past is None else f64(past))
    p = 0.0 if past is None else np.abs(f64(past))
    got = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past, **kw)
    assert got[1].shape == a.shape and got[2].shape == b.shape and got[1].dtype == got[2].dtype == torch.float32
    close(got[0], dx, np.abs(dx) * 2.0 ** -8 + sx * ((N + 2 * rank + 64) * E + 2.0 ** -18) + p * E + 1e-38, "dx")
    close(got[1], da, sa * (N + 3 * tokens + 128) * E + 1e-38, "da")
    close(got[2], db, sb * (3 * tokens + 64) * E + 1e-38, "db")
    return got


@pytest.mark.parametrize("rank", [1, 3, 8, 16, 24, 32, 33, 64, 100, 128])
@pytest.mark.parametrize("tokens", [1, 16, 17, 70])
def test_ranks(tokens, rank):
    check(*case(rank, tokens, 200, 131, rank, 4, "any"))


@pytest.mark.parametrize("tokens,K,N", [(1, 1, 1), (2, 7, 7), (31, 31, 63), (32, 64, 64), (33, 65, 65), (100, 1152, 1152),
                                        (257, 1235, 1111), (1371, 520, 9), (2000, 9, 1100), (4000, 96, 200),
                                        (20000, 40, 72)])
def test_sizes(tokens, K, N):
    check(*case(K, tokens, K, N, 24, 5, "mixed", torch.int64))
    check(*case(N, tokens, K, N, 8, 3, "blocks"))
    dy, x, hidden, a, b, _, _, _, _ = args = case(N + 1, tokens, K, N, 20, 1, "one")
    check(*args)
    _, hidden = sol.add_adapters(dy, x, a, b, hidden=True)
    check(dy, x, hidden, a, b, None, None, None, None)


@pytest.mark.parametrize("tokens,adapters", [(64, 48), (9, 700), (640, 64), (3000, 2)])
def test_many_adapters_and_none_for_some(tokens, adapters):
    got = check(*case(tokens, tokens, 136, 300, 16, adapters, "distinct"))
    if tokens < adapters:
        assert int((got[1].abs().amax((1, 2)) > 0).sum()) == tokens   # the others' gradients are zeros
    check(*case(tokens, tokens, 136, 300, 48, adapters, "any"))


def test_all_tokens_without_an_adapter():
    dy, x, hidden, a, b, c, _, past, _ = case(1, 70, 48, 64, 8, 2, "mixed")
    index = torch.full((70,), -1, dtype=torch.int32, device=device())
    index[69] = 5
    dy[3], x[4] = float("nan"), float("inf")
    plan = sol.adapter_plan(index, 2)
    dx, da, db = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    assert torch.equal(dx[:69], past[:69]) and torch.all(torch.isnan(dx[69]))
    assert torch.all(da == 0) and torch.all(db == 0)
    dx, _, _ = sol.adapters_backward(dy, x, hidden, a, b, c, plan)
    assert torch.all(dx[:69] == 0)


@pytest.mark.parametrize("offset", [0, 1, 3])
def test_strides_and_in_place(offset):
    tokens, K, N = 77, 90, 64
    dy, x, hidden, a, b, c, plan, past, index = case(3, tokens, K, N, 16, 3, "mixed")
    wide = draw(9, tokens, 3 * N + offset)
    dy_ = wide[:, N + offset:2 * N + offset]
    dy_.copy_(dy)
    x_ = draw(8, tokens, 2 * K + 1)[:, K + 1:]
    x_.copy_(x)
    room = draw(7, tokens, K + 13)
    keep = room.clone()
    past_ = room[:, offset:K + offset]
    past_.copy_(past)
    keep[:, offset:K + offset] = past
    want = check(dy, x, hidden, a, b, c, plan, past, index)
    got = sol.adapters_backward(dy_, x_, hidden, a, b, c, plan, past_, dx=past_)
    assert got[0] is past_ and all(torch.equal(p, q) for p, q in zip(want, got))
    keep[:, offset:K + offset] = want[0]
    assert torch.equal(room, keep)
    check(dy[:1].expand(tokens, N), x[:1].expand(tokens, K), hidden, a, b, c, plan, past[:1].expand(tokens, K), index)


def test_values_that_are_not_finite():
    """A token with an infinity spoils its dx and its adapter's gradients, no
    others.  They are infinite or NaN: h's pieces may have both signs or be 0, and
    an infinity times them added up is then NaN."""
    dy, x, hidden, a, b, c, plan, past, index = case(5, 90, 40, 48, 8, 3, "mixed")
    want = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    t = int((index == 1).nonzero()[-1])       # the last of its tile, whose other places repeat its row
    dy[t, 3] = float("inf")
    dx, da, db = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    others = torch.arange(90, device=device()) != t
    assert torch.equal(dx[others], want[0][others]) and not torch.any(torch.isfinite(dx[t]))
    assert torch.equal(da[[0, 2]], want[1][[0, 2]]) and torch.equal(db[[0, 2]], want[2][[0, 2]])
    assert not torch.any(torch.isfinite(db[1, 3])) and torch.equal(db[1, :3], want[2][1, :3])


def test_lengths_of_zero():
    a, b, c = weights(1, 2, 8, 40, 24)
    e = torch.empty(0, 24, dtype=torch.bfloat16, device=device())
    plan = sol.adapter_plan(torch.empty(0, dtype=torch.int32, device=device()), 2)
    dx, da, db = sol.adapters_backward(e, torch.empty(0, 40, dtype=torch.bfloat16, device=device()),
                                       torch.empty(0, 8, device=device()), a, b, c, plan)
    assert dx.shape == (0, 40) and torch.all(da == 0) and torch.all(db == 0)
    check(*case(2, 33, 40, 0, 8, 2, "mixed"))
    check(*case(2, 33, 0, 40, 8, 2, "mixed"))


def test_same_results_on_every_call_and_any_stream():
    dy, x, hidden, a, b, c, plan, past, _ = case(1, 3000, 320, 1448, 32, 6, "mixed")
    want = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    again = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(want, got, again))


def test_workspace_may_hold_anything():
    dy, x, hidden, a, b, c, plan, past, _ = case(1, 200, 96, 160, 16, 3, "any")
    want = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    need = sol.adapters_backward_workspace_bytes(200, 3, True, 160, 96, 16)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=device())     # NaN in every format
    got = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past, workspace=ws)
    assert all(torch.equal(p.nan_to_num(7.0), q.nan_to_num(7.0)) for p, q in zip(want, got))


def test_gradients_against_differences():
    """<dx, u>, <da, u>, <db, u> against central differences of the float64
    definition, which is bilinear: a step of 2^-6 has no error of its own.  The
    FP32 gradients' is within 2^-13 of the terms' magnitudes (N + 3 tokens + 128
    roundings), dx's BF16 one within 2^-8."""
    tokens, K, N, rank, adapters = 37, 24, 40, 6, 3
    dy, x, hidden, a, b, c, plan, past, index = case(11, tokens, K, N, rank, adapters, "mixed")
    dx, da, db = sol.adapters_backward(dy, x, hidden, a, b, c, plan, past)
    at, w, p = index.cpu().numpy(), f64(dy), f64(past)

    def loss(x, a, b):
        return float(np.sum(w * R.add_adapters(np.zeros((tokens, N)), x, a, b, f64(c), at)[0]) + np.sum(p * x))
    v = [f64(x), f64(a), f64(b)]
    rng = np.random.default_rng(1)
    step = 2.0 ** -6
    for i, (got, rel) in enumerate(((dx, 2.0 ** -8), (da, 2.0 ** -13), (db, 2.0 ** -13))):
        for _ in range(4):
            u = rng.standard_normal(v[i].shape)
            up, down = [t.copy() for t in v], [t.copy() for t in v]
            up[i] += step * u
            down[i] -= step * u
            want = (loss(*up) - loss(*down)) / (2 * step)
            size = float(np.sum(np.abs(f64(got) * u)))
            assert abs(float(np.sum(f64(got) * u)) - want) <= rel * size + 1e-9


def test_graph_replay_with_a_plan_written_again():
    dy, x, hidden, a, b, c, plan, past, index = case(1, 130, 96, 160, 16, 4, "mixed")

    def step():
        sol.adapter_plan(index, 4, plan)
        _, h = sol.add_adapters(dy, x, a, b, c, plan, hidden=True)
        return (h, *sol.adapters_backward(dy, x, h, a, b, c, plan, past))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(draw(10 + i, 130, 96))
        index.copy_(index_of(20 + i, 130, 4, "mixed"))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(kept, want))
