"""Low-rank adapters beside a linear against float64, element by element:
plans of every kind, sizes around the tiles' edges, every rank's shape, strided
and misaligned rows, in place, tokens without an adapter and past the last.

Bounds, in units of E = 2^-24: a hidden value is an FP32 sum of K exact products
in some order, K + 16 roundings at most; it enters the second product as two
BF16 pieces, within 2^-18 of it; that product's FP32 sums round at most 2 rank +
8 times; then one multiply-add and the rounding to BF16 (2^-8 covers it with a
step into the next binade)."""
import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
BF16 = torch.bfloat16


def f64(t):
    return t.detach().cpu().double().numpy()


def draw(seed, *shape, scale=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).to(device())


def weights(seed, adapters, rank, K, N):
    return (draw(seed, adapters, rank, K, scale=max(K, 1) ** -0.5), draw(seed + 1, adapters, N, rank, scale=0.3),
            torch.linspace(0.5, 2.0, adapters).to(device()))


def index_of(seed, tokens, adapters, kind, dtype=torch.int32):
    rng = np.random.default_rng(seed)
    if kind == "mixed":
        i = rng.integers(-1, adapters, tokens)
    elif kind == "blocks":
        i = np.sort(rng.integers(0, 7, tokens)) * 5 % adapters
    elif kind == "distinct":
        i = rng.permutation(max(tokens, adapters))[:tokens] % adapters
    else:
        i = rng.integers(-3, adapters + 2, tokens)     # past the last adapter, too
    return torch.from_numpy(i).to(dtype).to(device())


def close(got, want, bound, label):
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), label
    ok = ~np.isnan(want)
    worst = float(np.max(np.abs(got - want)[ok] / bound[ok])) if ok.any() else 0.0
    say(f"  {label}: worst |err| / bound {worst:.3f}")
    assert worst <= 1.0, label


def check_forward(y, x, a, b, scales, index, plan, **kw):
    at = np.zeros(x.shape[0], np.int64) if index is None else index.cpu().numpy()
    c = np.ones(a.shape[0]) if scales is None else f64(scales)
    out, hid, size, hid_size = R.add_adapters(f64(y), f64(x), f64(a), f64(b), c, at)
    K, rank = a.shape[2], a.shape[1]
    y64 = f64(y)
    got, hidden = sol.add_adapters(y, x, a, b, scales, plan, hidden=True, **kw)
    close(hidden, hid, hid_size * (K + 16) * E + 1e-38, "hidden")
    close(got, out, np.abs(out) * 2.0 ** -8 + size * ((K + 2 * rank + 32) * E + 2.0 ** -18) + np.abs(y64) * E + 1e-38, "out")
    return got, hidden


# ---- the plan -------------------------------------------------------------

def plan_ref(index, adapters):
    """The layout that the kernels read: first tiles, first places, tokens, tiles."""
    g = np.where(index < 0, adapters, np.minimum(index, adapters + 1))
    g = np.where((index >= adapters), adapters + 1, g).astype(np.int64)
    groups = adapters + 2
    counts = np.bincount(g, minlength=groups)
    places = np.concatenate(([0], np.cumsum(counts)))
    tiles_of = -(-counts // 32)
    first = np.concatenate(([0], np.cumsum(tiles_of)))
    tiles = [(e, places[e] + 32 * i, min(32, counts[e] - 32 * i)) for e in range(groups) for i in range(tiles_of[e])]
    return first, places, np.argsort(g, kind="stable"), tiles


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("tokens,adapters,kind", [(1, 1, "mixed"), (5, 3, "any"), (33, 1, "any"), (64, 48, "distinct"),
                                                  (1371, 5, "any"), (8192, 2, "blocks"), (20001, 7, "any"),
                                                  (700, 1500, "any"), (26574, 64, "mixed"), (9, 3000, "distinct")])
def test_plan(dtype, tokens, adapters, kind):
    index = index_of(tokens, tokens, adapters, kind, dtype)
    plan = sol.adapter_plan(index, adapters)
    first, places, order, tiles = plan_ref(index.cpu().numpy().astype(np.int64), adapters)
    p = plan.buffer.cpu().numpy()
    heads = (adapters + 3 + 3) // 4 * 4
    assert np.array_equal(p[:adapters + 3], first) and np.array_equal(p[heads:heads + adapters + 3], places)
    assert np.array_equal(p[2 * heads:2 * heads + tokens], order)
    rest = p[2 * heads + (tokens + 3) // 4 * 4:].reshape(-1, 4)
    assert np.array_equal(rest[:len(tiles), :3], np.array(tiles).reshape(-1, 3)) and np.all(rest[len(tiles):, 2] == 0)


def test_plan_of_no_tokens_and_written_again():
    empty = sol.adapter_plan(torch.empty(0, dtype=torch.int32, device=device()), 3)
    assert torch.all(empty.buffer[:6] == 0)
    a, b, c = weights(1, 3, 8, 16, 24)
    out, hidden = sol.add_adapters(draw(1, 0, 24), draw(2, 0, 16), a, b, c, empty, hidden=True)
    assert out.shape == (0, 24) and hidden.shape == (0, 8)
    one, two = index_of(1, 50, 3, "any"), index_of(2, 50, 3, "any")
    plan = sol.adapter_plan(one, 3)
    assert sol.adapter_plan(two, 3, plan) is plan
    n = 2 * 8 + 50
    assert torch.equal(plan.buffer[:n], sol.adapter_plan(two, 3).buffer[:n])


# ---- forward --------------------------------------------------------------

@pytest.mark.parametrize("rank", [1, 3, 8, 16, 24, 32, 33, 64, 100, 128])
@pytest.mark.parametrize("tokens", [1, 16, 17, 33])
def test_ranks(tokens, rank):
    K, N, adapters = 200, 131, 4
    a, b, c = weights(rank, adapters, rank, K, N)
    index = index_of(rank, tokens, adapters, "any")
    check_forward(draw(1, tokens, N), draw(2, tokens, K), a, b, c, index, sol.adapter_plan(index, adapters))


@pytest.mark.parametrize("tokens,K,N", [(1, 1, 1), (2, 7, 7), (15, 8, 16), (31, 31, 63), (32, 64, 64), (33, 65, 65),
                                        (100, 1152, 1152), (257, 1235, 1111), (1371, 520, 9), (4000, 96, 200),
                                        (30000, 40, 72)])
def test_sizes(tokens, K, N):
    for rank, adapters, kind in ((24, 5, "mixed"), (8, 3, "blocks")):
        a, b, c = weights(K, adapters, rank, K, N)
        index = index_of(tokens, tokens, adapters, kind, torch.int64)
        check_forward(draw(1, tokens, N), draw(2, tokens, K), a, b, c, index, sol.adapter_plan(index, adapters))
    a, b, _ = weights(N, 1, 20, K, N)
    check_forward(draw(3, tokens, N), draw(4, tokens, K), a, b, None, None, None)


@pytest.mark.parametrize("tokens,adapters,K,N", [(64, 48, 2432, 7296), (200, 200, 1152, 1152), (9, 3000, 64, 64)])
def test_an_adapter_a_token(tokens, adapters, K, N):
    a, b, c = weights(tokens, adapters, 32 if adapters < 1000 else 8, K, N)
    index = index_of(5, tokens, adapters, "distinct")
    check_forward(draw(1, tokens, N), draw(2, tokens, K), a, b, c, index, sol.adapter_plan(index, adapters))


@pytest.mark.parametrize("tokens,K,N,rank", [(1, 9728, 640, 64), (70, 9001, 130, 33), (40, 2432, 200, 128),
                                             (300, 4000, 64, 100), (9, 100000, 40, 24)])
def test_wide_adapters(tokens, K, N, rank):
    """a of 2^18 elements or more: h is formed by several workgroups in a launch of its own."""
    adapters = 3
    a, b, c = weights(tokens, adapters, rank, K, N)
    index = index_of(tokens, tokens, adapters, "any")
    plan = sol.adapter_plan(index, adapters)
    x, y = draw(1, tokens, K), draw(2, tokens, N)
    out, _ = check_forward(y, x, a, b, c, index, plan)
    need = sol.add_adapters_workspace_bytes(tokens, adapters, True, N, K, rank)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=device())
    assert need and torch.equal(sol.add_adapters(y, x, a, b, c, plan, workspace=ws)[0].nan_to_num(7.0), out.nan_to_num(7.0))


@pytest.mark.parametrize("offset", [0, 1, 3])
def test_strides_in_place_and_what_lies_between(offset):
    """The k part of a packed QKV buffer, in place, from columns of a wider x."""
    tokens, K, N, adapters = 77, 90, 64, 3
    wide = draw(1, tokens, 2 * K + offset)
    qkv = draw(2, tokens, 3 * N + offset)
    x, y = wide[:, offset:offset + K], qkv[:, N + offset:2 * N + offset]
    a, b, c = weights(3, adapters, 16, K, N)
    index = index_of(4, tokens, adapters, "mixed")
    plan = sol.adapter_plan(index, adapters)
    want, _ = sol.add_adapters(y, x, a, b, c, plan)
    before = qkv.clone()
    got, _ = check_forward(y, x, a, b, c, index, plan, out=y)
    assert got is y and torch.equal(y, want)
    before[:, N + offset:2 * N + offset] = want
    assert torch.equal(qkv, before)
    # into rows of another buffer, between which nothing is written
    room = draw(5, tokens, 100)
    keep = room.clone()
    y.copy_(draw(6, tokens, N))
    sol.add_adapters(y, x, a, b, c, plan, out=room[:, 7:7 + N])
    keep[:, 7:7 + N] = sol.add_adapters(y, x, a, b, c, plan)[0]
    assert torch.equal(room, keep)
    # one row of x and of y for all tokens
    check_forward(y[:1].expand(tokens, N), x[:1].expand(tokens, K), a, b, c, index, plan)


def test_tokens_without_an_adapter_keep_their_y():
    tokens, K, N = 70, 64, 80
    a, b, c = weights(1, 2, 8, K, N)
    index = torch.full((tokens,), -1, dtype=torch.int32, device=device())
    index[5], index[66] = 1, 9
    x, y = draw(2, tokens, K), draw(3, tokens, N)
    x[3] = float("nan")
    plan = sol.adapter_plan(index, 2)
    out, hidden = sol.add_adapters(y, x, a, b, c, plan, hidden=True)
    none = torch.ones(tokens, dtype=torch.bool, device=device())
    none[5] = none[66] = False
    assert torch.equal(out[none], y[none]) and torch.all(hidden[none] == 0)
    assert torch.all(torch.isnan(out[66])) and torch.all(torch.isnan(hidden[66]))
    assert not torch.equal(out[5], y[5]) and torch.all(torch.isfinite(out[5]))
    kept = y.clone()
    sol.add_adapters(y, x, a, b, c, plan, out=y)
    assert torch.equal(y[none], kept[none]) and torch.equal(y[5], out[5])


def test_values_that_are_not_finite_stay_with_their_token():
    tokens, K, N = 40, 72, 50
    a, b, _ = weights(1, 1, 12, K, N)
    x, y = draw(2, tokens, K), draw(3, tokens, N)
    want, _ = sol.add_adapters(y, x, a, b)
    x[7, 3], y[9, 4] = float("nan"), float("inf")
    x[11] = 0
    x[11, 0] = float("inf")
    out, hidden = sol.add_adapters(y, x, a, b, hidden=True)
    others = torch.ones(tokens, dtype=torch.bool, device=device())
    others[[7, 9, 11]] = False
    assert torch.equal(out[others], want[others]) and torch.all(torch.isnan(out[7])) and torch.isinf(out[9, 4])
    # an infinite h: infinite or NaN as in any order of its products, no finite value
    assert torch.all(torch.isinf(hidden[11])) and not torch.any(torch.isfinite(out[11]))


def test_features_of_length_zero():
    a, b, c = weights(1, 2, 8, 0, 24)
    index = index_of(1, 10, 2, "mixed")
    plan = sol.adapter_plan(index, 2)
    y = draw(1, 10, 24)
    out, hidden = sol.add_adapters(y, draw(2, 10, 0), a, b, c, plan, hidden=True)
    assert torch.equal(out, y) and torch.all(hidden == 0)
    a, b, c = weights(1, 2, 8, 24, 0)
    x = draw(2, 10, 24)
    out, hidden = sol.add_adapters(draw(1, 10, 0), x, a, b, c, plan, hidden=True)
    want = R.add_adapters(np.zeros((10, 0)), f64(x), f64(a), f64(b), f64(c), index.cpu().numpy())
    assert out.shape == (10, 0)
    close(hidden, want[1], want[3] * 40 * E + 1e-38, "hidden")


def test_same_results_on_every_call_and_any_stream():
    tokens, K, N, adapters = 3000, 320, 448, 6
    a, b, c = weights(1, adapters, 32, K, N)
    index = index_of(2, tokens, adapters, "mixed")
    x, y = draw(3, tokens, K), draw(4, tokens, N)
    want = sol.add_adapters(y, x, a, b, c, sol.adapter_plan(index, adapters), hidden=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plan = sol.adapter_plan(index, adapters, stream=side)
    got = sol.add_adapters(y, x, a, b, c, plan, hidden=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_graph_replay_with_a_plan_written_again():
    tokens, K, N, adapters = 130, 96, 160, 4
    a, b, c = weights(1, adapters, 16, K, N)
    x, y, index = draw(2, tokens, K), draw(3, tokens, N), index_of(4, tokens, adapters, "any")
    plan = sol.adapter_plan(index, adapters)

    def step():
        sol.adapter_plan(index, adapters, plan)
        return sol.add_adapters(y, x, a, b, c, plan, hidden=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(draw(10 + i, tokens, K))
        index.copy_(index_of(20 + i, tokens, adapters, "any"))
        graph.replay()
        want = sol.add_adapters(y, x, a, b, c, sol.adapter_plan(index, adapters), hidden=True)
        torch.cuda.synchronize()
        assert all(torch.equal(p.nan_to_num(7.0), q.nan_to_num(7.0)) for p, q in zip(held, want))


@pytest.mark.parametrize("fill", ["zeros", "any"])
def test_plan_that_is_not_written_yet(fill):
    """The memory of a plan that only a graph has written so far may hold anything: what the calls give is
    undefined, but nothing outside their outputs is written and every kernel ends."""
    tokens, adapters, K, N, rank = 300, 5, 200, 130, 16
    x, y, dy = draw(1, tokens, K), draw(2, tokens, N), draw(3, tokens, N)
    a, b, c = weights(4, adapters, rank, K, N)
    plan = sol.adapter_plan(index_of(6, tokens, adapters, "any"), adapters)
    g = torch.Generator().manual_seed(7)
    n = plan.buffer.numel()
    plan.buffer.copy_(torch.randint(-2 ** 31, 2 ** 31, (n,), generator=g) if fill == "any" else torch.zeros(n))
    room, dx_room = (torch.full((tokens + 2, w + 8), 3.0, dtype=BF16, device=device()) for w in (N, K))
    out, dx = room[1:-1, 4:-4], dx_room[1:-1, 4:-4]
    say(f"  plan of {fill}")
    _, hidden = sol.add_adapters(y, x, a, b, c, plan, hidden=True, out=out)
    hidden.zero_()
    _, da, db = sol.adapters_backward(dy, x, hidden, a, b, c, plan, dx=dx)
    torch.cuda.synchronize()
    for whole in (room, dx_room):
        edges = whole.clone()
        edges[1:-1, 4:-4] = 3.0
        assert bool((edges == 3.0).all())
    if fill == "zeros":   # no token has a tile
        assert bool((out == 3.0).all()) and bool((dx == 3.0).all()) and not da.any() and not db.any()
