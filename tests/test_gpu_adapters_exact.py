"""Low-rank adapters where every sum is exact in FP32, so that results are the
definition's to the last bit: h and g have 24 bits and all of them reach what
is formed from them; infinite weights; gradients of tokens taken in runs.

With x = (p, q, r, 0 ..) of whole numbers p from 128 to 254, q and r up to 255,
rank element 0 holds h = p + q 2^-8 + r 2^-16, which fills FP32's 24 bits; two
others hold -p and -q 2^-8.  b takes all three once: r 2^-16 is left, 8 bits that
BF16 holds.  Any order of the sums is exact: all values are multiples of 2^-16
below 2^8."""
import pytest
import torch

import paper_2604_06916_amd as sol
from gpu_util import device
from test_gpu_adapted_maxsize import check_adapters

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def parts(seed, tokens, width, places):
    """[tokens, width] with p, q, r in three columns, and r 2^-16."""
    g = torch.Generator().manual_seed(seed)
    v = torch.zeros(tokens, width)
    for at, (lo, hi) in zip(places, ((128, 255), (0, 256), (0, 256))):
        v[:, at] = torch.randint(lo, hi, (tokens,), generator=g).float()
    return v.to(BF16).to(device()), (v[:, places[2]] * 2.0 ** -16).to(device())


def columns(rank, width, places, all_of):
    """(w [rank, width] that gives h, -p, -q 2^-8 from those columns, b's row)."""
    w, row = torch.zeros(rank, width), torch.zeros(rank)
    for i, at in enumerate(places):
        w[all_of[0], at] = 2.0 ** (-8 * i)
    w[all_of[1], places[0]], w[all_of[2], places[1]] = -1.0, -2.0 ** -8
    row[list(all_of)] = 1.0
    return w.to(BF16).to(device()), row.to(BF16).to(device())


def index_of(tokens, adapters):
    g = torch.Generator().manual_seed(tokens)
    return torch.randint(0, adapters, (tokens,), generator=g, dtype=torch.int32).to(device())


@pytest.mark.parametrize("tokens,K,N,rank,adapters", [
    (1, 3, 1, 3, 1), (5, 40, 70, 8, 2), (70, 200, 131, 24, 3), (33, 64, 128, 32, 2), (300, 90, 64, 33, 5), (64, 100, 200, 64, 1),
    (40, 300, 200, 100, 3), (50, 129, 333, 128, 2), (12000, 16, 24, 32, 2), (20000, 24, 40, 64, 1), (15000, 9, 16, 128, 3),
    (9, 9000, 40, 32, 2), (35, 5000, 70, 128, 3)])
def test_all_bits_of_h_reach_the_output(tokens, K, N, rank, adapters):
    places, ranks = (0, K // 2, K - 1), (0, rank - 1, rank // 2)
    x, left = parts(tokens, tokens, K, places)
    w, row = columns(rank, K, places, ranks)
    a, b = w.expand(adapters, rank, K).contiguous(), row.expand(adapters, N, rank).contiguous()
    plan = None if adapters == 1 else sol.adapter_plan(index_of(tokens, adapters), adapters)
    y = torch.zeros(tokens, N, dtype=BF16, device=device())
    out, hidden = sol.add_adapters(y, x, a, b, None, plan, hidden=True)
    assert torch.equal(hidden, x.float() @ w.float().t())
    assert torch.equal(out.float(), left[:, None].expand(tokens, N))


@pytest.mark.parametrize("tokens,K,N,rank,adapters", [
    (1, 1, 3, 3, 1), (5, 70, 40, 8, 2), (70, 131, 200, 24, 3), (33, 128, 64, 32, 2), (300, 64, 90, 33, 5), (64, 200, 100, 64, 1),
    (40, 200, 300, 100, 3), (50, 333, 1129, 128, 2), (12000, 24, 16, 32, 2), (20000, 40, 24, 64, 1), (15000, 16, 9, 128, 3)])
def test_all_bits_of_g_reach_dx(tokens, K, N, rank, adapters):
    places, ranks = (0, N // 2, N - 1), (0, rank - 1, rank // 2)
    dy, left = parts(tokens, tokens, N, places)
    w, row = columns(rank, N, places, ranks)
    b = w.t().contiguous().expand(adapters, N, rank).contiguous()
    a = row[:, None].expand(adapters, rank, K).contiguous()
    plan = None if adapters == 1 else sol.adapter_plan(index_of(tokens, adapters), adapters)
    x, hidden = torch.zeros(tokens, K, dtype=BF16, device=device()), torch.zeros(tokens, rank, device=device())
    dx, da, db = sol.adapters_backward(dy, x, hidden, a, b, None, plan)
    assert torch.equal(dx.float(), left[:, None].expand(tokens, K)) and not da.any() and not db.any()


@pytest.mark.parametrize("tokens,K,N,rank", [(1, 1, 1, 1), (7, 40, 33, 8), (90, 65, 130, 24), (40, 200, 64, 64), (33, 72, 96, 128)])
def test_all_bits_of_g_and_h_reach_da_and_db(tokens, K, N, rank):
    """A token an adapter.  b is 1 in each column's own rank element, dy and x are 1, the scale fills 24
    bits: g is the number of a rank element's columns times the scale, here one column or none."""
    g = torch.Generator().manual_seed(tokens)
    b = torch.zeros(tokens, N, rank)
    n = min(N, rank)
    b[:, torch.arange(n), torch.arange(n)] = 1.0
    scales = (torch.randint(2 ** 23, 2 ** 24, (tokens,), generator=g).float() * 2.0 ** -23).to(device())
    hidden = (torch.randint(-2 ** 24, 2 ** 24, (tokens, rank), generator=g).float() * 2.0 ** -20).to(device())
    a = torch.zeros(tokens, rank, K, dtype=BF16, device=device())
    dy, x = torch.ones(tokens, N, dtype=BF16, device=device()), torch.ones(tokens, K, dtype=BF16, device=device())
    index = torch.randperm(tokens, generator=g).int().to(device())
    plan = sol.adapter_plan(index, tokens)
    _, da, db = sol.adapters_backward(dy, x, hidden, a, b.to(BF16).to(device()), scales, plan)
    want = torch.zeros(tokens, rank, K, device=device())
    want[:, :n] = scales[:, None, None]
    assert torch.equal(da, want)
    _, _, db = sol.adapters_backward(dy, x, hidden, a, b.to(BF16).to(device()), None, plan)
    assert torch.equal(db[index.long()], hidden[:, None].expand(tokens, N, rank))


@pytest.mark.parametrize("rank", [1, 4, 8, 12, 24, 40, 72, 128])
@pytest.mark.parametrize("tokens", [3, 40])
def test_an_infinite_weight_is_met_once(rank, tokens):
    """b's last rank element is infinite: the output is what the definition gives, an infinity of
    h's sign, where all pieces of h have that sign (here positive: p, q and r below 128)."""
    K, N = 70, 50
    x = torch.zeros(tokens, K)
    x[:, :3] = torch.tensor([255.0, 3.0, 5.0])
    a = torch.zeros(1, rank, K)
    a[:, -1, :3] = torch.tensor([1.0, 2.0 ** -8, 2.0 ** -16])
    b = torch.zeros(1, N, rank)
    b[:, ::2, -1] = float("inf")
    b[:, 1::4, -1] = -float("inf")
    y = torch.ones(tokens, N, dtype=BF16, device=device())
    out, hidden = sol.add_adapters(y, *(t.to(BF16).to(device()) for t in (x, a, b)), hidden=True)
    want = (1 + b[:, :, -1]).expand(tokens, N).to(device())
    assert torch.equal(out.float(), want)
    assert torch.equal(hidden[:, -1].cpu(), torch.full((tokens,), 255 + 3 * 2.0 ** -8 + 5 * 2.0 ** -16))


@pytest.mark.parametrize("rank", [8, 24, 32, 40, 128])
@pytest.mark.parametrize("tokens", [2, 50, 12000])
def test_weights_at_any_address(rank, tokens):
    """a and b at odd elements of their memory give what aligned ones give."""
    K, N = 66, 75
    g = torch.Generator().manual_seed(rank)
    room = [torch.randn(n, generator=g).to(BF16).to(device()) for n in (rank * K + 1, N * rank + 1)]
    a, b = room[0][1:].view(1, rank, K), room[1][1:].view(1, N, rank)
    x, y = (torch.randn(tokens, w, generator=g).to(BF16).to(device()) for w in (K, N))
    want = sol.add_adapters(y, x, a.clone(), b.clone(), hidden=True)
    got = sol.add_adapters(y, x, a, b, hidden=True)
    assert a.data_ptr() % 4 == b.data_ptr() % 4 == 2 and all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("tokens,K,N,rank,adapters,sparse", [(70000, 64, 2048, 128, 3, 64), (1300000, 40, 72, 8, 7, 4),
                                                             (600000, 33, 129, 40, 2, 8)])
def test_gradients_of_tokens_in_several_runs(tokens, K, N, rank, adapters, sparse):
    """So many that g's shares take more than a run of tiles holds: sums over runs that end inside an
    adapter's tiles, adapters of one run alone, tokens without one in the last."""
    size = sol.adapters_backward_workspace_bytes
    assert size(tokens, adapters, True, N, K, rank) < size(tokens // 4, adapters, True, N, K, rank) * 2
    check_adapters(tokens, K, N, rank, adapters, sparse, exact=True)


def test_runs_in_a_graph_and_in_place():
    tokens, K, N, rank, adapters = 70000, 64, 2048, 128, 3
    g = torch.Generator(device=device()).manual_seed(3)
    normal = lambda *s: torch.randn(*s, generator=g, device=device()).to(BF16)
    dy, x, past = normal(tokens, N), normal(tokens, K), normal(tokens, K)
    a, b, hidden = normal(adapters, rank, K), normal(adapters, N, rank), normal(tokens, rank).float()
    plan = sol.adapter_plan(index_of(tokens, adapters), adapters)
    dx = past.clone()
    call = lambda: sol.adapters_backward(dy, x, hidden, a, b, None, plan, dx, dx=dx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        dy.copy_(normal(tokens, N))
        dx.copy_(past)
        graph.replay()
        torch.cuda.synchronize()
        want = sol.adapters_backward(dy, x, hidden, a, b, None, plan, past)
        torch.cuda.synchronize()
        assert held[0] is dx and all(torch.equal(p, q) for p, q in zip(held, want))
