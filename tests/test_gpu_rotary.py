"""Rotary positions against float64, element by element: both layouts, every
type, part of the head, odd pair counts, packed QKV views, heads-first
buffers, in place, both position types and none, positions outside the table;
the transposed rotation; the table.

Bound: two products and their sum in FP32 (3 roundings of 2^-24 of the
products' magnitudes), then the type's unit roundoff."""
import math

import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
LAYOUTS = ["half", "interleaved"]


def f64(t):
    return t.detach().cpu().double().numpy()


def draw(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).to(device())


def make_table(rows, rotated):
    return sol.rotary_table(sol.rotary_frequencies(rotated), rows)


def check(got, t, table, at, layout, inverse, label=""):
    want, size = R.rotate(f64(t), f64(table), at, layout, inverse)
    u = UNIT[got.dtype]
    # copied elements are exact, rotated ones within the bound (the smallest
    # FP16 and BF16 numbers are half a step apart from 2^-25 on)
    bound = np.abs(want) * u + size * 2.0 ** -22 + 2.0 ** -24 * (got.dtype == torch.float16) + 1e-37
    bound[..., table.shape[1]:] = 0
    err = np.abs(f64(got) - want)
    assert np.all(err <= bound), (label, float(np.max(err - bound)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim,rotated", [(128, 128), (128, 80), (96, 32), (64, 64), (80, 44), (32, 2), (256, 250),
                                         (33, 18), (7, 6), (128, 0)])
def test_layouts_and_parts(dtype, layout, dim, rotated):
    T, H, G = 11, 6, 2
    table = make_table(40, rotated)
    qkv = draw(dim + rotated, T, H + 2 * G, dim, dtype=dtype)
    q, k = qkv[:, :H], qkv[:, H:H + G]
    before = qkv.clone()
    at = np.arange(T)
    for inverse in (False, True):
        a, b = sol.rotary(q, k, table, layout=layout, inverse=inverse)
        check(a, q, table, at, layout, inverse)
        check(b, k, table, at, layout, inverse)
    assert torch.equal(qkv, before)
    # in place in the packed buffer: the same, and v untouched
    c, d = sol.rotary(q, k, table, layout=layout, inverse=True, q_out=q, k_out=k)
    assert c is q and d is k and torch.equal(q, a) and torch.equal(k, b)
    assert torch.equal(qkv[:, H + G:], before[:, H + G:])
    # q alone
    e, none = sol.rotary(before[:, :H], None, table, layout=layout, inverse=True)
    assert none is None and torch.equal(e, a)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
@pytest.mark.parametrize("tokens", [0, 1, 2, 63, 1000])
def test_positions(layout, kind, tokens):
    table = make_table(300, 64)
    q, k = draw(1, tokens, 5, 64), draw(2, tokens, 1, 64)
    at = torch.randint(300, (tokens,), generator=torch.Generator().manual_seed(tokens), dtype=kind)
    a, b = sol.rotary(q, k, table, at.to(device()), layout)
    check(a, q, table, at.numpy(), layout, False)
    check(b, k, table, at.numpy(), layout, False)
    a, b = sol.rotary(q, k, table, None, layout)
    check(a, q, table, np.arange(tokens) % 300, layout, False, "sequences of the table's length")


def test_positions_outside_the_table():
    table = make_table(16, 32)
    q = draw(1, 6, 3, 48)
    for kind, bad in ((torch.int32, [3, -1, 16, 15, 2 ** 31 - 1, -2 ** 31]),
                      (torch.int64, [3, -1, 16, 15, 2 ** 40, -2 ** 62])):
        a, _ = sol.rotary(q, None, table, torch.tensor(bad, dtype=kind, device=device()))
        out = torch.tensor([1, 2, 4, 5], device=device())
        assert torch.all(torch.isnan(a[out][..., :32])) and torch.equal(a[out][..., 32:], q[out][..., 32:])
        for i in (0, 3):
            check(a[i:i + 1], q[i:i + 1], table, np.array([bad[i]]), "half", False)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_strides(layout):
    table = make_table(50, 40)
    T, H, D = 13, 4, 56
    at = np.arange(T)
    heads_first = draw(1, H, T, D).transpose(0, 1)
    odd = draw(2, T, H * 61 + 3)[:, 1:1 + H * 61].view(T, H, 61)[..., 2:2 + D]       # odd strides and offset
    out = draw(3, H, T, D + 5).transpose(0, 1)[..., :D]
    a, b = sol.rotary(heads_first, odd, table, layout=layout, q_out=out)
    assert a is out
    check(a, heads_first, table, at, layout, False)
    check(b, odd, table, at, layout, False)
    same = heads_first.clone(memory_format=torch.preserve_format)
    sol.rotary(same, None, table, layout=layout, q_out=same)
    assert torch.equal(same, a)
    # all heads read one (stride 0): the outputs are apart
    one = draw(4, T, 1, D).expand(T, H, D)
    a, _ = sol.rotary(one, None, table, layout=layout)
    check(a, one, table, at, layout, False)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_gradient(layout):
    """The transposed rotation is the gradient: <rotate(q), d> = <q,
    transposed(d)> for every q and d, and it undoes the rotation up to the
    magnitude's square."""
    f = sol.rotary_frequencies(48)
    table = sol.rotary_table(f, 30, magnitude=1.25)
    q, d = draw(1, 30, 3, 64, dtype=torch.float32), draw(2, 30, 3, 64, dtype=torch.float32)
    y, _ = sol.rotary(q, None, table, layout=layout)
    dq, _ = sol.rotary(d, None, table, layout=layout, inverse=True)
    left, right = float((y.double() * d.double()).sum()), float((q.double() * dq.double()).sum())
    size = float((y.double() * d.double()).abs().sum())
    assert abs(left - right) <= size * 2.0 ** -21
    back, _ = sol.rotary(y, None, table, layout=layout, inverse=True)
    assert torch.allclose(back[..., :48], 1.5625 * q[..., :48], rtol=0, atol=1e-5)
    # central differences of the float64 definition
    h = 1e-5
    t, w, tab = f64(q), f64(d), f64(table)
    rng = np.random.Generator(np.random.PCG64(3))
    e = rng.standard_normal(t.shape)
    at = np.arange(30)
    num = sum(s * np.sum(w * R.rotate(t + s * h * e, tab, at, layout)[0]) for s in (1, -1)) / (2 * h)
    assert abs(float(np.sum(f64(dq) * e)) - num) <= np.sum(np.abs(f64(dq) * e)) * 2.0 ** -20 + 1e-6


def test_table():
    """Angles in 64 bits: FP32 of cos and sin of the float64 angle, which is
    itself within 2^-53 of position x frequency (2^-21 at 2^31 radians)."""
    f = sol.rotary_frequencies(64, base=5e5)
    at = torch.tensor([0, 1, 77, 4607, 131071, 2 ** 31 - 1, -5], device=device())
    t = sol.rotary_table(f, at)
    ang = at.cpu().double()[:, None] * f
    want = torch.cat((ang.cos(), ang.sin()), 1)
    assert t.dtype == torch.float32 and float((t.cpu().double() - want).abs().max()) <= 2.0 ** -24 + 2.0 ** -40
    assert torch.equal(sol.rotary_table(f, 200), sol.rotary_table(f, torch.arange(200, device=device())))
    out = torch.empty(200, 64, device=device())
    assert sol.rotary_table(f, 200, magnitude=0.5, out=out) is out
    assert torch.equal(out, 0.5 * sol.rotary_table(f, 200))
    assert sol.rotary_table(f, 0).shape == (0, 64) and sol.rotary_table(f[:0], 5).shape == (5, 0)


def test_image_positions():
    """Three axes, as an image's tokens have: text row, image row, column."""
    f = torch.cat([sol.rotary_frequencies(n) for n in (16, 56, 56)])
    at = torch.randint(0, 64, (90, 3), generator=torch.Generator().manual_seed(1))
    t = sol.rotary_table(f, at.to(device()), axis_pairs=[8, 28, 28])
    axis = torch.tensor([0] * 8 + [1] * 28 + [2] * 28)
    ang = at[:, axis].double() * f
    assert float((t.cpu().double() - torch.cat((ang.cos(), ang.sin()), 1)).abs().max()) <= 2.0 ** -24


def test_frequencies():
    f = sol.rotary_frequencies(128)
    assert torch.equal(sol.rotary_frequencies(128, scaling="linear", factor=4.0), f / 4)
    b = sol.rotary_frequencies(128, scaling="base", factor=8.0)
    assert b[0] == f[0] and math.isclose(float(b[-1]), float(f[-1]) / 8, rel_tol=1e-12)
    p = sol.rotary_frequencies(128, scaling="by-parts", factor=8.0, original_length=4096)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(p[turns > 32], f[turns > 32]) and torch.allclose(p[turns < 1], f[turns < 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    assert bool(mid.any()) and bool(torch.all((p[mid] < f[mid]) & (p[mid] > f[mid] / 8)))


def test_large_and_graph():
    """More tokens than one round of workgroups, replayed from a graph."""
    table = make_table(512, 64)
    qkv = draw(7, 4096, 24, 64)
    q, k = qkv[:, :8], qkv[:, 8:16]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sol.rotary(q, k, table)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sol.rotary(q, k, table)
    for i in range(3):
        qkv.copy_(draw(20 + i, 4096, 24, 64))
        graph.replay()
        torch.cuda.synchronize()
        want = sol.rotary(q, k, table)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(got[0], q, table, np.arange(4096) % 512, "half", False)
    say("  4096 tokens, 16 heads: replays equal eager calls")
