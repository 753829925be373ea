"""The norm with the residual's addition and its backward pass against
float64, element by element: every type, with and without residual, gain and
groups, widths from 1 past every number of waves a row takes, strided and
misaligned rows, in place.

Bounds, fixed by the arithmetic: u is the unit roundoff of the type.  The
mean square of a row is a sum of at most 48 FP32 squares a lane, six steps
across the wave and eight waves, so rho is within (48 + 6 + 8) / 2 + 3 < 2^-18
(in units of 2^-24) relative; the products after it add 2^-23.  A gain's
gradient is a sum of FP32 terms, each within 2^-18, added in an order of at
most rows + 64 roundings."""
import numpy as np
import pytest
import torch

import oracle.nvfp4 as O
import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}
REL = 2.0 ** -18
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def f64(t):
    return t.detach().cpu().double().numpy()


def draw(seed, rows, width, dtype, scale=1.0, stride=None, offset=0):
    """[rows, width] on the GPU, rows `stride` apart, `offset` elements into its storage."""
    g = torch.Generator().manual_seed(seed)
    stride = stride or width
    flat = (scale * torch.randn(offset + max(rows, 1) * stride, generator=g)).to(dtype).to(device())
    return flat[offset:].as_strided((rows, width), (stride, 1), offset)


def check(got, want, rel, extra, dtype, label):
    got = f64(got)
    bound = np.abs(want) * (UNIT[dtype] + rel) + extra * (1 + UNIT[dtype]) + TINY[dtype]
    worst = float(np.max(np.abs(got - want) / bound)) if want.size else 0.0
    say(f"  {label}: worst |err| / bound {worst:.3f}")
    assert worst <= 1.0, label


WIDTHS = [1, 7, 8, 33, 512, 1152, 1235, 3073, 6144, 6151, 12289, 24576]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_forward(dtype, width):
    rows = 6
    x, r = draw(width, rows, width, dtype), draw(width + 1, rows, width, dtype, 3.0)
    g = (1 + draw(width + 2, 3, width, dtype, 0.3))
    s, y = R.add_rmsnorm(f64(x), f64(r), f64(g), 1e-5)
    out, total = sol.add_rmsnorm(x, r, g, 1e-5)
    check(total, s, 0.0, np.abs(s) * 2.0 ** -24, dtype, "sum")
    check(out, y, REL, 0.0, dtype, "norm")
    # without a residual or a gain
    s, y = R.add_rmsnorm(f64(x))
    out, total = sol.add_rmsnorm(x)
    assert total is None
    check(out, y, REL, 0.0, dtype, "plain norm")


@pytest.mark.parametrize("rows", [0, 1, 3, 5, 1000])
def test_row_counts_and_graph_of_groups(rows):
    for groups in {1, rows} - {0}:
        x = draw(rows, rows, 160, torch.bfloat16)
        g = draw(rows + 1, groups, 160, torch.bfloat16)
        out, _ = sol.add_rmsnorm(x, None, g)
        check(out, R.add_rmsnorm(f64(x), None, f64(g))[1], REL, 0.0, torch.bfloat16, f"{rows} rows, {groups} groups")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width,stride,offset", [(96, 101, 1), (1152, 3459, 3), (1235, 1235, 5), (40, 64, 0)])
def test_strides_alignment_and_in_place(dtype, width, stride, offset):
    rows = 9
    x, r = draw(1, rows, width, dtype, 1.0, stride, offset), draw(2, rows, width, dtype, 1.0, stride + 2, offset + 1)
    gains = draw(3, 3, 2 * width, dtype)[:, width:]           # every second vector of a modulation
    s, y = R.add_rmsnorm(f64(x), f64(r), f64(gains))
    out = draw(4, rows, width, dtype, 1.0, stride + 1, 1)
    keep = draw(4, 1, rows * (stride + 1) + 1, dtype)
    got, total = sol.add_rmsnorm(x, r, gains, out=out, sum_out=r)
    assert got is out and total is r
    check(got, y, REL, 0.0, dtype, "norm")
    check(r, s, 0.0, np.abs(s) * 2.0 ** -24, dtype, "sum in the residual's place")
    # nothing between the rows was touched
    whole = out.as_strided((1, rows * (stride + 1) + 1), (1, 1), 0)
    between = torch.ones(rows * (stride + 1) + 1, dtype=torch.bool)
    for i in range(rows):
        between[1 + i * (stride + 1): 1 + i * (stride + 1) + width] = False
    assert torch.equal(whole[0].cpu()[between], keep[0].cpu()[between])
    # the output in x's place
    y = R.add_rmsnorm(f64(x), None, f64(gains))[1]
    got, _ = sol.add_rmsnorm(x, None, gains, out=x)
    check(x, y, REL, 0.0, dtype, "norm in place")
    # one row for all (stride 0)
    one = draw(5, 1, width, dtype).expand(rows, width)
    out, total = sol.add_rmsnorm(r, one)
    check(out, R.add_rmsnorm(f64(r), f64(one))[1], REL, 0.0, dtype, "broadcast residual")


def decoded(codes, scales, kind):
    if kind == "mxfp8":
        return R.mxfp8_values(codes, scales)
    return O.mxfp4_unscaled_ref(codes, scales)


@pytest.mark.parametrize("kind", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [32, 96, 1152, 3072, 6176, 12288])
def test_quantized_output(kind, dtype, width):
    """Every block's scale and every code is that of a value within 2^-18
    (and the products' 2^-23) of the float64 one."""
    rows = 5
    x = draw(width, rows, width, dtype) * torch.exp2(torch.arange(rows, device=device()) - 2.0).to(dtype)[:, None]
    r = draw(width + 1, rows, width, dtype)
    x[:, :32] = 0                                              # a block of zeros, one of tiny values
    r[:, :32] = 0
    x[2, 32:64] *= 2.0 ** -12
    r[2, 32:64] *= 2.0 ** -12
    g = draw(width + 2, 1, width, dtype)[0]
    s, y = R.add_rmsnorm(f64(x), f64(r), f64(g))
    codes, scales, total = getattr(sol, f"{kind}_add_rmsnorm")(x, r, g)
    check(total, s, 0.0, np.abs(s) * 2.0 ** -24, dtype, "sum")
    c, sc = codes.cpu().numpy(), scales.cpu().numpy().astype(np.int64)
    emax, most = (8, 448.0) if kind == "mxfp8" else (2, 6.0)
    amax = np.abs(y).reshape(rows, -1, 32).max(2)
    d = 2.0 ** -17
    assert np.all((R.block_scale_bytes(amax * (1 - d), emax) <= sc) & (sc <= R.block_scale_bytes(amax * (1 + d), emax)))
    unit = np.repeat(np.exp2(sc - 127.0), 32, axis=1)
    got = decoded(c, scales.cpu().numpy(), kind) / unit
    table = R.E4M3 if kind == "mxfp8" else np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    mid = (table[1:] + table[:-1]) / 2

    def nearest(a, side):
        return table[np.searchsorted(mid, a, side=side)]
    a = np.abs(y) / unit
    low, high = nearest(a * (1 - d), "left"), nearest(a * (1 + d), "right")
    assert np.all((low <= np.abs(got)) & (np.abs(got) <= high) & (np.abs(got) <= most))
    assert np.all((got == 0) | (np.sign(got) == np.sign(y)))
    exact = float(np.mean(np.abs(got) == nearest(a, "left")))
    say(f"  {kind} {width}: {exact:.5f} of the codes are those of the float64 value")
    assert exact > 0.999


def test_mxfp4_output_feeds_the_gemm():
    x = draw(1, 70, 256, torch.bfloat16)
    w = draw(2, 48, 256, torch.bfloat16)
    wq = sol.mxfp4_quantize(w)
    codes, scales, _ = sol.mxfp4_add_rmsnorm(x)
    out = sol.mxfp4_gemm(codes, scales, *wq)
    want = O.mxfp4_gemm_ref(codes.cpu().numpy(), scales.cpu().numpy(), *(t.cpu().numpy() for t in wq))
    assert np.linalg.norm(f64(out) - want) <= 2e-3 * np.linalg.norm(want)


def test_special_values():
    for dtype in TYPES:
        x = draw(1, 6, 64, dtype)
        x[0] = 0
        x[1, 5] = float("nan")
        x[2, 7] = float("inf")
        x[3] = torch.finfo(dtype).tiny
        out, _ = sol.add_rmsnorm(x)
        assert torch.all(out[0] == 0) and torch.all(torch.isnan(out[1])) and torch.isnan(out[2, 7])
        assert torch.all(out[2, :7] == 0)
        check(out[3:], R.add_rmsnorm(f64(x[3:]))[1], REL, 0.0, dtype, "the smallest normal numbers")
        codes, _, _ = sol.mxfp8_add_rmsnorm(x)
        assert torch.all(codes[0] == 0) and torch.all((codes[1] & 127) == 127)
        # eps = 0 on a row of zeros: 0 times infinity
        assert torch.all(torch.isnan(sol.add_rmsnorm(x[:1], eps=0.0)[0]))


def test_residual_cancels():
    x = draw(3, 4, 128, torch.float32)
    out, total = sol.add_rmsnorm(x, -x)
    assert torch.all(out == 0) and torch.all(total == 0)


# ---- backward -------------------------------------------------------------

def check_backward(dy, s, g, dsum, dtype, eps=1e-5, **kw):
    ds, dg, size, terms = R.rmsnorm_backward(f64(dy), f64(s), None if g is None else f64(g),
                                             None if dsum is None else f64(dsum), eps)
    want_extra = size * REL + (0 if dsum is None else (np.abs(f64(dsum)) + size) * 2.0 ** -23)
    dx, dgain = sol.rmsnorm_backward(dy, s, g, dsum, eps, **kw)
    check(dx, ds, 0.0, want_extra, dtype, "dx")
    if g is None:
        assert dgain is None
        return dx
    assert dgain.dtype == torch.float32 and dgain.shape == g.shape
    bound = terms * (REL + (s.shape[0] + 64) * 2.0 ** -24) + 1e-30
    worst = float(np.max(np.abs(f64(dgain).reshape(dg.shape) - dg) / bound)) if dg.size else 0.0
    say(f"  dgain: worst |err| / bound {worst:.3f}")
    assert worst <= 1.0
    return dx


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_backward(dtype, width):
    rows = 12
    dy, s, dsum = (draw(width + i, rows, width, dtype) for i in range(3))
    check_backward(dy, s, 1 + draw(width + 3, 3, width, dtype, 0.3), dsum, dtype)
    check_backward(dy, s, draw(width + 3, 1, width, dtype)[0], None, dtype)
    check_backward(dy, s, None, dsum, dtype)


@pytest.mark.parametrize("rows,groups", [(1, 1), (2, 2), (9, 3), (777, 1), (5000, 1), (6000, 6), (600, 600)])
def test_backward_rows_and_groups(rows, groups):
    dy, s = draw(rows, rows, 104, torch.bfloat16), draw(rows + 1, rows, 104, torch.bfloat16)
    check_backward(dy, s, draw(rows + 2, groups, 104, torch.bfloat16), None, torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_strides_and_in_place(dtype):
    rows, width = 10, 131
    dy, s = draw(1, rows, width, dtype, 1.0, 140, 3), draw(2, rows, width, dtype, 1.0, 133, 1)
    dsum = draw(3, rows, width, dtype, 1.0, 150, 1)
    g = draw(4, 2, 3 * width, dtype)[:, width:2 * width]
    a = check_backward(dy, s, g, dsum, dtype)
    for place in (dsum, dy):
        d, ds_ = dy.clone(), dsum.clone()
        dx, _ = sol.rmsnorm_backward(dy, s, g, dsum, 1e-5, dx=place)
        assert dx is place and torch.equal(dx, a)
        dy.copy_(d)
        dsum.copy_(ds_)


def test_backward_without_rows():
    e = torch.empty(0, 96, dtype=torch.bfloat16, device=device())
    dx, dg = sol.rmsnorm_backward(e, e, torch.ones(2, 96, dtype=torch.bfloat16, device=device()))
    assert dx.shape == (0, 96) and torch.all(dg == 0)


def test_same_results_on_every_call_and_any_stream():
    dy, s, g = (draw(i, 3000, 1152, torch.bfloat16) for i in range(3))
    g = g[:4]
    a = sol.rmsnorm_backward(dy, s, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = sol.rmsnorm_backward(dy, s, g, stream=side)
    n = sol.add_rmsnorm(dy, s, g, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    m = sol.add_rmsnorm(dy, s, g)
    assert all(torch.equal(x, y) for x, y in zip(a + m, b + n))


def test_gradient_against_differences():
    """<dx, d> and <dgain, e> against central differences of the float64
    definition: step 1e-5, error of the difference about 1e-9 relative, of
    the FP32 gradient 2^-17 of the terms' magnitudes."""
    rng = np.random.Generator(np.random.PCG64(5))
    rows, width = 7, 201
    x, r, w = (rng.standard_normal((rows, width)).astype(np.float32) for _ in range(3))
    g = rng.standard_normal((1, width)).astype(np.float32)
    a = [torch.from_numpy(t).to(device()) for t in (x, r, w, g)]
    _, total = sol.add_rmsnorm(a[0], a[1], a[3], 1e-3)
    dx, dg = sol.rmsnorm_backward(a[2], total, a[3], None, 1e-3)

    def loss(x, r, g):
        return float(np.sum(w.astype(np.float64) * R.add_rmsnorm(x, r, g, 1e-3)[1]))
    h = 1e-5
    x, r, g = (t.astype(np.float64) for t in (x, r, g))
    for _ in range(4):
        d, e = rng.standard_normal(x.shape), rng.standard_normal(g.shape)
        for got, num, dirn in ((dx, loss(x + h * d, r, g) - loss(x - h * d, r, g), d),
                               (dx, loss(x, r + h * d, g) - loss(x, r - h * d, g), d),
                               (dg, loss(x, r, g + h * e) - loss(x, r, g - h * e), e)):
            size = float(np.sum(np.abs(f64(got) * dirn)))
            assert abs(float(np.sum(f64(got) * dirn)) - num / (2 * h)) <= size * 2.0 ** -16 + 1e-6


def test_graph_replay():
    x, r, g = draw(1, 200, 1152, torch.bfloat16), draw(2, 200, 1152, torch.bfloat16), draw(3, 4, 1152, torch.bfloat16)
    dy = draw(4, 200, 1152, torch.bfloat16)

    def step():
        y, s = sol.add_rmsnorm(x, r, g)
        c = sol.mxfp8_add_rmsnorm(x, r, g)
        return (y, s, *c, *sol.rmsnorm_backward(dy, s, g))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        x.copy_(draw(10 + i, 200, 1152, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


# ---- rows that share a wave -----------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 5, 8, 9, 16, 31, 32, 64, 65, 96, 128, 200, 255, 256, 257])
@pytest.mark.parametrize("rows", [1, 63, 64, 1030])
def test_narrow_rows(dtype, width, rows):
    """As few lanes a row as hold it: every lane count, rows that fill no
    workgroup, one NaN row among them."""
    x, r, dy = (draw(width + i, rows, width, dtype) for i in range(3))
    g = 1 + draw(width + 3, 1, width, dtype, 0.3)[0]
    s, y = R.add_rmsnorm(f64(x), f64(r), f64(g))
    out, total = sol.add_rmsnorm(x, r, g)
    check(out, y, REL, 0.0, dtype, "norm")
    check(total, s, 0.0, np.abs(s) * 2.0 ** -24, dtype, "sum")
    check_backward(dy, x, g, r, dtype)
    check_backward(dy, x, None, None, dtype)
    if rows > 1:
        x[rows // 2, width // 2] = float("nan")
        bad, _ = sol.add_rmsnorm(x, r, g)
        keep = [i for i in range(rows) if i != rows // 2]
        assert torch.equal(bad[keep], out[keep]) and torch.all(torch.isnan(bad[rows // 2]))
    if width % 32 == 0 and rows > 1:
        c = sol.mxfp8_add_rmsnorm(x[:rows // 2], r[:rows // 2], g)
        assert np.linalg.norm(R.mxfp8_values(c[0].cpu().numpy(), c[1].cpu().numpy()) - y[:rows // 2]) <= \
            2.0 ** -4 * np.linalg.norm(y[:rows // 2])


@pytest.mark.parametrize("rows,groups,width", [(4, 1, 12000), (33, 1, 4000), (64, 2, 136), (256, 1, 128), (257, 1, 128),
                                               (8192, 4, 128), (96, 96, 40)])
def test_backward_one_and_several_workgroups(rows, groups, width):
    """Around the largest row count that one workgroup takes alone."""
    for dtype in TYPES:
        dy, s = draw(rows, rows, width, dtype), draw(rows + 1, rows, width, dtype)
        check_backward(dy, s, draw(rows + 2, groups, width, dtype), None, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1000, 2100, 4101, 9000, 16390, 20480, 22528])
def test_widths_between(dtype, width):
    """Widths at which a lane holds one to six runs of a row on one to eight waves."""
    rows = 9
    x, r = draw(width, rows, width, dtype), draw(width + 1, rows, width, dtype)
    g = draw(width + 2, 3, width, dtype)
    s, y = R.add_rmsnorm(f64(x), f64(r), f64(g))
    out, total = sol.add_rmsnorm(x, r, g)
    check(total, s, 0.0, np.abs(s) * 2.0 ** -24, dtype, "sum")
    check(out, y, REL, 0.0, dtype, "norm")
    check_backward(x, r, g, total, dtype)


@pytest.mark.parametrize("kind", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [992, 4128, 9024, 16416, 20480, 24576])
def test_quantized_widths_between(kind, dtype, width):
    test_quantized_output(kind, dtype, width)


@pytest.mark.parametrize("rows,groups", [(9000, 1), (12000, 3), (70000, 1), (72000, 6)])
def test_backward_many_rows(rows, groups):
    """One round of workgroups a compute unit, and two."""
    dy, s = draw(rows, rows, 104, torch.bfloat16), draw(rows + 1, rows, 104, torch.bfloat16)
    check_backward(dy, s, draw(rows + 2, groups, 104, torch.bfloat16), None, torch.bfloat16)
