"""Edges of the operators around the linears on the GPU: operands and values
that the tests of the single operators do not reach."""
import numpy as np
import pytest
import torch

import oracle.nvfp4 as O
import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def f64(t):
    return t.detach().cpu().double().numpy()


# ---- the table's frequencies ----------------------------------------------

@pytest.mark.parametrize("view", [lambda f: f[::2], lambda f: f[7:8].expand(24), lambda f: f.flip(0)[1::3]])
def test_table_of_strided_frequencies(view):
    """A view of device frequencies gives the table of its values."""
    f = view(sol.rotary_frequencies(96).to(device()))
    assert torch.equal(sol.rotary_table(f, 40), sol.rotary_table(f.cpu().clone(), 40))


# ---- packed buffers -------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("order", [(0, 2, 1, 3), (0, 1, 2, 3), (1, 0, 2, 3), (2, 1, 0, 3)])
def test_rotary_in_place_in_packed_buffers(dtype, layout, order):
    """q, k and v of one buffer in every order of tokens, heads and the three:
    turned in place as out of place, v untouched."""
    T, H, D, rotated = 9, 5, 56, 36
    t = torch.randn(T, 3, H, D, generator=torch.Generator().manual_seed(3)).to(dtype).to(device())
    # a buffer laid out in this order, seen as [tokens, 3, heads, dim]
    t = t.permute(order).contiguous().permute([order.index(i) for i in range(4)])
    q, k, v = (t[:, i] for i in range(3))
    keep = v.clone()
    table = sol.rotary_table(sol.rotary_frequencies(rotated), 20)
    want = sol.rotary(q.contiguous(), k.contiguous(), table, layout=layout)
    out = torch.empty_like(t)
    got = sol.rotary(q, k, table, layout=layout, q_out=out[:, 0], k_out=out[:, 1])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    sol.rotary(q, k, table, layout=layout, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, keep)


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_in_columns_of_one_buffer(dtype):
    """Operands and outputs that are columns of one buffer: as with buffers of
    their own, and the columns beside them untouched."""
    rows, width = 37, 150
    g = torch.Generator().manual_seed(4)
    t = torch.randn(rows, 5, width, generator=g).to(dtype).to(device())
    x, r, total, out, other = (t[:, i] for i in range(5))
    gain = torch.randn(1, width, generator=g).to(dtype).to(device())
    keep = t.clone()
    y, s = sol.add_rmsnorm(x.contiguous(), r.contiguous(), gain)
    sol.add_rmsnorm(x, r, gain, out=out, sum_out=total)
    assert torch.equal(out, y) and torch.equal(total, s)
    assert torch.equal(x, keep[:, 0]) and torch.equal(r, keep[:, 1]) and torch.equal(other, keep[:, 4])
    dx, dgain = sol.rmsnorm_backward(x.contiguous(), s, gain, r.contiguous())
    got, got_gain = sol.rmsnorm_backward(x, total, gain, r, dx=out)
    assert got is out and torch.equal(out, dx) and torch.equal(got_gain, dgain) and torch.equal(other, keep[:, 4])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [24, 1152, 6151])
def test_gradient_in_the_place_of_x(dtype, width):
    g = torch.Generator().manual_seed(width)
    dy, x, gain = (torch.randn(n, width, generator=g).to(dtype).to(device()) for n in (50, 50, 2))
    dx, dgain = sol.rmsnorm_backward(dy, x, gain)
    got, again = sol.rmsnorm_backward(dy, x, gain, dx=x)
    assert got is x and torch.equal(x, dx) and torch.equal(again, dgain)


# ---- gradients with eps = 0 -----------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,groups,width", [(1, 1, 1152), (1, 1, 24), (9, 3, 200), (5, 1, 6151), (101, 1, 104),
                                               (4429, 1, 2432), (8858, 2, 96), (3001, 1, 12000)])
def test_gradients_without_eps(dtype, rows, groups, width):
    """eps = 0 and no row of zeros: the slots of a workgroup that have no row
    add nothing, whether the group's sums are one workgroup's or several's.

    dx: REL 2^-18 of the magnitudes it is formed from, and the type's
    rounding; dgain: that of its terms and a rounding a row."""
    g = torch.Generator().manual_seed(rows + width)
    dy, s, gain = (torch.randn(n, width, generator=g).to(dtype).to(device()) for n in (rows, rows, groups))
    dx, dgain = sol.rmsnorm_backward(dy, s, gain, eps=0.0)
    want, want_gain, size, terms = R.rmsnorm_backward(f64(dy), f64(s), f64(gain), None, 0.0)
    unit = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]
    tiny = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}[dtype]
    assert np.all(np.abs(f64(dx) - want) <= np.abs(want) * unit + size * 2.0 ** -18 * (1 + unit) + tiny)
    assert np.all(np.abs(f64(dgain) - want_gain) <= terms * (2.0 ** -18 + (rows + 64) * 2.0 ** -24) + 1e-30)


@pytest.mark.parametrize("rows", [3, 700])
def test_gradients_of_a_zero_row_without_eps(rows):
    """0 times infinity is the row's own: its dx and its group's dgain are NaN, no other's."""
    g = torch.Generator().manual_seed(rows)
    dy, s, gain = (torch.randn(n, 72, generator=g).to(device()) for n in (2 * rows, 2 * rows, 2))
    s[1] = 0
    dx, dgain = sol.rmsnorm_backward(dy, s, gain, eps=0.0)
    keep = torch.arange(2 * rows, device=device()) != 1
    assert torch.all(torch.isnan(dx[1])) and torch.all(torch.isfinite(dx[keep]))
    assert torch.all(torch.isnan(dgain[0])) and torch.all(torch.isfinite(dgain[1]))


# ---- infinities and the range of the quantized norms ----------------------

def quantized(kind, x, **kw):
    """(decoded values, scale bytes, codes) of the norm of x."""
    codes, scales, _ = getattr(sol, f"{kind}_add_rmsnorm")(x, **kw)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    return (R.mxfp8_values(c, s) if kind == "mxfp8" else O.mxfp4_unscaled_ref(c, s)), s.astype(np.int64), c


@pytest.mark.parametrize("kind", ["same", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_with_an_infinity(kind, dtype):
    """rho = 0: the infinite elements are NaN and the finite ones 0, in every form of the output."""
    g = torch.Generator().manual_seed(8)
    x = torch.randn(4, 320, generator=g).to(dtype).to(device())
    x[1, 70] = float("inf")
    x[2, 5] = float("-inf")
    x[2, 319] = float("inf")
    finite = torch.isfinite(x).cpu().numpy()
    if kind == "same":
        y = f64(sol.add_rmsnorm(x)[0])
        assert np.all(np.isnan(y[~finite])) and np.all(y[1:3][finite[1:3]] == 0)
        return
    y, scales, codes = quantized(kind, x)
    assert np.all(y[1:3][finite[1:3]] == 0)
    if kind == "mxfp8":
        assert np.all((codes[~finite] & 127) == 127)
    blocks = finite.reshape(4, -1, 32).all(2)
    assert np.all(scales[1:3][blocks[1:3]] == 0)
    # the rows beside them are as they are alone
    alone, s, _ = quantized(kind, x[[0, 3]])
    assert np.array_equal(y[[0, 3]], alone) and np.array_equal(scales[[0, 3]], s)


@pytest.mark.parametrize("kind", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e-36, 1e-30, 1e-22, 1e-19, 1e-10, 1e10, 1e18, 1e20, 1e30, 1e36])
def test_quantized_norm_of_large_and_small_rows(kind, dtype, size):
    """The squares and rho are formed in 64 bits: rows between 2^-126 and 2^126
    give what rows of 1 give.  Scales as in the definition (amax within 2^-17),
    elements within half a step of theirs."""
    g = torch.Generator().manual_seed(9)
    x = (size * torch.randn(5, 160, generator=g)).to(dtype).to(device())
    want = R.add_rmsnorm(f64(x), None, None, 0.0)[1]
    got, scales, _ = quantized(kind, x, eps=0.0)
    emax, most, step, least = (8, 448.0, 2.0 ** -4, 2.0 ** -10) if kind == "mxfp8" else (2, 6.0, 0.25, 0.25)
    amax, d = np.abs(want).reshape(5, -1, 32).max(2), 2.0 ** -17
    assert np.all((R.block_scale_bytes(amax * (1 - d), emax) <= scales) & (scales <= R.block_scale_bytes(amax * (1 + d), emax)))
    unit = np.repeat(np.exp2(scales - 127.0), 32, axis=1)
    v = np.clip(want / unit, -most, most)
    assert np.all(np.abs(got / unit - v) <= np.abs(v) * (step + d) + least)


# ---- allocations ----------------------------------------------------------

def allocating_calls():
    x = torch.randn(32, 64, generator=torch.Generator().manual_seed(1)).bfloat16().to(device())
    w = sol.nvfp4_quantize(x)
    m = sol.mxfp4_quantize(x)
    table = sol.rotary_table(sol.rotary_frequencies(16), 32)
    heads = x.view(32, 4, 16)
    m8 = sol.mxfp8_add_rmsnorm(x)[:2]
    return {"nvfp4_quantize": lambda: sol.nvfp4_quantize(x), "mxfp4_quantize": lambda: sol.mxfp4_quantize(x),
            "nvfp4_gemm": lambda: sol.nvfp4_gemm(*w, *w), "mxfp4_gemm": lambda: sol.mxfp4_gemm(*m, *m),
            "nvfp4_linear": lambda: sol.nvfp4_linear(x, *w), "mxfp4_linear": lambda: sol.mxfp4_linear(x, *m),
            "add_rmsnorm": lambda: sol.add_rmsnorm(x, x), "mxfp4_add_rmsnorm": lambda: sol.mxfp4_add_rmsnorm(x),
            "rmsnorm_backward": lambda: sol.rmsnorm_backward(x, x, x[0]), "rotary": lambda: sol.rotary(heads, heads, table),
            "nvfp4_weight_linear": lambda: sol.nvfp4_weight_linear(x, *w),
            "mxfp8_linear": lambda: sol.mxfp8_linear(*m8, *m)}


def test_allocations_are_seen_by_dispatch_modes():
    """Outputs and workspaces that a call allocates go through torch's
    dispatcher while a mode looks on, and hold the same results."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Seen(TorchDispatchMode):
        def __init__(self):
            super().__init__()
            self.empties = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            self.empties += "empty" in str(func)
            return func(*args, **(kwargs or {}))
    for name, call in allocating_calls().items():
        want = call()
        with Seen() as seen:
            got = call()
        assert seen.empties > 0, name
        pairs = zip(want, got) if isinstance(want, tuple) else [(want, got)]
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in pairs), name


def test_results_with_deterministic_algorithms():
    calls = allocating_calls()
    want = {name: call() for name, call in calls.items()}
    torch.use_deterministic_algorithms(True)
    try:
        got = {name: call() for name, call in calls.items()}
    finally:
        torch.use_deterministic_algorithms(False)
    for name in calls:
        pairs = zip(want[name], got[name]) if isinstance(want[name], tuple) else [(want[name], got[name])]
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in pairs), name
