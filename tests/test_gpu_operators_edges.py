"""Edges of the operators around the linears on the GPU: operands and values
that the tests of the single operators do not reach."""
import numpy as np
import pytest
import torch

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
