"""Refusals of the low-rank adapters' calls, without a GPU: the C-ABI's status
codes before any HIP call and the binding's ValueErrors; and the oracle against
torch's autograd in 64 bits."""
import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from test_operators_host import EALIGN, EINVAL, ESHAPE, EWORKSPACE, OK, Reached, T, apart, at, meta  # noqa: F401


def plan(index=apart(0), nb=4, tokens=40, adapters=3, p=apart(1), pb=1 << 20):
    return sol.lib.solfp4_adapter_plan(index, nb, tokens, adapters, p, pb, None)


def test_plan_refusals():
    need = sol.adapter_plan_bytes(40, 3)
    assert need >= 4 * 40 and need % 16 == 0 and sol.adapter_plan_bytes(0, 1) > 0
    assert sol.adapter_plan_bytes(-1, 3) == 0 == sol.adapter_plan_bytes(4, 0) == sol.adapter_plan_bytes(4, 65537)
    assert sol.adapter_plan_bytes(1 << 27, 1) == 0
    assert plan(tokens=-1) == EINVAL and plan(adapters=0) == EINVAL and plan(adapters=65537) == ESHAPE
    assert plan(tokens=1 << 27) == ESHAPE and plan(nb=2) == EINVAL and plan(index=None) == EINVAL and plan(p=None) == EINVAL
    assert plan(index=at(2)) == EALIGN and plan(index=at(4), nb=8) == EALIGN and plan(p=at(8)) == EALIGN
    assert plan(pb=need - 1) == EWORKSPACE and plan(p=apart(0)) == EINVAL


def forward(y=apart(0), ys=64, x=apart(1), xs=32, a=apart(2), b=apart(3), c=apart(4), E=3, p=apart(5), out=apart(6),
            os=64, h=apart(7), ws=apart(8), wsb=1 << 30, tokens=40, N=64, K=32, rank=8):
    return sol.lib.solfp4_add_adapters(y, ys, x, xs, a, b, c, E, p, out, os, h, ws, wsb, tokens, N, K, rank, None)


def test_forward_refusals():
    for bad in (dict(tokens=-1), dict(N=-1), dict(K=-1), dict(rank=0), dict(E=0), dict(y=None), dict(x=None), dict(a=None),
                dict(b=None), dict(out=None), dict(p=None), dict(ys=-1), dict(os=63), dict(os=0)):
        assert forward(**bad) == EINVAL, bad
    for bad in (dict(tokens=1 << 27), dict(N=1 << 22), dict(K=1 << 22), dict(rank=129), dict(E=65537), dict(xs=1 << 60)):
        assert forward(**bad) == ESHAPE, bad
    for bad in (dict(y=at(1)), dict(x=at(1)), dict(a=at(1)), dict(b=at(1)), dict(out=at(1)), dict(c=at(2)), dict(h=at(2)),
                dict(p=at(8))):
        assert forward(**bad) == EALIGN, bad
    # out over anything but y in place, hidden over anything
    for over in range(1, 6):
        assert forward(out=apart(over)) == EINVAL
    for over in range(0, 7):
        assert forward(h=apart(over)) == EINVAL
    assert forward(out=at(2)) == EINVAL and forward(out=apart(0), os=65) == EINVAL
    size = sol.add_adapters_workspace_bytes
    assert size(40, 3, True, 64, 32, 8) == 0 == size(40, 3, True, 64, 32, 129) == size(100000, 3, True, 64, 9728, 64)
    big = dict(K=9728, rank=64, xs=9728)
    need = size(40, 3, True, 64, 9728, 64)
    assert need > 0 and forward(ws=None, wsb=0, x=None) == EINVAL
    assert forward(ws=None, **big) == EWORKSPACE and forward(wsb=need - 1, **big) == EWORKSPACE
    assert forward(ws=at(8), **big) == EALIGN
    for over in range(0, 8):
        assert forward(ws=apart(over), **big) == EINVAL
    assert forward(tokens=0, x=None, y=None, out=None) == OK and forward(N=0, K=0, h=None, a=None, b=None) == OK


def back(dy=apart(0), x=apart(1), h=apart(2), a=apart(3), b=apart(4), c=apart(5), E=3, p=apart(6), past=apart(7),
         dx=apart(8), dxs=32, da=apart(9), db=apart(10), ws=apart(11), wsb=1 << 30, tokens=40, N=64, K=32, rank=8):
    return sol.lib.solfp4_adapters_backward(dy, 64, x, 32, h, a, b, c, E, p, past, 32, dx, dxs, da, db, ws, wsb, tokens, N,
                                            K, rank, None)


def test_backward_refusals():
    size = sol.adapters_backward_workspace_bytes
    need = size(40, 3, True, 64, 32, 8)
    assert need > 0 and size(40, 0, True, 64, 32, 8) == 0 == size(40, 3, True, 64, 32, 129) == size(40, 3, True, -1, 32, 8)
    assert size(26574, 2, True, 7296, 2432, 32) < 1 << 28
    for bad in (dict(tokens=-1), dict(rank=0), dict(E=0), dict(dy=None), dict(x=None), dict(h=None), dict(a=None),
                dict(b=None), dict(p=None), dict(dx=None), dict(da=None), dict(db=None), dict(dxs=31)):
        assert back(**bad) == EINVAL, bad
    assert back(rank=129) == ESHAPE and back(N=1 << 22) == ESHAPE
    for bad in (dict(dy=at(1)), dict(h=at(2)), dict(da=at(2)), dict(db=at(2)), dict(ws=at(8)), dict(past=at(1))):
        assert back(**bad) == EALIGN, bad
    assert back(ws=None) == EWORKSPACE and back(wsb=need - 1) == EWORKSPACE
    for over in range(0, 7):
        assert back(dx=apart(over)) == EINVAL
    for name in ("da", "db", "ws"):
        for over in range(0, 9):
            assert back(**{name: apart(over)}) == EINVAL, (name, over)
    assert back(da=apart(10)) == EINVAL and back(ws=apart(9)) == EINVAL and back(dx=at((7 << 32) + 2)) == EINVAL


def test_binding_refusals(meta, monkeypatch):  # noqa: F811
    y, x, a, b = T(40, 64), T(40, 32), T(3, 8, 32), T(3, 64, 8)
    f32 = torch.float32
    made = sol.AdapterPlan(40, 3, T(sol.adapter_plan_bytes(40, 3) // 4, dtype=torch.int32))
    with pytest.raises(Reached):
        sol.adapter_plan(T(40, dtype=torch.int64), 3)
    for bad in (T(40, dtype=torch.int16), T(40, 1, dtype=torch.int32), T(80, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            sol.adapter_plan(bad, 3)
    for adapters, given in ((0, None), (65537, None), (2, made), (3, 5)):
        with pytest.raises(ValueError):
            sol.adapter_plan(T(40, dtype=torch.int32), adapters, given)
    with pytest.raises(Reached):
        sol.add_adapters(y, x, a, b, None, made, hidden=True)
    with pytest.raises(Reached):
        sol.add_adapters(y, x, a[:1], b[:1])
    for bad in (dict(plan=None), dict(plan=made.buffer), dict(plan=sol.AdapterPlan(41, 3, made.buffer)),
                dict(plan=sol.AdapterPlan(40, 3, made.buffer[1:])), dict(scales=T(2, dtype=f32)), dict(scales=T(3)),
                dict(out=T(40, 63)), dict(hidden=T(40, 8)), dict(hidden=T(40, 9, dtype=f32)), dict(y=T(39, 64)),
                dict(x=T(40, 31)), dict(x=T(40, 32, dtype=torch.float16)), dict(a=T(3, 0, 32)), dict(a=T(3, 129, 32)),
                dict(b=T(3, 8, 64)), dict(b=T(2, 64, 8)), dict(a=T(3, 32, 8).transpose(1, 2)), dict(y=T(64, 40).t()),
                dict(x=3)):
        kw = dict(y=y, x=x, a=a, b=b, plan=made)
        kw.update(bad)
        with pytest.raises(ValueError):
            sol.add_adapters(**kw)
    h = T(40, 8, dtype=f32)
    with pytest.raises(Reached):
        sol.adapters_backward(y, x, h, a, b, None, made, x)
    for bad in (dict(hidden=T(40, 8)), dict(hidden=None), dict(past=T(40, 31)), dict(dx=T(40, 33)), dict(da=T(3, 8, 32)),
                dict(db=T(3, 8, 64, dtype=f32)), dict(plan=None), dict(workspace=T(16, dtype=torch.uint8))):
        kw = dict(dy=y, x=x, hidden=h, a=a, b=b, plan=made)
        kw.update(bad)
        with pytest.raises(ValueError):
            sol.adapters_backward(**kw)


def test_oracle_against_autograd_in_64_bits():
    g = torch.Generator().manual_seed(3)
    tokens, K, N, rank, adapters = 23, 9, 7, 3, 4
    x, a, b, past, dy = (torch.randn(*s, generator=g, dtype=torch.float64) for s in
                         ((tokens, K), (adapters, rank, K), (adapters, N, rank), (tokens, K), (tokens, N)))
    y, c = torch.randn(tokens, N, generator=g, dtype=torch.float64), torch.tensor([0.5, 1.0, 2.0, -1.0], dtype=torch.float64)
    index = torch.randint(-1, 3, (tokens,), generator=g)
    leaves = [t.clone().requires_grad_() for t in (x, a, b)]
    e = index.clamp(min=0)
    add = torch.einsum("tnr,trk,tk->tn", leaves[2][e], leaves[1][e], leaves[0]) * (c[e] * (index >= 0))[:, None]
    out, hidden, _, _ = R.add_adapters(y.numpy(), x.numpy(), a.numpy(), b.numpy(), c.numpy(), index.numpy())
    np.testing.assert_allclose(out, (y + add).detach().numpy(), rtol=1e-12, atol=1e-12)
    grads = torch.autograd.grad((add * dy).sum() + (leaves[0] * past).sum(), leaves)
    got = R.adapters_backward(dy.numpy(), x.numpy(), hidden, a.numpy(), b.numpy(), c.numpy(), index.numpy(), past.numpy())
    for v, want in zip(got[:3], grads):
        np.testing.assert_allclose(v, want.numpy(), rtol=1e-11, atol=1e-12)
