"""Refusals of the layer norm's calls, without a GPU: the C-ABI's status codes
before any HIP call and the binding's ValueErrors; and the oracle against
torch's definition in 64 bits."""
import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from test_operators_host import EALIGN, EINVAL, ESHAPE, EWORKSPACE, OK, Reached, T, apart, at, meta  # noqa: F401


def norm(type=0, x=apart(0), xs=64, r=apart(1), rs=64, g=apart(2), gs=64, t=apart(5), ts=64, groups=1, eps=1e-6,
         s=apart(3), ss=64, out=apart(4), os=64, rows=4, width=64):
    return sol.lib.solfp4_add_layernorm(type, x, xs, r, rs, g, gs, t, ts, groups, eps, s, ss, out, os, rows, width, None)


def qnorm(fn, type=0, x=apart(0), g=None, t=None, codes=apart(4), scales=apart(5), rows=4, width=64, groups=1):
    return fn(type, x, 64, None, 0, g, 64, t, 64, groups, 1e-6, None, 0, codes, scales, rows, width, None)


def test_norm_refusals():
    assert norm(type=3) == EINVAL and norm(type=-1) == EINVAL
    assert norm(rows=-1) == EINVAL and norm(width=-1) == EINVAL and norm(rows=1 << 31) == ESHAPE
    assert norm(width=24577) == ESHAPE and norm(groups=0) == EINVAL and norm(groups=3) == ESHAPE
    assert norm(eps=-1.0) == EINVAL and norm(eps=float("nan")) == EINVAL
    assert norm(x=None) == EINVAL and norm(s=None) == EINVAL and norm(out=None) == EINVAL
    assert norm(t=at(1)) == EALIGN and norm(type=2, t=at(2)) == EALIGN and norm(ts=-1) == EINVAL
    assert norm(ts=1 << 60, groups=4) == ESHAPE
    # what is written over the shift, the gain, the residual or the sum
    assert norm(t=apart(4)) == EINVAL and norm(t=apart(3)) == EINVAL and norm(g=apart(4)) == EINVAL
    assert norm(out=apart(1)) == EINVAL and norm(out=apart(3)) == EINVAL and norm(s=at(64)) == EINVAL
    assert norm(rows=0, x=None) == OK and norm(width=0, x=None) == OK
    for fn in (sol.lib.mxfp8_add_layernorm, sol.lib.mxfp4_add_layernorm):
        assert qnorm(fn, width=48) == ESHAPE and qnorm(fn, codes=None) == EINVAL
        assert qnorm(fn, scales=at(8)) == EALIGN and qnorm(fn, type=9) == EINVAL
        assert qnorm(fn, t=apart(4)) == EINVAL and qnorm(fn, t=apart(5)) == EINVAL
        assert qnorm(fn, rows=0, x=None, codes=None, scales=None) == OK


def back(type=0, dy=apart(0), x=apart(1), g=apart(2), groups=1, ds=apart(3), dx=apart(4), dxs=64, dg=apart(5),
         dt=apart(7), ws=apart(6), wsb=1 << 20, rows=4, width=64, eps=1e-6):
    return sol.lib.solfp4_layernorm_backward(type, dy, 64, x, 64, g, 64, groups, ds, 64, eps, dx, dxs, dg, dt, ws, wsb,
                                             rows, width, None)


def test_backward_refusals():
    need = sol.layernorm_backward_workspace_bytes(4, 64, 1)
    assert need == 2 * sol.rmsnorm_backward_workspace_bytes(4, 64, 1)
    assert sol.layernorm_backward_workspace_bytes(4, 64, 3) == 0 == sol.layernorm_backward_workspace_bytes(0, 64, 1)
    assert back(type=7) == EINVAL and back(rows=-2) == EINVAL and back(width=1 << 15) == ESHAPE
    assert back(groups=3) == ESHAPE and back(groups=0) == EINVAL and back(rows=65536, groups=65536) == ESHAPE
    assert back(dy=None) == EINVAL and back(x=None) == EINVAL and back(dx=None) == EINVAL
    assert back(dx=at(64)) == EINVAL and back(dxs=32) == EINVAL and back(eps=-1.0) == EINVAL
    assert back(ws=None) == EWORKSPACE and back(wsb=need - 1) == EWORKSPACE and back(ws=at(8)) == EALIGN
    assert back(dg=None, ws=None) == EWORKSPACE and back(dg=None, wsb=need // 2 - 1) == EWORKSPACE
    assert back(dg=at(2)) == EALIGN and back(dt=at(2)) == EALIGN
    # the outputs over each other, over what is read, over the workspace
    for over in (apart(5), apart(4), apart(0), apart(1), apart(2), apart(3), apart(6)):
        assert back(dt=over) == EINVAL
    assert back(dt=apart(5), rows=0) == EINVAL


def test_binding_refusals(meta):  # noqa: F811
    x, g = T(8, 64), T(2, 64)
    with pytest.raises(Reached):
        sol.add_layernorm(x, x, g, g)
    for bad in (dict(shift=T(3, 64)), dict(shift=T(64), gain=g), dict(gain=g, shift=T(4, 64)), dict(shift=T(2, 63)),
                dict(shift=T(2, 64, dtype=torch.float32)), dict(shift=3.0), dict(eps=-1.0), dict(sum_out=x),
                dict(shift=T(64, 2).t()), dict(gain=T(3, 64)), dict(out=T(8, 63))):
        with pytest.raises(ValueError):
            sol.add_layernorm(x, **bad)
    for fn in (sol.mxfp8_add_layernorm, sol.mxfp4_add_layernorm):
        with pytest.raises(ValueError):
            fn(T(8, 48))
        with pytest.raises(ValueError):
            fn(x, codes=T(8, 64))
    with pytest.raises(Reached):
        sol.layernorm_backward(x, x, None, g)
    for bad in (dict(dgain=T(64, dtype=torch.float32)), dict(dshift=T(64, dtype=torch.float32)),
                dict(shift=g, dshift=T(2, 64)), dict(gain=g, shift=T(64)), dict(dsum=T(8, 63)), dict(eps=float("nan")),
                dict(gain=g, workspace=T(1, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            sol.layernorm_backward(x, x, **bad)


def test_oracle_against_torch_in_64_bits():
    g = torch.Generator().manual_seed(3)
    x, r, w, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((6, 33), (6, 33), (33,), (33,)))
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    y = torch.nn.functional.layer_norm(leaves[0] + r, (33,), leaves[1], leaves[2], 1e-3)
    s, want, _ = R.add_layernorm(x.numpy(), r.numpy(), w.numpy(), b.numpy(), 1e-3)
    np.testing.assert_allclose(y.detach().numpy(), want, rtol=1e-12, atol=1e-12)
    dy, past = torch.randn(6, 33, generator=g, dtype=torch.float64), torch.randn(6, 33, generator=g, dtype=torch.float64)
    grads = torch.autograd.grad((y * dy).sum() + (past * leaves[0]).sum(), leaves)
    ds, dg, dt, *_ = R.layernorm_backward(dy.numpy(), s, w.numpy(), 1, past.numpy(), 1e-3)
    for got, expect in zip((ds, dg[0], dt[0]), grads):
        np.testing.assert_allclose(got, expect.numpy(), rtol=1e-11, atol=1e-12)
