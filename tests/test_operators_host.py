"""Refusals of the operators around the linears, without a GPU: the C-ABI's
status codes before any HIP call, and the binding's ValueErrors (on torch's
meta device, the call stopped where it would pick its stream); and the
oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import oracle.nvfp4 as O
import oracle.operators as R
import paper_2604_06916_amd as sol
from paper_2604_06916_amd import _binding as B

OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE = 0, -1, -2, -3, -4


def at(n):
    return ctypes.c_void_p(0x7F0000000000 + n)


def apart(i):
    return at(i << 32)


def norm(type=0, x=apart(0), xs=64, r=apart(1), rs=64, g=apart(2), gs=64, groups=1, eps=1e-6, s=apart(3), ss=64,
         out=apart(4), os=64, rows=4, width=64):
    return sol.lib.solfp4_add_rmsnorm(type, x, xs, r, rs, g, gs, groups, eps, s, ss, out, os, rows, width, None)


def qnorm(fn, type=0, x=apart(0), g=None, codes=apart(4), scales=apart(5), rows=4, width=64, groups=1):
    return fn(type, x, 64, None, 0, g, 64, groups, 1e-6, None, 0, codes, scales, rows, width, None)


def test_norm_refusals():
    assert norm(type=3) == EINVAL and norm(type=-1) == EINVAL
    assert norm(rows=-1) == EINVAL and norm(width=-1) == EINVAL and norm(rows=1 << 31) == ESHAPE
    assert norm(width=24577) == ESHAPE
    assert norm(groups=0) == EINVAL and norm(groups=3) == ESHAPE
    assert norm(eps=-1.0) == EINVAL and norm(eps=float("nan")) == EINVAL
    assert norm(x=None) == EINVAL and norm(s=None) == EINVAL and norm(out=None) == EINVAL
    assert norm(x=at(1)) == EALIGN and norm(type=2, g=at(2)) == EALIGN
    assert norm(xs=-64) == EINVAL and norm(os=63) == EINVAL and norm(ss=1) == EINVAL
    assert norm(xs=1 << 60) == ESHAPE
    # the output over the residual or the sum; the sum shifted against x
    assert norm(out=apart(1)) == EINVAL and norm(out=apart(3)) == EINVAL
    assert norm(s=at(64)) == EINVAL
    assert norm(rows=0, x=None) == OK and norm(width=0, x=None) == OK
    for fn in (sol.lib.mxfp8_add_rmsnorm, sol.lib.mxfp4_add_rmsnorm):
        assert qnorm(fn, width=48) == ESHAPE and qnorm(fn, codes=None) == EINVAL
        assert qnorm(fn, scales=at(8)) == EALIGN and qnorm(fn, type=9) == EINVAL
        assert qnorm(fn, rows=0, x=None, codes=None, scales=None) == OK


def back(type=0, dy=apart(0), x=apart(1), g=apart(2), groups=1, ds=apart(3), dx=apart(4), dxs=64, dg=apart(5),
         ws=apart(6), wsb=1 << 20, rows=4, width=64, eps=1e-6):
    return sol.lib.solfp4_rmsnorm_backward(type, dy, 64, x, 64, g, 64, groups, ds, 64, eps, dx, dxs, dg, ws, wsb,
                                           rows, width, None)


def test_backward_refusals():
    need = sol.rmsnorm_backward_workspace_bytes(4, 64, 1)
    assert need >= 64 * 4 and sol.rmsnorm_backward_workspace_bytes(4, 64, 3) == 0
    assert sol.rmsnorm_backward_workspace_bytes(0, 64, 1) == 0
    assert back(type=7) == EINVAL and back(rows=-2) == EINVAL and back(width=1 << 15) == ESHAPE
    assert back(groups=3) == ESHAPE and back(groups=0) == EINVAL and back(rows=65536, groups=65536) == ESHAPE
    assert back(dy=None) == EINVAL and back(x=None) == EINVAL and back(dx=None) == EINVAL
    assert back(dx=at(64)) == EINVAL and back(dxs=32) == EINVAL and back(eps=-1.0) == EINVAL
    assert back(ws=None) == EWORKSPACE and back(wsb=need - 1) == EWORKSPACE and back(ws=at(8)) == EALIGN
    assert back(dg=at(2)) == EALIGN


def rot(type=0, layout=0, q=apart(0), qt=512, qh=128, qo=apart(1), qot=512, qoh=128, H=4, k=None, kt=0, kh=0, ko=None,
        kot=0, koh=0, G=0, table=apart(8), rows=16, pos=None, pb=0, tokens=4, dim=128, rotated=128):
    return sol.lib.solfp4_rotary(type, layout, 0, q, qt, qh, qo, qot, qoh, H, k, kt, kh, ko, kot, koh, G, table, rows,
                                 pos, pb, tokens, dim, rotated, None)


def test_rotary_refusals():
    assert rot(type=5) == EINVAL and rot(layout=2) == EINVAL
    assert rot(rotated=3) == ESHAPE and rot(rotated=130) == ESHAPE and rot(rotated=-2) == EINVAL
    assert rot(tokens=-1) == EINVAL and rot(H=-1) == EINVAL
    assert rot(q=None) == EINVAL and rot(qo=None) == EINVAL and rot(table=None) == EINVAL and rot(rows=0) == EINVAL
    assert rot(pos=apart(9)) == EINVAL and rot(pos=apart(9), pb=2) == EINVAL and rot(pb=4) == EINVAL
    assert rot(q=at(1)) == EALIGN and rot(table=at(2)) == EALIGN and rot(pos=at(4), pb=8) == EALIGN
    assert rot(qt=-1) == EINVAL and rot(qt=1 << 62) == ESHAPE
    # output heads on top of each other; an output shifted against its input, or over the other operand
    assert rot(qoh=64) == EINVAL and rot(qot=400) == EINVAL
    assert rot(qo=at(256)) == EINVAL
    assert rot(k=apart(1), kt=512, kh=128, ko=apart(3), kot=512, koh=128, G=4) == EINVAL
    assert rot(tokens=0, q=None) == OK and rot(H=0, q=None) == OK


def test_rotary_table_refusals():
    def table(pos=None, rows=8, f=apart(1), pairs=16, counts=None, axes=1, out=apart(2)):
        c = None if counts is None else (ctypes.c_int64 * len(counts))(*counts)
        return sol.lib.solfp4_rotary_table(pos, rows, f, pairs, c, axes, 1.0, out, None)
    assert table(rows=-1) == EINVAL and table(axes=0) == EINVAL and table(axes=2) == EINVAL
    assert table(pos=apart(3), axes=5, counts=[4] * 5) == ESHAPE
    assert table(pos=apart(3), axes=2, counts=[4, 4]) == ESHAPE and table(pos=apart(3), axes=2, counts=[20, 4]) == ESHAPE
    assert table(pos=apart(3), axes=2, counts=[-4, 20]) == EINVAL
    assert table(f=None) == EINVAL and table(out=None) == EINVAL and table(f=at(4)) == EALIGN
    assert table(rows=0, f=None, out=None) == OK


@pytest.mark.parametrize("kind", ["nvfp4", "mxfp4", "mxfp8"])
def test_weight_linear_refusals(kind):
    def call(x=apart(0), xs=apart(1), wc=apart(2), ws=apart(3), wg=apart(4), bias=None, out=apart(5), M=4, N=8, K=64):
        if kind == "nvfp4":
            return sol.lib.nvfp4_weight_linear(x, wc, ws, wg, bias, out, M, N, K, None)
        if kind == "mxfp4":
            return sol.lib.mxfp4_weight_linear(x, wc, ws, bias, out, M, N, K, None)
        return sol.lib.mxfp8_linear(x, xs, wc, ws, bias, out, M, N, K, None)
    assert call(M=-1) == EINVAL and call(N=-1) == EINVAL and call(K=-32) == EINVAL
    assert call(K=40) == ESHAPE and call(K=1 << 24) == ESHAPE and call(N=1 << 22) == ESHAPE and call(M=1 << 31) == ESHAPE
    assert call(x=None) == EINVAL and call(wc=None) == EINVAL and call(ws=None) == EINVAL and call(out=None) == EINVAL
    assert call(x=at(8)) == EALIGN and call(out=at(2)) == EALIGN and call(bias=at(2)) == EALIGN
    assert call(M=0, out=None, x=None) == OK and call(N=0, out=None) == OK
    if kind == "nvfp4":
        assert call(wg=None) == EINVAL and call(K=16, x=None) == EINVAL
    else:
        assert call(K=16) == ESHAPE
    if kind == "mxfp8":
        assert call(xs=None) == EINVAL and call(xs=at(4)) == EALIGN


def test_gain_over_what_is_written_is_refused():
    assert norm(g=apart(4)) == EINVAL and norm(g=apart(3)) == EINVAL and back(g=apart(4)) == EINVAL
    assert norm(g=at((4 << 32) + 2 * 64 * 3)) == EINVAL


# ---- the binding ----------------------------------------------------------

class Reached(Exception):
    pass


@pytest.fixture()
def meta(monkeypatch):
    monkeypatch.setattr(B, "_is_gpu", lambda t: t.device.type == "meta")

    def stop(stream, device):
        raise Reached()
    monkeypatch.setattr(B, "_stream", stop)


def T(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")


def test_binding_norm(meta):
    x = T(6, 64)
    for good in (dict(), dict(residual=T(6, 64), gain=T(64)), dict(gain=T(3, 64)), dict(gain=T(2, 128)[:, 64:]),
                 dict(residual=T(6, 100)[:, 3:67], sum_out=T(6, 64))):
        with pytest.raises(Reached):
            sol.add_rmsnorm(x, **good)
        with pytest.raises(Reached):
            sol.mxfp8_add_rmsnorm(x, **good)
    for bad in (dict(residual=T(6, 63)), dict(residual=T(6, 64, dtype=torch.float16)), dict(gain=T(4, 64)),
                dict(gain=T(63)), dict(gain=T(64, dtype=torch.float32)), dict(gain=T(1, 1, 64)), dict(eps=-1.0),
                dict(sum_out=T(6, 64)), dict(residual=T(64, 6).t()), dict(residual=torch.zeros(6, 64).bfloat16()),
                dict(gain=3), dict(residual=T(5, 64))):
        with pytest.raises(ValueError):
            sol.add_rmsnorm(x, **bad)
        with pytest.raises(ValueError):
            sol.mxfp4_add_rmsnorm(x, **bad)
    for bad in (T(6, 64, dtype=torch.float64), T(64), "x", T(64, 6).t()):
        with pytest.raises(ValueError):
            sol.add_rmsnorm(bad)
    with pytest.raises(ValueError):
        sol.mxfp8_add_rmsnorm(T(6, 48))
    with pytest.raises(ValueError):
        sol.mxfp8_add_rmsnorm(x, codes=T(6, 32, dtype=torch.uint8))
    with pytest.raises(ValueError):
        sol.add_rmsnorm(x, out=T(6, 65))


def test_binding_backward(meta):
    x = T(6, 64)
    with pytest.raises(Reached):
        sol.rmsnorm_backward(x, x, T(2, 64), x)
    for args, kw in (((T(6, 63), x), {}), ((x, x, T(4, 64)), {}), ((x, x, None), dict(dgain=T(64, dtype=torch.float32))),
                     ((x, x, T(64)), dict(dgain=T(64))), ((x, x, None, T(5, 64)), {}), ((x, x), dict(dx=T(6, 60))),
                     ((x, x, T(64)), dict(workspace=T(4, dtype=torch.uint8))), ((x, x), dict(eps=-1.0)), ((x, 3), {})):
        with pytest.raises(ValueError):
            sol.rmsnorm_backward(*args, **kw)


def test_binding_rotary(meta):
    q, k, t = T(5, 4, 64), T(5, 2, 64), T(9, 32, dtype=torch.float32)
    with pytest.raises(Reached):
        sol.rotary(q, k, t, T(5, dtype=torch.int32), "interleaved")
    with pytest.raises(Reached):
        sol.rotary(q, None, t)
    for args, kw in (((q, T(5, 2, 63), t), {}), ((q, T(4, 2, 64), t), {}), ((q, T(5, 2, 64, dtype=torch.float16), t), {}),
                     ((q, k, T(9, 33, dtype=torch.float32)), {}), ((q, k, T(9, 66, dtype=torch.float32)), {}),
                     ((q, k, T(9, 32)), {}), ((q, k, T(0, 32, dtype=torch.float32)), {}),
                     ((q, k, t, T(4, dtype=torch.int64)), {}), ((q, k, t, T(5, dtype=torch.int16)), {}),
                     ((q, k, t), dict(layout="both")), ((q, None, t), dict(k_out=k)), ((q, k, t), dict(q_out=k)),
                     ((T(5, 64), k, t), {}), ((T(5, 4, 64, dtype=torch.float64), None, t), {}),
                     ((T(5, 64, 4).transpose(1, 2), None, t), {}), ((q, 5, t), {})):
        with pytest.raises(ValueError):
            sol.rotary(*args, **kw)


def test_binding_table():
    for bad in (dict(rotated=3), dict(rotated=8, scaling="other"), dict(rotated=8, base=0.0),
                dict(rotated=8, scaling="by-parts"), dict(rotated=2, scaling="base", factor=2.0),
                dict(rotated=8, scaling="by-parts", original_length=10, low_turns=4.0, high_turns=4.0)):
        with pytest.raises(ValueError):
            sol.rotary_frequencies(**bad)
    f = sol.rotary_frequencies(8)
    for args, kw in (((f.float(), 4), dict(device="cuda")), ((f, -1), dict(device="cuda")),
                     ((f, torch.zeros(3, dtype=torch.int32)), {}), ((f, torch.zeros(3, dtype=torch.int64)), {}),
                     ((f, 4), dict(axis_pairs=[3], device="cuda"))):
        with pytest.raises(ValueError):
            sol.rotary_table(*args, **kw)


def test_binding_weight_linear(meta):
    u8 = lambda *s: T(*s, dtype=torch.uint8)   # noqa: E731
    x, g = T(3, 64), T(1, dtype=torch.float32)
    with pytest.raises(Reached):
        sol.nvfp4_weight_linear(x, u8(5, 32), u8(5, 4), g, T(5))
    with pytest.raises(Reached):
        sol.mxfp4_weight_linear(x, u8(5, 32), u8(5, 2))
    with pytest.raises(Reached):
        sol.mxfp8_linear(u8(3, 64), u8(3, 2), u8(5, 32), u8(5, 2))
    for bad in (lambda: sol.nvfp4_weight_linear(x, u8(5, 32), u8(5, 2), g),
                lambda: sol.nvfp4_weight_linear(x, u8(5, 31), u8(5, 4), g),
                lambda: sol.nvfp4_weight_linear(x, u8(5, 32), u8(5, 4), 1.0),
                lambda: sol.nvfp4_weight_linear(x.float(), u8(5, 32), u8(5, 4), g),
                lambda: sol.mxfp4_weight_linear(x, u8(5, 32), u8(5, 4)),
                lambda: sol.mxfp4_weight_linear(T(3, 48), u8(5, 24), u8(5, 1)),
                lambda: sol.mxfp4_weight_linear(x, u8(5, 32), u8(5, 2), T(4)),
                lambda: sol.mxfp8_linear(u8(3, 64), u8(3, 4), u8(5, 32), u8(5, 2)),
                lambda: sol.mxfp8_linear(x, u8(3, 2), u8(5, 32), u8(5, 2)),
                lambda: sol.mxfp8_linear(u8(3, 64), u8(3, 2), u8(5, 32), u8(5, 2), None, T(3, 6))):
        with pytest.raises(ValueError):
            bad()


# ---- the oracle's pins ----------------------------------------------------

def test_oracle_gradients_against_differences():
    rng = np.random.Generator(np.random.PCG64(1))
    x, w, d = (rng.standard_normal((6, 20)) for _ in range(3))
    g, e = rng.standard_normal((3, 20)), rng.standard_normal((3, 20))
    f = lambda x, g: np.sum(w * R.add_rmsnorm(x, None, g, 1e-2)[1])   # noqa: E731
    ds, dg, _, _ = R.rmsnorm_backward(w, x, g, None, 1e-2)
    h = 1e-6
    assert np.isclose((f(x + h * d, g) - f(x - h * d, g)) / (2 * h), np.sum(ds * d), rtol=1e-7)
    assert np.isclose((f(x, g + h * e) - f(x, g - h * e)) / (2 * h), np.sum(dg * e), rtol=1e-7)
    # a mistake in the mean's term is seen
    wrong = ds + 1e-3 * x
    assert not np.isclose((f(x + h * d, g) - f(x - h * d, g)) / (2 * h), np.sum(wrong * d), rtol=1e-5)


def test_oracle_rotation_keeps_lengths_and_layouts_agree():
    rng = np.random.Generator(np.random.PCG64(2))
    t = rng.standard_normal((5, 2, 12))
    ang = rng.standard_normal((7, 4))
    table = np.concatenate((np.cos(ang), np.sin(ang)), 1)
    at = np.array([0, 6, 3, 3, 1])
    y, _ = R.rotate(t, table, at, "half")
    assert np.allclose((y ** 2).sum(-1), (t ** 2).sum(-1)) and np.array_equal(y[..., 8:], t[..., 8:])
    assert np.allclose(R.rotate(y, table, at, "half", inverse=True)[0], t)
    perm = np.array([0, 4, 1, 5, 2, 6, 3, 7, 8, 9, 10, 11])
    z, _ = R.rotate(t[..., perm], table, at, "interleaved")
    assert np.allclose(z, y[..., perm])
    assert np.isclose(y[0, 0, 1], t[0, 0, 1] * np.cos(ang[0, 1]) - t[0, 0, 5] * np.sin(ang[0, 1]))


def test_oracle_mxfp8():
    assert np.array_equal(R.e4m3_encode(R.E4M3), np.arange(127))
    assert R.e4m3_encode(np.array([1e9, -1e9, -0.0, 2.0 ** -10, 3 * 2.0 ** -10])).tolist() == [126, 254, 128, 0, 2]
    assert R.block_scale_bytes(np.array([0.0, 448.0, 256.0, 255.9, 1.0, 1e300]), 8).tolist() == [0, 127, 127, 126, 119, 254]
    v = R.mxfp8_values(np.full((1, 32), 0xB8, np.uint8), np.array([[128]], np.uint8))
    assert np.all(v == -2.0) and O.e4m3_decode(np.array([0x38], np.uint8))[0] == 1.0
