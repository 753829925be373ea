"""Float64 definitions of the operators around the linears: the norm with the
residual's addition and its gradients, rotary positions, products with 4-bit
weights, the MXFP8 encoding.  Plain and slow; no code of the GPU path."""
from __future__ import annotations

import numpy as np

from . import nvfp4 as O


def _gain(gain, rows, width):
    if gain is None:
        return np.ones((rows, width))
    g = np.asarray(gain, np.float64).reshape(-1, width)
    return np.repeat(g, rows // g.shape[0], axis=0) if rows else np.ones((0, width))


def add_rmsnorm(x, residual=None, gain=None, eps=1e-6):
    """(sum, norm of the sum), both float64 and unrounded."""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    rho = 1.0 / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps)
    return s, s * rho * _gain(gain, *s.shape)


def rmsnorm_backward(dy, s, gain=None, dsum=None, eps=1e-6):
    """(ds, dgain [groups, width], and the two magnitudes that the FP32
    evaluation's error goes by: of ds per element, of dgain's summands)."""
    dy, s = np.asarray(dy, np.float64), np.asarray(s, np.float64)
    rows, width = s.shape
    groups = 1 if gain is None else np.asarray(gain).reshape(-1, width).shape[0]
    rho = 1.0 / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps)
    G = dy * _gain(gain, rows, width)
    ds = rho * (G - s * rho ** 2 * np.mean(G * s, axis=1, keepdims=True))
    size = rho * (np.abs(G) + np.abs(s) * rho ** 2 * np.mean(np.abs(G * s), axis=1, keepdims=True))
    if dsum is not None:
        ds = ds + dsum
    n = (dy * s * rho).reshape(groups, rows // groups, width)
    return ds, n.sum(1), size, np.abs(n).sum(1)


def rotate(t, table, positions, layout, inverse=False):
    """Rotary positions on t [tokens, heads, dim]; (result, sum of the
    magnitudes that each element is formed from)."""
    t, table = np.asarray(t, np.float64), np.asarray(table, np.float64)
    R = table.shape[1]
    h = R // 2
    c, s = table[positions, None, :h], table[positions, None, h:]
    if inverse:
        s = -s
    first, second = (slice(0, h), slice(h, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
    u, v = t[..., first], t[..., second]
    out, size = t.copy(), np.abs(t)
    out[..., first], out[..., second] = u * c - v * s, u * s + v * c
    size[..., first], size[..., second] = abs(u * c) + abs(v * s), abs(u * s) + abs(v * c)
    return out, size


E4M3 = O.e4m3_decode(np.arange(127, dtype=np.uint8))     # ascending magnitudes


def e4m3_encode(v):
    """Codes of float64 values: nearest, ties to the even code, saturating."""
    a = np.abs(v)
    mid = (E4M3[1:] + E4M3[:-1]) / 2
    i = np.searchsorted(mid, a, side="left")       # a == mid: the lower code
    tie = (i < mid.size) & (a == mid[np.minimum(i, mid.size - 1)])
    i = i + (tie & (i % 2 == 1))
    return (i + 128 * np.signbit(v)).astype(np.uint8)


def block_scale_bytes(amax, emax):
    """E8M0 bytes floor(log2(amax)) - emax + 127, clamped to 0..254; 0 for 0."""
    _, e = np.frexp(amax)
    return np.where(amax > 0, np.clip(e - 1 - emax + 127, 0, 254), 0)


def mxfp8_values(codes, scales):
    """Decoded values [rows, K] of MXFP8 codes and scales."""
    rows, K = codes.shape
    v = O.e4m3_decode(codes & 127) * np.where(codes & 128, -1.0, 1.0)
    return (v.reshape(rows, K // 32, 32) * O.e8m0_decode(scales)[..., None]).reshape(rows, K)
