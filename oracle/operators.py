"""Float64 definitions of the operators around the linears: the norm with the
residual's addition and its gradients, the layer norm and its, rotary positions, products with 4-bit
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


def add_layernorm(x, residual=None, gain=None, shift=None, eps=1e-6):
    """(sum, layer norm of the sum, and for every element the magnitude that
    an FP32 evaluation's error goes by, in units of its rounding)."""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    rows, width = s.shape
    c = s - s.mean(axis=1, keepdims=True)
    rho = 1.0 / np.sqrt(np.mean(c * c, axis=1, keepdims=True) + eps)
    n, g = c * rho, _gain(gain, rows, width)
    t = np.zeros_like(s) if shift is None else _gain(shift, rows, width)
    far = rho * np.sqrt(np.mean(s * s, axis=1, keepdims=True))
    size = np.abs(g) * (rho * np.abs(s) + far + np.abs(n) * (40 + 2 * far) + 68) + 2 * (np.abs(n * g) + np.abs(t))
    return s, n * g + t, size


def layernorm_backward(dy, s, gain=None, groups=1, dsum=None, eps=1e-6):
    """(ds, dgain, dshift [groups, width]; magnitudes that the FP32 evaluation's
    error goes by: of ds per element, of dgain's and of dshift's summands; and
    the normalised rows' own)."""
    dy, s = np.asarray(dy, np.float64), np.asarray(s, np.float64)
    rows, width = s.shape
    c = s - s.mean(axis=1, keepdims=True)
    q = np.mean(c * c, axis=1, keepdims=True)
    rho = 1.0 / np.sqrt(q + eps)
    G = dy * _gain(gain, rows, width)
    mean = lambda v: np.mean(v, axis=1, keepdims=True)
    ds = rho * (G - mean(G) - c * rho ** 2 * mean(G * c))
    size = rho * (np.abs(G) + mean(np.abs(G)) + (np.abs(c) + np.sqrt(q)) * rho ** 2 *
                  (mean(np.abs(G * c)) + np.sqrt(q) * mean(np.abs(G))))
    if dsum is not None:
        ds = ds + dsum
    split = lambda v: v.reshape(groups, rows // groups, width).sum(1)
    return ds, split(dy * c * rho), split(dy), size, split(np.abs(dy * c * rho)), split(np.abs(dy))


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


def add_adapters(y, x, a, b, scales, index):
    """(out, hidden, and the magnitudes that their FP32 evaluation's errors go
    by: sum of |a x| per hidden value, of |scale b| (|a| |x|) per output) of
    adapters a [E, rank, K], b [E, N, rank] on tokens with these indices."""
    out, hid = np.array(y, np.float64), np.zeros((x.shape[0], a.shape[1]))
    size, hid_size = np.zeros_like(out), np.zeros_like(hid)
    for e in range(a.shape[0]):
        t = np.flatnonzero(index == e)
        hid[t], hid_size[t] = x[t] @ a[e].T, np.abs(x[t]) @ np.abs(a[e]).T
        out[t] += scales[e] * (hid[t] @ b[e].T)
        size[t] = abs(scales[e]) * (hid_size[t] @ np.abs(b[e]).T)
    bad = index >= a.shape[0]
    out[bad] = hid[bad] = np.nan
    return out, hid, size, hid_size


def adapters_backward(dy, x, hidden, a, b, scales, index, past=None):
    """(dx, da, db, and of each the sum of the magnitudes that it is formed
    from: |a| (|scale b| |dy|) for dx, over the tokens for da and db)."""
    dx = np.zeros_like(x, dtype=np.float64) if past is None else np.array(past, np.float64)
    da, db = np.zeros(a.shape), np.zeros(b.shape)
    sizes = [np.zeros_like(v) for v in (dx, da, db)]
    for e in range(a.shape[0]):
        t, c = np.flatnonzero(index == e), scales[e]
        g, g_size = c * (dy[t] @ b[e]), abs(c) * (np.abs(dy[t]) @ np.abs(b[e]))
        dx[t] += g @ a[e]
        da[e], db[e] = g.T @ x[t], c * (dy[t].T @ hidden[t])
        sizes[0][t] = g_size @ np.abs(a[e])
        sizes[1][e], sizes[2][e] = g_size.T @ np.abs(x[t]), abs(c) * (np.abs(dy[t]).T @ np.abs(hidden[t]))
    dx[index >= a.shape[0]] = np.nan
    return (dx, da, db, *sizes)
