"""Linears of few tokens with 4-bit weights against float64, element by
element (gpu_util.assert_per_element's bound: FP32 sums in any order, one
BF16 rounding): NVFP4 and MXFP4 weights with BF16 activations, MXFP8
activations with MXFP4 weights; token counts around every tile, widths and
reduction lengths that fill none, zeros, special values."""
import numpy as np
import pytest
import torch

import oracle.nvfp4 as O
import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import (abs_products, assert_per_element, bf16_from_dev, bf16_to_dev, device, f32_to_dev, poison_bf16,
                      u8_to_dev)
from workloads import draw_activations, draw_bias, draw_weights

pytestmark = pytest.mark.gpu

KINDS = ["nvfp4", "mxfp4", "mxfp8"]


def weight(kind, N, K, seed):
    """(device operands, values without the tensor scale, alpha)."""
    bits = draw_weights(N, K, 0.02, seed)
    if kind == "nvfp4":
        c, s, a = O.nvfp4_quantize_ref(bits)
        return (u8_to_dev(c), u8_to_dev(s), f32_to_dev(a)), O.nvfp4_unscaled_ref(c, s), a
    c, s = O.mxfp4_quantize_ref(bits)
    return (u8_to_dev(c), u8_to_dev(s)), O.mxfp4_unscaled_ref(c, s), np.float32(1)


def activations(kind, M, K, seed):
    bits = draw_activations("outlier4x20", M, K, seed) if M else np.empty((0, K), np.uint16)
    if kind != "mxfp8":
        return (bf16_to_dev(bits),), O.bf16_bits_to_f32(bits).astype(np.float64)
    v = O.bf16_bits_to_f32(bits).astype(np.float64).reshape(M, K // 32, 32)
    sc = R.block_scale_bytes(np.abs(v).max(2, initial=0.0), 8).astype(np.uint8)
    codes = R.e4m3_encode(v / np.exp2(sc.astype(np.float64) - 127)[..., None]).reshape(M, K)
    return (u8_to_dev(codes), u8_to_dev(sc)), R.mxfp8_values(codes, sc)


def call(kind, x, w, bias=None, out=None, **kw):
    f = {"nvfp4": sol.nvfp4_weight_linear, "mxfp4": sol.mxfp4_weight_linear, "mxfp8": sol.mxfp8_linear}[kind]
    return f(*x, *w, bias, out, **kw)


def check(kind, M, N, K, seed, bias=True):
    x, xv = activations(kind, M, K, seed)
    w, wv, alpha = weight(kind, N, K, seed + 1)
    b = draw_bias(N, 0.02, seed + 2) if bias else None
    out = poison_bf16((M, N))
    assert call(kind, x, w, None if b is None else bf16_to_dev(b), out) is out
    ref = float(alpha) * (xv @ wv.T)
    if b is not None:
        ref = ref + O.bf16_bits_to_f32(b).astype(np.float64)
    assert_per_element(bf16_from_dev(out), ref, abs_products(xv, wv), alpha, K, b, f"{kind} {M}x{N}x{K}: ")
    return x, w, out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M", [1, 2, 4, 5, 13, 16, 17, 31, 32, 33, 48, 49, 64, 65, 130])
def test_token_counts(kind, M):
    check(kind, M, 80, 288, 100 + M)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N", [1, 15, 16, 17, 33, 63, 64, 65, 129, 1235])
def test_widths(kind, N):
    check(kind, 3, N, 160, 200 + N, bias=N % 2 == 1)
    check(kind, 37, N, 160, 300 + N, bias=N % 2 == 0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("K", [16, 32, 48, 64, 112, 128, 144, 256, 272, 480, 512, 1040, 1056, 2240, 4128, 12288])
def test_reduction_lengths(kind, K):
    if kind != "nvfp4" and K % 32:
        K += 16
    check(kind, 1, 48, K, 400 + K)
    check(kind, 20, 48, K, 500 + K)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N,K", [(1, 1152, 1152), (4, 4608, 1152), (64, 2304, 2432), (7, 18432, 256)])
def test_layer_sizes(kind, M, N, K):
    check(kind, M, N, K, 700 + M)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N,K", [(3, 700, 1056), (3, 4117, 544), (2, 16401, 288), (16, 700, 928), (16, 4117, 1056),
                                   (9, 8209, 288), (40, 1235, 416), (64, 3001, 672), (64, 4499, 1184), (33, 9001, 288)])
def test_every_tile(kind, M, N, K):
    """Ragged shapes on either side of each change of tile (on 256 compute units)."""
    check(kind, M, N, K, 800 + M)
    if kind == "nvfp4":
        check(kind, M, N, K + 16, 900 + M, bias=False)


@pytest.mark.parametrize("kind", KINDS)
def test_empty_sizes(kind):
    for M, N, K in ((0, 16, 32), (3, 0, 32), (0, 0, 0)):
        x, _ = activations(kind, M, K, 1) if K else ((torch.empty(M, 0, dtype=torch.uint8 if kind == "mxfp8" else
                                                                  torch.bfloat16, device=device()),
                                                     *([torch.empty(M, 0, dtype=torch.uint8, device=device())]
                                                       if kind == "mxfp8" else [])), None)
        w = [torch.empty(N, K // 2, dtype=torch.uint8, device=device()),
             torch.empty(N, K // (16 if kind == "nvfp4" else 32), dtype=torch.uint8, device=device())]
        w += [torch.ones(1, device=device())] if kind == "nvfp4" else []
        assert call(kind, x, w).shape == (M, N)
    # K == 0: the bias, or zeros
    u8 = dict(dtype=torch.uint8, device=device())
    x = [torch.empty(5, 0, **u8), torch.empty(5, 0, **u8)] if kind == "mxfp8" else \
        [torch.empty(5, 0, dtype=torch.bfloat16, device=device())]
    w = [torch.empty(9, 0, **u8), torch.empty(9, 0, **u8)] + ([torch.ones(1, device=device())] if kind == "nvfp4" else [])
    b = torch.randn(9, device=device()).bfloat16()
    assert torch.equal(call(kind, x, w, b), b.expand(5, 9)) and torch.all(call(kind, x, w) == 0)


@pytest.mark.parametrize("kind", ["nvfp4", "mxfp4"])
def test_every_code_and_scale(kind):
    """One-hot activations read the weight back: every code with every scale
    byte, exactly (weight rows with values beyond BF16's range excepted)."""
    K = 128
    block = 16 if kind == "nvfp4" else 32
    top = 127 if kind == "nvfp4" else 255        # E4M3 0x7F and E8M0 0xFF are NaN
    N = top
    sc = np.repeat(np.arange(top, dtype=np.uint8)[:, None], K // block, 1)
    codes = (np.arange(K // 2, dtype=np.int64)[None, :] * 17 + 5 * np.arange(N)[:, None]) & 255
    codes = codes.astype(np.uint8)
    values = (O.nvfp4_unscaled_ref if kind == "nvfp4" else O.mxfp4_unscaled_ref)(codes, sc)
    w = [u8_to_dev(codes), u8_to_dev(sc)] + ([f32_to_dev(1.0)] if kind == "nvfp4" else [])
    x = torch.eye(K, dtype=torch.bfloat16, device=device())
    got = O.bf16_bits_to_f32(bf16_from_dev(call(kind, [x], w))).astype(np.float64)
    # results below FP32's smallest normal number may be flushed to zero
    fits = (np.abs(values) < 2.0 ** 128).all(1)
    assert fits.sum() >= N - 2
    got, values = got[:, fits], values[fits]
    normal = np.abs(values.T) >= 2.0 ** -126
    assert np.array_equal(got[normal], values.T[normal])
    assert np.all(np.abs(got[~normal]) <= 2.0 ** -126)


def test_every_mxfp8_code_and_scale():
    """One-hot weights read the activations back."""
    K = 256
    eye = np.zeros((K, K // 2), np.uint8)
    k = np.arange(K)
    eye[k, k // 2] = np.where(k % 2, 0x20, 0x02)     # E2M1 code 2: 1.0
    w = [u8_to_dev(eye), u8_to_dev(np.full((K, K // 32), 127, np.uint8))]
    codes = np.tile(np.arange(256, dtype=np.uint8), (64, 1))
    codes[(codes & 127) == 127] = 0                  # without the NaN codes
    sc = np.repeat((100 + np.arange(64, dtype=np.uint8))[:, None], K // 32, 1)
    got = O.bf16_bits_to_f32(bf16_from_dev(sol.mxfp8_linear(u8_to_dev(codes), u8_to_dev(sc), *w))).astype(np.float64)
    assert np.array_equal(got, R.mxfp8_values(codes, sc))


def test_nan_and_infinity_stay_in_their_row():
    for kind in KINDS:
        x, _ = activations(kind, 6, 160, 9)
        w, _, _ = weight(kind, 40, 160, 10)
        clean = call(kind, x, w)
        if kind == "mxfp8":
            x[0][2, 70] = 0x7F
        else:
            x[0][2, 70] = float("nan")
            x[0][4, 3] = float("inf")
        got = call(kind, x, w)
        assert torch.all(torch.isnan(got[2]))
        keep = [0, 1, 3, 5] + ([4] if kind == "mxfp8" else [])
        assert torch.equal(got[keep], clean[keep])
        if kind != "mxfp8":
            assert not torch.any(torch.isfinite(got[4]))


def test_same_results_streams_and_graph():
    for kind in KINDS:
        x, _ = activations(kind, 12, 1056, 3)
        w, _, _ = weight(kind, 500, 1056, 4)
        a = call(kind, x, w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        b = call(kind, x, w, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c = call(kind, x, w)
        for i in range(3):
            x[0].copy_(activations(kind, 12, 1056, 30 + i)[0][0])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c, call(kind, x, w))
