"""Block scales of the layer norm's 8- and 4-bit forms next to powers of two:
every row's gain puts one element of each block as near to a power of two as
FP32 allows, 2^-25 on average, where an FP32 evaluation falls on either side.

The sum is exact (no residual) and a scale goes by the value in 64 bits, so it is
the float64 norm's, unless that lies within 2^-40 of the power of two."""
import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu


def f64(t):
    return t.cpu().double().numpy()


@pytest.mark.parametrize("kind,emax", [("mxfp8", 8), ("mxfp4", 2)])
@pytest.mark.parametrize("width,mean", [(64, 0.0), (96, 3.0), (2240, 0.5), (6176, 100.0), (64, 2.0e4)])
@pytest.mark.parametrize("shifted", [False, True])
def test_scales_next_to_powers_of_two(kind, emax, width, mean, shifted):
    rows, eps = max(64, 60000 // width), 1e-6
    rng = np.random.default_rng(width)
    x = (rng.standard_normal((rows, width)) + mean).astype(np.float32)
    shift = rng.uniform(-0.5, 0.5, (rows, width)).astype(np.float32) if shifted else None
    _, n, _ = R.add_layernorm(x, None, None, None, eps)
    gain = (0.01 * rng.standard_normal((rows, width))).astype(np.float32)
    at = np.arange(0, width, 32) + rng.integers(0, 32, width // 32)
    power = np.exp2(rng.integers(0, 4, at.size))
    gain[:, at] = ((power - (0 if shift is None else shift[:, at])) / n[:, at]).astype(np.float32)
    dev = lambda v: None if v is None else torch.from_numpy(v).to(device())
    _, y, _ = R.add_layernorm(x, None, gain, shift, eps)
    amax = np.abs(y).reshape(rows, -1, 32).max(2)
    _, scales, _ = getattr(sol, f"{kind}_add_layernorm")(dev(x), None, dev(gain), dev(shift), eps)
    sc, d = scales.cpu().numpy(), 2.0 ** -40
    near = np.abs(amax / np.broadcast_to(power, amax.shape) - 1)
    low, high = R.block_scale_bytes(amax * (1 - d), emax), R.block_scale_bytes(amax * (1 + d), emax)
    wrong = (sc < low) | (sc > high)
    say(f"  {int(np.sum(near < 2.0 ** -22))} of {amax.size} blocks within 2^-22 of a power of two, {int(wrong.sum())} wrong")
    assert np.sum(near < 2.0 ** -22) > amax.size // 4 and not wrong.any()
