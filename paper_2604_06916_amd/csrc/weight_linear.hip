// Products of few tokens with 4-bit weights: BF16 activations that stay
// BF16 with NVFP4 or MXFP4 weights, and MXFP8 activations with MXFP4 weights.
//
//   out[m][n] = bf16(alpha * sum_k x[m][k] (s q)[n][k] + bias[n])
//
// One wave per weight row and four tokens: a lane takes every 64th run of 32
// weights (16 bytes of codes).  FP32 throughout, one rounding.
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

constexpr int kWLTokens = 4;
constexpr int kWLThreads = 256;

__device__ __forceinline__ float e2m1_value(uint32_t c) {
  // 0, .5, 1, 1.5, 2, 3, 4, 6
  const uint32_t m = c & 7u;
  const float v = m < 2u ? 0.5f * (float)m : __uint_as_float(((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
  return c & 8u ? -v : v;
}

__device__ __forceinline__ float e8m0_value(uint32_t b) {
  return b ? __uint_as_float(b << 23) : 0x1p-127f;
}

__device__ __forceinline__ float e4m3_signed(uint32_t c) {
  if ((c & 127u) == 127u) return __builtin_nanf("");
  const float v = e4m3_value(c & 127u);
  return c & 128u ? -v : v;
}

template <int kFormat, bool kX8>
__global__ __launch_bounds__(kWLThreads) void weight_linear_kernel(WeightLinearArgs a) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t cols = (a.N + kWLThreads / kWave - 1) / (kWLThreads / kWave);
  const int64_t n = blockIdx.x % cols * (kWLThreads / kWave) + threadIdx.x / kWave;
  if (n >= a.N) return;
  const int64_t m0 = blockIdx.x / cols * kWLTokens;
  float acc[kWLTokens] = {};
  constexpr int kGroup = kFormat == SOLFP4_FORMAT_NVFP4 ? 16 : 32;
  // units of one group: 16 or 32 weights
  for (int64_t g = lane; g < a.K / kGroup; g += kWave) {
    const uint32_t sb = a.w_scales[n * (a.K / kGroup) + g];
    const float s = kFormat == SOLFP4_FORMAT_NVFP4 ? e4m3_value(sb) : e8m0_value(sb);
    for (int k = 0; k < kGroup; k += 2) {
      const int64_t at = g * kGroup + k;
      const uint32_t c = a.w_codes[(n * a.K + at) / 2];
      const float w0 = e2m1_value(c & 15u) * s, w1 = e2m1_value(c >> 4) * s;
#pragma unroll
      for (int m = 0; m < kWLTokens; ++m) {
        if (m0 + m >= a.M) break;
        const int64_t xi = (m0 + m) * a.K + at;
        float x0, x1;
        if constexpr (kX8) {
          const uint8_t* xc = static_cast<const uint8_t*>(a.x);
          const float xs = e8m0_value(a.x_scales[xi / 32]);
          x0 = e4m3_signed(xc[xi]) * xs;
          x1 = e4m3_signed(xc[xi + 1]) * xs;
        } else {
          const uint16_t* xb = static_cast<const uint16_t*>(a.x);
          x0 = __uint_as_float((uint32_t)xb[xi] << 16);
          x1 = __uint_as_float((uint32_t)xb[xi + 1] << 16);
        }
        acc[m] += x0 * w0;
        acc[m] += x1 * w1;
      }
    }
  }
  const float alpha = a.w_global ? a.w_global[0] : 1.0f;
  const float b = a.bias ? __uint_as_float((uint32_t)a.bias[n] << 16) : 0.0f;
#pragma unroll
  for (int m = 0; m < kWLTokens; ++m) {
    const float t = wave_sum(acc[m]);
    if (lane == 0 && m0 + m < a.M)
      a.out[(m0 + m) * a.N + n] = (uint16_t)pack_bf16(__builtin_fmaf(alpha, t, b), 0.0f);
  }
}

int64_t weight_linear_groups(int64_t M, int64_t N) {
  return ((N + kWLThreads / kWave - 1) / (kWLThreads / kWave)) * ((M + kWLTokens - 1) / kWLTokens);
}

hipError_t launch_weight_linear(int w_format, bool x_mxfp8, const WeightLinearArgs& a, hipStream_t stream) {
  if (a.M == 0 || a.N == 0) return hipSuccess;
  const dim3 grid((unsigned)weight_linear_groups(a.M, a.N)), block(kWLThreads);
  if (x_mxfp8) return launch_kernel(weight_linear_kernel<SOLFP4_FORMAT_MXFP4, true>, grid, block, stream, a);
  if (w_format == SOLFP4_FORMAT_NVFP4)
    return launch_kernel(weight_linear_kernel<SOLFP4_FORMAT_NVFP4, false>, grid, block, stream, a);
  return launch_kernel(weight_linear_kernel<SOLFP4_FORMAT_MXFP4, false>, grid, block, stream, a);
}

}  // namespace solfp4
