// What the root-mean-square norm and the layer norm share: how rows lie on
// waves, sums over a row, the 8- and 4-bit codes, and the last step of the
// gains' gradients.
#pragma once

#include "elements.h"
#include "kernels.h"

namespace solfp4 {

// max over the aligned lane quad (quad_perm DPP: lanes 1,0,3,2 then 2,3,0,1)
__device__ __forceinline__ uint32_t quad_max_bits(uint32_t v) {
  v = max(v, dpp_of<0xB1>(v));
  return max(v, dpp_of<0x4E>(v));
}

// y / 2^(scale - 127), exact
__device__ __forceinline__ float inverse_scale(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// E4M3, nearest with ties to even, saturating at 448; NaN stays NaN
__device__ __forceinline__ float clamp_e4m3(float v) {
  v = v > 448.0f ? 448.0f : v;
  return v < -448.0f ? -448.0f : v;
}

__device__ __forceinline__ u32x2_t e4m3_codes(const float (&y)[8], float inv) {
  int c[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    c[h] = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(y[4 * h] * inv), clamp_e4m3(y[4 * h + 1] * inv), 0, false);
    c[h] = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(y[4 * h + 2] * inv), clamp_e4m3(y[4 * h + 3] * inv), c[h], true);
  }
  return u32x2_t{(uint32_t)c[0], (uint32_t)c[1]};
}

__device__ __forceinline__ uint32_t e2m1_codes(const float (&y)[8], float inv) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0] * inv, y[1] * inv, 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2] * inv, y[3] * inv, 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4] * inv, y[5] * inv, 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6] * inv, y[7] * inv, 1.0f, 3);
  return c;
}

// How rows lie on the waves of a workgroup: a row on `wpr` whole waves, or
// on `lanes` lanes of one (both powers of two; kRuns == 1 only).
struct RowShape {
  int wpr, lanes, runs;
  __host__ __device__ int waves_slots(int waves) const { return waves / wpr * (kWave / lanes); }   // rows of a workgroup
};

// This thread's row slot in its workgroup, its lane in the row, and the
// columns between its runs.
template <int kRuns>
struct Place {
  int wave, slot, lane, step;
  __device__ __forceinline__ explicit Place(RowShape sh) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l = threadIdx.x & (kWave - 1);
    slot = wave / sh.wpr;
    lane = (wave & (sh.wpr - 1)) * kWave + l;
    step = sh.wpr * kWave * 8;
    if (kRuns == 1 && sh.lanes < kWave) {
      slot = wave * (kWave / sh.lanes) + l / sh.lanes;
      lane = l & (sh.lanes - 1);
    }
  }
};

// The sums of v[0 .. n) over a row's lanes, waves in wave order; every wave
// of the workgroup calls it.  kAgain: the waves may still read what an earlier
// call left in this lds (callers that alternate between two need no wait: a
// wave is past its reads of one when it reaches the other's).
template <bool kAgain = true, int n, typename T>
__device__ __forceinline__ void row_sum(T (&v)[n], T (*lds)[n], int wave, RowShape sh) {
#pragma unroll
  for (int i = 0; i < n; ++i) v[i] = lanes_sum(v[i], sh.lanes);
  if (sh.wpr == 1) return;
  if (kAgain) __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
    for (int i = 0; i < n; ++i) lds[wave][i] = v[i];
  __syncthreads();
  const int first = wave & -sh.wpr;
#pragma unroll
  for (int i = 0; i < n; ++i) v[i] = lds[first][i];
#pragma unroll 1
  for (int w = 1; w < sh.wpr; ++w)
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] += lds[first + w][i];
}

// a b + c, one rounding (the build contracts nothing by itself)
__device__ __forceinline__ float fused(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fused(double a, double b, double c) { return __builtin_fma(a, b, c); }
__device__ __forceinline__ double fused(float a, float b, double c) { return fused((double)a, (double)b, c); }

// v^-1/2 in 64 bits, for 8- and 4-bit outputs: the FP32 root of v scaled by an
// even power of two to [1/2, 2), where FP32 holds it whatever v is, and two
// Newton steps: 2^-22, 2^-43, beyond 2^-50.  The root of 0, infinity and NaN is
// what it is.
__device__ __forceinline__ double inverse_root(double v) {
  const int half = __builtin_amdgcn_frexp_exp(v) >> 1;
  const double m = __builtin_ldexp(v, -2 * half);
  double rho = 1.0f / __builtin_sqrtf((float)m);
  if (rho > 0.0 && rho < __builtin_inf())
#pragma unroll
    for (int i = 0; i < 2; ++i) rho = rho * (1.5 - 0.5 * m * rho * rho);
  return __builtin_ldexp(rho, -half);
}

// Runs a lane above which a row of the forward pass gets more waves.  More of
// a row a lane costs registers and so waves in flight, more waves a barrier:
// BF16 8192 x 2240 takes 26.1 us with up to three and 27.6 with six (25.5 with
// two, but 9000 x 1235 18.7 and 22.6), FP32 9216 x 3072 80.8, 84.7 and 97.1 with
// one, two and six.
template <int kType>
constexpr int kNormRuns = kType == SOLFP4_F32 ? 1 : 3;

// The shape for this width: the fewest waves that need at most `most` runs
// a lane; a row that fits half a wave on as few lanes as hold it.
static RowShape row_shape(int64_t width, int most) {
  const int64_t all = (width + 7) / 8;
  RowShape sh = {1, kWave, 1};
  while (sh.wpr < kNormMaxWaves && all > (int64_t)sh.wpr * kWave * most) sh.wpr *= 2;
  sh.runs = (int)((all + sh.wpr * kWave - 1) / (sh.wpr * kWave));
  while (sh.lanes > 1 && all <= sh.lanes / 2) sh.lanes /= 2;
  return sh;
}

// Runs a lane above which a row gets more waves: with these the kernel takes
// at most 128 registers, and two workgroups share a CU.
template <int kType>
constexpr int kBackRuns = kType == SOLFP4_F32 ? 2 : 3;

// dg[group][col] = sum of the group's parts, each of kFoldSlices threads
// taking every kFoldSlices-th part, their sums added in slice order; a
// thread's loads go out kFoldDeep at a time, so that up to 256 parts cost one
// round trip (195 parts of 1235 columns: 2.7 us, 3.2 in a loop of eight).
constexpr int kFoldCols = 64, kFoldSlices = 16, kFoldDeep = 16;

__device__ __forceinline__ void fold_parts(const float* __restrict__ partial, float* __restrict__ dgain, int64_t width,
                                           int parts) {
  __shared__ float sums[kFoldSlices][kFoldCols];
  const int c = threadIdx.x % kFoldCols, z = threadIdx.x / kFoldCols;
  const int64_t col = (int64_t)blockIdx.x * kFoldCols + c, group = blockIdx.y;
  float t = 0.0f;
  if (col < width) {
    const float* p = partial + group * parts * width + col;
    for (int i = z; i < parts; i += kFoldSlices * kFoldDeep) {
      float v[kFoldDeep];
#pragma unroll
      for (int u = 0; u < kFoldDeep; ++u) v[u] = i + u * kFoldSlices < parts ? p[(i + u * kFoldSlices) * width] : 0.0f;
#pragma unroll
      for (int u = 0; u < kFoldDeep; ++u) t += v[u];
    }
  }
  sums[z][c] = t;
  __syncthreads();
  if (z || col >= width) return;
#pragma unroll
  for (int i = 1; i < kFoldSlices; ++i) t += sums[i][c];
  dgain[group * width + col] = t;
}

}  // namespace solfp4
