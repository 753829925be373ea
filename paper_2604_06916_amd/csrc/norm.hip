// Root-mean-square norm of rows, with the residual's addition and an output
// in the rows' type, in MXFP8 or in MXFP4; and its backward pass.
//
//   s = x + r,  rho = (mean(s^2) + eps)^-1/2,  y = s rho g
//   G = dy g,   ds = rho (G - s rho^2 mean(G s)) + dsum,   dg = sum over rows of dy s rho
//
// Everything between a load and a store is FP32: the norm sees the FP32 sum
// (y is rounded once, not norm-of-a-rounded-sum), and the stored sum is that
// sum rounded once.
//
// A row belongs to `wpr` waves (1, 2, 4 or 8; as few as hold it in
// kNormMaxRuns runs of 8 elements a lane), so a row is read once, stays in
// registers, and for most widths is reduced inside one wave without a
// barrier.  Bound by memory: 8 bytes an element in BF16 (7.03 with MXFP8
// output).
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

// max over the aligned lane quad (quad_perm DPP: lanes 1,0,3,2 then 2,3,0,1)
__device__ __forceinline__ uint32_t quad_max_bits(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, false));
  return v;
}

// The E8M0 byte of a 32-element block held by a lane quad, 8 values a lane:
// floor(log2(amax)) - kEmax + 127, at least 0, for elements whose largest
// exponent is kEmax.  A NaN has the largest pattern of all, so it gives the
// largest scale and stays a NaN where the elements have one.
template <int kEmax>
__device__ __forceinline__ uint32_t block_scale(const float (&y)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(y[e]) & 0x7FFFFFFFu);
  const uint32_t f = quad_max_bits(m) >> 23;
  return f > kEmax ? f - kEmax : 0u;
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

// y, the 8 values at column `col` of a row (n of them inside it), to the output.
template <int kType, int kOut>
__device__ __forceinline__ void emit(const NormArgs& a, int64_t row, int64_t col, int64_t n, const float (&y)[8]) {
  if constexpr (kOut == kNormSame) {
    store_run<kType>(a.out, row * a.out_stride + col, n, from_f32<kType>(y));
  } else {
    // the four lanes of a block are inside the row or outside it together
    const uint32_t sc = block_scale<(kOut == kNormMxfp8 ? 8 : 2)>(y);
    const float inv = inverse_scale(sc);
    if constexpr (kOut == kNormMxfp8)
      *reinterpret_cast<u32x2_t*>(a.codes + row * a.width + col) = e4m3_codes(y, inv);
    else
      *reinterpret_cast<uint32_t*>(a.codes + (row * a.width + col) / 2) = e2m1_codes(y, inv);
    if ((threadIdx.x & 3) == 0) a.scales[(row * a.width + col) / 32] = (uint8_t)sc;
  }
}

// The sum of v over the `wpr` waves of this wave's row; every wave of the
// workgroup calls it.
__device__ __forceinline__ float row_sum(float v, float* lds, int wpr) {
  v = wave_sum(v);
  if (wpr == 1) return v;
  const int wave = threadIdx.x / kWave, first = wave / wpr * wpr;
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) lds[wave] = v;
  __syncthreads();
  float t = 0.0f;
  for (int w = 0; w < wpr; ++w) t += lds[first + w];
  return t;
}

template <int kType, int kOut, int kRuns>
__global__ __launch_bounds__(512) void add_rmsnorm_kernel(NormArgs a, int wpr) {
  __shared__ float lds[kNormMaxWaves];
  const int waves = blockDim.x / kWave;
  const int wave = threadIdx.x / kWave;
  const int64_t row = (int64_t)blockIdx.x * (waves / wpr) + wave / wpr;
  const int lane = (wave % wpr) * kWave + (threadIdx.x & (kWave - 1));
  const int step = wpr * kWave * 8;
  const bool in = row < a.rows;
  float s[kRuns][8];
  Run<kType> x[kRuns], r[kRuns], g[kRuns];
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int64_t col = (int64_t)i * step + lane * 8, n = in ? a.width - col : 0;
    x[i] = r[i] = g[i] = zero_run<kType>();
    if (n > 0) {
      x[i] = load_run<kType>(a.x, row * a.x_stride + col, n);
      if (a.residual) r[i] = load_run<kType>(a.residual, row * a.residual_stride + col, n);
      if (a.gain) g[i] = load_run<kType>(a.gain, row / a.group_rows * a.gain_stride + col, n);
    }
  }
  float q = 0.0f;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int64_t col = (int64_t)i * step + lane * 8, n = in ? a.width - col : 0;
    to_f32<kType>(x[i], s[i]);
    if (a.residual) {
      float v[8];
      to_f32<kType>(r[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] += v[e];
      if (n > 0) store_run<kType>(a.sum, row * a.sum_stride + col, n, from_f32<kType>(s[i]));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) q += s[i][e] * s[i][e];
  }
  q = row_sum(q, lds, wpr);
  const float rho = 1.0f / __builtin_sqrtf(q / (float)a.width + a.eps);
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int64_t col = (int64_t)i * step + lane * 8, n = in ? a.width - col : 0;
    float v[8];
    if (a.gain) to_f32<kType>(g[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[i][e] *= rho;
      if (a.gain) s[i][e] *= v[e];
    }
    if (n > 0) emit<kType, kOut>(a, row, col, n, s[i]);
  }
}

// Waves of a row, and runs a lane, for this width.
static void row_shape(int64_t width, int* wpr, int* runs) {
  const int64_t all = (width + 7) / 8;
  *wpr = 1;
  while (*wpr < kNormMaxWaves && all > (int64_t)*wpr * kWave * kNormMaxRuns) *wpr *= 2;
  *runs = (int)((all + *wpr * kWave - 1) / (*wpr * kWave));
}

template <int kType, int kOut>
static hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  int wpr, runs;
  row_shape(a.width, &wpr, &runs);
  const int waves = wpr > 4 ? wpr : 4, slots = waves / wpr;
  const dim3 grid((unsigned)((a.rows + slots - 1) / slots)), block(waves * kWave);
  switch (runs) {
    case 1: return launch_kernel(add_rmsnorm_kernel<kType, kOut, 1>, grid, block, stream, a, wpr);
    case 2: return launch_kernel(add_rmsnorm_kernel<kType, kOut, 2>, grid, block, stream, a, wpr);
    case 3: return launch_kernel(add_rmsnorm_kernel<kType, kOut, 3>, grid, block, stream, a, wpr);
    case 4: return launch_kernel(add_rmsnorm_kernel<kType, kOut, 4>, grid, block, stream, a, wpr);
    case 5: return launch_kernel(add_rmsnorm_kernel<kType, kOut, 5>, grid, block, stream, a, wpr);
    default: return launch_kernel(add_rmsnorm_kernel<kType, kOut, 6>, grid, block, stream, a, wpr);
  }
}

template <int kType>
static hipError_t launch_norm_type(const NormArgs& a, int out, hipStream_t stream) {
  if (out == kNormSame) return launch_norm<kType, kNormSame>(a, stream);
  if (out == kNormMxfp8) return launch_norm<kType, kNormMxfp8>(a, stream);
  return launch_norm<kType, kNormMxfp4>(a, stream);
}

hipError_t launch_add_rmsnorm(int type, int out, const NormArgs& a, hipStream_t stream) {
  if (a.rows == 0 || a.width == 0) return hipSuccess;
  if (type == SOLFP4_BF16) return launch_norm_type<SOLFP4_BF16>(a, out, stream);
  if (type == SOLFP4_F16) return launch_norm_type<SOLFP4_F16>(a, out, stream);
  return launch_norm_type<SOLFP4_F32>(a, out, stream);
}

// ---- backward -------------------------------------------------------------

// ds of every row, and each workgroup's share of dg: a workgroup takes the
// rows [part * part_rows, ...) of one group, its row slots one row after
// another, and keeps dg of its columns in registers; at the end the slots'
// sums are added in slot order and stored as one row of the workspace.
template <int kType, int kRuns>
__global__ __launch_bounds__(512) void rmsnorm_backward_kernel(NormBackArgs a, int wpr) {
  __shared__ float lds[kNormMaxWaves];
  __shared__ __attribute__((aligned(16))) float fold[512 * 8];
  const int waves = blockDim.x / kWave, slots = waves / wpr;
  const int slot = threadIdx.x / kWave / wpr;
  const int lane = threadIdx.x - slot * wpr * kWave;
  const int step = wpr * kWave * 8;
  const int64_t group = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int64_t first = group * a.group_rows + part * a.part_rows;
  const int64_t last = min(first + a.part_rows, (group + 1) * a.group_rows);
  float dg[kRuns][8] = {};
  for (int64_t base = first; base < last; base += slots) {
    const int64_t row = base + slot;
    const bool in = row < last;
    float s[kRuns][8], G[kRuns][8];
    float q = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int64_t col = (int64_t)i * step + lane * 8, n = in ? a.width - col : 0;
      Run<kType> x = zero_run<kType>(), d = x, g = x;
      if (n > 0) {
        x = load_run<kType>(a.x, row * a.x_stride + col, n);
        d = load_run<kType>(a.dy, row * a.dy_stride + col, n);
        if (a.gain) g = load_run<kType>(a.gain, group * a.gain_stride + col, n);
      }
      to_f32<kType>(x, s[i]);
      to_f32<kType>(d, G[i]);
      float v[8];
      to_f32<kType>(g, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = a.gain ? G[i][e] * v[e] : G[i][e];
        q += s[i][e] * s[i][e];
        b += w * s[i][e];
      }
    }
    q = row_sum(q, lds, wpr);
    b = row_sum(b, lds, wpr);
    const float rho = 1.0f / __builtin_sqrtf(q / (float)a.width + a.eps);
    const float k = b / (float)a.width * rho * rho;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int64_t col = (int64_t)i * step + lane * 8, n = in ? a.width - col : 0;
      if (n <= 0) continue;
      float v[8], out[8];
      if (a.gain) to_f32<kType>(load_run<kType>(a.gain, group * a.gain_stride + col, n), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = a.gain ? G[i][e] * v[e] : G[i][e];
        dg[i][e] += G[i][e] * (s[i][e] * rho);
        out[e] = rho * (w - s[i][e] * k);
      }
      if (a.dsum) {
        to_f32<kType>(load_run<kType>(a.dsum, row * a.dsum_stride + col, n), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] += v[e];
      }
      store_run<kType>(a.dx, row * a.dx_stride + col, n, from_f32<kType>(out));
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) fold[threadIdx.x * 8 + e] = dg[i][e];
    __syncthreads();
    if (slot) continue;
    const int64_t col = (int64_t)i * step + lane * 8;
    if (col >= a.width) continue;
    for (int z = 1; z < slots; ++z)
#pragma unroll
      for (int e = 0; e < 8; ++e) dg[i][e] += fold[(z * wpr * kWave + lane) * 8 + e];
    for (int e = 0; e < 8; ++e)
      if (col + e < a.width) a.partial[(int64_t)blockIdx.x * a.width + col + e] = dg[i][e];
  }
}

// dg[group][col] = sum of the group's parts, each of kFoldSlices threads
// taking every kFoldSlices-th part, their sums added in slice order.
constexpr int kFoldCols = 64, kFoldSlices = 16;

__global__ __launch_bounds__(kFoldCols * kFoldSlices) void dgain_kernel(const float* __restrict__ partial,
                                                                         float* __restrict__ dgain, int64_t width,
                                                                         int parts) {
  __shared__ float sums[kFoldSlices][kFoldCols];
  const int c = threadIdx.x % kFoldCols, z = threadIdx.x / kFoldCols;
  const int64_t col = (int64_t)blockIdx.x * kFoldCols + c, group = blockIdx.y;
  float t = 0.0f;
  if (col < width)
    for (int p = z; p < parts; p += kFoldSlices) t += partial[(group * parts + p) * width + col];
  sums[z][c] = t;
  __syncthreads();
  if (z || col >= width) return;
  for (int i = 1; i < kFoldSlices; ++i) t += sums[i][c];
  dgain[group * width + col] = t;
}

// Workgroups a group's rows are dealt to: two a compute unit over all
// groups, but at least kPartMinRows rows each, so that the partial sums stay
// a small share of the rows' bytes.
constexpr int64_t kPartMinRows = 8;

int64_t rmsnorm_backward_parts(int64_t rows, int64_t groups) {
  if (rows == 0 || groups == 0) return 0;
  const int64_t per = rows / groups;
  int64_t parts = (2 * (int64_t)device_cu_count() + groups - 1) / groups;
  if (parts > (per + kPartMinRows - 1) / kPartMinRows) parts = (per + kPartMinRows - 1) / kPartMinRows;
  const int64_t part_rows = (per + parts - 1) / parts;
  return (per + part_rows - 1) / part_rows;
}

template <int kType>
static hipError_t launch_back(const NormBackArgs& a, int64_t groups, hipStream_t stream) {
  int wpr, runs;
  row_shape(a.width, &wpr, &runs);
  const int waves = wpr > 4 ? wpr : 4;
  const dim3 grid((unsigned)(groups * a.parts)), block(waves * kWave);
  switch (runs) {
    case 1: return launch_kernel(rmsnorm_backward_kernel<kType, 1>, grid, block, stream, a, wpr);
    case 2: return launch_kernel(rmsnorm_backward_kernel<kType, 2>, grid, block, stream, a, wpr);
    case 3: return launch_kernel(rmsnorm_backward_kernel<kType, 3>, grid, block, stream, a, wpr);
    case 4: return launch_kernel(rmsnorm_backward_kernel<kType, 4>, grid, block, stream, a, wpr);
    case 5: return launch_kernel(rmsnorm_backward_kernel<kType, 5>, grid, block, stream, a, wpr);
    default: return launch_kernel(rmsnorm_backward_kernel<kType, 6>, grid, block, stream, a, wpr);
  }
}

hipError_t launch_rmsnorm_backward(int type, NormBackArgs a, float* dgain, hipStream_t stream) {
  const int64_t groups = a.groups;
  if (a.width == 0 || groups == 0) return hipSuccess;
  hipError_t e = hipSuccess;
  const int64_t parts = rmsnorm_backward_parts(a.rows, groups);
  if (parts) {
    a.group_rows = a.rows / groups;
    a.parts = (int)parts;
    a.part_rows = (a.group_rows + parts - 1) / parts;
    if (type == SOLFP4_BF16) e = launch_back<SOLFP4_BF16>(a, groups, stream);
    else if (type == SOLFP4_F16) e = launch_back<SOLFP4_F16>(a, groups, stream);
    else e = launch_back<SOLFP4_F32>(a, groups, stream);
  }
  if (e != hipSuccess || !dgain) return e;
  const dim3 grid((unsigned)((a.width + kFoldCols - 1) / kFoldCols), (unsigned)groups);
  return launch_kernel(dgain_kernel, grid, dim3(kFoldCols * kFoldSlices), stream, (const float*)a.partial, dgain,
                       a.width, (int)parts);
}

}  // namespace solfp4
