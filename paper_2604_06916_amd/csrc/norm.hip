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
// A row belongs to `wpr` waves (1, 2, 4 or 8; as few as hold it in kNormRuns,
// at most kNormMaxRuns, runs of 8 elements a lane), so a row is read once and
// stays in registers between the sum and the output.  Rows of at most 256
// elements (contiguous heads of q or k) share a wave: 32 lanes a row or fewer
// (kRuns == 1).
//
// Bound by memory: 8 bytes an element in BF16 with a residual, 7.03 with MXFP8
// output.  BF16, 8192 x 2240 in 8 groups 26.1 us, 5.6 TB/s; 18432 x 3072 to MXFP8
// 71.8 us, 5.5 TB/s (a 1 GB copy moves 5.0, a 0.2 GB one 5.4); one row of 1152
// 3.2 us, a launch.
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

// max over the aligned lane quad (quad_perm DPP: lanes 1,0,3,2 then 2,3,0,1)
__device__ __forceinline__ uint32_t quad_max_bits(uint32_t v) {
  v = max(v, dpp_of<0xB1>(v));
  return max(v, dpp_of<0x4E>(v));
}

// The E8M0 byte of a 32-element block held by a lane quad, 8 values y = s rho g
// a lane: floor(log2(amax)) - kEmax + 127, at least 0, for elements whose
// largest exponent is kEmax.  A NaN has the largest pattern of all, so it
// gives the largest scale and stays a NaN where the elements have one.
//
// An FP32 amax next to a power of two may lie on the wrong side of it, which
// would double or halve the scale: within 4 units (y is within 3, the
// roundings of rho and the two products) the comparison is made in 64 bits.
// That takes a rho of more than 32 bits, for which the row's squares are
// summed in 64.
template <int kEmax>
__device__ __forceinline__ uint32_t block_scale(const float (&y)[8], const float (&s)[8], const float (&g)[8],
                                                double rho) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(y[e]) & 0x7FFFFFFFu);
  m = quad_max_bits(m);
  uint32_t f = m >> 23;
  if (((m + 4u) & 0x7FFFFFu) < 8u) {   // alike in the quad
    f = (m + 4u) >> 23;
    const double power = __uint_as_float(f << 23);
    uint32_t reached = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float t = s[e];
      asm volatile("" : "+v"(t));   // converted here, where it is rarely needed, and not kept in 64 bits
      reached |= __builtin_fabs((double)t * rho * (double)g[e]) >= power;
    }
    if (!quad_max_bits(reached)) --f;
  }
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
// of the workgroup calls it.
template <int n, typename T>
__device__ __forceinline__ void row_sum(T (&v)[n], T (*lds)[n], int wave, RowShape sh) {
#pragma unroll
  for (int i = 0; i < n; ++i) v[i] = lanes_sum(v[i], sh.lanes);
  if (sh.wpr == 1) return;
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
    for (int i = 0; i < n; ++i) lds[wave][i] = v[i];
  __syncthreads();
  const int first = wave & -sh.wpr;
#pragma unroll
  for (int i = 0; i < n; ++i) v[i] = lds[first][i];
  for (int w = 1; w < sh.wpr; ++w)
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] += lds[first + w][i];
}

// a b + c, one rounding (the build contracts nothing by itself)
__device__ __forceinline__ float fused(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fused(double a, double b, double c) { return __builtin_fma(a, b, c); }
__device__ __forceinline__ double fused(float a, float b, double c) { return fused((double)a, (double)b, c); }

template <int kType, int kOut, int kRuns>
__global__ __launch_bounds__(kNormMaxWaves * kWave) void add_rmsnorm_kernel(NormArgs a, RowShape sh) {
  using Sum = std::conditional_t<kOut == kNormSame, float, double>;   // block_scale
  __shared__ Sum lds[kNormMaxWaves][1];
  const Place<kRuns> at_(sh);
  const int64_t row = a.first + (int64_t)blockIdx.x * sh.waves_slots(blockDim.x / kWave) + at_.slot;
  const int lane = at_.lane, step = at_.step;
  const int width = row < a.rows ? (int)a.width : 0;   // no elements of a row past the last
  const int64_t at = row < a.rows ? row : 0;
  const uint8_t* xr = row_of<kType>(a.x, at, a.x_stride);
  const uint8_t* rr = row_of<kType>(a.residual, at, a.residual_stride);
  const uint8_t* gr = row_of<kType>(a.gain, (uint32_t)at / (uint32_t)a.group_rows, a.gain_stride);
  Run<kType> x[kRuns], r[kRuns], g[kRuns];
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = width - col;
    x[i] = r[i] = zero_run<kType>();
    g[i] = one_run<kType>();
    if (n > 0) {
      x[i] = load_run<kType>(xr, col, n);
      if (a.residual) r[i] = load_run<kType>(rr, col, n);
      if (a.gain) g[i] = load_run<kType>(gr, col, n);
    }
  }
  float s[kRuns][8];
  Sum q[1] = {0};
  uint8_t* sr = row_of<kType>(a.sum, at, a.sum_stride);
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = width - col;
    to_f32<kType>(x[i], s[i]);
    if (a.residual) {
      float v[8];
      to_f32<kType>(r[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] += v[e];
      if (n > 0) store_run<kType>(sr, col, n, from_f32<kType>(s[i]));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) q[0] = fused(s[i][e], s[i][e], q[0]);
  }
  row_sum(q, lds, at_.wave, sh);
  Sum rho;
  if constexpr (kOut == kNormSame) {
    rho = 1.0f / __builtin_sqrtf(q[0] / (float)a.width + a.eps);
  } else {
    // The FP32 root of v scaled by an even power of two to [1/2, 2), where FP32
    // holds it whatever v is, and two Newton steps: 2^-22, 2^-43, beyond
    // 2^-50.  The root of 0, infinity and NaN is what it is.
    const double v = q[0] / (double)a.width + (double)a.eps;
    const int half = __builtin_amdgcn_frexp_exp(v) >> 1;
    const double m = __builtin_ldexp(v, -2 * half);
    rho = 1.0f / __builtin_sqrtf((float)m);
    if (rho > 0.0 && rho < __builtin_inf())
#pragma unroll
      for (int i = 0; i < 2; ++i) rho = rho * (1.5 - 0.5 * m * rho * rho);
    rho = __builtin_ldexp(rho, -half);
  }
  const float rho32 = (float)rho;
  uint8_t* outr = row_of<kType>(a.out, at, a.out_stride);
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = width - col;
    float v[8], y[8];
    forget(g[i]);
    to_f32<kType>(g[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = s[i][e] * rho32 * v[e];
    if (n <= 0) continue;
    if constexpr (kOut == kNormSame) {
      store_run<kType>(outr, col, n, from_f32<kType>(y));
    } else {
      // the four lanes of a block are inside the row or outside it together
      const uint32_t sc = block_scale<(kOut == kNormMxfp8 ? 8 : 2)>(y, s[i], v, rho);
      const float inv = inverse_scale(sc);
      if constexpr (kOut == kNormMxfp8)
        *reinterpret_cast<u32x2_t*>(a.codes + at * a.width + col) = e4m3_codes(y, inv);
      else
        *reinterpret_cast<uint32_t*>(a.codes + (at * a.width + col) / 2) = e2m1_codes(y, inv);
      if ((threadIdx.x & 3) == 0) a.scales[(at * a.width + col) / 32] = (uint8_t)sc;
    }
  }
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

template <int kType, int kOut>
static auto norm_kernel(int runs) {
  switch (runs) {
    case 1: return add_rmsnorm_kernel<kType, kOut, 1>;
    case 2: return add_rmsnorm_kernel<kType, kOut, 2>;
    case 3: return add_rmsnorm_kernel<kType, kOut, 3>;
    case 4: return add_rmsnorm_kernel<kType, kOut, 4>;
    case 5: return add_rmsnorm_kernel<kType, kOut, 5>;
    default: return add_rmsnorm_kernel<kType, kOut, 6>;
  }
}

template <int kType, int kOut>
static hipError_t launch_norm(NormArgs a, hipStream_t stream) {
  const RowShape sh = row_shape(a.width, kNormRuns<kType>);
  const int waves = sh.wpr > 4 ? sh.wpr : 4, slots = sh.waves_slots(waves);
  const int64_t most = kMaxThreads / (waves * kWave) * slots;   // rows of one launch
  for (a.first = 0; a.first < a.rows; a.first += most) {
    const int64_t rows = a.rows - a.first < most ? a.rows - a.first : most;
    const hipError_t e = launch_kernel(norm_kernel<kType, kOut>(sh.runs), dim3((unsigned)((rows + slots - 1) / slots)),
                                       dim3(waves * kWave), stream, a, sh);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
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

// Runs a lane above which a row gets more waves: with these the kernel takes
// at most 128 registers, and two workgroups share a CU.
template <int kType>
constexpr int kBackRuns = kType == SOLFP4_F32 ? 2 : 3;

// ds of every row, and each workgroup's share of dg: a workgroup of eight
// waves takes every `parts`-th run of as many rows as it holds of one group,
// so that the chip reads one window of the operands at a time (contiguous
// blocks of rows a workgroup were slower), and keeps dg of its columns in
// registers; at the end the slots' sums are added in slot order and stored as
// one row of the workspace.  All of a row's loads go out before the first use
// and stay as they were read (converted again after the reduction: half the
// registers of FP32 copies, twice the waves).  Holding the next row's loads
// beside them was slower, 130 us for 126, by the registers.
//
// Bound by memory, 8 bytes an element in BF16 with dsum: 26574 x 2432 in 6
// groups 108 us with the sums of dg, 4.8 TB/s; FP32 777 x 1235 8.1 + 2.7 us.
template <int kType, int kRuns>
__global__ __launch_bounds__(kNormMaxWaves * kWave, kRuns <= kBackRuns<kType> ? 4 : 2) void rmsnorm_backward_kernel(NormBackArgs a, RowShape sh) {
  __shared__ float lds[kNormMaxWaves][2];
  __shared__ __attribute__((aligned(16))) float fold[kRuns][kNormMaxWaves * kWave * 8];
  const Place<kRuns> at_(sh);
  const int slots = sh.waves_slots(kNormMaxWaves), slot = at_.slot, lane = at_.lane, step = at_.step;
  const int group = blockIdx.x / a.parts, part = blockIdx.x - group * a.parts;
  const uint32_t rows = (uint32_t)a.group_rows;   // a hop past its end still fits 32 bits
  const int64_t row0 = group * a.group_rows;
  Run<kType> g[kRuns];
  const uint8_t* gr = row_of<kType>(a.gain, group, a.gain_stride);
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = (int)a.width - col;
    g[i] = one_run<kType>();
    if (a.gain && n > 0) g[i] = load_run<kType>(gr, col, n);
  }
  float dg[kRuns][8] = {};
  for (uint32_t base = part * slots; base < rows; base += a.parts * slots) {
    const bool in = base + slot < rows;
    const int64_t row = row0 + (in ? base + slot : base);
    const int width = in ? (int)a.width : 0;
    const uint8_t* xr = row_of<kType>(a.x, row, a.x_stride);
    const uint8_t* dr = row_of<kType>(a.dy, row, a.dy_stride);
    const uint8_t* er = row_of<kType>(a.dsum, row, a.dsum_stride);
    Run<kType> x[kRuns], d[kRuns], ex[kRuns];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int col = i * step + lane * 8, n = width - col;
      x[i] = d[i] = ex[i] = zero_run<kType>();
      if (n > 0) {
        x[i] = load_run<kType>(xr, col, n);
        d[i] = load_run<kType>(dr, col, n);
        if (a.dsum) ex[i] = load_run<kType>(er, col, n);
      }
    }
    float qb[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      float s[8], D[8], v[8];
      to_f32<kType>(x[i], s);
      to_f32<kType>(d[i], D);
      to_f32<kType>(g[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        qb[0] = fused(s[e], s[e], qb[0]);
        qb[1] = fused(D[e] * v[e], s[e], qb[1]);
      }
    }
    row_sum(qb, lds, at_.wave, sh);
    // 0 where the slot has no row: with eps = 0 its zeros would add 0 times infinity to dg
    const float rho = in ? 1.0f / __builtin_sqrtf(qb[0] / (float)a.width + a.eps) : 0.0f;
    const float k = qb[1] / (float)a.width * rho * rho;
    uint8_t* outr = row_of<kType>(a.dx, row, a.dx_stride);
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int col = i * step + lane * 8, n = width - col;
      float s[8], D[8], v[8], out[8];
      forget(x[i]);
      forget(d[i]);
      forget(g[i]);
      to_f32<kType>(x[i], s);
      to_f32<kType>(d[i], D);
      to_f32<kType>(g[i], v);
      to_f32<kType>(ex[i], out);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dg[i][e] = fused(D[e], s[e] * rho, dg[i][e]);
        out[e] = fused(rho, fused(s[e], -k, D[e] * v[e]), out[e]);
      }
      if (n > 0) store_run<kType>(outr, col, n, from_f32<kType>(out));
    }
  }
  if (!a.partial) return;
  float* part_row = a.partial + (int64_t)blockIdx.x * a.width;
  // every slot's sums to LDS, then each thread adds some columns'
  const int cols = sh.wpr * sh.lanes * 8;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    floatx4_t* to = reinterpret_cast<floatx4_t*>(fold[i] + slot * cols + lane * 8);
    to[0] = floatx4_t{dg[i][0], dg[i][1], dg[i][2], dg[i][3]};
    to[1] = floatx4_t{dg[i][4], dg[i][5], dg[i][6], dg[i][7]};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    for (int c = threadIdx.x; c < cols; c += kNormMaxWaves * kWave) {
      float t = fold[i][c];
      for (int z = 1; z < slots; ++z) t += fold[i][z * cols + c];
      if (i * step + c < a.width) part_row[i * step + c] = t;
    }
  }
}

// dg[group][col] = sum of the group's parts, each of kFoldSlices threads
// taking every kFoldSlices-th part, their sums added in slice order; a
// thread's loads go out kFoldDeep at a time, so that up to 256 parts cost one
// round trip (195 parts of 1235 columns: 2.7 us, 3.2 in a loop of eight).
constexpr int kFoldCols = 64, kFoldSlices = 16, kFoldDeep = 16;

__global__ __launch_bounds__(kFoldCols * kFoldSlices) void dgain_kernel(const float* __restrict__ partial,
                                                                         float* __restrict__ dgain, int64_t width,
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

// Workgroups a group's rows are dealt to: over all groups at most two a
// compute unit (one round: with 516 on 256 CUs, 26574 x 2432 took 126 us, with
// 510 107), or one where they then take fewer than kBackDeep rounds of rows
// each (FP32, one and two a CU: 1311 x 3072 18.7 and 18.5 us, 777 x 9728 36.0 and
// 40.8, but 2304 x 5600, nine rounds, 47.3 and 43.9).  Up to kOnePass rounds
// stay on one workgroup, which then needs no second launch.  (Rounds by FP32's
// shape for all types: the workspace does not depend on the type.)
constexpr int64_t kOnePass = 2, kBackDeep = 8;

int64_t rmsnorm_backward_parts(int64_t rows, int64_t width, int64_t groups) {
  if (rows == 0 || groups == 0) return 0;
  const int64_t cus = device_cu_count();
  const int64_t slots = row_shape(width, kBackRuns<SOLFP4_F32>).waves_slots(kNormMaxWaves);
  const int64_t rounds = (rows / groups + slots - 1) / slots;
  if (rounds <= kOnePass) return 1;
  const int64_t parts = (rounds * groups < kBackDeep * cus ? cus : 2 * cus) / groups;
  return parts < 1 ? 1 : parts < rounds ? parts : rounds;
}

template <int kType>
static hipError_t launch_back(const NormBackArgs& a, int64_t groups, hipStream_t stream) {
  const RowShape sh = row_shape(a.width, kBackRuns<kType>);
  const dim3 grid((unsigned)(groups * a.parts)), block(kNormMaxWaves * kWave);
  switch (sh.runs) {
    case 1: return launch_kernel(rmsnorm_backward_kernel<kType, 1>, grid, block, stream, a, sh);
    case 2: return launch_kernel(rmsnorm_backward_kernel<kType, 2>, grid, block, stream, a, sh);
    case 3: return launch_kernel(rmsnorm_backward_kernel<kType, 3>, grid, block, stream, a, sh);
    case 4: return launch_kernel(rmsnorm_backward_kernel<kType, 4>, grid, block, stream, a, sh);
    case 5: return launch_kernel(rmsnorm_backward_kernel<kType, 5>, grid, block, stream, a, sh);
    default: return launch_kernel(rmsnorm_backward_kernel<kType, 6>, grid, block, stream, a, sh);
  }
}

hipError_t launch_rmsnorm_backward(int type, NormBackArgs a, float* dgain, hipStream_t stream) {
  const int64_t groups = a.groups;
  if (a.width == 0 || groups == 0) return hipSuccess;
  hipError_t e = hipSuccess;
  const int64_t parts = rmsnorm_backward_parts(a.rows, a.width, groups);
  if (parts == 1 && dgain) a.partial = dgain;   // the one workgroup's sums are the group's
  if (parts) {
    a.group_rows = a.rows / groups;
    a.parts = (int)parts;
    if (type == SOLFP4_BF16) e = launch_back<SOLFP4_BF16>(a, groups, stream);
    else if (type == SOLFP4_F16) e = launch_back<SOLFP4_F16>(a, groups, stream);
    else e = launch_back<SOLFP4_F32>(a, groups, stream);
  }
  if (e != hipSuccess || !dgain || parts == 1) return e;
  const dim3 grid((unsigned)((a.width + kFoldCols - 1) / kFoldCols), (unsigned)groups);
  return launch_kernel(dgain_kernel, grid, dim3(kFoldCols * kFoldSlices), stream, (const float*)a.partial, dgain,
                       a.width, (int)parts);
}

}  // namespace solfp4
