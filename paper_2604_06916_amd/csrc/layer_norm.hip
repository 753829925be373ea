// Layer norm of rows with a gain and a shift, with the residual's addition
// and an output in the rows' type, in MXFP8 or in MXFP4; and its backward pass.
//
//   s = x + r,  m = mean(s),  rho = (mean((s - m)^2) + eps)^-1/2
//   n = (s - m) rho,  y = n g + t
//   G = dy g,  ds = rho (G - mean(G) - n mean(G n)) + dsum
//   dg = sum over rows of dy n,  dt = sum over rows of dy
//
// Rows lie on waves as in the root-mean-square norm and are read once.  The
// statistics take two sums over the registers: the mean, then the differences
// d = s - m and their squares.  The second sum of d corrects the first: m is
// rounded to FP32, so a row far from zero (1000 +- 1) would keep an error of
// 2^-24 of its mean in every element; with d's own mean taken off, elements
// are right to 2^-24 of themselves, and mean(d^2) - mean(d)^2 loses nothing,
// since mean(d) is 2^-24 of m.  With 8- and 4-bit outputs the sums are in 64 bits,
// of unrounded differences from a mean that needs no such correction.
//
// Bound by memory: 8 bytes an element in BF16 with a residual, 7.03 with MXFP8
// output: 8192 x 2240 BF16 in 8 groups 26.8 us, 5.5 TB/s; 26574 x 2432 to MXFP8 93 us,
// 4.9 TB/s; one row of 1152 4.3 us of which 2.3 are an empty launch.
#include "norm_common.h"

namespace solfp4 {

// The E8M0 byte of a 32-element block held by a lane quad, 8 values y = n g + t
// a lane, as the root-mean-square norm's: floor(log2(amax)) - kEmax + 127, at
// least 0.  Where y is the difference of two larger numbers its error goes by
// those: `size` is the lane's largest |n g| + |t| + |off rho g|, off what m lacks
// to the mean, and y is within 6 roundings of 2^-24 of it (s - m, less off, rho,
// the two products and the sum; where off outweighs the element, s - m and it
// once more).  An amax within 2^-21 size of a power of two is formed in 64 bits,
// from s itself: s - m is rounded, and that alone can reach over the power.
template <int kEmax, typename F>
__device__ __forceinline__ uint32_t block_scale(const float (&y)[8], float size, F y64) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(y[e]) & 0x7FFFFFFFu);
  m = quad_max_bits(m);
  const float near = __uint_as_float(quad_max_bits(__float_as_uint(size))) * 0x1p-21f, amax = __uint_as_float(m);
  const float below = amax > near ? amax - near : 0.0f;
  uint32_t f = m >> 23;
  if (__float_as_uint(below) >> 23 != __float_as_uint(amax + near) >> 23 && f < 255u) {   // alike in the quad
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double v = __builtin_fabs(y64(e));
      const int b = v > 0.0 ? __builtin_amdgcn_frexp_exp(v) - 1 + 127 : 0;
      top = max(top, (uint32_t)max(b, 0));
    }
    f = quad_max_bits(top);
  }
  return f > kEmax ? f - kEmax : 0u;
}

// A variance that its rounding took below 0 (a row of equal elements); NaN stays NaN
template <typename T>
__device__ __forceinline__ T not_negative(T v) { return v < 0 ? 0 : v; }

// s - m of a lane's run, 0 where the row has no elements (the first n of the run exist)
__device__ __forceinline__ void differences(float (&s)[8], float m, int n, bool whole) {
  const float from = n > 0 ? m : 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] -= from;
  if (!whole)
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = e < n ? s[e] : 0.0f;
}

template <int kType, int kOut, int kRuns>
__global__ __launch_bounds__(kNormMaxWaves * kWave) void add_layernorm_kernel(LayerNormArgs p, RowShape sh) {
  using Sum = std::conditional_t<kOut == kNormSame, float, double>;   // block_scale
  constexpr int kSums = kOut == kNormSame ? 2 : 1;   // d where the mean is rounded, and d^2
  __shared__ Sum lds[kNormMaxWaves][kSums];
  __shared__ Sum lds_mean[kNormMaxWaves][1];
  const NormArgs& a = p.n;
  const Place<kRuns> at_(sh);
  const int64_t row = a.first + (int64_t)blockIdx.x * sh.waves_slots(blockDim.x / kWave) + at_.slot;
  const int lane = at_.lane, step = at_.step;
  const int width = row < a.rows ? (int)a.width : 0;   // no elements of a row past the last
  const int64_t at = row < a.rows ? row : 0;
  const int64_t group = (uint32_t)at / (uint32_t)a.group_rows;
  const uint8_t* xr = row_of<kType>(a.x, at, a.x_stride);
  const uint8_t* rr = row_of<kType>(a.residual, at, a.residual_stride);
  const uint8_t* gr = row_of<kType>(a.gain, group, a.gain_stride);
  const uint8_t* tr = row_of<kType>(p.shift, group, p.shift_stride);
  Run<kType> x[kRuns], r[kRuns], g[kRuns], t[kRuns];
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = width - col;
    x[i] = r[i] = t[i] = zero_run<kType>();
    g[i] = one_run<kType>();
    if (n > 0) {
      x[i] = load_run<kType>(xr, col, n);
      if (a.residual) r[i] = load_run<kType>(rr, col, n);
      if (a.gain) g[i] = load_run<kType>(gr, col, n);
      if (p.shift) t[i] = load_run<kType>(tr, col, n);
    }
  }
  float s[kRuns][8];
  Sum mean[1] = {0};
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
    for (int e = 0; e < 8; ++e) mean[0] += s[i][e];
  }
  row_sum<false>(mean, lds_mean, at_.wave, sh);
  const Sum mean_ = mean[0] / (Sum)a.width;
  const float m = (float)mean_;
  Sum q[kSums] = {};
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int n = width - (i * step + lane * 8);
    if constexpr (kOut == kNormSame) {
      differences(s[i], m, n, (a.width & 7) == 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        q[0] += s[i][e];
        q[1] = fused(s[i][e], s[i][e], q[1]);
      }
    } else {   // a run is inside the row or outside it
      const double from = n > 0 ? mean_ : 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double d = (double)s[i][e] - from;
        q[0] = fused(d, d, q[0]);
      }
    }
  }
  row_sum<false>(q, lds, at_.wave, sh);
  Sum off, var;   // mean - m
  if constexpr (kOut == kNormSame) {
    off = q[0] / (Sum)a.width, var = not_negative(q[1] / (Sum)a.width - off * off);
  } else {
    off = mean_ - m, var = q[0] / (Sum)a.width;
  }
  Sum rho;
  if constexpr (kOut == kNormSame) rho = 1.0f / __builtin_sqrtf(var + a.eps);
  else rho = inverse_root(var + (double)a.eps);
  const float rho32 = (float)rho, off32 = (float)off, far = __builtin_fabsf(off32 * rho32);
  uint8_t* outr = row_of<kType>(a.out, at, a.out_stride);
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = width - col;
    float v[8], w[8], y[8];
    forget(g[i]);
    forget(t[i]);
    to_f32<kType>(g[i], v);
    to_f32<kType>(t[i], w);
    float size = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = kOut == kNormSame ? s[i][e] : s[i][e] - m;
      const float ng = (d - off32) * rho32 * v[e];
      y[e] = ng + w[e];
      size = __builtin_fmaxf(size, fused(far, __builtin_fabsf(v[e]), __builtin_fabsf(ng) + __builtin_fabsf(w[e])));
    }
    if (n <= 0) continue;
    if constexpr (kOut == kNormSame) {
      store_run<kType>(outr, col, n, from_f32<kType>(y));
    } else {
      // the four lanes of a block are inside the row or outside it together
      const uint32_t sc = block_scale<(kOut == kNormMxfp8 ? 8 : 2)>(y, size, [&](int e) {
        float x = s[i][e];
        asm volatile("" : "+v"(x));   // converted here, where it is rarely needed, and not kept in 64 bits
        return ((double)x - mean_) * rho * (double)v[e] + (double)w[e];
      });
      const float inv = inverse_scale(sc);
      if constexpr (kOut == kNormMxfp8)
        *reinterpret_cast<u32x2_t*>(a.codes + at * a.width + col) = e4m3_codes(y, inv);
      else
        *reinterpret_cast<uint32_t*>(a.codes + (at * a.width + col) / 2) = e2m1_codes(y, inv);
      if ((threadIdx.x & 3) == 0) a.scales[(at * a.width + col) / 32] = (uint8_t)sc;
    }
  }
}

template <int kType, int kOut>
static auto norm_kernel(int runs) {
  switch (runs) {
    case 1: return add_layernorm_kernel<kType, kOut, 1>;
    case 2: return add_layernorm_kernel<kType, kOut, 2>;
    case 3: return add_layernorm_kernel<kType, kOut, 3>;
    case 4: return add_layernorm_kernel<kType, kOut, 4>;
    case 5: return add_layernorm_kernel<kType, kOut, 5>;
    default: return add_layernorm_kernel<kType, kOut, 6>;
  }
}

template <int kType, int kOut>
static hipError_t launch_norm(LayerNormArgs a, hipStream_t stream) {
  const RowShape sh = row_shape(a.n.width, kNormRuns<kType>);
  const int waves = sh.wpr > 4 ? sh.wpr : 4, slots = sh.waves_slots(waves);
  const int64_t most = kMaxThreads / (waves * kWave) * slots;   // rows of one launch
  for (a.n.first = 0; a.n.first < a.n.rows; a.n.first += most) {
    const int64_t rows = a.n.rows - a.n.first < most ? a.n.rows - a.n.first : most;
    const hipError_t e = launch_kernel(norm_kernel<kType, kOut>(sh.runs), dim3((unsigned)((rows + slots - 1) / slots)),
                                       dim3(waves * kWave), stream, a, sh);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int kType>
static hipError_t launch_norm_type(const LayerNormArgs& a, int out, hipStream_t stream) {
  if (out == kNormSame) return launch_norm<kType, kNormSame>(a, stream);
  if (out == kNormMxfp8) return launch_norm<kType, kNormMxfp8>(a, stream);
  return launch_norm<kType, kNormMxfp4>(a, stream);
}

hipError_t launch_add_layernorm(int type, int out, const LayerNormArgs& a, hipStream_t stream) {
  if (a.n.rows == 0 || a.n.width == 0) return hipSuccess;
  if (type == SOLFP4_BF16) return launch_norm_type<SOLFP4_BF16>(a, out, stream);
  if (type == SOLFP4_F16) return launch_norm_type<SOLFP4_F16>(a, out, stream);
  return launch_norm_type<SOLFP4_F32>(a, out, stream);
}

// ---- backward -------------------------------------------------------------

// Runs a lane above which a row gets more waves.  A row needs two exchanges
// between its waves, so in 16 bits one wave with all of the row in up to 256
// registers, two waves a SIMD, is faster than two to four waves with 128 (BF16
// with up to six and two runs: 26574 x 2432 121 and 143 us, 6000 x 9728 125 and
// 141, 30000 x 1152 67 and 78; 10000 x 5600 122 and 119).  FP32 rows would spill
// (12000 x 2432 102 us with two, 108 with three).
template <int kType>
constexpr int kLayerBackRuns = kType == SOLFP4_F32 ? 2 : 6;

// ds of every row, and each workgroup's share of dg and dt: rows are dealt to
// the workgroups as in the root-mean-square norm's backward pass, all of a
// row's loads go out before the first use and stay as they were read.  dt is
// summed in LDS and the gain kept there, each lane's in places of its own: with
// all of it in registers the kernel spilled (26574 x 2432 BF16 371 us).
//
// Bound by memory, 8 bytes an element in BF16 with dsum, and by how few waves
// hold it in flight: 26574 x 2432 in 6 groups 120 us, 4.3 TB/s; FP32 1009 x 1283
// 13.3 us.
// kWhole: the width is a multiple of 8.
template <int kType, int kRuns, bool kWhole>
__global__ __launch_bounds__(kNormMaxWaves * kWave, 2) void layernorm_backward_kernel(LayerNormBackArgs p, RowShape sh) {
  __shared__ float lds[kNormMaxWaves][4], lds_mean[kNormMaxWaves][1];
  __shared__ __attribute__((aligned(16))) float fold[kRuns][kNormMaxWaves * kWave * 8];
  const NormBackArgs& a = p.n;
  const Place<kRuns> at_(sh);
  const int slots = sh.waves_slots(kNormMaxWaves), slot = at_.slot, lane = at_.lane, step = at_.step;
  const int group = blockIdx.x / a.parts, part = blockIdx.x - group * a.parts;
  const uint32_t rows = (uint32_t)a.group_rows;   // a hop past its end still fits 32 bits
  const int64_t row0 = group * a.group_rows;
  // the gain, each lane's in places of its own
  constexpr bool kGainInLds = kRuns <= kLayerBackRuns<kType>;
  __shared__ u32x4_t gains[kGainInLds ? kRuns * kRunPieces<kType> : 1][kNormMaxWaves * kWave];
  Run<kType> g[kGainInLds ? 1 : kRuns];
  const uint8_t* gr = row_of<kType>(a.gain, group, a.gain_stride);
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int col = i * step + lane * 8, n = (int)a.width - col;
    Run<kType> v = one_run<kType>();
    if (a.gain && n > 0) v = load_run<kType>(gr, col, n);
    if constexpr (kGainInLds) {
#pragma unroll
      for (int k = 0; k < kRunPieces<kType>; ++k) gains[i * kRunPieces<kType> + k][threadIdx.x] = v.p[k];
    } else {
      g[i] = v;
    }
  }
  const auto gain_run = [&](int i) {
    if constexpr (kGainInLds) {
      Run<kType> v;
      asm volatile("" ::: "memory");   // read again where it is used again
#pragma unroll
      for (int k = 0; k < kRunPieces<kType>; ++k) v.p[k] = gains[i * kRunPieces<kType> + k][threadIdx.x];
      return v;
    } else {
      forget(g[i]);
      return g[i];
    }
  };
  const int cols = sh.wpr * sh.lanes * 8;
  float dg[kRuns][8] = {};
  floatx4_t* const mine = reinterpret_cast<floatx4_t*>(fold[0] + slot * cols + lane * 8);
  constexpr int kNext = kNormMaxWaves * kWave * 2;   // from a run's place to the next's, in fours
  if (p.shift_partial)
#pragma unroll
    for (int i = 0; i < kRuns; ++i) mine[i * kNext] = mine[i * kNext + 1] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t base = part * slots; base < rows; base += a.parts * slots) {
    const bool in = base + slot < rows;
    const int64_t row = row0 + (in ? base + slot : base);
    const int width = in ? (int)a.width : 0;
    using Row = std::conditional_t<(kRuns > 1), BufferRow<kType, kWhole>, LaneRow<kType>>;
    const Row xr(row_of<kType>(a.x, row, a.x_stride), width), dr(row_of<kType>(a.dy, row, a.dy_stride), width);
    const Row er(row_of<kType>(a.dsum, row, a.dsum_stride), a.dsum ? width : 0);
    Run<kType> x[kRuns], d[kRuns], ex[kRuns];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int col = i * step + lane * 8, n = width - col;
      x[i] = xr.load(col, n);
      d[i] = dr.load(col, n);
      ex[i] = er.load(col, a.dsum ? n : 0);
    }
    float mean[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kRuns; ++i) mean[0] = add_run<kType>(x[i], mean[0]);
    row_sum<false>(mean, lds_mean, at_.wave, sh);
    const float m = mean[0] / (float)a.width;
    float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // d, d^2, G, G d
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      float s[8], D[8], v[8];
      forget(x[i]);
      to_f32<kType>(x[i], s);
      differences(s, m, width - (i * step + lane * 8), kWhole);
      to_f32<kType>(d[i], D);
      to_f32<kType>(gain_run(i), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float G = D[e] * v[e];
        q[0] += s[e];
        q[1] = fused(s[e], s[e], q[1]);
        q[2] += G;
        q[3] = fused(G, s[e], q[3]);
      }
    }
    row_sum<false>(q, lds, at_.wave, sh);
    const float off = q[0] / (float)a.width;
    // 0 where the slot has no row: with eps = 0 its zeros would add 0 times infinity to dg
    const float rho = in ? 1.0f / __builtin_sqrtf(not_negative(q[1] / (float)a.width - off * off) + a.eps) : 0.0f;
    const float mg = q[2] / (float)a.width;
    const float k = fused(-off, q[2], q[3]) / (float)a.width * rho;   // mean(G n)
    const float away = -off * rho;
    const Row outr(row_of<kType>(a.dx, row, a.dx_stride), width);
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int col = i * step + lane * 8, n = width - col;
      float s[8], D[8], v[8], out[8];
      forget(x[i]);
      forget(d[i]);
      to_f32<kType>(x[i], s);
      to_f32<kType>(d[i], D);
      to_f32<kType>(gain_run(i), v);
      to_f32<kType>(ex[i], out);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float nrm = fused(s[e] - m, rho, away);
        dg[i][e] = fused(D[e], nrm, dg[i][e]);
        out[e] = fused(rho, fused(nrm, -k, fused(D[e], v[e], -mg)), out[e]);
      }
      outr.store(col, n, from_f32<kType>(out));
      if (p.shift_partial) {
        mine[i * kNext] += floatx4_t{D[0], D[1], D[2], D[3]};
        mine[i * kNext + 1] += floatx4_t{D[4], D[5], D[6], D[7]};
      }
      __builtin_amdgcn_sched_barrier(0);   // one run's values at a time in registers
    }
  }
  // every slot's sums in LDS: each thread adds some columns'
  const bool narrow = kRuns == 1 && sh.lanes < kWave;   // several slots a wave
  const int parts_of = narrow ? kNormMaxWaves : slots;
  const auto share = [&](float* partial) {
    float* part_row = partial + (int64_t)blockIdx.x * a.width;
    if (narrow) {
      // a wave's slots first, by lane exchange: up to 512 slots one after another took 7 us
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = mine[e / 4][e % 4];
        for (int hop = sh.lanes; hop < kWave; hop *= 2) v[e] += __shfl_xor(v[e], hop, kWave);
      }
      __syncthreads();
      floatx4_t* to = reinterpret_cast<floatx4_t*>(fold[0] + at_.wave * cols + lane * 8);
      if ((threadIdx.x & (kWave - 1)) < sh.lanes) {
        to[0] = floatx4_t{v[0], v[1], v[2], v[3]};
        to[1] = floatx4_t{v[4], v[5], v[6], v[7]};
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      for (int c = threadIdx.x; c < cols; c += kNormMaxWaves * kWave) {
        float t = fold[i][c];
        for (int z = 1; z < parts_of; ++z) t += fold[i][z * cols + c];
        if (i * step + c < a.width) part_row[i * step + c] = t;
      }
    }
  };
  if (p.shift_partial) {
    share(p.shift_partial);
    __syncthreads();
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    mine[i * kNext] = floatx4_t{dg[i][0], dg[i][1], dg[i][2], dg[i][3]};
    mine[i * kNext + 1] = floatx4_t{dg[i][4], dg[i][5], dg[i][6], dg[i][7]};
  }
  share(a.partial);
}

// dg and dt from the workgroups' shares, one a slice of the grid.
__global__ __launch_bounds__(kFoldCols * kFoldSlices) void layernorm_sums_kernel(const float* __restrict__ partial,
                                                                                  float* __restrict__ dgain,
                                                                                  const float* __restrict__ shift_partial,
                                                                                  float* __restrict__ dshift,
                                                                                  int64_t width, int parts) {
  const bool shift = blockIdx.z || !dgain;
  fold_parts(shift ? shift_partial : partial, shift ? dshift : dgain, width, parts);
}

template <int kType, bool kWhole>
static auto back_kernel(int runs) {
  switch (runs) {
    case 1: return layernorm_backward_kernel<kType, 1, kWhole>;
    case 2: return layernorm_backward_kernel<kType, 2, kWhole>;
    case 3: return layernorm_backward_kernel<kType, 3, kWhole>;
    case 4: return layernorm_backward_kernel<kType, 4, kWhole>;
    case 5: return layernorm_backward_kernel<kType, 5, kWhole>;
    default: return layernorm_backward_kernel<kType, 6, kWhole>;
  }
}

template <int kType>
static hipError_t launch_back(const LayerNormBackArgs& a, hipStream_t stream) {
  const RowShape sh = row_shape(a.n.width, kLayerBackRuns<kType>);
  return launch_kernel(a.n.width % 8 ? back_kernel<kType, false>(sh.runs) : back_kernel<kType, true>(sh.runs),
                       dim3((unsigned)(a.n.groups * a.n.parts)), dim3(kNormMaxWaves * kWave), stream, a, sh);
}

hipError_t launch_layernorm_backward(int type, LayerNormBackArgs a, float* dgain, float* dshift, hipStream_t stream) {
  NormBackArgs& n = a.n;
  if (n.width == 0 || n.groups == 0) return hipSuccess;
  hipError_t e = hipSuccess;
  const int64_t parts = rmsnorm_backward_parts(n.rows, n.width, n.groups);
  if (parts == 1) n.partial = dgain, a.shift_partial = dshift;   // the one workgroup's sums are the group's
  if (parts) {
    n.group_rows = n.rows / n.groups;
    n.parts = (int)parts;
    if (type == SOLFP4_BF16) e = launch_back<SOLFP4_BF16>(a, stream);
    else if (type == SOLFP4_F16) e = launch_back<SOLFP4_F16>(a, stream);
    else e = launch_back<SOLFP4_F32>(a, stream);
  }
  const unsigned sums = (dgain ? 1 : 0) + (dshift ? 1 : 0);
  if (e != hipSuccess || !sums || parts == 1) return e;
  const dim3 grid((unsigned)((n.width + kFoldCols - 1) / kFoldCols), (unsigned)n.groups, sums);
  return launch_kernel(layernorm_sums_kernel, grid, dim3(kFoldCols * kFoldSlices), stream,
                       dgain ? (const float*)n.partial : nullptr, dgain, (const float*)a.shift_partial, dshift, n.width,
                       (int)parts);
}

}  // namespace solfp4
