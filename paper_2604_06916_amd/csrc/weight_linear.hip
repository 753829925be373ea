// Products of few tokens with 4-bit weights: BF16 activations that stay
// BF16 with NVFP4 or MXFP4 weights, and MXFP8 activations with MXFP4 weights.
//
//   out[m][n] = bf16(alpha * sum_k x[m][k] (s q)[n][k] + bias[n])
//
// Bound by reading the weight once.  A workgroup makes 16 NT outputs of
// 16 MT tokens; its waves share the reduction: each takes a run of K steps
// of 128, and their FP32 partial sums are added in wave order through LDS.
// So even a narrow layer has enough 16-byte loads in flight, and the result
// does not depend on timing.
//
// A lane holds 32 consecutive weights of one row a step (16 bytes of codes);
// lane group g of four takes weights 32 g .. 32 g + 31.  For BF16 activations
// four v_mfma_f32_16x16x32_bf16 take 8 of them each, against the same 8
// activations of a token (a permutation of K, alike on both sides).  Weights
// become BF16 exactly: s q has at most 6 significant bits (E4M3 times E2M1),
// or 2 and a power of two.  So do MXFP8 activations (4 bits and a power of
// two).  The scaled matrix instruction would take E2M1 against E4M3 as they
// are, but adds its 128 products with fewer bits than FP32: with 20-fold
// outliers among the activations its result was off by up to 1.4 times what
// any order of FP32 sums can be, at K = 160.
//
// Tokens are the columns of the matrix instruction, so up to 16 cost what
// one does; token rows past M repeat the last one and are not stored.
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

constexpr int kWLStep = 128;      // K a step

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// An E8M0 byte as the converters take it (they read the exponent field: 0 is 2^-127).
__device__ __forceinline__ float e8m0_float(uint32_t b) { return __uint_as_float(b << 23); }

// 8 E4M3 activations (two words) as BF16, times the block's scale
__device__ __forceinline__ bf16x8_t activations8(uint32_t lo, uint32_t hi, float s) {
  u32x4_t r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true));
  return __builtin_bit_cast(bf16x8_t, r);
}

// 8 weights (one word of codes) as BF16, times the block's scale
template <int kFormat>
__device__ __forceinline__ bf16x8_t weights8(uint32_t c, float s) {
  u32x4_t r;
  if constexpr (kFormat == SOLFP4_FORMAT_MXFP4) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  } else {
    const floatx2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    const floatx2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    const floatx2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    const floatx2_t e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    r[0] = pack_bf16(a.x * s, a.y * s);
    r[1] = pack_bf16(b.x * s, b.y * s);
    r[2] = pack_bf16(d.x * s, d.y * s);
    r[3] = pack_bf16(e.x * s, e.y * s);
  }
  return __builtin_bit_cast(bf16x8_t, r);
}

// A lane's operands of one step
template <bool kX8, int MT, int NT>
struct Step {
  u32x4_t w[NT];
  uint32_t ws[NT];                 // scale bytes of the lane's 32 weights
  u32x4_t x[MT][kX8 ? 2 : 4];
  uint32_t xs[MT];                 // kX8
};

template <int kFormat, bool kX8, int MT, int NT, int W, int U>
__global__ __launch_bounds__(W * kWave) void weight_linear_kernel(WeightLinearArgs a, int tiles_m) {
  __shared__ floatx4_t part[W][NT * MT][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)(blockIdx.x / tiles_m) * (16 * NT);
  const int64_t m0 = (int64_t)(blockIdx.x % tiles_m) * (16 * MT);
  constexpr int kBlocks = kFormat == SOLFP4_FORMAT_NVFP4 ? 2 : 1;   // scale bytes of 32 weights
  const int K = (int)a.K;
  const int steps = (K + kWLStep - 1) / kWLStep;
  const int first = steps * wave / W, last = steps * (wave + 1) / W;

  const uint8_t *wc[NT], *ws[NT], *x[MT], *xs[MT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t n = min(n0 + 16 * t + r, a.N - 1);
    wc[t] = a.w_codes + n * (K / 2) + 16 * g;
    ws[t] = a.w_scales + n * (K / (32 / kBlocks)) + kBlocks * g;
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = min(m0 + 16 * t + r, a.M - 1);
    x[t] = static_cast<const uint8_t*>(a.x) + m * K * (kX8 ? 1 : 2) + (kX8 ? 32 : 64) * g;
    xs[t] = kX8 ? a.x_scales + m * (K / 32) + g : nullptr;
  }

  floatx4_t acc[NT][MT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < MT; ++u) acc[t][u] = floatx4_t{0, 0, 0, 0};

  // loads of step s; a step that K ends in loads only what is there and
  // leaves zeros (weights and activations both: zero times what lies
  // past the end could be a NaN)
  auto load = [&](Step<kX8, MT, NT>& o, int s) {
    const int left = K - s * kWLStep;
    if (left >= kWLStep) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        o.w[t] = *reinterpret_cast<const u32x4_at2*>(wc[t] + s * (kWLStep / 2));
        const uint8_t* p = ws[t] + s * (kWLStep / 32 * kBlocks);
        if constexpr (kBlocks == 2) {
          typedef uint16_t u16_at1 __attribute__((aligned(1)));
          o.ws[t] = *reinterpret_cast<const u16_at1*>(p);
        } else {
          o.ws[t] = *p;
        }
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if constexpr (kX8) {
          o.x[t][0] = *reinterpret_cast<const u32x4_at2*>(x[t] + s * kWLStep);
          o.x[t][1] = *reinterpret_cast<const u32x4_at2*>(x[t] + s * kWLStep + 16);
          o.xs[t] = xs[t][s * (kWLStep / 32)];
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            o.x[t][j] = *reinterpret_cast<const u32x4_at2*>(x[t] + s * (2 * kWLStep) + 16 * j);
        }
      }
      return;
    }
    const int mine = left - 32 * g;   // of the lane's 32 elements, those inside K: a multiple of 16
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      o.w[t] = u32x4_t{0, 0, 0, 0};
      o.ws[t] = 0;
      const uint8_t* p = ws[t] + s * (kWLStep / 32 * kBlocks);
      const uint8_t* c = wc[t] + s * (kWLStep / 2);
      if (mine >= 32) {
        o.w[t] = *reinterpret_cast<const u32x4_at2*>(c);
        o.ws[t] = p[0] | (kBlocks == 2 ? (uint32_t)p[kBlocks - 1] << 8 : 0u);
      } else if (mine > 0) {
        typedef u32x2_t u32x2_at2 __attribute__((aligned(2)));
        const u32x2_t h = *reinterpret_cast<const u32x2_at2*>(c);
        o.w[t][0] = h.x;
        o.w[t][1] = h.y;
        o.ws[t] = p[0];
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      o.xs[t] = 0;
      if constexpr (kX8) {
        o.x[t][0] = o.x[t][1] = u32x4_t{0, 0, 0, 0};
        if (mine > 0) {   // whole blocks
          o.x[t][0] = *reinterpret_cast<const u32x4_at2*>(x[t] + s * kWLStep);
          o.x[t][1] = *reinterpret_cast<const u32x4_at2*>(x[t] + s * kWLStep + 16);
          o.xs[t] = xs[t][s * (kWLStep / 32)];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          o.x[t][j] = u32x4_t{0, 0, 0, 0};
          if (8 * j < mine) o.x[t][j] = *reinterpret_cast<const u32x4_at2*>(x[t] + s * (2 * kWLStep) + 16 * j);
        }
      }
    }
  };

  auto compute = [&](const Step<kX8, MT, NT>& o) {
    bf16x8_t x[MT][4];
#pragma unroll
    for (int u = 0; u < MT; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (kX8)
          x[u][j] = activations8(o.x[u][j / 2][2 * (j & 1)], o.x[u][j / 2][2 * (j & 1) + 1], e8m0_float(o.xs[u]));
        else
          x[u][j] = __builtin_bit_cast(bf16x8_t, o.x[u][j]);
      }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float s[2];
      if constexpr (kBlocks == 2) {
        s[0] = __builtin_amdgcn_cvt_f32_fp8((int)o.ws[t], 0);
        s[1] = __builtin_amdgcn_cvt_f32_fp8((int)o.ws[t], 1);
      } else {
        s[0] = s[1] = e8m0_float(o.ws[t]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8_t w = weights8<kFormat>(o.w[t][j], s[j / 2]);
#pragma unroll
        for (int u = 0; u < MT; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[u][j], acc[t][u], 0, 0, 0);
      }
    }
  };

  for (int s = first; s < last; s += U) {
    Step<kX8, MT, NT> o[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < last) load(o[u], s + u);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < last) compute(o[u]);
  }

#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < MT; ++u) part[wave][t * MT + u][lane] = acc[t][u];
  __syncthreads();

  // a lane of tile (t, u) holds outputs n0 + 16 t + 4 g .. + 3 of token m0 + 16 u + r
  const float alpha = kFormat == SOLFP4_FORMAT_NVFP4 ? a.w_global[0] : 1.0f;
  for (int q = wave; q < NT * MT; q += W) {
    floatx4_t v = part[0][q][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += part[w][q][lane];
    const int64_t n = n0 + 16 * (q / MT) + 4 * g, m = m0 + 16 * (q % MT) + r;
    if (m >= a.M || n >= a.N) continue;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float b = a.bias && n + e < a.N ? __uint_as_float((uint32_t)a.bias[n + e] << 16) : 0.0f;
      y[e] = __builtin_fmaf(alpha, v[e], b);
    }
    const uint32_t p0 = pack_bf16(y[0], y[1]), p1 = pack_bf16(y[2], y[3]);
    uint16_t* o = a.out + m * a.N + n;
    if (n + 4 <= a.N) {
      typedef u32x2_t u32x2_at2 __attribute__((aligned(2)));
      *reinterpret_cast<u32x2_at2*>(o) = u32x2_t{p0, p1};
    } else {
      o[0] = (uint16_t)p0;
      if (n + 1 < a.N) o[1] = (uint16_t)(p0 >> 16);
      if (n + 2 < a.N) o[2] = (uint16_t)p1;
    }
  }
}

static int tokens_tile(int64_t M) { return M <= 16 ? 1 : M <= 32 ? 2 : 4; }

// 16-column tiles of a workgroup
static int column_tiles(int64_t M, int64_t N) {
  (void)M;
  return N >= 4096 ? 2 : 1;
}

int64_t weight_linear_groups(int64_t M, int64_t N) {
  const int mt = tokens_tile(M), nt = column_tiles(M, N);
  return ((N + 16 * nt - 1) / (16 * nt)) * ((M + 16 * mt - 1) / (16 * mt));
}

template <int kFormat, bool kX8, int MT, int NT>
static hipError_t launch_tile(const WeightLinearArgs& a, hipStream_t stream) {
  constexpr int W = 8, U = MT == 1 ? 4 : 2;
  const int tiles_m = (int)((a.M + 16 * MT - 1) / (16 * MT));
  return launch_kernel(weight_linear_kernel<kFormat, kX8, MT, NT, W, U>, dim3((unsigned)weight_linear_groups(a.M, a.N)),
                       dim3(W * kWave), stream, a, tiles_m);
}

template <int kFormat, bool kX8>
static hipError_t launch_format(const WeightLinearArgs& a, hipStream_t stream) {
  const int mt = tokens_tile(a.M), nt = column_tiles(a.M, a.N);
  if (mt == 1) return nt == 1 ? launch_tile<kFormat, kX8, 1, 1>(a, stream) : launch_tile<kFormat, kX8, 1, 2>(a, stream);
  if (mt == 2) return nt == 1 ? launch_tile<kFormat, kX8, 2, 1>(a, stream) : launch_tile<kFormat, kX8, 2, 2>(a, stream);
  return nt == 1 ? launch_tile<kFormat, kX8, 4, 1>(a, stream) : launch_tile<kFormat, kX8, 4, 2>(a, stream);
}

hipError_t launch_weight_linear(int w_format, bool x_mxfp8, const WeightLinearArgs& a, hipStream_t stream) {
  if (a.M == 0 || a.N == 0) return hipSuccess;
  if (x_mxfp8) return launch_format<SOLFP4_FORMAT_MXFP4, true>(a, stream);
  if (w_format == SOLFP4_FORMAT_NVFP4) return launch_format<SOLFP4_FORMAT_NVFP4, false>(a, stream);
  return launch_format<SOLFP4_FORMAT_MXFP4, false>(a, stream);
}

}  // namespace solfp4
