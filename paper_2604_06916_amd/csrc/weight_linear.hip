// Products of few tokens with 4-bit weights: BF16 activations that stay
// BF16 with NVFP4 or MXFP4 weights, and MXFP8 activations with MXFP4 weights.
//
//   out[m][n] = bf16(alpha * sum_k x[m][k] (s q)[n][k] + bias[n])
//
// Bound by reading the weight once: 4 x 18432 x 3072 NVFP4 8.9 us, 3.6 TB/s, of
// which loads, scales and the reduction alone take 7.5 to 8.5; 64 x 9728 x 2432
// MXFP8 9.7 us, the activations' way through L2 and LDS to 304 tiles of columns.
// A workgroup makes 16 NT outputs of 16 MT tokens; its waves share the
// reduction: each takes a run of K steps of 128, and their FP32 partial sums
// are added in wave order through LDS.  So even a narrow layer has enough
// 16-byte loads in flight, and the result does not depend on timing.
//
// A lane holds 32 consecutive weights of one row a step (16 bytes of codes);
// lane group g of four takes weights 32 g .. 32 g + 31.  For BF16 activations
// four v_mfma_f32_16x16x32_bf16 take 8 of them each, against the same 8
// activations of a token (a permutation of K, alike on both sides).  Weights
// become BF16 exactly: s q has at most 6 significant bits (E4M3 times E2M1),
// or 2 and a power of two.  So do MXFP8 activations (4 bits and a power of
// two) from 2^-133, BF16's smallest, on.  The scaled matrix instruction would
// take E2M1 against E4M3 as they are, but adds its 128 products with fewer
// bits than FP32: with 20-fold outliers among the activations its result was
// off by up to 1.4 times what any order of FP32 sums can be, at K = 160.
//
// Tokens are the columns of the matrix instruction, so up to 16 cost what
// one does; columns past M hold anything and are not stored.
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

constexpr int kWLStep = 128;      // K a step

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Between one wave's LDS accesses by some lanes and by others: they keep their
// order (the hardware runs a wave's LDS instructions in theirs, so no wait is
// needed).
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

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

// A workgroup's waves work alone until the end: each moves its steps from
// memory to a buffer of its own in LDS and reads the matrix instructions'
// operands from there.  Loads straight into operand order put every lane of
// a load on another row, one cache line a lane, and the address path (one
// line a cycle) took longer than the memory: 4 x 18432 x 3072 19 us that
// way.  Here 4 (weights), 16 (BF16) or 8 (MXFP8) neighbouring lanes read one
// row's 64, 256 or 128 bytes of a step.
//
// Loads of the activations alone in operand order, 64 bytes of a row by four
// lanes, were slower still (32 x 9728 x 2432 NVFP4 12.4 us for 9.2): the address
// path takes them at half its rate.
//
// kWhole: K % 128 == 0, no partial step.  One step is in flight in registers
// and one in the LDS buffer (two or four in registers: slower or the same).
// Pieces of 16 bytes are stored at their number XOR the row's, so that 16
// lanes that read one piece of 16 rows reach all banks.  Scales come four
// steps at a time for each wave by itself (all waves' steps at once by the
// workgroup: slower, by the barrier).
template <int kFormat, bool kX8, bool kWhole, int MT, int NT, int XR, int W>
__global__ __launch_bounds__(W * kWave) void weight_linear_kernel(WeightLinearArgs a, int tiles_m) {
  constexpr bool kNv = kFormat == SOLFP4_FORMAT_NVFP4;
  constexpr int kScaleStep = kNv ? 8 : 4;              // scale bytes of a row's step
  constexpr int kScaleRow = 4 * kScaleStep;            // of four steps: one batch
  constexpr int kStage = (NT + XR) * 1024, kPart = NT * MT * 1024, kScales = NT * 16 * kScaleRow;
  constexpr int kBuf = (kStage + kScales > kPart ? kStage + kScales : kPart);
  __shared__ __attribute__((aligned(16))) uint8_t lds[W][kBuf];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);   // uniform: offsets by step stay scalar
  const int r = lane & 15, g = lane >> 4;
  // the tiles of the same columns on one XCD, whose L2 then gets their weights
  // once (64 x 9728 x 2432 MXFP8 10.4 us and 27 MB read, 9.7 so)
  int tile_m = 0, tile_n = blockIdx.x;
  if (tiles_m > 1) tile_coords(tiles_m, gridDim.x / tiles_m, tile_m, tile_n);
  const int64_t n0 = (int64_t)tile_n * (16 * NT), m0 = (int64_t)tile_m * (16 * MT);
  // rows of this tile inside the operands
  const int rows_n = a.N - n0 < 16 * NT ? (int)(a.N - n0) : 16 * NT;
  const int rows_m = a.M - m0 < 16 * MT ? (int)(a.M - m0) : 16 * MT;
  const int K = (int)a.K;
  const int steps = (K + kWLStep - 1) / kWLStep;
  const int first = steps * wave / W, last = steps * (wave + 1) / W;
  uint8_t* const lw = lds[wave];
  uint8_t* const lx = lw + NT * 1024;
  uint8_t* const ls = lw + kStage;

  // weights: lane l moves piece l % 4 (32 weights) of row l / 4
  const int w_row = K / 2;
  const __amdgpu_buffer_rsrc_t rw = uniform_rsrc(a.w_codes + n0 * w_row, (int64_t)rows_n * w_row);
  const int wr = lane >> 2, wp = lane & 3;
  uint32_t w_off[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) w_off[t] = (uint32_t)((16 * t + wr) * w_row + 16 * wp);
  uint8_t* const w_to = lw + wr * 64 + 16 * (wp ^ (wr >> 2));
  const uint8_t* const w_from = lw + r * 64 + 16 * (g ^ (r >> 2));
  // activations: lane l moves piece l % P of row l / P (+ 64 / P a load)
  constexpr int P = kX8 ? 8 : 16;
  constexpr int kTokens = XR * 64 / P;   // rows in LDS: fewer than 16 MT where M has no more; others repeat them
  const int x_row = K * (kX8 ? 1 : 2);
  const __amdgpu_buffer_rsrc_t rx =
      uniform_rsrc(static_cast<const uint8_t*>(a.x) + m0 * x_row, (int64_t)rows_m * x_row);
  const int xr = lane / P, xp = lane % P;
  uint32_t x_off[XR];
#pragma unroll
  for (int j = 0; j < XR; ++j) x_off[j] = (uint32_t)((j * (64 / P) + xr) * x_row + 16 * xp);
  // MXFP8's scales: lane (r, g) holds block g of token r
  const uint8_t* xs[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) xs[t] = kX8 ? a.x_scales + (m0 + (16 * t + r < rows_m ? 16 * t + r : rows_m - 1)) * (K / 32) + g : nullptr;
  // weight scales: a batch's kScaleRow bytes of a row in pieces of 16
  constexpr int kScalePieces = kScaleRow / 16;
  constexpr int kScaleLoads = (NT * 16 * kScalePieces + kWave - 1) / kWave;
  const int scale_row = K / (kNv ? 16 : 32);
  const __amdgpu_buffer_rsrc_t rs =
      uniform_rsrc(a.w_scales + n0 * scale_row, (int64_t)rows_n * scale_row);
  uint32_t s_off[kScaleLoads];
#pragma unroll
  for (int i = 0; i < kScaleLoads; ++i) {
    const int p = i * kWave + lane;
    s_off[i] = (uint32_t)(p / kScalePieces * scale_row + 16 * (p % kScalePieces));
  }

  struct Regs {
    u32x4_t w[NT], x[XR];
    uint32_t xs[MT];
  };
  // Step s into registers.  Where K ends inside it, pieces past the end are
  // zeros: the activations' too, since zero times what lies there could be NaN.
  auto load = [&](Regs& o, int s) {
    if (kWhole || K - s * kWLStep >= kWLStep) {
#pragma unroll
      for (int t = 0; t < NT; ++t) o.w[t] = __builtin_amdgcn_raw_buffer_load_b128(rw, w_off[t], s * (kWLStep / 2), 0);
#pragma unroll
      for (int j = 0; j < XR; ++j)
        o.x[j] = __builtin_amdgcn_raw_buffer_load_b128(rx, x_off[j], s * (kWLStep * (kX8 ? 1 : 2)), 0);
      if constexpr (kX8) {
#pragma unroll
        for (int t = 0; t < MT; ++t) o.xs[t] = xs[t][s * (kWLStep / 32)];
      }
      return;
    }
    const int left = K - s * kWLStep;
    constexpr uint32_t kOutside = 0x80000000u;   // beyond any operand's range (below 2^31): reads zero
#pragma unroll
    for (int t = 0; t < NT; ++t)
      o.w[t] = __builtin_amdgcn_raw_buffer_load_b128(rw, 32 * wp < left ? w_off[t] + s * (kWLStep / 2) : kOutside, 0, 0);
#pragma unroll
    for (int j = 0; j < XR; ++j)
      o.x[j] = __builtin_amdgcn_raw_buffer_load_b128(
          rx, (kX8 ? 16 : 8) * xp < left ? x_off[j] + s * (kWLStep * (kX8 ? 1 : 2)) : kOutside, 0, 0);
    if constexpr (kX8) {
#pragma unroll
      for (int t = 0; t < MT; ++t) o.xs[t] = 32 * g < left ? xs[t][s * (kWLStep / 32)] : 0u;
    }
  };
  // half of the last 32 weights can be the next row's (K % 32 == 16)
  auto trim = [&](Regs& o, int s) {
    if constexpr (kNv && !kWhole) {
      if (K - s * kWLStep - 32 * wp == 16) {
#pragma unroll
        for (int t = 0; t < NT; ++t) o.w[t][2] = o.w[t][3] = 0;
      }
    }
  };
  // Scales of the four steps from s on; bytes past the row's end are zeros.
  // Near it the load starts early enough to end with the row (a load's range
  // check would drop bytes that share a word with the operand's end) and the
  // bytes are moved down; rows under 16 bytes go byte by byte.
  auto load_scales = [&](u32x4_t (&o)[kScaleLoads], int s) {
    const int at = s * kScaleStep;
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
      const int p = i * kWave + lane;
      if (kScaleLoads * kWave > NT * 16 * kScalePieces && p >= NT * 16 * kScalePieces) continue;
      if (at + kScaleRow <= scale_row) {
        o[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, s_off[i], at, 0);
        continue;
      }
      const int n = scale_row - at - 16 * (p % kScalePieces);   // bytes from the piece to the row's end
      if (scale_row >= 16) {
        const int back = n >= 16 ? 0 : n > 0 ? 16 - n : 16;
        u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(rs, n > 0 ? s_off[i] + at - back : s_off[i], 0, 0);
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d] = __builtin_amdgcn_alignbyte(d < 3 ? v[d + 1] : 0u, v[d], back & 3);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int d = 0; d < 4; ++d) v[d] = back & (4 << h) ? (d + (1 << h) < 4 ? v[d + (1 << h)] : 0u) : v[d];
#pragma unroll
        for (int d = 0; d < 4; ++d) o[i][d] = back & 16 ? 0u : v[d];
        continue;
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint32_t v = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b)
          if (4 * d + b < n) v |= (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rs, s_off[i] + at + 4 * d + b, 0, 0) << (8 * b);
        o[i][d] = v;
      }
    }
  };

  floatx4_t acc[NT][MT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < MT; ++u) acc[t][u] = floatx4_t{0, 0, 0, 0};

  u32x4_t sreg[kScaleLoads];
  Regs c;
  if (first < last) {
    load_scales(sreg, first);
    load(c, first);
  }

  for (int s = first; s < last; s += 4) {
    wave_order();
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
      if (i * kWave + lane < NT * 16 * kScalePieces)
        *reinterpret_cast<u32x4_t*>(ls + 16 * (i * kWave + lane)) = sreg[i];
    if (s + 4 < last) load_scales(sreg, s + 4);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (s + v >= last) break;
      if (s + v == steps - 1) trim(c, s + v);
      if (v > 0) wave_order();
#pragma unroll
      for (int t = 0; t < NT; ++t) *reinterpret_cast<u32x4_t*>(w_to + t * 1024) = c.w[t];
#pragma unroll
      for (int j = 0; j < XR; ++j) {
        const int row = j * (64 / P) + xr;
        *reinterpret_cast<u32x4_t*>(lx + row * (16 * P) + 16 * (xp ^ (row & (P - 1)))) = c.x[j];
      }
      wave_order();
      uint32_t sx[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) sx[t] = kX8 ? c.xs[t] : 0u;
      if (s + v + 1 < last) load(c, s + v + 1);

      bf16x8_t x[MT][4];
#pragma unroll
      for (int u = 0; u < MT; ++u) {
        const int row = (16 * u + r) & (kTokens - 1);
        if constexpr (kX8) {
          u32x4_t h[2];
#pragma unroll
          for (int j = 0; j < 2; ++j)
            h[j] = *reinterpret_cast<const u32x4_t*>(lx + row * 128 + 16 * ((2 * g + j) ^ (row & 7)));
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[u][j] = activations8(h[j / 2][2 * (j & 1)], h[j / 2][2 * (j & 1) + 1], e8m0_float(sx[u]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[u][j] = *reinterpret_cast<const bf16x8_t*>(lx + row * 256 + 16 * ((4 * g + j) ^ (row & 15)));
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(w_from + t * 1024);
        const uint8_t* sc = ls + (16 * t + r) * kScaleRow + v * kScaleStep;
        float f[2];
        if constexpr (kNv) {
          const int two = *reinterpret_cast<const uint16_t*>(sc + 2 * g);
          f[0] = __builtin_amdgcn_cvt_f32_fp8(two, 0);
          f[1] = __builtin_amdgcn_cvt_f32_fp8(two, 1);
        } else {
          f[0] = f[1] = e8m0_float(sc[g]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8_t b = weights8<kFormat>(w[j], f[j / 2]);
#pragma unroll
          for (int u = 0; u < MT; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, x[u][j], acc[t][u], 0, 0, 0);
        }
      }
    }
  }

  // each wave's sums in place of its buffer, after its reads
  wave_order();
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < MT; ++u) reinterpret_cast<floatx4_t*>(lw)[(t * MT + u) * kWave + lane] = acc[t][u];
  __syncthreads();

  // a lane of tile (t, u) holds outputs n0 + 16 t + 4 g .. + 3 of token m0 + 16 u + r
  const float alpha = kNv ? a.w_global[0] : 1.0f;
  for (int q = wave; q < NT * MT; q += W) {
    floatx4_t v = reinterpret_cast<const floatx4_t*>(lds[0])[q * kWave + lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += reinterpret_cast<const floatx4_t*>(lds[w])[q * kWave + lane];
    const int64_t n = n0 + 16 * (q / MT) + 4 * g, m = m0 + 16 * (q % MT) + r;
    if (m >= a.M || n >= a.N) continue;
    typedef u32x2_t u32x2_at2 __attribute__((aligned(2)));
    float y[4];
    u32x2_t b = u32x2_t{0, 0};
    if (a.bias) {
      if (n + 4 <= a.N) {
        b = *reinterpret_cast<const u32x2_at2*>(a.bias + n);
      } else {
        b.x = a.bias[n] | (n + 1 < a.N ? (uint32_t)a.bias[n + 1] << 16 : 0u);
        b.y = n + 2 < a.N ? a.bias[n + 2] : 0u;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = __builtin_fmaf(alpha, v[e], __uint_as_float(e & 1 ? b[e / 2] & 0xFFFF0000u : b[e / 2] << 16));
    const uint32_t p0 = pack_bf16(y[0], y[1]), p1 = pack_bf16(y[2], y[3]);
    uint16_t* o = a.out + m * a.N + n;
    if (n + 4 <= a.N) {
      *reinterpret_cast<u32x2_at2*>(o) = u32x2_t{p0, p1};
    } else {
      o[0] = (uint16_t)p0;
      if (n + 1 < a.N) o[1] = (uint16_t)(p0 >> 16);
      if (n + 2 < a.N) o[2] = (uint16_t)p1;
    }
  }
}

// The tile of a shape (us: NVFP4, MXFP4, MXFP8 x MXFP4).  A step brings 256 bytes a
// token and 64 a column into a wave's buffer, so wide tiles save the
// activations' way from L2 and LDS; narrow ones make more workgroups and
// shorter steps.
//
// Up to 16 tokens, 16 columns a workgroup while that is at most one a CU.
// Past it, 32 columns (16 x 4500 x 12288 16.1, 14.9, 14.7 with 16 columns, 12.9, 10.6,
// 10.7 with 32), of eight waves up to one workgroup a CU and of four beyond (16 x
// 8300 x 5600 13.8, 12.2, 12.1 and 13.2, 11.7, 11.7), of which more fit a CU.  So `few`
// tokens that one load brings (4 in BF16, 8 in MXFP8) keep 16 columns: 16 waves up
// to one workgroup a CU (4 x 3072 x 12288 8.1, 6.9, 7.7 with 8 and 7.5, 6.2, 6.4
// with 16), then eight (4 x 4500 x 12288 13.0, 10.6, 11.0 with 16 and 11.8, 9.6,
// 9.9 with 8), and four once eight would start a second round of workgroups
// (more than four a CU: 8 x 18000 x 512 5.6, 5.0, 4.8 and 4.2, 3.9, 4.1).
//
// Beyond, 32 tokens a workgroup, and 16, 32 or 64 columns.  16 up to half a CU
// of 32-column workgroups (64 x 1235 x 9728 11.4, 10.4, 9.0; 14.5, 12.0, 10.9 with
// 32), 32 up to a whole one (64 x 3072 x 12288 17.6, 14.5, 14.7; 22.8, 21.2, 22.3
// with 16), 64 while those are at most one a CU (64 x 4500 x 12288 25.6, 19.8, 19.9;
// 30.5, 24.5, 25.9 with 32 and four waves, the best of the others), and past that
// 32 again, of four waves (64 x 9728 x 2432 12.3, 10.6, 9.8; 16.4, 14.1, 10.5 with
// eight, 13.8, 10.8, 10.2 with 64 columns).
struct Tile {
  int mt, nt, waves;
  int64_t groups(int64_t M, int64_t N) const { return ((M + 16 * mt - 1) / (16 * mt)) * ((N + 16 * nt - 1) / (16 * nt)); }
};

static Tile tile_of(int64_t M, int64_t N, bool few) {
  const int64_t cus = device_cu_count();
  if (M <= 16) {
    const int64_t narrow = Tile{1, 1, 0}.groups(M, N);
    if (few) return {1, 1, narrow <= cus ? 16 : narrow <= 4 * cus ? 8 : 4};
    if (narrow <= cus) return {1, 1, 8};
    return {1, 2, Tile{1, 2, 0}.groups(M, N) <= cus ? 8 : 4};
  }
  const int64_t wide = Tile{2, 2, 0}.groups(M, N);
  if (wide <= cus / 2) return {2, 1, 8};
  if (wide <= cus) return {2, 2, 8};
  if (Tile{2, 4, 0}.groups(M, N) <= cus) return {2, 4, 8};
  return {2, 2, 4};
}

template <int kFormat, bool kX8, int MT, int NT, int XR, int W>
static hipError_t launch_tile(const WeightLinearArgs& a, hipStream_t stream) {
  const auto kernel = a.K % kWLStep == 0 ? weight_linear_kernel<kFormat, kX8, true, MT, NT, XR, W>
                                         : weight_linear_kernel<kFormat, kX8, false, MT, NT, XR, W>;
  // tokens of one launch, by whole tiles (N < 2^22 leaves at least one)
  const int64_t most = kMaxThreads / (W * kWave) / Tile{MT, NT, W}.groups(1, a.N) * (16 * MT);
  for (int64_t m = 0; m < a.M; m += most) {
    WeightLinearArgs p = a;
    p.M = a.M - m < most ? a.M - m : most;
    p.x = static_cast<const uint8_t*>(a.x) + m * a.K * (kX8 ? 1 : 2);
    if (kX8) p.x_scales += m * (a.K / 32);
    p.out += m * a.N;
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)Tile{MT, NT, W}.groups(p.M, p.N)), dim3(W * kWave), stream,
                                       p, (int)((p.M + 16 * MT - 1) / (16 * MT)));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int kFormat, bool kX8>
static hipError_t launch_format(const WeightLinearArgs& a, hipStream_t stream) {
  constexpr int kFull = kX8 ? 2 : 4;   // loads of 16 tokens' step
  // as few activation rows as one load brings need no more LDS than that
  const bool few = a.M <= 16 / kFull;
  const Tile t = tile_of(a.M, a.N, few);
  if (few) {
    if (t.waves == 16) return launch_tile<kFormat, kX8, 1, 1, 1, 16>(a, stream);
    if (t.waves == 8) return launch_tile<kFormat, kX8, 1, 1, 1, 8>(a, stream);
    return launch_tile<kFormat, kX8, 1, 1, 1, 4>(a, stream);
  }
  if (t.mt == 1) {
    if (t.nt == 1) return launch_tile<kFormat, kX8, 1, 1, kFull, 8>(a, stream);
    if (t.waves == 8) return launch_tile<kFormat, kX8, 1, 2, kFull, 8>(a, stream);
    return launch_tile<kFormat, kX8, 1, 2, kFull, 4>(a, stream);
  }
  if (t.nt == 1) return launch_tile<kFormat, kX8, 2, 1, 2 * kFull, 8>(a, stream);
  if (t.nt == 4) return launch_tile<kFormat, kX8, 2, 4, 2 * kFull, 8>(a, stream);
  if (t.waves == 8) return launch_tile<kFormat, kX8, 2, 2, 2 * kFull, 8>(a, stream);
  return launch_tile<kFormat, kX8, 2, 2, 2 * kFull, 4>(a, stream);
}

hipError_t launch_weight_linear(int w_format, bool x_mxfp8, const WeightLinearArgs& a, hipStream_t stream) {
  if (a.M == 0 || a.N == 0) return hipSuccess;
  if (x_mxfp8) return launch_format<SOLFP4_FORMAT_MXFP4, true>(a, stream);
  if (w_format == SOLFP4_FORMAT_NVFP4) return launch_format<SOLFP4_FORMAT_NVFP4, false>(a, stream);
  return launch_format<SOLFP4_FORMAT_MXFP4, false>(a, stream);
}

}  // namespace solfp4
