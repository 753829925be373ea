// What the adapters' kernels share: the plan, matrix operands, roundings.
#pragma once

#include "elements.h"
#include "kernels.h"

namespace solfp4 {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 8 consecutive BF16 values of `row` from element `at`, of which n exist (zeros after them).
__device__ __forceinline__ bf16x8_t operand8(const uint16_t* row, uint32_t at, int n) {
  if (n <= 0) return __builtin_bit_cast(bf16x8_t, u32x4_t{0, 0, 0, 0});
  return __builtin_bit_cast(bf16x8_t, load_run<SOLFP4_BF16>(reinterpret_cast<const uint8_t*>(row), at, n).p[0]);
}

// The same where all 8 exist.
__device__ __forceinline__ bf16x8_t operand8(const uint16_t* at) {
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_at2*>(at));
}

// FP32 values as a sum of BF16 pieces, each the rest rounded to nearest: two
// hold 16 bits of a value and three all 24.  Where the value is no finite
// number (or rounds to none), the further pieces are 0, so a product with it
// is what the value's is.
template <int kPieces>
__device__ __forceinline__ void split_bf16(const float (&v)[8], bf16x8_t (&out)[kPieces]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
  for (int p = 0; p < kPieces; ++p) {
    u32x4_t w;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      w[e / 2] = pack_bf16(rest[e], rest[e + 1]);
      const float lo = __uint_as_float(w[e / 2] << 16), hi = __uint_as_float(w[e / 2] & 0xFFFF0000u);
      rest[e] = __builtin_fabsf(lo) < __builtin_inff() ? rest[e] - lo : 0.0f;
      rest[e + 1] = __builtin_fabsf(hi) < __builtin_inff() ? rest[e + 1] - hi : 0.0f;
    }
    out[p] = __builtin_bit_cast(bf16x8_t, w);
  }
}

__device__ __forceinline__ floatx4_t mfma(bf16x8_t a, bf16x8_t b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A tile: up to kAdapterTile tokens of one group, at places first .. first +
// count - 1 of the plan's order.
struct Tile {
  int group, first, count;
};

// As read, without waiting for it: made uniform where it is used.
__device__ __forceinline__ Tile load_tile(const AdapterTokens& t, int i) {
  if (t.plan) {
    const int* p = t.plan + t.tiles_at + 4 * (int64_t)i;
    return {p[0], p[1], p[2]};
  }
  const int64_t first = (int64_t)i * kAdapterTile, left = t.tokens - first;
  return {0, (int)first, (int)(left < kAdapterTile ? left : kAdapterTile)};
}

__device__ __forceinline__ Tile uniform(Tile t) {
  return {__builtin_amdgcn_readfirstlane(t.group), __builtin_amdgcn_readfirstlane(t.first),
          __builtin_amdgcn_readfirstlane(t.count)};
}

// The token at place `at` of the order.
__device__ __forceinline__ int64_t token_at(const AdapterTokens& t, int at) {
  return t.plan ? t.plan[t.order_at + at] : at;
}

}  // namespace solfp4
