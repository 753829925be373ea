// What the adapters' kernels share: the plan, matrix operands, roundings.
#pragma once

#include "elements.h"
#include "kernels.h"

namespace solfp4 {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 8 consecutive BF16 values of `row` from element `at`; zeros from element `end`
// (uniform), the row's end, on.  One load without a branch: near the end of the
// row's last 8 values, moved down (element by element, each with a branch and a
// wait, 1371 x 1235 x 1111 took 25 us).
__device__ __forceinline__ bf16x8_t operand8(const uint16_t* row, uint32_t at, uint32_t end) {
  u32x4_t v = {0, 0, 0, 0};
  if (end < 8) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (at + e < end) v[e / 2] |= (uint32_t)row[at + e] << (16 * (e & 1));
    return __builtin_bit_cast(bf16x8_t, v);
  }
  const uint32_t from = min(at, end - 8), by = at - from;
  v = *reinterpret_cast<const u32x4_at2*>(row + from);
  if (by & 4) v = u32x4_t{v.z, v.w, 0, 0};
  if (by & 2) v = u32x4_t{v.y, v.z, v.w, 0};
  if (by & 1)
    v = u32x4_t{__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16),
                __builtin_amdgcn_alignbit(v.w, v.z, 16), v.w >> 16};
  if (by >= 8) v = u32x4_t{0, 0, 0, 0};
  return __builtin_bit_cast(bf16x8_t, v);
}

// The same where all 8 exist.
__device__ __forceinline__ bf16x8_t operand8(const uint16_t* at) {
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_at2*>(at));
}

// A lane's kCols (8 or 4) consecutive columns of a row.
template <int kCols>
struct LaneRun {
  typedef uint32_t words_t __attribute__((ext_vector_type(kCols / 2)));
  typedef words_t words_at2_t __attribute__((aligned(2)));
  words_t w;
  // Columns col and up, where all of them exist, or zeros from column `end` on.
  __device__ __forceinline__ void load(const uint16_t* row, uint32_t col, uint32_t end, bool whole) {
    if (whole) {
      w = *reinterpret_cast<const words_at2_t*>(row + col);
    } else {
      const u32x4_t v = __builtin_bit_cast(u32x4_t, operand8(row, col, end));
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) w[i] = v[i];
    }
  }
  // The same in two steps, so that the first waits for nothing: near the row's end
  // its last kCols values, which settle() then moves down.
  __device__ __forceinline__ void load_raw(const uint16_t* row, uint32_t col, uint32_t end) {
    if (end < kCols) load(row, col, end, false);
    else w = *reinterpret_cast<const words_at2_t*>(row + min(col, end - kCols));
  }
  __device__ __forceinline__ void settle(uint32_t col, uint32_t end) {
    if (end < kCols) return;
    const uint32_t by = col - min(col, end - kCols);
    constexpr int kWords = kCols / 2;
#pragma unroll
    for (int hop = kWords / 2; hop; hop /= 2)
      if (by & 2 * hop)
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = i + hop < kWords ? w[i + hop] : 0;
    if (by & 1)
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = i + 1 < kWords ? __builtin_amdgcn_alignbit(w[i + 1], w[i], 16) : w[i] >> 16;
    if (by >= kCols) w = words_t{};
  }
  __device__ __forceinline__ float value(int e) const {
    return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[kCols]) {
#pragma unroll
    for (int e = 0; e < kCols; e += 2) w[e / 2] = pack_bf16(v[e], v[e + 1]);
  }
  __device__ __forceinline__ void store(uint16_t* row, uint32_t col, uint32_t end, bool whole) const {
    if (whole) {
      *reinterpret_cast<words_at2_t*>(row + col) = w;
    } else {
#pragma unroll
      for (int e = 0; e < kCols; ++e)
        if (col + e < end) row[col + e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
  }
};

// Between one wave's LDS writes by some lanes and reads by others: the hardware
// keeps a wave's LDS instructions in order, the compiler is told to.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
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

// As read, without waiting for it: made uniform, and within the plan's bounds,
// where it is used.
__device__ __forceinline__ Tile load_tile(const AdapterTokens& t, int i) {
  if (t.plan) {
    const int* p = t.plan + t.tiles_at + 4 * (int64_t)i;
    return {p[0], p[1], p[2]};
  }
  const int64_t first = (int64_t)i * kAdapterTile, left = t.tokens - first;
  return {0, (int)first, (int)(left < kAdapterTile ? left : kAdapterTile)};
}

// A plan's memory that no call has written yet (a captured one before its first
// replay) may hold anything: wrong results, but no access outside the operands.
__device__ __forceinline__ Tile uniform(const AdapterTokens& t, Tile tile) {
  const uint32_t group = (uint32_t)__builtin_amdgcn_readfirstlane(tile.group);
  const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane(tile.first);
  const uint32_t count = (uint32_t)__builtin_amdgcn_readfirstlane(tile.count);
  const uint32_t place = min(first, (uint32_t)t.tokens - 1u);
  return {(int)min(group, (uint32_t)t.adapters + 1u), (int)place,
          (int)min(min(count, (uint32_t)kAdapterTile), (uint32_t)t.tokens - place)};
}

// The token at place `at` of the order: as read, and within its bounds.
__device__ __forceinline__ uint32_t raw_token(const AdapterTokens& t, int at) {
  return t.plan ? (uint32_t)t.plan[t.order_at + at] : (uint32_t)at;
}
__device__ __forceinline__ uint32_t bounded_token(const AdapterTokens& t, uint32_t token) {
  return t.plan ? min(token, (uint32_t)t.tokens - 1u) : token;
}
__device__ __forceinline__ int64_t token_at(const AdapterTokens& t, int at) { return bounded_token(t, raw_token(t, at)); }

}  // namespace solfp4
