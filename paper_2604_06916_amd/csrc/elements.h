// Runs of 8 elements of the operators' types (BF16, FP16, FP32) as FP32 values.
#pragma once

#include "device_common.h"
#include "solfp4.h"

namespace solfp4 {

// Vectors at any element boundary: rows of odd width or stride start at 2- or
// 4-byte addresses, where unaligned vector-memory access (on under HSA)
// still takes one 16-byte instruction.
typedef u32x4_t u32x4_at2 __attribute__((aligned(2)));
typedef u32x4_t u32x4_at4 __attribute__((aligned(4)));

template <int kType>
constexpr int kElemBytes = kType == SOLFP4_F32 ? 4 : 2;

// 16-byte pieces of a run of 8 elements
template <int kType>
constexpr int kRunPieces = kElemBytes<kType> * 8 / 16;

// A run as loaded: no conversion until it is used, so a loop's loads go out together.
template <int kType>
struct Run {
  u32x4_t p[kRunPieces<kType>];
};

template <int kType>
__device__ __forceinline__ Run<kType> zero_run() {
  Run<kType> r;
#pragma unroll
  for (int i = 0; i < kRunPieces<kType>; ++i) r.p[i] = u32x4_t{0, 0, 0, 0};
  return r;
}

// The run at element `at` of `base`, of which the first n elements exist
// (n >= 8: one vector load per piece; else element loads, zeros after them).
template <int kType>
__device__ __forceinline__ Run<kType> load_run(const void* base, int64_t at, int64_t n) {
  const uint8_t* a = static_cast<const uint8_t*>(base) + at * kElemBytes<kType>;
  Run<kType> r = zero_run<kType>();
  if (n >= 8) {
#pragma unroll
    for (int i = 0; i < kRunPieces<kType>; ++i) {
      if constexpr (kType == SOLFP4_F32)
        r.p[i] = *reinterpret_cast<const u32x4_at4*>(a + 16 * i);
      else
        r.p[i] = *reinterpret_cast<const u32x4_at2*>(a + 16 * i);
    }
    return r;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e) {
    if (e >= n) break;
    if constexpr (kType == SOLFP4_F32)
      r.p[e / 4][e % 4] = reinterpret_cast<const uint32_t*>(a)[e];
    else
      r.p[0][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(a)[e] << (16 * (e & 1));
  }
  return r;
}

template <int kType>
__device__ __forceinline__ void to_f32(const Run<kType>& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (kType == SOLFP4_F32) {
      v[e] = __uint_as_float(r.p[e / 4][e % 4]);
    } else if constexpr (kType == SOLFP4_BF16) {
      const uint32_t w = r.p[0][e / 2];
      v[e] = __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    } else {
      v[e] = (float)as_h2(r.p[0][e / 2])[e & 1];
    }
  }
}

// Each value rounded once (nearest, ties to even).
template <int kType>
__device__ __forceinline__ Run<kType> from_f32(const float (&v)[8]) {
  Run<kType> r;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    if constexpr (kType == SOLFP4_F32) {
      r.p[e / 4][e % 4] = __float_as_uint(v[e]);
      r.p[e / 4][e % 4 + 1] = __float_as_uint(v[e + 1]);
    } else if constexpr (kType == SOLFP4_BF16) {
      r.p[0][e / 2] = pack_bf16(v[e], v[e + 1]);
    } else {
      r.p[0][e / 2] = h2_as_u32(half2_t{(_Float16)v[e], (_Float16)v[e + 1]});
    }
  }
  return r;
}

template <int kType>
__device__ __forceinline__ void store_run(void* base, int64_t at, int64_t n, const Run<kType>& r) {
  uint8_t* a = static_cast<uint8_t*>(base) + at * kElemBytes<kType>;
  if (n >= 8) {
#pragma unroll
    for (int i = 0; i < kRunPieces<kType>; ++i) {
      if constexpr (kType == SOLFP4_F32)
        *reinterpret_cast<u32x4_at4*>(a + 16 * i) = r.p[i];
      else
        *reinterpret_cast<u32x4_at2*>(a + 16 * i) = r.p[i];
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e) {
    if (e >= n) break;
    if constexpr (kType == SOLFP4_F32)
      reinterpret_cast<uint32_t*>(a)[e] = r.p[e / 4][e % 4];
    else
      reinterpret_cast<uint16_t*>(a)[e] = (uint16_t)(r.p[0][e / 2] >> (16 * (e & 1)));
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

}  // namespace solfp4
