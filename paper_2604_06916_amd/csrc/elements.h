// Runs of 8 elements of the operators' types (BF16, FP16, FP32) as FP32 values.
#pragma once

#include <type_traits>

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

// Eight ones.
template <int kType>
__device__ __forceinline__ Run<kType> one_run() {
  constexpr uint32_t k = kType == SOLFP4_F32 ? 0x3F800000u : kType == SOLFP4_BF16 ? 0x3F803F80u : 0x3C003C00u;
  Run<kType> r;
#pragma unroll
  for (int i = 0; i < kRunPieces<kType>; ++i) r.p[i] = u32x4_t{k, k, k, k};
  return r;
}

// Row `row` of an operand (both uniform over the wave, so the address stays
// scalar and a lane adds its 32-bit offset).
template <int kType>
__device__ __forceinline__ const uint8_t* row_of(const void* base, int64_t row, int64_t stride) {
  return static_cast<const uint8_t*>(base) + row * stride * kElemBytes<kType>;
}
template <int kType>
__device__ __forceinline__ uint8_t* row_of(void* base, int64_t row, int64_t stride) {
  return static_cast<uint8_t*>(base) + row * stride * kElemBytes<kType>;
}

// The run at element `at` of `base`, of which the first n elements exist
// (n >= 8: one vector load per piece; else element loads, zeros after them).
template <int kType>
__device__ __forceinline__ Run<kType> load_run(const uint8_t* base, uint32_t at, int n) {
  const uint8_t* a = base + at * kElemBytes<kType>;
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
    if constexpr (kType == SOLFP4_F32) {
      if (e < n) r.p[e / 4][e % 4] = reinterpret_cast<const uint32_t*>(a)[e];
    } else {
      if (e < n) r.p[0][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(a)[e] << (16 * (e & 1));
    }
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
__device__ __forceinline__ void store_run(uint8_t* base, uint32_t at, int n, const Run<kType>& r) {
  uint8_t* a = base + at * kElemBytes<kType>;
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
    if constexpr (kType == SOLFP4_F32) {
      if (e < n) reinterpret_cast<uint32_t*>(a)[e] = r.p[e / 4][e % 4];
    } else {
      if (e < n) reinterpret_cast<uint16_t*>(a)[e] = (uint16_t)(r.p[0][e / 2] >> (16 * (e & 1)));
    }
  }
}

// Hides that the run is as it was, so that its conversion is made again
// where it is used again and no FP32 copy is kept in between.
template <int kType>
__device__ __forceinline__ void forget(Run<kType>& r) {
#pragma unroll
  for (int i = 0; i < kRunPieces<kType>; ++i) asm volatile("" : "+v"(r.p[i]));
}

// Sums over lanes, in every lane, without LDS: neighbours, quads and half
// rows by DPP, then rows of 16 and halves of 32 by lane swaps.
template <int kCtrl, typename T>
__device__ __forceinline__ T dpp_of(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), kCtrl, 0xF, 0xF, false));
  } else {
    const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
    return __builtin_bit_cast(T, u32x2_t{(uint32_t)__builtin_amdgcn_mov_dpp((int)w.x, kCtrl, 0xF, 0xF, false),
                                         (uint32_t)__builtin_amdgcn_mov_dpp((int)w.y, kCtrl, 0xF, 0xF, false)});
  }
}

template <int kLanes, typename T>
__device__ __forceinline__ T swapped_sum(T v) {
  auto swap = [](uint32_t w) {
    if constexpr (kLanes == 16) return __builtin_amdgcn_permlane16_swap(w, w, false, false);
    else return __builtin_amdgcn_permlane32_swap(w, w, false, false);
  };
  if constexpr (sizeof(T) == 4) {
    const auto h = swap(__builtin_bit_cast(uint32_t, v));
    return __builtin_bit_cast(T, (uint32_t)h[0]) + __builtin_bit_cast(T, (uint32_t)h[1]);
  } else {
    const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
    const auto x = swap(w.x), y = swap(w.y);
    return __builtin_bit_cast(T, u32x2_t{(uint32_t)x[0], (uint32_t)y[0]}) +
           __builtin_bit_cast(T, u32x2_t{(uint32_t)x[1], (uint32_t)y[1]});
  }
}

// Over each aligned group of `lanes` lanes (a power of two, uniform).
template <typename T>
__device__ __forceinline__ T lanes_sum(T v, int lanes) {
  if (lanes > 1) v += dpp_of<0xB1>(v);      // quad_perm 1,0,3,2
  if (lanes > 2) v += dpp_of<0x4E>(v);      // quad_perm 2,3,0,1
  if (lanes > 4) v += dpp_of<0x141>(v);     // row_half_mirror
  if (lanes > 8) v += dpp_of<0x140>(v);     // row_mirror
  if (lanes > 16) v = swapped_sum<16>(v);
  if (lanes > 32) v = swapped_sum<32>(v);
  return v;
}

}  // namespace solfp4
