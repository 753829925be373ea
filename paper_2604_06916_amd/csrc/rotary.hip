// Rotary positions on q and k, and the table of their cosines and sines.
//
// Pair i of a head (elements i and i + R/2 in the half layout, 2i and 2i + 1
// in the interleaved one, R elements rotated) at a token of position p:
//   (u, v) -> (u c - v s, u s + v c),   c, s = table[p][i], table[p][R/2 + i]
// The transposed rotation (s -> -s) takes the outputs' gradients to the
// inputs'.  Elements R.. of a head are copied.  FP32 between a load and a
// store.
//
// A lane takes the same 16-byte pieces of every head of its token that its
// slot reaches, so the table's row is read once per slot and not once per
// head (a row is 2 R FP32 bytes against 2 R of a BF16 head).  Bound by
// memory: each element is read and written once.
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

constexpr int kRotaryThreads = 256;

template <typename T>
__device__ __forceinline__ float load_elem(const T* p) {
  return (float)*p;
}

// 16-byte piece of VE elements as FP32
template <int kType, int VE>
__device__ __forceinline__ void piece_to_f32(u32x4_t p, float (&v)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    if constexpr (kType == SOLFP4_F32)
      v[e] = __uint_as_float(p[e]);
    else if constexpr (kType == SOLFP4_BF16)
      v[e] = __uint_as_float(e & 1 ? p[e / 2] & 0xFFFF0000u : p[e / 2] << 16);
    else
      v[e] = (float)as_h2(p[e / 2])[e & 1];
  }
}

template <int kType, int VE>
__device__ __forceinline__ u32x4_t piece_from_f32(const float (&v)[VE]) {
  u32x4_t p;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (kType == SOLFP4_F32)
      p[w] = __float_as_uint(v[w]);
    else if constexpr (kType == SOLFP4_BF16)
      p[w] = pack_bf16(v[2 * w], v[2 * w + 1]);
    else
      p[w] = h2_as_u32(half2_t{(_Float16)v[2 * w], (_Float16)v[2 * w + 1]});
  }
  return p;
}

// n (1 to VE) elements at p; the rest zero
template <int kType, int VE>
__device__ __forceinline__ u32x4_t load_piece(const uint8_t* p, int n) {
  if (n >= VE) {
    if constexpr (kType == SOLFP4_F32) return *reinterpret_cast<const u32x4_at4*>(p);
    return *reinterpret_cast<const u32x4_at2*>(p);
  }
  u32x4_t r = u32x4_t{0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < VE - 1; ++e) {
    if (e >= n) continue;
    if constexpr (kType == SOLFP4_F32)
      r[e] = reinterpret_cast<const uint32_t*>(p)[e];
    else
      r[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
  }
  return r;
}

template <int kType, int VE>
__device__ __forceinline__ void store_piece(uint8_t* p, int n, u32x4_t r) {
  if (n >= VE) {
    if constexpr (kType == SOLFP4_F32)
      *reinterpret_cast<u32x4_at4*>(p) = r;
    else
      *reinterpret_cast<u32x4_at2*>(p) = r;
    return;
  }
#pragma unroll
  for (int e = 0; e < VE - 1; ++e) {
    if (e >= n) continue;
    if constexpr (kType == SOLFP4_F32)
      reinterpret_cast<uint32_t*>(p)[e] = r[e];
    else
      reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(r[e / 2] >> (16 * (e & 1)));
  }
}

// One lane's unit: piece `c` of the heads slot, slot + slots, ... of a token.
// Pieces below `turning` hold pairs (half: VE pairs in two pieces R/2
// elements apart; interleaved: VE/2 pairs in one), the others copy.
template <int kType, bool kInterleaved>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a, int position_bytes, float sign,
                                                                int turning, int pieces, int slots) {
  constexpr int VE = 16 / kElemBytes<kType>;
  constexpr int kPairs = kInterleaved ? VE / 2 : VE;
  const int64_t unit = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x;
  const int c = (int)(unit % pieces);
  const int64_t rest = unit / pieces;
  const int slot = (int)(rest % slots);
  const int64_t token = rest / slots;
  if (token >= a.tokens) return;
  const int half = a.rotated / 2;
  const bool copies = c >= turning;
  // first element and count of the lane's piece (and of its partner R/2 further on)
  const int at = copies ? a.rotated + (c - turning) * VE : kInterleaved ? c * VE : c * VE;
  const int n = min(VE, copies ? a.dim - at : kInterleaved ? a.rotated - at : half - at);
  float cs[kPairs], sn[kPairs];
  if (!copies) {
    int64_t p = token % a.table_rows;
    if (position_bytes == 4) p = static_cast<const int32_t*>(a.positions)[token];
    if (position_bytes == 8) p = static_cast<const int64_t*>(a.positions)[token];
    const bool known = p >= 0 && p < a.table_rows;
    const float* t = a.table + (known ? p : 0) * a.rotated + (kInterleaved ? at / 2 : at);
    const int pairs = kInterleaved ? n / 2 : n;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      // a position outside the table turns into NaN
      cs[i] = !known ? __builtin_nanf("") : i < pairs ? t[i] : 0.0f;
      sn[i] = !known ? __builtin_nanf("") : i < pairs ? sign * t[half + i] : 0.0f;
    }
  }
  const int heads = a.q.heads + a.k.heads;
  for (int h = slot; h < heads; h += slots) {
    const bool first = h < a.q.heads;
    const RotaryOperand& o = first ? a.q : a.k;
    const int hh = first ? h : h - a.q.heads;
    const uint8_t* in = static_cast<const uint8_t*>(o.in) +
                        (token * o.in_token + hh * o.in_head + at) * kElemBytes<kType>;
    uint8_t* out = static_cast<uint8_t*>(o.out) + (token * o.out_token + hh * o.out_head + at) * kElemBytes<kType>;
    const u32x4_t pu = load_piece<kType, VE>(in, n);
    if (copies) {
      store_piece<kType, VE>(out, n, pu);
      continue;
    }
    float u[VE];
    piece_to_f32<kType, VE>(pu, u);
    if constexpr (kInterleaved) {
      float r[VE];
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        r[2 * i] = u[2 * i] * cs[i] - u[2 * i + 1] * sn[i];
        r[2 * i + 1] = u[2 * i] * sn[i] + u[2 * i + 1] * cs[i];
      }
      store_piece<kType, VE>(out, n, piece_from_f32<kType, VE>(r));
    } else {
      const int64_t apart = (int64_t)half * kElemBytes<kType>;
      float v[VE], ru[VE], rv[VE];
      piece_to_f32<kType, VE>(load_piece<kType, VE>(in + apart, n), v);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        ru[i] = u[i] * cs[i] - v[i] * sn[i];
        rv[i] = u[i] * sn[i] + v[i] * cs[i];
      }
      store_piece<kType, VE>(out, n, piece_from_f32<kType, VE>(ru));
      store_piece<kType, VE>(out + apart, n, piece_from_f32<kType, VE>(rv));
    }
  }
}

template <int kType>
static hipError_t launch_rotary_type(bool interleaved, bool inverse, int position_bytes, const RotaryArgs& a,
                                     hipStream_t stream) {
  constexpr int VE = 16 / kElemBytes<kType>;
  const int span = interleaved ? a.rotated : a.rotated / 2;
  const int turning = (span + VE - 1) / VE;
  const int pieces = turning + (a.dim - a.rotated + VE - 1) / VE;
  const int heads = a.q.heads + a.k.heads;
  const int slots = heads < 4 ? heads : 4;
  const int64_t units = a.tokens * slots * pieces;
  const dim3 grid((unsigned)((units + kRotaryThreads - 1) / kRotaryThreads)), block(kRotaryThreads);
  const float sign = inverse ? -1.0f : 1.0f;
  return interleaved ? launch_kernel(rotary_kernel<kType, true>, grid, block, stream, a, position_bytes, sign,
                                     turning, pieces, slots)
                     : launch_kernel(rotary_kernel<kType, false>, grid, block, stream, a, position_bytes, sign,
                                     turning, pieces, slots);
}

hipError_t launch_rotary(int type, bool interleaved, bool inverse, int position_bytes, const RotaryArgs& a,
                         hipStream_t stream) {
  if (a.tokens == 0 || a.dim == 0 || a.q.heads + a.k.heads == 0) return hipSuccess;
  if (type == SOLFP4_BF16) return launch_rotary_type<SOLFP4_BF16>(interleaved, inverse, position_bytes, a, stream);
  if (type == SOLFP4_F16) return launch_rotary_type<SOLFP4_F16>(interleaved, inverse, position_bytes, a, stream);
  return launch_rotary_type<SOLFP4_F32>(interleaved, inverse, position_bytes, a, stream);
}

// The angle and its cosine and sine in 64 bits, each rounded once: an FP32
// product of a position of 10^5 and its frequency is off by up to 2^-8 turns'
// worth of angle already.
__global__ __launch_bounds__(kRotaryThreads) void rotary_table_kernel(RotaryTableArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x;
  const int64_t row = unit / a.pairs;
  const int i = (int)(unit % a.pairs);
  if (row >= a.rows) return;
  int axis = 0;
  while (axis < a.axes - 1 && i >= a.axis_end[axis]) ++axis;
  const int64_t p = a.positions ? a.positions[row * a.axes + axis] : row;
  double s, c;
  sincos((double)p * a.frequencies[i], &s, &c);
  float* t = a.table + row * 2 * a.pairs + i;
  t[0] = (float)(c * a.magnitude);
  t[a.pairs] = (float)(s * a.magnitude);
}

hipError_t launch_rotary_table(const RotaryTableArgs& a, hipStream_t stream) {
  const int64_t units = a.rows * a.pairs;
  if (units == 0) return hipSuccess;
  return launch_kernel(rotary_table_kernel, dim3((unsigned)((units + kRotaryThreads - 1) / kRotaryThreads)),
                       dim3(kRotaryThreads), stream, a);
}

}  // namespace solfp4
