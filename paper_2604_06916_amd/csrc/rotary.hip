// Rotary positions on q and k, and the table of their cosines and sines.
//
// Pair i of a head (elements i and i + R/2 in the half layout, 2i and 2i + 1
// in the interleaved one, R elements rotated) at a token of position p:
//   (u, v) -> (u c - v s, u s + v c),   c, s = table[p][i], table[p][R/2 + i]
// The transposed rotation (s -> -s) takes the outputs' gradients to the
// inputs'.  Elements R.. of a head are copied.  FP32 between a load and a
// store.
//
// A wave takes the heads of one token (or, where they are few, of several):
// a lane one 16-byte piece of every `slots`-th head, or the piece and its
// partner R/2 elements further on, so its cosines and sines are read once for
// all of them, and the loads of kRotaryHeads heads go out together.
//
// Bound by memory: each element is read and written once.  BF16, 18432 tokens
// of 24 + 24 heads of 128, interleaved: 84 us, 5.4 TB/s (a 1 GB copy moves 5.0, a
// 0.2 GB one 5.4); F16, 1998 tokens of 19 + 19 heads, 80 of 128 turned, positions
// given: 8.8 us in the caches, 4.5 TB/s; one token 2.4 us, a launch.
#include "elements.h"
#include "kernels.h"

namespace solfp4 {

constexpr int kRotaryThreads = 256;

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

// Heads of a lane at most, all in flight together: more share the turns'
// loads, fewer leave more waves (18432 tokens of 48 heads of 128, BF16
// interleaved and 9000 in FP32, 64 turned: 107 and 113 us with one, 86 and 87 with
// two, 84 and 92 with three, 91 and 128 with four, 155 and 181 with six).
constexpr int kRotaryHeads = 2;

// n of the kPairs floats at p, the rest zero
template <int kPairs>
__device__ __forceinline__ void load_turns(const float* p, int n, float (&v)[kPairs]) {
  if (n >= kPairs) {
    if constexpr (kPairs == 2) {
      typedef u32x2_t u32x2_at4 __attribute__((aligned(4)));
      const u32x2_t w = *reinterpret_cast<const u32x2_at4*>(p);
      v[0] = __uint_as_float(w.x);
      v[1] = __uint_as_float(w.y);
    } else {
#pragma unroll
      for (int i = 0; i < kPairs; i += 4) {
        const u32x4_t w = *reinterpret_cast<const u32x4_at4*>(p + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i + e] = __uint_as_float(w[e]);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kPairs; ++i) v[i] = i < n ? p[i] : 0.0f;
}

// How a launch's lanes share the work.  A head has `pieces` pieces: below
// `turning` they hold pairs (half: VE pairs in two pieces R/2 elements apart;
// interleaved: VE/2 pairs in one), the others copy.  A wave holds `lanes` of
// them at a time (all, or 64 in each of `blocks` waves), `slots` heads of
// `packed` tokens; `parts` waves share a token's heads.
struct RotaryShape {
  int turning, pieces, lanes, blocks, slots, packed, parts;
};

template <int kType, bool kInterleaved>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a, RotaryShape sh, int position_bytes,
                                                                float sign) {
  constexpr int VE = 16 / kElemBytes<kType>;
  constexpr int kPairs = kInterleaved ? VE / 2 : VE;
  uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kRotaryThreads / kWave) + threadIdx.x / kWave);
  const int lane = threadIdx.x & (kWave - 1);
  uint32_t block = 0, part = 0;
  if (sh.blocks > 1) block = unit % sh.blocks, unit /= sh.blocks;
  if (sh.parts > 1) part = unit % sh.parts, unit /= sh.parts;
  const int at_slot = lane / sh.lanes, c = (int)block * sh.lanes + lane - at_slot * sh.lanes;
  const int sub = at_slot / sh.slots;
  const int64_t token = a.first + (int64_t)unit * sh.packed + sub;
  if (c >= sh.pieces || sub >= sh.packed || token >= a.tokens) return;
  const int half = a.rotated / 2;
  const bool copies = c >= sh.turning;
  // First element and count of the lane's piece (and of its partner R/2
  // further on).  The last piece of a span that it does not fill starts early
  // instead: a whole vector that repeats elements of the lane before.  Both
  // lanes have read them before either writes (in place they are the same
  // memory: one wave, one load, and the fence below), and write the same values.
  const int span = copies ? a.dim - a.rotated : kInterleaved ? a.rotated : half;
  int at = (copies ? c - sh.turning : c) * VE;
  if (sh.blocks == 1 && span >= VE) at = min(at, span - VE);
  const int n = min(VE, span - at);
  if (copies) at += a.rotated;
  float cs[kPairs], sn[kPairs];
  if (!copies) {
    int64_t p = token;
    if (position_bytes == 4) p = static_cast<const int32_t*>(a.positions)[token];
    else if (position_bytes == 8) p = static_cast<const int64_t*>(a.positions)[token];
    else if (a.table_rows < a.tokens) p = (uint32_t)token % (uint32_t)a.table_rows;
    const bool known = p >= 0 && p < a.table_rows;
    const float* t = a.table + (known ? p : 0) * a.rotated + (kInterleaved ? at / 2 : at);
    load_turns<kPairs>(t, kInterleaved ? n / 2 : n, cs);
    load_turns<kPairs>(t + half, kInterleaved ? n / 2 : n, sn);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      // a position outside the table turns into NaN
      cs[i] = known ? cs[i] : __builtin_nanf("");
      sn[i] = known ? sign * sn[i] : __builtin_nanf("");
    }
  }
  const uint8_t* qi = static_cast<const uint8_t*>(a.q.in) + (token * a.q.in_token + at) * kElemBytes<kType>;
  const uint8_t* ki = static_cast<const uint8_t*>(a.k.in) + (token * a.k.in_token + at) * kElemBytes<kType>;
  uint8_t* qo = static_cast<uint8_t*>(a.q.out) + (token * a.q.out_token + at) * kElemBytes<kType>;
  uint8_t* ko = static_cast<uint8_t*>(a.k.out) + (token * a.k.out_token + at) * kElemBytes<kType>;
  const int64_t apart = (int64_t)half * kElemBytes<kType>;
  const int heads = a.q.heads + a.k.heads, hop = sh.slots * sh.parts;
  const int h0 = at_slot - sub * sh.slots + (int)part * sh.slots;
  u32x4_t pu[kRotaryHeads], pv[kRotaryHeads];
  uint8_t* out[kRotaryHeads];
#pragma unroll
  for (int j = 0; j < kRotaryHeads; ++j) {
    const int h = h0 + j * hop;
    if (h >= heads) continue;
    const bool first = h < a.q.heads;
    const int64_t hh = first ? h : h - a.q.heads;
    const uint8_t* in = (first ? qi : ki) + hh * (first ? a.q.in_head : a.k.in_head) * kElemBytes<kType>;
    out[j] = (first ? qo : ko) + hh * (first ? a.q.out_head : a.k.out_head) * kElemBytes<kType>;
    pu[j] = load_piece<kType, VE>(in, n);
    if (!kInterleaved && !copies) pv[j] = load_piece<kType, VE>(in + apart, n);
  }
  // no lane's store before another's load
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < kRotaryHeads; ++j) {
    if (h0 + j * hop >= heads) continue;
    if (copies) {
      store_piece<kType, VE>(out[j], n, pu[j]);
      continue;
    }
    float u[VE];
    piece_to_f32<kType, VE>(pu[j], u);
    if constexpr (kInterleaved) {
      float r[VE];
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        r[2 * i] = u[2 * i] * cs[i] - u[2 * i + 1] * sn[i];
        r[2 * i + 1] = u[2 * i] * sn[i] + u[2 * i + 1] * cs[i];
      }
      store_piece<kType, VE>(out[j], n, piece_from_f32<kType, VE>(r));
    } else {
      float v[VE], ru[VE], rv[VE];
      piece_to_f32<kType, VE>(pv[j], v);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        ru[i] = u[i] * cs[i] - v[i] * sn[i];
        rv[i] = u[i] * sn[i] + v[i] * cs[i];
      }
      store_piece<kType, VE>(out[j], n, piece_from_f32<kType, VE>(ru));
      store_piece<kType, VE>(out[j] + apart, n, piece_from_f32<kType, VE>(rv));
    }
  }
}

// Waves wanted a CU; with fewer tokens their heads are split.
constexpr int64_t kRotaryWaves = 16;

// The shape of a call's launches, for vectors of VE elements.
static RotaryShape rotary_shape(int VE, bool interleaved, int64_t tokens, int64_t dim, int64_t rotated, int64_t heads) {
  const int64_t span = interleaved ? rotated : rotated / 2;
  RotaryShape sh;
  sh.turning = (int)((span + VE - 1) / VE);
  sh.pieces = sh.turning + (int)((dim - rotated + VE - 1) / VE);
  sh.blocks = (sh.pieces + kWave - 1) / kWave;
  sh.lanes = sh.blocks > 1 ? kWave : sh.pieces;
  const int fit = kWave / sh.lanes;
  sh.slots = heads < fit ? (int)heads : fit;
  sh.packed = fit / sh.slots;
  const int64_t rounds = (heads + sh.slots - 1) / sh.slots, units = (tokens + sh.packed - 1) / sh.packed;
  const int64_t least = (rounds + kRotaryHeads - 1) / kRotaryHeads;
  const int64_t wanted = (kRotaryWaves * device_cu_count() + units - 1) / units;
  sh.parts = (int)(wanted < least ? least : wanted < rounds ? wanted : rounds);
  return sh;
}

template <int kType>
static hipError_t launch_rotary_type(bool interleaved, bool inverse, int position_bytes, RotaryArgs a,
                                     hipStream_t stream) {
  const RotaryShape sh = rotary_shape(16 / kElemBytes<kType>, interleaved, a.tokens, a.dim, a.rotated,
                                      (int64_t)a.q.heads + a.k.heads);
  constexpr int kWaves = kRotaryThreads / kWave;
  // waves of `packed` tokens, and so tokens of one launch (heads x dim below
  // 2^31 are fewer than 2^26 waves)
  const int64_t each = (int64_t)sh.parts * sh.blocks;
  const int64_t most = kMaxThreads / kRotaryThreads * kWaves / each * sh.packed;
  const float sign = inverse ? -1.0f : 1.0f;
  const int64_t tokens = a.tokens;
  for (a.first = 0; a.first < tokens; a.first += most) {
    a.tokens = tokens - a.first < most ? tokens : a.first + most;   // the last workgroup ends with the launch's tokens
    const int64_t waves = (a.tokens - a.first + sh.packed - 1) / sh.packed * each;
    const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves)), block(kRotaryThreads);
    const hipError_t e = launch_kernel(interleaved ? rotary_kernel<kType, true> : rotary_kernel<kType, false>, grid,
                                       block, stream, a, sh, position_bytes, sign);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_rotary(int type, bool interleaved, bool inverse, int position_bytes, const RotaryArgs& a,
                         hipStream_t stream) {
  if (a.tokens == 0 || a.dim == 0 || a.q.heads + a.k.heads == 0) return hipSuccess;
  if (type == SOLFP4_BF16) return launch_rotary_type<SOLFP4_BF16>(interleaved, inverse, position_bytes, a, stream);
  if (type == SOLFP4_F16) return launch_rotary_type<SOLFP4_F16>(interleaved, inverse, position_bytes, a, stream);
  return launch_rotary_type<SOLFP4_F32>(interleaved, inverse, position_bytes, a, stream);
}

// The angle and its cosine and sine in 64 bits, each rounded once: an FP32
// product of a position of 10^5 and its frequency is off by up to 2^-8 radians
// already.
__global__ __launch_bounds__(kRotaryThreads) void rotary_table_kernel(RotaryTableArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x;
  const int64_t row = a.first + unit / a.pairs;
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

hipError_t launch_rotary_table(RotaryTableArgs a, hipStream_t stream) {
  if (a.rows == 0 || a.pairs == 0) return hipSuccess;
  const int64_t most = kMaxThreads / kRotaryThreads * kRotaryThreads / a.pairs;   // rows of one launch
  const int64_t rows = a.rows;
  for (a.first = 0; a.first < rows; a.first += most) {
    a.rows = rows - a.first < most ? rows : a.first + most;   // the last workgroup ends with the launch's rows
    const int64_t units = (a.rows - a.first) * a.pairs;
    const hipError_t e = launch_kernel(rotary_table_kernel, dim3((unsigned)((units + kRotaryThreads - 1) / kRotaryThreads)),
                                       dim3(kRotaryThreads), stream, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace solfp4
