// Low-rank adapters beside a shared linear, many at once:
//
//   h_t = a_e x_t,  out_t = y_t + c_e b_e h_t,  e the adapter of token t
//
// x [tokens][K], y [tokens][N] and the adapters' a [rank][K], b [N][rank] are
// BF16; h is FP32 (rank values a token) and goes into the second product as
// three BF16 pieces, all 24 of its bits: y may cancel what the adapters add.
//
// A workgroup takes a tile of up to 32 tokens of one adapter (the plan brings
// them together) and a range of N: its waves share K, add their shares of h in
// LDS in wave order, and share the columns.
//
// Bound by memory: x once, y once in and once out; a and b come from L2, as
// often as there are tiles.  So every access to a token's row covers whole
// lines: 16 lanes read 256 bytes of it (with 64 bytes a row an instruction, as a
// matrix operand lies, a copy of 26574 x 7296 takes 210 us, with 128 or more
// 165).  x goes through LDS into operand order.  In the second product tokens
// are the result's rows and a lane holds 8 consecutive columns of four of them:
// column m of block q is n = 8 m + q.  In the first, tokens are the columns, and
// row 4 g + i of blocks 2 c and 2 c + 1 is rank element 32 c + 8 g + i and four
// further on, so h is the second product's operand as it stands.
//
// 26574 tokens 2432 -> 7296, rank 32: 219 us, 4.2 TB/s (a copy of its bytes 5.0);
// 8192 tokens 2240 -> 6720 50 to 63 us, by what of its 257 MB the 256 MB cache keeps;
// 64 tokens of 48 adapters 12.9 us, where most tiles have one token and a and b come
// from HBM once; 1 token 1152 -> 1152, rank 16 5.7 us.
#include <limits.h>

#include "adapters.h"

namespace solfp4 {

// ---- plan -----------------------------------------------------------------

// Tokens come to their groups by a counting sort that keeps their order: they are
// cut to segments, one a wave, which counts its tokens of every group; one
// workgroup adds the counts up, group by group and segment by segment, to first
// places; and each wave puts its tokens there.  A token is read twice, and a
// count belongs to one wave, so results have no order of atomics in them.
//
// Three launches that wait for each other: 13.5 us for 64 tokens of 48 adapters, 17 for
// 26574 of 6, 91 for a million of 4, 3.1 ms for a million of 60000 (with a workgroup a
// group that read all of the index 13, 25, 782 and 124 ms).
constexpr int kPlanThreads = 1024, kPlanDeep = 4;   // fours of counts a thread
constexpr int kSegmentWaves = 4;   // of a workgroup
constexpr int64_t kSegment = 128, kMostSegments = 2048, kCounts = 16384;

typedef int i32x4_t __attribute__((ext_vector_type(4)));

struct Segments {
  int64_t each, counts_at;   // tokens of a segment; word of the counts in the plan, [group][segment]
  int count;
};

// Segments of kSegment tokens or more, and so few that adding up their counts,
// 0.4 ns each, takes no longer than their waves do, 2.6 us for 64 tokens (a million
// tokens of 1000 adapters: 230 us, 456 without), and that the counts take no more
// words than there are tokens (but for kCounts, or one segment's).
static Segments segments_of(const AdapterTokens& t) {
  const int64_t groups = t.adapters + 2, fit = (t.tokens + kCounts) / groups;
  int64_t n = (t.tokens + kSegment - 1) / kSegment;
  n = n < kMostSegments ? n : kMostSegments;
  n = n < fit ? n : fit;
  while (n > 1 && n * n * groups > 128 * t.tokens) n = n * 7 / 8;
  n = n < 1 ? 1 : n;
  const int64_t each = ((t.tokens + n - 1) / n + kWave - 1) / kWave * kWave;
  return {each, t.tiles_at + 4 * t.max_tiles, (int)n};
}

AdapterTokens adapter_tokens(const void* plan, int64_t tokens, int64_t adapters) {
  AdapterTokens t = {static_cast<const int*>(plan), tokens, (int)adapters, 0, 0, 0, 0};
  const int64_t groups = adapters + 2, heads = (groups + 1 + 3) / 4 * 4;
  t.places_at = heads;
  t.order_at = 2 * heads;
  t.tiles_at = t.order_at + (tokens + 3) / 4 * 4;
  t.max_tiles = (tokens + kAdapterTile - 1) / kAdapterTile;
  if (plan) t.max_tiles += groups < tokens ? groups : tokens;   // each group may end inside a tile
  return t;
}

size_t adapter_plan_bytes(int64_t tokens, int64_t adapters) {
  const AdapterTokens t = adapter_tokens(&t, tokens, adapters);   // any address: as with a plan
  const Segments s = segments_of(t);
  return (size_t)(s.counts_at + ((adapters + 2) * s.count + 3) / 4 * 4) * 4;
}

template <typename Index>
__device__ __forceinline__ int group_of(const Index* index, int64_t i, int adapters) {
  const Index v = index[i];
  return v < 0 ? adapters : v < adapters ? (int)v : adapters + 1;
}

// The lanes, of those with a token, whose group is this lane's.
__device__ __forceinline__ uint64_t lanes_alike(int group, bool has, int groups) {
  uint64_t alike = __ballot(has);
  for (int bit = 0; groups - 1 >> bit; ++bit) {
    const bool set = group >> bit & 1;
    const uint64_t with = __ballot(set);
    alike &= set ? with : ~with;
  }
  return alike;
}

// f(token, whether there is one, its group, the lanes of that group), 64 tokens at a time.
template <typename Index, typename F>
__device__ __forceinline__ void each_of_segment(const Index* index, const AdapterTokens& t, const Segments& s, int segment,
                                                int lane, F f) {
  const int64_t first = segment * s.each, end = min(first + s.each, t.tokens);
  int64_t i = first + lane;
  int next = i < end ? group_of(index, i, t.adapters) : 0;
  for (int64_t base = first; base < end; base += kWave, i += kWave) {
    const int group = next;
    const bool has = i < end;
    if (i + kWave < end) next = group_of(index, i + kWave, t.adapters);
    f((int)i, has, group, lanes_alike(group, has, t.adapters + 2));
  }
}

template <typename Index>
__global__ __launch_bounds__(kSegmentWaves* kWave) void plan_counts_kernel(const Index* __restrict__ index, AdapterTokens t,
                                                                          Segments s, int* plan) {
  const int segment = blockIdx.x * kSegmentWaves + threadIdx.x / kWave, lane = threadIdx.x % kWave;
  if (segment >= s.count) return;
  int* const counts = plan + s.counts_at + segment;
  const int64_t n = (int64_t)(t.adapters + 2) * s.count;
  for (int64_t g = lane; g < t.adapters + 2; g += kWave) counts[g * s.count] = 0;
  if (segment == 0 && lane < (-n & 3)) plan[s.counts_at + n + lane] = 0;   // up to whole fours
  __threadfence();
  each_of_segment(index, t, s, segment, lane, [&](int, bool has, int group, uint64_t alike) {
    if (has && lane == __builtin_ctzll(alike)) atomicAdd(counts + (int64_t)group * s.count, __builtin_popcountll(alike));
  });
}

// Sums of v over the workgroup's threads before this one; `at` goes on by the sum over all.
__device__ __forceinline__ int sum_before(int v, int& at, int (&sums)[kPlanThreads / kWave]) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  int upto = v;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int o = __shfl_up(upto, d, kWave);
    if (lane >= d) upto += o;
  }
  __syncthreads();
  if (lane == kWave - 1) sums[wave] = upto;
  __syncthreads();
  int before = at + upto - v;
#pragma unroll
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    if (w < wave) before += sums[w];
    at += sums[w];
  }
  return before;
}

// One workgroup: the counts become first places, and the groups' first places and
// first tiles follow from them.
__global__ __launch_bounds__(kPlanThreads) void plan_starts_kernel(AdapterTokens t, Segments s, int* plan) {
  __shared__ int sums[kPlanThreads / kWave];
  const int groups = t.adapters + 2;
  const int64_t n = (int64_t)groups * s.count;
  int* const counts = plan + s.counts_at;
  int at = 0;
  // a thread's counts follow each other, fours whose last may reach past the end
  i32x4_t* const fours = reinterpret_cast<i32x4_t*>(counts) + threadIdx.x * kPlanDeep;
  const int64_t left = (n + 3) / 4 - threadIdx.x * kPlanDeep;
  i32x4_t v[kPlanDeep];
  const auto load = [&](int64_t base) {
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u) v[u] = base + u < left ? fours[base + u] : i32x4_t{0, 0, 0, 0};
  };
  load(0);
  for (int64_t base = 0; base < (n + 3) / 4; base += kPlanThreads * kPlanDeep) {
    i32x4_t now[kPlanDeep];
    int sum = 0;
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u) {
      now[u] = v[u];
      sum += now[u].x + now[u].y + now[u].z + now[u].w;
    }
    load(base + kPlanThreads * kPlanDeep);
    int place = sum_before(sum, at, sums);
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u) {
      i32x4_t to;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        to[k] = place;
        place += now[u][k];
      }
      if (base + u < left) fours[base + u] = to;
    }
  }
  __syncthreads();
  int tiles = 0;
  for (int base = 0; base < groups; base += kPlanThreads) {
    const int g = base + threadIdx.x;
    const int from = g < groups ? counts[(int64_t)g * s.count] : 0;
    const int to = g + 1 < groups ? counts[(int64_t)(g + 1) * s.count] : (int)t.tokens;
    const int first = sum_before(g < groups ? (to - from + kAdapterTile - 1) / kAdapterTile : 0, tiles, sums);
    if (g < groups) plan[g] = first, plan[t.places_at + g] = from;
  }
  if (threadIdx.x == 0) plan[groups] = tiles, plan[t.places_at + groups] = (int)t.tokens;
  if (threadIdx.x < (-n & 3)) counts[n + threadIdx.x] = 0;
}

// The tokens to their places; the workgroups after those, a thread a tile, find
// its group among the groups' first tiles.
template <typename Index>
__global__ __launch_bounds__(kSegmentWaves* kWave) void plan_order_kernel(const Index* __restrict__ index, AdapterTokens t,
                                                                         Segments s, int* plan) {
  constexpr int kThreads = kSegmentWaves * kWave;
  const int segment = blockIdx.x * kSegmentWaves + threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int workgroups = (s.count + kSegmentWaves - 1) / kSegmentWaves, groups = t.adapters + 2;
  if ((int)blockIdx.x < workgroups) {
    if (segment >= s.count) return;
    int* const places = plan + s.counts_at + segment;
    each_of_segment(index, t, s, segment, lane, [&](int token, bool has, int group, uint64_t alike) {
      const int leader = has ? __builtin_ctzll(alike) : 0;
      int place = 0;
      if (has && lane == leader) place = atomicAdd(places + (int64_t)group * s.count, __builtin_popcountll(alike));
      place = __shfl(place, leader, kWave) + __builtin_popcountll(alike & ((1ull << lane) - 1));
      asm volatile("" : "+v"(place) : : "memory");   // these places before the next 64 tokens'
      if (has && place < t.tokens) plan[t.order_at + place] = token;
    });
    __threadfence();
    // zeros, as behind the last tile
    for (int64_t g = lane; g < groups; g += kWave) places[g * s.count] = 0;
    return;
  }
  const int64_t i = (int64_t)(blockIdx.x - workgroups) * kThreads + threadIdx.x;
  if (i >= t.max_tiles) return;
  int* tile = plan + t.tiles_at + 4 * i;
  int group = 0, first = 0, count = 0;
  if (i < plan[groups]) {
    int lo = 0, hi = groups;   // the last group whose first tile is i or before
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (plan[mid] <= i) lo = mid; else hi = mid;
    }
    group = lo;
    const int end = plan[t.places_at + group + 1];
    first = plan[t.places_at + group] + (int)(i - plan[group]) * kAdapterTile;
    count = min(end - first, kAdapterTile);
  }
  tile[0] = group, tile[1] = first, tile[2] = count, tile[3] = 0;
}

template <typename Index>
static hipError_t launch_plan(const Index* index, const AdapterTokens& t, int* plan, hipStream_t stream) {
  const Segments s = segments_of(t);
  constexpr int kThreads = kSegmentWaves * kWave;
  const unsigned workgroups = (unsigned)((s.count + kSegmentWaves - 1) / kSegmentWaves);
  const unsigned tiles = (unsigned)((t.max_tiles + kThreads - 1) / kThreads);
  hipError_t e = launch_kernel(plan_counts_kernel<Index>, dim3(workgroups), dim3(kThreads), stream, index, t, s, plan);
  if (e == hipSuccess) e = launch_kernel(plan_starts_kernel, dim3(1), dim3(kPlanThreads), stream, t, s, plan);
  if (e == hipSuccess)
    e = launch_kernel(plan_order_kernel<Index>, dim3(workgroups + tiles), dim3(kThreads), stream, index, t, s, plan);
  return e;
}

hipError_t launch_adapter_plan(const void* index, int index_bytes, int64_t tokens, int64_t adapters, void* plan,
                               hipStream_t stream) {
  const AdapterTokens t = adapter_tokens(plan, tokens, adapters);
  int* p = static_cast<int*>(plan);
  return index_bytes == 4 ? launch_plan(static_cast<const int32_t*>(index), t, p, stream)
                          : launch_plan(static_cast<const int64_t*>(index), t, p, stream);
}

// ---- forward --------------------------------------------------------------

constexpr int kStepK = 128;   // of a wave's step

// kChunks: 32s of the rank; kLane: columns of a lane a step (8, or 4 where b
// takes too many registers or there are few tiles: b then comes a step ahead);
// kWholeRank: the rank is a multiple of 8.  kPart: both products, or h's shares
// of a range of K alone, or the second product from such shares.
enum { kBoth, kShares, kFromShares };
template <int kChunks, int kLane, int kWaves, bool kWholeRank, int kPart>
__global__ __launch_bounds__(kWaves * kWave, 2) void add_adapters_kernel(AdapterArgs p) {
  constexpr int kBlocks = 2 * kChunks;   // 16s of the rank
  constexpr int kStepN = 16 * kLane;
  constexpr bool kAhead = kLane == 4 && kChunks < 4;
  constexpr int kRow = kStepK * 2 + 16;  // a row of x in LDS: 16 rows at one column lie in all banks
  constexpr int kAStep = 4 / kChunks;    // 32s of K whose rows of a are held at once
  constexpr int kPlaces = 2 * kBlocks * kWave;   // of four values of h
  constexpr int kXBytes = kPart == kFromShares ? 0 : kWaves * kAdapterTile * kRow;
  constexpr int kShareBytes = (kPart == kFromShares ? 1 : kWaves) * kPlaces * 16;
  // the waves' tiles of x, then their shares of h
  __shared__ __attribute__((aligned(16))) uint8_t room[kXBytes > kShareBytes ? kXBytes : kShareBytes];
  // the third piece of h, where three in registers would spill (13000 tokens 2432 ->
  // 7296, rank 64: 180 us)
  constexpr int kHeld = kChunks == 1 ? 3 : 2;
  __shared__ bf16x8_t low[kHeld == 3 ? 1 : 2 * kChunks][kWave];
  floatx4_t(*const share)[2 * kBlocks][kWave] = reinterpret_cast<floatx4_t(*)[2 * kBlocks][kWave]>(room);
  // with 8 tiles or more a tile's ranges run on one XCD, whose L2 then has its rows
  const int ranges = kPart == kShares ? p.k_splits : p.splits, at = blockIdx.x / p.xcds;
  const int index = at / ranges * p.xcds + blockIdx.x % p.xcds, split = at % ranges;
  if (index >= p.t.max_tiles) return;
  const Tile tile = uniform(p.t, load_tile(p.t, index));
  if (tile.count == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int m = lane % 16, g = lane / 16;
  const bool two = tile.count > 16;          // tokens in both blocks of 16
  const bool real = tile.group < p.t.adapters;
  // a lane reads and writes rows g + 4 i of the tile; the last row again past its end
  uint32_t token[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) token[i] = (uint32_t)token_at(p.t, tile.first + min(g + 4 * i, tile.count - 1));
  // as an operand's row or column, m is row 4 (m % 4) + m / 4 of its block, so that results are of rows g + 4 i
  const int row = m % 4 * 4 + m / 4;

  bf16x8_t h[2][kChunks][kHeld];   // h's pieces of this lane's tokens
  if (kPart == kFromShares && real) {
    const floatx4_t* from = static_cast<const floatx4_t*>(p.shares) + (int64_t)index * p.k_splits * kPlaces;
    for (int i = threadIdx.x; i < (two ? kPlaces : kPlaces / 2); i += kWaves * kWave) {
      floatx4_t v = from[i];
      for (int k = 1; k < p.k_splits; ++k) v += from[k * kPlaces + i];
      share[0][i / kWave][i % kWave] = v;
    }
  } else if (real) {
    floatx4_t acc[2][kBlocks];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) acc[j][r] = floatx4_t{0, 0, 0, 0};
    const uint16_t* a = p.a + (int64_t)tile.group * p.rank * p.K;
    const uint16_t* ar[kBlocks];
#pragma unroll
    for (int r = 0; r < kBlocks; ++r)   // rows past the rank: any, their results are set to 0
      ar[r] = a + (int64_t)min(r / 2 * 32 + m / 4 * 8 + r % 2 * 4 + m % 4, p.rank - 1) * p.K;
    uint8_t* const xs = room + wave * kAdapterTile * kRow;
    bf16x8_t x[8];
    const auto load = [&](int k0) {
      const int k = k0 + 8 * m;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (4 * i >= tile.count) continue;
        const uint16_t* xr = p.x + token[i] * p.x_stride;
        x[i] = k0 + kStepK <= p.K ? operand8(xr + k) : operand8(xr, k, p.K);
      }
    };
    const int first = kPart == kShares ? split * p.k_cols : 0, last = kPart == kShares ? min(p.K, first + p.k_cols) : p.K;
    int k0 = first + wave * kStepK;
    if (k0 < last) load(k0);
    for (; k0 < last; k0 += kWaves * kStepK) {
      const int k1 = k0 + kWaves * kStepK;
      bf16x8_t av[kBlocks][kAStep];
      const auto load_a = [&](int s0) {
#pragma unroll
        for (int s = 0; s < kAStep; ++s)
#pragma unroll
          for (int r = 0; r < kBlocks; ++r) {
            const int k = k0 + 32 * (s0 + s) + 8 * g;
            av[r][s] = k0 + kStepK <= p.K ? operand8(ar[r] + k) : operand8(ar[r], k, p.K);
          }
      };
      load_a(0);
      wave_order();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (4 * i < tile.count)
          *reinterpret_cast<u32x4_t*>(xs + (g + 4 * i) * kRow + 16 * m) = __builtin_bit_cast(u32x4_t, x[i]);
      if (k1 < last) load(k1);
      wave_order();
#pragma unroll
      for (int s0 = 0; s0 < 4; s0 += kAStep) {
        if (s0) load_a(s0);
#pragma unroll
        for (int s = 0; s < kAStep; ++s)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (j && !two) continue;
            const bf16x8_t xv = __builtin_bit_cast(
                bf16x8_t, *reinterpret_cast<const u32x4_t*>(xs + (row + 16 * j) * kRow + 64 * (s0 + s) + 16 * g));
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) acc[j][r] = mfma(av[r][s], xv, acc[j][r]);
          }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) share[wave][j * kBlocks + r][lane] = acc[j][r];
    __syncthreads();
    // each thread adds some places' shares, in wave order, into the first
    for (int i = threadIdx.x; i < kPlaces; i += kWaves * kWave) {
      floatx4_t* const s = &share[0][i / kWave][i % kWave];
      floatx4_t v = *s;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += share[w][i / kWave][i % kWave];
      if (kPart == kShares) static_cast<floatx4_t*>(p.shares)[((int64_t)index * p.k_splits + split) * kPlaces + i] = v;
      else *s = v;
    }
  }
  if (kPart == kShares) return;
  if (real) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const floatx4_t lo = share[0][j * kBlocks + 2 * c][lane], hi = share[0][j * kBlocks + 2 * c + 1][lane];
        const int r0 = 32 * c + 8 * g;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = r0 + e < p.rank ? (e < 4 ? lo[e % 4] : hi[e % 4]) : 0.0f;
        if (p.hidden && split == 0 && wave == 0 && row + 16 * j < tile.count && r0 < p.rank)
          store_run<SOLFP4_F32>(
              reinterpret_cast<uint8_t*>(p.hidden + token_at(p.t, tile.first + row + 16 * j) * p.rank), r0, p.rank - r0,
              from_f32<SOLFP4_F32>(v));
        bf16x8_t piece[3];
        split_bf16(v, piece);
#pragma unroll
        for (int s = 0; s < kHeld; ++s) h[j][c][s] = piece[s];
        if (kHeld == 2 && wave == 0) low[j * kChunks + c][lane] = piece[2];
      }
    if (kHeld == 2) __syncthreads();
  } else if (p.hidden && split == 0) {
    const float v = tile.group == p.t.adapters ? 0.0f : __builtin_nanf("");
    for (int i = threadIdx.x; i < tile.count * p.rank; i += kWaves * kWave)
      p.hidden[token_at(p.t, tile.first + i / p.rank) * p.rank + i % p.rank] = v;
  }

  const float scale = !real ? 0.0f : p.scales ? p.scales[tile.group] : 1.0f;
  const uint16_t* b = p.b + (real ? (int64_t)tile.group * p.N * p.rank : 0);
  const __amdgpu_buffer_rsrc_t whole_b = uniform_rsrc(b, real ? p.N * p.rank * 2 : 0);   // below 2^30 bytes
  const int end = min(p.N, (split + 1) * p.split_cols);
  LaneRun<kLane> y[8];
  const auto load = [&](int n0) {
    const int col = n0 + kLane * m;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (4 * i >= tile.count) continue;
      const uint16_t* yr = p.y + token[i] * p.y_stride;
      y[i].load(yr, col, p.N, n0 + kStepN <= p.N);
    }
  };
  bf16x8_t bv[kLane][kChunks];
  const auto load_b = [&](int n0) {
    if (!real) return;
#pragma unroll
    for (int q = 0; q < kLane; ++q) {
      const int n = min(n0 + kLane * m + q, p.N - 1);   // past the last column: any, not stored
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int r0 = 32 * c + 8 * g;
        // zeros past the rank, where an infinite weight times an h of 0 would be NaN: from past the buffer
        if constexpr (kWholeRank)
          bv[q][c] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(
                                                      whole_b, n * p.rank * 2 + (r0 < p.rank ? 2 * r0 : INT_MIN), 0, 0));
        else
          bv[q][c] = operand8(b + (int64_t)n * p.rank, r0, p.rank);
      }
    }
  };
  int n0 = split * p.split_cols + wave * kStepN;
  if (n0 < end) load(n0);
  if (kAhead && n0 < end) load_b(n0);
  for (; n0 < end; n0 += kWaves * kStepN) {
    const int n1 = n0 + kWaves * kStepN, col = n0 + kLane * m;
    bf16x8_t now_b[kLane][kChunks];
    if (!kAhead) load_b(n0);
#pragma unroll
    for (int q = 0; q < kLane; ++q)
#pragma unroll
      for (int c = 0; c < kChunks; ++c) now_b[q][c] = bv[q][c];
    if (kAhead && n1 < end) load_b(n1);
    LaneRun<kLane> now[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) now[i] = y[i];
    if (n1 < end) load(n1);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (j && !two) continue;
      floatx4_t acc[kLane];
#pragma unroll
      for (int q = 0; q < kLane; ++q) acc[q] = floatx4_t{0, 0, 0, 0};
      if (real) {
        int at = lane;
        if (kHeld == 2) asm volatile("" : "+v"(at));   // read here and not kept over the steps
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
          for (int s = 2; s >= 0; --s) {
            const bf16x8_t piece = s < kHeld ? h[j][c][s] : low[j * kChunks + c][at];
#pragma unroll
            for (int q = 0; q < kLane; ++q) acc[q] = mfma(piece, now_b[q][c], acc[q]);
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (g + 4 * i + 16 * j >= tile.count) continue;
        float v[kLane];
#pragma unroll
        for (int q = 0; q < kLane; ++q) {
          v[q] = now[4 * j + i].value(q);
          if (real) v[q] = __builtin_fmaf(scale, acc[q][i], v[q]);
          if (tile.group > p.t.adapters) v[q] = __builtin_nanf("");
        }
        now[4 * j + i].set(v);
        now[4 * j + i].store(p.out + token[4 * j + i] * p.out_stride, col, p.N, n0 + kStepN <= p.N);
      }
    }
  }
}

template <int kChunks, int kLane, int kWaves, int kPart>
static hipError_t launch_part(const AdapterArgs& a, hipStream_t stream) {
  const int64_t tiles = (a.t.max_tiles + a.xcds - 1) / a.xcds * a.xcds;
  const dim3 grid((unsigned)(tiles * (kPart == kShares ? a.k_splits : a.splits))), block(kWaves * kWave);
  if (a.rank % 8 == 0) return launch_kernel(add_adapters_kernel<kChunks, kLane, kWaves, true, kPart>, grid, block, stream, a);
  return launch_kernel(add_adapters_kernel<kChunks, kLane, kWaves, false, kPart>, grid, block, stream, a);
}

// Ranges of at least one step that a tile's `size` is cut to, at most `want`; their width.
static int cut(int64_t size, int64_t step, int64_t want, int* width) {
  const int64_t steps = size > step ? (size + step - 1) / step : 1;
  const int64_t ranges = want < 1 ? 1 : want < steps ? want : steps, each = (steps + ranges - 1) / ranges;
  *width = (int)(each * step);
  return (int)((steps + each - 1) / each);
}

// h in a launch of its own, its K shared by several workgroups, and the second
// product in another: where a tile's ranges would each go through a large a
// again (1 token 9728 -> 9728, rank 64: 38.9 us in one launch and 14.1 in two;
// 2048 tokens 2240 -> 2240, rank 64 23.1 and 20.5; 64 tokens of 48 adapters 2432 -> 7296,
// rank 32 12.6 and 13.2; 1 token 1152 -> 1152, rank 16 5.8 and 8.5).
constexpr int64_t kTwoLaunches = (int64_t)1 << 18;   // elements of one adapter's a
constexpr int kHWaves = 4, kOutWaves = 8;

static bool two_launches(const AdapterTokens& t, int64_t K, int64_t rank) {
  return t.max_tiles > 0 && t.max_tiles < device_cu_count() && rank * K >= kTwoLaunches;
}
static int h_ranges(const AdapterTokens& t, int64_t K, int* width) {
  return cut(K, kStepK * kHWaves, 2 * device_cu_count() / t.max_tiles, width);
}

size_t add_adapters_bytes(const AdapterTokens& t, int64_t K, int64_t rank) {
  if (!two_launches(t, K, rank)) return 0;
  int width;
  const int chunks = rank <= 32 ? 1 : rank <= 64 ? 2 : 4;
  return (size_t)(t.max_tiles * h_ranges(t, K, &width)) * 4 * chunks * kWave * sizeof(floatx4_t);
}

// A workgroup a tile where there are more than 1.25 tiles a CU, else ranges of a
// tile's columns, with more waves and shorter steps (8192 tokens 2240 -> 2240, 266
// tiles, 30 us so and 38 the other way; 12000 tokens 2432 -> 7296, 377 tiles, 113
// and 110).
template <int kChunks>
static hipError_t launch_rank(AdapterArgs a, hipStream_t stream) {
  const int64_t tiles = a.t.max_tiles, cus = device_cu_count();
  a.xcds = (int)(tiles < kXcds ? tiles : kXcds);
  if (a.shares) {
    a.k_splits = h_ranges(a.t, a.K, &a.k_cols);
    a.splits = cut(a.N, 64, cus / tiles, &a.split_cols);
    const hipError_t e = launch_part<kChunks, 4, kHWaves, kShares>(a, stream);
    return e != hipSuccess ? e : launch_part<kChunks, 4, kOutWaves, kFromShares>(a, stream);
  }
  if constexpr (kChunks == 4) {   // LDS holds four waves' shares of h
    a.splits = cut(a.N, 64, cus / tiles, &a.split_cols);
    return launch_part<4, 4, 4, kBoth>(a, stream);
  } else if (4 * tiles < 5 * cus) {
    a.splits = cut(a.N, 64, cus / tiles, &a.split_cols);
    return launch_part<kChunks, 4, 8, kBoth>(a, stream);
  } else {
    a.splits = cut(a.N, 128, 1, &a.split_cols);
    return launch_part<kChunks, 8, 4, kBoth>(a, stream);
  }
}

hipError_t launch_add_adapters(AdapterArgs a, void* workspace, hipStream_t stream) {
  a.shares = two_launches(a.t, a.K, a.rank) ? workspace : nullptr;
  if (a.t.tokens == 0 || (a.N == 0 && !a.hidden)) return hipSuccess;
  if (a.rank <= 32) return launch_rank<1>(a, stream);
  if (a.rank <= 64) return launch_rank<2>(a, stream);
  return launch_rank<4>(a, stream);
}

}  // namespace solfp4
