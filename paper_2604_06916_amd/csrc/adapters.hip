// Low-rank adapters beside a shared linear, many at once:
//
//   h_t = a_e x_t,  out_t = y_t + c_e b_e h_t,  e the adapter of token t
//
// x [tokens][K], y [tokens][N] and the adapters' a [rank][K], b [N][rank] are
// BF16; h is FP32 (rank values a token) and goes into the second product as
// two BF16 pieces, 16 of its bits, so that its rounding (2^-17) is far below
// the output's.
//
// A workgroup takes a tile of up to 32 tokens of one adapter (the plan brings
// them together) and a range of N: its waves share K, add their shares of h in
// LDS in wave order, and share the columns.  Tokens are the columns of the
// matrix instructions; the rows, r in the first product and n in the second,
// are dealt so that a lane's results are consecutive: row 4 g + i of blocks 2 u
// and 2 u + 1 is element 32 u + 8 g + i and four further on.  So h is the second
// product's operand as it stands, and a wave reads and writes 64 bytes of each
// token's row an instruction.
//
// Bound by memory: x once, y once in and once out; a and b come from L2, as
// often as there are tiles.
#include "adapters.h"

namespace solfp4 {

// ---- plan -----------------------------------------------------------------

constexpr int kPlanThreads = 1024, kPlanDeep = 8;

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
  return (size_t)(t.tiles_at + 4 * t.max_tiles) * 4;
}

template <typename Index>
__device__ __forceinline__ int group_of(const Index* index, int64_t i, int adapters) {
  const Index v = index[i];
  return v < 0 ? adapters : v < adapters ? (int)v : adapters + 1;
}

// A workgroup a group: counts the tokens of the groups before its own, then
// puts its tokens behind them in their order.  Each reads the index twice, so
// no workgroup waits for another.
template <typename Index>
__global__ __launch_bounds__(kPlanThreads) void plan_order_kernel(const Index* __restrict__ index, AdapterTokens t,
                                                                  int* __restrict__ plan) {
  constexpr int kWaves = kPlanThreads / kWave;
  __shared__ int sums[kWaves];
  const int group = blockIdx.x, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  int before = 0;
  for (int64_t base = 0; base < t.tokens; base += kPlanThreads * kPlanDeep) {
    int g[kPlanDeep];
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u) {
      const int64_t i = base + u * kPlanThreads + threadIdx.x;
      g[u] = i < t.tokens ? group_of(index, i, t.adapters) : group;
    }
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u) before += g[u] < group;
  }
  before = lanes_sum(before, kWave);
  if (lane == 0) sums[wave] = before;
  __syncthreads();
  int at = 0;
  for (int w = 0; w < kWaves; ++w) at += sums[w];
  if (threadIdx.x == 0) plan[t.places_at + group] = at;
  for (int64_t base = 0; base < t.tokens; base += kPlanThreads * kPlanDeep) {
    // a thread's kPlanDeep tokens follow each other, so that places ascend with them
    const int64_t first = base + (int64_t)threadIdx.x * kPlanDeep;
    uint32_t mine = 0;
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u)
      if (first + u < t.tokens && group_of(index, first + u, t.adapters) == group) mine |= 1u << u;
    const int n = __builtin_popcount(mine);
    int below = n;   // of this lane and the lanes before it
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int o = __shfl_up(below, d, kWave);
      if (lane >= d) below += o;
    }
    __syncthreads();
    if (lane == kWave - 1) sums[wave] = below;
    __syncthreads();
    int place = at + below - n;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) place += sums[w];
      at += sums[w];
    }
#pragma unroll
    for (int u = 0; u < kPlanDeep; ++u)
      if (mine >> u & 1) plan[t.order_at + place++] = (int)(first + u);
  }
  if (threadIdx.x == 0 && group == t.adapters + 1) plan[t.places_at + group + 1] = at;
}

// First tile of every group: one workgroup adds up the groups' tiles.
__global__ __launch_bounds__(kPlanThreads) void plan_starts_kernel(AdapterTokens t, int* __restrict__ plan) {
  constexpr int kWaves = kPlanThreads / kWave;
  __shared__ int sums[kWaves];
  const int groups = t.adapters + 2, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int* places = plan + t.places_at;
  int at = 0;
  for (int base = 0; base < groups; base += kPlanThreads) {
    const int g = base + threadIdx.x;
    const int n = g < groups ? (places[g + 1] - places[g] + kAdapterTile - 1) / kAdapterTile : 0;
    int upto = n;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int o = __shfl_up(upto, d, kWave);
      if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    int first = at + upto - n;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) first += sums[w];
      at += sums[w];
    }
    if (g < groups) plan[g] = first;
  }
  if (threadIdx.x == 0) plan[groups] = at;
}

// The tiles: a thread finds its tile's group among the groups' first tiles.
__global__ __launch_bounds__(256) void plan_tiles_kernel(AdapterTokens t, int* __restrict__ plan) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= t.max_tiles) return;
  const int groups = t.adapters + 2;
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

hipError_t launch_adapter_plan(const void* index, int index_bytes, int64_t tokens, int64_t adapters, void* plan,
                               hipStream_t stream) {
  const AdapterTokens t = adapter_tokens(plan, tokens, adapters);
  int* p = static_cast<int*>(plan);
  const dim3 groups((unsigned)(adapters + 2)), block(kPlanThreads);
  hipError_t e = index_bytes == 4
                     ? launch_kernel(plan_order_kernel<int32_t>, groups, block, stream, (const int32_t*)index, t, p)
                     : launch_kernel(plan_order_kernel<int64_t>, groups, block, stream, (const int64_t*)index, t, p);
  if (e == hipSuccess) e = launch_kernel(plan_starts_kernel, dim3(1), block, stream, t, p);
  if (e == hipSuccess && t.max_tiles > 0)
    e = launch_kernel(plan_tiles_kernel, dim3((unsigned)((t.max_tiles + 255) / 256)), dim3(256), stream, t, p);
  return e;
}

// ---- forward --------------------------------------------------------------

constexpr int kStepK = 64, kStepN = 64;   // of a wave's step

// kChunks: 32s of the rank; kWholeRank: the rank is a multiple of 8.
template <int kChunks, int kWaves, bool kWholeRank>
__global__ __launch_bounds__(kWaves * kWave) void add_adapters_kernel(AdapterArgs p) {
  constexpr int kBlocks = 2 * kChunks;   // 16s of the rank
  constexpr bool kAhead = kChunks < 4;   // the next step's loads go out before this one's products
  __shared__ floatx4_t share[kWaves][2 * kBlocks][kWave];
  // the column ranges of a tile run on one XCD, where its rows are then in L2
  const int id = blockIdx.x, at = id / kXcds;
  const int64_t index = (int64_t)(at / p.splits) * kXcds + id % kXcds;
  const int split = at % p.splits;
  if (index >= p.t.max_tiles) return;
  const Tile tile = uniform(load_tile(p.t, (int)index));
  if (tile.count == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int m = lane % 16, g = lane / 16;
  const bool two = tile.count > 16;          // tokens in both blocks of 16
  const bool real = tile.group < p.t.adapters;
  int64_t token[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) token[j] = token_at(p.t, tile.first + min(m + 16 * j, tile.count - 1));

  bf16x8_t h[2][kChunks][2];   // two pieces of h of this lane's tokens
  if (real) {
    floatx4_t acc[2][kBlocks];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) acc[j][r] = floatx4_t{0, 0, 0, 0};
    const uint16_t* a = p.a + (int64_t)tile.group * p.rank * p.K;
    const uint16_t *xr[2], *ar[kBlocks];
#pragma unroll
    for (int j = 0; j < 2; ++j) xr[j] = p.x + token[j] * p.x_stride;
#pragma unroll
    for (int r = 0; r < kBlocks; ++r)   // rows past the rank: any, their results are set to 0
      ar[r] = a + (int64_t)min(r / 2 * 32 + m / 4 * 8 + r % 2 * 4 + m % 4, p.rank - 1) * p.K;
    struct Step {
      bf16x8_t x[2][2], a[kBlocks][2];
    };
    const auto load = [&](int k0, Step& v) {
      const int k = k0 + 8 * g;
      const bool whole = k0 + kStepK <= p.K;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int at = k + 32 * s, n = p.K - at;
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (j == 0 || two) v.x[j][s] = whole ? operand8(xr[j] + at) : operand8(xr[j], at, n);
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) v.a[r][s] = whole ? operand8(ar[r] + at) : operand8(ar[r], at, n);
      }
    };
    Step now, next;
    int k0 = wave * kStepK;
    if (k0 < p.K) load(k0, now);
    for (; k0 < p.K; k0 += kWaves * kStepK) {
      const int k1 = k0 + kWaves * kStepK;
      if (kAhead && k1 < p.K) load(k1, next);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
          acc[0][r] = mfma(now.a[r][s], now.x[0][s], acc[0][r]);
          if (two) acc[1][r] = mfma(now.a[r][s], now.x[1][s], acc[1][r]);
        }
      if (!kAhead && k1 < p.K) load(k1, now);
      if (kAhead) now = next;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) share[wave][j * kBlocks + r][lane] = acc[j][r];
    __syncthreads();
    // each thread adds some places' shares, in wave order, into the first
    for (int i = threadIdx.x; i < 2 * kBlocks * kWave; i += kWaves * kWave) {
      floatx4_t* const s = &share[0][i / kWave][i % kWave];
      floatx4_t v = *s;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += share[w][i / kWave][i % kWave];
      *s = v;
    }
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
        if (p.hidden && split == 0 && wave == 0 && m + 16 * j < tile.count)
          store_run<SOLFP4_F32>(reinterpret_cast<uint8_t*>(p.hidden + token[j] * p.rank), r0, p.rank - r0,
                                from_f32<SOLFP4_F32>(v));
        split_bf16(v, h[j][c]);
      }
  } else if (p.hidden && split == 0) {
    const float v = tile.group == p.t.adapters ? 0.0f : __builtin_nanf("");
    for (int i = threadIdx.x; i < tile.count * p.rank; i += kWaves * kWave)
      p.hidden[token_at(p.t, tile.first + i / p.rank) * p.rank + i % p.rank] = v;
  }

  const float scale = !real ? 0.0f : p.scales ? p.scales[tile.group] : 1.0f;
  const uint16_t* b = p.b + (real ? (int64_t)tile.group * p.N * p.rank : 0);
  const int end = min(p.N, (split + 1) * p.split_cols);
  struct Step {
    Run<SOLFP4_BF16> y[2][2];
    bf16x8_t b[4][kChunks];
  };
  const auto load = [&](int n0, Step& v) {
    const bool whole = n0 + kStepN <= p.N;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (j == 1 && !two) continue;
      const uint16_t* yr = p.y + token[j] * p.y_stride;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int col = n0 + 32 * u + 8 * g;
        v.y[j][u].p[0] = __builtin_bit_cast(u32x4_t, whole ? operand8(yr + col) : operand8(yr, col, p.N - col));
      }
    }
    if (!real) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = min(n0 + q / 2 * 32 + m / 4 * 8 + q % 2 * 4 + m % 4, p.N - 1);   // past the last column: any, not stored
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        // past the rank: any of the row, times an h of 0
        const int r0 = 32 * c + 8 * g;
        if constexpr (kWholeRank) v.b[q][c] = operand8(b + (int64_t)n * p.rank + min(r0, p.rank - 8));
        else v.b[q][c] = operand8(b + (int64_t)n * p.rank, r0, p.rank - r0);
      }
    }
  };
  Step now, next;
  int n0 = split * p.split_cols + wave * kStepN;
  if (n0 < end) load(n0, now);
  for (; n0 < end; n0 += kWaves * kStepN) {
    const int n1 = n0 + kWaves * kStepN;
    if (kAhead && n1 < end) load(n1, next);
    floatx4_t acc[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[j][q] = floatx4_t{0, 0, 0, 0};
    if (real)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
          for (int s = 1; s >= 0; --s) {
            acc[0][q] = mfma(now.b[q][c], h[0][c][s], acc[0][q]);
            if (two) acc[1][q] = mfma(now.b[q][c], h[1][c][s], acc[1][q]);
          }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (m + 16 * j >= tile.count) continue;
      uint8_t* o = reinterpret_cast<uint8_t*>(p.out + token[j] * p.out_stride);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int col = n0 + 32 * u + 8 * g;
        float v[8];
        to_f32<SOLFP4_BF16>(now.y[j][u], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = real ? __builtin_fmaf(scale, acc[j][2 * u + e / 4][e % 4], v[e]) : v[e];
          if (tile.group > p.t.adapters) v[e] = __builtin_nanf("");
        }
        const Run<SOLFP4_BF16> r = from_f32<SOLFP4_BF16>(v);
        if (n0 + kStepN <= p.N) store_run<SOLFP4_BF16>(o, col, 8, r);
        else if (col < p.N) store_run<SOLFP4_BF16>(o, col, p.N - col, r);
      }
    }
    if (!kAhead && n1 < end) load(n1, now);
    if (kAhead) now = next;
  }
}

template <int kChunks, int kWaves>
static hipError_t launch_forward(const AdapterArgs& a, dim3 grid, hipStream_t stream) {
  const dim3 block(kWaves * kWave);
  if (a.rank % 8 == 0) return launch_kernel(add_adapters_kernel<kChunks, kWaves, true>, grid, block, stream, a);
  return launch_kernel(add_adapters_kernel<kChunks, kWaves, false>, grid, block, stream, a);
}

template <int kChunks>
static hipError_t launch_rank(AdapterArgs a, hipStream_t stream) {
  const int64_t tiles = a.t.max_tiles, steps = a.N > kStepN ? (a.N + kStepN - 1) / kStepN : 1;
  const int64_t cus = device_cu_count();
  // column ranges a tile, so that there is a workgroup a CU
  int64_t splits = tiles < cus ? cus / tiles : 1;
  splits = splits < steps ? splits : steps;
  splits = splits < 1 ? 1 : splits;
  const int64_t each = (steps + splits - 1) / splits;
  a.split_cols = (int)(each * kStepN);
  a.splits = (int)((steps + each - 1) / each);
  const dim3 grid((unsigned)((tiles + kXcds - 1) / kXcds * kXcds * a.splits));
#ifndef FW
#define FW 4
#endif
  if constexpr (kChunks < 4)   // more shares than LDS holds twice
    if (tiles < 3 * cus) return launch_forward<kChunks, 8>(a, grid, stream);
  if constexpr (kChunks == 1) return launch_forward<kChunks, FW>(a, grid, stream);
  return launch_forward<kChunks, 4>(a, grid, stream);
}

hipError_t launch_add_adapters(const AdapterArgs& a, hipStream_t stream) {
  if (a.t.tokens == 0 || (a.N == 0 && !a.hidden)) return hipSuccess;
  if (a.rank <= 32) return launch_rank<1>(a, stream);
  if (a.rank <= 64) return launch_rank<2>(a, stream);
  return launch_rank<4>(a, stream);
}

}  // namespace solfp4
