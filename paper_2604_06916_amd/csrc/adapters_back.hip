// Gradients of low-rank adapters:
//
//   g_t = c_e b_e^T dy_t          dx_t = past_t + a_e^T g_t
//   db_e = c_e sum_t dy_t h_t^T   da_e = sum_t g_t x_t^T      t the tokens of e
//
// dy and x are read once.  A first pass takes dy: a wave holds 16 kCols of its
// columns for db's sums over a run of tiles (slice) and adds its share of g,
// which needs all of N: the waves of a workgroup add theirs in LDS, the
// workgroups' go through the workspace.  A second kernel adds those and writes
// g as the matrix operands that the third needs, which takes x, past and dx: a
// wave holds 16 kCols columns of da.  The last adds the slices' da and db.
// All sums have a fixed order, so results are the same on every call.
//
// Both passes multiply by a token's values twice: once with the token's row
// as it lies in memory (g, dx) and once summed over tokens, for which the row's
// columns must be lanes and the tokens the reduction: the tile goes through
// LDS and comes back transposed (ds_read_b64_tr_b16).
//
// FP32 factors (h, g) enter the products as BF16 pieces: three, all 24 bits,
// for da and db, which are FP32; two for dx, which is BF16.
//
// Slices and tiles: slice s of tiles_each tiles leaves its sums of adapter e in
// slot s + e.  Tiles are sorted by adapter, so two slices of one adapter or two
// adapters of one slice never share a slot.
#include "adapters.h"

namespace solfp4 {

namespace {

constexpr int kWaves = 8;        // of a workgroup of the first pass
constexpr int kXWaves = 4;       // of the second, whose waves go by themselves

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t* lds_short4_t;

// Blocks of 16 columns of a wave, so that the sums take 64 registers.
constexpr int cols_of(int chunks) { return 8 / chunks; }

// How the work is dealt and where everything lies in the workspace.
struct Deal {
  int64_t tiles;
  int units_n, chunks_n, units_x;       // waves' columns of N and K; workgroups along N
  int slices_n, each_n, slices_x, each_x;
  int64_t slots_n, slots_x;
  int64_t share, pieces2, pieces3, db, da, bytes;   // offsets of floatx4_t places, bytes at the end
};

struct BackArgs {
  AdapterBackArgs p;
  Deal d;
  floatx4_t* ws;
};

Deal deal(const AdapterTokens& t, int64_t N, int64_t K, int64_t rank) {
  const int chunks = rank <= 32 ? 1 : rank <= 64 ? 2 : 4, cols = 16 * cols_of(chunks), blocks = 2 * chunks;
  const int64_t cus = device_cu_count();
  Deal d = {};
  d.tiles = t.max_tiles;
  d.units_n = (int)((N + cols - 1) / cols);
  d.units_x = (int)((K + cols - 1) / cols);
  d.chunks_n = (d.units_n + kWaves - 1) / kWaves;
  const auto slices = [&](int64_t want, int* each) {
    want = want < 1 ? 1 : want < d.tiles ? want : d.tiles;
    *each = (int)(want > 0 ? (d.tiles + want - 1) / want : 1);
    return (int)((d.tiles + *each - 1) / *each);
  };
  d.slices_n = slices(d.chunks_n ? cus / d.chunks_n : 1, &d.each_n);
  d.slices_x = slices(d.units_x ? 8 * cus / d.units_x : 1, &d.each_x);
  d.slots_n = d.slices_n + t.adapters;
  d.slots_x = d.slices_x + t.adapters;
  const int64_t frag = blocks * kWave;
  int64_t at = 0;
  const auto take = [&](int64_t n) {
    const int64_t was = at;
    at += n;
    return was;
  };
  d.share = take((int64_t)d.chunks_n * d.tiles * 2 * frag);
  d.pieces2 = take(d.tiles * chunks * 2 * 2 * kWave);
  d.pieces3 = take(d.tiles * 3 * frag);
  d.db = take(d.slots_n * d.units_n * cols_of(chunks) * frag);
  d.da = take(d.slots_x * d.units_x * cols_of(chunks) * frag);
  d.bytes = at * 16;
  return d;
}

__device__ __forceinline__ bf16x8_t none8() { return __builtin_bit_cast(bf16x8_t, u32x4_t{0, 0, 0, 0}); }

// One wave's tile in LDS, [token][column]; rows 32 bytes apart beyond their
// columns, so that the eight rows that half a wave reads lie in different banks.
template <int kCols>
struct TileLds {
  static constexpr int kRow = kCols * 32 + 32;
  uint8_t* base;
  __device__ __forceinline__ void put(int token, int col, bf16x8_t v) const {
    *reinterpret_cast<u32x4_t*>(base + token * kRow + col * 2) = __builtin_bit_cast(u32x4_t, v);
  }
  // Block c with the columns as lanes: element j of lane (m, g) is column 16 c + m of token 16 (j / 4) + 4 g + j % 4.
  __device__ __forceinline__ bf16x8_t transposed(int c, int lane) const {
    const int i = lane % 16, g = lane / 16;
    short4_t v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint8_t* at = base + (16 * h + 4 * g + i / 4) * kRow + (16 * c + i % 4 * 4) * 2;
      v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)at);
    }
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// The two tokens of a lane in a tile, m and m + 16 (the last one where the tile ends before).
struct Pair {
  int64_t token[2];
};
__device__ __forceinline__ Pair pair_of(const AdapterTokens& t, const Tile& tile, int m) {
  Pair p;
#pragma unroll
  for (int j = 0; j < 2; ++j) p.token[j] = token_at(t, tile.first + min(m + 16 * j, tile.count - 1));
  return p;
}

// A tile's rows as they lie: element k of [j][s] is column col0 + 32 s + 8 g + k of token m + 16 j.
template <int kCols>
struct Rows {
  bf16x8_t v[2][kCols / 2];
  __device__ __forceinline__ void load(const uint16_t* base, int64_t stride, const Pair& pair, int col0, int cols,
                                       int g) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint16_t* row = base + pair.token[j] * stride;
#pragma unroll
      for (int s = 0; s < kCols / 2; ++s) {
        const int c = col0 + 32 * s + 8 * g;
        v[j][s] = col0 + 16 * kCols <= cols ? operand8(row + c) : operand8(row, c, cols);
      }
    }
  }
  // zeros in the place of tokens past the tile's end
  __device__ __forceinline__ void clear(int count, int m) {
    if (count == kAdapterTile) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int s = 0; s < kCols / 2; ++s)
        if (m + 16 * j >= count) v[j][s] = none8();
  }
};

// ---- the pass over dy -----------------------------------------------------

template <int kChunks>
__global__ __launch_bounds__(kWaves * kWave, 2) void adapters_back_y_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks, kCols = cols_of(kChunks);
  constexpr int kRounds = kChunks == 4 ? 2 : 1, kShared = 2 * kBlocks / kRounds;   // LDS holds all shares of a round
  __shared__ floatx4_t share[kWaves][kShared][kWave];
  __shared__ bf16x8_t factor[3][kBlocks][kWave];
  __shared__ __attribute__((aligned(16))) uint8_t tiles[kWaves][kAdapterTile * TileLds<kCols>::kRow];
  const AdapterBackArgs& p = q.p;
  const int slice = blockIdx.x / q.d.chunks_n, chunk = blockIdx.x - slice * q.d.chunks_n;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int m = lane % 16, g = lane / 16;
  // the chunk's units, dealt evenly; a wave without one only keeps step
  const int from = (int)((int64_t)q.d.units_n * chunk / q.d.chunks_n);
  const int to = (int)((int64_t)q.d.units_n * (chunk + 1) / q.d.chunks_n);
  const int unit = from + wave;
  const bool works = unit < to;
  const int col0 = unit * 16 * kCols;
  const TileLds<kCols> lds{tiles[wave]};

  floatx4_t acc[kCols][kBlocks];
  bf16x8_t bt[kBlocks][kCols / 2];
  int group = -1;
  const auto flush = [&] {
    if (group >= 0 && works) {
      floatx4_t* to_ = q.ws + q.d.db + ((int64_t)(slice + group) * q.d.units_n + unit) * kCols * kBlocks * kWave + lane;
#pragma unroll
      for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) to_[(c * kBlocks + r) * kWave] = acc[c][r];
    }
  };
  const auto begin = [&](int e) {
    group = e;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) acc[c][r] = floatx4_t{0, 0, 0, 0};
    // b^T: row 4 g + i of block r is rank element 32 (r / 2) + 8 g + 4 (r % 2) + i
    const uint16_t* b = p.b + (int64_t)e * p.N * p.rank;
#pragma unroll
    for (int r = 0; r < kBlocks; ++r) {
      const int at = 32 * (r / 2) + m / 4 * 8 + r % 2 * 4 + m % 4;
#pragma unroll
      for (int s = 0; s < kCols / 2; ++s) {
        u32x4_t w = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int n = col0 + 32 * s + 8 * g + k;
          if (works && n < p.N && at < p.rank) w[k / 2] |= (uint32_t)b[(int64_t)n * p.rank + at] << (16 * (k & 1));
        }
        bt[r][s] = __builtin_bit_cast(bf16x8_t, w);
      }
    }
  };

  const int first = slice * q.d.each_n, end = min(first + q.d.each_n, (int)q.d.tiles);
  for (int i = first; i < end; ++i) {
    const Tile tile = uniform(load_tile(p.t, i));
    if (tile.count == 0 || tile.group >= p.t.adapters) break;   // adapters' tiles come first
    const Pair pair = pair_of(p.t, tile, m);
    Rows<kCols> dy;
    if (works) {
      dy.load(p.dy, p.dy_stride, pair, col0, p.N, g);
      dy.clear(tile.count, m);
    }
    if (tile.group != group) {
      flush();
      begin(tile.group);
    }
    // h as an operand, its tokens in the transposed tile's order
    for (int r = wave; r < kBlocks; r += kWaves) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int t = 16 * (k / 4) + 4 * g + k % 4, at = 16 * r + m;
        v[k] = t < tile.count && at < p.rank ? p.hidden[token_at(p.t, tile.first + t) * p.rank + at] : 0.0f;
      }
      bf16x8_t piece[3];
      split_bf16(v, piece);
#pragma unroll
      for (int s = 0; s < 3; ++s) factor[s][r][lane] = piece[s];
    }
    __syncthreads();
    floatx4_t part[2][kBlocks];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) part[j][r] = floatx4_t{0, 0, 0, 0};
    if (works) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int s = 0; s < kCols / 2; ++s) lds.put(m + 16 * j, 32 * s + 8 * g, dy.v[j][s]);
      wave_order();
#pragma unroll
      for (int s = 0; s < kCols / 2; ++s)
#pragma unroll
        for (int r = 0; r < kBlocks; ++r)
#pragma unroll
          for (int j = 0; j < 2; ++j) part[j][r] = mfma(bt[r][s], dy.v[j][s], part[j][r]);
      bf16x8_t z[kCols];
#pragma unroll
      for (int c = 0; c < kCols; ++c) z[c] = lds.transposed(c, lane);
#pragma unroll
      for (int r = 0; r < kBlocks; ++r)
#pragma unroll
        for (int s = 2; s >= 0; --s) {
          const bf16x8_t f = factor[s][r][lane];
#pragma unroll
          for (int c = 0; c < kCols; ++c) acc[c][r] = mfma(f, z[c], acc[c][r]);
        }
      wave_order();
    }
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
      if (round) __syncthreads();
#pragma unroll
      for (int v = 0; v < kShared; ++v) {
        const int at = round * kShared + v;
        share[wave][v][lane] = part[at / kBlocks][at % kBlocks];
      }
      __syncthreads();
      floatx4_t* to_ = q.ws + q.d.share + (((int64_t)chunk * q.d.tiles + i) * kRounds + round) * kShared * kWave;
      for (int k = threadIdx.x; k < kShared * kWave; k += kWaves * kWave) {
        floatx4_t v = share[0][k / kWave][k % kWave];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += share[w][k / kWave][k % kWave];
        to_[k] = v;
      }
    }
  }
  flush();
}

// ---- g from its shares ----------------------------------------------------

template <int kChunks>
__global__ __launch_bounds__(256) void adapters_back_g_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks, kRow = 16 * kBlocks + 1;
  __shared__ float gs[kAdapterTile][kRow];
  const AdapterBackArgs& p = q.p;
  const int i = blockIdx.x;
  const Tile tile = uniform(load_tile(p.t, i));
  if (tile.count == 0 || tile.group >= p.t.adapters) return;
  const float scale = p.scales ? p.scales[tile.group] : 1.0f;
  const floatx4_t* from = q.ws + q.d.share + (int64_t)i * 2 * kBlocks * kWave;
  const int64_t hop = q.d.tiles * 2 * kBlocks * kWave;
  for (int k = threadIdx.x; k < kBlocks * kWave; k += 256) {
    // eight values of a token, from two blocks
    const int lane = k % kWave, jc = k / kWave, j = jc / kChunks, c = jc % kChunks;
    const int at = (j * kBlocks + 2 * c) * kWave + lane;
    floatx4_t lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    for (int n = 0; n < q.d.chunks_n; ++n) {
      lo += from[n * hop + at];
      hi += from[n * hop + at + kWave];
    }
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = scale * (e < 4 ? lo[e % 4] : hi[e % 4]);
      gs[lane % 16 + 16 * j][32 * c + lane / 16 * 8 + e] = v[e];
    }
    bf16x8_t piece[2];
    split_bf16(v, piece);
#pragma unroll
    for (int s = 0; s < 2; ++s)
      q.ws[q.d.pieces2 + (((int64_t)i * kChunks + c) * 2 + j) * 2 * kWave + s * kWave + lane] =
          __builtin_bit_cast(floatx4_t, piece[s]);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < kBlocks * kWave; k += 256) {
    const int lane = k % kWave, r = k / kWave, g = lane / 16;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gs[16 * (e / 4) + 4 * g + e % 4][16 * r + lane % 16];
    bf16x8_t piece[3];
    split_bf16(v, piece);
#pragma unroll
    for (int s = 0; s < 3; ++s)
      q.ws[q.d.pieces3 + ((int64_t)i * 3 + s) * kBlocks * kWave + r * kWave + lane] =
          __builtin_bit_cast(floatx4_t, piece[s]);
  }
}

// ---- the pass over x ------------------------------------------------------

template <int kChunks>
__global__ __launch_bounds__(kXWaves * kWave, 2) void adapters_back_x_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks, kCols = cols_of(kChunks);
  constexpr int kRun = kCols < 4 ? kCols : 4, kRuns = kCols / kRun;   // blocks whose columns a lane holds in a row
  __shared__ __attribute__((aligned(16))) uint8_t tiles[kXWaves][kAdapterTile * TileLds<kCols>::kRow];
  const AdapterBackArgs& p = q.p;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int64_t id = (int64_t)blockIdx.x * kXWaves + wave;
  const int slice = (int)(id / q.d.units_x), unit = (int)(id - (int64_t)slice * q.d.units_x);
  if (slice >= q.d.slices_x) return;
  const int m = lane % 16, g = lane / 16, col0 = unit * 16 * kCols;
  const TileLds<kCols> lds{tiles[wave]};

  floatx4_t acc[kCols][kBlocks];
  bf16x8_t at[kCols][kChunks];
  int group = -1;
  const auto flush = [&] {
    if (group >= 0 && group < p.t.adapters) {
      floatx4_t* to = q.ws + q.d.da + ((int64_t)(slice + group) * q.d.units_x + unit) * kCols * kBlocks * kWave + lane;
#pragma unroll
      for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) to[(c * kBlocks + r) * kWave] = acc[c][r];
    }
  };
  const auto begin = [&](int e) {
    group = e;
    if (e >= p.t.adapters) return;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
      for (int r = 0; r < kBlocks; ++r) acc[c][r] = floatx4_t{0, 0, 0, 0};
    // a^T: row 4 g + i of block c is column 16 kRun (c / kRun) + 4 kRun g + 4 (c % kRun) + i
    const uint16_t* a = p.a + (int64_t)e * p.rank * p.K;
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      const int col = col0 + c / kRun * 16 * kRun + m / 4 * 4 * kRun + c % kRun * 4 + m % 4;
#pragma unroll
      for (int h = 0; h < kChunks; ++h) {
        u32x4_t w = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = 32 * h + 8 * g + k;
          if (col < p.K && r < p.rank) w[k / 2] |= (uint32_t)a[(int64_t)r * p.K + col] << (16 * (k & 1));
        }
        at[c][h] = __builtin_bit_cast(bf16x8_t, w);
      }
    }
  };

  const int first = slice * q.d.each_x, end = min(first + q.d.each_x, (int)q.d.tiles);
  for (int i = first; i < end; ++i) {
    const Tile tile = uniform(load_tile(p.t, i));
    if (tile.count == 0) break;
    const bool real = tile.group < p.t.adapters;
    const Pair pair = pair_of(p.t, tile, m);
    if (tile.group != group) {
      flush();
      begin(tile.group);
    }
    bf16x8_t two[kChunks][2][2];
    if (real) {
      Rows<kCols> x;
      x.load(p.x, p.x_stride, pair, col0, p.K, g);
      x.clear(tile.count, m);
#pragma unroll
      for (int h = 0; h < kChunks; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int s = 0; s < 2; ++s)
            two[h][j][s] = __builtin_bit_cast(
                bf16x8_t, q.ws[q.d.pieces2 + (((int64_t)i * kChunks + h) * 2 + j) * 2 * kWave + s * kWave + lane]);
      wave_order();
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int s = 0; s < kCols / 2; ++s) lds.put(m + 16 * j, 32 * s + 8 * g, x.v[j][s]);
      wave_order();
      bf16x8_t z[kCols];
#pragma unroll
      for (int c = 0; c < kCols; ++c) z[c] = lds.transposed(c, lane);
#pragma unroll
      for (int r = 0; r < kBlocks; ++r)
#pragma unroll
        for (int s = 2; s >= 0; --s) {
          const bf16x8_t f = __builtin_bit_cast(
              bf16x8_t, q.ws[q.d.pieces3 + ((int64_t)i * 3 + s) * kBlocks * kWave + r * kWave + lane]);
#pragma unroll
          for (int c = 0; c < kCols; ++c) acc[c][r] = mfma(f, z[c], acc[c][r]);
        }
    }
#pragma unroll
    for (int u = 0; u < kRuns; ++u) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int col = col0 + u * 16 * kRun + g * 4 * kRun;
        floatx4_t d[kRun];
#pragma unroll
        for (int c = 0; c < kRun; ++c) d[c] = floatx4_t{0, 0, 0, 0};
        if (real)
#pragma unroll
          for (int c = 0; c < kRun; ++c)
#pragma unroll
            for (int h = 0; h < kChunks; ++h)
#pragma unroll
              for (int s = 1; s >= 0; --s) d[c] = mfma(at[u * kRun + c][h], two[h][j][s], d[c]);
        if (m + 16 * j >= tile.count) continue;
        const uint8_t* pr = reinterpret_cast<const uint8_t*>(p.past + pair.token[j] * p.past_stride);
        uint8_t* o = reinterpret_cast<uint8_t*>(p.dx + pair.token[j] * p.dx_stride);
#pragma unroll
        for (int w = 0; w < kRun / 2; ++w) {
          const int c0 = col + 8 * w, n = p.K - c0;
          if (n <= 0) continue;
          float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
          if (p.past) to_f32<SOLFP4_BF16>(load_run<SOLFP4_BF16>(pr, c0, n), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (real) v[e] += d[2 * w + e / 4][e % 4];
            if (tile.group > p.t.adapters) v[e] = __builtin_nanf("");
          }
          store_run<SOLFP4_BF16>(o, c0, n, from_f32<SOLFP4_BF16>(v));
        }
      }
    }
  }
  flush();
}

// ---- da and db from the slices' sums --------------------------------------

// One thread a place of four rank elements of a column; db first, then da.
template <int kChunks>
__global__ __launch_bounds__(256) void adapters_back_sums_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks, kCols = cols_of(kChunks);
  const AdapterBackArgs& p = q.p;
  const int64_t per_n = (int64_t)q.d.units_n * kCols * kBlocks * kWave, per_x = (int64_t)q.d.units_x * kCols * kBlocks * kWave;
  const int64_t all = p.t.adapters * (per_n + per_x);
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
    const bool is_db = id < p.t.adapters * per_n;
    const int64_t k = is_db ? id : id - p.t.adapters * per_n, per = is_db ? per_n : per_x;
    const int e = (int)(k / per);
    const int64_t place = k - e * per;
    int begin = 0, end = (int)q.d.tiles;   // the adapter's tiles
    if (p.t.plan) begin = p.t.plan[e], end = p.t.plan[e + 1];
    floatx4_t v = {0, 0, 0, 0};
    if (begin < end) {
      const int each = is_db ? q.d.each_n : q.d.each_x;
      const floatx4_t* from = q.ws + (is_db ? q.d.db : q.d.da) + place;
      for (int s = begin / each; s <= (end - 1) / each; ++s) v += from[(s + e) * per];
    }
    const int lane = (int)(place % kWave), r = (int)(place / kWave % kBlocks);
    const int64_t col = place / kWave / kBlocks * 16 + lane % 16;
    const int at = 16 * r + lane / 16 * 4, left = p.rank - at;
    if (is_db) {
      if (col >= p.N) continue;
      const float scale = p.scales ? p.scales[e] : 1.0f;
      float* to = p.db + ((int64_t)e * p.N + col) * p.rank + at;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < left) to[c] = scale * v[c];
    } else {
      if (col >= p.K) continue;
      float* to = p.da + ((int64_t)e * p.rank + at) * p.K + col;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < left) to[c * (int64_t)p.K] = v[c];
    }
  }
}

template <int kChunks>
hipError_t launch_back(const BackArgs& q, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (q.d.tiles > 0) {
    if (q.d.chunks_n > 0)
      e = launch_kernel(adapters_back_y_kernel<kChunks>, dim3((unsigned)(q.d.chunks_n * q.d.slices_n)),
                        dim3(kWaves * kWave), stream, q);
    if (e == hipSuccess && q.d.units_x > 0)
      e = launch_kernel(adapters_back_g_kernel<kChunks>, dim3((unsigned)q.d.tiles), dim3(256), stream, q);
    const int64_t waves = (int64_t)q.d.units_x * q.d.slices_x;
    if (e == hipSuccess && q.d.units_x > 0)
      e = launch_kernel(adapters_back_x_kernel<kChunks>, dim3((unsigned)((waves + kXWaves - 1) / kXWaves)),
                        dim3(kXWaves * kWave), stream, q);
  }
  if (e != hipSuccess) return e;
  const int64_t places = (int64_t)q.p.t.adapters * (q.d.units_n + q.d.units_x) * cols_of(kChunks) * 2 * kChunks * kWave;
  if (places == 0) return hipSuccess;
  const int64_t wgs = (places + 255) / 256, most = 1 << 20;
  return launch_kernel(adapters_back_sums_kernel<kChunks>, dim3((unsigned)(wgs < most ? wgs : most)), dim3(256), stream, q);
}

}  // namespace

size_t adapters_backward_bytes(const AdapterTokens& t, int64_t N, int64_t K, int64_t rank) {
  return (size_t)deal(t, N, K, rank).bytes;
}

hipError_t launch_adapters_backward(const AdapterBackArgs& a, void* workspace, hipStream_t stream) {
  const BackArgs q = {a, deal(a.t, a.N, a.K, a.rank), static_cast<floatx4_t*>(workspace)};
  if (a.rank <= 32) return launch_back<1>(q, stream);
  if (a.rank <= 64) return launch_back<2>(q, stream);
  return launch_back<4>(q, stream);
}

}  // namespace solfp4
