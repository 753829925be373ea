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
// Bound by memory, dy, x and past once in and dx once out, and by how few waves
// hold it in flight, two workgroups a CU of up to 256 registers: 26574 tokens 2432 ->
// 7296, rank 32 228 to 232 us, 3.4 TB/s (112 to 118 us for dy, 13 for g, 94 to 96 for
// x, 12 for the slices); 8192 tokens 2240 -> 6720 87 to 91 us.  With few tokens by the
// four launches: 1 token 1152 -> 1152 20 us.  At a rank of 128 by g: its shares are as
// many bytes as dy, and every wave of the pass over x reads 48 KB of its pieces a tile
// for 2 KB of x (6600 tokens 2432 -> 7296 241 us).
//
// Both passes multiply by a token's values twice: once with the token's row
// as it lies in memory (g, dx) and once summed over tokens, for which the row's
// columns must be lanes and the tokens the reduction: the tile goes through
// LDS and comes back transposed (ds_read_b64_tr_b16).
//
// FP32 factors (h, g) enter the products as three BF16 pieces, all 24 bits, also
// for dx, which is BF16: past may cancel what the adapters add.
//
// Slices and tiles: slice s of tiles_each tiles leaves its sums of adapter e in
// slot s + e.  Tiles are sorted by adapter, so two slices of one adapter or two
// adapters of one slice never share a slot.
//
// Shares and pieces of g grow with the tokens, at a rank of 128 to more than dy
// (a million tokens 9728 -> 9728 would take 20 GB): past kRunBytes of them the
// tiles are taken in runs, all launches for each, and a run's sums are added to
// the da and db of those before it.
#include "adapters.h"

namespace solfp4 {

namespace {

// Waves of a workgroup of the first pass: two workgroups a CU that wait for each
// other's waves less, but more shares of g through the workspace, four times as
// many values with a rank of 128 (26574 tokens 2432 -> 7296, rank 32: 258 us with 4,
// 280 with 8; 13000 tokens, rank 64 212 and 201; 6600 tokens, rank 128 392 and 302,
// before the later steps).
constexpr int y_waves(int chunks) { return chunks == 1 ? 4 : 8; }
constexpr int kXWaves = 4;       // of the second, whose waves go by themselves

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t* lds_short4_t;

// Blocks of 16 columns of a wave, so that the sums take 64 registers; in the
// second pass, which holds x, past and g's pieces beside them, 32 where rows stay
// whole lines (26574 tokens 2432 -> 7296, rank 32: 229 us with four blocks, 270 with
// eight, whose registers spill).
constexpr int cols_of(int chunks) { return 8 / chunks; }
constexpr int x_cols(int chunks) { return chunks == 1 ? 4 : cols_of(chunks); }

// Most bytes of g's shares and pieces of a run (of one tile, if that has more).
// Rank 128, 2432 -> 7296, 26574 and 50000 tokens: 905 and 1689 us with 256 MiB, 913
// and 1691 in one run of 0.5 and 0.9 GiB, 959 and 1740 with 128 MiB.
constexpr int64_t kRunBytes = (int64_t)256 << 20;

// How a run's work is dealt and where everything lies in the workspace.
struct Deal {
  int64_t tiles;                        // of a run
  int units_n, chunks_n, units_x;       // waves' columns of N and K; workgroups along N
  int slices_n, each_n, slices_x, each_x;
  int64_t slots_n, slots_x;
  int64_t share, rows_g, tokens_g, db, da, bytes;   // offsets of floatx4_t places, bytes at the end
  int64_t share_each, rows_each, tokens_each;       // places of a tile
};

struct BackArgs {
  AdapterBackArgs p;
  Deal d;        // share, rows_g and tokens_g: of the plan's first tile, were it in this run
  floatx4_t* ws;
  int begin, end;   // the run's tiles
};

Deal deal(const AdapterTokens& t, int64_t N, int64_t K, int64_t rank) {
  const int chunks = rank <= 32 ? 1 : rank <= 64 ? 2 : 4, blocks = 2 * chunks;
  const int cols = 16 * cols_of(chunks), x_wide = 16 * x_cols(chunks);
  const int64_t cus = device_cu_count();
  Deal d = {};
  d.units_n = (int)((N + cols - 1) / cols);
  d.units_x = (int)((K + x_wide - 1) / x_wide);
  const int waves = y_waves(chunks);
  d.chunks_n = (d.units_n + waves - 1) / waves;
  const int64_t frag = blocks * kWave;
  d.share_each = 2 * frag, d.rows_each = chunks * 2 * 3 * kWave, d.tokens_each = 3 * frag;
  const int64_t each = (d.chunks_n * d.share_each + d.rows_each + d.tokens_each) * 16;
  const int64_t most = each < kRunBytes ? kRunBytes / each : 1, runs = (t.max_tiles + most - 1) / most;
  d.tiles = runs ? (t.max_tiles + runs - 1) / runs : 0;
  const auto slices = [&](int64_t want, int* each) {
    want = want < 1 ? 1 : want < d.tiles ? want : d.tiles;
    *each = (int)(want > 0 ? (d.tiles + want - 1) / want : 1);
    return (int)((d.tiles + *each - 1) / *each);
  };
  d.slices_n = slices(d.chunks_n ? 8 * cus / (waves * d.chunks_n) : 1, &d.each_n);
  d.slices_x = slices(d.units_x ? 8 * cus / d.units_x : 1, &d.each_x);
  d.slots_n = d.slices_n + t.adapters;
  d.slots_x = d.slices_x + t.adapters;
  int64_t at = 0;
  const auto take = [&](int64_t n) {
    const int64_t was = at;
    at += n;
    return was;
  };
  d.share = take(d.chunks_n * d.tiles * d.share_each);
  d.rows_g = take(d.tiles * d.rows_each);
  d.tokens_g = take(d.tiles * d.tokens_each);
  d.db = take(d.slots_n * d.units_n * cols_of(chunks) * frag);
  d.da = take(d.slots_x * d.units_x * x_cols(chunks) * frag);
  d.bytes = at * 16;
  return d;
}

__device__ __forceinline__ bf16x8_t none8() { return __builtin_bit_cast(bf16x8_t, u32x4_t{0, 0, 0, 0}); }

// Columns as lanes of a matrix in LDS whose rows lie `stride` bytes apart: element j
// of lane (m, g) is row 16 (j / 4) + 4 g + j % 4 of column first + hop (m / 4) + m % 4.
__device__ __forceinline__ bf16x8_t transposed_read(uint8_t* base, int stride, int first, int hop, int lane) {
  const int i = lane % 16, g = lane / 16;
  short4_t v[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_short4_t)(base + (16 * h + 4 * g + i / 4) * stride + (first + i % 4 * hop) * 2));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

// One wave's tile in LDS, [token][column]; rows 32 bytes apart beyond their
// columns, so that the eight rows that half a wave reads lie in different banks.
template <int kCols>
struct TileLds {
  static constexpr int kRow = kCols * 32 + 32;
  uint8_t* base;
  __device__ __forceinline__ void put(int row, int m, const LaneRun<kCols>& v) const {
    *reinterpret_cast<typename LaneRun<kCols>::words_t*>(base + row * kRow + m * kCols * 2) = v.w;
  }
  // Its columns apart: column kCols m + c in the place of column 16 c + m.
  __device__ __forceinline__ void spread(int row, int m, const LaneRun<kCols>& v) const {
#pragma unroll
    for (int c = 0; c < kCols; ++c)
      *reinterpret_cast<uint16_t*>(base + row * kRow + (16 * c + m) * 2) = (uint16_t)(v.w[c / 2] >> (16 * (c & 1)));
  }
  // As it lies: element j of lane (m, g) is column 32 s + 16 (j / 4) + 4 g + j % 4 of row `row`.
  __device__ __forceinline__ bf16x8_t plain(int row, int s, int g) const {
    const uint8_t* at = base + row * kRow + 64 * s + 8 * g;
    const u32x2_t lo = *reinterpret_cast<const u32x2_t*>(at), hi = *reinterpret_cast<const u32x2_t*>(at + 32);
    return __builtin_bit_cast(bf16x8_t, u32x4_t{lo.x, lo.y, hi.x, hi.y});
  }
  // Block c with the columns as lanes.
  __device__ __forceinline__ bf16x8_t transposed(int c, int lane) const {
    return transposed_read(base, kRow, 16 * c, 4, lane);
  }
};

// A tile's tokens, one a lane (twice; the last again past the tile's end), so
// that rows' addresses wait for no load of their own.
struct Tokens {
  int mine;
  __device__ __forceinline__ void load(const AdapterTokens& t, const Tile& tile, int lane) {
    mine = (int)raw_token(t, tile.first + min(lane % kAdapterTile, tile.count - 1));
  }
  // before the first use, and not at once: that waits for the load (26574 tokens 229 -> 241 us)
  __device__ __forceinline__ void bound(const AdapterTokens& t) { mine = (int)bounded_token(t, (uint32_t)mine); }
  __device__ __forceinline__ int64_t row(int i) const { return (uint32_t)__shfl(mine, i, kWave); }
};

// The tiles of a slice, looked up ahead of their use: at work on tile i, the
// tokens of i + 1 are there, those of i + 2 on their way and tile i + 3 is read.
// Loads come back in order, so a look-up that waited would wait for the rows
// before it.
struct Tiles {
  const AdapterTokens& t;
  int end, lane;
  Tile tile, next, later, raw;
  Tokens tokens, tokens_next, tokens_later;
  __device__ __forceinline__ Tile at(int i) const { return i < end ? load_tile(t, i) : Tile{0, 0, 0}; }
  __device__ __forceinline__ Tiles(const AdapterTokens& t, int first, int end, int lane) : t(t), end(end), lane(lane) {
    tile = uniform(t, at(first)), next = uniform(t, at(first + 1)), raw = at(first + 2);
    if (tile.count) tokens.load(t, tile, lane), tokens.bound(t);
    if (next.count) tokens_next.load(t, next, lane);
  }
  __device__ __forceinline__ void look(int i) {   // at work on tile i
    later = uniform(t, raw);
    if (later.count) tokens_later.load(t, later, lane);
    raw = at(i + 3);
  }
  __device__ __forceinline__ void advance() {
    tile = next, tokens = tokens_next;
    if (tile.count) tokens.bound(t);
    next = later, tokens_next = tokens_later;
  }
};

// A tile's rows: 16 lanes read kCols columns each of one row, whole lines where
// the rank lets a wave have 64 columns or more; a lane has rows g + 4 i.
template <int kCols>
struct Rows {
  LaneRun<kCols> v[8];
  // kRaw: settle() is called before the first use.
  template <bool kRaw = false>
  __device__ __forceinline__ void load(const uint16_t* base, int64_t stride, const Tokens& tokens, int col0, int cols,
                                       int m, int g) {
    if (col0 + 16 * kCols <= cols) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i].load(base + tokens.row(g + 4 * i) * stride, col0 + kCols * m, cols, true);
    } else if constexpr (!kRaw) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i].load(base + tokens.row(g + 4 * i) * stride, col0 + kCols * m, cols, false);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i].load_raw(base + tokens.row(g + 4 * i) * stride, col0 + kCols * m, cols);
    }
  }
  // Before the first use, and not at once: that waits for the loads, and all
  // waves for the one with the row's end (8192 tokens 2240 -> 6720, where it has 64
  // of its 128 columns, 109 us, so 87).  In the second pass, whose waves do not
  // wait for each other, rows' ends are moved at once: with this there its rows
  // of whole lines lost 3%.
  __device__ __forceinline__ void settle(int col0, int cols, int m) {
    if (col0 + 16 * kCols <= cols) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i].settle(col0 + kCols * m, cols);
  }
  // to LDS, with zeros in the place of tokens past the tile's end
  __device__ __forceinline__ void put(const TileLds<kCols>& lds, int count, int m, int g) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (count < kAdapterTile && g + 4 * i >= count) v[i].w = typename LaneRun<kCols>::words_t{};
      lds.put(g + 4 * i, m, v[i]);
    }
  }
};

// acc += factor^T tile, the tile's columns as lanes; factor(r, s) is piece s of
// block r.  kHeld: the factors are in registers, and a block of columns is at a time.
template <int kCols, int kBlocks, bool kHeld, typename F>
__device__ __forceinline__ void add_products(floatx4_t (&acc)[kCols][kBlocks], const TileLds<kCols>& lds, int lane,
                                             F factor) {
  if constexpr (kHeld) {
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      const bf16x8_t z = lds.transposed(c, lane);
#pragma unroll
      for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) acc[c][r] = mfma(factor(r, s), z, acc[c][r]);
    }
  } else {
    bf16x8_t z[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) z[c] = lds.transposed(c, lane);
#pragma unroll
    for (int r = 0; r < kBlocks; ++r)
#pragma unroll
      for (int s = 2; s >= 0; --s) {
        const bf16x8_t f = factor(r, s);
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c][r] = mfma(f, z[c], acc[c][r]);
      }
  }
}

// ---- the pass over dy -----------------------------------------------------

template <int kChunks>
__global__ __launch_bounds__(y_waves(kChunks) * kWave, 2) void adapters_back_y_kernel(BackArgs q) {
  constexpr int kWaves = y_waves(kChunks), kBlocks = 2 * kChunks, kCols = cols_of(kChunks);
  constexpr int kHBlocks = (kBlocks + kWaves - 1) / kWaves;   // blocks of h that a wave makes an operand
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
    // b^T through LDS: row 4 g + i of block r is rank element 32 (r / 2) + 8 g + 4 (r % 2) + i.
    // All of the wave's columns, 8 KB, are loaded at once, and pass through LDS in
    // squares of 32 columns and 32 rank elements, as many at a time as fit.
    if (!works) return;
    int rank = p.rank, row = lane / (2 * kBlocks);
    asm volatile("" : "+s"(rank), "+v"(row));   // rows' places made here and not kept over the tiles
    const uint16_t* b = p.b + (int64_t)e * p.N * rank;
    constexpr int kFit = 4 / kChunks, kSquareRow = 72, kSquare = 32 * kSquareRow;
    static_assert(kFit * kSquare <= kAdapterTile * TileLds<kCols>::kRow, "the squares' place");
    const int piece = lane % (2 * kBlocks);
    u32x4_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int n = col0 + row + i * (32 / kBlocks);
      const uint16_t* br = b + (int64_t)min(n, p.N - 1) * rank;
      v[i] = __builtin_bit_cast(u32x4_t, rank == 16 * kBlocks ? operand8(br + 8 * piece) : operand8(br, 8 * piece, rank));
      if (n >= p.N) v[i] = u32x4_t{0, 0, 0, 0};
    }
#pragma unroll
    for (int round = 0; round < 4 / kFit; ++round) {
      wave_order();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = row + i * (32 / kBlocks), square = at / 32 * kChunks + piece / 4;
        if (square / kFit != round) continue;
        u32x2_t* to_ = reinterpret_cast<u32x2_t*>(lds.base + square % kFit * kSquare + at % 32 * kSquareRow + piece % 4 * 16);
        to_[0] = u32x2_t{v[i].x, v[i].y};
        to_[1] = u32x2_t{v[i].z, v[i].w};
      }
      wave_order();
#pragma unroll
      for (int f = 0; f < kFit; ++f)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int square = round * kFit + f;
          bt[square % kChunks * 2 + r][square / kChunks] =
              transposed_read(lds.base + f * kSquare, kSquareRow, 4 * r, 8, lane);
        }
    }
    wave_order();
  };

  const int first = q.begin + slice * q.d.each_n, end = min(first + q.d.each_n, q.end);
  // the next tile's rows and its h come while a tile is worked on
  Tiles tiles_(p.t, first, end, lane);
  Tile& tile = tiles_.tile;
  Tokens& tokens = tiles_.tokens;
  Rows<kCols> dy;
  float hv[kHBlocks][8];
  const auto is_real = [&] { return tile.count && tile.group < p.t.adapters; };   // adapters' tiles come first
  const auto fetch = [&] {
#pragma unroll
    for (int u = 0; u < kHBlocks; ++u) {
      const int r = wave + u * kWaves;
      if (r >= kBlocks) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int t = 16 * (k / 4) + 4 * g + k % 4, at = 16 * r + m;
        const int64_t token = tokens.row(t);
        hv[u][k] = t < tile.count && at < p.rank ? p.hidden[token * p.rank + at] : 0.0f;
      }
    }
    if (works) dy.template load<true>(p.dy, p.dy_stride, tokens, col0, p.N, m, g);
  };
  int i = first;
  while (is_real()) {
    begin(tile.group);
    fetch();
    for (bool more = true; more; ++i) {
      tiles_.look(i);
      if (works) {
        dy.settle(col0, p.N, m);
        dy.put(lds, tile.count, m, g);
      }
      // h as an operand, its tokens in the transposed tile's order
#pragma unroll
      for (int u = 0; u < kHBlocks; ++u) {
        const int r = wave + u * kWaves;
        if (r >= kBlocks) continue;
        bf16x8_t piece[3];
        split_bf16(hv[u], piece);
#pragma unroll
        for (int s = 0; s < 3; ++s) factor[s][r][lane] = piece[s];
      }
      tiles_.advance();
      more = is_real() && tile.group == group;
      if (more) fetch();
      __syncthreads();
      floatx4_t part[2][kBlocks];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) part[j][r] = floatx4_t{0, 0, 0, 0};
      if (works) {
#pragma unroll
        for (int s = 0; s < kCols / 2; ++s)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const bf16x8_t v = lds.plain(m + 16 * j, s, g);
#pragma unroll
            for (int r = 0; r < kBlocks; ++r) part[j][r] = mfma(bt[r][s], v, part[j][r]);
          }
        add_products<kCols, kBlocks, false>(acc, lds, lane, [&](int r, int s) { return factor[s][r][lane]; });
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
}

// ---- g from its shares ----------------------------------------------------

template <int kChunks>
__global__ __launch_bounds__(256) void adapters_back_g_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks, kRow = 16 * kBlocks + 1;
  __shared__ float gs[kAdapterTile][kRow];
  const AdapterBackArgs& p = q.p;
  const int i = q.begin + blockIdx.x;
  const Tile tile = uniform(p.t, load_tile(p.t, i));
  if (tile.count == 0 || tile.group >= p.t.adapters) return;
  const float scale = p.scales ? p.scales[tile.group] : 1.0f;
  const floatx4_t* from = q.ws + q.d.share + (int64_t)i * 2 * kBlocks * kWave;
  const int64_t hop = q.d.tiles * 2 * kBlocks * kWave;
  for (int k = threadIdx.x; k < kBlocks * kWave; k += 256) {
    // eight values of a token, from two blocks
    const int lane = k % kWave, jc = k / kWave, j = jc / kChunks, c = jc % kChunks;
    const int at = (j * kBlocks + 2 * c) * kWave + lane;
    floatx4_t lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    // in order, eight workgroups' loads at a time (one by one each waits for the one before)
    for (int n = 0; n < q.d.chunks_n; n += 8) {
      floatx4_t u[2][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool has = n + i < q.d.chunks_n;
        u[0][i] = has ? from[(n + i) * hop + at] : floatx4_t{0, 0, 0, 0};
        u[1][i] = has ? from[(n + i) * hop + at + kWave] : floatx4_t{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) lo += u[0][i], hi += u[1][i];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      gs[lane % 16 + 16 * j][32 * c + lane / 16 * 8 + e] = scale * (e < 4 ? lo[e % 4] : hi[e % 4]);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < kBlocks * kWave; k += 256) {
    // row 4 g + i of the result is row g + 4 i of the tile, as in the forward pass
    const int lane = k % kWave, m = lane % 16, jc = k / kWave, j = jc / kChunks, c = jc % kChunks;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gs[m % 4 * 4 + m / 4 + 16 * j][32 * c + e / 4 * 16 + lane / 16 * 4 + e % 4];
    bf16x8_t piece[3];
    split_bf16(v, piece);
#pragma unroll
    for (int s = 0; s < 3; ++s)
      q.ws[q.d.rows_g + (((int64_t)i * kChunks + c) * 2 + j) * 3 * kWave + s * kWave + lane] =
          __builtin_bit_cast(floatx4_t, piece[s]);
  }
  for (int k = threadIdx.x; k < kBlocks * kWave; k += 256) {
    const int lane = k % kWave, r = k / kWave, g = lane / 16;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gs[16 * (e / 4) + 4 * g + e % 4][16 * r + lane % 16];
    bf16x8_t piece[3];
    split_bf16(v, piece);
#pragma unroll
    for (int s = 0; s < 3; ++s)
      q.ws[q.d.tokens_g + ((int64_t)i * 3 + s) * kBlocks * kWave + r * kWave + lane] =
          __builtin_bit_cast(floatx4_t, piece[s]);
  }
}

// ---- the pass over x ------------------------------------------------------

template <int kChunks>
__global__ __launch_bounds__(kXWaves * kWave, 2) void adapters_back_x_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks, kCols = x_cols(kChunks);
  constexpr bool kHeld = kChunks == 1;   // g's pieces fit in registers
  // g's pieces for dx half a tile at a time, and above rank 64 both halves late, where
  // more at once would spill (13000 tokens 2432 -> 7296, rank 64: 201 us, 214 with both
  // halves ahead, 205 with both late; 8192 tokens 2240 -> 2240, rank 128: 154 us;
  // of two pieces 151, and 185 with both halves ahead)
  constexpr int kHalves = kChunks == 1 ? 2 : 1;
  constexpr bool kLate = kChunks == 4;
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
    // a^T through LDS: column m of block c is column kCols m + c, so that a lane's
    // results follow each other
    int K = p.K, row = g;
    asm volatile("" : "+s"(K), "+v"(row));   // rows' places made here and not kept over the tiles
    const uint16_t* a = p.a + (int64_t)e * p.rank * K;
#pragma unroll
    for (int h = 0; h < kChunks; ++h) {
      LaneRun<kCols> v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 32 * h + row + 4 * i;
        v[i].load(a + (int64_t)min(r, p.rank - 1) * K, col0 + kCols * m, K, col0 + 16 * kCols <= K);
        if (r >= p.rank) v[i].w = typename LaneRun<kCols>::words_t{};
      }
      wave_order();
#pragma unroll
      for (int i = 0; i < 8; ++i) lds.spread(g + 4 * i, m, v[i]);
      wave_order();
#pragma unroll
      for (int c = 0; c < kCols; ++c) at[c][h] = lds.transposed(c, lane);
      wave_order();
      __builtin_amdgcn_sched_barrier(0);   // one step's loads at a time in registers
    }
  };

  const int first = q.begin + slice * q.d.each_x, end = min(first + q.d.each_x, q.end);
  // x ahead as in the pass over dy; past of the tile itself, needed last
  Tiles tiles_(p.t, first, end, lane);
  Tile& tile = tiles_.tile;
  Tokens& tokens = tiles_.tokens;
  Rows<kCols> x;
  const auto piece3 = [&](int i, int r, int s) {
    return __builtin_bit_cast(bf16x8_t, q.ws[q.d.tokens_g + ((int64_t)i * 3 + s) * kBlocks * kWave + r * kWave + lane]);
  };
  int i = first;
  while (tile.count) {
    begin(tile.group);
    const bool real = group < p.t.adapters;
    if (real) x.load(p.x, p.x_stride, tokens, col0, p.K, m, g);
    for (bool more = true; more; ++i) {
      tiles_.look(i);
      const Tile now = tile;
      const Tokens of_now = tokens;
      // g's operands first, past after them: loads come back in order
      bf16x8_t gd[kHalves][kChunks][3], three[kHeld ? kBlocks : 1][3];
      const auto load_gd = [&](bf16x8_t(&to)[kChunks][3], int j) {
#pragma unroll
        for (int h = 0; h < kChunks; ++h)
#pragma unroll
          for (int s = 0; s < 3; ++s)
            to[h][s] = __builtin_bit_cast(
                bf16x8_t, q.ws[q.d.rows_g + (((int64_t)i * kChunks + h) * 2 + j) * 3 * kWave + s * kWave + lane]);
      };
      if (real) {
#pragma unroll
        for (int r = 0; r < (kHeld ? kBlocks : 0); ++r)
#pragma unroll
          for (int s = 0; s < 3; ++s) three[r][s] = piece3(i, r, s);
#pragma unroll
        for (int j = 0; j < (kLate ? 0 : kHalves); ++j) load_gd(gd[j], j);
        wave_order();
        x.put(lds, now.count, m, g);
        wave_order();
      }
      Rows<kCols> add;
      if (p.past) {
        add.load(p.past, p.past_stride, of_now, col0, p.K, m, g);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) add.v[k].w = typename LaneRun<kCols>::words_t{};
      }
      tiles_.advance();
      more = tile.count && tile.group == group;
      if (more && real) x.load(p.x, p.x_stride, tokens, col0, p.K, m, g);
      if (real) {
        add_products<kCols, kBlocks, kHeld>(acc, lds, lane, [&](int r, int s) {
          if constexpr (kHeld) return three[r][s];
          else return piece3(i, r, s);
        });
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (real) {
          if (kHalves == 1 && (kLate || j)) load_gd(gd[0], j);
          // two columns of a lane's rows at a time
#pragma unroll
          for (int c = 0; c < kCols; c += 2) {
            floatx4_t d[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int h = 0; h < kChunks; ++h)
#pragma unroll
              for (int s = 2; s >= 0; --s)
#pragma unroll
                for (int u = 0; u < 2; ++u) d[u] = mfma(gd[kHalves == 1 ? 0 : j][h][s], at[c + u][h], d[u]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              LaneRun<kCols>& o = add.v[4 * j + k];
              o.w[c / 2] = pack_bf16(o.value(c) + d[0][k], o.value(c + 1) + d[1][k]);
            }
          }
        } else if (now.group > p.t.adapters) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int c = 0; c < kCols / 2; ++c) add.v[4 * j + k].w[c] = 0x7FC07FC0u;   // NaN
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t token = of_now.row(g + 4 * k + 16 * j);
          if (g + 4 * k + 16 * j < now.count)
            add.v[4 * j + k].store(p.dx + token * p.dx_stride, col0 + kCols * m, p.K, col0 + 16 * kCols <= p.K);
        }
      }
    }
    flush();
  }
}

// ---- da and db from the slices' sums --------------------------------------

// One thread a place of four rank elements of a column; db first, then da.
template <int kChunks>
__global__ __launch_bounds__(256) void adapters_back_sums_kernel(BackArgs q) {
  constexpr int kBlocks = 2 * kChunks;
  const AdapterBackArgs& p = q.p;
  const int64_t per_n = (int64_t)q.d.units_n * cols_of(kChunks) * kBlocks * kWave;
  const int64_t per_x = (int64_t)q.d.units_x * x_cols(kChunks) * kBlocks * kWave;
  const int64_t all = p.t.adapters * (per_n + per_x);
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
    const bool is_db = id < p.t.adapters * per_n;
    const int64_t k = is_db ? id : id - p.t.adapters * per_n, per = is_db ? per_n : per_x;
    const int e = (int)(k / per);
    const int64_t place = k - e * per;
    int begin = q.begin, end = q.end;   // the adapter's tiles in this run
    if (p.t.plan) begin = max(p.t.plan[e], begin), end = min(p.t.plan[e + 1], end);
    if (q.begin && begin >= end) continue;
    begin -= q.begin, end -= q.begin;
    floatx4_t v = {0, 0, 0, 0};
    if (begin < end) {
      const int each = is_db ? q.d.each_n : q.d.each_x;
      const floatx4_t* from = q.ws + (is_db ? q.d.db : q.d.da) + place;
      // in order, eight loads at a time
      const int s1 = (end - 1) / each;
      for (int s = begin / each; s <= s1; s += 8) {
        floatx4_t u[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = s + k <= s1 ? from[(s + k + e) * per] : floatx4_t{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) v += u[k];
      }
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
        if (c < left) to[c] = q.begin ? to[c] + scale * v[c] : scale * v[c];
    } else {
      if (col >= p.K) continue;
      float* to = p.da + ((int64_t)e * p.rank + at) * p.K + col;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < left) to[c * (int64_t)p.K] = q.begin ? to[c * (int64_t)p.K] + v[c] : v[c];
    }
  }
}

template <int kChunks>
hipError_t launch_run(const BackArgs& q, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (q.end > q.begin) {
    if (q.d.chunks_n > 0)
      e = launch_kernel(adapters_back_y_kernel<kChunks>, dim3((unsigned)(q.d.chunks_n * q.d.slices_n)),
                        dim3(y_waves(kChunks) * kWave), stream, q);
    if (e == hipSuccess && q.d.units_x > 0)
      e = launch_kernel(adapters_back_g_kernel<kChunks>, dim3((unsigned)(q.end - q.begin)), dim3(256), stream, q);
    const int64_t waves = (int64_t)q.d.units_x * q.d.slices_x;
    if (e == hipSuccess && q.d.units_x > 0)
      e = launch_kernel(adapters_back_x_kernel<kChunks>, dim3((unsigned)((waves + kXWaves - 1) / kXWaves)),
                        dim3(kXWaves * kWave), stream, q);
  }
  if (e != hipSuccess) return e;
  const int64_t columns = (int64_t)q.d.units_n * cols_of(kChunks) + (int64_t)q.d.units_x * x_cols(kChunks);   // 16s
  const int64_t places = q.p.t.adapters * columns * 2 * kChunks * kWave;
  if (places == 0) return hipSuccess;
  const int64_t wgs = (places + 255) / 256, most = 1 << 20;
  return launch_kernel(adapters_back_sums_kernel<kChunks>, dim3((unsigned)(wgs < most ? wgs : most)), dim3(256), stream, q);
}

template <int kChunks>
hipError_t launch_back(BackArgs q, hipStream_t stream) {
  const Deal d = q.d;
  const int64_t tiles = q.p.t.max_tiles;
  int64_t begin = 0;
  do {   // once without a tile, for da and db of 0
    q.begin = (int)begin, q.end = (int)(begin + d.tiles < tiles ? begin + d.tiles : tiles);
    q.d.share = d.share - begin * d.share_each;
    q.d.rows_g = d.rows_g - begin * d.rows_each;
    q.d.tokens_g = d.tokens_g - begin * d.tokens_each;
    const hipError_t e = launch_run<kChunks>(q, stream);
    if (e != hipSuccess) return e;
    begin += d.tiles;
  } while (begin < tiles);
  return hipSuccess;
}

}  // namespace

size_t adapters_backward_bytes(const AdapterTokens& t, int64_t N, int64_t K, int64_t rank) {
  return (size_t)deal(t, N, K, rank).bytes;
}

hipError_t launch_adapters_backward(const AdapterBackArgs& a, void* workspace, hipStream_t stream) {
  const BackArgs q = {a, deal(a.t, a.N, a.K, a.rank), static_cast<floatx4_t*>(workspace), 0, 0};
  if (a.rank <= 32) return launch_back<1>(q, stream);
  if (a.rank <= 64) return launch_back<2>(q, stream);
  return launch_back<4>(q, stream);
}

}  // namespace solfp4
