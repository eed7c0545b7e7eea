// Attention of few query rows of a KV head over a cache in pages: over all rows that its tokens see, or over the rows of chosen blocks.
#pragma once

#include <type_traits>

#include "paged_attention.h"
#include "wave_scan.h"

namespace dapq {

// Over chosen blocks: an item is one KV head of one token, with its query heads, up to kMostRowCols of them, as columns.
struct SparseParams : PagedAttentionParams {
  const int32_t *idx, *count;
  int32_t block_shift, n_select;
  int32_t parts_each;  // workgroups of an item
  int32_t most_tiles;  // of n_select blocks, or of all that there are, if they are fewer
};
template <bool SPARSE>
using RowParams = std::conditional_t<SPARSE, SparseParams, PagedAttentionParams>;

namespace {

constexpr int kTile = 32;     // cache rows that a wave takes at a time
constexpr int kRowWaves = 4;  // of a workgroup
constexpr unsigned kNoPage = 0xffffffffu;

// ---- how the row kernel shares out the rows ---------------------------------------------------------------------------
// An item is one KV head of one sequence and layer, with all columns (new tokens x query heads of the KV head).  Where there are many items a
// workgroup has one each.  Where there are few and long ones, every item is cut into parts of about the same length (`share`), as many as the chip holds
// workgroups in all, so that sequences of any lengths share it evenly; a part has a workgroup, and a second kernel joins an item's parts, in order.
// (Shares of one long axis of all tiles, with workgroups that go on into the next item, are as even, but a second item in a workgroup starts all over:
// 300 rows, 1 sequence 13.5 us, where a share happened to be a divisor of an item 12.1 with 1000.)
struct Sequence {
  int first, tokens;  // its new tokens
  int before;         // rows held before them
  int tiles;          // of an item; 0 if it has no new tokens
};

__device__ __forceinline__ Sequence sequence(const PagedAttentionParams& p, int b) {
  Sequence s;
  s.first = p.cu_new == nullptr ? b * p.each_new : p.cu_new[b];
  s.tokens = p.cu_new == nullptr ? p.each_new : p.cu_new[b + 1] - s.first;
  s.tokens = s.tokens < p.max_new ? s.tokens : p.max_new;
  s.before = p.lengths[b];
  s.tiles = 0;
  if (s.tokens > 0) {
    const int n = rows_seen(p, s.before, s.tokens - 1);
    s.tiles = n > kTile ? (n + kTile - 1) / kTile : 1;  // (an item without rows has its zeros to write)
  }
  return s;
}
// The same in all lanes.
__device__ __forceinline__ Sequence uniform_sequence(const PagedAttentionParams& p, int b) {
  Sequence s = sequence(p, b);
  return {uniform(s.first), uniform(s.tokens), uniform(s.before), uniform(s.tiles)};
}
// The tiles of 64 sequences from number b0 on, one sequence to a lane: its own, and the sum of an item's tiles up to and with it.
struct Tiles {
  Sequence own;
  uint32_t upto;  // (64 x at most 2^25)
};
__device__ __forceinline__ Tiles tiles_of_64(const PagedAttentionParams& p, int b0, int lane) {
  Tiles t;
  t.own = {0, 0, 0, 0};
  if (b0 + lane < p.batch) t.own = sequence(p, b0 + lane);
  t.upto = wave_scan<OpAdd>((uint32_t)t.own.tiles);
  return t;
}
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ Sequence from_lane(const Sequence& s, int lane) {
  return {__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.tokens, lane), __builtin_amdgcn_readlane(s.before, lane),
          __builtin_amdgcn_readlane(s.tiles, lane)};
}
// a / b of values that are the same in all lanes, inv = 1.0f / b.
__device__ __forceinline__ int64_t divide(int64_t a, int b, float inv) {
  return a < kQuotientMax ? __builtin_amdgcn_readfirstlane(quotient((int)a, inv)) : uniform64(a / b);
}
// The length of a part: at least a tile to a wave, and so that the parts of all items, each rounded up, are no more than the chip's workgroups: one more
// to an item than its tiles over the share, and the items have left `spare` of them for that quotient.
__device__ __forceinline__ int share_of(const PagedAttentionParams& p, int64_t tiles) {
  const int64_t share = divide(tiles * p.items + p.spare - 1, p.spare, p.inv_spare);
  return (int)(share < kRowWaves ? kRowWaves : (share < 1 << 30 ? share : 1 << 30));
}
__device__ __forceinline__ uint32_t parts_of(int tiles, int share) { return ((uint32_t)tiles + (uint32_t)share - 1) / (uint32_t)share; }

// A part of an item in the workspace: weighted sums, references and sums of weights of its columns.
template <int COLS>
struct Part {
  static constexpr int kFloats = COLS * (kHeadDim + 2);
};

// One wave per 32 rows at a time, the waves of a workgroup in turn over a part of an item; both products on v_mfma_f32_16x16x32_bf16.
//   logits   D[row][column] = K (A operand, 16 rows x 32 channels) x q (B operand); a lane has four rows of one column.
//   weights  2^(c * logit - ref) in fp32; ref only moves, and the sums are rescaled, where a logit lies more than kHeadroom binades above it.
//   output   D[column][channel] += weights (A) x V (B); a weight enters as two bf16 numbers, the leading 8 bits of its significand and the next 8.
//            What is cut off is less than 2^-15 of a weight and 2^-17 on average, always downwards, while the sum below the fraction has all 24 bits: 2^-9 of half a
//            step of the result.  A third number would be another product for every eight channels where columns exceed 8.
//            V is transposed in registers: a lane loads the same 8 channels of 8 rows.
// Bound by bytes where there are enough items: bf16, 256 sequences of 1000 rows, 8 KV heads 182 us (5.8 TB/s), in 4 bits 55 (5.1 TB/s, where 335 vector
// instructions a tile begin to count: three waves to a SIMD, two take 63); one item alone takes 0.27 us a tile in bf16, 0.17 in 4 bits, behind 5 to 6 us.  In 8 bits 64
// sequences of 4000 rows 94 us (5.8 TB/s), 0.19 us a tile.
// BLOCKS: blocks of 16 columns; 0: up to 8 columns, whose leading and following parts take the two halves of one block.
// SPLIT: a workgroup has a part of an item; else an item (and nothing is to be joined).
// SPARSE: of chosen blocks; their rows, one block after the other, are what tiles are cut from.  64 tokens over 2048 rows each, 8 KV heads: bf16 95 us (5.7 TB/s), in 8 bits 53, in 4 29.
template <int FMT, int BLOCKS, int CAP, bool SPLIT, bool SPARSE>
__global__ __launch_bounds__(64 * kRowWaves, BLOCKS == 2 ? 2 : 3) void paged_rows_kernel(RowParams<SPARSE> p) {
  touch_args<sizeof(RowParams<SPARSE>)>();
  constexpr bool kHalf = BLOCKS == 0;
  constexpr int NB = kHalf ? 1 : BLOCKS, kCols = kHalf ? 8 : 16 * BLOCKS;
  constexpr int kWaveFloats = NB * 16 * (kHeadDim + 2);
  constexpr bool kQueriesInLds = NB == 2;  // (there are no registers for them)
  static_assert(!kQueriesInLds || kRowWaves == 4, "a wave brings in half a block");
  extern __shared__ float lds[];  // [waves]: weighted sums, references, sums of weights; queries
  bf16x8* queries = reinterpret_cast<bf16x8*>(lds + kRowWaves * kWaveFloats);
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* mine = lds + wave * kWaveFloats;
  const int g = p.group;
  // the columns of up to 8: the second half of a block has what the leading parts of the weights leave
  const unsigned rest_mask = n >= 8 ? 0xffff0000u : 0u;
  const float rest_factor = n >= 8 ? 1.0f + 0x1p-22f : 1.0f;

  // the entries of the table that the halves of the tile at `row` have (of the last page, past the table)
  auto entries_of = [&](int64_t table, int64_t row, int* a, int* b) {
    const int64_t last = p.pool.max_pages - 1, e0 = row >> p.pool.page_shift, e1 = (row + 16) >> p.pool.page_shift;
    *a = p.pool.table[table + (e0 < last ? e0 : last)];
    *b = p.pool.table[table + (e1 < last ? e1 : last)];
  };
  int entry0 = -1, entry1 = -1;
  // of chosen blocks: the first rows of the halves of the tile at row `row` of the chosen ones; entries past the count may hold anything
  int row_of0 = -1, row_of1 = -1;
  const int32_t* chosen = nullptr;
  auto blocks_of = [&](int64_t row) {
    if constexpr (SPARSE) {
      auto first_row = [&](int64_t r) {
        const int64_t slot = r >> p.block_shift;
        const int block = chosen[slot < p.n_select ? slot : p.n_select - 1];
        const int64_t in_pool = block < 0 ? -1 : ((int64_t)block << p.block_shift) + (r & ((1 << p.block_shift) - 1));
        return (int)(in_pool < (int64_t)p.pool.max_pages << p.pool.page_shift ? in_pool : -1);
      };
      row_of0 = first_row(row);
      row_of1 = first_row(row + 16);
    }
  };
  auto entries_of_blocks = [&](int64_t table) {
    entry0 = p.pool.table[table + (row_of0 < 0 ? 0 : row_of0 >> p.pool.page_shift)];
    entry1 = p.pool.table[table + (row_of1 < 0 ? 0 : row_of1 >> p.pool.page_shift)];
  };
  // this workgroup's item, and its part of it
  int seq, item, part = 0, parts = 1;
  int begin = 0, end = 0;  // SPARSE: the part's tiles
  Sequence s;
  int seen_of_token = 0, chosen_count = 0;  // SPARSE
  if constexpr (SPARSE) {
    const int at = blockIdx.x / p.pool.n_kv_heads, layer = at / p.total_new, r = at - layer * p.total_new;  // (the same in all lanes)
    chosen = p.idx + (int64_t)blockIdx.x * p.n_select;
    item = layer * p.pool.n_kv_heads + (blockIdx.x - at * p.pool.n_kv_heads);
    part = blockIdx.y;
    parts = p.parts_each;
    const int kept = p.count[blockIdx.x];
    // parts are cut from the most rows that there may be, so that the first blocks are on their way before the count is known; blocks named more than once may be
    // more yet, which the last part has
    begin = uniform(p.most_tiles * part / parts);
    end = uniform(p.most_tiles * (part + 1) / parts);
    blocks_of((begin + wave + (int64_t)kRowWaves * lane) * kTile);
    int t;
    if (!find_token(p.cu_new, p.batch, p.each_new, p.max_new, r, lane, &seq, &t)) return;
    seq = uniform(seq);
    entries_of_blocks((int64_t)seq * p.pool.max_pages);
    const int before = uniform(p.lengths[seq]);
    const int64_t most = (int64_t)p.pool.max_pages << p.pool.page_shift, n = (int64_t)before + t + 1;
    seen_of_token = uniform((int)(n < 0 ? 0 : (n < most ? n : most)));
    chosen_count = uniform(kept < 0 ? 0 : (kept < p.n_select ? kept : p.n_select));
    const int64_t rows = (int64_t)chosen_count << p.block_shift;
    s = {r, 1, before, (int)((rows + kTile - 1) / kTile)};
    end = end < s.tiles && part + 1 < parts ? end : s.tiles;
  } else if constexpr (SPLIT) {
    Tiles t = tiles_of_64(p, 0, lane);
    int64_t total = from_lane(t.upto, 63);
    for (int b0 = 64; b0 < p.batch; b0 += 64) total += from_lane(tiles_of_64(p, b0, lane).upto, 63);
    const int share = share_of(p, total);
    int at = blockIdx.x;  // (from the start of the 64 sequences)
    uint32_t own, upto;
    for (seq = 0;;) {
      own = parts_of(t.own.tiles, share);
      upto = wave_scan<OpAdd>(own);
      const int all = (int)from_lane(upto, 63) * p.items;
      if (at < all) break;
      at -= all;
      seq += 64;
      if (seq >= p.batch) return;
      t = tiles_of_64(p, seq, lane);
    }
    const int l = __builtin_ctzll(__ballot(upto > (uint32_t)uniform_quotient(at, p.items, p.inv_items)));
    seq += l;
    s = from_lane(t.own, l);
    parts = (int)from_lane(own, l);
    at -= ((int)from_lane(upto, l) - parts) * p.items;
    item = uniform_quotient(at, parts, 1.0f / (float)parts);  // layer * Hkv + head
    part = at - item * parts;
  } else {
    seq = (int)divide(blockIdx.x, p.items, p.inv_items);
    item = blockIdx.x - seq * p.items;
    // the first entries of the table are on their way before it is known how many of them count
    entries_of((int64_t)seq * p.pool.max_pages, (wave + (int64_t)kRowWaves * lane) * kTile, &entry0, &entry1);
    s = uniform_sequence(p, seq);
    if (s.tiles == 0) return;
  }
  // (constants of all rows' kernel, and no test there whether a row is negative: with both as variables 3200 rows in 4 bits took 21.4 us for 21.0)
  const int tile0 = SPARSE ? begin : (SPLIT ? uniform((int)((int64_t)s.tiles * part / parts)) : 0);
  const int tile1 = SPARSE ? end : (SPLIT ? uniform((int)((int64_t)s.tiles * (part + 1) / parts)) : s.tiles);

  {
    const int layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
    const int col0 = SPARSE ? blockIdx.z * kCols : 0;  // (of a token's query heads, where they are more than kCols)
    const int cols = SPARSE ? (g - col0 < kCols ? g - col0 : kCols) : s.tokens * g;
    auto token_of = [&](int col) { return SPARSE ? 0 : quotient(col, p.inv_group); };
    auto sees = [&](int token) { return SPARSE ? seen_of_token : rows_seen(p, s.before, token); };
    // the columns of this lane: query rows as operand, and what they see
    bf16x8 qf[kQueriesInLds ? 1 : NB][4];
    int vis[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      int col = kHalf ? opaque(n) & 7 : 16 * t + opaque(n);
      col = col < cols ? col : cols - 1;
      const int token = token_of(col), h = head * g + col0 + col - token * g;
      vis[t] = sees(token);
      const uint16_t* src = p.q + layer * p.q_stride_layer + (int64_t)(s.first + token) * p.q_stride_row + (int64_t)h * p.q_stride_head;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (kQueriesInLds && 2 * t + (i >> 1) != wave) continue;
        const bf16x8 x = *reinterpret_cast<const bf16x8*>(src + (FMT == kBf16 ? 32 * i + 8 * kg : 32 * kg + 8 * i));
        if constexpr (kQueriesInLds) queries[(t * 4 + i) * 64 + lane] = x;
        else qf[t][i] = x;
      }
    }
    if (kQueriesInLds) __syncthreads();
    __builtin_amdgcn_sched_barrier(0);  // (loads of queries behind those of the first tile would be waited for in every step)
    const int seen_by_all = sees(0), seen_by_last = sees(s.tokens - 1);

    int64_t chosen_rows = 0;
    if constexpr (SPARSE) chosen_rows = (int64_t)chosen_count << p.block_shift;
    // pages of this wave's tiles, 64 tiles at a time, one to a lane
    // as the number of 16 rows that the halves of a tile are (the rows of a pool over 16: below 2^32)
    unsigned half0 = kNoPage, half1 = kNoPage;
    auto load_pages = [&](int k) {
      const int64_t row = ((int64_t)tile0 + wave + (int64_t)kRowWaves * (k + opaque(lane))) * kTile;
      if constexpr (SPARSE) {
        if (k > 0) {
          blocks_of(row);
          entries_of_blocks((int64_t)seq * p.pool.max_pages);
        }
        if (row >= chosen_rows) row_of0 = -1;
        if (row + 16 >= chosen_rows) row_of1 = -1;
      } else if (SPLIT || k > 0) {
        entries_of((int64_t)seq * p.pool.max_pages, row, &entry0, &entry1);
      }
      auto sixteen = [&](int page, int64_t r) {
        const bool there = row < (int64_t)tile1 * kTile && (!SPARSE || r >= 0) && r >> p.pool.page_shift < p.pool.max_pages && page >= 0 && page < p.pool.n_pages;
        return there ? (unsigned)((page_row(p.pool, layer, page, head) + (r & ((1 << p.pool.page_shift) - 1))) >> 4) : kNoPage;
      };
      half0 = sixteen(entry0, SPARSE ? row_of0 : row);
      half1 = sixteen(entry1, SPARSE ? row_of1 : row + 16);
    };
    struct Rows {
      unsigned at[2];
      bool ok[2];
      int row[2];  // the halves' first rows
    };
    auto rows_of = [&](int k) {
      if ((k & 63) == 0) load_pages(k);
      const unsigned a = __builtin_amdgcn_readlane(half0, k & 63), b = __builtin_amdgcn_readlane(half1, k & 63);
      Rows r = {{a, b}, {a != kNoPage, b != kNoPage}, {0, 0}};
      if constexpr (SPARSE) {
        r.row[0] = __builtin_amdgcn_readlane(row_of0, k & 63);
        r.row[1] = __builtin_amdgcn_readlane(row_of1, k & 63);
      }
      return r;
    };
    // A tile in registers.  Keys: the operand (bf16), or a row's group of 32 channels to a lane.  Values: 8 channels of the rows
    // 16 * (e / 4) + 4 * kg + e % 4.
    constexpr int kBytes = kCodeBytes<FMT>, kKeyLoads = FMT == kBf16 ? 4 : kBytes / 64;
    struct Buffer {
      u32x4 kf[2][kKeyLoads];
      unsigned ks[2];
      u32x4 vt[FMT == kBf16 ? 8 : 1];
      unsigned vc[8][FMT == kE4m3 ? 2 : 1];
      u32x4 vs[2];
      Rows rows;
    };
    Buffer b;
    // (through descriptors of 16 rows each: the address of a lane is an offset of 32 bits, and what is on no page is not read)
    const unsigned k_at = n * kBytes + kg * (FMT == kBf16 ? 16 : kBytes / 4), v_at = 4 * kg * kBytes + n * (kBytes / 16);
    auto rows16 = [&](uint8_t* pool, const Rows& r, int hf, int bytes) {
      return __builtin_amdgcn_make_buffer_rsrc(pool + (uint64_t)(r.ok[hf] ? r.at[hf] : 0) * (16 * bytes), 0, r.ok[hf] ? 16 * bytes : 0, 0x00020000);
    };
    auto load_k = [&](const Rows& r) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const auto src = rows16(p.pool.k, r, hf, kBytes);
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) b.kf[hf][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (int)k_at + i * (FMT == kBf16 ? 64 : 16), 0, 0));
        if constexpr (FMT != kBf16) b.ks[hf] = __builtin_amdgcn_raw_buffer_load_b8(rows16(p.pool.k_scales, r, hf, 4), n * 4 + kg, 0, 0);
      }
    };
    auto load_v = [&](const Rows& r) {
      b.rows = r;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const auto src = rows16(p.pool.v, r, hf, kBytes);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (FMT == kFp4) {
            b.vc[4 * hf + e][0] = __builtin_amdgcn_raw_buffer_load_b32(src, (int)v_at + e * kBytes, 0, 0);
          } else if constexpr (FMT == kE4m3) {
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(src, (int)v_at + e * kBytes, 0, 0));
            b.vc[4 * hf + e][0] = x[0], b.vc[4 * hf + e][1] = x[1];
          } else b.vt[4 * hf + e] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (int)v_at + e * kRowBytes, 0, 0));
        }
        if constexpr (FMT != kBf16) b.vs[hf] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows16(p.pool.v_scales, r, hf, 4), 16 * kg, 0, 0));
      }
    };

    f32x4 acc[NB][8];
    float ref[NB], sum[NB];
    bool seen[NB];  // (by this lane's rows)
#pragma unroll
    for (int t = 0; t < NB; ++t) {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[t][j] = {0.0f, 0.0f, 0.0f, 0.0f};
      ref[t] = kLowest;
      sum[t] = 0.0f;
      seen[t] = false;
    }

    bool apart = false;  // whether there are such values
    // Tile number k of this wave, and the loads of the next one as the registers of this one are spent: always, or the waits could not count them.
    auto step = [&](int k) {
      const int row0 = (tile0 + wave + kRowWaves * k) * kTile;
      const Rows now = b.rows;
      auto row_at = [&](int e) { return (SPARSE ? now.row[e >> 2] : row0 + 16 * (e >> 2)) + 4 * kg + (e & 3); };
      const bool partial = (SPARSE ? (now.row[0] > now.row[1] ? now.row[0] : now.row[1]) + 16 > seen_by_all : row0 + kTile > seen_by_all) || !now.ok[0] || !now.ok[1];
      float xs[NB][8];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        f32x4 d[NB];
#pragma unroll
        for (int t = 0; t < NB; ++t) d[t] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4 a;
          if constexpr (FMT == kFp4) a = fp4_unpack8(b.kf[hf][0][i], group_scale(b.ks[hf]));
          else if constexpr (FMT == kE4m3) a = e4m3_unpack8(b.kf[hf][i >> 1][2 * (i & 1)], b.kf[hf][i >> 1][2 * (i & 1) + 1], group_scale(b.ks[hf]));
          else a = b.kf[hf][i];
#pragma unroll
          for (int t = 0; t < NB; ++t)
            d[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), kQueriesInLds ? queries[(t * 4 + i) * 64 + lane] : qf[kQueriesInLds ? 0 : t][i], d[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) xs[t][4 * hf + v] = capped<CAP>(p, d[t][v]);
      }
      const Rows next = rows_of(k + 1);
      load_k(next);
      __builtin_amdgcn_sched_barrier(0);
      u32x4 hi[NB], lo[NB];  // the weights as A operand
#pragma unroll
      for (int t = 0; t < NB; ++t) {
        float(&x)[8] = xs[t];
        if (partial) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool there = (row_at(e) < vis[t]) & now.ok[e >> 2];
            seen[t] |= there;
            if (!there) x[e] = -INFINITY;
          }
        } else {
          seen[t] = true;
        }
        float m = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) m = fmaxf(m, x[e]);
        if (CAP == kNoCap) m *= p.c;
        if (__any(m > ref[t] + kHeadroom)) {
          m = fmaxf(m, __shfl_xor(m, 16, 64));
          m = fmaxf(m, __shfl_xor(m, 32, 64));
          const float moved = fmaxf(ref[t], m);
          const float f = __builtin_amdgcn_exp2f(ref[t] - moved);
          ref[t] = moved;
          sum[t] *= f;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float fv = __shfl(f, 4 * kg + v, 64);  // (row 4 * kg + v of the sums is column 4 * kg + v)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[t][j][v] *= fv;
          }
        }
        unsigned w[8], w2[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = __builtin_amdgcn_exp2f(CAP != kNoCap ? x[e] - ref[t] : fmaf(x[e], p.c, -ref[t]));
          sum[t] += y;
          // what the leading part leaves, and 2^-22 of the weight, which keeps it from 0 where a value is infinite
          const float rest = fmaf(y, kHalf ? rest_factor : 1.0f + 0x1p-22f, -__uint_as_float(__float_as_uint(y) & (kHalf ? rest_mask : 0xffff0000u)));
          w[e] = __float_as_uint(kHalf ? rest : y);
          w2[e] = __float_as_uint(rest);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          hi[t][e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302u);
          lo[t][e] = __builtin_amdgcn_perm(w2[2 * e + 1], w2[2 * e], 0x07060302u);
        }
      }
      float vscale[8];  // codes: of the rows, for this lane's channels
#pragma unroll
      for (int e = 0; e < 8; ++e) vscale[e] = FMT != kBf16 ? group_scale((b.vs[e >> 2][e & 3] >> (8 * (n >> 2))) & 255u) : 0.0f;
      if (partial) {
        // Rows that no column sees may hold anything, and 0 times it must be 0.  A value that is infinite or no number, in a row that some columns
        // see and others don't, is added to the former by itself, in LDS.
        bool odd = false;
        float top = 0.0f;  // FP4: the largest scale of such rows
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int row = row_at(e);
          const bool none = row >= seen_by_last || !now.ok[e >> 2];
          if constexpr (FMT == kFp4) {
            if (none) {
              b.vc[e][0] = 0;
              vscale[e] = 1.0f;
            }
            if (!SPARSE) top = fmaxf(top, row >= seen_by_all ? vscale[e] : 0.0f);
          } else if constexpr (FMT == kE4m3) {
            if (none) {
              b.vc[e][0] = b.vc[e][1] = 0;
              vscale[e] = 1.0f;
            }
            if (!SPARSE) odd |= row >= seen_by_all && (e4m3_past(b.vc[e][0], vscale[e]) | e4m3_past(b.vc[e][1], vscale[e])) != 0;
          } else {
            if (none) b.vt[e] = u32x4{0, 0, 0, 0};
            if (!SPARSE && row >= seen_by_all) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const unsigned bad = infinite_bits(b.vt[e][i]);
                odd |= bad != 0;
                b.vt[e][i] &= ~bad;
              }
            }
          }
        }
        if (!SPARSE && __any(odd || top > kLargestFp4Scale)) {
          if constexpr (FMT != kBf16) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (row0 + 16 * (e >> 2) + 4 * kg + (e & 3) < seen_by_all) continue;
              if constexpr (FMT == kFp4) b.vc[e][0] = fp4_finite8(b.vc[e][0], vscale[e]);
              else b.vc[e][0] = e4m3_finite4(b.vc[e][0], vscale[e]), b.vc[e][1] = e4m3_finite4(b.vc[e][1], vscale[e]);
              if (vscale[e] > 0x1p127f) vscale[e] = 1.0f;  // (0 without a scale is no number)
            }
          }
          if (!apart) {
            for (int i = lane; i < kCols * kHeadDim; i += 64) mine[i] = 0.0f;
            apart = true;
          }
#pragma unroll 1
          for (int row = row0 > seen_by_all ? row0 : seen_by_all; row < row0 + kTile && row < seen_by_last; ++row) {  // once more, two channels to a lane
            const int i = row - row0;
            if (!(i < 16 ? now.ok[0] : now.ok[1])) continue;
            const int64_t at = (int64_t)(i < 16 ? now.at[0] : now.at[1]) * 16 + (i & 15);
            unsigned u;
            if constexpr (FMT == kFp4) u = fp4_unpack2((unsigned)p.pool.v[at * kBytes + lane], group_scale(p.pool.v_scales[at * 4 + (lane >> 4)]), 0);
            else if constexpr (FMT == kE4m3)
              u = e4m3_unpack2(*reinterpret_cast<const uint16_t*>(p.pool.v + at * kBytes + 2 * lane), group_scale(p.pool.v_scales[at * 4 + (lane >> 4)]), 0);
            else u = *reinterpret_cast<const unsigned*>(p.pool.v + at * kRowBytes + lane * 4);
            u &= infinite_bits(u);
            if (!__any(u != 0)) continue;
#pragma unroll 1
            for (int col = 0; col < cols; ++col) {
              if (row >= rows_seen(p, s.before, quotient(col, p.inv_group))) continue;
              mine[col * kHeadDim + 2 * lane] += __uint_as_float(u << 16);
              mine[col * kHeadDim + 2 * lane + 1] += __uint_as_float(u & 0xffff0000u);
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // channels 8 * n + 2 * i and the one behind it
        unsigned x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (FMT == kFp4) x[e] = fp4_unpack2(b.vc[e][0], vscale[e], i);
          else if constexpr (FMT == kE4m3) x[e] = e4m3_unpack2(b.vc[e][i >> 1], vscale[e], i & 1);
          else x[e] = b.vt[e][i];
        }
#pragma unroll
        for (int j = 2 * i; j < 2 * i + 2; ++j) {
          u32x4 vb;
#pragma unroll
          for (int e = 0; e < 4; ++e) vb[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int t = 0; t < NB; ++t) {
            acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi[t]), __builtin_bit_cast(bf16x8, vb), acc[t][j], 0, 0, 0);
            if constexpr (!kHalf)
              acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo[t]), __builtin_bit_cast(bf16x8, vb), acc[t][j], 0, 0, 0);
          }
        }
      }
      load_v(next);
      __builtin_amdgcn_sched_barrier(0);
    };
    if (tile0 + wave < tile1) {
      const int tiles = (tile1 - tile0 - wave + kRowWaves - 1) / kRowWaves;
      const Rows first = rows_of(0);
      load_k(first);
      load_v(first);
      __builtin_amdgcn_sched_barrier(0);
      for (int k = 0; k < tiles; ++k) step(k);
    }

    // what the waves have, in LDS
    if (apart) {
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[t][j][v] += mine[(kHalf ? (4 * kg + v) & 7 : 16 * t + 4 * kg + v) * kHeadDim + 8 * n + j];
    }
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      float w = sum[t];
      w += __shfl_xor(w, 16, 64);
      w += __shfl_xor(w, 32, 64);
      const uint64_t any = __ballot(seen[t]);
      const bool column = (any >> n | any >> (n + 16) | any >> (n + 32) | any >> (n + 48)) & 1;
      const int n8 = opaque(8 * n);
      if (kg == 0) {
        mine[NB * 16 * kHeadDim + 16 * t + n] = column ? ref[t] : -INFINITY;  // (no row was seen)
        mine[NB * 16 * (kHeadDim + 1) + 16 * t + n] = w;
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        f32x4* dst = reinterpret_cast<f32x4*>(mine + (16 * t + 4 * kg + v) * kHeadDim + n8);
        dst[0] = f32x4{acc[t][0][v], acc[t][1][v], acc[t][2][v], acc[t][3][v]};
        dst[1] = f32x4{acc[t][4][v], acc[t][5][v], acc[t][6][v], acc[t][7][v]};
      }
    }
    __syncthreads();
    const bool whole = !SPLIT || parts == 1;
    const int64_t own_part = SPARSE ? ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * parts + part : blockIdx.x;
    float* mine_of = p.parts + own_part * Part<kCols>::kFloats;
    for (int e = opaque(tid); e < cols * (kHeadDim / 2); e += 64 * kRowWaves) {
      const int col = e / (kHeadDim / 2), c = 2 * (e % (kHeadDim / 2));
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) m = fmaxf(m, lds[w * kWaveFloats + NB * 16 * kHeadDim + col]);
      f32x2 o = {0.0f, 0.0f};
      float total = 0.0f;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) {  // (in order)
        const float* from_wave = lds + w * kWaveFloats;
        const float r = from_wave[NB * 16 * kHeadDim + col];
        const float f = r == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r - m);
        f32x2 x = *reinterpret_cast<const f32x2*>(from_wave + col * kHeadDim + c);
        if constexpr (kHalf) x += *reinterpret_cast<const f32x2*>(from_wave + (col + 8) * kHeadDim + c);
        if (r != -INFINITY) {
          o[0] = fmaf(f, x[0], o[0]);
          o[1] = fmaf(f, x[1], o[1]);
          total = fmaf(f, from_wave[NB * 16 * (kHeadDim + 1) + col], total);
        }
      }
      if (whole) {
        const int token = token_of(col), h = head * g + col0 + col - token * g;
        bf16x2 result;
        result[0] = (__bf16)(m == -INFINITY ? 0.0f : o[0] / total);
        result[1] = (__bf16)(m == -INFINITY ? 0.0f : o[1] / total);
        *reinterpret_cast<bf16x2*>(p.out + (((int64_t)layer * p.total_new + s.first + token) * p.n_q_heads + h) * kHeadDim + c) = result;
      } else {
        *reinterpret_cast<f32x2*>(mine_of + col * kHeadDim + c) = o;
        if (c == 0) {
          mine_of[kCols * kHeadDim + col] = m;
          mine_of[kCols * (kHeadDim + 1) + col] = total;
        }
      }
    }
  }
}

// The items that several workgroups share.  WAVES: a column has all waves of a workgroup, which take its parts in turn and meet in LDS (few items, many
// parts), or one (32 sequences, 32 columns, 2 parts each: the whole call 150 -> 138 us).
// EARLY: parts whose sums are asked for before their weights are known.
constexpr int kJoinWaves = 8, kJoinEarly = 4;
template <int COLS, int WAVES, bool SPARSE, int EARLY = kJoinEarly>
__global__ __launch_bounds__(64 * kJoinWaves) void paged_join_kernel(RowParams<SPARSE> p) {
  __shared__ float wave_sums[kJoinWaves][kHeadDim + 2];
  const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : uniform(threadIdx.x >> 6);
  const int col = WAVES == 1 ? blockIdx.y * kJoinWaves + uniform(threadIdx.x >> 6) : blockIdx.y;
  int64_t first = 0;  // the workgroup that has the item's first part
  int parts, item, col0 = 0;
  Sequence s;
  if constexpr (SPARSE) {
    const int at = blockIdx.x / p.pool.n_kv_heads, layer = at / p.total_new, r = at - layer * p.total_new;
    int seq, t;
    if (!find_token(p.cu_new, p.batch, p.each_new, p.max_new, r, lane, &seq, &t)) return;
    item = layer * p.pool.n_kv_heads + (blockIdx.x - at * p.pool.n_kv_heads);
    col0 = blockIdx.z * COLS;
    if (col >= COLS || col0 + col >= p.group) return;
    parts = p.parts_each;
    first = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * parts;
    s = {r, 1, 0, 0};
  } else {
    const int seq = (int)divide(blockIdx.x, p.items, p.inv_items);
    item = blockIdx.x - seq * p.items;
    Tiles t = tiles_of_64(p, 0, lane);
    int64_t total = from_lane(t.upto, 63);
    for (int b0 = 64; b0 < p.batch; b0 += 64) total += from_lane(tiles_of_64(p, b0, lane).upto, 63);
    const int share = share_of(p, total);
    for (int b0 = 0; b0 < (seq & ~63); b0 += 64) {
      first += (int)from_lane(wave_scan<OpAdd>(parts_of(t.own.tiles, share)), 63) * p.items;
      t = tiles_of_64(p, b0 + 64, lane);
    }
    s = from_lane(t.own, seq & 63);
    const uint32_t own = parts_of(t.own.tiles, share);
    parts = (int)from_lane(own, seq & 63);
    if (parts <= 1 || col >= s.tokens * p.group) return;
    first += ((int)from_lane(wave_scan<OpAdd>(own), seq & 63) - parts) * p.items + item * parts;
  }
  constexpr bool kFew = EARLY >= 16;  // (no more parts than the lanes of a row, which meet without the LDS crossbar)
  auto first16 = [](float x, auto op) {
    x = op(x, __uint_as_float(dpp<kRor1>(__float_as_uint(x))));
    x = op(x, __uint_as_float(dpp<kRor2>(__float_as_uint(x))));
    x = op(x, __uint_as_float(dpp<kRor4>(__float_as_uint(x))));
    x = op(x, __uint_as_float(dpp<kRor8>(__float_as_uint(x))));
    return __uint_as_float((unsigned)uniform((int)__float_as_uint(x)));
  };
  auto part = [&](int i) { return p.parts + (int64_t)(first + i) * Part<COLS>::kFloats; };
  float m = -INFINITY, sum = 0.0f;
  f32x2 o = {0.0f, 0.0f};
  for (int i0 = wave; i0 < parts; i0 += WAVES * 64) {  // 64 parts of this wave, one to a lane
    const int mine = i0 + WAVES * lane, n = (parts - i0 + WAVES - 1) / WAVES < 64 ? (parts - i0 + WAVES - 1) / WAVES : 64;
    const float r = mine < parts ? part(mine)[COLS * kHeadDim + col] : -INFINITY;
    float w = mine < parts ? part(mine)[COLS * (kHeadDim + 1) + col] : 0.0f;
    f32x2 early[EARLY];  // (their loads need no weights)
#pragma unroll
    for (int i = 0; i < EARLY; ++i) early[i] = *reinterpret_cast<const f32x2*>(part(i0 + WAVES * (i < n ? i : n - 1)) + col * kHeadDim + 2 * lane);
    float top = r;
    if constexpr (kFew) top = first16(top, [](float a, float b) { return fmaxf(a, b); });
    else for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float moved = fmaxf(m, top);
    if (moved == -INFINITY) continue;
    const float f = __builtin_amdgcn_exp2f(r - moved), before = __builtin_amdgcn_exp2f(m - moved);  // (parts without a row: 0)
    w = f == 0.0f && r == -INFINITY ? 0.0f : w * f;
    if constexpr (kFew) w = first16(w, [](float a, float b) { return a + b; });
    else for (int d = 32; d > 0; d >>= 1) w += __shfl_xor(w, d, 64);
    sum = m == -INFINITY ? w : fmaf(sum, before, w);
    if (m != -INFINITY) o *= before;
    m = moved;
    auto add = [&](int i, f32x2 x) {
      const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i));
      if (__builtin_amdgcn_readlane(__float_as_uint(r), i) == 0xff800000u) return;
      o[0] = fmaf(fi, x[0], o[0]);
      o[1] = fmaf(fi, x[1], o[1]);
    };
#pragma unroll
    for (int i = 0; i < EARLY; ++i)
      if (i < n) add(i, early[i]);
#pragma unroll 4
    for (int i = EARLY; i < n; ++i) add(i, *reinterpret_cast<const f32x2*>(part(i0 + WAVES * i) + col * kHeadDim + 2 * lane));
  }
  if constexpr (WAVES > 1) {
    *reinterpret_cast<f32x2*>(&wave_sums[wave][2 * lane]) = o;
    if (lane == 0) {
      wave_sums[wave][kHeadDim] = m;
      wave_sums[wave][kHeadDim + 1] = sum;
    }
    __syncthreads();
    if (wave != 0) return;
    const int waves = parts < WAVES ? parts : WAVES;
    m = -INFINITY;
    for (int w = 0; w < waves; ++w) m = fmaxf(m, wave_sums[w][kHeadDim]);
    o = f32x2{0.0f, 0.0f};
    sum = 0.0f;
    for (int w = 0; w < waves; ++w) {  // (in order)
      if (wave_sums[w][kHeadDim] == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f(wave_sums[w][kHeadDim] - m);
      o[0] = fmaf(f, wave_sums[w][2 * lane], o[0]);
      o[1] = fmaf(f, wave_sums[w][2 * lane + 1], o[1]);
      sum = fmaf(f, wave_sums[w][kHeadDim + 1], sum);
    }
  }
  const int layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
  const int token = SPARSE ? 0 : quotient(col, p.inv_group), h = head * p.group + col0 + col - token * p.group;
  bf16x2 result;
  result[0] = (__bf16)(m == -INFINITY ? 0.0f : o[0] / sum);
  result[1] = (__bf16)(m == -INFINITY ? 0.0f : o[1] / sum);
  *reinterpret_cast<bf16x2*>(p.out + (((int64_t)layer * p.total_new + s.first + token) * p.n_q_heads + h) * kHeadDim + 2 * lane) = result;
}

int row_cols(int64_t cols) { return cols <= 8 ? 8 : (cols <= 16 ? 16 : 32); }
template <int BLOCKS>
constexpr int kRowLds = kRowWaves * (BLOCKS == 0 ? 1 : BLOCKS) * 16 * (kHeadDim + 2) * 4 + (BLOCKS == 2 ? 8192 : 0);

}  // namespace
}  // namespace dapq
