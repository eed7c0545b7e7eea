// Attention of a step's tokens over a cache in pages.
#include "paged_attention.h"
#include "wave_scan.h"

namespace dapq {
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
// instructions a tile begin to count: three waves to a SIMD, two take 63); one item alone takes 0.27 us a tile in bf16, 0.16 in 4 bits, behind 5 to 6 us.
// BLOCKS: blocks of 16 columns; 0: up to 8 columns, whose leading and following parts take the two halves of one block.
// SPLIT: a workgroup has a part of an item; else an item (and nothing is to be joined).
template <int FMT, int BLOCKS, int CAP, bool SPLIT>
__global__ __launch_bounds__(64 * kRowWaves, BLOCKS == 2 ? 2 : 3) void paged_rows_kernel(PagedAttentionParams p) {
  touch_args<sizeof(PagedAttentionParams)>();
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
  // this workgroup's item, and its part of it
  int seq, item, part = 0, parts = 1;
  Sequence s;
  if constexpr (SPLIT) {
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
  const int tile0 = SPLIT ? uniform((int)((int64_t)s.tiles * part / parts)) : 0;
  const int tile1 = SPLIT ? uniform((int)((int64_t)s.tiles * (part + 1) / parts)) : s.tiles;

  {
    const int layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
    const int cols = s.tokens * g;
    // the columns of this lane: query rows as operand, and what they see
    bf16x8 qf[kQueriesInLds ? 1 : NB][4];
    int vis[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      int col = kHalf ? opaque(n) & 7 : 16 * t + opaque(n);
      col = col < cols ? col : cols - 1;
      const int token = quotient(col, p.inv_group), h = head * g + col - token * g;
      vis[t] = rows_seen(p, s.before, token);
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
    const int seen_by_all = rows_seen(p, s.before, 0), seen_by_last = rows_seen(p, s.before, s.tokens - 1);

    // pages of this wave's tiles, 64 tiles at a time, one to a lane
    // as the number of 16 rows that the halves of a tile are (the rows of a pool over 16: below 2^32)
    unsigned half0 = kNoPage, half1 = kNoPage;
    auto load_pages = [&](int k) {
      const int64_t row = ((int64_t)tile0 + wave + (int64_t)kRowWaves * (k + opaque(lane))) * kTile;
      if (SPLIT || k > 0) entries_of((int64_t)seq * p.pool.max_pages, row, &entry0, &entry1);
      auto sixteen = [&](int page, int64_t r) {
        const bool there = row < (int64_t)tile1 * kTile && r >> p.pool.page_shift < p.pool.max_pages && page >= 0 && page < p.pool.n_pages;
        return there ? (unsigned)((page_row(p.pool, layer, page, head) + (r & ((1 << p.pool.page_shift) - 1))) >> 4) : kNoPage;
      };
      half0 = sixteen(entry0, row);
      half1 = sixteen(entry1, row + 16);
    };
    struct Rows {
      unsigned at[2];
      bool ok[2];
    };
    auto rows_of = [&](int k) {
      if ((k & 63) == 0) load_pages(k);
      const unsigned a = __builtin_amdgcn_readlane(half0, k & 63), b = __builtin_amdgcn_readlane(half1, k & 63);
      return Rows{{a, b}, {a != kNoPage, b != kNoPage}};
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
      const bool partial = row0 + kTile > seen_by_all || !now.ok[0] || !now.ok[1];
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
            const bool there = (row0 + 16 * (e >> 2) + 4 * kg + (e & 3) < vis[t]) & now.ok[e >> 2];
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
          const int row = row0 + 16 * (e >> 2) + 4 * kg + (e & 3);
          const bool none = row >= seen_by_last || !now.ok[e >> 2];
          if constexpr (FMT == kFp4) {
            if (none) {
              b.vc[e][0] = 0;
              vscale[e] = 1.0f;
            }
            top = fmaxf(top, row >= seen_by_all ? vscale[e] : 0.0f);
          } else if constexpr (FMT == kE4m3) {
            if (none) {
              b.vc[e][0] = b.vc[e][1] = 0;
              vscale[e] = 1.0f;
            }
            odd |= row >= seen_by_all && (e4m3_past(b.vc[e][0], vscale[e]) | e4m3_past(b.vc[e][1], vscale[e])) != 0;
          } else {
            if (none) b.vt[e] = u32x4{0, 0, 0, 0};
            if (row >= seen_by_all) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const unsigned bad = infinite_bits(b.vt[e][i]);
                odd |= bad != 0;
                b.vt[e][i] &= ~bad;
              }
            }
          }
        }
        if (__any(odd || top > kLargestScale<kFp4>)) {
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
    float* mine_of = p.parts + (int64_t)blockIdx.x * Part<kCols>::kFloats;
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
        const int token = quotient(col, p.inv_group), h = head * g + col - token * g;
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
constexpr int kJoinWaves = 8, kJoinEarly = 4;
template <int COLS, int WAVES>
__global__ __launch_bounds__(64 * kJoinWaves) void paged_join_kernel(PagedAttentionParams p) {
  __shared__ float wave_sums[kJoinWaves][kHeadDim + 2];
  const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : uniform(threadIdx.x >> 6);
  const int seq = (int)divide(blockIdx.x, p.items, p.inv_items), item = blockIdx.x - seq * p.items;
  const int col = WAVES == 1 ? blockIdx.y * kJoinWaves + uniform(threadIdx.x >> 6) : blockIdx.y;
  Tiles t = tiles_of_64(p, 0, lane);
  int64_t total = from_lane(t.upto, 63);
  for (int b0 = 64; b0 < p.batch; b0 += 64) total += from_lane(tiles_of_64(p, b0, lane).upto, 63);
  const int share = share_of(p, total);
  int first = 0;  // the workgroup that has the item's first part
  for (int b0 = 0; b0 < (seq & ~63); b0 += 64) {
    first += (int)from_lane(wave_scan<OpAdd>(parts_of(t.own.tiles, share)), 63) * p.items;
    t = tiles_of_64(p, b0 + 64, lane);
  }
  const Sequence s = from_lane(t.own, seq & 63);
  const uint32_t own = parts_of(t.own.tiles, share);
  const int parts = (int)from_lane(own, seq & 63);
  if (parts <= 1 || col >= s.tokens * p.group) return;
  first += ((int)from_lane(wave_scan<OpAdd>(own), seq & 63) - parts) * p.items + item * parts;
  auto part = [&](int i) { return p.parts + (int64_t)(first + i) * Part<COLS>::kFloats; };
  float m = -INFINITY, sum = 0.0f;
  f32x2 o = {0.0f, 0.0f};
  for (int i0 = wave; i0 < parts; i0 += WAVES * 64) {  // 64 parts of this wave, one to a lane
    const int mine = i0 + WAVES * lane, n = (parts - i0 + WAVES - 1) / WAVES < 64 ? (parts - i0 + WAVES - 1) / WAVES : 64;
    const float r = mine < parts ? part(mine)[COLS * kHeadDim + col] : -INFINITY;
    float w = mine < parts ? part(mine)[COLS * (kHeadDim + 1) + col] : 0.0f;
    f32x2 early[kJoinEarly];  // (their loads need no weights)
#pragma unroll
    for (int i = 0; i < kJoinEarly; ++i) early[i] = *reinterpret_cast<const f32x2*>(part(i0 + WAVES * (i < n ? i : n - 1)) + col * kHeadDim + 2 * lane);
    float top = r;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float moved = fmaxf(m, top);
    if (moved == -INFINITY) continue;
    const float f = __builtin_amdgcn_exp2f(r - moved), before = __builtin_amdgcn_exp2f(m - moved);  // (parts without a row: 0)
    w = f == 0.0f && r == -INFINITY ? 0.0f : w * f;
    for (int d = 32; d > 0; d >>= 1) w += __shfl_xor(w, d, 64);
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
    for (int i = 0; i < kJoinEarly; ++i)
      if (i < n) add(i, early[i]);
#pragma unroll 4
    for (int i = kJoinEarly; i < n; ++i) add(i, *reinterpret_cast<const f32x2*>(part(i0 + WAVES * i) + col * kHeadDim + 2 * lane));
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
  const int token = quotient(col, p.inv_group), h = head * p.group + col - token * p.group;
  bf16x2 result;
  result[0] = (__bf16)(m == -INFINITY ? 0.0f : o[0] / sum);
  result[1] = (__bf16)(m == -INFINITY ? 0.0f : o[1] / sum);
  *reinterpret_cast<bf16x2*>(p.out + (((int64_t)layer * p.total_new + s.first + token) * p.n_q_heads + h) * kHeadDim + 2 * lane) = result;
}

int row_cols(int64_t cols) { return cols <= 8 ? 8 : (cols <= 16 ? 16 : 32); }

// How a call of up to 32 columns is run: a function of the descriptors alone, which the workspace follows.
struct RowPlan {
  bool split;
  int groups, spare;  // workgroups of a split call; those that are left when every item has one
};
RowPlan row_plan(const dapq_pages* p, int cols) {
  const int64_t tiles = ((int64_t)p->max_pages * p->page_rows + kTile - 1) / kTile;  // of an item, at most
  const int64_t items = (int64_t)p->n_layers * p->batch * p->n_kv_heads;
  RowPlan plan;
  // An item takes some 6 us and `tile` for each tile of it, a workgroup's four waves one after the other; parts take `join` more, and what their bytes take
  // of the chip.  Us, parts / items, 8 KV heads, bf16, sequences x rows: 1 x 600 10.6 / 9.7, 1 x 1000 11.9 / 13.6, 1 x 8000 17.2 / 74.3, 4 x 1000 13.0 / 14.2,
  // 8 x 1000 15.0 / 14.4, 8 x 2000 19.4 / 22.7, 16 x 2000 34.0 / 30.0, 16 x 4000 57.5 / 55.5, 24 x 2000 47 / 37; in 4 bits 1 x 1000 11.3 / 9.8, 1 x 2000
  // 11.5 / 15.2, 8 x 1000 12.2 / 10.0, 8 x 2000 13.7 / 15.4, 16 x 2000 16.3 / 15.6, 16 x 4000 21.2 / 26.3, 31 x 2000 20.8 / 16.2.
  const bool fp4 = p->format == DAPQ_PAGES_FP4;
  const double tile = fp4 ? 0.16 : 0.27, bytes = (fp4 ? 4352 : 16384) / 6.5e6, join = fp4 ? 6.5 : 5.5;
  // Lengths are not known here, only the table's width: from 30 us an item on parts also keep a long sequence from outlasting the others (8 KV heads, bf16, 16
  // sequences of 1024..8192 rows 58 / 98, 32 of them 120 / 123; 64 of 1000..4000 122 / 122).
  plan.split = items <= 4096 && ((double)tiles * (tile - bytes * (double)items) > join || (double)tiles * tile > 30.0);
  // At least as many workgroups as the chip holds, and enough to an item that parts come in several lengths (32 columns, 32 sequences of 1024..8192 rows, two to an
  // item 138 us, four 131, six 134; 8 columns, 256 sequences of 4000 rows 709, 734, 751).
  const int64_t resident = cols == 32 ? 512 : 768, wanted = (cols == 32 ? 4 : 2) * items, chip = resident > wanted ? resident : wanted;
  const int64_t groups = (tiles + kRowWaves - 1) / kRowWaves * items;
  plan.groups = (int)(groups < chip ? groups : chip);
  plan.spare = (int)(chip - items);
  return plan;
}

template <int FMT, int BLOCKS, bool SPLIT>
int launch_rows(const dapq_pages* pages, const PagedAttentionParams& p, hipStream_t stream) {
  constexpr int kCols = BLOCKS == 0 ? 8 : 16 * BLOCKS, kBytes = kRowWaves * (BLOCKS == 0 ? 1 : BLOCKS) * 16 * (kHeadDim + 2) * 4 + (BLOCKS == 2 ? 8192 : 0);
  const Cap cap = cap_of(p);
  auto kernel = cap == kNoCap ? paged_rows_kernel<FMT, BLOCKS, kNoCap, SPLIT>
                              : (cap == kSmallCap ? paged_rows_kernel<FMT, BLOCKS, kSmallCap, SPLIT> : paged_rows_kernel<FMT, BLOCKS, kLargeCap, SPLIT>);
  const int rc = set_max_dynamic_lds(reinterpret_cast<const void*>(kernel), kBytes);
  if (rc != DAPQ_OK) return rc;
  const unsigned items = (unsigned)(pages->batch * p.items);  // (below 2^24)
  hipLaunchKernelGGL(kernel, dim3(SPLIT ? (unsigned)p.groups : items), dim3(64 * kRowWaves), kBytes, stream, p);
  DAPQ_HIP_LAUNCH_CHECK("paged_rows_kernel");
  if (SPLIT) {
    const unsigned cols = (unsigned)(p.max_new * p.group);
    if (items < 128) hipLaunchKernelGGL((paged_join_kernel<kCols, kJoinWaves>), dim3(items, cols), dim3(64 * kJoinWaves), 0, stream, p);
    else hipLaunchKernelGGL((paged_join_kernel<kCols, 1>), dim3(items, (cols + kJoinWaves - 1) / kJoinWaves), dim3(64 * kJoinWaves), 0, stream, p);
    DAPQ_HIP_LAUNCH_CHECK("paged_join_kernel");
  }
  return DAPQ_OK;
}
template <int FMT, bool SPLIT>
int launch_rows(const dapq_pages* pages, const PagedAttentionParams& p, int cols, hipStream_t stream) {
  return cols == 8 ? launch_rows<FMT, 0, SPLIT>(pages, p, stream) : (cols == 16 ? launch_rows<FMT, 1, SPLIT>(pages, p, stream) : launch_rows<FMT, 2, SPLIT>(pages, p, stream));
}
int launch_rows(const dapq_pages* pages, PagedAttentionParams p, int cols, hipStream_t stream) {
  const RowPlan plan = row_plan(pages, cols);
  p.groups = plan.groups;
  p.spare = plan.spare;
  p.inv_spare = 1.0f / (float)plan.spare;
  if (pages->format == DAPQ_PAGES_FP4) return plan.split ? launch_rows<kFp4, true>(pages, p, cols, stream) : launch_rows<kFp4, false>(pages, p, cols, stream);
  if (pages->format == DAPQ_PAGES_E4M3) return plan.split ? launch_rows<kE4m3, true>(pages, p, cols, stream) : launch_rows<kE4m3, false>(pages, p, cols, stream);
  return plan.split ? launch_rows<kBf16, true>(pages, p, cols, stream) : launch_rows<kBf16, false>(pages, p, cols, stream);
}

int check_attention(const dapq_pages* pages, const dapq_step* step) {
  int rc = check_pages(pages);
  if (rc == DAPQ_OK) rc = check_step(pages, step);
  if (rc != DAPQ_OK) return rc;
  auto stride_ok = [](int64_t s) { return s >= 0 && s % 8 == 0; };
  DAPQ_REQUIRE(stride_ok(step->q_stride_layer) && stride_ok(step->q_stride_row) && stride_ok(step->q_stride_head) && step->q_stride_row >= kHeadDim,
               DAPQ_ERR_UNSUPPORTED, "q strides of the step must be non-negative multiples of 8 elements (row >= 128)");
  DAPQ_REQUIRE(isfinite(step->scale) && step->scale > 0.0f, DAPQ_ERR_INVALID_ARG, "scale must be finite and > 0");
  DAPQ_REQUIRE(isfinite(step->softcap) && step->softcap >= 0.0f, DAPQ_ERR_INVALID_ARG, "softcap must be finite and >= 0");
  // The factors that the kernels have (scale or softcap in binary units, scale / softcap) are normal numbers: an infinite one times a product of 0 is no number,
  // and one of a few bits rounds every score.
  DAPQ_REQUIRE(step->scale <= 0x1p126f && step->softcap <= 0x1p126f, DAPQ_ERR_UNSUPPORTED, "scale (%g) or softcap (%g) exceeds 2^126", step->scale, step->softcap);
  const double ratio = step->softcap > 0.0f ? (double)step->scale / step->softcap : 1.0;
  DAPQ_REQUIRE(ratio >= 0x1p-110 && ratio <= 0x1p110, DAPQ_ERR_UNSUPPORTED, "scale (%g) / softcap (%g) must be from 2^-110 to 2^110", step->scale, step->softcap);
  DAPQ_REQUIRE(step->n_q_heads <= 65535 && step->total_new * step->n_q_heads < (int64_t)1 << 31, DAPQ_ERR_UNSUPPORTED,
               "n_q_heads (%d) exceeds 65535, or total_new (%lld) query rows of all heads 2^31", step->n_q_heads, (long long)step->total_new);
  return DAPQ_OK;
}

}  // namespace
}  // namespace dapq

using namespace dapq;

extern "C" DAPQ_API size_t dapq_paged_attention_workspace_bytes(const dapq_pages* pages, const dapq_step* step) {
  if (check_attention(pages, step) != DAPQ_OK) return 0;
  const int64_t cols = (int64_t)most_new(pages, step) * (step->n_q_heads / pages->n_kv_heads);
  if (cols > kMostRowCols) return turn_workspace_bytes(pages, step);
  const RowPlan plan = row_plan(pages, row_cols(cols));
  return plan.split ? align_up((size_t)plan.groups * row_cols(cols) * (kHeadDim + 2) * sizeof(float), 256) : 256;
}

extern "C" DAPQ_API int dapq_paged_attention(const dapq_pages* pages, const dapq_step* step, const void* q, void* out, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  const int rc = check_attention(pages, step);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(q != nullptr && out != nullptr, DAPQ_ERR_INVALID_ARG, "q and out must not be NULL");
  DAPQ_REQUIRE(((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) == 0, DAPQ_ERR_UNSUPPORTED,
               "q and out must be 16-byte aligned");
  if (step->total_new == 0 || step->max_new == 0) return DAPQ_OK;
  const size_t need = dapq_paged_attention_workspace_bytes(pages, step);
  DAPQ_REQUIRE(workspace != nullptr, DAPQ_ERR_INVALID_ARG, "workspace is NULL");
  DAPQ_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255) == 0, DAPQ_ERR_UNSUPPORTED, "workspace is not 256-byte aligned");
  DAPQ_REQUIRE(workspace_bytes >= need, DAPQ_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  PagedAttentionParams p;
  p.pool = page_pool(pages);
  p.q = static_cast<const uint16_t*>(q);
  p.out = static_cast<uint16_t*>(out);
  p.cu_new = step->cu_new;
  p.lengths = step->lengths;
  p.q_stride_layer = step->q_stride_layer; p.q_stride_row = step->q_stride_row; p.q_stride_head = step->q_stride_head;
  p.batch = pages->batch;
  p.total_new = (int32_t)step->total_new;
  p.each_new = (int32_t)(step->total_new / pages->batch);
  p.max_new = most_new(pages, step);
  p.n_q_heads = step->n_q_heads;
  p.parts = static_cast<float*>(workspace);
  p.group = step->n_q_heads / pages->n_kv_heads;
  p.items = pages->n_layers * pages->n_kv_heads;
  p.inv_group = 1.0f / (float)p.group;
  p.inv_items = 1.0f / (float)p.items;
  p.cap = step->softcap * kLog2e;
  p.c = step->softcap > 0.0f ? step->scale / step->softcap : step->scale * kLog2e;
  const int64_t cols = (int64_t)p.max_new * p.group;
  if (cols <= kMostRowCols) return launch_rows(pages, p, row_cols(cols), static_cast<hipStream_t>(stream));
  return launch_turn(pages, step, p, static_cast<hipStream_t>(stream));
}
