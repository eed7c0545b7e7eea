// Attention of many tokens over a cache in pages: a conversation's next turn behind what the eviction kept of the earlier ones.
#include "paged_attention.h"
#include "wave_scan.h"

namespace dapq {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kTurnTile = 64;   // cache rows of a tile
constexpr int kTurnWaves = 4;
constexpr int kTurnTileBytes = kTurnTile * kRowBytes;  // of K or V in LDS, as bf16
constexpr int kTurnCols = 32 * kTurnWaves;   // of a workgroup
constexpr int kTurnRows = kTurnTile / kTurnWaves;  // that a wave brings in: 16, which are on one page

struct TurnParams : PagedAttentionParams {
  int32_t blocks, splits;  // blocks of columns of all sequences, at most; parts of the rows
};

// Where 16 bytes of a row of a tile lie in LDS: the chunks of a row are permuted by its number, so that 16 rows' same chunks, and
// four rows' same four chunks, fall on all banks.
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * kRowBytes + ((chunk ^ ((row & 3) << 2 | (row >> 2 & 3))) << 4); }

__device__ __forceinline__ int tokens_of(const TurnParams& p, int b) {
  const int n = p.cu_new == nullptr ? p.each_new : p.cu_new[b + 1] - p.cu_new[b];
  return n < p.max_new ? (n > 0 ? n : 0) : p.max_new;
}
// The sequence that a block of columns belongs to (-1: none), and its number there.
__device__ __forceinline__ int find_block(const TurnParams& p, int lane, int* block) {
  if (p.cu_new == nullptr) {
    const int each = (tokens_of(p, 0) * p.group + kTurnCols - 1) / kTurnCols, seq = uniform(*block / each);
    *block -= seq * each;
    return seq < p.batch ? seq : -1;
  }
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    const uint32_t n = b0 + lane < p.batch ? (uint32_t)((tokens_of(p, b0 + lane) * p.group + kTurnCols - 1) / kTurnCols) : 0;
    const uint32_t upto = wave_scan<OpAdd>(n);
    const uint64_t past = __ballot(upto > (uint32_t)*block);
    if (past != 0) {
      const int l = __builtin_ctzll(past);
      *block -= __builtin_amdgcn_readlane((int)(upto - n), l);
      return b0 + l;
    }
    *block -= __builtin_amdgcn_readlane((int)upto, 63);
  }
  return -1;
}

// A workgroup has a block of columns (new tokens x query heads of one KV head, token by token), 32 to a wave, and all rows that they see
// or one of `splits` parts of them.  Tiles of 64 rows pass through LDS as bf16, in two buffers; while a tile is used the next one is on its way to
// registers.  Both products run on v_mfma_f32_32x32x16_bf16:
//   logits   D[row][column] = K (A operand) x q (B operand): a lane has 16 rows of one column, lane and lane ^ 32 the 32 rows of a column
//   output   D[channel][column] += V (A, transposed by the reads from LDS) x weights (B): the lane's weights are the operand as they are, since the
//            order of the rows is free, and a column's factors are the lane's own
// Bound by the two kinds of arithmetic, which two waves to a SIMD overlap in part (matrix instructions 38 % of a SIMD's time, vector ones 45 %), at the
// 2.0 of 2.4 GHz that the card's power leaves: eight turns of 200..2500 tokens behind 983 rows 390 us (777 TFLOP/s), in 4 bits 390, in 8 401; 100 tokens of 8 query
// heads a KV head behind 100000 rows 415 (790).  64 columns to a wave, one wave to a SIMD: 560; eight waves to a workgroup: 438; one half's weights among
// the other half's products: 396..404.
// Weights enter as one bf16, rounded to nearest: an error of 2^-9 of a weight, independent from row to row, below the rounding of the result where
// more than a few rows count; a second part would take half as many matrix instructions again.
template <int FMT, int CAP, bool SPLIT>
__global__ __launch_bounds__(64 * kTurnWaves, 8 / kTurnWaves) void paged_turn_kernel(TurnParams p) {
  extern __shared__ char lds[];  // K of two tiles, V of two tiles; flags of four tiles
  // of a tile: 1 for values that are not finite, 2 << i for rows 16 * i .. on no page.  Tile t's are written in step t - 1, read in step t and cleared
  // in step t + 2, with a barrier at the end of every step.
  int* flags = reinterpret_cast<int*>(lds + 4 * kTurnTileBytes);
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int g = p.group;
  int block = uniform((int)(blockIdx.x / (unsigned)p.items));
  const int item = blockIdx.x - block * p.items, layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
  const int seq = uniform(find_block(p, lane, &block));
  if (seq < 0) return;
  block = uniform(block);
  const int tokens = uniform(tokens_of(p, seq)), before = uniform(p.lengths[seq]);
  const int first_row = uniform(p.cu_new == nullptr ? seq * p.each_new : p.cu_new[seq]);  // of q and out
  const int cols = tokens * g;
  block = (cols + kTurnCols - 1) / kTurnCols - 1 - block;  // (the longest first)
  const int col0 = block * kTurnCols, col_end = cols - col0 < kTurnCols ? cols : col0 + kTurnCols;
  const int token0 = uniform(col0 / g), rest0 = col0 - token0 * g;
  const int seen_by_all = uniform(rows_seen(p, before, token0)), seen_by_last = uniform(rows_seen(p, before, (col_end - 1) / g));
  const int tiles = seen_by_last > 0 ? (seen_by_last + kTurnTile - 1) / kTurnTile : 0;
  const int tile0 = SPLIT ? uniform((int)((int64_t)tiles * blockIdx.y / p.splits)) : 0;
  const int tile1 = SPLIT ? uniform((int)((int64_t)tiles * (blockIdx.y + 1) / p.splits)) : tiles;

  const bool active = col0 + wave * 32 < col_end;  // (a wave without columns only brings in)
  // this lane's columns
  bf16x8 q[8];
  int vis;
  {
    int col = wave * 32 + l32;
    col = col0 + col < col_end ? col : col_end - 1 - col0;
    const int step = quotient(rest0 + col, p.inv_group), h = head * g + rest0 + col - step * g;
    vis = rows_seen(p, before, token0 + step);
    const uint16_t* src = p.q + layer * p.q_stride_layer + (int64_t)(first_row + token0 + step) * p.q_stride_row + (int64_t)h * p.q_stride_head;
#pragma unroll
    for (int c = 0; c < 8; ++c) q[c] = *reinterpret_cast<const bf16x8*>(src + 16 * c + 8 * half);
  }

  // (There before the loop: the waits in it would count them, and with them the rows that are on their way.)
#pragma unroll
  for (int c = 0; c < 8; ++c) asm volatile("" : "+v"(q[c]));

  // Bringing in: this wave's rows of a tile, in registers, then in LDS.
  const int32_t* table = p.pool.table + (int64_t)seq * p.pool.max_pages;
  constexpr int kBytes = kCodeBytes<FMT>, kLoads = kTurnRows * kBytes / 1024;
  u32x4 kr[kLoads], vr[kLoads];  // bf16: load j has row 4 * j + lane / 16; codes: a lane has a group of row lane / 4
  unsigned ks = 0, vs = 0;
  int loaded_row = 0;  // the first of the rows in the registers
  bool loaded_page = false;
  // A tile's entry of the table is read one tile ahead of its rows and looked at with them, since a wait for it is one for every load before it.
  auto entry_of = [&](int tile) { return ((int64_t)tile * kTurnTile + kTurnRows * wave) >> p.pool.page_shift; };
  auto page_of = [&](int tile) {
    const int64_t e = entry_of(tile);
    return table[e < p.pool.max_pages ? e : p.pool.max_pages - 1];
  };
  auto load_rows = [&](int tile, int page) {
    page = uniform(page);
    page = tile < tile1 && entry_of(tile) < p.pool.max_pages && page < p.pool.n_pages ? page : -1;
    loaded_row = tile * kTurnTile + kTurnRows * wave;
    loaded_page = page >= 0;
    int rows = seen_by_last - loaded_row;
    rows = uniform(page < 0 || rows < 0 ? 0 : (rows < kTurnRows ? rows : kTurnRows));
    const int64_t at = uniform64(page_row(p.pool, layer, page < 0 ? 0 : page, head) + (loaded_row & ((1 << p.pool.page_shift) - 1)));
    const auto ksrc = __builtin_amdgcn_make_buffer_rsrc(p.pool.k + at * kBytes, 0, rows * kBytes, 0x00020000);  // (past the rows: zeros)
    const auto vsrc = __builtin_amdgcn_make_buffer_rsrc(p.pool.v + at * kBytes, 0, rows * kBytes, 0x00020000);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int at_lane = FMT == kBf16 ? lane * 16 + j * 1024 : lane * (kBytes / 4) + j * 16;
      kr[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ksrc, at_lane, 0, 0));
      vr[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vsrc, at_lane, 0, 0));
    }
    if constexpr (FMT != kBf16) {
      ks = __builtin_amdgcn_raw_buffer_load_b8(__builtin_amdgcn_make_buffer_rsrc(p.pool.k_scales + at * 4, 0, rows * 4, 0x00020000), lane, 0, 0);
      vs = __builtin_amdgcn_raw_buffer_load_b8(__builtin_amdgcn_make_buffer_rsrc(p.pool.v_scales + at * 4, 0, rows * 4, 0x00020000), lane, 0, 0);
    }
  };
  auto store_rows = [&](int buffer, int tile) {
    char* kt = lds + buffer * kTurnTileBytes;
    char* vt = kt + 2 * kTurnTileBytes;
    bool odd = false;  // a value that is not finite in a row that some columns see and others don't: 0 times it would not be 0
    if constexpr (FMT != kBf16) {
      const int row = kTurnRows * wave + (lane >> 2);
      float scale = group_scale(vs);
      bool past = loaded_row + (lane >> 2) >= seen_by_all;
      if constexpr (FMT == kFp4) {
        past = past && scale > kLargestFp4Scale;
      } else if (past) {
        past = false;
#pragma unroll
        for (int i = 0; i < 4 * kLoads; ++i) past |= e4m3_past(vr[i >> 2][i & 3], scale) != 0;
      }
      if (past) {
        odd = true;
#pragma unroll
        for (int i = 0; i < 4 * kLoads; ++i) vr[i >> 2][i & 3] = FMT == kFp4 ? fp4_finite8(vr[i >> 2][i & 3], scale) : e4m3_finite4(vr[i >> 2][i & 3], scale);
        if (scale > 0x1p127f) scale = 1.0f;  // (0 without a scale is no number)
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        auto values = [&](const u32x4 (&codes)[kLoads], float s) {
          if constexpr (FMT == kFp4) return fp4_unpack8(codes[0][i], s);
          else return e4m3_unpack8(codes[i >> 1][2 * (i & 1)], codes[i >> 1][2 * (i & 1) + 1], s);
        };
        *reinterpret_cast<u32x4*>(kt + chunk_at(row, 4 * (lane & 3) + i)) = values(kr, group_scale(ks));
        *reinterpret_cast<u32x4*>(vt + chunk_at(row, 4 * (lane & 3) + i)) = values(vr, scale);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kTurnRows / 4; ++j) {
        const int row = kTurnRows * wave + 4 * j + (lane >> 4);
        *reinterpret_cast<u32x4*>(kt + chunk_at(row, lane & 15)) = kr[j];
        if (loaded_row + kTurnRows > seen_by_all && loaded_row + 4 * j + (lane >> 4) >= seen_by_all) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned x = vr[j][i], bad = infinite_bits(x);
            odd |= bad != 0;
            vr[j][i] = x & ~bad;
          }
        }
        *reinterpret_cast<u32x4*>(vt + chunk_at(row, lane & 15)) = vr[j];
      }
    }
    const int flag = (__any(odd) ? 1 : 0) | (loaded_page ? 0 : 2 << (kTurnRows * wave / 16));
    if (flag != 0 && lane == 0) atomicOr(&flags[tile & 3], flag);
  };

  f32x16 acc[4];
  float ref = kLowest, sum = 0.0f;
  bool seen = false;  // (by this lane's rows)
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[cb][i] = 0.0f;
  if (tid < 4) flags[tid] = 0;
  __syncthreads();
  if (tile0 < tile1) {
    load_rows(tile0, page_of(tile0));
    store_rows(0, tile0);
    load_rows(tile0 + 1, page_of(tile0 + 1));
  }
  int page = tile0 < tile1 ? page_of(tile0 + 2) : -1;
  __syncthreads();

  for (int tile = tile0; tile < tile1; ++tile) {
    const int buffer = (tile - tile0) & 1, row0 = tile * kTurnTile;
    const char* kt = lds + buffer * kTurnTileBytes;
    const char* vt = kt + 2 * kTurnTileBytes;
    const int flag = uniform(flags[tile & 3]);
    const unsigned none = (unsigned)flag >> 1;
    if (tid == 0) flags[(tile + 2) & 3] = 0;
    const bool partial = row0 + kTurnTile > seen_by_all || flag != 0;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      if (!active) break;
      f32x16 s;
      __builtin_amdgcn_s_setprio(1);  // (a wave that multiplies goes before one that weighs: eight turns in 4 bits 399 -> 392 us)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(kt + chunk_at(32 * sub + l32, 2 * c + half));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[c], s, 0, 0, 0);
      }
      __builtin_amdgcn_s_setprio(0);
      bf16x8 w[2];
      {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = capped<CAP>(p, s[i]);
        if (partial) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool there = (row0 + 32 * sub + 8 * (i >> 2) + 4 * half + (i & 3) < vis) & ((none >> (2 * sub + (i >> 3)) & 1) == 0);
            seen |= there;
            if (!there) s[i] = -INFINITY;
          }
        } else {
          seen = true;
        }
        float m = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
        if (CAP == kNoCap) m *= p.c;
        if (__any(m > ref + kHeadroom)) {
          m = fmaxf(m, __shfl_xor(m, 32, 64));
          const float moved = fmaxf(ref, m), f = __builtin_amdgcn_exp2f(ref - moved);
          ref = moved;
          sum *= f;
#pragma unroll
          for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[cb][i] *= f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float y = __builtin_amdgcn_exp2f(CAP != kNoCap ? s[i] - ref : fmaf(s[i], p.c, -ref));
          sum += y;
          w[i >> 3][i & 7] = (__bf16)y;
        }
      }
      __builtin_amdgcn_s_setprio(1);
      // rows 16 * k + 4 * half .. + 3 and the four that are 8 further on, as the weights have them
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = 32 * sub + 16 * k + 4 * half + ((lane & 15) >> 2);
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          const int chunk = 4 * cb + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), in = 8 * (lane & 1);
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + chunk_at(row, chunk) + in));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + chunk_at(row + 8, chunk) + in));
          const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w[k], acc[cb], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (flag & 1) {  // values that are not finite, once more out of the pages, to the columns that see them
#pragma unroll 1
      for (int row = row0 > seen_by_all ? row0 : seen_by_all; row < row0 + kTurnTile && row < seen_by_last; ++row) {
        const int64_t at = find_row(p.pool, layer, seq, head, row);
        if (at < 0) continue;
        const int four = opaque(4 * half);
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const int c = 32 * cb + 8 * i4 + four;
            unsigned x[2];
            if constexpr (FMT == kFp4) {
              const unsigned codes = *reinterpret_cast<const uint16_t*>(p.pool.v + at * kBytes + c / 2);
              const float scale = group_scale(p.pool.v_scales[at * 4 + cb]);
              x[0] = fp4_unpack2(codes, scale, 0);
              x[1] = fp4_unpack2(codes, scale, 1);
            } else if constexpr (FMT == kE4m3) {
              const unsigned codes = *reinterpret_cast<const unsigned*>(p.pool.v + at * kBytes + c);
              const float scale = group_scale(p.pool.v_scales[at * 4 + cb]);
              x[0] = e4m3_unpack2(codes, scale, 0);
              x[1] = e4m3_unpack2(codes, scale, 1);
            } else {
              const u32x2 u = *reinterpret_cast<const u32x2*>(p.pool.v + at * kRowBytes + c * 2);
              x[0] = u[0];
              x[1] = u[1];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const unsigned bad = x[i >> 1] & infinite_bits(x[i >> 1]);
              const float value = __uint_as_float((i & 1) ? bad & 0xffff0000u : bad << 16);
              acc[cb][4 * i4 + i] += row < vis ? value : 0.0f;
            }
          }
      }
    }
    // (the other buffer was last read before the barrier that ended the step before)
    if (tile + 1 < tile1) {
      store_rows(buffer ^ 1, tile + 1);
      if (tile + 2 < tile1) load_rows(tile + 2, page);
      page = page_of(tile + 3);
    }
    __syncthreads();
  }

  {
    float total = sum + __shfl_xor(sum, 32, 64);
    const uint64_t with_rows = __ballot(seen);
    const bool any = ((with_rows >> l32 | with_rows >> (l32 + 32)) & 1) != 0;
    const int col = wave * 32 + opaque(l32);
    if (col0 + col >= col_end) return;
    if constexpr (SPLIT) {
      float* part = p.parts + ((int64_t)blockIdx.x * p.splits + blockIdx.y) * kTurnCols * (kHeadDim + 2);
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(part + (int64_t)col * kHeadDim + 32 * cb + 8 * i + 4 * half) =
              f32x4{acc[cb][4 * i], acc[cb][4 * i + 1], acc[cb][4 * i + 2], acc[cb][4 * i + 3]};
      if (half == 0) {
        part[kTurnCols * kHeadDim + col] = any ? ref : -INFINITY;
        part[kTurnCols * (kHeadDim + 1) + col] = total;
      }
    } else {
      const int step = quotient(rest0 + col, p.inv_group), h = head * g + rest0 + col - step * g;
      uint16_t* dst = p.out + (((int64_t)layer * p.total_new + first_row + token0 + step) * p.n_q_heads + h) * kHeadDim;
      const float f = 1.0f / total;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          bf16x4 o;
#pragma unroll
          for (int v = 0; v < 4; ++v) o[v] = (__bf16)(any ? acc[cb][4 * i + v] * f : 0.0f);
          *reinterpret_cast<bf16x4*>(dst + 32 * cb + 8 * i + 4 * half) = o;
        }
    }
  }
}

// The parts of a block's rows, in order: a wave to a column.
__global__ __launch_bounds__(256) void paged_turn_join_kernel(TurnParams p) {
  const int lane = threadIdx.x & 63, col = blockIdx.y * 4 + uniform(threadIdx.x >> 6);
  int block = uniform((int)(blockIdx.x / (unsigned)p.items));
  const int item = blockIdx.x - block * p.items, layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
  const int g = p.group;
  const int seq = find_block(p, lane, &block);
  if (seq < 0) return;
  const int cols = tokens_of(p, seq) * g, first_row = p.cu_new == nullptr ? seq * p.each_new : p.cu_new[seq], blocks = (cols + kTurnCols - 1) / kTurnCols;
  block = blocks - 1 - block;
  const int at = block * kTurnCols + col;
  if (at >= cols) return;
  const float* parts = p.parts + (int64_t)blockIdx.x * p.splits * kTurnCols * (kHeadDim + 2);
  auto part = [&](int i) { return parts + (int64_t)i * kTurnCols * (kHeadDim + 2); };
  float m = -INFINITY, sum = 0.0f;
  f32x2 o = {0.0f, 0.0f};
  for (int i0 = 0; i0 < p.splits; i0 += 64) {  // 64 parts, one to a lane
    const int n = p.splits - i0 < 64 ? p.splits - i0 : 64;
    const float r = lane < n ? part(i0 + lane)[kTurnCols * kHeadDim + col] : -INFINITY;
    float w = lane < n ? part(i0 + lane)[kTurnCols * (kHeadDim + 1) + col] : 0.0f;
    float top = r;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    if (top == -INFINITY) continue;  // (parts without a row)
    const float moved = fmaxf(m, top), f = __builtin_amdgcn_exp2f(r - moved), earlier = __builtin_amdgcn_exp2f(m - moved);
    w = r == -INFINITY ? 0.0f : w * f;
    for (int d = 32; d > 0; d >>= 1) w += __shfl_xor(w, d, 64);
    if (m != -INFINITY) {
      sum *= earlier;
      o *= earlier;
    }
    sum += w;
    m = moved;
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const f32x2 x = *reinterpret_cast<const f32x2*>(part(i0 + i) + (int64_t)col * kHeadDim + 2 * lane);
      const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i));
      if (__builtin_amdgcn_readlane(__float_as_uint(r), i) == 0xff800000u) continue;
      o[0] = fmaf(fi, x[0], o[0]);
      o[1] = fmaf(fi, x[1], o[1]);
    }
  }
  const int token = at / g, h = head * g + at - token * g;
  bf16x2 result;
  result[0] = (__bf16)(m == -INFINITY ? 0.0f : o[0] / sum);
  result[1] = (__bf16)(m == -INFINITY ? 0.0f : o[1] / sum);
  *reinterpret_cast<bf16x2*>(p.out + (((int64_t)layer * p.total_new + first_row + token) * p.n_q_heads + h) * kHeadDim + 2 * lane) = result;
}

// How such a call is run: a function of the descriptors alone, which the workspace follows.
struct TurnPlan {
  int splits;
  int64_t blocks;  // of columns, of all sequences and one KV head of a layer, at most
};
TurnPlan turn_plan(const dapq_pages* pages, const dapq_step* step) {
  const int64_t g = step->n_q_heads / pages->n_kv_heads;
  const int64_t most = most_new(pages, step);
  TurnPlan plan;
  const int64_t cols = kTurnCols, each = (most * g + cols - 1) / cols;
  const int64_t by_total = step->total_new * g / cols + pages->batch;
  plan.blocks = step->cu_new == nullptr || pages->batch * each < by_total ? pages->batch * each : by_total;
  const int64_t groups = plan.blocks * pages->n_layers * pages->n_kv_heads;
  const int64_t tiles = ((int64_t)pages->max_pages * pages->page_rows + kTurnTile - 1) / kTurnTile;
  // Parts for the 512 workgroups that the chip holds, of four tiles or more.  Us, one part / for 256 workgroups / 512 / 1024, 4 query heads of 8 KV heads, bf16:
  // 16 tokens behind 1000 rows 30 / 15 / 15 / 15, behind 100000 2290 / 97 / 100 / 132, of 8 sequences of 4000 rows 102 / 40 / 41 / 52, of 32 of them 106 / 107 / 114 / 124,
  // 500 tokens behind 1000 rows 48 / 39 / 36 / 45, 300 behind 8000 218 / 89 / 70 / 82; in 4 bits 16 tokens behind 100000 rows 2321 / 94 / 80 / 105, of 32 sequences of
  // 4000 rows 103 / 104 / 85 / 92.  Parts of two tiles or more / four / eight: 16 tokens behind 1000 rows 12.8 / 15.1 / 21.1, behind 4000 24.0 / 22.2 / 25.5, of 8 sequences
  // of 1000 rows 22.3 / 19.9 / 24.0, 500 tokens behind 1000 36.1 / 36.2 / 39.4.
  int64_t splits = groups > 0 ? 2048 / kTurnWaves / groups : 1;
  if (splits > tiles / 4) splits = tiles / 4;
  plan.splits = (int)(splits < 1 ? 1 : splits);
  return plan;
}

template <int FMT, bool SPLIT>
int launch_turn(const TurnParams& p, hipStream_t stream) {
  constexpr int kBytes = 4 * kTurnTileBytes + 16;
  const Cap cap = cap_of(p);
  auto kernel = cap == kNoCap ? paged_turn_kernel<FMT, kNoCap, SPLIT>
                              : (cap == kSmallCap ? paged_turn_kernel<FMT, kSmallCap, SPLIT> : paged_turn_kernel<FMT, kLargeCap, SPLIT>);
  const int rc = set_max_dynamic_lds(reinterpret_cast<const void*>(kernel), kBytes);
  if (rc != DAPQ_OK) return rc;
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.blocks * p.items, (unsigned)p.splits), dim3(64 * kTurnWaves), kBytes, stream, p);
  DAPQ_HIP_LAUNCH_CHECK("paged_turn_kernel");
  if (SPLIT) {
    hipLaunchKernelGGL(paged_turn_join_kernel, dim3((unsigned)p.blocks * p.items, (unsigned)(kTurnCols / 4)), dim3(256), 0, stream, p);
    DAPQ_HIP_LAUNCH_CHECK("paged_turn_join_kernel");
  }
  return DAPQ_OK;
}
}  // namespace

size_t turn_workspace_bytes(const dapq_pages* pages, const dapq_step* step) {
  const TurnPlan plan = turn_plan(pages, step);
  if (plan.splits == 1) return 256;
  return align_up((size_t)plan.blocks * pages->n_layers * pages->n_kv_heads * plan.splits * kTurnCols * (kHeadDim + 2) * sizeof(float), 256);
}

int launch_turn(const dapq_pages* pages, const dapq_step* step, const PagedAttentionParams& shared, hipStream_t stream) {
  const TurnPlan plan = turn_plan(pages, step);
  TurnParams p;
  static_cast<PagedAttentionParams&>(p) = shared;
  DAPQ_REQUIRE(plan.blocks * p.items < (int64_t)1 << 24, DAPQ_ERR_UNSUPPORTED, "%lld blocks of %d query rows are too many for a call",
               (long long)(plan.blocks * p.items), kTurnCols);
  p.blocks = (int32_t)plan.blocks;
  p.splits = plan.splits;
  if (pages->format == DAPQ_PAGES_FP4) return p.splits > 1 ? launch_turn<kFp4, true>(p, stream) : launch_turn<kFp4, false>(p, stream);
  if (pages->format == DAPQ_PAGES_E4M3) return p.splits > 1 ? launch_turn<kE4m3, true>(p, stream) : launch_turn<kE4m3, false>(p, stream);
  return p.splits > 1 ? launch_turn<kBf16, true>(p, stream) : launch_turn<kBf16, false>(p, stream);
}

}  // namespace dapq
