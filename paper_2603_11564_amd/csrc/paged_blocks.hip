// Which blocks of a cache in pages a token reads: bounds of the keys of a block, and the blocks whose keys the queries may score highest.
#include "kernel_args.h"
#include "paged_attention.h"
#include "paged_blocks.h"
#include "wave_scan.h"

namespace dapq {

int check_blocks(const dapq_pages* p, const dapq_blocks* b, bool need_bounds) {
  DAPQ_REQUIRE(b != nullptr, DAPQ_ERR_INVALID_ARG, "blocks is NULL");
  DAPQ_REQUIRE(b->block_rows >= 16 && b->block_rows <= p->page_rows && (b->block_rows & (b->block_rows - 1)) == 0, DAPQ_ERR_UNSUPPORTED,
               "block_rows (%d) must be a power of two from 16 to page_rows (%d)", b->block_rows, p->page_rows);
  DAPQ_REQUIRE(b->n_select >= 1 && b->n_select <= 4096, DAPQ_ERR_UNSUPPORTED, "n_select (%d) must be from 1 to 4096", b->n_select);
  DAPQ_REQUIRE(b->n_first >= 0 && b->n_last >= 1 && (int64_t)b->n_first + b->n_last <= b->n_select, DAPQ_ERR_INVALID_ARG,
               "n_first (%d) must not be negative, n_last (%d) at least 1, and both together no more than n_select (%d)", b->n_first, b->n_last,
               b->n_select);
  if (need_bounds) {
    DAPQ_REQUIRE(b->bounds != nullptr && b->scales != nullptr, DAPQ_ERR_INVALID_ARG, "bounds and scales of the blocks must not be NULL");
    DAPQ_REQUIRE((reinterpret_cast<uintptr_t>(b->bounds) & 15) == 0, DAPQ_ERR_UNSUPPORTED, "bounds of the blocks must be 16-byte aligned");
  }
  return DAPQ_OK;
}

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---- dapq_paged_bounds ----------------------------------------------------------------------------------------------------
struct BoundsParams {
  PagePool pool;
  uint8_t *bounds, *scales;
  const int32_t *first, *lengths;
  int32_t block_shift, max_rows;
};

// Two bf16 as whole numbers of 16 bits that sort as they do, and back.  An infinity and what is no number lie past all others, at both ends.
__device__ __forceinline__ unsigned sortable(unsigned x) {
  return x ^ (__builtin_bit_cast(unsigned, __builtin_bit_cast(s16x2, x) >> (short)15) & 0x7fff7fffu);
}
__device__ __forceinline__ unsigned upper_of(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ unsigned lower_of(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}

// 16 lanes have a row, eight channels to a lane.  SHARED: a wave has a block, four rows at a time, which meet at the end; else four blocks, one to 16 lanes, so that
// what a block costs beside its rows is shared by four.  Bound by bytes in bf16 (8 layers of 32768 rows, 537 MB, 97 us: 5.6 TB/s), by conversions and comparisons of codes.  Keys are compared as whole numbers, two to an instruction (a float to an instruction: 8 layers of
// 32768 rows in blocks of 64 in 8 and in 4 bits 62 us, now 58 and 42).
template <int FMT, bool SHARED>
__global__ __launch_bounds__(256) void paged_bounds_kernel(BoundsParams p) {
  touch_args<sizeof(BoundsParams)>();
  const int lane = threadIdx.x & 63, ch = lane & 15, part = lane >> 4;
  const int layer = blockIdx.y / p.pool.n_kv_heads, head = blockIdx.y - layer * p.pool.n_kv_heads, seq = blockIdx.z;
  const int first = p.first == nullptr || p.first[seq] < 0 ? 0 : p.first[seq];
  const int64_t bound = (int64_t)first + p.max_rows, length = p.lengths[seq] < bound ? p.lengths[seq] : bound;
  const int of_call = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t block = (int64_t)(first >> p.block_shift) + (SHARED ? of_call : 4 * of_call + part);
  if ((block + 1) << p.block_shift > length) return;  // (16 lanes agree)
  const int64_t row0 = find_row(p.pool, layer, seq, head, block << p.block_shift);
  if (row0 < 0) return;
  u32x4 hi, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) hi[i] = 0x80008000u, lo[i] = 0x7fff7fffu;
  constexpr int kStep = SHARED ? 4 : 1;
#pragma unroll(SHARED ? 4 : 8)
  for (int r = SHARED ? part : 0; r < 1 << p.block_shift; r += kStep) {
    const int64_t row = row0 + r;
    u32x4 x;
    if constexpr (FMT == kBf16) {
      x = *reinterpret_cast<const u32x4*>(p.pool.k + row * kRowBytes + ch * 16);
    } else {
      const float s = group_scale(p.pool.k_scales[row * 4 + (ch >> 2)]);
      if constexpr (FMT == kFp4) {
        x = fp4_unpack8(*reinterpret_cast<const unsigned*>(p.pool.k + row * kCodeBytes<FMT> + ch * 4), s);
      } else {
        const u32x2 c = *reinterpret_cast<const u32x2*>(p.pool.k + row * kCodeBytes<FMT> + ch * 8);
        x = e4m3_unpack8(c[0], c[1], s);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned whole = sortable(x[i]);
      hi[i] = upper_of(hi[i], whole), lo[i] = lower_of(lo[i], whole);
    }
  }
  unsigned largest = 0;  // of the magnitudes
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int d = 16; SHARED && d < 64; d *= 2) {
      hi[i] = upper_of(hi[i], (unsigned)__shfl_xor((int)hi[i], d, 64));
      lo[i] = lower_of(lo[i], (unsigned)__shfl_xor((int)lo[i], d, 64));
    }
    hi[i] = sortable(hi[i]), lo[i] = sortable(lo[i]);
    largest = larger(largest, larger(larger_magnitude(hi[i]), larger_magnitude(lo[i])));
  }
  largest = larger(largest, dpp<kRor1>(largest));  // (of the 16 lanes that have a row)
  largest = larger(largest, dpp<kRor2>(largest));
  largest = larger(largest, dpp<kRor4>(largest));
  largest = larger(largest, dpp<kRor8>(largest));
  const bool bad = largest >= 0x7f80u;
  const int unit = unit_byte(bad ? 0 : largest);
  const float per = power_of_two(254 - unit);
  const int64_t at = row0 >> p.block_shift;
  // (of a block that a wave shares the lanes of part 0 store the upper bounds, those of part 1 the lower ones)
#pragma unroll
  for (int side = 0; side < (SHARED ? 1 : 2); ++side) {
    const bool upper = SHARED ? part == 0 : side == 0;
    u32x2 w = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned two = upper ? hi[i >> 1] : lo[i >> 1];
      const float y = __uint_as_float(i & 1 ? two & 0xffff0000u : two << 16) * per, x = upper ? ceilf(y) : floorf(y);
      const int whole = bad ? 0 : (int)fminf(fmaxf(x, -127.0f), 127.0f);
      w[i >> 2] |= ((unsigned)whole & 255u) << (8 * (i & 3));
    }
    if (!SHARED || part < 2) *reinterpret_cast<u32x2*>(p.bounds + at * (2 * kHeadDim) + (upper ? 0 : kHeadDim) + ch * 8) = w;
  }
  if ((SHARED ? lane : ch) == 0) p.scales[at] = (uint8_t)(bad ? 255 : unit);
}

// ---- dapq_paged_select ----------------------------------------------------------------------------------------------------
// Scores as whole numbers that sort as they do.  No score, which is finite, comes near the last two.
constexpr unsigned kNoBlock = 0, kBadBlock = 0xfffffffeu, kEndBlock = 0xffffffffu;
__device__ __forceinline__ unsigned key_of(float score) {
  const unsigned u = __float_as_uint(score);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

struct SelectParams {
  PagePool pool;
  const uint8_t *bounds, *scales;
  const uint16_t* q;
  int32_t *idx, *count;
  const int32_t *cu_new, *lengths;
  unsigned* keys;  // of the workspace: [layer][token][KV head][stride]
  int64_t q_stride_layer, q_stride_row, q_stride_head, stride;
  int32_t batch, total_new, each_new, max_new, group, items;  // items: layers * Hkv
  int32_t block_shift, n_select, n_first, n_last;
  int32_t chunk, chunks, cols_log2;  // tiles of 16 blocks of a workgroup; such chunks of a sequence; columns of a token, a power of two
  int32_t col_tiles;                 // that a workgroup has in LDS
  float inv_items;
};

__device__ __forceinline__ int blocks_seen(const SelectParams& p, int before, int t) {
  const int most = p.pool.max_pages << p.pool.page_shift, n = (before < 1 << 30 ? before : 1 << 30) + t + 1;  // (rows are below 2^30, tokens no more than 2^25)
  return ((n < 0 ? 0 : (n < most ? n : most)) + (1 << p.block_shift) - 1) >> p.block_shift;
}

// Four keys, each the largest of the 2^log2 lanes that a lane stands among (up to 16).  Lanes that agree already are taken by mirrors of 8 and 16 lanes.
constexpr int kMirror8 = 0x141, kMirror16 = 0x140;
template <int CTRL>
__device__ __forceinline__ void with_lanes(u32x4& x) {
#pragma unroll
  for (int v = 0; v < 4; ++v) x[v] = larger(x[v], dpp<CTRL>(x[v]));
}
__device__ __forceinline__ void largest_of_lanes(u32x4& x, int log2) {
  if (log2 == 0) return;
  with_lanes<kXor1>(x);
  if (log2 == 1) return;
  with_lanes<kXor2>(x);
  if (log2 == 2) return;
  with_lanes<kMirror8>(x);
  if (log2 == 3) return;
  with_lanes<kMirror16>(x);
}

// What is kept of a token's keys: those above `least`, and of those equal to it the first `equal`.
struct Cut {
  unsigned least, equal;
};

// The bin that the want-th largest of 256 bins' entries lies in, the same in all lanes: its number, what of `want` falls to it, and its entries.
struct Bin {
  unsigned at, want, entries;
};
__device__ __forceinline__ Bin find_bin(const unsigned* bins, unsigned want, int lane) {
  const u32x4 x = *reinterpret_cast<const u32x4*>(bins + 252 - 4 * lane);  // from the top
  const unsigned own = x[0] + x[1] + x[2] + x[3], upto = wave_scan<OpAdd>(own);
  const int l = __builtin_ctzll(__ballot(upto >= want));
  unsigned rest = want - (unsigned)__builtin_amdgcn_readlane((int)(upto - own), l);
  unsigned bin = 255u - 4u * l;
#pragma unroll
  for (int i = 3; i > 0; --i) {
    const unsigned n = (unsigned)__builtin_amdgcn_readlane((int)x[i], l);
    if (rest <= n) return {bin, rest, n};
    rest -= n;
    --bin;
  }
  return {bin, rest, (unsigned)__builtin_amdgcn_readlane((int)x[0], l)};
}

// The cut of a token's keys.  The range that scores take is cut into 256 bins, then the bin that the last kept key lies in, until all of a bin is kept or it is
// one key; every wave reads the bins by itself, so that a round is one barrier.  each(f) calls f with each of a thread's keys.
template <int WAVES>
struct CutLds {
  __attribute__((aligned(16))) unsigned bins[4][256];
  unsigned range[WAVES][4];  // of a wave: least and largest key, keys, ends
};
template <int WAVES, typename EACH>
__device__ __forceinline__ Cut find_cut(const SelectParams& p, CutLds<WAVES>& lds, EACH each) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (tid < 256) lds.bins[i][tid] = 0;
  unsigned low = kEndBlock, high = 0, n = 0, ends = 0;
  each([&](unsigned x) {
    n += x != kNoBlock;
    ends += x == kEndBlock;
    low = x != kNoBlock && x < low ? x : low;
    high = x != kEndBlock && x > high ? x : high;
  });
  low = wave_reduce<OpMin>(low);
  high = wave_reduce<OpMax>(high);
  n = wave_sum(n);
  ends = wave_sum(ends);
  if (lane == 0) {
    lds.range[wave][0] = low;
    lds.range[wave][1] = high;
    lds.range[wave][2] = n;
    lds.range[wave][3] = ends;
  }
  __syncthreads();
  n = ends = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    low = low < lds.range[w][0] ? low : lds.range[w][0];
    high = larger(high, lds.range[w][1]);
    n += lds.range[w][2];
    ends += lds.range[w][3];
  }
  low = (unsigned)uniform((int)low), high = (unsigned)uniform((int)high);
  if (n <= (unsigned)p.n_select) return {kNoBlock, 0};  // all
  unsigned want = (unsigned)p.n_select - (unsigned)uniform((int)ends);
  if (want == 0) return {kEndBlock - 1, 0};
  // keys from `low` on, below low + 2^bits, in bins of 2^shift
  int shift = high - low < 256u ? 0 : 24 - __builtin_clz(high - low);
  int bits = 32;
  for (int round = 0;; ++round) {
    each([&](unsigned k) {
      const unsigned x = k - low;
      if (k != kNoBlock && k != kEndBlock && k >= low && (bits == 32 || x >> bits == 0)) atomicAdd(&lds.bins[round][x >> shift], 1u);
    });
    __syncthreads();
    const Bin bin = find_bin(lds.bins[round], want, lane);
    low += bin.at << shift;
    want = bin.want;
    if (bin.entries == want) return {low - 1, 0};  // the whole bin
    if (shift == 0) return {low, want};
    bits = shift;
    shift = shift > 8 ? shift - 8 : 0;
  }
}

// The n_select largest keys of a token and KV head, of equal ones the first, in order.  A workgroup has the keys in registers, REGS times four in a row to a thread.
// A chain of four barriers and, as a kernel, three trips to memory: 64 of 2048 for 8 items 4.8 us, for 1024 7.6, of 2063 for 12800 55 (of 8 KB each: 1.9 TB/s).
template <int WAVES, int REGS>
struct Choice {
  static constexpr int kTurn = 256 * WAVES;  // keys that the workgroup takes at a time
  static_assert(WAVES * REGS <= 64, "a lane for the sum of each");
  struct Lds {
    CutLds<WAVES> cut;
    unsigned sums[WAVES * REGS];
  };
  // k: this thread's keys kTurn * r + 4 * tid .. + 3; row: layer, token and head as idx has them
  static __device__ __forceinline__ void run(const SelectParams& p, Lds& lds, u32x4 (&k)[REGS], int blocks, int64_t row) {
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
#pragma unroll
    for (int r = 0; r < REGS; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (kTurn * r + 4 * tid + j >= blocks) k[r][j] = kNoBlock;
    const Cut cut = find_cut<WAVES>(p, lds.cut, [&](auto f) {
#pragma unroll
      for (int r = 0; r < REGS; ++r) {
        if (r > 0 && kTurn * r >= blocks) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) f(k[r][j]);
      }
    });
    // in order, before a thread's keys: above the cut in the low half, equal to it in the high one
    unsigned upto[REGS];
#pragma unroll
    for (int r = 0; r < REGS; ++r) {
      unsigned both = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) both += (unsigned)(k[r][j] > cut.least) + ((unsigned)(k[r][j] == cut.least && k[r][j] != kNoBlock) << 16);
      upto[r] = wave_scan<OpAdd>(both);
      if (lane == 63) lds.sums[WAVES * r + wave] = upto[r];
      upto[r] -= both;
    }
    __syncthreads();
    const unsigned sum = lane < WAVES * REGS ? lds.sums[lane] : 0, before = wave_scan<OpAdd>(sum);
    int32_t* out = p.idx + row * p.n_select;
#pragma unroll
    for (int r = 0; r < REGS; ++r) {
      unsigned here = upto[r] + (unsigned)__builtin_amdgcn_readlane((int)(before - sum), WAVES * r + wave);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned above = here & 0xffffu, equal = here >> 16;
        const bool same = k[r][j] == cut.least && k[r][j] != kNoBlock;
        if (k[r][j] > cut.least || (same && equal < cut.equal)) out[above + (equal < cut.equal ? equal : cut.equal)] = kTurn * r + 4 * tid + j;
        here += (unsigned)(k[r][j] > cut.least) + ((unsigned)same << 16);
      }
    }
    if (tid == 0) {
      const unsigned all = (unsigned)__builtin_amdgcn_readlane((int)before, 63);
      p.count[row] = (int)((all & 0xffffu) + (all >> 16 < cut.equal ? all >> 16 : cut.equal));
    }
  }
};

constexpr int kAhead = 1;
constexpr int kColTiles = 8, kColTileBytes = 4096;  // column tiles in LDS, at most; u+ and u- of 16 columns, and as much is a tile of bounds

// The score is a product of whole numbers of 8 bits, 256 long: with u+ = max(u, 0) and u- = min(u, 0), max(u * upper, u * lower) = u+ * upper + u- * lower.
// D[block][column] = bounds (A, 16 blocks) x (u+, u-) (B, 16 columns: query heads of a token, padded to a power of two) on v_mfma_i32_16x16x64_i8, exact.
// Bound by the bytes of the bounds where tokens are few: 64 sequences of 32768 rows, 8 KV heads, blocks of 16 (269 MB) 53 us with the choice (5.1 TB/s), of 4096..32768 rows
// in blocks of 32 (73 MB) 20.  A workgroup brings the columns of some tokens into LDS as operands, then each wave takes tiles of 16 blocks.  16 lanes load a block, whole lines of
// it, and the tile is turned in LDS: loaded as operands, 64 bytes of 16 blocks at a time, lines left the cache between their halves (22.6 us, with more tiles on their way 24 and 27).
// Many tokens are bound by a chain of some 40 vector instructions to a tile and 16 columns, and its waits: 200 tokens of 8 sequences of 8192..32768 rows 62 us.
// COLUMNS: kOne: one column tile in all, whose operand stays in registers; kMany; kWide: a token has more than 16 query heads, and several column tiles.
// REGS: of the Choice of the same workgroup, which has all tiles of the sequence and keeps their keys in LDS; 0: the keys go to the workspace.
enum Columns { kOne, kMany, kWide };
template <int COLUMNS, int WAVES, int REGS>
__global__ __launch_bounds__(64 * WAVES) void paged_scores_kernel(SelectParams p) {
  touch_args<sizeof(SelectParams)>();
  constexpr bool WIDE = COLUMNS == kWide, WHOLE = REGS > 0;
  extern __shared__ char lds[];  // column tiles; a tile of bounds to a wave; the units of the columns; WHOLE: keys
  float* units = reinterpret_cast<float*>(lds + (p.col_tiles + WAVES) * kColTileBytes);
  unsigned* whole_keys = reinterpret_cast<unsigned*>(units + 16 * p.col_tiles);
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
  const int wave = uniform(tid >> 6);
  char* turned = lds + (p.col_tiles + wave) * kColTileBytes;
  // (chunks of the same number follow each other: workgroups go round the chip's eight parts, and late chunks are those that sequences do not have)
  const int all_items = p.items * p.batch, chunk = blockIdx.x / all_items, of_item = blockIdx.x - chunk * all_items;
  const int seq = uniform_quotient(of_item, p.items, p.inv_items), item = of_item - seq * p.items;
  const int layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
  // the pages of the first tile are on their way before it is known whether there is one
  const int32_t* table = p.pool.table + (int64_t)seq * p.pool.max_pages;
  const int to_page = p.pool.page_shift - p.block_shift;  // blocks of a page, log2
  auto page_of = [&](int k) {
    const int e = (16 * k + n) >> to_page;
    return table[e < p.pool.max_pages ? e : p.pool.max_pages - 1];
  };
  int pages[kAhead + 1];
#pragma unroll
  for (int i = 0; i <= kAhead; ++i) pages[i] = page_of(chunk * p.chunk + wave + i * WAVES);
  const int first = uniform(p.cu_new == nullptr ? seq * p.each_new : p.cu_new[seq]);
  int tokens = p.cu_new == nullptr ? p.each_new : uniform(p.cu_new[seq + 1]) - first;
  tokens = tokens < p.max_new ? tokens : p.max_new;
  if (tokens <= 0) return;
  const int before = uniform(p.lengths[seq]);
  const int tiles = (blocks_seen(p, before, tokens - 1) + 15) >> 4, tile0 = chunk * p.chunk, tile1 = tile0 + p.chunk < tiles ? tile0 + p.chunk : tiles;
  if (!WHOLE && tile0 >= tile1) return;
  // A tile is asked for kAhead tiles before it is used, its pages one tile earlier.
  struct Tile {
    i32x4 a[4];
    int scale;  // -1 on no page
  };
  const int64_t head_of_layer = ((int64_t)layer * p.pool.n_pages * p.pool.n_kv_heads + head) << to_page;
  auto fetch = [&](Tile& tile, int k, int page) {
    const int block = 16 * k + n;
    const bool there = k < tile1 && page >= 0 && page < p.pool.n_pages && block >> to_page < p.pool.max_pages;
    // (blocks of a pool are below 2^32)
    const unsigned at = there ? (unsigned)(head_of_layer + (((int64_t)page * p.pool.n_kv_heads) << to_page) + (block & ((1 << to_page) - 1))) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned of_lane = (unsigned)__shfl((int)at, 4 * i + kg, 64);
      tile.a[i] = *reinterpret_cast<const i32x4*>(p.bounds + (uint64_t)of_lane * (2 * kHeadDim) + ((n ^ (4 * i + kg)) << 4));
    }
    const int scale = p.scales[at];
    tile.scale = there ? scale : -1;
  };
  const int log2 = WIDE ? 4 : p.cols_log2, each = 16 >> log2;  // tokens of a column tile
  const int all = WIDE ? (p.group + 15) >> 4 : (tokens + each - 1) / each;  // column tiles: of a token, or of the sequence
  const int middle0 = p.n_first, middle1 = blocks_seen(p, before, 0) - p.n_last;  // blocks that all tokens score
  for (int64_t t0 = WIDE ? blockIdx.y : 0; t0 < (WIDE ? tokens : 1); t0 += gridDim.y) {
    for (int c0 = WIDE ? 0 : blockIdx.y * p.col_tiles; c0 < all; c0 += WIDE ? p.col_tiles : (int)gridDim.y * p.col_tiles) {
      const int here = COLUMNS == kOne ? 1 : (all - c0 < p.col_tiles ? all - c0 : p.col_tiles);
      Tile ring[kAhead + 1];
      if (t0 > blockIdx.y || c0 > 0)
#pragma unroll
        for (int i = 0; i <= kAhead; ++i) pages[i] = page_of(tile0 + wave + i * WAVES);
      // 16 lanes to a column, eight channels to a lane; columns that there are not are the last one that there is
      const int col = tid >> 4 & 15, o = tid & 15;
      auto query = [&](int c) {
        c = c < here ? c : here - 1;
        int token = WIDE ? (int)t0 : (c0 + c) * each + (col >> log2), h = WIDE ? (c0 + c) * 16 + col : col & ((1 << log2) - 1);
        token = token < tokens ? token : tokens - 1;
        h = head * p.group + (h < p.group ? h : p.group - 1);
        return *reinterpret_cast<const u32x4*>(p.q + layer * p.q_stride_layer + (int64_t)(first + token) * p.q_stride_row + (int64_t)h * p.q_stride_head + 8 * o);
      };
      u32x4 x = query(tid >> 8);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) fetch(ring[i], tile0 + wave + i * WAVES, pages[i]);
      int page = pages[kAhead];
      for (int c = tid >> 8; c < here; c += WAVES / 4) {
        const u32x4 next = query(c + WAVES / 4);
        unsigned largest = larger(larger(larger_magnitude(x[0]), larger_magnitude(x[1])), larger(larger_magnitude(x[2]), larger_magnitude(x[3])));
        largest = larger(largest, dpp<kRor1>(largest));
        largest = larger(largest, dpp<kRor2>(largest));
        largest = larger(largest, dpp<kRor4>(largest));
        largest = larger(largest, dpp<kRor8>(largest));
        const bool bad = largest >= 0x7f80u;
        const int unit = unit_byte(bad ? 0 : largest);
        const float per = power_of_two(254 - unit);
        u32x2 up = {0, 0}, down = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned two = x[e >> 1];
          const float f = __uint_as_float(e & 1 ? two & 0xffff0000u : two << 16);
          const int whole = bad ? 0 : (int)rintf(fminf(fmaxf(f * per, -127.0f), 127.0f));
          up[e >> 2] |= (unsigned)(whole > 0 ? whole : 0) << (8 * (e & 3));
          down[e >> 2] |= ((unsigned)(whole < 0 ? whole : 0) & 255u) << (8 * (e & 3));
        }
        char* at = lds + c * kColTileBytes + (((o >> 3) * 64 + (o >> 1 & 3) * 16 + col) * 16 + (o & 1) * 8);
        *reinterpret_cast<u32x2*>(at) = up;
        *reinterpret_cast<u32x2*>(at + 2048) = down;
        if (o == 0) units[c * 16 + col] = power_of_two(unit);
        x = next;
      }
      __syncthreads();
      i32x4 own[4];  // kOne: the column tile's operand
      float own_unit = 0.0f;
      auto operand = [&](int c, int i) { return reinterpret_cast<const i32x4*>(lds + c * kColTileBytes)[64 * i + lane]; };
      if constexpr (COLUMNS == kOne) {
#pragma unroll
        for (int i = 0; i < 4; ++i) own[i] = operand(0, i);
        own_unit = units[n];
      }
      // where the keys of this lane's token, in the first column tile here, are written; of the next one `next` further on
      const int token0 = WIDE ? (int)t0 : c0 * each + (n >> log2);
      const int64_t next = WHOLE ? each * p.stride : (int64_t)each * p.pool.n_kv_heads * p.stride;
      unsigned* const to0 = (WHOLE ? whole_keys + (n >> log2) * p.stride : p.keys + (((int64_t)layer * p.total_new + first + token0) * p.pool.n_kv_heads + head) * p.stride) + 4 * kg;
      const bool writes = (n & ((1 << log2) - 1)) == 0;
      auto use = [&](const Tile& tile, int k) {
        // 16 lanes have brought in a block, whole lines of it; as operand a lane has its own: through LDS, with the 16 bytes of a block permuted by its number
        i32x4 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<i32x4*>(turned + 1024 * i + 16 * lane) = tile.a[i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const i32x4*>(turned + 256 * n + (((4 * i + kg) ^ n) << 4));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the next tile goes through the same place)
        const bool plain = 16 * k >= middle0 && 16 * k + 16 <= middle1 && !__any(tile.scale < 0 || tile.scale == 255);
        float factor[4];  // of this lane's blocks
        const float mine = power_of_two(tile.scale < 0 ? 0 : tile.scale);
#pragma unroll
        for (int v = 0; v < 4; ++v) factor[v] = __shfl(mine, 4 * kg + v, 64);
        auto put = [&](u32x4 keys, int c) {
          const int token = WIDE ? token0 : token0 + c * each;
          largest_of_lanes(keys, log2);
          if (!plain) {
            const int seen = blocks_seen(p, before, token);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int block = 16 * k + 4 * kg + v, s = __shfl(tile.scale, 4 * kg + v, 64);
              if (s == 255) keys[v] = kBadBlock;
              if (block < p.n_first || block >= seen - p.n_last) keys[v] = kEndBlock;
              if (block >= seen || s < 0) keys[v] = kNoBlock;
            }
          }
          u32x4* to = reinterpret_cast<u32x4*>(to0 + (WIDE ? 0 : c * next) + 16 * k);
          if (writes && token < tokens) {
            if (WIDE && c0 > 0) {  // (what this lane has written for the query heads before these)
              const u32x4 old = *to;
#pragma unroll
              for (int v = 0; v < 4; ++v) keys[v] = larger(keys[v], old[v]);
            }
            *to = keys;
          }
        };
        u32x4 of_token = {0, 0, 0, 0};
#pragma unroll 2
        for (int c = 0; c < here; ++c) {
          i32x4 sum = {0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], COLUMNS == kOne ? own[i] : operand(c, i), sum, 0, 0, 0);
          const float unit = COLUMNS == kOne ? own_unit : units[c * 16 + n];
          u32x4 keys;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            keys[v] = key_of((float)sum[v] * unit * factor[v]);
            of_token[v] = larger(of_token[v], keys[v]);
          }
          if (!WIDE) put(keys, c);
        }
        if (WIDE) put(of_token, 0);
      };
      for (int k0 = tile0 + wave; k0 < tile1; k0 += (kAhead + 1) * WAVES) {
#pragma unroll
        for (int i = 0; i <= kAhead; ++i) {
          const int k = k0 + i * WAVES;
          fetch(ring[(i + kAhead) % (kAhead + 1)], k + kAhead * WAVES, page);
          page = page_of(k + (kAhead + 1) * WAVES);
          if (k < tile1) use(ring[i], k);
        }
      }
      if constexpr (WHOLE) {
        using C = Choice<WAVES, REGS>;
        __shared__ typename C::Lds choice;
        __syncthreads();
        for (int t = c0 * each; t < tokens && t < (c0 + 1) * each; ++t) {
          const unsigned* keys = whole_keys + (t - c0 * each) * p.stride;
          const int blocks = blocks_seen(p, before, t);
          u32x4 k[REGS];
#pragma unroll
          for (int r = 0; r < REGS; ++r) k[r] = C::kTurn * r + 4 * tid < blocks ? *reinterpret_cast<const u32x4*>(keys + C::kTurn * r + 4 * tid) : u32x4{0, 0, 0, 0};
          C::run(p, choice, k, blocks, ((int64_t)layer * p.total_new + first + t) * p.pool.n_kv_heads + head);
        }
        return;  // (a workgroup has one column tile)
      }
      if (COLUMNS != kOne) __syncthreads();
    }
  }
}

template <int WAVES, int REGS>
__global__ __launch_bounds__(64 * WAVES) void paged_choose_kernel(SelectParams p) {
  touch_args<sizeof(SelectParams)>();
  using C = Choice<WAVES, REGS>;
  __shared__ typename C::Lds lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int row = blockIdx.x / p.pool.n_kv_heads;  // layer * total_new + token
  const unsigned* keys = p.keys + (int64_t)blockIdx.x * p.stride;
  u32x4 k[REGS];
  auto load = [&](int r, int end) { k[r] = C::kTurn * r + 4 * tid < end ? *reinterpret_cast<const u32x4*>(keys + C::kTurn * r + 4 * tid) : u32x4{0, 0, 0, 0}; };
  constexpr bool kEarly = WAVES * REGS <= 8;  // (the few keys of a narrow table are on their way before it is known how many of them count)
  if constexpr (kEarly)
#pragma unroll
    for (int r = 0; r < REGS; ++r) load(r, (int)p.stride);
  int seq, t;
  if (!find_token(p.cu_new, p.batch, p.each_new, p.max_new, row % p.total_new, lane, &seq, &t)) return;
  const int blocks = uniform(blocks_seen(p, p.lengths[seq], t));
  if constexpr (!kEarly)
#pragma unroll
    for (int r = 0; r < REGS; ++r) load(r, blocks);  // (a row has room for whole tiles)
  C::run(p, lds, k, blocks, blockIdx.x);
}

// The same of any number of keys, read again from memory for every round (one choice of 25000 blocks 18 us).
constexpr int kLongWaves = 16;
__global__ __launch_bounds__(64 * kLongWaves) void paged_choose_long_kernel(SelectParams p) {
  touch_args<sizeof(SelectParams)>();
  constexpr int kTurn = 256 * kLongWaves;
  __shared__ CutLds<kLongWaves> lds;
  __shared__ unsigned sums[2][kLongWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int row = blockIdx.x / p.pool.n_kv_heads;  // layer * total_new + token
  int seq, t;
  if (!find_token(p.cu_new, p.batch, p.each_new, p.max_new, row % p.total_new, lane, &seq, &t)) return;
  const int blocks = uniform(blocks_seen(p, p.lengths[seq], t));
  const unsigned* keys = p.keys + (int64_t)blockIdx.x * p.stride;
  auto four = [&](int i) {  // (a row has room for whole tiles, of which the last may hold keys past `blocks`: no blocks)
    return i < blocks ? *reinterpret_cast<const u32x4*>(keys + i) : u32x4{kNoBlock, kNoBlock, kNoBlock, kNoBlock};
  };
  const Cut cut = find_cut<kLongWaves>(p, lds, [&](auto f) {
#pragma unroll 4
    for (int i = 4 * tid; i < blocks; i += kTurn) {
      const u32x4 k = four(i);
#pragma unroll
      for (int j = 0; j < 4; ++j) f(i + j < blocks ? k[j] : kNoBlock);
    }
  });
  int32_t* out = p.idx + (int64_t)blockIdx.x * p.n_select;
  unsigned above = 0, equal = 0;  // so far
  u32x4 next = four(4 * tid);
  for (int i0 = 0, turn = 0; i0 < blocks; i0 += kTurn, turn ^= 1) {
    u32x4 k = next;
    next = four(i0 + kTurn + 4 * tid);
    unsigned both = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + 4 * tid + j >= blocks) k[j] = kNoBlock;
      both += (unsigned)(k[j] > cut.least) + ((unsigned)(k[j] == cut.least && k[j] != kNoBlock) << 16);
    }
    const unsigned upto = wave_scan<OpAdd>(both);
    if (lane == 63) sums[turn][wave] = upto;
    __syncthreads();  // (the sums of the turn before last are overwritten behind it)
    const unsigned sum = lane < kLongWaves ? sums[turn][lane] : 0, scan = wave_scan<OpAdd>(sum);
    const unsigned all = (unsigned)__builtin_amdgcn_readlane((int)scan, 63), before = upto - both + (unsigned)__builtin_amdgcn_readlane((int)(scan - sum), wave);
    unsigned a = above + (before & 0xffffu), e = equal + (before >> 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool same = k[j] == cut.least && k[j] != kNoBlock;
      if (k[j] > cut.least || (same && e < cut.equal)) out[a + (e < cut.equal ? e : cut.equal)] = i0 + 4 * tid + j;
      a += k[j] > cut.least;
      e += same;
    }
    above += all & 0xffffu;
    equal += all >> 16;
  }
  if (tid == 0) p.count[blockIdx.x] = (int)(above + (equal < cut.equal ? equal : cut.equal));
}

struct SelectPlan {
  int64_t stride, chunk, chunks, columns;  // columns: workgroups along the column tiles
  int cols_log2, col_tiles;
  bool whole;  // a workgroup scores all blocks of a sequence and KV head and chooses them
  int waves, lds;
};
int columns_log2(const dapq_pages* pages, const dapq_step* step) {
  int log2 = 0;
  while (1 << log2 < step->n_q_heads / pages->n_kv_heads) ++log2;
  return log2;
}
int64_t column_tiles(int group, int cols_log2, int64_t most) {
  const int64_t each = cols_log2 < 4 ? 16 >> cols_log2 : 1;
  return cols_log2 > 4 ? (group + 15) / 16 : (most + each - 1) / each;
}
// One kernel, a workgroup for all blocks of an item and a column tile of at most two tokens, or a kernel for chunks of blocks and one for the choice; `most` new tokens of a
// sequence, `items` sequences x KV heads x layers.  A workgroup takes 0.11 us a tile of its own, where the bytes of all take 0.75 ns (half of the table in use), and a second kernel
// some 3 us.  With several column tiles every workgroup reads the bounds, which pays while they are few.  Us, one kernel / two, 8 KV heads, 4 query heads a KV head, sequences x blocks: 1 x 128 6.5 / 8.9, 1 x 512 8.9 / 9.1, 1 x 2048 20.0 / 9.4, 8 x 512 9.1 / 9.8,
// 16 x 2048 20.9 / 21.4, 16 x 256..8192 65 / 42, 32 x 1024 16.0 / 20.5, 64 x 512 16.6 / 20.9, 64 x 2048 53 / 64, two tokens of 64 x 256 15.0 / 16.2; 8 query heads, four tokens of 16 x 512 12.3 /
// 13.5, of 64 x 64 11.2 / 14.6, of 64 x 256 25.4 / 18.1, eight of 64 x 64 18.5 / 21.0; 16 query heads, two tokens of 16 x 512 9.8 / 13.0, four of 32 x 512..2048 50 / 32.
// Lengths are not known here: one sequence that fills a table of 2048 / 4096 / 8192 blocks among 63 of 63 blocks 17.7 / 21.0, 30.7 / 34.1, 53.8 / 57.2 (in calls of their own 10.9, 13.7, 17.4
// and 6.0).  Its blocks are one workgroup's in either form, since chunks are cut for as many long sequences as there are; the second kernel is 3 us behind here too.
// fewest: the items; or 1, to ask whether calls of fewer items are one kernel as well (fewer tokens and items meet all other conditions too).
bool in_one_kernel(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step, int64_t most, int64_t items, int64_t fewest) {
  const int cols_log2 = columns_log2(pages, step);
  const int64_t tiles = (most_blocks(pages, blocks) + 15) / 16, each = cols_log2 < 4 ? 16 >> cols_log2 : 1, of_tile = most < each ? most : each;  // tokens of a column tile
  const int64_t col_tiles = column_tiles(step->n_q_heads / pages->n_kv_heads, cols_log2, most);
  auto bytes_of = [&](int64_t n) { return 0.75e-3 * (double)(tiles * n); };
  return cols_log2 <= 4 && of_tile <= 2 && col_tiles <= 16 && 16 * tiles <= 8192 && items < 1 << 20 && 0.11 * (double)tiles < 3.0 + 0.5 * bytes_of(fewest) &&
         (col_tiles <= 1 || bytes_of(items) * (double)col_tiles < 9.0);
}
SelectPlan select_plan(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  SelectPlan plan;
  const int64_t tiles = (most_blocks(pages, blocks) + 15) / 16;
  plan.stride = 16 * tiles;
  const int group = step->n_q_heads / pages->n_kv_heads;
  plan.cols_log2 = columns_log2(pages, step);
  const int64_t most = most_new(pages, step), tiles_of_columns = column_tiles(group, plan.cols_log2, most);
  plan.col_tiles = (int)(tiles_of_columns < kColTiles ? (tiles_of_columns < 1 ? 1 : tiles_of_columns) : kColTiles);
  plan.columns = plan.cols_log2 > 4 ? most : (tiles_of_columns + plan.col_tiles - 1) / plan.col_tiles;
  plan.columns = plan.columns < 1 ? 1 : (plan.columns > 65535 ? 65535 : plan.columns);
  const int64_t items = (int64_t)pages->n_layers * pages->batch * pages->n_kv_heads;
  plan.whole = in_one_kernel(pages, blocks, step, most, items, items);
  plan.waves = plan.whole && plan.stride > 256 ? 8 : 4;
  if (plan.whole) {
    plan.col_tiles = 1;
    plan.columns = tiles_of_columns < 1 ? 1 : tiles_of_columns;
  }
  plan.lds = plan.col_tiles * (kColTileBytes + 64) + plan.waves * kColTileBytes;
  if (plan.whole) {
    const int64_t each = plan.cols_log2 < 4 ? 16 >> plan.cols_log2 : 1;
    plan.lds += (int)((most < each ? most : each) * plan.stride * 4);
    plan.chunk = tiles;
  } else {
    // Chunks for some 1024 workgroups: four tokens of 32 sequences of 512..2048 blocks, scores with 512 / 768 / 1024 / 1536 / 2048 workgroups 26.3 / 24.8 / 23.2 / 24.3 / 24.5 us.
    // No fewer than 4 tiles, one to a wave.
    plan.chunk = (tiles * items * plan.columns + 1023) / 1024;
    plan.chunk = plan.chunk < 4 ? 4 : (plan.chunk < tiles ? (plan.chunk + 3) / 4 * 4 : (tiles + 3) / 4 * 4);
  }
  plan.chunks = (tiles + plan.chunk - 1) / plan.chunk;
  return plan;
}

int check_select(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  int rc = check_pages(pages);
  if (rc == DAPQ_OK) rc = check_blocks(pages, blocks, true);
  if (rc == DAPQ_OK) rc = check_step(pages, step);
  if (rc == DAPQ_OK) rc = check_queries(step);
  if (rc != DAPQ_OK) return rc;
  // (a launch holds fewer than 2^32 threads along an axis)
  DAPQ_REQUIRE((int64_t)pages->n_layers * step->total_new * pages->n_kv_heads < (int64_t)1 << 22, DAPQ_ERR_UNSUPPORTED,
               "n_layers * total_new * n_kv_heads (%lld) must be below 2^22", (long long)(pages->n_layers * step->total_new * pages->n_kv_heads));
  DAPQ_REQUIRE(step->n_q_heads <= 65535, DAPQ_ERR_UNSUPPORTED, "n_q_heads (%d) exceeds 65535", step->n_q_heads);
  return DAPQ_OK;
}

}  // namespace

}  // namespace dapq

using namespace dapq;

extern "C" DAPQ_API int dapq_paged_bounds(const dapq_pages* pages, const dapq_blocks* blocks, const int32_t* first, const int32_t* lengths, int32_t max_rows,
                                          void* stream) {
  int rc = check_pages(pages);
  if (rc == DAPQ_OK) rc = check_blocks(pages, blocks, true);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(lengths != nullptr, DAPQ_ERR_INVALID_ARG, "lengths must not be NULL");
  DAPQ_REQUIRE(max_rows >= 0, DAPQ_ERR_INVALID_ARG, "max_rows (%d) must not be negative", max_rows);
  DAPQ_REQUIRE(pages->batch <= 65535, DAPQ_ERR_UNSUPPORTED, "batch (%d) exceeds 65535", pages->batch);
  if (max_rows == 0) return DAPQ_OK;
  BoundsParams p;
  p.pool = page_pool(pages);
  p.bounds = reinterpret_cast<uint8_t*>(blocks->bounds);
  p.scales = blocks->scales;
  p.first = first;
  p.lengths = lengths;
  p.block_shift = __builtin_ctz((unsigned)blocks->block_rows);
  p.max_rows = max_rows;
  const int64_t all = most_blocks(pages, blocks), most = ((int64_t)max_rows + blocks->block_rows - 1) / blocks->block_rows;
  // 8 layers of 32768 rows, us, a block of 16 rows shared by a wave / not, of 32, of 64: bf16 106 / 113, 101 / 108, 99 / 99; in 8 bits 85 / 62, 69 / 65, 58 / 57; in 4 bits
  // 78 / 42, 53 / 35, 42 / 32, but 64 blocks of 64 rows 4.2 / 6.6.  In bf16 bytes bound both, and rows that follow each other are read at once by the first.
  // Of 128 rows, the same call repeated, 43 / 45 in 8 bits and 34 / 29 in 4, of 256 43 / 42 and 32 / 32; one layer of them 8.1 / 14.0, 6.4 / 10.0 and 10.9 / 24.8, 7.3 / 17.7.  A token
  // of 64 sequences, 16 / 32 / 64 / 128 / 256 rows: 3.2 / 4.6, 3.4 / 6.2, 4.1 / 9.6, 5.1 / 16.5, 7.4 / 30.  Above 32 rows the shared form is never far behind and far ahead where blocks are
  // few; below, the other one wins with many blocks and loses up to 3 us with few.  The rule knows no number of blocks, so that in 4 bits many blocks of 64 pay a third more.
  const bool shared = pages->format == DAPQ_PAGES_BF16 || blocks->block_rows > 32;
  const int of_group = shared ? 4 : 16;  // blocks
  const int64_t groups = ((most < all ? most : all) + of_group - 1) / of_group;
  DAPQ_REQUIRE(groups * 256 < (int64_t)1 << 32, DAPQ_ERR_UNSUPPORTED, "max_rows (%d) is too large", max_rows);
  auto kernel = pages->format == DAPQ_PAGES_BF16 ? paged_bounds_kernel<kBf16, true>
                : pages->format == DAPQ_PAGES_FP4 ? (shared ? paged_bounds_kernel<kFp4, true> : paged_bounds_kernel<kFp4, false>)
                                                  : (shared ? paged_bounds_kernel<kE4m3, true> : paged_bounds_kernel<kE4m3, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)(pages->n_layers * pages->n_kv_heads), (unsigned)pages->batch), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_bounds_kernel");
  return DAPQ_OK;
}

extern "C" DAPQ_API size_t dapq_paged_select_workspace_bytes(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  if (check_select(pages, blocks, step) != DAPQ_OK) return 0;
  // Enough for every smaller step as well, however its tokens are packed: one of fewer items may take two kernels where this one takes one, whose keys are no more than these.
  const int64_t most = step->max_new < step->total_new ? step->max_new : step->total_new, items = (int64_t)pages->n_layers * pages->batch * pages->n_kv_heads;
  if (in_one_kernel(pages, blocks, step, most, items, 1)) return 256;
  const int64_t rows = (int64_t)pages->n_layers * step->total_new * pages->n_kv_heads, stride = 16 * ((most_blocks(pages, blocks) + 15) / 16);
  return align_up((size_t)(rows < 1 ? 1 : rows) * stride * sizeof(unsigned), 256);
}

extern "C" DAPQ_API int dapq_paged_select(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step, const void* q, int32_t* idx,
                                          int32_t* count, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_select(pages, blocks, step);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(q != nullptr && idx != nullptr && count != nullptr, DAPQ_ERR_INVALID_ARG, "q, idx and count must not be NULL");
  DAPQ_REQUIRE((reinterpret_cast<uintptr_t>(q) & 15) == 0, DAPQ_ERR_UNSUPPORTED, "q must be 16-byte aligned");
  if (step->total_new == 0 || step->max_new == 0) return DAPQ_OK;
  rc = check_workspace(workspace, workspace_bytes, dapq_paged_select_workspace_bytes(pages, blocks, step));
  if (rc != DAPQ_OK) return rc;
  const SelectPlan plan = select_plan(pages, blocks, step);
  SelectParams p;
  p.pool = page_pool(pages);
  p.bounds = reinterpret_cast<const uint8_t*>(blocks->bounds);
  p.scales = blocks->scales;
  p.q = static_cast<const uint16_t*>(q);
  p.idx = idx;
  p.count = count;
  p.cu_new = step->cu_new;
  p.lengths = step->lengths;
  p.keys = static_cast<unsigned*>(workspace);
  p.q_stride_layer = step->q_stride_layer; p.q_stride_row = step->q_stride_row; p.q_stride_head = step->q_stride_head;
  p.stride = plan.stride;
  p.batch = pages->batch;
  p.total_new = (int32_t)step->total_new;
  p.each_new = (int32_t)(step->total_new / pages->batch);
  p.max_new = most_new(pages, step);
  p.group = step->n_q_heads / pages->n_kv_heads;
  p.items = pages->n_layers * pages->n_kv_heads;
  p.block_shift = __builtin_ctz((unsigned)blocks->block_rows);
  p.n_select = blocks->n_select; p.n_first = blocks->n_first; p.n_last = blocks->n_last;
  p.chunk = (int32_t)plan.chunk;
  p.chunks = (int32_t)plan.chunks;
  p.cols_log2 = plan.cols_log2;
  p.inv_items = 1.0f / (float)p.items;
  p.col_tiles = plan.col_tiles;
  const hipStream_t on = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)((int64_t)p.items * p.batch * p.chunks), (unsigned)plan.columns);
  if (plan.whole) {
    auto kernel = plan.waves == 4 ? paged_scores_kernel<kOne, 4, 1> : (plan.stride <= 2048 ? paged_scores_kernel<kOne, 8, 1> : paged_scores_kernel<kOne, 8, 4>);
    rc = set_max_dynamic_lds(reinterpret_cast<const void*>(kernel), 9 * kColTileBytes + 64 + 2 * 8192 * 4);
    if (rc != DAPQ_OK) return rc;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * plan.waves), plan.lds, on, p);
    DAPQ_HIP_LAUNCH_CHECK("paged_scores_kernel");
    return DAPQ_OK;
  }
  hipLaunchKernelGGL((plan.cols_log2 > 4 ? paged_scores_kernel<kWide, 4, 0> : (plan.col_tiles == 1 ? paged_scores_kernel<kOne, 4, 0> : paged_scores_kernel<kMany, 4, 0>)),
                     grid, dim3(256), plan.lds, on, p);
  DAPQ_HIP_LAUNCH_CHECK("paged_scores_kernel");
  const unsigned rows = (unsigned)((int64_t)p.items * p.total_new);
  // A workgroup chooses for an item, with its keys in registers, up to 32 to a thread.  200 tokens of 8 sequences (12800 items), us: up to 1024 blocks 256 threads 30, 64 threads 21, but
  // 64 threads 9.5 for 7.9 with 2048 items, 14.5 for 9.7 with 1536 of 2048 blocks, and 90 for 55 with 12800 of 4096 blocks; 1024 threads waited for each other for 364 us.
  if (plan.stride <= 1024) hipLaunchKernelGGL((paged_choose_kernel<4, 1>), dim3(rows), dim3(256), 0, on, p);
  else if (plan.stride <= 2048) hipLaunchKernelGGL((paged_choose_kernel<4, 2>), dim3(rows), dim3(256), 0, on, p);
  else if (plan.stride <= 4096) hipLaunchKernelGGL((paged_choose_kernel<4, 4>), dim3(rows), dim3(256), 0, on, p);
  else if (plan.stride <= 8192) hipLaunchKernelGGL((paged_choose_kernel<8, 4>), dim3(rows), dim3(512), 0, on, p);
  else if (plan.stride <= 16384) hipLaunchKernelGGL((paged_choose_kernel<8, 8>), dim3(rows), dim3(512), 0, on, p);
  else hipLaunchKernelGGL(paged_choose_long_kernel, dim3(rows), dim3(64 * kLongWaves), 0, on, p);
  DAPQ_HIP_LAUNCH_CHECK("paged_choose_kernel");
  return DAPQ_OK;
}
