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

// A wave has a block: 16 lanes to a row, eight channels to a lane, four rows at a time; the four meet at the end.
template <int FMT>
__global__ __launch_bounds__(256) void paged_bounds_kernel(BoundsParams p) {
  touch_args<sizeof(BoundsParams)>();
  const int lane = threadIdx.x & 63, ch = lane & 15, part = lane >> 4;
  const int layer = blockIdx.y / p.pool.n_kv_heads, head = blockIdx.y - layer * p.pool.n_kv_heads, seq = blockIdx.z;
  const int first = p.first == nullptr || p.first[seq] < 0 ? 0 : p.first[seq];
  const int64_t bound = (int64_t)first + p.max_rows, length = p.lengths[seq] < bound ? p.lengths[seq] : bound;
  const int64_t block = (int64_t)(first >> p.block_shift) + blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((block + 1) << p.block_shift > length) return;
  const int64_t row0 = find_row(p.pool, layer, seq, head, block << p.block_shift);
  if (row0 < 0) return;
  float hi[8], lo[8];
  unsigned largest = 0;  // of the magnitudes, infinities and NaN among them
#pragma unroll
  for (int i = 0; i < 8; ++i) hi[i] = -INFINITY, lo[i] = INFINITY;
#pragma unroll 4
  for (int r = part; r < 1 << p.block_shift; r += 4) {
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
      const float a = __uint_as_float(x[i] << 16), b = __uint_as_float(x[i] & 0xffff0000u);
      hi[2 * i] = fmaxf(hi[2 * i], a), lo[2 * i] = fminf(lo[2 * i], a);
      hi[2 * i + 1] = fmaxf(hi[2 * i + 1], b), lo[2 * i + 1] = fminf(lo[2 * i + 1], b);
      largest = larger(largest, larger_magnitude(x[i]));
    }
  }
#pragma unroll
  for (int d = 16; d < 64; d *= 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], d, 64));
      lo[i] = fminf(lo[i], __shfl_xor(lo[i], d, 64));
    }
  }
  largest = wave_reduce<OpMax>(largest);
  const bool bad = largest >= 0x7f80u;
  const int unit = unit_byte(largest);
  const float per = power_of_two(254 - unit);
  const int64_t at = row0 >> p.block_shift;
  // (the lanes of part 0 store the upper bounds, those of part 1 the lower ones)
  unsigned w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = part == 0 ? ceilf(hi[i] * per) : floorf(lo[i] * per);
    const int whole = bad ? 0 : (int)fminf(fmaxf(x, -127.0f), 127.0f);
    w[i >> 2] |= ((unsigned)whole & 255u) << (8 * (i & 3));
  }
  if (part < 2) *reinterpret_cast<u32x2*>(p.bounds + at * (2 * kHeadDim) + part * kHeadDim + ch * 8) = u32x2{w[0], w[1]};
  if (lane == 0) p.scales[at] = (uint8_t)(bad ? 255 : unit);
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
  float inv_items, inv_chunks;
};

__device__ __forceinline__ int blocks_seen(const SelectParams& p, int before, int t) {
  const int64_t most = (int64_t)p.pool.max_pages << p.pool.page_shift, n = (int64_t)before + t + 1;
  return (int)(((n < 0 ? 0 : (n < most ? n : most)) + (1 << p.block_shift) - 1) >> p.block_shift);
}

// Largest of the 2^log2 lanes that a lane stands among (up to 16).
__device__ __forceinline__ float largest_of_lanes(float x, int log2) {
  auto with = [&](float y) { return fmaxf(x, y); };
  if (log2 >= 1) x = with(__uint_as_float(dpp<kXor1>(__float_as_uint(x))));
  if (log2 >= 2) x = with(__uint_as_float(dpp<kXor2>(__float_as_uint(x))));
  if (log2 >= 3) x = with(__shfl_xor(x, 4, 64));
  if (log2 >= 4) x = with(__shfl_xor(x, 8, 64));
  return x;
}

// The score is a product of whole numbers of 8 bits, 256 long: with u+ = max(u, 0) and u- = min(u, 0), max(u * upper, u * lower) = u+ * upper + u- * lower.
// D[block][column] = bounds (A, 16 blocks) x (u+, u-) (B, 16 columns: query heads of a token, padded to a power of two) on v_mfma_i32_16x16x64_i8, exact.
// Bound by the bytes of the bounds.  A wave has a tile of 16 blocks at a time.
__global__ __launch_bounds__(256) void paged_scores_kernel(SelectParams p) {
  touch_args<sizeof(SelectParams)>();
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  const int of_item = uniform_quotient(blockIdx.x, p.chunks, p.inv_chunks), chunk = blockIdx.x - of_item * p.chunks;
  const int seq = uniform_quotient(of_item, p.items, p.inv_items), item = of_item - seq * p.items;
  const int layer = item / p.pool.n_kv_heads, head = item - layer * p.pool.n_kv_heads;
  const int first = uniform(p.cu_new == nullptr ? seq * p.each_new : p.cu_new[seq]);
  int tokens = p.cu_new == nullptr ? p.each_new : uniform(p.cu_new[seq + 1]) - first;
  tokens = tokens < p.max_new ? tokens : p.max_new;
  if (tokens <= 0) return;
  const int before = uniform(p.lengths[seq]);
  const int tiles = (blocks_seen(p, before, tokens - 1) + 15) >> 4, tile0 = chunk * p.chunk, tile1 = tile0 + p.chunk < tiles ? tile0 + p.chunk : tiles;
  if (tile0 >= tile1) return;
  const int wide = p.cols_log2 > 4 ? p.cols_log2 - 4 : 0;  // a token has 2^wide column tiles
  const int each = p.cols_log2 < 4 ? 4 - p.cols_log2 : 0;  // or a column tile 2^each tokens
  for (int64_t t0 = (int64_t)blockIdx.y << each; t0 < tokens; t0 += (int64_t)gridDim.y << each) {
    const int token = (int)t0 + (n >> p.cols_log2);
    const int seen = token < tokens ? blocks_seen(p, before, token) : 0;
    for (int k0 = tile0 + wave; k0 < tile1; k0 += 4) {
      const int64_t row = (int64_t)(16 * k0 + n) << p.block_shift;
      const int64_t at = row >> p.pool.page_shift < p.pool.max_pages ? find_row(p.pool, layer, seq, head, row) >> p.block_shift : -1;
      i32x4 a[4];
      const uint8_t* src = p.bounds + (at < 0 ? 0 : at) * (2 * kHeadDim) + 16 * kg;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = at < 0 ? i32x4{0, 0, 0, 0} : *reinterpret_cast<const i32x4*>(src + 64 * i);
      const int scale = at < 0 ? -1 : p.scales[at];
      float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      for (int w = 0; w < 1 << wide; ++w) {
        const int col = wide ? 16 * w + n : n & ((1 << p.cols_log2) - 1);
        const bool real = token < tokens && col < p.group;
        // the column's whole numbers: channels 16 * kg .. + 15 and 64 further on
        const uint16_t* qs = p.q + layer * p.q_stride_layer + (int64_t)(first + (real ? token : 0)) * p.q_stride_row + (int64_t)(head * p.group + (real ? col : 0)) * p.q_stride_head;
        u32x4 x[4];
        unsigned largest = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = *reinterpret_cast<const u32x4*>(qs + 64 * (i >> 1) + 16 * kg + 8 * (i & 1));
#pragma unroll
          for (int j = 0; j < 4; ++j) largest = larger(largest, larger_magnitude(x[i][j]));
        }
        largest = larger(largest, (unsigned)__shfl_xor((int)largest, 16, 64));
        largest = larger(largest, (unsigned)__shfl_xor((int)largest, 32, 64));
        const bool bad = largest >= 0x7f80u;
        const int unit = unit_byte(bad ? 0 : largest);
        const float per = power_of_two(254 - unit);
        i32x4 d = {0, 0, 0, 0};
        i32x4 up[2], down[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            unsigned u = 0, v = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned two = x[2 * i + (j >> 1)][2 * (j & 1) + (e >> 1)];
              const float f = __uint_as_float(e & 1 ? two & 0xffff0000u : two << 16);
              const int whole = bad ? 0 : (int)rintf(fminf(fmaxf(f * per, -127.0f), 127.0f));
              u |= (unsigned)(whole > 0 ? whole : 0) << (8 * e);
              v |= ((unsigned)(whole < 0 ? whole : 0) & 255u) << (8 * e);
            }
            up[i][j] = (int)u;
            down[i][j] = (int)v;
          }
#pragma unroll
        for (int i = 0; i < 2; ++i) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], up[i], d, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[2 + i], down[i], d, 0, 0, 0);
        const float two_to_f = power_of_two(unit);
#pragma unroll
        for (int v = 0; v < 4; ++v) best[v] = fmaxf(best[v], real ? (float)d[v] * two_to_f : -INFINITY);
      }
      u32x4 keys;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float top = largest_of_lanes(best[v], p.cols_log2);
        const int block = 16 * k0 + 4 * kg + v, s = __shfl(scale, 4 * kg + v, 64);
        const unsigned scored = s == 255 ? kBadBlock : key_of(top * power_of_two(s < 0 ? 0 : s));
        keys[v] = block >= seen || s < 0 ? kNoBlock : (block < p.n_first || block >= seen - p.n_last ? kEndBlock : scored);
      }
      if (token < tokens && (n & ((1 << (p.cols_log2 < 4 ? p.cols_log2 : 4)) - 1)) == 0)
        *reinterpret_cast<u32x4*>(p.keys + (((int64_t)layer * p.total_new + first + token) * p.pool.n_kv_heads + head) * p.stride + 16 * k0 + 4 * kg) = keys;
    }
  }
}

// The n_select largest keys of a token and KV head, of equal ones the first: a workgroup finds the smallest key that is kept, eight bits at a time, then
// writes down in order what lies above it and as many of its like as there is room for.
__global__ __launch_bounds__(256) void paged_choose_kernel(SelectParams p) {
  touch_args<sizeof(SelectParams)>();
  __shared__ unsigned bins[256];
  __shared__ unsigned found[2];
  __shared__ unsigned wave_sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int row = blockIdx.x / p.pool.n_kv_heads;  // layer * total_new + token
  const int r = row % p.total_new;
  int seq, t;
  if (!find_token(p.cu_new, p.batch, p.each_new, p.max_new, r, lane, &seq, &t)) return;
  const int blocks = blocks_seen(p, uniform(p.lengths[seq]), t);
  const unsigned* keys = p.keys + (int64_t)blockIdx.x * p.stride;
  unsigned least = 0, want = (unsigned)p.n_select;  // the kept keys' leading bits so far; how many of those with the same are kept
  for (int shift = 24; shift >= 0; shift -= 8) {
    bins[tid] = 0;
    __syncthreads();
    for (int i = tid; i < blocks; i += 256) {
      const unsigned k = keys[i];
      if (k != kNoBlock && (shift == 24 || (k ^ least) >> (shift + 8) == 0)) atomicAdd(&bins[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    // bins from the top: thread tid has bin 255 - tid
    const unsigned mine = bins[255 - tid];
    unsigned upto = wave_scan<OpAdd>(mine);
    if (lane == 63) wave_sums[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += wave_sums[w];
    if (tid == 255) found[0] = upto < want ? ~0u : 0u;  // (fewer keys than wanted: only in the first round)
    __syncthreads();
    if (found[0] == ~0u) {
      least = kNoBlock;
      want = 0;
      break;
    }
    if (upto >= want && upto - mine < want) found[1] = (unsigned)(255 - tid), found[0] = want - (upto - mine);
    __syncthreads();
    least |= found[1] << shift;
    want = found[0];
    __syncthreads();
  }
  // `want` of the keys equal to `least` (none of the keys of no block), and all above
  int32_t* out = p.idx + (int64_t)blockIdx.x * p.n_select;
  unsigned above = 0, equal = 0;  // so far
  for (int i0 = 0; i0 < blocks; i0 += 1024) {
    unsigned k[4];
    unsigned a = 0, e = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + 4 * tid + j;
      k[j] = i < blocks ? keys[i] : kNoBlock;
      a += k[j] > least;
      e += k[j] == least;
    }
    const unsigned both = a | e << 16;
    unsigned upto = wave_scan<OpAdd>(both);
    __syncthreads();
    if (lane == 63) wave_sums[wave] = upto;
    __syncthreads();
    unsigned all = 0;
    for (int w = 0; w < 4; ++w) {
      if (w < wave) upto += wave_sums[w];
      all += wave_sums[w];
    }
    unsigned a0 = above + ((upto - both) & 0xffffu), e0 = equal + ((upto - both) >> 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool take = k[j] > least || (k[j] == least && e0 < want);
      if (take) out[a0 + (e0 < want ? e0 : want)] = i0 + 4 * tid + j;
      a0 += k[j] > least;
      e0 += k[j] == least;
    }
    above += all & 0xffffu;
    equal += all >> 16;
  }
  if (tid == 0) p.count[blockIdx.x] = (int)(above + (equal < want ? equal : want));
}

struct SelectPlan {
  int64_t stride, chunk, chunks, col_tiles;
  int cols_log2;
};
SelectPlan select_plan(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  SelectPlan plan;
  const int64_t tiles = (most_blocks(pages, blocks) + 15) / 16;
  plan.stride = 16 * tiles;
  const int group = step->n_q_heads / pages->n_kv_heads;
  plan.cols_log2 = 0;
  while (1 << plan.cols_log2 < group) ++plan.cols_log2;
  const int64_t each = plan.cols_log2 < 4 ? 16 >> plan.cols_log2 : 1;
  plan.col_tiles = (most_new(pages, step) + each - 1) / each;
  if (plan.col_tiles > 65535) plan.col_tiles = 65535;
  const int64_t items = (int64_t)pages->n_layers * pages->batch * pages->n_kv_heads;
  plan.chunk = (tiles * items + 2047) / 2048;
  plan.chunk = plan.chunk < 4 ? 4 : (plan.chunk + 3) / 4 * 4;
  plan.chunks = (tiles + plan.chunk - 1) / plan.chunk;
  return plan;
}

int check_select(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  int rc = check_pages(pages);
  if (rc == DAPQ_OK) rc = check_blocks(pages, blocks, true);
  if (rc == DAPQ_OK) rc = check_step(pages, step);
  if (rc == DAPQ_OK) rc = check_queries(step);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE((int64_t)pages->n_layers * step->total_new * pages->n_kv_heads < (int64_t)1 << 24, DAPQ_ERR_UNSUPPORTED,
               "n_layers * total_new * n_kv_heads (%lld) must be below 2^24", (long long)(pages->n_layers * step->total_new * pages->n_kv_heads));
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
  const int64_t groups = ((most < all ? most : all) + 3) / 4;  // (below 2^24: blocks are below 2^26)
  auto kernel = pages->format == DAPQ_PAGES_BF16 ? paged_bounds_kernel<kBf16> : (pages->format == DAPQ_PAGES_FP4 ? paged_bounds_kernel<kFp4> : paged_bounds_kernel<kE4m3>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)(pages->n_layers * pages->n_kv_heads), (unsigned)pages->batch), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_bounds_kernel");
  return DAPQ_OK;
}

extern "C" DAPQ_API size_t dapq_paged_select_workspace_bytes(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  if (check_select(pages, blocks, step) != DAPQ_OK) return 0;
  const int64_t rows = (int64_t)pages->n_layers * step->total_new * pages->n_kv_heads;
  return align_up((size_t)(rows < 1 ? 1 : rows) * select_plan(pages, blocks, step).stride * sizeof(unsigned), 256);
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
  p.inv_chunks = 1.0f / (float)p.chunks;
  hipLaunchKernelGGL(paged_scores_kernel, dim3((unsigned)((int64_t)p.items * p.batch * p.chunks), (unsigned)plan.col_tiles), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_scores_kernel");
  hipLaunchKernelGGL(paged_choose_kernel, dim3((unsigned)((int64_t)p.items * p.total_new)), dim3(256), 0, static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_choose_kernel");
  return DAPQ_OK;
}
