// Rows into and out of a cache in pages: the rows that an eviction kept (Sec. 4.2, last paragraph), the rows of new tokens with
// their rotation (Sec. 4.1: decoding goes on at position L_p), and back out as bf16.
#include <math.h>

#include "kernel_args.h"
#include "paged.h"
#include "rope_math.h"

namespace dapq {

int check_pages(const dapq_pages* p) {
  DAPQ_REQUIRE(p != nullptr, DAPQ_ERR_INVALID_ARG, "pages is NULL");
  DAPQ_REQUIRE(p->n_layers >= 1 && p->batch >= 1 && p->n_kv_heads >= 1 && p->n_pages >= 1 && p->max_pages >= 1, DAPQ_ERR_INVALID_ARG,
               "n_layers (%d), batch (%d), n_kv_heads (%d), n_pages (%d) and max_pages (%d) of the pages must be >= 1", p->n_layers,
               p->batch, p->n_kv_heads, p->n_pages, p->max_pages);
  DAPQ_REQUIRE(p->head_dim == kHeadDim, DAPQ_ERR_UNSUPPORTED, "head_dim %d is not supported (128 only)", p->head_dim);
  DAPQ_REQUIRE(p->format == DAPQ_PAGES_BF16 || p->format == DAPQ_PAGES_FP4, DAPQ_ERR_INVALID_ARG, "format (%d) is none of DAPQ_PAGES_*",
               p->format);
  DAPQ_REQUIRE(p->page_rows >= 16 && p->page_rows <= 1024 && (p->page_rows & (p->page_rows - 1)) == 0, DAPQ_ERR_UNSUPPORTED,
               "page_rows (%d) must be a power of two from 16 to 1024", p->page_rows);
  DAPQ_REQUIRE((int64_t)p->max_pages * p->page_rows < (int64_t)1 << 30, DAPQ_ERR_UNSUPPORTED,
               "max_pages (%d) * page_rows (%d) must be below 2^30", p->max_pages, p->page_rows);
  DAPQ_REQUIRE((int64_t)p->n_layers * p->n_kv_heads <= 65535, DAPQ_ERR_UNSUPPORTED, "n_layers * n_kv_heads (%lld) of the pages exceeds 65535",
               (long long)p->n_layers * p->n_kv_heads);
  DAPQ_REQUIRE((int64_t)p->n_layers * p->batch * p->n_kv_heads < (int64_t)1 << 24, DAPQ_ERR_UNSUPPORTED,
               "n_layers * batch * n_kv_heads (%lld) of the pages must be below 2^24", (long long)p->n_layers * p->batch * p->n_kv_heads);
  DAPQ_REQUIRE((int64_t)p->n_pages * p->page_rows / 16 <= ((int64_t)0xfffffff0 / ((int64_t)p->n_layers * p->n_kv_heads)), DAPQ_ERR_UNSUPPORTED,
               "n_pages (%d) of page_rows (%d) are more than 2^36 rows of all layers and heads", p->n_pages, p->page_rows);
  DAPQ_REQUIRE(p->k != nullptr && p->v != nullptr && p->table != nullptr, DAPQ_ERR_INVALID_ARG, "k, v and table of the pages must not be NULL");
  uintptr_t bits = reinterpret_cast<uintptr_t>(p->k) | reinterpret_cast<uintptr_t>(p->v);
  if (p->format == DAPQ_PAGES_FP4) {
    DAPQ_REQUIRE(p->k_scales != nullptr && p->v_scales != nullptr, DAPQ_ERR_INVALID_ARG, "FP4 pages need k_scales and v_scales");
    bits |= reinterpret_cast<uintptr_t>(p->k_scales) | reinterpret_cast<uintptr_t>(p->v_scales);
  }
  DAPQ_REQUIRE((bits & 15) == 0, DAPQ_ERR_UNSUPPORTED, "the pools of the pages must be 16-byte aligned");
  return DAPQ_OK;
}

int check_step(const dapq_pages* p, const dapq_step* s) {
  DAPQ_REQUIRE(s != nullptr, DAPQ_ERR_INVALID_ARG, "step is NULL");
  DAPQ_REQUIRE(s->n_q_heads >= 1 && s->n_q_heads % p->n_kv_heads == 0, DAPQ_ERR_INVALID_ARG,
               "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", s->n_q_heads, p->n_kv_heads);
  DAPQ_REQUIRE(s->total_new >= 0 && s->max_new >= 0, DAPQ_ERR_INVALID_ARG, "total_new (%lld) and max_new (%d) must not be negative",
               (long long)s->total_new, s->max_new);
  // (a launch holds fewer than 2^32 threads along an axis)
  DAPQ_REQUIRE(s->total_new <= (int64_t)1 << 25, DAPQ_ERR_UNSUPPORTED, "total_new (%lld) exceeds 2^25", (long long)s->total_new);
  DAPQ_REQUIRE(s->cu_new != nullptr || s->total_new % p->batch == 0, DAPQ_ERR_INVALID_ARG,
               "without cu_new total_new (%lld) must be a multiple of batch (%d)", (long long)s->total_new, p->batch);
  DAPQ_REQUIRE(s->lengths != nullptr, DAPQ_ERR_INVALID_ARG, "lengths of the step must not be NULL");
  return DAPQ_OK;
}

namespace {

// Bytes moved from which rows go past the caches, as dapq_gather's do: us without -> with hints, 983 rows of 32 layers (258 MB) 53.0 -> 46.0 (5.6 TB/s),
// 512 rows of 8 prompts and 32 layers into 4 bits and back out 279 -> 261, 16 sequences of 512..2048 rows, 8 layers, read (1.5 GB) 293 -> 263 (5.8 TB/s).
constexpr int64_t kStreamOut = (int64_t)8 << 20, kStreamIn = (int64_t)192 << 20, kStreamRead = (int64_t)8 << 20;

bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }
bool aligned16(const void* a, const void* b) { return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15) == 0; }

template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned x) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;                               // lanes of a quad
constexpr int kRor1 = 0x121, kRor2 = 0x122, kRor4 = 0x124, kRor8 = 0x128;  // of 16 lanes
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

// STREAM: past the caches.
template <bool STREAM, typename T>
__device__ __forceinline__ void put(T* at, T x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, at);
  else *at = x;
}
template <bool STREAM, typename T>
__device__ __forceinline__ T get(const T* at) {
  if constexpr (STREAM) return __builtin_nontemporal_load(at);
  else return *at;
}

// A row of 16 lanes with 8 channels each into the pool.
template <bool FP4, bool STREAM>
__device__ __forceinline__ void put_row16(uint8_t* rows, uint8_t* scales, int64_t row, int ch, u32x4 x) {
  if constexpr (!FP4) {
    put<STREAM>(reinterpret_cast<u32x4*>(rows + row * kRowBytes + ch * 16), x);
  } else {
    unsigned m = larger(larger(larger_magnitude(x[0]), larger_magnitude(x[1])), larger(larger_magnitude(x[2]), larger_magnitude(x[3])));
    m = larger(m, dpp<kXor1>(m));
    m = larger(m, dpp<kXor2>(m));
    const unsigned s = fp4_scale_byte(m);
    put<STREAM>(reinterpret_cast<unsigned*>(rows + row * kFp4RowBytes + ch * 4), fp4_pack8(x, s));
    unsigned all = s << (8 * (ch >> 2));
    all |= dpp<kRor4>(all);
    all |= dpp<kRor8>(all);
    if (ch == 0) put<STREAM>(reinterpret_cast<unsigned*>(scales + row * 4), all);
  }
}

// ---- dapq_paged_gather --------------------------------------------------------------------------------------------------
struct PagedGatherParams {
  PagePool pool;
  const uint16_t *k, *v;
  const int32_t *idx, *count, *cu_seqlens;
  int64_t k_stride_layer, k_stride_seq, k_stride_head, k_stride_token;
  int64_t v_stride_layer, v_stride_seq, v_stride_head, v_stride_token;
  int32_t batch, budget, seq_len;  // seq_len: dense batches
};

// As gather_kernel, 16 lanes move a row with one 16-byte load each; a lane group has two rows, and K and V of each, whose place is looked up once.
// STREAM_IN, STREAM_OUT: hints of the loads and stores of rows.
template <bool FP4, bool STREAM_IN, bool STREAM_OUT>
__global__ __launch_bounds__(256) void paged_gather_kernel(PagedGatherParams p) {
  touch_args<sizeof(PagedGatherParams)>();
  constexpr int ROWS = 2;
  const int ch = threadIdx.x & 15;
  const int slot0 = blockIdx.x * (16 * ROWS) + (threadIdx.x >> 4);
  const int layer = blockIdx.y / p.pool.n_kv_heads, kv = blockIdx.y - layer * p.pool.n_kv_heads;
  const int seq = blockIdx.z;
  const int64_t head = ((int64_t)layer * p.batch + seq) * p.pool.n_kv_heads + kv;
  const int n = p.count[head] < p.budget ? p.count[head] : p.budget;
  if (slot0 >= n) return;
  int64_t start;
  int L;
  if (p.cu_seqlens == nullptr) {
    L = p.seq_len;
    start = (int64_t)seq * L;
  } else {
    start = p.cu_seqlens[seq];
    L = p.cu_seqlens[seq + 1] - (int)start;
  }
  const uint16_t* k = p.k + layer * p.k_stride_layer + seq * p.k_stride_seq + kv * p.k_stride_head;
  const uint16_t* v = p.v + layer * p.v_stride_layer + seq * p.v_stride_seq + kv * p.v_stride_head;
  int j[ROWS];
  int64_t to[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int slot = slot0 + 16 * r;
    j[r] = slot < n ? p.idx[head * p.budget + slot] : -1;
    to[r] = slot < n ? find_row(p.pool, layer, seq, kv, slot) : -1;
  }
  u32x4 x[ROWS][2];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    x[r][0] = x[r][1] = u32x4{0, 0, 0, 0};
    if (j[r] >= 0 && j[r] < L && to[r] >= 0) {  // (the 16 lanes of a row agree)
      x[r][0] = get<STREAM_IN>(reinterpret_cast<const u32x4*>(k + (start + j[r]) * p.k_stride_token) + ch);
      x[r][1] = get<STREAM_IN>(reinterpret_cast<const u32x4*>(v + (start + j[r]) * p.v_stride_token) + ch);
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (j[r] < 0 || j[r] >= L || to[r] < 0) continue;
    put_row16<FP4, STREAM_OUT>(p.pool.k, p.pool.k_scales, to[r], ch, x[r][0]);
    put_row16<FP4, STREAM_OUT>(p.pool.v, p.pool.v_scales, to[r], ch, x[r][1]);
  }
}

// ---- dapq_paged_append --------------------------------------------------------------------------------------------------
struct PagedAppendParams {
  PagePool pool;
  const uint16_t *k, *v;
  const int32_t *positions, *cu_new, *lengths;
  int64_t k_stride_layer, k_stride_row, k_stride_head;
  int64_t v_stride_layer, v_stride_row, v_stride_head;
  double exponent;  // of rope_angle
  int32_t batch, total_new, each_new, max_new;  // each_new: tokens of a sequence without cu_new
  int32_t pairing, run, k_runs;                 // run: heads of a wave, k_runs: such runs of the keys (then as many of the values)
};

// The sequence of token r and its number there, the same in all lanes; false if the token is none of a sequence's first max_new.
__device__ __forceinline__ bool find_token(const int32_t* cu_new, int batch, int each_new, int max_new, int r, int lane, int* seq, int* t) {
  if (cu_new == nullptr) {
    *seq = r / each_new;
    *t = r - *seq * each_new;
  } else {
    int before = 0, start = 0;  // sequences that end at or before r
    for (int b0 = 0; b0 < batch; b0 += 64) {
      const int end = b0 + lane < batch ? cu_new[b0 + lane + 1] : 0x7fffffff;
      const int n = __popcll(__ballot(end <= r));
      before += n;
      if (n > 0) start = __shfl(end, n - 1, 64);
      if (n < 64) break;
    }
    *seq = before;
    *t = r - start;
    if (before >= batch) return false;
  }
  return *t < max_new;
}

// A wave has one token of one layer and a run of its heads, two at a time, a half wave each: lane c of a half has the channels 2c, 2c + 1
// and 64 + 2c, 65 + 2c, which hold both channels of two pairs in either pairing.  A lane evaluates one angle of the row, in fp64 as
// dapq_rope_apply does, and has the two that it needs from other lanes.
// A small call is a chain of trips to memory (one token, 8 heads 4 us); 10000 tokens of 8 heads take 20 us (4.0 TB/s).
template <bool FP4>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendParams p) {
  touch_args<sizeof(PagedAppendParams)>();
  const int lane = threadIdx.x & 63, c = lane & 31;
  const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int layer = blockIdx.z;
  if (r >= p.total_new) return;
  int seq, t;
  if (!find_token(p.cu_new, p.batch, p.each_new, p.max_new, r, lane, &seq, &t)) return;
  const int64_t row0 = find_row(p.pool, layer, seq, 0, (int64_t)p.lengths[seq] + t);
  if (row0 < 0) return;
  const bool is_v = (int)blockIdx.y >= p.k_runs;
  const int hd0 = (is_v ? blockIdx.y - p.k_runs : blockIdx.y) * p.run;
  const int hd1 = hd0 + p.run < p.pool.n_kv_heads ? hd0 + p.run : p.pool.n_kv_heads;
  const uint16_t* src = is_v ? p.v + layer * p.v_stride_layer + (int64_t)r * p.v_stride_row : p.k + layer * p.k_stride_layer + (int64_t)r * p.k_stride_row;
  const int64_t stride_head = is_v ? p.v_stride_head : p.k_stride_head;
  uint8_t* rows = is_v ? p.pool.v : p.pool.k;
  uint8_t* scales = is_v ? p.pool.v_scales : p.pool.k_scales;
  const bool rotate = !is_v && p.positions != nullptr;
  const int own = lane >> 5;  // of two heads
  auto source = [&](int hd) { return reinterpret_cast<const unsigned*>(src + (int64_t)(hd < hd1 ? hd : hd1 - 1) * stride_head) + c; };
  unsigned a = source(hd0 + own)[0], b = source(hd0 + own)[32];  // (on their way while the angle is evaluated)
  double sn0 = 0, cs0 = 1, sn1 = 0, cs1 = 1;
  if (rotate) {
    double sn, cs;
    rope_angle(p.positions[r], lane, p.exponent, &sn, &cs);
    const int a0 = p.pairing == 0 ? 2 * c : c, a1 = p.pairing == 0 ? 2 * c + 1 : c + 32;
    sn0 = __shfl(sn, a0, 64);
    cs0 = __shfl(cs, a0, 64);
    sn1 = __shfl(sn, a1, 64);
    cs1 = __shfl(cs, a1, 64);
  }
  for (int hd = hd0 + own; hd - own < hd1; hd += 2) {
    const bool mine = hd < hd1;
    const unsigned next_a = source(hd + 2)[0], next_b = source(hd + 2)[32];
    if (rotate) {
      auto lo = [](unsigned x) { return bf16_to_f64((uint16_t)x); };
      auto hi = [](unsigned x) { return bf16_to_f64((uint16_t)(x >> 16)); };
      auto pack = [](double x, double y) { return (unsigned)f64_to_bf16(x) | ((unsigned)f64_to_bf16(y) << 16); };
      const double a0 = lo(a), a1 = hi(a), b0 = lo(b), b1 = hi(b);
      if (p.pairing == 0) {
        a = pack(a0 * cs0 - b0 * sn0, a1 * cs1 - b1 * sn1);
        b = pack(b0 * cs0 + a0 * sn0, b1 * cs1 + a1 * sn1);
      } else {
        a = pack(a0 * cs0 - a1 * sn0, a1 * cs0 + a0 * sn0);
        b = pack(b0 * cs1 - b1 * sn1, b1 * cs1 + b0 * sn1);
      }
    }
    const int64_t row = row0 + ((int64_t)hd << p.pool.page_shift);
    if constexpr (!FP4) {
      if (mine) {
        unsigned* dst = reinterpret_cast<unsigned*>(rows + row * kRowBytes) + c;
        dst[0] = a;
        dst[32] = b;
      }
    } else {
      unsigned ma = larger_magnitude(a), mb = larger_magnitude(b);  // of the 16 lanes that have a group's channels
      ma = larger(ma, dpp<kRor1>(ma)), mb = larger(mb, dpp<kRor1>(mb));
      ma = larger(ma, dpp<kRor2>(ma)), mb = larger(mb, dpp<kRor2>(mb));
      ma = larger(ma, dpp<kRor4>(ma)), mb = larger(mb, dpp<kRor4>(mb));
      ma = larger(ma, dpp<kRor8>(ma)), mb = larger(mb, dpp<kRor8>(mb));
      const unsigned sa = fp4_scale_byte(ma), sb = fp4_scale_byte(mb);
      // a byte of each half of the row to a lane; the four of a quad become a dword
      unsigned ca = sa == kFp4Bad ? 0u : __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, a), fp4_scale(sa), 0);
      unsigned cb = sb == kFp4Bad ? 0u : __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, b), fp4_scale(sb), 0);
      ca = (ca & 255u) << (8 * (c & 3)), cb = (cb & 255u) << (8 * (c & 3));
      ca |= dpp<kXor1>(ca), cb |= dpp<kXor1>(cb);
      ca |= dpp<kXor2>(ca), cb |= dpp<kXor2>(cb);
      if (mine && (c & 3) == 0) {
        unsigned* dst = reinterpret_cast<unsigned*>(rows + row * kFp4RowBytes) + (c >> 2);
        dst[0] = ca;
        dst[8] = cb;
      }
      if (mine && (c & 15) == 0) {
        scales[row * 4 + (c >> 4)] = (uint8_t)sa;
        scales[row * 4 + 2 + (c >> 4)] = (uint8_t)sb;
      }
    }
    a = next_a;
    b = next_b;
  }
}

// ---- dapq_paged_read ----------------------------------------------------------------------------------------------------
struct PagedReadParams {
  PagePool pool;
  const int32_t* lengths;
  uint16_t *k_out, *v_out;
  int32_t batch, max_rows;
};

// 16 lanes to a row, two rows of K and of V to a lane group.
template <bool FP4, bool STREAM>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedReadParams p) {
  touch_args<sizeof(PagedReadParams)>();
  constexpr int ROWS = 2;
  const int ch = threadIdx.x & 15;
  const int layer = blockIdx.y / p.pool.n_kv_heads, kv = blockIdx.y - layer * p.pool.n_kv_heads;
  const int seq = blockIdx.z;
  const int i0 = blockIdx.x * (16 * ROWS) + (threadIdx.x >> 4);
  const int n = p.lengths[seq] < p.max_rows ? p.lengths[seq] : p.max_rows;
  if (i0 >= n) return;
  const int64_t out = ((((int64_t)layer * p.batch + seq) * p.pool.n_kv_heads + kv) * p.max_rows + i0) * kHeadDim + ch * 8;
  int64_t row[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) row[r] = i0 + 16 * r < n ? find_row(p.pool, layer, seq, kv, i0 + 16 * r) : -1;
  u32x4 x[ROWS][2];
  unsigned scale[ROWS][2];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (row[r] < 0) continue;
    if constexpr (FP4) {
      x[r][0][0] = *reinterpret_cast<const unsigned*>(p.pool.k + row[r] * kFp4RowBytes + ch * 4);
      x[r][1][0] = *reinterpret_cast<const unsigned*>(p.pool.v + row[r] * kFp4RowBytes + ch * 4);
      scale[r][0] = p.pool.k_scales[row[r] * 4 + (ch >> 2)];
      scale[r][1] = p.pool.v_scales[row[r] * 4 + (ch >> 2)];
    } else {
      x[r][0] = get<STREAM>(reinterpret_cast<const u32x4*>(p.pool.k + row[r] * kRowBytes + ch * 16));
      x[r][1] = get<STREAM>(reinterpret_cast<const u32x4*>(p.pool.v + row[r] * kRowBytes + ch * 16));
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (row[r] < 0) continue;
    if constexpr (FP4) {
      x[r][0] = fp4_unpack8(x[r][0][0], fp4_scale(scale[r][0]));
      x[r][1] = fp4_unpack8(x[r][1][0], fp4_scale(scale[r][1]));
    }
    put<STREAM>(reinterpret_cast<u32x4*>(p.k_out + out + 16 * r * kHeadDim), x[r][0]);
    put<STREAM>(reinterpret_cast<u32x4*>(p.v_out + out + 16 * r * kHeadDim), x[r][1]);
  }
}

}  // namespace
}  // namespace dapq

using namespace dapq;

extern "C" DAPQ_API int dapq_paged_gather(const dapq_shape* shape, const dapq_pages* pages, const void* k, const void* v, const int32_t* idx,
                                          const int32_t* count, int32_t budget, void* stream) {
  int rc = check_shape(shape, false, true, true);
  if (rc == DAPQ_OK) rc = check_pages(pages);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(shape->n_layers == pages->n_layers && shape->batch == pages->batch && shape->n_kv_heads == pages->n_kv_heads, DAPQ_ERR_INVALID_ARG,
               "layers, batch and KV heads of shape (%d, %d, %d) and pages (%d, %d, %d) differ", shape->n_layers, shape->batch, shape->n_kv_heads,
               pages->n_layers, pages->batch, pages->n_kv_heads);
  DAPQ_REQUIRE(k != nullptr && v != nullptr && idx != nullptr && count != nullptr, DAPQ_ERR_INVALID_ARG, "k, v, idx and count must not be NULL");
  DAPQ_REQUIRE(budget >= 1, DAPQ_ERR_INVALID_ARG, "budget (%d) must be >= 1", budget);
  DAPQ_REQUIRE(aligned16(k, v), DAPQ_ERR_UNSUPPORTED, "k and v must be 16-byte aligned");
  PagedGatherParams p;
  p.pool = page_pool(pages);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.idx = idx;
  p.count = count;
  p.cu_seqlens = shape->cu_seqlens;
  p.k_stride_layer = shape->k_stride_layer; p.k_stride_seq = shape->k_stride_seq;
  p.k_stride_head = shape->k_stride_head; p.k_stride_token = shape->k_stride_token;
  p.v_stride_layer = shape->v_stride_layer; p.v_stride_seq = shape->v_stride_seq;
  p.v_stride_head = shape->v_stride_head; p.v_stride_token = shape->v_stride_token;
  p.batch = shape->batch;
  p.budget = budget;
  p.seq_len = (int32_t)(shape->total_tokens / shape->batch);
  DAPQ_REQUIRE(shape->batch <= 65535, DAPQ_ERR_UNSUPPORTED, "batch (%d) exceeds 65535", shape->batch);
  // no more rows than the table has a place for
  const int64_t rows = (int64_t)pages->max_pages * pages->page_rows;
  const unsigned blocks = (unsigned)(((budget < rows ? budget : rows) + 31) / 32);
  // bytes read and written where every head keeps its whole budget
  const int64_t moved = (int64_t)shape->n_layers * shape->batch * shape->n_kv_heads * (budget < rows ? budget : rows) * 2 *
                        (kRowBytes + (pages->format == DAPQ_PAGES_FP4 ? kFp4RowBytes + 4 : kRowBytes));
  DAPQ_REQUIRE((uint64_t)blocks * 256 < (uint64_t)1 << 32, DAPQ_ERR_UNSUPPORTED, "budget (%d) is too large", budget);
  const bool fp4 = pages->format == DAPQ_PAGES_FP4;
  auto kernel = fp4 ? paged_gather_kernel<true, false, false> : paged_gather_kernel<false, false, false>;
  if (moved >= kStreamOut) kernel = fp4 ? paged_gather_kernel<true, false, true> : paged_gather_kernel<false, false, true>;
  if (moved >= kStreamIn) kernel = fp4 ? paged_gather_kernel<true, true, true> : paged_gather_kernel<false, true, true>;
  hipLaunchKernelGGL(kernel, dim3(blocks, (unsigned)(shape->n_layers * shape->n_kv_heads), (unsigned)shape->batch), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_gather_kernel");
  return DAPQ_OK;
}

extern "C" DAPQ_API int dapq_paged_append(const dapq_pages* pages, const dapq_step* step, const void* k_new, const void* v_new,
                                          const int32_t* positions, double theta, int32_t pairing, void* stream) {
  int rc = check_pages(pages);
  if (rc == DAPQ_OK) rc = check_step(pages, step);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(k_new != nullptr && v_new != nullptr, DAPQ_ERR_INVALID_ARG, "k_new and v_new must not be NULL");
  if (positions != nullptr) {
    DAPQ_REQUIRE(pairing == 0 || pairing == 1, DAPQ_ERR_INVALID_ARG, "pairing must be 0 (half) or 1 (interleaved)");
    DAPQ_REQUIRE(theta > 0.0 && isfinite(theta), DAPQ_ERR_INVALID_ARG, "theta must be finite and > 0");
  }
  DAPQ_REQUIRE(aligned16(k_new, v_new), DAPQ_ERR_UNSUPPORTED, "k_new and v_new must be 16-byte aligned");
  DAPQ_REQUIRE(stride_ok(step->k_stride_layer) && stride_ok(step->k_stride_row) && stride_ok(step->k_stride_head) && step->k_stride_row >= kHeadDim,
               DAPQ_ERR_UNSUPPORTED, "k strides of the step must be non-negative multiples of 8 elements (row >= 128)");
  DAPQ_REQUIRE(stride_ok(step->v_stride_layer) && stride_ok(step->v_stride_row) && stride_ok(step->v_stride_head) && step->v_stride_row >= kHeadDim,
               DAPQ_ERR_UNSUPPORTED, "v strides of the step must be non-negative multiples of 8 elements (row >= 128)");
  if (step->total_new == 0 || step->max_new == 0) return DAPQ_OK;
  PagedAppendParams p;
  p.pool = page_pool(pages);
  p.k = static_cast<const uint16_t*>(k_new);
  p.v = static_cast<const uint16_t*>(v_new);
  p.positions = positions;
  p.cu_new = step->cu_new;
  p.lengths = step->lengths;
  p.k_stride_layer = step->k_stride_layer; p.k_stride_row = step->k_stride_row; p.k_stride_head = step->k_stride_head;
  p.v_stride_layer = step->v_stride_layer; p.v_stride_row = step->v_stride_row; p.v_stride_head = step->v_stride_head;
  p.exponent = positions != nullptr ? rope_exponent(theta, kHeadDim) : 0.0;
  p.batch = pages->batch;
  p.total_new = (int32_t)step->total_new;
  p.each_new = (int32_t)(step->total_new / pages->batch);
  p.max_new = step->max_new;
  p.pairing = pairing;
  // Heads of a wave: the angles of a row are worth sharing, but a small call wants a wave for every two heads (64 tokens, 8 heads, in 4 bits with reading
  // back: 11.0 us in runs of eight, 9.8 in runs of two).
  p.run = 2;
  while (p.run < 32 && p.run < pages->n_kv_heads && step->total_new * pages->n_layers * ((pages->n_kv_heads + 2 * p.run - 1) / (2 * p.run)) >= 2048) p.run *= 2;
  p.k_runs = (pages->n_kv_heads + p.run - 1) / p.run;
  hipLaunchKernelGGL(pages->format == DAPQ_PAGES_FP4 ? paged_append_kernel<true> : paged_append_kernel<false>,
                     dim3((unsigned)((step->total_new + 3) / 4), (unsigned)(2 * p.k_runs), (unsigned)pages->n_layers), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_append_kernel");
  return DAPQ_OK;
}

extern "C" DAPQ_API int dapq_paged_read(const dapq_pages* pages, const int32_t* lengths, int32_t max_rows, void* k_out, void* v_out, void* stream) {
  int rc = check_pages(pages);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(lengths != nullptr && k_out != nullptr && v_out != nullptr, DAPQ_ERR_INVALID_ARG, "lengths, k_out and v_out must not be NULL");
  DAPQ_REQUIRE(max_rows >= 1, DAPQ_ERR_INVALID_ARG, "max_rows (%d) must be >= 1", max_rows);
  DAPQ_REQUIRE(aligned16(k_out, v_out), DAPQ_ERR_UNSUPPORTED, "k_out and v_out must be 16-byte aligned");
  DAPQ_REQUIRE(pages->batch <= 65535, DAPQ_ERR_UNSUPPORTED, "batch (%d) exceeds 65535", pages->batch);
  PagedReadParams p;
  p.pool = page_pool(pages);
  p.lengths = lengths;
  p.k_out = static_cast<uint16_t*>(k_out);
  p.v_out = static_cast<uint16_t*>(v_out);
  p.batch = pages->batch;
  p.max_rows = max_rows;
  const int64_t rows = (int64_t)pages->max_pages * pages->page_rows;  // (below 2^30: 2^33 threads would be too many)
  const uint64_t blocks = (uint64_t)(((max_rows < rows ? max_rows : rows) + 31) / 32);
  DAPQ_REQUIRE(blocks * 256 < (uint64_t)1 << 32, DAPQ_ERR_UNSUPPORTED, "max_rows (%d) is too large", max_rows);
  const int64_t moved = (int64_t)pages->n_layers * pages->batch * pages->n_kv_heads * (max_rows < rows ? max_rows : rows) * 2 *
                        (kRowBytes + (pages->format == DAPQ_PAGES_FP4 ? kFp4RowBytes + 4 : kRowBytes));
  auto kernel = pages->format == DAPQ_PAGES_FP4 ? (moved >= kStreamRead ? paged_read_kernel<true, true> : paged_read_kernel<true, false>)
                                                : (moved >= kStreamRead ? paged_read_kernel<false, true> : paged_read_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, (unsigned)(pages->n_layers * pages->n_kv_heads), (unsigned)pages->batch), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_read_kernel");
  return DAPQ_OK;
}
