// What the kernels of paged attention share: a step's tokens, what they see, capped scores.
#pragma once

#include <math.h>

#include "kernel_args.h"
#include "paged.h"

namespace dapq {

struct PagedAttentionParams {
  PagePool pool;
  const uint16_t* q;
  uint16_t* out;
  const int32_t *cu_new, *lengths;
  int64_t q_stride_layer, q_stride_row, q_stride_head;
  float* parts;  // of the workspace
  int32_t batch, total_new, each_new, max_new, n_q_heads;
  int32_t group, items, groups, spare;  // query heads of a KV head; layers * Hkv; of the row kernel: workgroups, and those that items leave
  float inv_group, inv_items, inv_spare;
  float c, cap;       // c: scale * log2(e), with a cap scale / softcap; cap: softcap * log2(e)
};

// New tokens of a sequence, at most.
inline int32_t most_new(const dapq_pages* pages, const dapq_step* step) {
  const int64_t n = step->cu_new == nullptr ? step->total_new / pages->batch : step->total_new;
  return (int32_t)(step->max_new < n ? step->max_new : n);
}

// The columns (new tokens x query heads of a KV head) that the row kernel takes, two blocks of 16: it reads a row in place, where the turn kernel passes it through
// LDS and has 128 columns to a workgroup, used or not.  Us, row / turn kernel, 8 KV heads, 32 columns: 1 sequence of 1000 rows 14.8 / 14.1, of 100000 84.6 / 96.2, 32 of 4000
// 108.5 / 106.3, 64 of 1000 54.3 / 52.6; in 4 bits 16.3 / 14.6, 40.3 / 72.8, 45.4 / 74.0, 24.4 / 35.8.  4 columns: 11.8 / 13.4, 82.9 / 94.7, 97.9 / 100.6, 48.4 / 50.9; in 4 bits
// 9.2 / 14.1, 31.3 / 70.6, 36.4 / 69.6, 14.6 / 34.4.
constexpr int kMostRowCols = 32;
// Checks that the calls of attention share, and the parameters of their kernels (host).
int check_queries(const dapq_step* step);
int check_attention(const dapq_pages* pages, const dapq_step* step);
int check_buffers(const void* q, const void* out);
int check_workspace(const void* workspace, size_t bytes, size_t need);
PagedAttentionParams attention_params(const dapq_pages* pages, const dapq_step* step, const void* q, void* out, void* workspace);
size_t turn_workspace_bytes(const dapq_pages* pages, const dapq_step* step);
int launch_turn(const dapq_pages* pages, const dapq_step* step, const PagedAttentionParams& p, hipStream_t stream);

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kHeadroom = 4.0f;      // binades that a logit may lie above the reference of its column
constexpr float kLowest = -3.4028234663852886e38f;  // where references start: finite, a logit of -inf then weighs 0
constexpr float kLog2e = 1.4426950408889634f;

// A value that the compiler can't trace: what is computed from it inside a loop is not kept in registers around the loop.
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// The rows that token t sees.
__device__ __forceinline__ int rows_seen(const PagedAttentionParams& p, int before, int t) {
  const int64_t most = (int64_t)p.pool.max_pages << p.pool.page_shift, n = (int64_t)before + t + 1;
  return (int)(n < 0 ? 0 : (n < most ? n : most));
}
// The bits of those of the two bf16 of a dword that are infinite or no number.
__device__ __forceinline__ unsigned infinite_bits(unsigned x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// log2 of a weight before the reference is taken off: c * logit, or with a cap cap * log2(e) * tanh(logit * scale / cap), where
// tanh(z) = 1 - 2 / (1 + exp(2 z)) is off by some 2^-22.  Up to a cap of 64 that is an error of a score below 2^-16, as much as the
// dot product's own; with a larger cap scores below a quarter of it take the series instead, whose first term left out is below 2^-22 z.
// (The series costs: eight turns with a cap of 65 594 us, with one of 50 490.)
enum Cap { kNoCap, kSmallCap, kLargeCap };
constexpr float kMostSmallCap = 64.0f;
template <int CAP>
__device__ __forceinline__ float capped(const PagedAttentionParams& p, float d) {
  if constexpr (CAP == kNoCap) return d;  // (times p.c where it is used)
  const float z = d * p.c;
  const float big = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * (2.0f * kLog2e))), 1.0f);
  if constexpr (CAP == kSmallCap) return p.cap * big;
  const float u = z * z;
  const float small = z * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  return p.cap * (fabsf(z) < 0.25f ? small : big);
}
inline Cap cap_of(const PagedAttentionParams& p) { return !(p.cap > 0.0f) ? kNoCap : (p.cap <= kMostSmallCap * kLog2e ? kSmallCap : kLargeCap); }

}  // namespace
}  // namespace dapq
