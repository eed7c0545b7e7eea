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
  int32_t group, items, groups, least_share;  // query heads of a KV head; layers * Hkv; workgroups of the row kernel; fewest tiles of one
  float inv_group, inv_items, inv_groups;
  float c, cap;       // c: scale * log2(e), with a cap scale / softcap; cap: softcap * log2(e)
};

// The call with more columns (new tokens x query heads of a KV head) than the row kernel takes.
constexpr int kMostRowCols = 32;
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

// log2 of a weight before the reference is taken off: c * logit, or with a cap cap * log2(e) * tanh(logit * scale / cap).
template <bool CAP>
__device__ __forceinline__ float capped(const PagedAttentionParams& p, float d) {
  if constexpr (!CAP) return d;  // (times p.c where it is used)
  // tanh(z) = 1 - 2 / (1 + exp(2 z)) loses what z is smaller than 1 by: below 1/4 the series, whose first term left out is below 2^-22 z
  const float z = d * p.c;
  const float big = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * (2.0f * kLog2e))), 1.0f);
  const float u = z * z;
  const float small = z * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  return p.cap * (fabsf(z) < 0.25f ? small : big);
}

}  // namespace
}  // namespace dapq
