// Attention of a step's tokens over a cache in pages.
#include <math.h>

#include "paged.h"

namespace dapq {
namespace {

struct PagedAttentionParams {
  PagePool pool;
  const uint16_t* q;
  uint16_t* out;
  const int32_t *cu_new, *lengths;
  int64_t q_stride_layer, q_stride_row, q_stride_head;
  int32_t batch, total_new, each_new, max_new, n_q_heads;
  float scale, softcap;
};

// A wave to a token and query head: the logits of 64 rows at a time, one to a lane, then their values, two channels to a lane.
template <bool FP4>
__global__ __launch_bounds__(64) void paged_attention_kernel(PagedAttentionParams p) {
  __shared__ float q[kHeadDim];
  const int lane = threadIdx.x, r = blockIdx.x, h = blockIdx.y, layer = blockIdx.z;
  const int kv = h / (p.n_q_heads / p.pool.n_kv_heads);
  int seq = 0, start = 0;
  if (p.cu_new == nullptr) {
    seq = r / p.each_new;
    start = seq * p.each_new;
  } else {
    while (seq < p.batch && p.cu_new[seq + 1] <= r) ++seq;
    if (seq >= p.batch) return;
    start = p.cu_new[seq];
  }
  if (r - start >= p.max_new) return;
  const int64_t most = (int64_t)p.pool.max_pages << p.pool.page_shift;
  const int64_t seen = (int64_t)p.lengths[seq] + (r - start) + 1;
  const int visible = (int)(seen < most ? seen : most);
  const uint16_t* src = p.q + layer * p.q_stride_layer + (int64_t)r * p.q_stride_row + h * p.q_stride_head;
  q[lane] = __uint_as_float((unsigned)src[lane] << 16);
  q[lane + 64] = __uint_as_float((unsigned)src[lane + 64] << 16);
  __syncthreads();
  auto value = [&](const uint8_t* rows, const uint8_t* scales, int64_t row, int c8) {
    if constexpr (FP4) return fp4_unpack8(*reinterpret_cast<const unsigned*>(rows + row * kFp4RowBytes + c8 * 4), fp4_scale(scales[row * 4 + (c8 >> 2)]));
    else return *reinterpret_cast<const u32x4*>(rows + row * kRowBytes + c8 * 16);
  };
  float m = -INFINITY, sum = 0.0f, o[2] = {0.0f, 0.0f};
  for (int i0 = 0; i0 < visible; i0 += 64) {
    const int64_t row = i0 + lane < visible ? find_row(p.pool, layer, seq, kv, i0 + lane) : -1;
    float x = -INFINITY;
    if (row >= 0) {
      x = 0.0f;
      for (int c8 = 0; c8 < 16; ++c8) {
        const u32x4 k = value(p.pool.k, p.pool.k_scales, row, c8);
        for (int i = 0; i < 4; ++i) {
          x = fmaf(q[8 * c8 + 2 * i], __uint_as_float(k[i] << 16), x);
          x = fmaf(q[8 * c8 + 2 * i + 1], __uint_as_float(k[i] & 0xffff0000u), x);
        }
      }
      x *= p.scale;
      if (p.softcap > 0.0f) x = p.softcap * tanhf(x / p.softcap);
    }
    float top = x;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    if (__ballot(row >= 0) == 0) continue;
    const float moved = fmaxf(fmaxf(m, top), -3.4028234663852886e38f);
    const float f = expf(m - moved);
    m = moved;
    const float w = row >= 0 ? expf(x - m) : 0.0f;
    float s = w;
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    sum = sum * f + s;
    o[0] *= f;
    o[1] *= f;
    for (int j = 0; j < 64; ++j) {
      const int64_t rj = __shfl(row, j, 64);
      const float wj = __shfl(w, j, 64);
      if (rj < 0) continue;
      const u32x4 v = value(p.pool.v, p.pool.v_scales, rj, lane >> 2);
      const unsigned u = v[lane & 3];
      o[0] = fmaf(wj, __uint_as_float(u << 16), o[0]);
      o[1] = fmaf(wj, __uint_as_float(u & 0xffff0000u), o[1]);
    }
  }
  const bool none = m == -INFINITY;  // no visible row is on a page
  bf16x2 result;
  result[0] = (__bf16)(none ? 0.0f : o[0] / sum);
  result[1] = (__bf16)(none ? 0.0f : o[1] / sum);
  *reinterpret_cast<bf16x2*>(p.out + (((int64_t)layer * p.total_new + r) * p.n_q_heads + h) * kHeadDim + 2 * lane) = result;
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
  DAPQ_REQUIRE(step->n_q_heads <= 65535, DAPQ_ERR_UNSUPPORTED, "n_q_heads (%d) exceeds 65535", step->n_q_heads);
  return DAPQ_OK;
}

}  // namespace
}  // namespace dapq

using namespace dapq;

extern "C" DAPQ_API size_t dapq_paged_attention_workspace_bytes(const dapq_pages* pages, const dapq_step* step) {
  return check_attention(pages, step) == DAPQ_OK ? 256 : 0;
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
  p.max_new = step->max_new;
  p.n_q_heads = step->n_q_heads;
  p.scale = step->scale;
  p.softcap = step->softcap;
  hipLaunchKernelGGL(pages->format == DAPQ_PAGES_FP4 ? paged_attention_kernel<true> : paged_attention_kernel<false>,
                     dim3((unsigned)step->total_new, (unsigned)step->n_q_heads, (unsigned)pages->n_layers), dim3(64), 0,
                     static_cast<hipStream_t>(stream), p);
  DAPQ_HIP_LAUNCH_CHECK("paged_attention_kernel");
  return DAPQ_OK;
}
