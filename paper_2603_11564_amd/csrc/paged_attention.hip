// Attention of a step's tokens over a cache in pages.
#include "paged_rows.h"

namespace dapq {
namespace {

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
  // (In 8 bits an item alone takes 0.19 a tile, but then 16 x 4000 would be items.)  In 8 bits 1 x 1000 10.9 / 10.7, 1 x 2000 10.8 / 16.7, 4 x 1000 12.3 / 10.8, 8 x 2000 15.9 / 18.0, 16 x 2000 20.5 / 18.3, 16 x 4000 30.7 / 35.7, 31 x 2000 28.1 / 22.4.
  const bool fp4 = p->format == DAPQ_PAGES_FP4, e4m3 = p->format == DAPQ_PAGES_E4M3;
  const double tile = fp4 ? 0.16 : (e4m3 ? 0.22 : 0.27), bytes = (fp4 ? 4352 : (e4m3 ? 8448 : 16384)) / 6.5e6, join = fp4 ? 6.5 : (e4m3 ? 6.0 : 5.5);
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
  constexpr int kCols = BLOCKS == 0 ? 8 : 16 * BLOCKS, kBytes = kRowLds<BLOCKS>;
  const Cap cap = cap_of(p);
  auto kernel = cap == kNoCap ? paged_rows_kernel<FMT, BLOCKS, kNoCap, SPLIT, false>
                              : (cap == kSmallCap ? paged_rows_kernel<FMT, BLOCKS, kSmallCap, SPLIT, false> : paged_rows_kernel<FMT, BLOCKS, kLargeCap, SPLIT, false>);
  const int rc = set_max_dynamic_lds(reinterpret_cast<const void*>(kernel), kBytes);
  if (rc != DAPQ_OK) return rc;
  const unsigned items = (unsigned)(pages->batch * p.items);  // (below 2^24)
  hipLaunchKernelGGL(kernel, dim3(SPLIT ? (unsigned)p.groups : items), dim3(64 * kRowWaves), kBytes, stream, p);
  DAPQ_HIP_LAUNCH_CHECK("paged_rows_kernel");
  if (SPLIT) {
    const unsigned cols = (unsigned)(p.max_new * p.group);
    if (items < 128) hipLaunchKernelGGL((paged_join_kernel<kCols, kJoinWaves, false>), dim3(items, cols), dim3(64 * kJoinWaves), 0, stream, p);
    else hipLaunchKernelGGL((paged_join_kernel<kCols, 1, false>), dim3(items, (cols + kJoinWaves - 1) / kJoinWaves), dim3(64 * kJoinWaves), 0, stream, p);
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

}  // namespace

int check_attention(const dapq_pages* pages, const dapq_step* step) {
  int rc = check_pages(pages);
  if (rc == DAPQ_OK) rc = check_step(pages, step);
  if (rc != DAPQ_OK) return rc;
  rc = check_queries(step);
  if (rc != DAPQ_OK) return rc;
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

int check_queries(const dapq_step* step) {
  auto stride_ok = [](int64_t s) { return s >= 0 && s % 8 == 0; };
  DAPQ_REQUIRE(stride_ok(step->q_stride_layer) && stride_ok(step->q_stride_row) && stride_ok(step->q_stride_head) && step->q_stride_row >= kHeadDim,
               DAPQ_ERR_UNSUPPORTED, "q strides of the step must be non-negative multiples of 8 elements (row >= 128)");
  return DAPQ_OK;
}

int check_buffers(const void* q, const void* out) {
  DAPQ_REQUIRE(q != nullptr && out != nullptr, DAPQ_ERR_INVALID_ARG, "q and out must not be NULL");
  DAPQ_REQUIRE(((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) == 0, DAPQ_ERR_UNSUPPORTED,
               "q and out must be 16-byte aligned");
  return DAPQ_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  DAPQ_REQUIRE(workspace != nullptr, DAPQ_ERR_INVALID_ARG, "workspace is NULL");
  DAPQ_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255) == 0, DAPQ_ERR_UNSUPPORTED, "workspace is not 256-byte aligned");
  DAPQ_REQUIRE(bytes >= need, DAPQ_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", bytes, need);
  return DAPQ_OK;
}

PagedAttentionParams attention_params(const dapq_pages* pages, const dapq_step* step, const void* q, void* out, void* workspace) {
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
  return p;
}

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
  int rc = check_attention(pages, step);
  if (rc != DAPQ_OK) return rc;
  rc = check_buffers(q, out);
  if (rc != DAPQ_OK) return rc;
  if (step->total_new == 0 || step->max_new == 0) return DAPQ_OK;
  rc = check_workspace(workspace, workspace_bytes, dapq_paged_attention_workspace_bytes(pages, step));
  if (rc != DAPQ_OK) return rc;
  const PagedAttentionParams p = attention_params(pages, step, q, out, workspace);
  const int64_t cols = (int64_t)p.max_new * p.group;
  if (cols <= kMostRowCols) return launch_rows(pages, p, row_cols(cols), static_cast<hipStream_t>(stream));
  return launch_turn(pages, step, p, static_cast<hipStream_t>(stream));
}
