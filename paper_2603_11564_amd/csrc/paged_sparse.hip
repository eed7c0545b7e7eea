// Attention of a step's tokens over chosen blocks of a cache in pages.
#include "paged_blocks.h"
#include "paged_rows.h"

namespace dapq {
namespace {

// How a call is run: a function of the descriptors alone, which the workspace follows.  Other than lengths, the rows of an item are known here: no more
// than n_select blocks.
struct SparsePlan {
  int cols, chunks;  // columns of the kernel, and how many such runs of a token's query heads there are
  int64_t items;
  int parts, tiles;
};
int64_t resident_workgroups(const SparsePlan& plan) { return plan.cols == 32 ? 512 : 768; }
SparsePlan sparse_plan(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  SparsePlan plan;
  const int group = step->n_q_heads / pages->n_kv_heads;
  plan.cols = row_cols(group);
  plan.chunks = (group + plan.cols - 1) / plan.cols;
  plan.items = (int64_t)pages->n_layers * step->total_new * pages->n_kv_heads;
  const int64_t all = most_blocks(pages, blocks), rows = (blocks->n_select < all ? blocks->n_select : all) * blocks->block_rows;
  const int64_t tiles = (rows + kTile - 1) / kTile;
  plan.tiles = (int)tiles;  // (up to 2^17: parts_each times it stays below 2^31)
  // Parts for as many workgroups as the chip holds at once, but of no fewer tiles than a workgroup has waves.  8 KV heads of one token, us with parts of
  // 2 / 4 / 8 tiles at least: 2048 rows of 4 query heads 9.8 / 9.3 / 10.5, of 8 query heads 10.2 / 10.2 / 11.4, 4096 rows 12.7 / 10.9 / 12.0.
  const int64_t resident = resident_workgroups(plan), items = plan.items * plan.chunks;
  int64_t parts = items > 0 ? resident / items : 1;
  if (parts > tiles / kRowWaves) parts = tiles / kRowWaves;
  plan.parts = (int)(parts < 1 ? 1 : parts);
  return plan;
}

template <int FMT, int BLOCKS, bool SPLIT>
int launch_sparse(const SparseParams& p, const SparsePlan& plan, hipStream_t stream) {
  constexpr int kCols = BLOCKS == 0 ? 8 : 16 * BLOCKS, kBytes = kRowLds<BLOCKS>;
  const Cap cap = cap_of(p);
  auto kernel = cap == kNoCap ? paged_rows_kernel<FMT, BLOCKS, kNoCap, SPLIT, true>
                              : (cap == kSmallCap ? paged_rows_kernel<FMT, BLOCKS, kSmallCap, SPLIT, true> : paged_rows_kernel<FMT, BLOCKS, kLargeCap, SPLIT, true>);
  const int rc = set_max_dynamic_lds(reinterpret_cast<const void*>(kernel), kBytes);
  if (rc != DAPQ_OK) return rc;
  hipLaunchKernelGGL(kernel, dim3((unsigned)plan.items, (unsigned)plan.parts, (unsigned)plan.chunks), dim3(64 * kRowWaves), kBytes, stream, p);
  DAPQ_HIP_LAUNCH_CHECK("paged_rows_kernel");
  if (SPLIT) {
    const unsigned cols = (unsigned)(p.group < kCols ? p.group : kCols);
    // Up to 16 parts (always so with 128 items, which leave 6 to each) are joined by a wave, whose first 16 lanes hold their weights.  More take eight waves:
    // 8 KV heads, us, one wave / eight, 32 parts 16.7 / 10.4, 96 parts 44 / 21.
    if (plan.parts > 16) hipLaunchKernelGGL((paged_join_kernel<kCols, kJoinWaves, true>), dim3((unsigned)plan.items, cols, (unsigned)plan.chunks), dim3(64 * kJoinWaves), 0, stream, p);
    else hipLaunchKernelGGL((paged_join_kernel<kCols, 1, true, 16>), dim3((unsigned)plan.items, (cols + kJoinWaves - 1) / kJoinWaves, (unsigned)plan.chunks), dim3(64 * kJoinWaves), 0, stream, p);
    DAPQ_HIP_LAUNCH_CHECK("paged_join_kernel");
  }
  return DAPQ_OK;
}
template <int FMT, int BLOCKS>
int launch_sparse(const SparseParams& p, const SparsePlan& plan, hipStream_t stream) {
  return plan.parts > 1 ? launch_sparse<FMT, BLOCKS, true>(p, plan, stream) : launch_sparse<FMT, BLOCKS, false>(p, plan, stream);
}
template <int FMT>
int launch_sparse(const SparseParams& p, const SparsePlan& plan, hipStream_t stream) {
  return plan.cols == 8 ? launch_sparse<FMT, 0>(p, plan, stream) : (plan.cols == 16 ? launch_sparse<FMT, 1>(p, plan, stream) : launch_sparse<FMT, 2>(p, plan, stream));
}

int check_sparse(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  int rc = check_attention(pages, step);
  if (rc == DAPQ_OK) rc = check_blocks(pages, blocks, false);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE((int64_t)pages->n_layers * step->total_new * pages->n_kv_heads < (int64_t)1 << 23, DAPQ_ERR_UNSUPPORTED,
               "n_layers * total_new * n_kv_heads (%lld) must be below 2^23", (long long)(pages->n_layers * step->total_new * pages->n_kv_heads));
  return DAPQ_OK;
}

}  // namespace
}  // namespace dapq

using namespace dapq;

extern "C" DAPQ_API size_t dapq_paged_sparse_attention_workspace_bytes(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step) {
  if (check_sparse(pages, blocks, step) != DAPQ_OK) return 0;
  // Enough for every smaller step as well, which may share out its items where this one has enough of them.
  const SparsePlan plan = sparse_plan(pages, blocks, step);
  const int64_t parts_each = plan.tiles / kRowWaves, most = plan.items * plan.chunks * parts_each, resident = resident_workgroups(plan);
  return parts_each > 1 ? align_up((size_t)(most < resident ? most : resident) * plan.cols * (kHeadDim + 2) * sizeof(float), 256) : 256;
}

extern "C" DAPQ_API int dapq_paged_sparse_attention(const dapq_pages* pages, const dapq_blocks* blocks, const dapq_step* step, const void* q, const int32_t* idx,
                                                    const int32_t* count, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_sparse(pages, blocks, step);
  if (rc != DAPQ_OK) return rc;
  DAPQ_REQUIRE(idx != nullptr && count != nullptr, DAPQ_ERR_INVALID_ARG, "idx and count must not be NULL");
  rc = check_buffers(q, out);
  if (rc != DAPQ_OK) return rc;
  if (step->total_new == 0 || step->max_new == 0) return DAPQ_OK;
  rc = check_workspace(workspace, workspace_bytes, dapq_paged_sparse_attention_workspace_bytes(pages, blocks, step));
  if (rc != DAPQ_OK) return rc;
  SparseParams p;
  static_cast<PagedAttentionParams&>(p) = attention_params(pages, step, q, out, workspace);
  p.idx = idx;
  p.count = count;
  p.block_shift = __builtin_ctz((unsigned)blocks->block_rows);
  p.n_select = blocks->n_select;
  const SparsePlan plan = sparse_plan(pages, blocks, step);
  p.parts_each = plan.parts;
  p.most_tiles = plan.tiles;
  const hipStream_t on = static_cast<hipStream_t>(stream);
  return pages->format == DAPQ_PAGES_BF16 ? launch_sparse<kBf16>(p, plan, on) : (pages->format == DAPQ_PAGES_FP4 ? launch_sparse<kFp4>(p, plan, on) : launch_sparse<kE4m3>(p, plan, on));
}
