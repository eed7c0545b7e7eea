// Blocks of a cache in pages, as the calls that choose them and those that read them share them.
#pragma once

#include "paged.h"

namespace dapq {

// Checks of the blocks' descriptor (host).  need_bounds: the call reads or writes bounds and scales.
int check_blocks(const dapq_pages* p, const dapq_blocks* b, bool need_bounds);
// Blocks that the table has room for.
inline int64_t most_blocks(const dapq_pages* p, const dapq_blocks* b) { return (int64_t)p->max_pages * p->page_rows / b->block_rows; }

namespace {

// Whole numbers of 8 bits in units of a power of two: the byte e + 127 of the least e in [-50, 50] with max <= 127 * 2^e, from the largest magnitude
// (the bits of a finite non-negative bf16).  max = (1 + m / 128) * 2^x, and 127 * 2^e = (1 + 126 / 128) * 2^(e + 6): e is x - 6, or x - 5 if m is 127.
constexpr int kLeastUnit = 127 - 50, kMostUnit = 127 + 50;
__device__ __forceinline__ int unit_byte(unsigned largest) {
  const int s = (int)((largest + 1) >> 7) - 6;
  return s < kLeastUnit ? kLeastUnit : (s > kMostUnit ? kMostUnit : s);
}
__device__ __forceinline__ float power_of_two(int byte) { return __uint_as_float((unsigned)byte << 23); }

}  // namespace
}  // namespace dapq
