// The page pool as the kernels see it, and the FP4 rows of it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dapq_internal.h"

namespace dapq {

struct PagePool {
  uint8_t *k, *v, *k_scales, *v_scales;
  const int32_t* table;
  int32_t n_pages, max_pages, page_shift, n_kv_heads;
};

// Checks of the descriptors that the paged calls share (host).
int check_pages(const dapq_pages* p);
int check_step(const dapq_pages* p, const dapq_step* s);
inline PagePool page_pool(const dapq_pages* p) {
  return {static_cast<uint8_t*>(p->k), static_cast<uint8_t*>(p->v), static_cast<uint8_t*>(p->k_scales),
          static_cast<uint8_t*>(p->v_scales), p->table, p->n_pages, p->max_pages, __builtin_ctz((unsigned)p->page_rows), p->n_kv_heads};
}

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kRowBytes = 2 * kHeadDim;      // of a bf16 row
constexpr int kFp4RowBytes = kHeadDim / 2;   // the codes of an FP4 row; and 4 scale bytes
constexpr float kLargestFp4Scale = 0x1p125f;  // of finite values: 6 * 2^125 is a bf16, 6 * 2^126 is not
constexpr unsigned kFp4Bad = 255;            // scale byte of a group with a value that is not finite

// Row number of slot 0 of a page of one head.
__device__ __forceinline__ int64_t page_row(const PagePool& p, int layer, int page, int head) {
  return (((int64_t)layer * p.n_pages + page) * p.n_kv_heads + head) << p.page_shift;
}
// Row number of row i of a sequence, or -1 if it is on no page.
__device__ __forceinline__ int64_t find_row(const PagePool& p, int layer, int64_t seq, int head, int64_t i) {
  const int64_t at = i >> p.page_shift;
  if (i < 0 || at >= p.max_pages) return -1;
  const int page = p.table[seq * p.max_pages + at];
  if (page < 0 || page >= p.n_pages) return -1;
  return page_row(p, layer, page, head) + (i & ((1 << p.page_shift) - 1));
}

// The scale byte of a group from its largest magnitude (the bits of a non-negative bf16, in the low half): the least e in [-125, 125] with
// max <= 7 * 2^e.  max = (1 + m / 128) * 2^x, and 7 * 2^e = 1.75 * 2^(e + 2): e is x - 2, or x - 1 if m > 96.  The biased exponent
// x + 127 is the byte's for e = x; 0x7f80 and more are an infinity or a NaN.
__device__ __forceinline__ unsigned fp4_scale_byte(unsigned largest) {
  const int s = (int)((largest + (127 - 96)) >> 7) - 2;  // (the sum carries into the exponent from m = 97 on)
  const int kept = s < 2 ? 2 : (s > 252 ? 252 : s);
  return largest >= 0x7f80u ? kFp4Bad : (unsigned)kept;
}
// 2^(s - 127) as the conversions take it, which look at the exponent's bits alone: 0 counts as 2^-127, 255 as no number.
__device__ __forceinline__ float fp4_scale(unsigned s) { return __uint_as_float(s << 23); }

// Eight values (four dwords of two bf16) as codes.  bad: the group is not finite.
__device__ __forceinline__ unsigned fp4_pack8(u32x4 x, unsigned scale_byte) {
  const float s = fp4_scale(scale_byte);
  const unsigned x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];  // (a bit_cast of a vector's element takes its first)
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x0), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x1), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x2), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x3), s, 3);
  return scale_byte == kFp4Bad ? 0u : c;
}
// Codes 2i and 2i + 1 of eight.
__device__ __forceinline__ unsigned fp4_unpack2(unsigned c, float s, int i) {
  switch (i) {
    case 0: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
    case 1: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
    case 2: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
    default: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  }
}
// Eight codes as bf16 values.  A group without a scale (255) is NaN: the conversion makes its values so.
__device__ __forceinline__ u32x4 fp4_unpack8(unsigned c, float s) {
  return u32x4{fp4_unpack2(c, s, 0), fp4_unpack2(c, s, 1), fp4_unpack2(c, s, 2), fp4_unpack2(c, s, 3)};
}

// Eight codes of which those are 0 whose values with the scale s are no finite bf16: all of them without a scale, 2 and more at 2^127, 4 and 6 at 2^126.
__device__ __forceinline__ unsigned fp4_finite8(unsigned c, float s) {
  const unsigned past = s > 0x1p127f ? ~0u : (s > 0x1p126f ? c >> 2 : (s > kLargestFp4Scale ? c >> 2 & c >> 1 : 0u));  // (in the lowest bit of each code)
  return c & ~((past & 0x11111111u) * 15u);
}

// The larger of the two magnitudes in a dword.
__device__ __forceinline__ unsigned larger_magnitude(unsigned x) {
  const unsigned a = x & 0x7fffu, b = (x >> 16) & 0x7fffu;
  return a > b ? a : b;
}

}  // namespace
}  // namespace dapq
