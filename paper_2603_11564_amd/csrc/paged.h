// The page pool as the kernels see it, and the FP4 and E4M3 rows of it.
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
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Formats, as the kernels' template arguments.
constexpr int kBf16 = DAPQ_PAGES_BF16, kFp4 = DAPQ_PAGES_FP4, kE4m3 = DAPQ_PAGES_E4M3;
constexpr int kRowBytes = 2 * kHeadDim;      // of a bf16 row
template <int FMT>
constexpr int kCodeBytes = FMT == kBf16 ? kRowBytes : (FMT == kFp4 ? kHeadDim / 2 : kHeadDim);  // of a row; codes have 4 scale bytes beside them
constexpr float kLargestFp4Scale = 0x1p125f;  // of finite values: 6 * 2^125 is a bf16 number, twice as much is not (E4M3: e4m3_past)
constexpr unsigned kNoScale = 255;           // scale byte of a group with a value that is not finite
// Bytes of a row with its scales (host).
inline int row_bytes(const dapq_pages* p) {
  return p->format == DAPQ_PAGES_BF16 ? kRowBytes : (p->format == DAPQ_PAGES_FP4 ? kCodeBytes<kFp4> : kCodeBytes<kE4m3>) + 4;
}

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
  return largest >= 0x7f80u ? kNoScale : (unsigned)kept;
}
// The same of E4M3: the least e in [-117, 119] with max <= 464 * 2^e.  464 = (1 + 104 / 128) * 2^8: e is x - 8, or x - 7 if m > 104.  2^-9, the least
// code's value, is then a normal bf16 number at every scale.
__device__ __forceinline__ unsigned e4m3_scale_byte(unsigned largest) {
  const int s = (int)((largest + (127 - 104)) >> 7) - 8;
  const int kept = s < 10 ? 10 : (s > 246 ? 246 : s);
  return largest >= 0x7f80u ? kNoScale : (unsigned)kept;
}
template <int FMT>
__device__ __forceinline__ unsigned scale_byte_of(unsigned largest) {
  return FMT == kFp4 ? fp4_scale_byte(largest) : e4m3_scale_byte(largest);
}
// 2^(s - 127) as the conversions take it, which look at the exponent's bits alone: 0 counts as 2^-127, 255 as no number.
__device__ __forceinline__ float group_scale(unsigned s) { return __uint_as_float(s << 23); }

// Eight values (four dwords of two bf16) as codes.  bad: the group is not finite.
__device__ __forceinline__ unsigned fp4_pack8(u32x4 x, unsigned scale_byte) {
  const float s = group_scale(scale_byte);
  const unsigned x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];  // (a bit_cast of a vector's element takes its first)
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x0), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x1), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x2), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x3), s, 3);
  return scale_byte == kNoScale ? 0u : c;
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

// Eight codes of FP4 of which those are 0 whose values with the scale s are no finite bf16: all of them without a scale, 2 and more at 2^127, 4 and 6 at 2^126.
__device__ __forceinline__ unsigned fp4_finite8(unsigned c, float s) {
  const unsigned past = s > 0x1p127f ? ~0u : (s > 0x1p126f ? c >> 2 : (s > kLargestFp4Scale ? c >> 2 & c >> 1 : 0u));  // (in the lowest bit of each code)
  return c & ~((past & 0x11111111u) * 15u);
}

// Two values as E4M3 codes, in the low half.  The conversion rounds to nearest, ties to even, and makes what is past the levels no number: only at the
// largest scale there may be such values, which become 448.
__device__ __forceinline__ unsigned e4m3_pack2(unsigned x, unsigned scale_byte) {
  if (scale_byte == 246u) {
    const unsigned most = 0x7f607f60u;  // 448 * 2^119
    const unsigned m = __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(u16x2, x & 0x7fff7fffu), __builtin_bit_cast(u16x2, most)));
    x = m | (x & 0x80008000u);
  }
  const s16x2 c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, __builtin_bit_cast(bf16x2, x), group_scale(scale_byte), 0);
  return scale_byte == kNoScale ? 0u : __builtin_bit_cast(unsigned, c) & 0xffffu;
}
__device__ __forceinline__ u32x2 e4m3_pack8(u32x4 x, unsigned scale_byte) {
  const unsigned x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  return u32x2{e4m3_pack2(x0, scale_byte) | e4m3_pack2(x1, scale_byte) << 16, e4m3_pack2(x2, scale_byte) | e4m3_pack2(x3, scale_byte) << 16};
}
// Codes 2i and 2i + 1 of four.  The code 127 is no number, and neither is any code of a group without a scale.
__device__ __forceinline__ unsigned e4m3_unpack2(unsigned c, float s, int i) {
  return i == 0 ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, 0))
                : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, 1));
}
__device__ __forceinline__ u32x4 e4m3_unpack8(unsigned c0, unsigned c1, float s) {
  return u32x4{e4m3_unpack2(c0, s, 0), e4m3_unpack2(c0, s, 1), e4m3_unpack2(c1, s, 0), e4m3_unpack2(c1, s, 1)};
}

// The highest bits of those of four E4M3 codes whose values with the scale s are no finite bf16: 127 at any scale, from 2^8 on (0x78) at 2^120, from 2^7
// on (0x70) at 2^121, ..., all of them without a scale.
__device__ __forceinline__ unsigned e4m3_past(unsigned c, float s) {
  const int over = (int)(__float_as_uint(s) >> 23) - (119 + 127);
  const unsigned to_bit = over <= 0 ? 1u : (over >= 9 ? 0x80u : 8u * over);  // takes the first such code to 128
  return ((c & 0x7f7f7f7fu) + to_bit * 0x01010101u) & 0x80808080u;
}
__device__ __forceinline__ unsigned e4m3_finite4(unsigned c, float s) { return c & ~((e4m3_past(c, s) >> 7) * 255u); }

// The larger of the two magnitudes in a dword.
__device__ __forceinline__ unsigned larger_magnitude(unsigned x) {
  const unsigned a = x & 0x7fffu, b = (x >> 16) & 0x7fffu;
  return a > b ? a : b;
}

template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned x) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;                               // lanes of a quad
constexpr int kRor1 = 0x121, kRor2 = 0x122, kRor4 = 0x124, kRor8 = 0x128;  // of 16 lanes
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

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

}  // namespace
}  // namespace dapq
