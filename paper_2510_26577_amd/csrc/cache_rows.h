// What the kernels of long caches share: where a position's rows lie, and the 4-bit rows' formats (include/tva_cache.h).
#ifndef TVA_CACHE_ROWS_H
#define TVA_CACHE_ROWS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tva.h"
#include "tva_cache.h"

namespace cache_rows {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A cache as the kernels see it: strides in units (elements for BF16 and E4M3, rows of one head for E2M1; one unit is
// unit_bytes bytes of K or V).
struct CacheView {
  char *k, *v;
  char *k_row_scale, *v_row_scale;
  const int32_t *cu_L, *page_table;
  int page_size, max_pages;
  uint32_t page_magic, page_bits;  // division by the page size, of positions below 2^30: page_of
  int64_t stride_page, stride_tok, stride_head;
};

// t / page_size, exact for t below 2^30 (page_magic is 2^(31 + page_bits) / page_size rounded up, 2^page_bits >= page_size)
__device__ __forceinline__ int page_of(const CacheView &c, int t) { return (int)(__umulhi((uint32_t)t * 2u, c.page_magic) >> c.page_bits); }

// Where position t of sequence b begins, head 0, in units.  The position is within the sequence's room.
__device__ __forceinline__ int64_t position_at(const CacheView &c, int b, int t) {
  if (c.page_table) {
    const int pi = page_of(c, t);
    const int page = c.page_table[(int64_t)b * c.max_pages + pi];
    return (int64_t)page * c.stride_page + (int64_t)(t - pi * c.page_size) * c.stride_tok;
  }
  return ((int64_t)c.cu_L[b] + t) * c.stride_tok;
}

// The same for one sequence and head, the look into the page table apart from what is made of it, so that a loop can look ahead:
// entry() is what is read (nothing in the dense form), at() the place.
template <bool PAGED>
struct Finder {
  const int32_t *table;
  int64_t base;
  __device__ __forceinline__ Finder(const CacheView &c, int b, int g) {
    if constexpr (PAGED) table = c.page_table + (int64_t)b * c.max_pages, base = g * c.stride_head;
    else table = nullptr, base = (int64_t)c.cu_L[b] * c.stride_tok + g * c.stride_head;
  }
  __device__ __forceinline__ int entry(const CacheView &c, int t) const {
    if constexpr (PAGED) return table[page_of(c, t)];
    else return 0;
  }
  __device__ __forceinline__ int64_t at(const CacheView &c, int t, int entry) const {
    if constexpr (PAGED) return base + (int64_t)entry * c.stride_page + (int64_t)(t - page_of(c, t) * c.page_size) * c.stride_tok;
    else return base + (int64_t)t * c.stride_tok;
  }
};
// Positions of sequence b that have a place: what a call writes stays below it.
__device__ __forceinline__ int64_t room_of(const CacheView &c, int b) {
  return c.page_table ? min((int64_t)c.max_pages * c.page_size, (int64_t)1 << 30) : (int64_t)c.cu_L[b + 1] - c.cu_L[b];
}

// Checks a cache argument and turns it into a view: TVA_OK or a negative status.
inline int view_of(const tva_cache &a, int Hkv, int D, bool need_v, CacheView *c) {
  if (a.kind < TVA_ROWS_BF16 || a.kind > TVA_ROWS_E2M1) return TVA_INVALID_ARG;
  const bool four = a.kind == TVA_ROWS_E2M1;
  if (!a.k || (need_v && !a.v)) return TVA_INVALID_ARG;
  if (four && (!a.k_row_scale || (need_v && !a.v_row_scale))) return TVA_INVALID_ARG;
  if (((uintptr_t)a.k | (uintptr_t)(need_v ? a.v : nullptr)) & 15) return TVA_INVALID_ARG;
  if (four && (((uintptr_t)a.k_row_scale & 3) || ((uintptr_t)(need_v ? a.v_row_scale : nullptr) & 1))) return TVA_INVALID_ARG;
  const bool dense = a.cu_L != nullptr, paged = a.page_table != nullptr;
  if (dense == paged) return TVA_INVALID_ARG;
  if (paged && (a.page_size <= 0 || a.max_pages <= 0)) return TVA_INVALID_ARG;
  if (paged && a.page_size > 1 << 30) return TVA_UNSUPPORTED;
  if (a.stride_page < 0 || a.stride_tok < 0 || a.stride_head < 0) return TVA_INVALID_ARG;
  const int unit = four ? D : a.kind == TVA_ROWS_E4M3 ? 16 : 8;
  if (a.stride_page % unit || a.stride_tok % unit || a.stride_head % unit) return TVA_INVALID_ARG;
  if (a.kind == TVA_ROWS_E4M3 && (!(a.k_scale >= 0.f) || !(a.v_scale >= 0.f))) return TVA_INVALID_ARG;
  const int per = four ? D : 1;
  c->k = (char *)a.k, c->v = (char *)a.v, c->k_row_scale = (char *)a.k_row_scale, c->v_row_scale = (char *)a.v_row_scale;
  c->cu_L = a.cu_L, c->page_table = a.page_table;
  c->page_size = paged ? a.page_size : 1, c->max_pages = a.max_pages;
  c->page_bits = 0;
  while ((1u << c->page_bits) < (uint32_t)c->page_size) ++c->page_bits;
  c->page_magic = (uint32_t)(((1ull << (31 + c->page_bits)) + (uint32_t)c->page_size - 1) / (uint32_t)c->page_size);
  c->stride_head = (a.stride_head ? a.stride_head : D) / per;
  c->stride_tok = (a.stride_tok ? a.stride_tok : (int64_t)Hkv * D) / per;
  c->stride_page = a.stride_page ? a.stride_page / per : (int64_t)c->page_size * c->stride_tok;
  return TVA_OK;
}

// A lane's number and that of the lane 32 further on, added
__device__ __forceinline__ float half_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float exponent_byte(uint32_t x) { return __uint_as_float(x << 23); }  // 2^(x - 127), x of 1 .. 254

// The eight codes of a word -> bf16 values times s (a power of two, so exact).
__device__ __forceinline__ bf16x8 widen8(uint32_t w, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace cache_rows
#endif
