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
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
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
__host__ __device__ __forceinline__ int page_of(const CacheView &c, int t) {
  return (int)((uint32_t)((uint64_t)((uint32_t)t * 2u) * c.page_magic >> 32) >> c.page_bits);
}

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
// entry() is what is read (nothing in the dense form), at() the place.  GAPS: entries below 0 are allowed among those that are looked up (pages
// given back): they are page 0 here, so that no place lies outside the cache.
template <bool PAGED, bool GAPS = false>
struct Finder {
  const int32_t *table;
  int64_t base;
  __host__ __device__ __forceinline__ Finder(const CacheView &c, int b, int g) {
    if constexpr (PAGED) table = c.page_table + (int64_t)b * c.max_pages, base = g * c.stride_head;
    else table = nullptr, base = (int64_t)c.cu_L[b] * c.stride_tok + g * c.stride_head;
  }
  __host__ __device__ __forceinline__ int entry_of(int page) const {
    if constexpr (!PAGED) return 0;
    else return GAPS && table[page] < 0 ? 0 : table[page];
  }
  __host__ __device__ __forceinline__ int entry(const CacheView &c, int t) const {
    if constexpr (PAGED) return entry_of(page_of(c, t));
    else return 0;
  }
  __host__ __device__ __forceinline__ int64_t at(const CacheView &c, int t, int entry) const {
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

// What 4, 8 or 16 neighbouring lanes hold, added up or the largest of it, in each of them: lanes exchanged inside the vector instructions
// (by shuffles through LDS each step waits for its answer)
template <int CTRL, class T>
__device__ __forceinline__ T exchanged(T x) {
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int N, class T, class F>
__device__ __forceinline__ T over_lanes(T x, F f) {
  static_assert(N == 4 || N == 8 || N == 16, "");
  x = f(x, exchanged<0xb1>(x));                        // lanes 1, 0, 3, 2
  x = f(x, exchanged<0x4e>(x));                        // lanes 2, 3, 0, 1
  if constexpr (N >= 8) x = f(x, exchanged<0x141>(x));  // eight lanes the other way round
  if constexpr (N >= 16) x = f(x, exchanged<0x140>(x)); // sixteen
  return x;
}

// |x| bits of the largest finite of eight bf16 numbers, and whether all are finite
__device__ __forceinline__ uint32_t largest(const u16x8 x, bool *finite) {
  uint32_t a = 0, all = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = x[i] & 0x7fff;
    a = m < 0x7f80 && m > a ? m : a;
    all = max(all, m);
  }
  *finite = all < 0x7f80;
  return a;
}
// Code of x / s by the borders between codes: s (at most 4 significant bits) times a border (3) is exact, and so are the comparisons.
// NaN compares false: 0.
__device__ __forceinline__ uint32_t code_of(float x, float s) {
  const float a = fabsf(x);
  const uint32_t c = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) + (a >= 3.5f * s) + (a > 5.f * s);
  return c | (a == a ? (__float_as_uint(x) >> 28) & 8u : 0u);
}
__device__ inline uint32_t codes_of(const u16x8 x, float s) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) w |= code_of(__uint_as_float((uint32_t)x[i] << 16), s) << (4 * i);
  return w;
}
// The same by the conversion instructions, for finite x of at most 6 s: they divide by a power of two and round to nearest even.
__device__ __forceinline__ uint32_t codes_k(const u16x8 x, float s) {
  uint32_t w = 0;
#define PAIR(i) bf16x2{__builtin_bit_cast(__bf16, (uint16_t)x[2 * i]), __builtin_bit_cast(__bf16, (uint16_t)x[2 * i + 1])}
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, PAIR(0), s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, PAIR(1), s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, PAIR(2), s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, PAIR(3), s, 3);
#undef PAIR
  return w;
}
// V's scale is no power of two: the quotient comes from a reciprocal and one correction, exact where it is a border (only equality
// with one is near enough to matter: x has 8 bits and s times a border 7).
__device__ __forceinline__ uint32_t codes_v(const u16x8 x, float s) {
  const float r = 1.f / s;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = __uint_as_float((uint32_t)x[i] << 16), q = a * r;
    y[i] = fmaf(fmaf(-q, s, a), r, q);
  }
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
  return w;
}

// Eight elements of a K row (LPR lanes have the row's, in order) -> their codes, and the scale byte of the 32 they are among.
// a = (1 + m/128) 2^(E-127) <= 6 * 2^e
template <int LPR>
__device__ __forceinline__ uint32_t round_k(const u16x8 k, uint32_t *scale) {
  bool fine;
  uint32_t a = largest(k, &fine);
  a = over_lanes<4>(a, [](uint32_t x, uint32_t y) { return max(x, y); });
  const int e = (int)(a >> 7) - 127 - ((a & 127) > 64 ? 1 : 2), kept = min(max(e, -96), 124);
  const float s = exponent_byte((uint32_t)(kept + 127));
  uint32_t w = codes_k(k, s);
  if (!(fine && e == kept)) w = codes_of(k, s);  // (what the instructions would do is not asked)
  *scale = (uint32_t)(kept + 127);
  return w;
}
// Eight elements of a V row -> their codes, and the row's scale: a = n/256 * 2^(E-126), the quotient by 6 rounded up to four bits
template <int LPR>
__device__ __forceinline__ uint32_t round_v(const u16x8 v, float *scale) {
  bool fine;
  uint32_t a = largest(v, &fine);
  a = over_lanes<LPR>(a, [](uint32_t x, uint32_t y) { return max(x, y); });
  const int n = 128 + (int)(a & 127), e = (int)(a >> 7) - 126;
  const float s = fminf(fmaxf(n < 192 ? ldexpf((float)((n + 11) / 12), e - 7) : ldexpf((float)((n + 23) / 24), e - 6), 0x1p-96f), 0x1p124f);
  uint32_t w = codes_v(v, s);
  if (!(fine && s > 0x1p-96f && s < 0x1p124f)) w = codes_of(v, s);
  *scale = s;
  return w;
}

// The eight codes of a word -> bf16 values times s (a power of two, so exact).
__device__ __forceinline__ bf16x8 widen8(uint32_t w, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Four consecutive E4M3 bytes' pairs -> bf16 (exact)
__device__ __forceinline__ bf16x8 widen8_e4m3(u32x2 w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace cache_rows
#endif
