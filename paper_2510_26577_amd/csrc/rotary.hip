// libtva: rotary positions, norms of heads, and the append to the cache (gfx950).  Entry points and their meaning:
// include/tva_layer.h.
//
// One kernel.  Large calls are bound by memory: every head is read once (its pair's half comes from another lane, not from memory) and written
// once.  A wave has one token and four pieces of 1 KB of its heads (8 lanes of 16 bytes to a head of 64, 16 to one of 128), all on the way while
// the token's position is found and one lane per pair computes its sine and cosine, which all heads share through LDS.  The grid is token x
// wave-wide piece in one dimension: with tokens and pieces apart waves start in another order (62 us in the place of 56).
//   8204 tokens of 64 + 8 heads of 128, half of each turned, interleaved, 288 MB   55 us  5.2 TB/s (a copy: 5.1)
//   16384 tokens of 32 + 8 heads of 128, normed, 336 MB                            68 us  4.9 TB/s
//   16396 of 32 + 8 + 8, normed, K and V to 4-bit rows, 352 MB                     85 us  4.1 TB/s (1.25 times the vector instructions)
//   the same not normed and to 16-bit rows, 384 MB, 75 us, to 8-bit rows, 352 MB, 73
// Small calls (a tree's nodes, 64 tokens) are one launch of 4.6 to 5.4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache_rows.h"
#include "sequences.h"
#include "tva.h"
#include "tva_cache.h"
#include "tva_layer.h"

namespace {

using namespace cache_rows;

constexpr int kWaves = 4;
constexpr int kRowsInFlight = 4;  // wave-wide pieces (of 64 / (D/8) heads) that a wave has on the way

struct RotateParams {
  const int32_t *cu_T, *L, *pos;
  const uint64_t *mask;
  const double *freq;
  const char *q, *k, *v;
  const uint16_t *q_norm, *k_norm;
  char *q_out, *k_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  CacheView c;
  float k_scale, v_scale;  // E4M3
  int32_t *L_out, *err_flag;
  int B, Hq, Hkv, sum_T, dims, words;
  int q_pieces, k_pieces, v_pieces, parts;  // wave-wide pieces of a token's q, k and v; waves per token
  float magnitude, eps;
};

__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Eight bf16 numbers / s -> E4M3 codes
__device__ __forceinline__ u32x2 eight_codes(const u16x8 x, float s) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float z = widen(x[i]) / s;
    y[i] = z == z ? fminf(fmaxf(z, -448.f), 448.f) : 0.f;
  }
  u32x2 w = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int h = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], h, true);
  }
  return w;
}

// One head's eight elements of this lane, to the cache row at unit `at` (head included)
template <int D, int KIND>
__device__ __forceinline__ void to_cache(const CacheView &c, bool is_v, int64_t at, int piece, const u16x8 x, float scale, bool valid) {
  constexpr int LPR = D / 8;
  char *base = is_v ? c.v : c.k;
  if constexpr (KIND == TVA_ROWS_BF16) {
    if (valid) *(u16x8 *)(base + (at + piece * 8) * 2) = x;
  } else if constexpr (KIND == TVA_ROWS_E4M3) {
    const u32x2 w = eight_codes(x, scale);
    if (valid) *(u32x2 *)(base + at + piece * 8) = w;
  } else if (is_v) {
    float s;
    const uint32_t w = round_v<LPR>(x, &s);
    if (valid) ((uint32_t *)base)[at * LPR + piece] = w;
    if (valid && piece == 0) ((uint16_t *)c.v_row_scale)[at] = (uint16_t)(__float_as_uint(s) >> 16);
  } else {
    uint32_t s;
    const uint32_t w = round_k<LPR>(x, &s);
    if (valid) ((uint32_t *)base)[at * LPR + piece] = w;
    if (valid && piece % 4 == 0) ((uint8_t *)c.k_row_scale)[at * (D / 32) + piece / 4] = (uint8_t)s;
  }
}

constexpr int kNoCache = -1;

// KIND: of the cache's rows, or kNoCache.  NORM: q's or k's heads are normed
template <int D, bool INTERLEAVED, int KIND, bool NORM>
__global__ void __launch_bounds__(64 * kWaves) rotate_kernel(const RotateParams p) {
  constexpr int LPR = D / 8, HEADS = 64 / LPR, U = kRowsInFlight;
  __shared__ float2 turns[kWaves][D / 2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (KIND != kNoCache && blockIdx.x == 0 && p.L_out)
    for (int b = threadIdx.x; b < p.B; b += 64 * kWaves) p.L_out[b] = p.L[b] + (p.cu_T[b + 1] - p.cu_T[b]);
  const uint32_t unit = blockIdx.x * kWaves + wave;
  const int64_t row = unit / (uint32_t)p.parts;
  const int first = (int)(unit - (uint32_t)row * (uint32_t)p.parts) * U;
  if (row >= p.sum_T) return;
  const int piece = lane % LPR;  // of the head: elements 8 piece ..
  const int half = p.dims / 16;  // pieces between the two elements of a pair
  const bool turned = piece * 8 < p.dims;
  const int other = INTERLEAVED || !turned ? piece : piece < half ? piece + half : piece - half;

  // ---- the rows (all reads come before the first write: the outputs may be the inputs) ----
  u16x8 x[U];
  int head[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = first + u;
    const bool is_q = at < p.q_pieces, is_k = !is_q && at < p.q_pieces + p.k_pieces;
    const int H = is_q ? p.Hq : p.Hkv;
    head[u] = (is_q ? at : is_k ? at - p.q_pieces : at - p.q_pieces - p.k_pieces) * HEADS + lane / LPR;
    const char *from = is_q ? p.q + row * p.q_stride * 2 : is_k ? p.k + row * p.k_stride * 2 : p.v + row * p.v_stride * 2;
    from += min(head[u], H - 1) * (D * 2);
    x[u] = u16x8{};
    if (at < p.q_pieces + p.k_pieces + p.v_pieces) x[u] = *(const u16x8 *)(from + piece * 16);
  }

  // the weights of the first heads' norm
  const uint16_t *norm = !NORM ? nullptr : first < p.q_pieces ? p.q_norm : p.k_norm;
  u16x8 w = {}, wz = {};
  if (NORM && norm) w = *(const u16x8 *)(norm + piece * 8), wz = *(const u16x8 *)(norm + other * 8);

  // ---- the token's place and position ----
  int b = 0, i = (int)row, P = 0, start = 0;
  if (p.cu_T) {
    const sequences::Place at = sequences::find(p.cu_T, p.L, p.B, row, [](int, int from) { return (int64_t)from; });
    b = at.b, i = (int)row - at.t0, start = at.L;
    if (i < 0 || (int)row >= at.t1) return;  // behind the last sequence
  }
  if (p.pos) {
    P = p.pos[row];
  } else if (p.mask) {
    int bits = 0;
    for (int w = 0; w < p.words; ++w) bits += (int)__popcll(p.mask[row * p.words + w]);
    P = start + bits - 1;
  } else {
    P = start + i;
  }
  if (lane < p.dims / 2) {
    // in turns: the whole ones are dropped in 64 bits
    const double t = (double)P * (p.freq[lane] * 0.15915494309189535);
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    turns[wave][lane] = make_float2(c * p.magnitude, s * p.magnitude);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // this lane's element e becomes x[e] * own[e] + its pair's other element * with[e], a norm's weights taken in
  float own[8], with[8];
  auto turn = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      own[e] = 1.f, with[e] = 0.f;
      if (turned) {
        const bool second = INTERLEAVED ? e % 2 : piece >= half;
        const float2 t = turns[wave][INTERLEAVED ? piece * 4 + e / 2 : (second ? piece - half : piece) * 8 + e];
        own[e] = t.x, with[e] = second ? t.y : -t.y;
      }
      if (NORM && norm) own[e] *= widen(w[e]), with[e] *= widen(INTERLEAVED ? w[e ^ 1] : wz[e]);
    }
  };
  turn();
  // What a norm multiplies a head by.  Without a cache the heads' sums are made together, so that none waits for another; with one that
  // takes registers that its rows' waves need (16396 prompt tokens to 4-bit rows and read back 106 us, one by one 100).
  auto norm_of = [&](int u) __attribute__((always_inline)) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(widen(x[u][e]), widen(x[u][e]), s);
    s = over_lanes<LPR>(s, [](float x, float y) { return x + y; });
    return 1.f / sqrtf(s * (1.f / D) + p.eps);
  };
  float by[U];
  if constexpr (NORM && KIND == kNoCache) {
#pragma unroll
    for (int u = 0; u < U; ++u) by[u] = norm_of(u);
  }
  bool room = false;
  int64_t at_cache = 0;
  if constexpr (KIND != kNoCache) {
    const int64_t slot = (int64_t)start + i;
    room = slot >= 0 && slot < room_of(p.c, b);
    // (a table's entry below 0 is no page: what a table is filled with behind a sequence's pages)
    if (room && p.c.page_table) room = p.c.page_table[(int64_t)b * p.c.max_pages + page_of(p.c, (int)slot)] >= 0;
    if (room) at_cache = position_at(p.c, b, (int)slot);
    else if (p.err_flag && first <= p.q_pieces && lane == 0) atomicCAS(p.err_flag, 0, 1 + b);
  }

  // ---- head by head ----
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = first + u;
    if (at >= p.q_pieces + p.k_pieces + p.v_pieces) return;
    const bool is_q = at < p.q_pieces, is_v = at >= p.q_pieces + p.k_pieces;
    const bool valid = head[u] < (is_q ? p.Hq : p.Hkv);
    if (is_v) {
      if constexpr (KIND != kNoCache)
        if (room) to_cache<D, KIND>(p.c, true, at_cache + head[u] * p.c.stride_head, piece, x[u], p.v_scale, valid);
      continue;
    }
    if (NORM && u > 0 && at == p.q_pieces) {  // k's heads have a norm of their own
      norm = p.k_norm;
      if (norm) w = *(const u16x8 *)(norm + piece * 8), wz = *(const u16x8 *)(norm + other * 8);
      turn();
    }
    u16x8 y = x[u];
    if constexpr (!INTERLEAVED) {
      u32x4 from = __builtin_bit_cast(u32x4, x[u]);
#pragma unroll
      for (int e = 0; e < 4; ++e) from[e] = (uint32_t)__builtin_amdgcn_ds_bpermute((lane - piece + other) * 4, (int)from[e]);
      y = __builtin_bit_cast(u16x8, from);
    }
    float f = 1.f;
    if (NORM && norm) {
      if constexpr (KIND == kNoCache) f = by[u];
      else f = norm_of(u);
    }
    u16x8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a = widen(x[u][e]), z = widen(y[INTERLEAVED ? e ^ 1 : e]);
      if (NORM) a *= f, z *= f;  // (first: what the weights make of an element that is not normed yet may be past fp32's range, f then 0)
      float r = a * own[e];
      if (turned) r = fmaf(z, with[e], r);  // (elements that are not turned are not mixed with others either: 0 * inf)
      out[e] = narrow(r);
    }
    if (is_q) {
      if (valid) *(u16x8 *)(p.q_out + (row * p.q_out_stride + head[u] * D + piece * 8) * 2) = out;
    } else {
      if (valid && p.k_out) *(u16x8 *)(p.k_out + (row * p.k_out_stride + head[u] * D + piece * 8) * 2) = out;
      if constexpr (KIND != kNoCache)
        if (room) to_cache<D, KIND>(p.c, false, at_cache + head[u] * p.c.stride_head, piece, out, p.k_scale, valid);
    }
  }
}

// A row stride as given, 0 = packed: below 0 if it is none
int64_t stride_of(int64_t given, int H, int D) { return given == 0 ? (int64_t)H * D : given % 8 || given < (int64_t)H * D ? -1 : given; }
bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }

int check_rotate(const tva_rotate_args *a, bool append, RotateParams *p) {
  if (!a || a->B < 0 || a->Hq < 0 || a->Hkv < 0 || a->sum_T < 0) return TVA_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return TVA_UNSUPPORTED;
  if (a->dims < 0 || a->dims > a->D) return TVA_INVALID_ARG;
  if (a->dims % 16) return TVA_UNSUPPORTED;
  if (!(a->eps >= 0.f) || !std::isfinite(a->magnitude)) return TVA_INVALID_ARG;
  p->cu_T = a->cu_T, p->L = a->L, p->B = a->B, p->sum_T = a->sum_T;
  if ((append || !a->pos) && a->B > 0 && (!a->cu_T || !a->L)) return TVA_INVALID_ARG;
  if (a->sum_T == 0) return TVA_OK;  // (tensors without rows need no place)
  if (!a->q && !a->k) return TVA_INVALID_ARG;
  if ((a->q && a->Hq < 1) || (a->k && a->Hkv < 1)) return TVA_INVALID_ARG;
  if ((a->q == nullptr) != (a->q_out == nullptr) || (a->k == nullptr && a->k_out) || (!append && a->k && !a->k_out)) return TVA_INVALID_ARG;
  if (a->dims > 0 && (!a->freq || ((uintptr_t)a->freq & 7))) return TVA_INVALID_ARG;
  if (!a->pos && a->anc_mask && (a->mask_words < 1 || a->mask_words > 2)) return TVA_UNSUPPORTED;
  if (!aligned(a->q) || !aligned(a->k) || !aligned(a->q_out) || !aligned(a->k_out) || !aligned(a->q_norm) || !aligned(a->k_norm)) return TVA_INVALID_ARG;
  p->q_stride = stride_of(a->q_stride, a->Hq, a->D), p->k_stride = stride_of(a->k_stride, a->Hkv, a->D);
  p->q_out_stride = stride_of(a->q_out_stride, a->Hq, a->D), p->k_out_stride = stride_of(a->k_out_stride, a->Hkv, a->D);
  if (p->q_stride < 0 || p->k_stride < 0 || p->q_out_stride < 0 || p->k_out_stride < 0) return TVA_INVALID_ARG;
  if (a->q && a->q_out == a->q && p->q_out_stride != p->q_stride) return TVA_INVALID_ARG;
  if (a->k && a->k_out == a->k && p->k_out_stride != p->k_stride) return TVA_INVALID_ARG;
  const int heads = 64 / (a->D / 8);
  p->pos = a->pos, p->mask = a->anc_mask, p->words = a->mask_words, p->freq = a->freq;
  p->q = (const char *)a->q, p->k = (const char *)a->k, p->q_norm = (const uint16_t *)a->q_norm, p->k_norm = (const uint16_t *)a->k_norm;
  p->q_out = (char *)a->q_out, p->k_out = (char *)a->k_out;
  p->Hq = a->Hq, p->Hkv = a->Hkv, p->dims = a->dims;
  p->q_pieces = a->q ? (a->Hq + heads - 1) / heads : 0, p->k_pieces = a->k ? (a->Hkv + heads - 1) / heads : 0;
  p->magnitude = a->magnitude == 0.f ? 1.f : a->magnitude, p->eps = a->eps;
  return TVA_OK;
}

template <int KIND>
int launch(const tva_rotate_args *a, RotateParams &p, hipStream_t st) {
  p.parts = std::max(1, (p.q_pieces + p.k_pieces + p.v_pieces + kRowsInFlight - 1) / kRowsInFlight);
  const int64_t blocks = std::max<int64_t>(1, ((int64_t)p.sum_T * p.parts + kWaves - 1) / kWaves);
  if (blocks > 0x3fffffff) return TVA_UNSUPPORTED;  // (waves are numbered in 32 bits)
  (void)hipGetLastError();
  auto go = [&](auto d, auto inter) {
    constexpr int D = decltype(d)::value;
    constexpr bool INTERLEAVED = decltype(inter)::value;
    if (p.q_norm || p.k_norm) hipLaunchKernelGGL((rotate_kernel<D, INTERLEAVED, KIND, true>), dim3((unsigned)blocks), dim3(64 * kWaves), 0, st, p);
    else hipLaunchKernelGGL((rotate_kernel<D, INTERLEAVED, KIND, false>), dim3((unsigned)blocks), dim3(64 * kWaves), 0, st, p);
  };
  auto shape = [&](auto d) {
    if (a->interleaved) go(d, std::true_type{});
    else go(d, std::false_type{});
  };
  if (a->D == 128) shape(std::integral_constant<int, 128>{});
  else shape(std::integral_constant<int, 64>{});
  return hipPeekAtLastError() == hipSuccess ? TVA_OK : TVA_HIP_ERROR;
}

}  // namespace

extern "C" {

int tva_rotate(const tva_rotate_args *a, void *stream) {
  RotateParams p{};
  const int rc = check_rotate(a, false, &p);
  if (rc != TVA_OK || a->sum_T == 0 || (a->B == 0 && (a->cu_T || !a->pos))) return rc;
  return launch<kNoCache>(a, p, (hipStream_t)stream);
}

int tva_cache_append(const tva_append_args *a, void *stream) {
  if (!a) return TVA_INVALID_ARG;
  RotateParams p{};
  int rc = check_rotate(&a->r, true, &p);
  if (rc != TVA_OK) return rc;
  if (a->r.sum_T > 0 && (!a->r.k || !a->v || !aligned(a->v))) return TVA_INVALID_ARG;
  p.v_stride = stride_of(a->v_stride, a->r.Hkv, a->r.D);
  if (p.v_stride < 0 || (a->L_out && a->L_out == a->r.L)) return TVA_INVALID_ARG;
  rc = view_of(a->cache, a->r.Hkv, a->r.D, true, &p.c);
  if (rc != TVA_OK) return rc;
  if (a->r.B == 0 || (a->r.sum_T == 0 && !a->L_out)) return TVA_OK;
  p.v = (const char *)a->v, p.v_pieces = p.k_pieces, p.L_out = a->L_out, p.err_flag = a->err_flag;
  p.k_scale = a->cache.k_scale == 0.f ? 1.f : a->cache.k_scale, p.v_scale = a->cache.v_scale == 0.f ? 1.f : a->cache.v_scale;
  const hipStream_t st = (hipStream_t)stream;
  if (a->cache.kind == TVA_ROWS_BF16) return launch<TVA_ROWS_BF16>(&a->r, p, st);
  if (a->cache.kind == TVA_ROWS_E4M3) return launch<TVA_ROWS_E4M3>(&a->r, p, st);
  return launch<TVA_ROWS_E2M1>(&a->r, p, st);
}

int tva_rotary_frequencies(int32_t scaling, int32_t dims, double base, double factor, double original, double low, double high, double *freq,
                           double *magnitude) {
  if (!freq || dims < 4 || dims % 2 || !(base > 1.0) || !std::isfinite(base)) return TVA_INVALID_ARG;
  if (scaling < TVA_ROTARY_PLAIN || scaling > TVA_ROTARY_RAMP) return TVA_INVALID_ARG;
  if (scaling != TVA_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return TVA_INVALID_ARG;
  const bool choice = scaling == TVA_ROTARY_WAVELENGTH || scaling == TVA_ROTARY_RAMP;
  if (choice && !(original > 0.0 && std::isfinite(original) && low > 0.0 && high > low && std::isfinite(high))) return TVA_INVALID_ARG;
  const double two_pi = 6.283185307179586;
  if (scaling == TVA_ROTARY_BASE) base *= std::pow(factor, dims / (dims - 2.0));
  // the pair (as a real number) that makes n turns over `original` positions
  auto pair_of = [&](double n) { return dims * std::log(original / (n * two_pi)) / (2.0 * std::log(base)); };
  double from = 0.0, to = 0.0;
  if (scaling == TVA_ROTARY_RAMP) {
    from = std::max(std::floor(pair_of(high)), 0.0), to = std::min(std::ceil(pair_of(low)), dims - 1.0);
    if (to - from < 0.001) to = from + 0.001;  // (a step)
  }
  for (int j = 0; j < dims / 2; ++j) {
    const double f = std::pow(base, -2.0 * j / dims);
    double keep = 1.0;
    if (scaling == TVA_ROTARY_LINEAR) keep = 0.0;
    else if (scaling == TVA_ROTARY_WAVELENGTH) keep = std::min(std::max((original * f / two_pi - low) / (high - low), 0.0), 1.0);
    else if (scaling == TVA_ROTARY_RAMP) keep = 1.0 - std::min(std::max((j - from) / (to - from), 0.0), 1.0);
    freq[j] = keep == 1.0 ? f : f * keep + f / factor * (1.0 - keep);
  }
  if (magnitude) *magnitude = scaling == TVA_ROTARY_RAMP ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return TVA_OK;
}

size_t tva_sizeof_rotate_args(void) { return sizeof(tva_rotate_args); }
size_t tva_sizeof_append_args(void) { return sizeof(tva_append_args); }

}  // extern "C"
