// libtva: eviction from K/V caches (gfx950).  Entry points and their meaning: include/tva_cache.h.
//
//   weigh_kernel   attention weights of cached keys, summed over a step's accepted rows.  S = Q K^T by 32x32x16 bf16 MFMAs with a
//                  key per lane: a wave holds the operands of its keys and streams row blocks past them, so that K is read once
//                  and a key's sum stays in its lane.  No atomics: a key has one wave.
//   choose_kernel  which slots of a weight row stay: one workgroup per row.  The n-th largest key is found digit by digit (8 bits,
//                  histograms in LDS), the kept set is then a bit per slot, and gaps and fillers are matched by rank.
//   shift_kernel   the rows that fill the gaps: sources and destinations are disjoint, so every row moves by itself.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cache_rows.h"
#include "tva.h"
#include "tva_cache.h"

namespace {

using namespace cache_rows;

constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------------------------------
// weights of keys
// ---------------------------------------------------------------------------------------
struct WeighParams {
  const int32_t *cu_T, *path, *path_len, *L, *first_pos;
  const __bf16 *q;
  const float *lse;
  CacheView c;
  float *weight;
  int32_t *pos;
  int64_t ld;
  int Hq, Hkv, G, max_rows, max_L;
  int blocks;  // of 32 keys, per wave
  float scale_log2;
};

// Four consecutive E4M3 bytes' pairs -> bf16 (exact)
__device__ __forceinline__ bf16x8 widen8_e4m3(u32x2 w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr int kWeighWaves = 4;

// What a lane reads of a K row, as it lies in the cache: elements 16 s + 8 half of step s (bf16), or half of the row per lane half.
template <int D, int KIND>
struct RawK {
  static constexpr int AHEAD = KIND == TVA_ROWS_BF16 ? 1 : KIND == TVA_ROWS_E4M3 ? 2 : 3;  // blocks on their way
  static constexpr int NS = D / 16, N = KIND == TVA_ROWS_BF16 ? NS : KIND == TVA_ROWS_E4M3 ? NS / 2 : NS / 4;
  u32x4 x[N];
  uint32_t scale;
  __device__ __forceinline__ void read(const CacheView &c, int64_t at, int half) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (KIND == TVA_ROWS_BF16) x[i] = *(const u32x4 *)(c.k + (at + i * 16 + half * 8) * 2);
      else if constexpr (KIND == TVA_ROWS_E4M3) x[i] = *(const u32x4 *)(c.k + at + half * (D / 2) + i * 16);
      else x[i] = *(const u32x4 *)(c.k + at * (D / 2) + half * (D / 4) + i * 16);
    }
    if constexpr (KIND == TVA_ROWS_E2M1) {
      if constexpr (D == 128) scale = *(const uint16_t *)(c.k_row_scale + at * 4 + half * 2);
      else scale = *(const uint8_t *)(c.k_row_scale + at * 2 + half);
    }
  }
  __device__ __forceinline__ bf16x8 operand(int s) const {
    if constexpr (KIND == TVA_ROWS_BF16) return __builtin_bit_cast(bf16x8, x[s]);
    else if constexpr (KIND == TVA_ROWS_E4M3) return widen8_e4m3(u32x2{x[s / 2][s % 2 * 2], x[s / 2][s % 2 * 2 + 1]});
    else return widen8(x[s / 4][s % 4], exponent_byte(s < 4 ? scale & 255 : scale >> 8));
  }
};

// Grid: waves of a sequence (head fastest: the heads of a token lie side by side in a token-major cache, and a workgroup's waves read
// whole lines of it), sequence.  A wave walks p.blocks blocks of 32 keys, the next block's rows on their way.
// The operands of the first 32 query rows (all there are, mostly) stay in registers; further ones are read again for every block of keys.
template <int D, int KIND, bool PAGED>
__global__ void __launch_bounds__(64 * kWeighWaves, D == 128 && KIND != TVA_ROWS_BF16 ? 3 : 4) weigh_kernel(const WeighParams p) {
  constexpr int NS = D / 16;
  __shared__ __align__(16) float lds[kWeighWaves][2][2][32];  // of the rows that stay, and of others
  const int b = blockIdx.y;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int id = blockIdx.x * kWeighWaves + wave, g = id % p.Hkv;
  const int key0 = (id / p.Hkv) * p.blocks * 32;
  const int t0 = p.cu_T[b], T = p.cu_T[b + 1] - t0;
  const int all = p.L[b], L = min(all, p.max_L);
  const int n = min(min(p.path ? p.path_len[b] : T, p.max_rows), all);
  const int end = min(L, key0 + p.blocks * 32);
  if (n <= 0 || key0 >= L) return;  // (no barriers below: a wave keeps to itself)
  const Finder<PAGED> find(p.c, b, g);
  auto own = [&](int key) __attribute__((always_inline)) { return min(key + l32, end - 1); };  // past the end: the last row
  constexpr int AHEAD = RawK<D, KIND>::AHEAD;
  // Loads return in the order they were asked for, and a wait is a count of those behind the one waited for: what a block needs (its
  // weights too) is asked for AHEAD blocks earlier, and always, so that the counts are known.
  const int old = all - n;  // positions below it are seen by every row
  float *const weight = p.weight + ((int64_t)b * p.Hkv + g) * p.ld;
  RawK<D, KIND> raw[AHEAD];
  float before[AHEAD];
  int entry[AHEAD];  // the page of this lane's key, looked up 2 AHEAD blocks earlier
  auto ask = [&](int u, int key) __attribute__((always_inline)) {
    raw[u].read(p.c, find.at(p.c, own(key), entry[u]), half);
    before[u] = weight[own(key)];
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) entry[u] = find.entry(p.c, own(key0 + 32 * u));
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) ask(u, key0 + 32 * u);
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) entry[u] = find.entry(p.c, own(key0 + 32 * (AHEAD + u)));

  const int R = T > 0 ? n * p.G : 0;  // (a sequence without rows has none to read, and the last one's would lie behind the tensors)
  // rows r0 .. r0+31: query operand (a row per lane), and in LDS minus log-sum-exp and the last position the row saw (-1: it does not count)
  auto rows_of = [&](int r0, bf16x8 (&q)[NS], float (&to)[2][32]) __attribute__((always_inline)) {
    const int r = min(r0 + l32, R - 1), i = r / p.G, head = g * p.G + (r - i * p.G);
    const int node = p.path ? p.path[(int64_t)b * p.max_rows + i] : i;
    const bool there = node >= 0 && node < T;
    const int64_t row = (int64_t)(t0 + (there ? node : 0)) * p.Hq + head;
    const float lse = p.lse[row];
    const bool counts = there && r0 + l32 < R && lse != -INFINITY;
    const __bf16 *from = p.q + row * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = *(const bf16x8 *)(from + (KIND == TVA_ROWS_BF16 ? s * 16 + half * 8 : half * (D / 2) + s * 8));
      if (!counts) q[s] = bf16x8{};  // (whatever it holds)
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (half == 0) to[0][l32] = counts ? -lse * kLog2e : -INFINITY, to[1][l32] = __int_as_float(counts ? old + i : -1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  // a block's products with a block of rows, as weights, added to this lane's key's sum (of this half's rows)
  auto weigh = [&](const bf16x8 (&k)[NS], const bf16x8 (&q)[NS], const float (&to)[2][32], int key, bool all_seen, float &sum) __attribute__((always_inline)) {
    f32x16 x = {};
#pragma unroll
    for (int s = 0; s < NS; ++s) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[s], k[s], x, 0, 0, 0);
    const float before = sum;
    auto add = [&](bool select) __attribute__((always_inline)) {
      sum = before;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const f32x4 l = *(const f32x4 *)(to[0] + 8 * c + 4 * half);
        f32x4 last = {};
        if (select) last = *(const f32x4 *)(to[1] + 8 * c + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = __builtin_amdgcn_exp2f(fmaf(x[c * 4 + e], p.scale_log2, l[e]));
          sum += !select || key + l32 <= __float_as_int(last[e]) ? w : 0.f;
        }
      }
    };
    if (all_seen) add(false);
    else add(true);
    // Rows that do not count have operands of 0 and -inf for minus their log-sum-exp, which gives 0 except with a key that is not finite
    // (0 * inf; 4-bit rows have none): such a block is gone through again, row by row.
    if (KIND != TVA_ROWS_E2M1 && all_seen && __any(sum != sum)) add(true);
  };

  bf16x8 q[NS];
  if (R > 0) {
    rows_of(0, q, lds[wave][0]);
  } else {
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = bf16x8{};
    if (half == 0) lds[wave][0][0][l32] = -INFINITY, lds[wave][0][1][l32] = __int_as_float(-1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  const int first_pos = p.pos && end > old ? p.first_pos[b] : 0;
  for (int base = key0;; base += 32 * AHEAD)
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int key = base + 32 * u;
      const int t = key + l32;
      bf16x8 k[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) k[s] = raw[u].operand(s);
      const bool all_seen = key + 32 <= old;
      float sum = 0.f;
      weigh(k, q, lds[wave][0], key, all_seen, sum);
      for (int r0 = 32; r0 < R; r0 += 32) {
        bf16x8 more[NS];
        rows_of(r0, more, lds[wave][1]);
        weigh(k, more, lds[wave][1], key, all_seen, sum);
      }
      const float w = half_sum(sum) + (t < old ? before[u] : 0.f);
      ask(u, key + 32 * AHEAD);
      entry[u] = find.entry(p.c, own(key + 64 * AHEAD));
      if (!half && t < end) {
        weight[t] = w;
        if (p.pos && t >= old) p.pos[((int64_t)b * p.Hkv + g) * p.ld + t] = first_pos + (t - old);
      }
      if (key + 32 >= end) return;
    }
}

// ---------------------------------------------------------------------------------------
// which slots stay
// ---------------------------------------------------------------------------------------
struct ChooseParams {
  const int32_t *L, *keep, *newest, *pos;
  const float *weight;
  int32_t *src, *L_out;
  int64_t ld, ld_src;
  int B, H, max_L, n_first, words, list;  // words: 64-slot words of the longest row; list: gaps listed at a time
};

constexpr int kChooseThreads = 512, kChooseWaves = kChooseThreads / 64, kCopies = 16;

// Slots in the order they are kept: larger first.  Protected above everything, NaN below, -0 as 0.
__device__ __forceinline__ uint32_t key_of(const ChooseParams &p, float w, bool safe) {
  if (safe) return 0xffffffffu;
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ int ones(uint64_t x) { return (int)__popcll(x); }
// The r-th set bit of w (r < popcount)
__device__ __forceinline__ int select_bit(uint64_t w, int r) {
  int at = 0;
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) {
    const int c = ones(w & ((1ull << s) - 1));
    if (r >= c) r -= c, w >>= s, at += s;
  }
  return at;
}

// Inclusive sum over the workgroup's threads, and its total
template <class T>
__device__ __forceinline__ T scan_threads(T x, T *part, T *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const T y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();  // (part may still be read)
  if (lane == 63) part[wave] = x;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kChooseWaves; ++w) {
    before += w < wave ? part[w] : 0;
    all += part[w];
  }
  *total = all;
  return x + before;
}

// ITEMS > 0: the row's keys stay in registers (L <= kChooseThreads * ITEMS); 0: they are read again in every pass.
template <int ITEMS>
__global__ void __launch_bounds__(kChooseThreads, 4) choose_kernel(const ChooseParams p) {
  extern __shared__ __align__(16) unsigned char lds[];
  uint64_t *above = (uint64_t *)lds, *equal = above + p.words;  // a bit per slot; above becomes the kept set
  uint64_t *part64 = equal + p.words;                            // kChooseWaves
  int *before = (int *)(part64 + kChooseWaves);                  // gaps before each word
  int *rank0 = before + p.words + 1;                             // kept slots from n on before each word
  int *hist = rank0 + p.words;                                   // [256][kCopies]
  int *part = hist + 256 * kCopies;                              // kChooseWaves, and what a pass finds
  int *list = part + 32;                                         // gaps by rank, p.list of them
  const int h = blockIdx.x, b = blockIdx.y, layer = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int L = min(max(p.L[b], 0), p.max_L), n = (int)min((int64_t)min(max(p.keep[b], 0), L), p.ld_src);
  if (h == 0 && layer == 0 && tid == 0 && p.L_out) p.L_out[b] = n;
  const int64_t r = ((int64_t)layer * p.B + b) * p.H + h;
  const float *weight = p.weight + r * p.ld;
  const int32_t *pos = p.pos ? p.pos + r * p.ld : nullptr;
  int32_t *src = p.src + r * p.ld_src;
  if (n == L) {
    for (int j = tid; j < n; j += kChooseThreads) src[j] = j;
    return;
  }
  if (n == 0) return;
  const int newest = p.newest ? p.newest[b] : 0x7fffffff;
  const bool ages = p.newest != nullptr;
  // Slots from L on count as the smallest key there is: they come last among equals, behind all that n < L can reach.
  // Reads are batched, ROUNDS of the workgroup at a time (one by one each waits for the one before: 512 rows of up to 32768 slots with
  // ages 164 us instead of 114).
  constexpr int ROUNDS = 4;
  auto read = [&](int t0, uint32_t (&k)[ROUNDS]) __attribute__((always_inline)) {
    float w[ROUNDS];
    int age[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) w[i] = weight[min(t0 + i * kChooseThreads, L - 1)];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) age[i] = pos ? pos[min(t0 + i * kChooseThreads, L - 1)] : t0 + i * kChooseThreads;
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      const int t = t0 + i * kChooseThreads;
      k[i] = t < L ? key_of(p, w[i], t < p.n_first || (ages && age[i] >= newest)) : 0;
    }
  };
  uint32_t keys[ITEMS > 0 ? ITEMS : 1];
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; i += ROUNDS) {
      uint32_t k[ROUNDS];
      read(i * kChooseThreads + tid, k);
#pragma unroll
      for (int j = 0; j < ROUNDS; ++j) keys[i + j] = k[j];
    }
  }
  auto each = [&](auto use) __attribute__((always_inline)) {
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) use(i * kChooseThreads + tid, keys[i]);
    } else {
      for (int t = tid; t - tid < L; t += ROUNDS * kChooseThreads) {
        uint32_t k[ROUNDS];
        read(t, k);
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) use(t + i * kChooseThreads, k[i]);
      }
    }
  };

  // ---- the n-th largest key: eight bits at a time, from the top
  uint32_t prefix = 0;
  int want = n;  // of the keys that begin with prefix, the want-th largest
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256 * kCopies; i += kChooseThreads) hist[i] = 0;
    __syncthreads();
    each([&](int, uint32_t k) __attribute__((always_inline)) {
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&hist[((k >> shift) & 255) * kCopies + (lane & (kCopies - 1))], 1);
    });
    __syncthreads();
    int mine = 0;
    const int digit = 255 - tid;  // thread 0 has the largest
    if (tid < 256)
      for (int c = 0; c < kCopies; ++c) mine += hist[digit * kCopies + ((c + lane) & (kCopies - 1))];
    int total;
    const int upto = scan_threads(mine, part, &total);
    if (tid < 256 && upto >= want && upto - mine < want) part[16] = digit, part[17] = want - (upto - mine);
    __syncthreads();
    prefix |= (uint32_t)part[16] << shift;
    want = part[17];
    __syncthreads();
  }
  // ---- a bit per slot: above the n-th key, equal to it (want of those stay, the lowest)
  each([&](int t, uint32_t k) __attribute__((always_inline)) {
    const uint64_t a = __ballot(k > prefix), e = __ballot(k == prefix);
    if (lane == 0 && (t >> 6) < p.words) above[t >> 6] = a, equal[t >> 6] = e;
  });
  __syncthreads();
  const int words = (L + 63) >> 6;
  for (int w0 = 0, ties = 0, gaps = 0, late = 0; w0 < words; w0 += kChooseThreads) {
    const int w = w0 + tid;
    const uint64_t e = w < words ? equal[w] : 0;
    int total;
    const int upto = scan_threads(ones(e), part, &total);
    const int take = want - (ties + upto - ones(e));  // of this word's ties
    ties += total;
    uint64_t kept = w < words ? above[w] : 0;
    if (take >= ones(e)) kept |= e;
    else if (take > 0) kept |= e & ((1ull << select_bit(e, take)) - 1);
    const int low = n - w * 64;  // slots of this word below n
    const uint64_t below = low >= 64 ? ~0ull : low > 0 ? (1ull << low) - 1 : 0;
    // gaps below n in the low half, kept slots from n on in the high half: neither sum passes 2^18
    const uint64_t mine = w < words ? (uint64_t)ones(~kept & below) | (uint64_t)ones(kept & ~below) << 32 : 0;
    uint64_t all;
    const uint64_t sums = scan_threads(mine, part64, &all) - mine;
    if (w < words) above[w] = kept, before[w] = gaps + (int)sums, rank0[w] = late + (int)(sums >> 32);
    gaps += (int)all, late += (int)(all >> 32);
    if (tid == 0) before[words] = gaps;  // (the last time: all of them)
  }
  __syncthreads();
  // ---- the map: the m-th gap is given the m-th kept slot from n on.  Gaps are listed by rank, as many as the list holds at a time (all
  // of them up to 16384 slots); a wave takes a word of slots
  const int n_gaps = before[words];
  for (int r0 = 0; r0 == 0 || r0 < n_gaps; r0 += p.list) {
    __syncthreads();
    for (int w = wave; w <= (n - 1) >> 6; w += kChooseWaves) {
      const uint64_t kept = above[w];
      const int t = w * 64 + lane;
      if (t >= n) continue;
      if (kept >> lane & 1) {
        if (r0 == 0) src[t] = t;
      } else {
        const int at = before[w] + ones(~kept & ((1ull << lane) - 1)) - r0;
        if (at >= 0 && at < p.list) list[at] = t;
      }
    }
    __syncthreads();
    for (int w = (n >> 6) + wave; w < words; w += kChooseWaves) {
      const uint64_t kept = above[w];
      const int t = w * 64 + lane, low = n - w * 64;
      const uint64_t late = low > 0 ? kept & (~0ull << low) : kept;
      const int at = rank0[w] + ones(late & ((1ull << lane) - 1)) - r0;
      if ((late >> lane & 1) && at >= 0 && at < p.list) src[list[at]] = t;
    }
  }
}

// ---------------------------------------------------------------------------------------
// the move
// ---------------------------------------------------------------------------------------
struct ShiftParams {
  const int32_t *n, *src;
  CacheView c;
  float *weight;
  int32_t *pos, *err_flag;
  int64_t ld, ld_src, layer_cache;  // layer_cache: units
  int B, H, Hkv, max_keep;
};

constexpr int kShiftWaves = 4;

// Grid: 256 slots, (sequence, head), layer; a wave takes 64 slots.
template <int D, int KIND>
__global__ void __launch_bounds__(64 * kShiftWaves) shift_kernel(const ShiftParams p) {
  constexpr int ROW = KIND == TVA_ROWS_BF16 ? D * 2 : KIND == TVA_ROWS_E4M3 ? D : D / 2;  // bytes
  constexpr int UNIT = KIND == TVA_ROWS_BF16 ? 2 : KIND == TVA_ROWS_E4M3 ? 1 : D / 2;
  constexpr int LPR = ROW / 16, RPI = 64 / LPR;  // lanes per row, rows at once
  __shared__ int64_t froms[kShiftWaves][64], tos[kShiftWaves][64];
  const int b = blockIdx.y / p.Hkv, g = blockIdx.y - b * p.Hkv, layer = blockIdx.z;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int n = min(p.n[b], p.max_keep);
  const int j = (blockIdx.x * kShiftWaves + wave) * 64 + lane;
  const int64_t r = ((int64_t)layer * p.B + b) * p.H + (p.H == 1 ? 0 : g);
  if (j - lane >= n) return;  // (a wave at a time; no barriers)
  const int old = j < n ? p.src[r * p.ld_src + j] : j;
  const int64_t room = room_of(p.c, b);
  const bool wrong = j < n && old != j && (old < p.n[b] || old >= room || j >= room || ((p.weight || p.pos) && old >= p.ld));
  if (wrong && p.err_flag) atomicCAS(p.err_flag, 0, 1 + b);
  const bool moves = j < n && old != j && !wrong;
  const uint64_t who = __ballot(moves);
  const int count = ones(who);
  if (moves) {
    const int at = ones(who & ((1ull << lane) - 1));
    const int64_t base = layer * p.layer_cache + g * p.c.stride_head;
    froms[wave][at] = base + position_at(p.c, b, old), tos[wave][at] = base + position_at(p.c, b, j);
    if (p.H != 1 || g == 0) {
      if (p.weight) p.weight[r * p.ld + j] = p.weight[r * p.ld + old];
      if (p.pos) p.pos[r * p.ld + j] = p.pos[r * p.ld + old];
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int piece = (lane % LPR) * 16;
#pragma unroll 2
  for (int i = lane / LPR; i < count; i += RPI) {
    const int64_t from = froms[wave][i], to = tos[wave][i];
    const u32x4 k = *(const u32x4 *)(p.c.k + from * UNIT + piece), v = *(const u32x4 *)(p.c.v + from * UNIT + piece);
    *(u32x4 *)(p.c.k + to * UNIT + piece) = k;
    *(u32x4 *)(p.c.v + to * UNIT + piece) = v;
    if constexpr (KIND == TVA_ROWS_E2M1) {
      if (lane % LPR == 0) {
        if constexpr (D == 128) ((uint32_t *)p.c.k_row_scale)[to] = ((const uint32_t *)p.c.k_row_scale)[from];
        else ((uint16_t *)p.c.k_row_scale)[to] = ((const uint16_t *)p.c.k_row_scale)[from];
        ((uint16_t *)p.c.v_row_scale)[to] = ((const uint16_t *)p.c.v_row_scale)[from];
      }
    }
  }
}

template <class F>
int by_kind(int D, int kind, F f) {
  auto of = [&](auto d) {
    if (kind == TVA_ROWS_BF16) f(d, std::integral_constant<int, TVA_ROWS_BF16>{});
    else if (kind == TVA_ROWS_E4M3) f(d, std::integral_constant<int, TVA_ROWS_E4M3>{});
    else f(d, std::integral_constant<int, TVA_ROWS_E2M1>{});
  };
  if (D == 128) of(std::integral_constant<int, 128>{});
  else of(std::integral_constant<int, 64>{});
  return hipPeekAtLastError() == hipSuccess ? TVA_OK : TVA_HIP_ERROR;
}

}  // namespace

extern "C" {

int tva_key_weights(const tva_key_weight_args *a, void *stream) {
  if (!a || a->B < 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv || a->max_rows < 0 || a->max_L < 0) return TVA_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return TVA_UNSUPPORTED;
  if (!(a->scale > 0.f) || a->ld < a->max_L) return TVA_INVALID_ARG;
  if (a->B == 0 || a->max_rows == 0 || a->max_L == 0) return TVA_OK;
  if (!a->cu_T || !a->L || !a->q || !a->lse || !a->weight || (a->path == nullptr) != (a->path_len == nullptr)) return TVA_INVALID_ARG;
  if (((uintptr_t)a->q & 15) || (a->pos && !a->first_pos)) return TVA_INVALID_ARG;
  WeighParams p{};
  const int rc = view_of(a->cache, a->Hkv, a->D, false, &p.c);
  if (rc != TVA_OK) return rc;
  p.cu_T = a->cu_T, p.path = a->path, p.path_len = a->path_len, p.L = a->L, p.first_pos = a->first_pos;
  p.q = (const __bf16 *)a->q, p.lse = a->lse, p.weight = a->weight, p.pos = a->pos, p.ld = a->ld;
  p.Hq = a->Hq, p.Hkv = a->Hkv, p.G = a->Hq / a->Hkv, p.max_rows = a->max_rows, p.max_L = a->max_L;
  const float ks = a->cache.kind == TVA_ROWS_E4M3 && a->cache.k_scale != 0.f ? a->cache.k_scale : 1.f;
  p.scale_log2 = a->scale * ks * kLog2e;
  // blocks per wave: as many as leave 4096 waves, at most 8 (16 x 16384 .. 32768 4-bit keys, before blocks that all rows
  // see had a form of their own, 66 us now: with 4 / 8 / 16 / 32 79 / 70.6 / 71.9 / 86 us)
  const int64_t all_blocks = ((int64_t)a->max_L + 31) / 32;
  p.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(8, all_blocks * a->B * a->Hkv / 4096));
  const int64_t waves = (all_blocks + p.blocks - 1) / p.blocks * a->Hkv, groups = (waves + kWeighWaves - 1) / kWeighWaves;
  if (a->B > 65535 || groups > 0x7fffffff || a->max_L > 1 << 29) return TVA_UNSUPPORTED;
  (void)hipGetLastError();
  return by_kind(a->D, a->cache.kind, [&](auto d, auto kind) {
    constexpr int D = decltype(d)::value, KIND = decltype(kind)::value;
    const dim3 grid((unsigned)groups, a->B), block(64 * kWeighWaves);
    if (a->cache.page_table) hipLaunchKernelGGL((weigh_kernel<D, KIND, true>), grid, block, 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL((weigh_kernel<D, KIND, false>), grid, block, 0, (hipStream_t)stream, p);
  });
}
size_t tva_sizeof_key_weight_args(void) { return sizeof(tva_key_weight_args); }

int tva_evict_select(const tva_evict_select_args *a, void *stream) {
  if (!a || a->B < 0 || a->H < 1 || a->max_L < 0 || a->n_layers < 0 || a->n_first < 0) return TVA_INVALID_ARG;
  if (a->max_L > TVA_EVICT_MAX_SLOTS) return TVA_UNSUPPORTED;
  if (a->ld < a->max_L || a->ld_src < 0) return TVA_INVALID_ARG;
  if (a->B == 0) return TVA_OK;
  if (!a->L || !a->keep || !a->weight || !a->src) return TVA_INVALID_ARG;
  if (a->L_out && (a->L_out == a->L || a->L_out == a->keep)) return TVA_INVALID_ARG;
  const int layers = a->n_layers > 0 ? a->n_layers : 1;
  if (a->B > 65535 || layers > 65535) return TVA_UNSUPPORTED;
  ChooseParams p{};
  p.L = a->L, p.keep = a->keep, p.newest = a->newest, p.pos = a->pos, p.weight = a->weight, p.src = a->src, p.L_out = a->L_out;
  p.ld = a->ld, p.ld_src = a->ld_src, p.B = a->B, p.H = a->H, p.max_L = a->max_L, p.n_first = a->n_first;
  p.words = (a->max_L + 63) / 64;
  p.list = std::min(a->max_L / 2 + 1, 8192);  // (there are no more gaps than kept slots behind them)
  const size_t bytes = (size_t)p.words * 24 + 4 + kChooseWaves * 8 + (256 * kCopies + 32 + p.list) * 4;
  const dim3 grid(a->H, a->B, layers), block(kChooseThreads);
  const hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  if (a->max_L <= 8 * kChooseThreads) hipLaunchKernelGGL(choose_kernel<8>, grid, block, bytes, st, p);
  else if (a->max_L <= 32 * kChooseThreads) hipLaunchKernelGGL(choose_kernel<32>, grid, block, bytes, st, p);
  else if (a->max_L <= 64 * kChooseThreads) hipLaunchKernelGGL(choose_kernel<64>, grid, block, bytes, st, p);
  else hipLaunchKernelGGL(choose_kernel<0>, grid, block, bytes, st, p);
  return hipPeekAtLastError() == hipSuccess ? TVA_OK : TVA_HIP_ERROR;
}
size_t tva_sizeof_evict_select_args(void) { return sizeof(tva_evict_select_args); }

int tva_evict_move(const tva_evict_move_args *a, void *stream) {
  if (!a || a->B < 0 || a->Hkv < 1 || a->max_keep < 0 || a->n_layers < 0 || (a->H != 1 && a->H != a->Hkv)) return TVA_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return TVA_UNSUPPORTED;
  if (a->ld_src < a->max_keep || a->layer_stride_cache < 0 || ((a->weight || a->pos) && a->ld < a->max_keep)) return TVA_INVALID_ARG;
  if (a->B == 0 || a->max_keep == 0) return TVA_OK;
  if (!a->n || !a->src) return TVA_INVALID_ARG;
  ShiftParams p{};
  const int rc = view_of(a->cache, a->Hkv, a->D, true, &p.c);
  if (rc != TVA_OK) return rc;
  const int unit = a->cache.kind == TVA_ROWS_E2M1 ? a->D : a->cache.kind == TVA_ROWS_E4M3 ? 16 : 8;
  if (a->layer_stride_cache % unit) return TVA_INVALID_ARG;
  const int layers = a->n_layers > 0 ? a->n_layers : 1;
  if ((int64_t)a->B * a->Hkv > 65535 || layers > 65535) return TVA_UNSUPPORTED;
  p.n = a->n, p.src = a->src, p.weight = a->weight, p.pos = a->pos, p.err_flag = a->err_flag, p.ld = a->ld, p.ld_src = a->ld_src;
  p.layer_cache = a->cache.kind == TVA_ROWS_E2M1 ? a->layer_stride_cache / a->D : a->layer_stride_cache;
  p.B = a->B, p.H = a->H, p.Hkv = a->Hkv, p.max_keep = a->max_keep;
  const dim3 grid((a->max_keep + 64 * kShiftWaves - 1) / (64 * kShiftWaves), a->B * a->Hkv, layers);
  (void)hipGetLastError();
  return by_kind(a->D, a->cache.kind, [&](auto d, auto kind) {
    hipLaunchKernelGGL((shift_kernel<decltype(d)::value, decltype(kind)::value>), grid, dim3(64 * kShiftWaves), 0, (hipStream_t)stream, p);
  });
}
size_t tva_sizeof_evict_move_args(void) { return sizeof(tva_evict_move_args); }

}  // extern "C"
