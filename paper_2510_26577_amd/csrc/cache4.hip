// libtva: caches of 4-bit rows (gfx950).  Entry points and formats: include/tva_cache.h.
//
//   store_rows_kernel  bf16 rows -> 4-bit rows: 8 elements per lane, D/8 lanes per row; the largest magnitudes (of 32
//                      elements for K, of the row for V) are integer maxima of bf16 bits over neighbouring lanes.
//   load_rows_kernel   the inverse.
//   four_bit_kernel    the verification attention: S^T = K Q^T and O^T = V^T P^T by 32x32x16 bf16 MFMAs, as in
//                      tva.hip, on tiles of 64 keys that every wave streams for itself.  A tile is 8.6 KB (D = 128), a
//                      quarter of a bf16 one, so that the next one waits in registers: K's bytes are the
//                      operand's own lanes' (a lane's key, half of the elements) and are widened there; V's pass
//                      through 4 KB of LDS that belong to the wave, because the transposing read (16 x 16 codes per 16
//                      lanes) wants rows.  No barrier in the loop.
//   join_kernel        merges the partial results of sequences that several workgroups share.
// Work is dealt out on the device (struct Deal): equal runs of tiles, whatever the sequences' lengths.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cache_rows.h"
#include "tva.h"
#include "tva_cache.h"

namespace {

using namespace cache_rows;

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------------------------------
// rows in, rows out
// ---------------------------------------------------------------------------------------
struct RowsParams {
  const int32_t *cu_T, *L, *path, *path_len;
  uint16_t *k_rows, *v_rows;
  CacheView c;
  int32_t *L_out, *err_flag;
  int Hkv, max_rows, n_layers;
  int64_t layer_rows;   // elements of k_rows / v_rows between layers
  int64_t layer_cache;  // rows of the cache between layers
};

// The row of k_rows / v_rows and the cache row of (sequence, j, head): false if there is none.
__device__ __forceinline__ bool find_row(const RowsParams &p, int b, int j, int g, int64_t *from, int64_t *to) {
  const int t0 = p.cu_T[b], T = p.cu_T[b + 1] - t0;
  int n = p.path ? p.path_len[b] : T;
  if (j >= (n < p.max_rows ? n : p.max_rows)) return false;
  const int node = p.path ? p.path[(int64_t)b * p.max_rows + j] : j;
  const int64_t pos = (int64_t)p.L[b] + j;
  if (node < 0 || node >= T || pos < 0 || pos >= room_of(p.c, b)) {
    if (p.err_flag && g == 0) atomicCAS(p.err_flag, 0, 1 + b);
    return false;
  }
  *from = (int64_t)t0 + node;
  *to = position_at(p.c, b, (int)pos) + g * p.c.stride_head;
  return true;
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
__device__ uint32_t codes_of(const u16x8 x, float s) {
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

// Layers that a workgroup takes its rows of at once: what leads to a row (lengths, path, page) is read once for them.
constexpr int kRowLayers = 4;

template <int D>
__global__ void __launch_bounds__(256) store_rows_kernel(const RowsParams p) {
  constexpr int LPR = D / 8;  // lanes per row
  const int b = blockIdx.y, layer0 = blockIdx.z * kRowLayers, here = min(p.n_layers - layer0, kRowLayers);
  const int idx = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, part = threadIdx.x % LPR;
  const int j = idx / p.Hkv, g = idx - j * p.Hkv;
  if (idx == 0 && part == 0 && layer0 == 0 && p.L_out) {
    const int n = p.path ? p.path_len[b] : p.cu_T[b + 1] - p.cu_T[b];
    p.L_out[b] = p.L[b] + (n < p.max_rows ? n : p.max_rows);
  }
  int64_t from, to;
  if (!find_row(p, b, j, g, &from, &to)) return;  // (the lanes of a row leave together)
  to += layer0 * p.layer_cache;
  const int64_t e = layer0 * p.layer_rows + (from * p.Hkv + g) * D + part * 8;
  u16x8 ks[kRowLayers], vs[kRowLayers];
#pragma unroll
  for (int l = 0; l < kRowLayers; ++l) {
    const int64_t at = e + min(l, here - 1) * p.layer_rows;
    ks[l] = *(const u16x8 *)(p.k_rows + at), vs[l] = *(const u16x8 *)(p.v_rows + at);
  }
#pragma unroll
  for (int l = 0; l < kRowLayers; ++l, to += p.layer_cache) {
    if (l >= here) return;
    const u16x8 k = ks[l], v = vs[l];
    bool fk, fv;
    uint32_t ak = largest(k, &fk), av = largest(v, &fv);
#pragma unroll
    for (int o = 1; o < LPR; o *= 2) {
      if (o < 4) ak = max(ak, (uint32_t)__shfl_xor((int)ak, o));
      av = max(av, (uint32_t)__shfl_xor((int)av, o));
    }
    // K: a = (1 + m/128) 2^(E-127) <= 6 * 2^e
    const int ek = (int)(ak >> 7) - 127 - ((ak & 127) > 64 ? 1 : 2), e2 = min(max(ek, -96), 124);
    // V: a = n/256 * 2^(E-126), the quotient by 6 rounded up to four bits
    const int n = 128 + (int)(av & 127), ev = (int)(av >> 7) - 126;
    const float sv = fminf(fmaxf(n < 192 ? ldexpf((float)((n + 11) / 12), ev - 7) : ldexpf((float)((n + 23) / 24), ev - 6), 0x1p-96f), 0x1p124f);
    const float sk = exponent_byte((uint32_t)(e2 + 127));
    const bool plain = fk && fv && ek == e2 && sv > 0x1p-96f && sv < 0x1p124f;  // (else: what the instructions would do is not asked)
    uint32_t wk = codes_k(k, sk), wv = codes_v(v, sv);
    if (!plain) wk = codes_of(k, sk), wv = codes_of(v, sv);
    ((uint32_t *)p.c.k)[to * LPR + part] = wk;
    ((uint32_t *)p.c.v)[to * LPR + part] = wv;
    if (part % 4 == 0) ((uint8_t *)p.c.k_row_scale)[to * (D / 32) + part / 4] = (uint8_t)(e2 + 127);
    if (part == 0) ((uint16_t *)p.c.v_row_scale)[to] = (uint16_t)(__float_as_uint(sv) >> 16);
  }
}

template <int D>
__global__ void __launch_bounds__(256) load_rows_kernel(const RowsParams p) {
  constexpr int LPR = D / 8;
  const int b = blockIdx.y, layer0 = blockIdx.z * kRowLayers, here = min(p.n_layers - layer0, kRowLayers);
  const int idx = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, part = threadIdx.x % LPR;
  const int j = idx / p.Hkv, g = idx - j * p.Hkv;
  int64_t to, from;
  if (!find_row(p, b, j, g, &to, &from)) return;
  from += layer0 * p.layer_cache;
  const int64_t e = layer0 * p.layer_rows + (to * p.Hkv + g) * D + part * 8;
  uint32_t k[kRowLayers], v[kRowLayers], sk[kRowLayers], sv[kRowLayers];
#pragma unroll
  for (int l = 0; l < kRowLayers; ++l) {
    const int64_t at = from + min(l, here - 1) * p.layer_cache;
    k[l] = ((const uint32_t *)p.c.k)[at * LPR + part], v[l] = ((const uint32_t *)p.c.v)[at * LPR + part];
    sk[l] = ((const uint8_t *)p.c.k_row_scale)[at * (D / 32) + part / 4], sv[l] = ((const uint16_t *)p.c.v_row_scale)[at];
  }
#pragma unroll
  for (int l = 0; l < kRowLayers; ++l) {
    if (l >= here) return;
    *(bf16x8 *)(p.k_rows + e + l * p.layer_rows) = widen8(k[l], exponent_byte(sk[l]));
    bf16x8 x = widen8(v[l], 1.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)((float)x[i] * __uint_as_float(sv[l] << 16));  // (at most 6 bits: exact)
    *(bf16x8 *)(p.v_rows + e + l * p.layer_rows) = x;
  }
}

// ---------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------
struct FourParams {
  const __bf16 *q, *k_tree, *v_tree;
  const int32_t *cu_T, *L, *parent;
  const uint64_t *mask;
  CacheView c;
  __bf16 *out;
  float *lse;
  float *part_out, *part_lse;  // [slots, Hkv, rows, D], [slots, Hkv, rows]
  int B, Hq, Hkv, G, W, max_L;
  int group, parts, rows;  // sequences whose tiles are dealt out together (1, or up to 64), among how many; rows of a slot
  float scale_log2;
};

// How the tiles of a group of sequences (64 cached keys each, and 64 of the tree's own) are dealt out: in order, in `parts` runs that
// differ by one tile at most, for one head and block of query rows.  A run may end inside a sequence and go on in the next: lengths
// that differ cost no balance, and the host need not know them.  A sequence that lies in one run is finished there; of others
// each run leaves a partial result (in slot run + sequence, which no two share) for join_kernel, which deals out the same way.
// A sequence by itself (group 1) has its tree's keys in a run of their own: such runs are short, and a tree's tile lasts as long as
// three of the cache.
struct Deal {
  int upto, tiles, t0, T, L;  // this lane's sequence: tiles of the group up to its end, its own; its first node, nodes, cached keys
  int total, parts;           // tiles and runs of the group
  int even, even_parts;       // tiles that are dealt out evenly, and among how many runs (the rest is the last run)
  __device__ __forceinline__ Deal(const FourParams &p, int first, int row0) {
    tiles = t0 = T = L = 0;
    if (p.group == 1) {
      t0 = p.cu_T[first], T = min(p.cu_T[first + 1] - t0, TVA_MAX_TREE), L = min(max(p.L[first], 0), p.max_L);
      const int cached = (L + 63) >> 6;
      if (T * p.G > row0) tiles = cached + ((T + 63) >> 6);
      upto = total = tiles;
      even = p.parts > 1 ? cached : total, even_parts = min(p.parts > 1 ? p.parts - 1 : 1, even);
      parts = total == 0 ? 0 : even_parts + (even < total);
    } else {
      const int lane = threadIdx.x & 63, b = first + lane;
      if (lane < p.group && b < p.B) {
        t0 = p.cu_T[b], T = min(p.cu_T[b + 1] - t0, TVA_MAX_TREE), L = min(max(p.L[b], 0), p.max_L);
        if (T * p.G > row0) tiles = ((L + 63) >> 6) + ((T + 63) >> 6);
      }
      upto = tiles;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
      }
      even = total = __builtin_amdgcn_readlane(upto, 63), even_parts = parts = min(p.parts, total);
    }
  }
  __device__ __forceinline__ static int divide(int64_t x, int y) { return x >> 32 ? (int)(x / y) : (int)((uint32_t)x / (uint32_t)y); }
  // the first tile of run i (i = parts: the end), and the run that tile x lies in
  __device__ __forceinline__ int begin(int i) const { return i < even_parts ? divide((int64_t)i * even, even_parts) : i < parts ? even : total; }
  __device__ __forceinline__ int run_of(int x) const { return x < even ? divide((int64_t)(x + 1) * even_parts + even - 1, even) - 1 : parts - 1; }
};

__device__ __forceinline__ float half_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

constexpr int kWaves = 4;

// A weight is rounded to bf16, the operand's type: half a step, 2^-8 of it.  Where many keys share a row the roundings cancel below that of
// the result; where few do they show.  So what the rounding leaves is multiplied too (2^-17 of a weight is then off) wherever a row's
// largest weight in a tile is more than this share of what the row has summed: no weight beyond an eighth of its row goes without.
constexpr float kLoThreshold = 0.125f;
// What is left of two numbers when their bf16 roundings (h) are taken from them, as bf16.  One instruction each, two where the
// rounding is widened first.  Its second operands, (-1, 0) and (0, -1), are in registers: as inline constants they are not read as bf16.
struct Remainders {
  uint32_t first = 0xbf80u, second = 0xbf800000u;
  __device__ __forceinline__ Remainders() { asm("" : "+s"(first), "+s"(second)); }
  __device__ __forceinline__ bf16x2 of(float x, float y, bf16x2 h) const {
    return bf16x2{(__bf16)__builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, first), x, false),
                  (__bf16)__builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, second), y, false)};
  }
};

// whether any of eight bf16 numbers is infinite or NaN
__device__ __forceinline__ bool not_finite(u32x4 x) {
  bool any = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) any |= (x[k] & 0x7f80) == 0x7f80 || (x[k] & 0x7f800000) == 0x7f800000;
  return any;
}

template <bool ONCE>
__device__ __forceinline__ u32x4 read16(const char *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4 *)p);
  else return *(const u32x4 *)p;
}

template <int D>
struct FourCfg {
  static constexpr int NS = D / 16;          // QK steps of 16 elements
  static constexpr int NJ = D / 32;          // 32-wide blocks of the output
  static constexpr int RB = D / 2;           // bytes of a row
  static constexpr int CH = RB / 16;         // 16-byte pieces of a row = wave-wide loads of a V tile
  static constexpr int RPL = 64 / CH;        // rows such a load covers
  static constexpr int KL = RB / 32;         // 16-byte pieces of a lane's half of a K row
  static constexpr int VT = 64 * RB;         // V tile
  // a wave's LDS: the V tile and its 64 scales; for a tree tile, NB blocks of bf16 rows n, n + NB, n + 2 NB ..., 32 bytes apart, so
  // that the four consecutive rows a transposing read takes together are in different banks
  static constexpr int NB = D / 8, BLK = 1024 + 32;
  static constexpr int WAVE_LDS = NB * BLK;
  static_assert(VT + 256 <= WAVE_LDS, "");
  static constexpr int TP = D + 4;           // floats between rows of an output patch
  static constexpr int PATCH = 32 * TP * 4;
  static constexpr int EXCHANGE = 2 * kWaves * 32 * 4;  // maxima and sums
  static constexpr int TREE = TVA_MAX_TREE * 4;
  static constexpr int LOOP_LDS = kWaves * WAVE_LDS + TREE;
  static constexpr int END_LDS = kWaves * PATCH + EXCHANGE;
  static constexpr int LDS = LOOP_LDS > END_LDS ? LOOP_LDS : END_LDS;
};

// Grid: KV head (fastest: with 8 heads one per XCD), block of WM * 32 query rows, run of tiles.  The four waves are WM row groups x
// 4 / WM key groups; every (4 / WM)th tile of a run's part of a sequence belongs to a key group.
// PG: 0 dense, 1 paged, 2 paged with pages of whole tiles (one table entry per tile, and as in the dense form addresses that are a
// scalar and a lane's offset).
// FORM kAlways: remainders in every tile, not in a block of their own where some row needs them.  So where several 32-row blocks share the
// keys, which is work of a few tiles per wave that need them all, or of three blocks (one sequence of 2048 keys, 60 nodes: 15.4 us, 16.6
// with the block, 14.5 without remainders); else few tiles need them (64 sequences of 4096 .. 16384 keys, 8 nodes: 182 us, 165, 160; 4
// of 16384 .. 32768, 48 nodes: 141 us, 124, 117).
// FORM kOnce: keys are read by nontemporal loads, where one block of rows reads them, a head's rows lie side by side and all of them are
// more than the last-level cache holds (64 sequences of 4096 .. 16384 keys, 8 nodes, head-major: 167 -> 164 us; 4 of 16384 .. 32768,
// which it holds, 40 -> 42; heads of a token-major cache share lines: 250 -> 306, 16 sequences of 2048 .. 4096 keys 34 -> 54).
enum { kPlain, kAlways, kOnce };
constexpr int64_t kLastLevel = 256ll << 20;  // bytes
template <int D, int WM, int PG, int FORM>
__global__ void __launch_bounds__(256, 2) four_bit_kernel(const FourParams p) {
  typedef FourCfg<D> C;
  constexpr int WK = kWaves / WM;
  constexpr bool ALWAYS = FORM == kAlways, ONCE = FORM == kOnce;
  __shared__ __align__(16) unsigned char lds[C::LDS];
  const int g = blockIdx.x, which = blockIdx.z / p.parts, run = blockIdx.z - which * p.parts;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wm = wave % WM, wk = wave / WM;
  const int row0 = blockIdx.y * (WM * 32);
  const Deal deal(p, which * p.group, row0);
  if (run >= deal.parts) return;
  int at_tile = deal.begin(run);
  const int stop = deal.begin(run + 1);

  while (true) {  // the run's part of one sequence after the other
    const int lb = __builtin_ctzll(__ballot(deal.upto > at_tile)), b = which * p.group + lb;
    const int tiles = __builtin_amdgcn_readlane(deal.tiles, lb), seq_end = __builtin_amdgcn_readlane(deal.upto, lb);
    const int x0 = at_tile - (seq_end - tiles), x1 = min(stop, seq_end) - (seq_end - tiles);  // of the sequence's tiles
    const bool whole = x1 - x0 == tiles;
    const int t0 = __builtin_amdgcn_readlane(deal.t0, lb), T = __builtin_amdgcn_readlane(deal.T, lb), L = __builtin_amdgcn_readlane(deal.L, lb);
    const int n_rows = T * p.G;
    const int n_cache = (L + 63) >> 6;

    // this lane's query row (column of S^T and O^T); rows past the end repeat the last one and are not written
    const int row = min(row0 + wm * 32 + l32, n_rows - 1);
    const int node = row / p.G, head = g * p.G + (row - node * p.G);
    const bool idle = row0 + wm * 32 >= n_rows;

    unsigned char *vt = lds + wave * C::WAVE_LDS;
    float *vsl = (float *)(vt + C::VT);

    // ---- what waits in registers: K and V bytes of a tile and their scales ----
    u32x4 kx[2][C::KL], vx[C::CH];
    // (scales stay in 16 bits, and what uses them takes the bits it needs: widened, the compiler lets them wait in the loop for what was
    // only just asked for)
    uint16_t ks[2], vs;
    const Finder<PG != 0> find(p.c, b, g);
    int entry = 0;        // the page of key `lane` of the tile after next (PG 2: of all its keys)
    uint32_t rs = 0;      // PG 1: the row of key `lane`
    int64_t base = 0;     // else: the row of the tile's first key
    const uint32_t step = (uint32_t)p.c.stride_tok;
    int last = 63;        // rows of the tile past its last key repeat that one and are masked
    const int cache_end = min(x1, n_cache);
    auto look = [&](int tile) __attribute__((always_inline)) {
      tile = min(tile, cache_end - 1);
      if constexpr (PG == 1) entry = find.entry(p.c, min(tile * 64 + lane, L - 1));
      if constexpr (PG == 2) entry = find.entry(p.c, tile * 64);
    };
    auto place = [&](int tile) __attribute__((always_inline)) {
      last = min(63, L - 1 - tile * 64);
      if constexpr (PG == 1) rs = (uint32_t)find.at(p.c, min(tile * 64 + lane, L - 1), entry);  // (row numbers have 32 bits)
      else base = find.at(p.c, tile * 64, __builtin_amdgcn_readfirstlane(entry));
    };
    // key r's row (PG 1), or its distance from the tile's first; and byte `at` of that row in a tensor of `size` bytes per row, where it
    // can be as a scalar and a lane's 32-bit offset
    auto row_of = [&](int r) __attribute__((always_inline)) -> uint32_t {
      if constexpr (PG == 1) return (uint32_t)__shfl((int)rs, r);
      else return __umul24(min(r, last), step);
    };
    auto byte_of = [&](const char *from, uint32_t row, int size, int at) __attribute__((always_inline)) -> const char * {
      if constexpr (PG == 1) return from + ((uint64_t)row * (uint32_t)size + (uint32_t)at);
      else return from + base * size + (uint32_t)(row * (uint32_t)size + at);
    };
    // What a lane works out from its number is worked out again in every tile: kept, it takes the registers that the loop needs, and
    // what is then read back from memory waits for all loads on their way.
    auto afresh = [&](int tile) __attribute__((always_inline)) {
      int x;
      asm("" : "=v"(x) : "0"(lane), "s"(tile));
      return x;
    };
    auto fetch_k = [&](int tile) __attribute__((always_inline)) {
      const int ln = afresh(tile), hf = ln >> 5;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t row = row_of(kb * 32 + (ln & 31));
        const char *from = byte_of(p.c.k, row, C::RB, hf * (C::RB / 2));
#pragma unroll
        for (int i = 0; i < C::KL; ++i) kx[kb][i] = read16<ONCE>(from + i * 16);
        if constexpr (D == 128) ks[kb] = *(const uint16_t *)byte_of(p.c.k_row_scale, row, 4, hf * 2);
        else ks[kb] = *(const uint8_t *)byte_of(p.c.k_row_scale, row, 2, hf);
      }
    };
    auto fetch_v = [&](int tile) __attribute__((always_inline)) {
      const int ln = afresh(tile);
#pragma unroll
      for (int i = 0; i < C::CH; ++i) vx[i] = read16<ONCE>(byte_of(p.c.v, row_of(i * C::RPL + ln / C::CH), C::RB, (ln % C::CH) * 16));
      if constexpr (PG == 1) vs = *(const uint16_t *)(p.c.v_row_scale + (uint64_t)rs * 2);
      else vs = *(const uint16_t *)byte_of(p.c.v_row_scale, row_of(ln), 2, 0);
    };

    int tile = x0 + wk;
    if (!idle && tile < cache_end) look(tile), place(tile), fetch_k(tile), fetch_v(tile), look(tile + WK);

    bf16x8 q[C::NS];
    const __bf16 *qrow = p.q + ((int64_t)(t0 + node) * p.Hq + head) * D + half * (D / 2);
#pragma unroll
    for (int s = 0; s < C::NS; ++s) q[s] = *(const bf16x8 *)(qrow + s * 8);

    // ancestor set of this lane's node, trimmed to the tree
    uint64_t anc0 = 0, anc1 = 0;
    if (x1 > n_cache) {
      if (p.mask) {
        const uint64_t *w = p.mask + (int64_t)(t0 + node) * p.W;
        anc0 = w[0];
        if (p.W > 1) anc1 = w[1];
      } else {
        int32_t *par = (int32_t *)(lds + kWaves * C::WAVE_LDS);
        if (tid < T) par[tid] = p.parent[t0 + tid];
        __syncthreads();
        int a = node;
        for (int step = 0; step < TVA_MAX_TREE; ++step) {
          if (a < 64) anc0 |= 1ull << a;
          else anc1 |= 1ull << (a - 64);
          const int up = par[a];
          if (up < 0 || up >= a) break;
          a = up;
        }
      }
      if (T < 64) anc0 &= (1ull << T) - 1, anc1 = 0;
      else if (T < 128) anc1 &= (1ull << (T - 64)) - 1;
    }

    f32x16 acc[C::NJ];
#pragma unroll
    for (int j = 0; j < C::NJ; ++j) acc[j] = f32x16{};
    float m = -INFINITY, l = 0.f;  // reference (log2 domain) and sum over this lane half's keys
    f32x16 s[2];
    // scores -> probabilities in place (log2 domain, fp32), O and l moved to a new reference where a row's maximum grew.  Returns whether
    // a row's largest one is beyond kLoThreshold.
    auto soften = [&]() __attribute__((always_inline)) -> bool {
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
      top = half_max(top) * p.scale_log2;
      // the reference moves only when it is exceeded by more than 2^8: probabilities stay below that
      if (__any(top > m + 8.f)) {
        const float to = fmaxf(m, top);
        const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
        m = to, l *= f;
#pragma unroll
        for (int j = 0; j < C::NJ; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[j][i] *= f;
      }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], p.scale_log2, -ref));
          l += s[kb][i];
        }
      return __any(__builtin_amdgcn_exp2f(top - ref) > kLoThreshold * half_sum(l));
    };
    const Remainders remainders;

    if (!idle) {
      for (; tile < cache_end; tile += WK) {
        // ---- S^T = K Q^T
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[kb] = f32x16{};
#pragma unroll
        for (int st = 0; st < C::NS; ++st)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const float sc = __uint_as_float(((uint32_t)ks[kb] << (st < C::NS / 2 || D == 64 ? 23 : 15)) & 0x7f800000u);  // exponent_byte
            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(kx[kb][st / 4][st % 4], sc), q[st], s[kb], 0, 0, 0);
          }
        const int left = L - tile * 64;
        // (the next tile, or the last one again: a branch here would leave the waits without a count to go by)
        place(min(tile + WK, cache_end - 1)), fetch_k(tile), look(tile + 2 * WK);
        if (left < 64) {
          const int mine = left - 4 * (afresh(tile) >> 5);
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (kb * 32 + 8 * (i / 4) + i % 4 >= mine) s[kb][i] = -INFINITY;
        }
        const bool fine = soften();
        const int ln = afresh(tile);
        // ---- V to LDS: piece c of row r lies at piece c ^ (r / 8) of its row, so that the 16 rows a transposing read takes
        // together (4 consecutive ones of each 8) are in different banks
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < C::CH; ++i) {
          const int r = i * C::RPL + ln / C::CH;
          *(u32x4 *)(vt + r * C::RB + (((ln % C::CH) ^ (r >> 3)) & (C::CH - 1)) * 16) = vx[i];
        }
        vsl[ln] = __uint_as_float((uint32_t)vs << 16);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        fetch_v(tile);
        // ---- O^T += V^T (P s_v)^T; codes are widened as they are, their row's scale is in the weight and rounded to bf16 with it
        // Remainders in a block of their own, which reads its operands for itself: kept for it, they would take registers in every tile.
        // (With ALWAYS: below.)
        if (!ALWAYS && fine) {
          int ln;
          asm volatile("" : "=v"(ln) : "0"(lane) : "memory");
          const int i16 = ln & 15, sub = (ln >> 4) & 1;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const int r = kb * 32 + 8 * (i16 >> 2) + 4 * (ln >> 5) + (i16 & 3);
            bf16x8 w[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 sc = *(const f32x4 *)(vsl + kb * 32 + 8 * i + 4 * (ln >> 5));
#pragma unroll
              for (int k = 0; k < 4; k += 2) {
                const float x = s[kb][i * 4 + k] * sc[k], y = s[kb][i * 4 + k + 1] * sc[k + 1];
                const bf16x2 rest = remainders.of(x, y, bf16x2{(__bf16)x, (__bf16)y});
                w[i / 2][(i % 2) * 4 + k] = rest[0], w[i / 2][(i % 2) * 4 + k + 1] = rest[1];
              }
            }
#pragma unroll
            for (int j = 0; j < C::NJ; ++j) {
              const i32x2 x = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
                  (__attribute__((address_space(3))) i32x2 *)(vt + r * C::RB + ((j ^ (r >> 3)) & (C::CH - 1)) * 16 + sub * 8));
#pragma unroll
              for (int a = 0; a < 2; ++a) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8((uint32_t)x[a], 1.f), w[a], acc[j], 0, 0, 0);
            }
          }
        }
        if constexpr (!ALWAYS) asm volatile("" ::: "memory");
        // (all operands are read ahead: each where it is used, 4 sequences of 16384 .. 32768 keys, 48 nodes, take 124 us instead of 117, before remainders)
        i32x2 c[2][C::NJ];
        f32x4 sc[2][4];
        {
          // this lane's row of the 16 x 16 codes its 16 lanes turn over: key slot i of its half, 8 bytes of elements
          const int i16 = ln & 15, sub = (ln >> 4) & 1;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const int r = kb * 32 + 8 * (i16 >> 2) + 4 * (ln >> 5) + (i16 & 3);
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[kb][i] = *(const f32x4 *)(vsl + kb * 32 + 8 * i + 4 * (ln >> 5));
#pragma unroll
            for (int j = 0; j < C::NJ; ++j)
              c[kb][j] = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
                  (__attribute__((address_space(3))) i32x2 *)(vt + r * C::RB + ((j ^ (r >> 3)) & (C::CH - 1)) * 16 + sub * 8));
          }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          bf16x8 w[2], low[2];
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
              const float x = s[kb][i * 4 + k] * sc[kb][i][k], y = s[kb][i * 4 + k + 1] * sc[kb][i][k + 1];
              const bf16x2 h = {(__bf16)x, (__bf16)y};
              w[i / 2][(i % 2) * 4 + k] = h[0], w[i / 2][(i % 2) * 4 + k + 1] = h[1];
              if constexpr (ALWAYS) {
                const bf16x2 rest = remainders.of(x, y, h);
                low[i / 2][(i % 2) * 4 + k] = rest[0], low[i / 2][(i % 2) * 4 + k + 1] = rest[1];
              }
            }
#pragma unroll
          for (int j = 0; j < C::NJ; ++j)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const bf16x8 v = widen8((uint32_t)c[kb][j][a], 1.f);
              acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[a], acc[j], 0, 0, 0);
              if constexpr (ALWAYS) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, low[a], acc[j], 0, 0, 0);
            }
        }
      }
      // ---- the tree's own keys, bf16: V goes to LDS while K's rows are fetched and multiplied
      for (; tile < x1; tile += WK) {
        const int first = (tile - n_cache) * 64, left = T - first;
        const int lane = afresh(tile), l32 = lane & 31, half = lane >> 5;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int n = 0; n < C::NB; ++n) {
          const int r = first + n + C::NB * (lane / C::NB);
          const __bf16 *from = p.v_tree + ((int64_t)(t0 + min(r, T - 1)) * p.Hkv + g) * D + (lane % C::NB) * 8;
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                           (__attribute__((address_space(3))) void *)(vt + n * C::BLK), 16, 0, 0);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
          const int key = first + kb * 32 + l32;
          const __bf16 *krow = p.k_tree + ((int64_t)(t0 + min(key, T - 1)) * p.Hkv + g) * D + half * (D / 2);
          if (kb * 32 < left) {
#pragma unroll
            for (int st = 0; st < C::NS; ++st)
              s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)(krow + st * 8), q[st], s[kb], 0, 0, 0);
          }
          const uint64_t word = first ? anc1 : anc0;
          const uint32_t bits = (uint32_t)(word >> (kb * 32));
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!((bits >> (8 * (i / 4) + 4 * half + i % 4)) & 1)) s[kb][i] = -INFINITY;
        }
        (void)soften();
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): V is in LDS
        asm volatile("" ::: "memory");
        // A node's V may hold what is not finite, and rows that do not see the node must not (0 * inf is NaN): such elements are taken
        // out of the tile, and rows that see them get them added
        bool odd = false;
#pragma unroll
        for (int n = 0; n < C::NB; ++n) odd |= not_finite(*(const u32x4 *)(vt + n * C::BLK + lane * 16));
        if (__any(odd)) {
          for (int n = 0; n < C::NB; ++n) {
            u32x4 x = *(const u32x4 *)(vt + n * C::BLK + lane * 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if ((x[k] & 0x7f80) == 0x7f80) x[k] &= 0xffff0000u;
              if ((x[k] & 0x7f800000) == 0x7f800000) x[k] &= 0xffffu;
            }
            *(u32x4 *)(vt + n * C::BLK + lane * 16) = x;
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          for (int k = 0; k < min(left, 64); ++k) {
            const bool sees = ((first ? anc1 : anc0) >> k) & 1;
            const __bf16 *vrow = p.v_tree + ((int64_t)(t0 + first + k) * p.Hkv + g) * D + 4 * half;
#pragma unroll
            for (int j = 0; j < C::NJ; ++j)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float v = (float)vrow[32 * j + 8 * (i / 4) + i % 4];
                if (sees && !__builtin_isfinite(v)) acc[j][i] += v;
              }
          }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            if (kb * 32 + a * 16 >= left) continue;
            bf16x8 w, low;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const bf16x2 h = {(__bf16)s[kb][a * 8 + i], (__bf16)s[kb][a * 8 + i + 1]}, rest = remainders.of(s[kb][a * 8 + i], s[kb][a * 8 + i + 1], h);
              w[i] = h[0], w[i + 1] = h[1], low[i] = rest[0], low[i + 1] = rest[1];
            }
            // 16 lanes turn over 4 rows x 16 elements: this lane's row (of keys 8 c + 4 half + 0..3) and 8-byte piece of it
            const int i16 = lane & 15, sub = (lane >> 4) & 1;
#pragma unroll
            for (int j = 0; j < C::NJ; ++j) {
              s16x4 c[2];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int r = 32 * kb + 16 * a + 8 * h + 4 * half + (i16 >> 2);
                c[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4 *)(vt + (r % C::NB) * C::BLK + (r / C::NB) * (D * 2) + j * 64 + sub * 32 + (i16 & 3) * 8));
              }
              const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(c[0], c[1], 0, 1, 2, 3, 4, 5, 6, 7));
              acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w, acc[j], 0, 0, 0);
              acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, low, acc[j], 0, 0, 0);  // (a tree's keys are few: in any case)
            }
          }
      }
    }

    // ---- the key groups' results joined, and O^T turned over to rows ----
    l = half_sum(l);
    __syncthreads();
    float *patch = (float *)lds, *maxima = (float *)(lds + kWaves * C::PATCH), *sums = maxima + kWaves * 32;
    if (half == 0) maxima[wave * 32 + l32] = m, sums[wave * 32 + l32] = l;
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < WK; ++k) top = fmaxf(top, maxima[(k * WM + wm) * 32 + l32]);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 x;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = acc[j][i * 4 + k] * f;
        *(f32x4 *)(patch + wave * (32 * C::TP) + l32 * C::TP + j * 32 + 8 * i + 4 * half) = x;
      }
    __syncthreads();
    constexpr int PIECES = WM * 32 * (D / 4);
    const int64_t slot = ((int64_t)(which * (p.parts + p.group) + run + lb) * p.Hkv + g) * p.rows;
    for (int x = tid; x < PIECES; x += 256) {
      const int r = x / (D / 4), d = (x - r * (D / 4)) * 4, w = r >> 5, rr = r & 31;
      if (row0 + r >= n_rows) break;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      float top_r = -INFINITY, sum = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) top_r = fmaxf(top_r, maxima[(k * WM + w) * 32 + rr]);
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const int at = k * WM + w;
        o += *(const f32x4 *)(patch + at * (32 * C::TP) + rr * C::TP + d);
        const float mk = maxima[at * 32 + rr];
        sum += mk == -INFINITY ? sums[at * 32 + rr] : sums[at * 32 + rr] * __builtin_amdgcn_exp2f(mk - top_r);  // (0, or NaN)
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;  // (NaN stays NaN)
      o *= inv;
      const float lse = sum == 0.f ? -INFINITY : (top_r + __builtin_amdgcn_logf(sum)) * kLn2;  // (logf: base 2)
      if (whole) {
        const int rnode = (row0 + r) / p.G, rhead = g * p.G + (row0 + r - rnode * p.G);
        const int64_t at = (int64_t)(t0 + rnode) * p.Hq + rhead;
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 y;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = (__bf16)o[k];
        *(bf16x4 *)(p.out + at * D + d) = y;
        if (d == 0 && p.lse) p.lse[at] = lse;
      } else {
        *(f32x4 *)(p.part_out + (slot + row0 + r) * D + d) = o;
        if (d == 0) p.part_lse[slot + row0 + r] = lse;
      }
    }
    at_tile = seq_end;
    if (at_tile >= stop) return;
    __syncthreads();  // (the patches are read before the next sequence's tiles take their place)
  }
}

// The parts of sequences that several runs share, merged: lse = log sum_s exp(lse_s), out = sum_s exp(lse_s - lse) out_s, D/4 lanes per
// row.  Grid: KV head, 1024 / D query rows, sequence (block_rows: the attention's).  Eight parts are in flight at a time.
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const FourParams p, int block_rows) {
  constexpr int LPR = D / 4, U = 8, ROWS = 256 / LPR;
  const int g = blockIdx.x, row = blockIdx.y * ROWS + threadIdx.x / LPR, row0 = blockIdx.y * ROWS / block_rows * block_rows, b = blockIdx.z, which = b / p.group, lb = b - which * p.group;
  const Deal deal(p, which * p.group, row0);
  const int tiles = __builtin_amdgcn_readlane(deal.tiles, lb), end = __builtin_amdgcn_readlane(deal.upto, lb);
  if (tiles == 0) return;
  const int first = deal.run_of(end - tiles), S = deal.run_of(end - 1) - first + 1;
  if (S == 1) return;
  const int t0 = __builtin_amdgcn_readlane(deal.t0, lb), n_rows = __builtin_amdgcn_readlane(deal.T, lb) * p.G;
  const int64_t stride = (int64_t)p.Hkv * p.rows, slot0 = (int64_t)(which * (p.parts + p.group) + first + lb) * stride + (int64_t)g * p.rows;
  const int d = (threadIdx.x % LPR) * 4;
  if (row >= n_rows) return;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;
  for (int s0 = 0; s0 < S; s0 += U) {
    float ls[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = slot0 + min(s0 + u, S - 1) * stride + row;
      ls[u] = p.part_lse[at];
      x[u] = *(const f32x4 *)(p.part_out + at * D + d);
    }
    float here = top;
#pragma unroll
    for (int u = 0; u < U; ++u) here = fmaxf(here, ls[u]);
    const float f = here == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((top - here) * kLog2e);
    o *= f, sum *= f, top = here;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u >= S || ls[u] == -INFINITY) continue;
      const float w = __builtin_amdgcn_exp2f((ls[u] - (top == -INFINITY ? 0.f : top)) * kLog2e);
      sum += w;
      o += x[u] * w;
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 y;
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = (__bf16)(o[k] * inv);
  const int node = row / p.G, head = g * p.G + (row - node * p.G);
  const int64_t at = (int64_t)(t0 + node) * p.Hq + head;
  *(bf16x4 *)(p.out + at * D + d) = y;
  if (d == 0 && p.lse) p.lse[at] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum) * kLn2;
}

struct FourPlan {
  int WM, blocks, group, groups, parts;
};
// 32-row workgroups while there is little work and one round of them holds it: their four waves split the keys, which costs no partial
// results (one sequence of 2048 keys, 56 nodes: 14.9 us with 32 rows, 17.2 with 64, 22.0 with 128; but 26 sequences of 7 keys, 64
// heads, 64 nodes 76 us with 32 rows, 43 with 128).  Else as many rows as divide the row groups without waste, so that fewer workgroups
// read the same keys, and 64 rows for an odd number from five on, which leaves one wave idle (4 sequences of 16384 .. 32768 keys, four heads
// to a KV head, with 32 / 64 / 128 rows: 24 nodes, three groups, 80.6 / 100.2 / 90.9 us; 48, six, 140 / 123 / 148; 56, seven, 157 / 149 /
// 155; 66, nine, 191 / 181 / 208; 80, ten, 217 / 188 / 215; 100, thirteen, 301 / 242 / 260; 112, fourteen, 308 / 246 / 269).
// Long work of several long sequences is dealt out over two workgroups per CU (a part of a sequence costs about four tiles of its own);
// a sequence by itself over one (the first case with 256 workgroups 14.8 us, with 512 18.5, before remainders), and one run at most is a
// round short of a workgroup rather than one too many.
void plan_four(const tva_attn4_args *a, FourPlan *pl) {
  constexpr int kSlots = 256, kTogether = 6, kLong = 32;
  const int G = a->Hq / a->Hkv;
  const int64_t rows = (int64_t)a->max_T * G, groups = std::max<int64_t>(1, (rows + 31) / 32);
  const int tiles = (a->max_L + 63) / 64 + (a->max_T + 63) / 64;
  const int64_t pairs = (int64_t)a->B * a->Hkv;
  if (a->plan_rows) pl->WM = a->plan_rows / 32;
  else pl->WM = groups == 1 || (pairs * groups <= 2 * kSlots && pairs * groups * tiles <= 8 * 2048) ? 1 : groups == 3 ? 1 : groups % 4 == 0 ? 4 : 2;
  const int WK = kWaves / pl->WM;
  pl->blocks = (int)((groups + pl->WM - 1) / pl->WM);
  const int64_t base = (int64_t)a->Hkv * pl->blocks;
  const int64_t load = pairs * pl->blocks * tiles / (2 * kSlots * WK);  // tiles a wave has where two workgroups per CU share them
  pl->groups = a->B > 1 && load >= kTogether && tiles >= kLong && a->num_splits == 0 ? (a->B + 63) / 64 : a->B;
  pl->group = (a->B + pl->groups - 1) / pl->groups;
  pl->groups = (a->B + pl->group - 1) / pl->group;
  int64_t parts = a->num_splits;
  if (parts == 0) {
    parts = std::max<int64_t>(1, (pl->group > 1 ? 2 * kSlots : kSlots) / (base * pl->groups));
    if (pl->group == 1) parts = std::min<int64_t>(parts, std::max(1, (tiles + WK - 1) / WK));  // a tile per wave
  }
  pl->parts = (int)std::max<int64_t>(1, std::min<int64_t>(parts, (int64_t)pl->group * tiles));
}

int check_four(const tva_attn4_args *a, bool shapes_only) {
  if (!a || a->B <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv) return TVA_INVALID_ARG;
  if (a->sum_T < 0 || a->max_T < 0 || a->max_L < 0 || a->num_splits < 0) return TVA_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return TVA_UNSUPPORTED;
  if (a->plan_rows != 0 && a->plan_rows != 32 && a->plan_rows != 64 && a->plan_rows != 128) return TVA_INVALID_ARG;
  if (a->max_T > TVA_MAX_TREE) return TVA_UNSUPPORTED;
  if (a->max_L > 1 << 29) return TVA_UNSUPPORTED;  // (page_of; positions are rounded up to whole tiles)
  if (shapes_only) return TVA_OK;
  if (!(a->scale > 0.f)) return TVA_INVALID_ARG;
  if (a->sum_T == 0) return TVA_OK;
  if (!a->cu_T || !a->L || !a->q || !a->k_tree || !a->v_tree || !a->out || (!a->anc_mask && !a->parent)) return TVA_INVALID_ARG;
  if (((uintptr_t)a->q | (uintptr_t)a->k_tree | (uintptr_t)a->v_tree | (uintptr_t)a->out) & 15) return TVA_INVALID_ARG;
  if (a->anc_mask && (a->mask_words < 1 || a->mask_words > 2 || a->mask_words * 64 < a->max_T)) return TVA_UNSUPPORTED;
  if (a->cache.kind != TVA_ROWS_E2M1) return TVA_UNSUPPORTED;
  return TVA_OK;
}

size_t four_bytes(const tva_attn4_args *a, const FourPlan &pl) {
  const size_t slots = (size_t)pl.groups * (pl.parts + pl.group), rows = (size_t)pl.blocks * pl.WM * 32;
  return pl.parts == 1 ? 0 : slots * a->Hkv * rows * (a->D + 1) * 4;
}

template <int D>
int launch_rows(const RowsParams &p, int B, int layers, bool load, hipStream_t st) {
  const int64_t groups = std::max<int64_t>(1, ((int64_t)p.max_rows * p.Hkv + 256 / (D / 8) - 1) / (256 / (D / 8)));  // (one writes L_out)
  if (groups > 0x7fffffff) return TVA_UNSUPPORTED;
  const dim3 grid((unsigned)groups, B, (layers + kRowLayers - 1) / kRowLayers);
  if (load) hipLaunchKernelGGL(load_rows_kernel<D>, grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(store_rows_kernel<D>, grid, dim3(256), 0, st, p);
  return hipPeekAtLastError() == hipSuccess ? TVA_OK : TVA_HIP_ERROR;
}

int run_rows(const tva_rows_args *a, bool load, void *stream) {
  if (!a || a->B < 0 || a->Hkv < 1 || a->max_rows < 0 || a->n_layers < 0) return TVA_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return TVA_UNSUPPORTED;
  if (a->B == 0) return TVA_OK;
  if (a->cache.kind != TVA_ROWS_E2M1) return a->cache.kind < 0 || a->cache.kind > TVA_ROWS_E2M1 ? TVA_INVALID_ARG : TVA_UNSUPPORTED;
  if (!a->cu_T || !a->L || (a->path == nullptr) != (a->path_len == nullptr)) return TVA_INVALID_ARG;
  if (!a->k_rows || !a->v_rows || (((uintptr_t)a->k_rows | (uintptr_t)a->v_rows) & 15)) return TVA_INVALID_ARG;
  if (a->L_out && (a->L_out == a->L || load)) return TVA_INVALID_ARG;
  if (a->layer_stride_cache < 0 || a->layer_stride_rows < 0 || a->layer_stride_cache % a->D || a->layer_stride_rows % 8) return TVA_INVALID_ARG;
  const int layers = a->n_layers > 0 ? a->n_layers : 1;
  if (a->B > 65535 || layers > 65535) return TVA_UNSUPPORTED;
  RowsParams p{};
  const int rc = view_of(a->cache, a->Hkv, a->D, true, &p.c);
  if (rc != TVA_OK) return rc;
  if (a->max_rows == 0 && !a->L_out) return TVA_OK;
  p.cu_T = a->cu_T, p.L = a->L, p.path = a->path, p.path_len = a->path_len;
  p.k_rows = (uint16_t *)a->k_rows, p.v_rows = (uint16_t *)a->v_rows;
  p.L_out = a->L_out, p.err_flag = a->err_flag, p.Hkv = a->Hkv, p.max_rows = a->max_rows, p.n_layers = layers;
  p.layer_rows = a->layer_stride_rows, p.layer_cache = a->layer_stride_cache / a->D;
  (void)hipGetLastError();
  return a->D == 128 ? launch_rows<128>(p, a->B, layers, load, (hipStream_t)stream) : launch_rows<64>(p, a->B, layers, load, (hipStream_t)stream);
}

}  // namespace

extern "C" {

int tva_cache_store(const tva_rows_args *a, void *stream) { return run_rows(a, false, stream); }
int tva_cache_load(const tva_rows_args *a, void *stream) { return run_rows(a, true, stream); }
size_t tva_sizeof_rows_args(void) { return sizeof(tva_rows_args); }

size_t tva_attn4_workspace_bytes(const tva_attn4_args *a) {
  FourPlan pl;
  if (check_four(a, true) != TVA_OK) return (size_t)-1;
  plan_four(a, &pl);
  return four_bytes(a, pl);
}

int32_t tva_attn4_plan_splits(const tva_attn4_args *a) {
  FourPlan pl;
  if (check_four(a, true) != TVA_OK) return -1;
  plan_four(a, &pl);
  return pl.parts;
}

int tva_tree_verify_attn_4bit(const tva_attn4_args *a, void *stream) {
  int rc = check_four(a, false);
  if (rc != TVA_OK) return rc;
  if (a->sum_T == 0 || a->max_T == 0) return TVA_OK;
  FourPlan pl;
  FourParams p{};
  rc = view_of(a->cache, a->Hkv, a->D, true, &p.c);
  if (rc != TVA_OK) return rc;
  plan_four(a, &pl);
  const size_t need = four_bytes(a, pl);
  if (need && (!a->workspace || ((uintptr_t)a->workspace & 15))) return TVA_INVALID_ARG;
  if (a->workspace_bytes < need) return TVA_WORKSPACE_TOO_SMALL;
  if ((int64_t)pl.groups * pl.parts > 65535 || a->B > 65535 || pl.blocks > 65535) return TVA_UNSUPPORTED;
  if (p.c.stride_tok * (a->D / 2) >= 1 << 24) return TVA_UNSUPPORTED;  // (offsets within a tile)
  p.q = (const __bf16 *)a->q, p.k_tree = (const __bf16 *)a->k_tree, p.v_tree = (const __bf16 *)a->v_tree;
  p.cu_T = a->cu_T, p.L = a->L, p.parent = a->parent, p.mask = a->anc_mask;
  p.out = (__bf16 *)a->out, p.lse = a->lse;
  p.rows = pl.blocks * pl.WM * 32;
  p.part_out = (float *)a->workspace, p.part_lse = p.part_out + (need ? need / 4 / (a->D + 1) * a->D : 0);
  p.B = a->B, p.Hq = a->Hq, p.Hkv = a->Hkv, p.G = a->Hq / a->Hkv, p.W = a->mask_words, p.max_L = a->max_L;
  p.group = pl.group, p.parts = pl.parts, p.scale_log2 = a->scale * kLog2e;
  const dim3 grid(a->Hkv, pl.blocks, pl.groups * pl.parts);
  const hipStream_t st = (hipStream_t)stream;
  const int pg = !a->cache.page_table ? 0 : a->cache.page_size % 64 ? 1 : 2;
  const bool once = p.c.stride_tok == 1 && (int64_t)a->B * a->max_L * a->Hkv * (a->D + a->D / 32 + 2) > kLastLevel;
  (void)hipGetLastError();
  auto launch = [&](auto d, auto wm) {
    constexpr int D = decltype(d)::value, WM = decltype(wm)::value;
    auto form = [&](auto f) {
      constexpr int FORM = decltype(f)::value;
      if (pg == 0) hipLaunchKernelGGL((four_bit_kernel<D, WM, 0, FORM>), grid, dim3(256), 0, st, p);
      else if (pg == 1) hipLaunchKernelGGL((four_bit_kernel<D, WM, 1, FORM>), grid, dim3(256), 0, st, p);
      else hipLaunchKernelGGL((four_bit_kernel<D, WM, 2, FORM>), grid, dim3(256), 0, st, p);
    };
    if constexpr (WM == 1) {
      if (pl.blocks > 1) form(std::integral_constant<int, kAlways>{});
      else if (once) form(std::integral_constant<int, kOnce>{});
      else form(std::integral_constant<int, kPlain>{});
    } else {
      form(std::integral_constant<int, kPlain>{});
    }
    if (pl.parts > 1 && hipPeekAtLastError() == hipSuccess)
      hipLaunchKernelGGL(join_kernel<D>, dim3(a->Hkv, (p.rows + 1024 / D - 1) / (1024 / D), a->B), dim3(256), 0, st, p, WM * 32);
  };
  auto shapes = [&](auto d) {
    if (pl.WM == 1) launch(d, std::integral_constant<int, 1>{});
    else if (pl.WM == 2) launch(d, std::integral_constant<int, 2>{});
    else launch(d, std::integral_constant<int, 4>{});
  };
  if (a->D == 128) shapes(std::integral_constant<int, 128>{});
  else shapes(std::integral_constant<int, 64>{});
  return hipPeekAtLastError() == hipSuccess ? TVA_OK : TVA_HIP_ERROR;
}

size_t tva_sizeof_attn4_args(void) { return sizeof(tva_attn4_args); }

}  // extern "C"
