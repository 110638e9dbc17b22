// libtva: attention of new tokens over the cache that holds them (gfx950).  Entry points and their meaning: include/tva_layer.h.
//
//   chunk_kernel  S^T = K Q^T and O^T = V^T P^T by 32x32x16 bf16 MFMAs, a query row per lane of a half, as in tva.hip and cache4.hip:
//                 the scores of a row then lie in the registers that the second product takes its weights from, and a row's maximum and
//                 sum are one lane exchange.  One pass over the keys with the running maximum and sum of the softmax.  A workgroup has
//                 32, 128 or 256 query rows (tokens x heads of a KV head: the heads share the keys) and walks tiles of its keys; only
//                 tiles that some row sees are walked: the first ones (of n_first), then those of the window or all.
//   merge_kernel  partial results of row blocks whose keys were split.
//
// 32 rows (single tokens, few new ones) wait for memory: four waves, each with 32-key tiles of its own that it brings and waits for alone, its
// next one on the way meanwhile.  64 sequences of 1024 seen keys: 56 us, 4.8 TB/s; 256 of 4096: 722 us, 5.9 TB/s (a copy: 5.1).
// 128 and 256 rows are bound by the instructions of a tile: all waves bring 64-key tiles to LDS together (through registers, K two tiles ahead;
// 8-bit rows are widened on the way) and read their operands there, K as rows, V by transposing reads.  2048 tokens behind 30000: 965 us,
// 1.08 PFLOP/s (a library product of 8192^3: 1.26 to 1.36); per matrix instruction, which takes the matrix unit 32 cycles, 5.6 vector
// instructions, an exponential among them, take the vector unit 34; counters have the matrix units busy for 51 % of the cycles, and the chip
// lowers its clock to 1.7 to 2.0 GHz under that load.  128 rows leave two workgroups to a compute
// unit, which fill each other's barriers and share long and short blocks; 256 bring every tile half as often.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cache_rows.h"
#include "sequences.h"
#include "tva.h"
#include "tva_cache.h"
#include "tva_layer.h"

namespace {

using namespace cache_rows;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ChunkParams {
  const __bf16 *q;
  const int32_t *cu_T, *L;
  const uint64_t *mask;
  CacheView c;
  __bf16 *out;
  float *lse;
  float *part_out, *part_lse;  // [blocks, parts, Hkv, rows of a block, D], [blocks, parts, Hkv, rows]
  int64_t q_stride;
  int B, Hq, Hkv, G, W, blocks, max_T;
  bool by_keys;  // how row blocks are numbered (Block)
  int each;
  int parts, part_keys;  // the most parts a block's tiles are cut into, and the keys of a part that it is cut for
  int window, n_first;   // window: 2^30 where there is none
  int longest;           // row blocks that are taken from the last on, before the others from the first on
  float scale_log2, v_scale;
};

// (The compiler takes what a wave finds by asking its lanes for a value per lane: said once, here.)
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A row block of one sequence: where its rows and its keys lie.
// Blocks are numbered in one of three ways, of which the launch takes one:
//   by their keys  up to 64 sequences: those with the most keys first, and of each its last block, which sees the most, first.  A lane per
//                  sequence finds where its blocks begin.  (16 sequences of 1 to 333 tokens behind 100 to 8000, 8-bit rows, one set of such
//                  lengths: 201 us, by rows 259; six other sets 203 to 265)
//   evenly         `each` for every sequence
//   by rows        a sequence's first is floor(cu_T[b] G / rows) + b: one of n rows has ceil(n / rows) of the numbers up to the next one's first,
//                  which are at least that many
// (Numbers without rows leave compute units idle where one workgroup for each was asked for: four trees of 60 nodes, 11 numbers by rows for 8
// blocks, 51 and 39 us.)
struct Block {
  int b, t0, T, L;
  int row0, rows;  // first row (token x head of the KV head) of the sequence, rows of this block
  int low, high;   // bounds of the positions that the rows have
  int end;         // key slots that a row may see
  __device__ __forceinline__ Block(const ChunkParams &p, int R, int number) {
    int64_t from;  // the number of its first one
    if (p.by_keys) {
      const int lane = threadIdx.x & 63, n = min(lane, p.B - 1), begin = p.cu_T[n], tokens = max(0, min(p.cu_T[n + 1] - begin, p.max_T)), cached = max(p.L[n], 0);
      const int blocks = lane < p.B ? (int)(((int64_t)tokens * p.G + R - 1) / R) : 0, keys = min(cached, p.window) + tokens;
      int start = 0;
      for (int x = 0; x < p.B; ++x) {
        const int other = __builtin_amdgcn_readlane(keys, x), many = __builtin_amdgcn_readlane(blocks, x);
        start += other > keys || (other == keys && x < lane) ? many : 0;
      }
      const uint64_t here = __ballot(number >= start && number < start + blocks);
      b = here ? __builtin_ctzll(here) : 0;
      t0 = __builtin_amdgcn_readlane(begin, b), T = __builtin_amdgcn_readlane(tokens, b), L = __builtin_amdgcn_readlane(cached, b);
      from = number - (__builtin_amdgcn_readlane(blocks, b) - 1 - (number - __builtin_amdgcn_readlane(start, b)));
      if (!here) T = 0, from = number;  // behind the last block: no rows
    } else if (p.each) {
      b = same((int)((uint32_t)number / (uint32_t)p.each)), from = (int64_t)b * p.each;
      t0 = p.cu_T[b], T = p.cu_T[b + 1] - t0, L = p.L[b];
    } else {
      auto first = [&](int n, int row) __attribute__((always_inline)) { return (int64_t)row * p.G / R + n; };
      const sequences::Place place = sequences::find(p.cu_T, p.L, p.B, number, first);
      b = same(place.b), t0 = same(place.t0), T = place.t1 - place.t0, L = place.L, from = first(b, t0);
      if (number < from) T = 0, from = number;  // in front of the first sequence (cu_T[0] > 0): no rows
    }
    T = same(min(T, p.max_T)), L = same(max(L, 0));
    const int64_t at = (number - from) * R, all = (int64_t)T * p.G;
    rows = same((int)max((int64_t)0, min((int64_t)R, all - at)));
    row0 = same((int)min(at, all));
    const int64_t room = room_of(p.c, b);
    if (p.mask) {
      low = L - 1, high = L + T - 1;
      end = (int)min((int64_t)L + T, room);
    } else {
      low = L + row0 / p.G, high = L + (row0 + max(rows, 1) - 1) / p.G;
      end = (int)min((int64_t)high + 1, room);
    }
    low = same(low), high = same(high), end = same(end);
  }
};
// Its tiles of KT keys: `first` of them from slot 0 on, then from tile `main` on, n in all.  Those that no row sees are left out.
struct Tiles {
  int first, main, n;
  __device__ __forceinline__ Tiles(const ChunkParams &p, const Block &k, int KT) {
    const int from = max(0, k.low - p.window + 1);
    main = min(from, max(k.end - 1, 0)) / KT;
    first = min(main, (min(p.n_first, from) + KT - 1) / KT);
    n = same(k.rows > 0 && k.end > 0 ? first + (k.end + KT - 1) / KT - main : 0);
    first = same(first), main = same(main);
  }
  __device__ __forceinline__ int at(int u) const { return u < first ? u : u - first + main; }
  __device__ __forceinline__ int parts(const ChunkParams &p, int KT) const {
    if (p.parts == 1) return 1;
    const uint32_t tiles = max(1, p.part_keys / KT);
    return same(max(1, min(p.parts, (int)((n + tiles - 1) / tiles))));
  }
};

__device__ __forceinline__ float half_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
// The larger, of each half, of |x| bits and those of eight bf16 numbers; and whether one of them is infinite or NaN
__device__ __forceinline__ u16x2 larger(u32x4 v, u16x2 x) {
#pragma unroll
  for (int k = 0; k < 4; ++k) x = __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, v[k] & 0x7fff7fffu));
  return x;
}
__device__ __forceinline__ bool not_finite(u16x2 x) { return max(x[0], x[1]) >= 0x7f80; }
__device__ __forceinline__ u32x4 finite_ones(u32x4 x) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if ((x[k] & 0x7f80) == 0x7f80) x[k] &= 0xffff0000u;
    if ((x[k] & 0x7f800000) == 0x7f800000) x[k] &= 0xffffu;
  }
  return x;
}

template <int D, int WM, int WK, int KB, int KIND>
struct ChunkCfg {
  static constexpr int WAVES = WM * WK, THREADS = 64 * WAVES;
  // 32-row workgroups: a wave brings tiles of its own and waits for no other; else the workgroup's waves bring one together
  static constexpr bool OWN = WM == 1;
  static constexpr int R = 32 * WM, KW = 32 * KB, KT = OWN ? KW : KW * WK;  // rows; keys of a tile that a wave multiplies, and of a tile
  static constexpr int STEP = OWN ? WK : 1;                                // tiles from one of a wave's to its next
  static constexpr int NS = D / 16, NJ = D / 32;
  // Bytes from row to row in LDS: spaced so that 16 rows of K at one 16-byte piece each, and four rows of V at 64 bytes of each, are in
  // different banks, and an operand's address is one register and constants.
  static constexpr int K_ROW = 2 * D + 16, V_ROW = 2 * D + 64;
  static constexpr int STAGES = OWN ? WK : 2;  // of K, and as many of V
  static constexpr int K_TILE = KT * K_ROW, V_TILE = KT * V_ROW;
  static constexpr int TOGETHER = OWN ? 1 : WAVES;                        // waves that bring a tile
  static constexpr int EPL = KIND == TVA_ROWS_BF16 || KT * D / 16 < 64 * TOGETHER ? 8 : 16;  // elements that a lane brings at once
  static constexpr int LPR = D / EPL, RPW = 64 / LPR;                     // lanes that bring a row, rows that a wave brings at once
  static constexpr int PIECES = EPL / 8;                                   // 16-byte pieces of bf16 that they become
  static constexpr int NP = KT / (RPW * TOGETHER);                        // reads per lane and tile (of K, and of V)
  static_assert(KT % (RPW * TOGETHER) == 0, "");
  static constexpr int TP = D + 4, PATCH = 32 * TP * 4;  // an output patch per wave, floats between its rows
  static constexpr int EXCHANGE = 2 * WAVES * 32 * 4;
  static constexpr int DEPTH = STAGES * (K_TILE + V_TILE), ODD = DEPTH + TVA_MAX_TREE * 4;  // LDS: tiles, depths of a tree's nodes, marks of tiles
  static constexpr int LOOP_LDS = ODD + 2 * WAVES * 4, END_LDS = WAVES * PATCH + EXCHANGE;
  static constexpr int LDS = LOOP_LDS > END_LDS ? LOOP_LDS : END_LDS;
  // remainders of the softmax weights are multiplied too (their rounding to bf16 would show; the shape waits for memory)
  static constexpr bool REST = WM == 1;
};

template <int N, class F>
__device__ __forceinline__ void times(F f) {
  if constexpr (N > 0) times<N - 1>(f), f(std::integral_constant<int, N - 1>{});
}
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Grid: KV head (fastest: with 8 heads one per XCD, whose L2 then holds one head's keys), part, row block: those that see the most keys first;
// where two workgroups per CU hold all of one sequence, the second ones from the first on, so that a long and a short one share a CU.
// PLACES: how a tile's rows are found.  kDense and kPages: the rows that a wave brings at once lie in a sequence, or a page, one after the
// other: scalar addresses and a lane's offset; kRows: each lane looks for its own (pages that such rows may straddle).
enum { kDense, kPages, kRows };
template <int D, int WM, int WK, int KB, int KIND, int PLACES, bool TREE>
__global__ void __launch_bounds__(64 * WM *WK, 2) chunk_kernel(const ChunkParams p) {
  typedef ChunkCfg<D, WM, WK, KB, KIND> C;
  __shared__ __align__(16) unsigned char lds[C::LDS];
  const int g = blockIdx.x, part = blockIdx.y, number = (int)blockIdx.z < p.longest ? p.blocks - 1 - blockIdx.z : blockIdx.z - p.longest;
  const Block k(p, C::R, number);
  const Tiles tiles(p, k, C::KT);
  const int parts = tiles.parts(p, C::KT);
  if (k.rows <= 0 || part >= parts) return;
  // (parts differ by a tile at most: the first n % parts have one more)
  const int each = parts == 1 ? tiles.n : (int)((uint32_t)tiles.n / (uint32_t)parts), more = tiles.n - each * parts;
  const int u0 = same(part * each + min(part, more)), u1 = same(u0 + each + (part < more));

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wm = wave % WM, wk = wave / WM;

  // ---- this lane's query row (column of S^T and O^T); rows past the end repeat the last one and are not written ----
  const int row = k.row0 + min(wm * 32 + l32, k.rows - 1);
  const int node = row / p.G, head = g * p.G + (row - node * p.G);
  bf16x8 q[C::NS];
  {
    const __bf16 *from = p.q + (int64_t)(k.t0 + node) * p.q_stride + head * D + half * 8;
#pragma unroll
    for (int s = 0; s < C::NS; ++s) q[s] = *(const bf16x8 *)(from + s * 16);
  }
  int P = k.L + node;
  uint64_t anc0 = 0, anc1 = 0;
  if constexpr (TREE) {
    int *depth = (int *)(lds + C::DEPTH);
    for (int i = tid; i < k.T; i += C::THREADS) {
      const uint64_t *words = p.mask + (int64_t)(k.t0 + i) * p.W;
      depth[i] = (int)__popcll(words[0]) + (p.W > 1 ? (int)__popcll(words[1]) : 0) - 1;
    }
    __syncthreads();
    const uint64_t *words = p.mask + (int64_t)(k.t0 + node) * p.W;
    anc0 = words[0], anc1 = p.W > 1 ? words[1] : 0;
    P = k.L + (int)__popcll(anc0) + (int)__popcll(anc1) - 1;
    if (k.T < 64) anc0 &= (1ull << k.T) - 1, anc1 = 0;
    else if (k.T < 128) anc1 &= (1ull << (k.T - 64)) - 1;
    for (uint64_t left = anc0; left; left &= left - 1) {  // what the window leaves of them
      const int j = __builtin_ctzll(left), at = k.L + depth[j];
      if (at <= P - p.window && at >= p.n_first) anc0 &= ~(1ull << j);
    }
    for (uint64_t left = anc1; left; left &= left - 1) {
      const int j = __builtin_ctzll(left), at = k.L + depth[64 + j];
      if (at <= P - p.window && at >= p.n_first) anc1 &= ~(1ull << j);
    }
  }
  const int behind = P - p.window;  // positions up to it are out of the window
  // Which of the 32 key slots from t on this lane's row sees, a bit each.  (Bits, not comparisons: those of a whole tile at once are more
  // than there are scalar registers.)
  auto below = [](int n) __attribute__((always_inline)) -> uint32_t { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
  auto sees = [&](int t) __attribute__((always_inline)) -> uint32_t {
    const uint32_t near = ~below(behind + 1 - t) | below(p.n_first - t);
    if constexpr (TREE) {
      const int j = t - k.L;  // the first one's number among the new tokens
      uint32_t bits = near & below(-j);
      if (j > -32) bits |= (uint32_t)(j < 0 ? anc0 << -j : j < 64 ? anc0 >> j : j < 128 ? anc1 >> (j - 64) : 0);
      if (j > 32 && j < 64) bits |= (uint32_t)(anc1 << (64 - j));
      return bits & below(k.end - t);
    } else {
      return near & below(min(P + 1, k.end) - t);
    }
  };
  // bounds over the wave's rows, the same for all its lanes
  int low = k.low, high = k.high;
  if constexpr (!TREE) {
    low = k.L + (k.row0 + min(wm * 32, k.rows - 1)) / p.G, high = k.L + (k.row0 + min(wm * 32 + 31, k.rows - 1)) / p.G;
    low = __builtin_amdgcn_readfirstlane(low), high = __builtin_amdgcn_readfirstlane(high);
  }
  // whether all rows with positions low .. high see the n slots from t on
  auto all_seen = [&](int t, int n, int low, int high) __attribute__((always_inline)) -> bool {
    return t + n <= k.end && t + n - 1 <= (TREE ? k.L - 1 : low) && (t > high - p.window || t + n <= p.n_first);
  };
  // the tiles all of which all those rows see, but for any of the first ones: a run of them
  auto run_of = [&](int low, int high, int *from, int *to) __attribute__((always_inline)) {
    const int whole = min(k.end, (TREE ? k.L : low + 1)) / C::KT;               // tiles below it end before what some row does not see
    const int near = max(high - p.window + C::KT, 0) / C::KT;                   // tiles from it on begin in all windows
    *from = same(max(near, tiles.main) - tiles.main + tiles.first), *to = same(whole - tiles.main + tiles.first);
  };
  int quiet0, quiet1, plain0, plain1;  // of the workgroup's rows, of the wave's
  run_of(k.low, k.high, &quiet0, &quiet1);
  run_of(low, high, &plain0, &plain1);

  // ---- tiles: global memory -> registers -> LDS ----
  const Finder<PLACES != kDense, true> find(p.c, k.b, g);
  const int piece = lane % C::LPR, lrow = lane / C::LPR, bring = C::OWN ? 0 : wave;
  const int last = k.end - 1, last_group = last - last % C::RPW;  // the last slot, and the first of the group that it is in
  constexpr int BYTES = KIND == TVA_ROWS_BF16 ? 2 : 1;            // of an element
  u32x4 kx[C::NP], vx[C::NP];
  int entry[PLACES == kRows ? C::NP : 1];  // kRows: the page of this lane's row of each read; kPages: lane i has that of read i, and
  uint32_t in_page = 0;                    // where its rows begin in the page, in bytes
  int64_t place[C::NP];                    // of the reads of K's tile, in bytes: V's are the same, later
  uint32_t within[C::NP];
  const uint32_t row_bytes = (uint32_t)(p.c.stride_tok * BYTES);
  // (a tile past the last one: the last again.  A branch would leave the waits without a count to go by)
  auto first_slot = [&](int u) __attribute__((always_inline)) { return tiles.at(min(u, u1 - 1)) * C::KT; };
  // (an entry below 0, a page given back that the window has left: its rows share a tile with rows that are seen; page 0 is read for it: GAPS)
  auto look = [&](int u) __attribute__((always_inline)) {
    const int t = first_slot(u);
    if constexpr (PLACES == kRows) {
#pragma unroll
      for (int i = 0; i < C::NP; ++i) entry[i] = find.entry(p.c, min(t + (i * C::TOGETHER + bring) * C::RPW + lrow, last));
    } else if constexpr (PLACES == kPages) {
      const int row = min(t + (min(lane, C::NP - 1) * C::TOGETHER + bring) * C::RPW, last_group), page = page_of(p.c, row);
      entry[0] = find.entry_of(page), in_page = (uint32_t)(row - page * p.c.page_size) * row_bytes;
    }
  };
  auto locate = [&](int u) __attribute__((always_inline)) {
    const int t = first_slot(u);
#pragma unroll
    for (int i = 0; i < C::NP; ++i) {
      const int row = t + (i * C::TOGETHER + bring) * C::RPW;
      if constexpr (PLACES == kRows) {
        place[i] = find.at(p.c, min(row + lrow, last), entry[i]) * BYTES;
        within[i] = piece * C::EPL * BYTES;
      } else if constexpr (PLACES == kPages) {
        // (the launch sees to it that a page has less than 2^32 bytes)
        place[i] = find.base * BYTES + (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(entry[0], i) * (uint32_t)(p.c.stride_page * BYTES)) +
                   (uint32_t)__builtin_amdgcn_readlane((int)in_page, i);
        within[i] = (uint32_t)min(lrow, last - min(row, last_group)) * row_bytes + (uint32_t)(piece * C::EPL * BYTES);
      } else {
        place[i] = find.base * BYTES + (int64_t)((uint64_t)(uint32_t)t * row_bytes);
        within[i] = (uint32_t)min((i * C::TOGETHER + bring) * C::RPW + lrow, last - t) * row_bytes + (uint32_t)(piece * C::EPL * BYTES);
      }
    }
  };
  auto read = [&](u32x4 (&x)[C::NP], const char *from) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::NP; ++i) {
      if constexpr (C::EPL * BYTES == 16) {
        x[i] = *(const u32x4 *)(from + place[i] + within[i]);
      } else {
        const u32x2 a = *(const u32x2 *)(from + place[i] + within[i]);
        x[i] = u32x4{a[0], a[1], 0, 0};
      }
    }
  };
  auto k_stage = [&](int stage) __attribute__((always_inline)) { return lds + stage * C::K_TILE; };
  auto v_stage = [&](int stage) __attribute__((always_inline)) { return lds + C::STAGES * C::K_TILE + stage * C::V_TILE; };
  // Tiles that some row does not see all of are looked through for values that are not finite: those go to LDS as 0 (a weight of 0 times
  // them is no 0), the tile is marked, and rows that see them get them added.  (With remainders every tile: an infinite value times a
  // remainder of 0 or below is no infinity.)
  auto careful_with = [&](int u) __attribute__((always_inline)) { return C::REST || u < quiet0 || u >= quiet1; };
  auto stash_k = [&](int stage, const u32x4 (&kx)[C::NP]) __attribute__((always_inline)) {
    unsigned char *to = k_stage(stage);
#pragma unroll
    for (int i = 0; i < C::NP; ++i) {
      const int r = (i * C::TOGETHER + bring) * C::RPW + lrow;
      if constexpr (KIND == TVA_ROWS_BF16) {
        *(u32x4 *)(to + r * C::K_ROW + piece * 16) = kx[i];
      } else {
#pragma unroll
        for (int h = 0; h < C::EPL / 8; ++h)
          *(bf16x8 *)(to + r * C::K_ROW + (C::EPL / 8 * piece + h) * 16) = widen8_e4m3(u32x2{kx[i][2 * h], kx[i][2 * h + 1]});
      }
    }
  };
  auto stash_v = [&](int stage) __attribute__((always_inline)) {
    unsigned char *to = v_stage(stage);
#pragma unroll
    for (int i = 0; i < C::NP; ++i) {
      const int r = (i * C::TOGETHER + bring) * C::RPW + lrow;
#pragma unroll
      for (int h = 0; h < C::PIECES; ++h) {
        u32x4 v = vx[i];
        if constexpr (KIND != TVA_ROWS_BF16) v = __builtin_bit_cast(u32x4, widen8_e4m3(u32x2{vx[i][2 * h], vx[i][2 * h + 1]}));
        *(u32x4 *)(to + r * C::V_ROW + (C::PIECES * piece + h) * 16) = v;
      }
    }
  };
  auto look_through = [&](int stage) __attribute__((always_inline)) {  // at what this lane has brought
    unsigned char *to = v_stage(stage);
    u16x2 x = {0, 0};
#pragma unroll
    for (int i = 0; i < C::NP * C::PIECES; ++i)
      x = larger(*(const u32x4 *)(to + ((i / C::PIECES * C::TOGETHER + bring) * C::RPW + lrow) * C::V_ROW + (C::PIECES * piece + i % C::PIECES) * 16), x);
    const bool odd = __any(not_finite(x));
    if (odd) {
      for (int i = 0; i < C::NP * C::PIECES; ++i) {
        u32x4 *v = (u32x4 *)(to + ((i / C::PIECES * C::TOGETHER + bring) * C::RPW + lrow) * C::V_ROW + (C::PIECES * piece + i % C::PIECES) * 16);
        *v = finite_ones(*v);
      }
    }
    if (lane == 0) ((int *)(lds + C::ODD))[(C::OWN ? 0 : stage * C::WAVES) + wave] = odd;
  };
  auto is_odd = [&](int u, int stage) __attribute__((always_inline)) -> bool {
    bool odd = false;
    if (careful_with(u)) {
#pragma unroll
      for (int w = 0; w < C::TOGETHER; ++w) odd |= ((const int *)(lds + C::ODD))[C::OWN ? wave : stage * C::WAVES + w] != 0;
    }
    return same(odd);
  };

  f32x16 acc[C::NJ];
#pragma unroll
  for (int j = 0; j < C::NJ; ++j) acc[j] = f32x16{};
  float m = -INFINITY, l = 0.f;  // reference (log2 domain) and sum over this lane half's keys

  // ---- what is done with 32 keys ----
  // S^T = K Q^T, of which row l32 of K is this lane's operand
  auto k_operand = [&](const unsigned char *kt, int kb, int st) __attribute__((always_inline)) {
    return *(const bf16x8 *)(kt + (kb * 32 + l32) * C::K_ROW + (st * 2 + half) * 16);
  };
  // O^T += V^T P^T, of 16 keys and 32 elements: 16 lanes turn over 4 rows x 16 elements, this lane's row (of keys 8 h + 4 half + 0..3) and 8-byte
  // piece of it
  const int i16 = lane & 15, sub = (lane >> 4) & 1;
  auto v_operand = [&](const unsigned char *vt, int kb, int a, int j) __attribute__((always_inline)) {
    s16x4 c[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 32 * kb + 16 * a + 8 * h + 4 * half + (i16 >> 2);
      c[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4 *)(vt + r * C::V_ROW + j * 64 + sub * 32 + (i16 & 3) * 8));
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(c[0], c[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto mask = [&](f32x16 &s, int t) __attribute__((always_inline)) {
    const uint32_t bits = sees(t) >> (4 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!((bits >> (8 * (i / 4) + i % 4)) & 1)) s[i] = -INFINITY;
  };
  auto add_odd = [&](int t0) __attribute__((always_inline)) {
    for (int t = t0; t < min(t0 + 32, k.end); ++t) {
      const bool here = sees(t) & 1;
      const int64_t at = find.at(p.c, t, find.entry(p.c, t));
#pragma unroll
      for (int j = 0; j < C::NJ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int d = 32 * j + 8 * (i / 4) + 4 * half + i % 4;
          float v;
          if constexpr (KIND == TVA_ROWS_BF16) v = (float)((const __bf16 *)p.c.v)[at + d];
          else v = (((const uint8_t *)p.c.v)[at + d] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f;
          if (here && !__builtin_isfinite(v)) acc[j][i] += v;
        }
    }
  };
  // A row's largest score (log2 domain) of 32 N keys; and whether the reference is to move: only where it is exceeded by more than 2^8, and
  // then for all rows of the wave.  Moving it brings l and O along.
  auto top_of = [&](auto &...s) __attribute__((always_inline)) -> float {
    float top = -INFINITY;
    auto take = [&](const f32x16 &x) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
    };
    (take(s), ...);
    return half_max(top) * p.scale_log2;
  };
  auto moves = [&](float top) __attribute__((always_inline)) -> bool { return __any(top > m + 8.f); };
  auto move_to = [&](float top) __attribute__((always_inline)) {
    const float to = fmaxf(m, top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
    m = to, l *= f;
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][i] *= f;
  };
  // Scores -> weights (bf16, and what their rounding leaves), their sum added to l
  auto soften = [&](const f32x16 &s, float ref, bf16x8 (&w)[2], bf16x8 (&rest)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -ref));
      l += x;
      w[i / 8][i % 8] = (__bf16)x;
      if constexpr (C::REST) rest[i / 8][i % 8] = (__bf16)(x - (float)w[i / 8][i % 8]);
    }
  };

  if constexpr (C::OWN) {
    static_assert(KB == 1, "");
    int u = u0 + wk;
    if (u < u1) {
      look(u);
      locate(u);
      read(kx, p.c.k), read(vx, p.c.v);
      look(u + C::STEP);
      for (; u < u1; u += C::STEP) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        stash_k(wave, kx);
        stash_v(wave);
        if (careful_with(u)) look_through(wave);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        locate(u + C::STEP);
        read(kx, p.c.k), read(vx, p.c.v);
        look(u + 2 * C::STEP);
        const int t = tiles.at(u) * C::KT;
        const bool masked = !all_seen(t, 32, low, high);
        f32x16 s = {};
#pragma unroll
        for (int st = 0; st < C::NS; ++st) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(k_stage(wave), 0, st), q[st], s, 0, 0, 0);
        if (masked) mask(s, t);
        const float top = top_of(s);
        if (moves(top)) move_to(top);
        bf16x8 w[2], rest[2];
        soften(s, m == -INFINITY ? 0.f : m, w, rest);
        if (is_odd(u, wave)) add_odd(t);
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int j = 0; j < C::NJ; ++j) {
            const bf16x8 v = v_operand(v_stage(wave), 0, a, j);
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[a], acc[j], 0, 0, 0);
            if constexpr (C::REST) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, rest[a], acc[j], 0, 0, 0);
          }
      }
    }
  } else if (u0 < u1) {
    static_assert(KB == 2 && WK == 1, "");
    // Beside the softmax of tile u run the products of tile u + 1's scores, beside those of O with tile u the search for tile u + 1's largest
    // scores: matrix and vector instructions of a wave that do not wait for each other.  K's tiles are therefore a tile ahead of V's.
    f32x16 s[2], next;
    {
      u32x4 k1[C::NP];
      look(u0);
      locate(u0);
      look(u0 + 1);
      read(kx, p.c.k), read(vx, p.c.v);
      locate(u0 + 1);
      look(u0 + 2);
      read(k1, p.c.k);
      stash_k(u0 & 1, kx), stash_v(u0 & 1);
      if (careful_with(u0)) look_through(u0 & 1);
      read(vx, p.c.v);
      locate(u0 + 2);
      look(u0 + 3);
      read(kx, p.c.k);
      stash_k(1 - (u0 & 1), k1);
      __syncthreads();
    }
    {
      const unsigned char *kt = k_stage(u0 & 1);
      s[0] = f32x16{}, s[1] = f32x16{};
#pragma unroll
      for (int st = 0; st < C::NS; ++st)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(kt, kb, st), q[st], s[kb], 0, 0, 0);
    }
    const int t = tiles.at(u0) * C::KT;
    if (!all_seen(t, C::KT, low, high)) mask(s[0], t), mask(s[1], t + 32);
    float top = top_of(s[0], s[1]);  // of s
    __syncthreads();                 // (K's first tile has been read)
    // A tile in the order in which it runs (left to itself the compiler has all products first and their operands' reads right before them):
    // per matrix instruction the softmax of EACH scores, in three steps of which each waits for none of its own turn, and an operand read AHEAD
    // matrix instructions ahead.  x holds the scores of half h of tile u, y those of the other; z takes those of half h of tile u + 1, then x
    // those of the other.
    //   scores z     | weights of x
    //   O with x's   | weights of y
    //   scores x     | largest of z
    //   O with y's   | largest of x
    constexpr int NS = C::NS, NP = 2 * C::NJ, AHEAD = WM == 4 ? 3 : 4, EACH = 16 / NS;
    static_assert(NS == NP, "");
    auto straight = [&](int u, f32x16 &x, f32x16 &y, f32x16 &z) __attribute__((always_inline)) {
      const float ref = m == -INFINITY ? 0.f : m;
      const unsigned char *kt = k_stage(1 - (u & 1)), *vt = v_stage(u & 1);
      bf16x8 ops[AHEAD], w[2][2];
      float arg[2][EACH], e[2][EACH];
      top = -INFINITY;
      auto fetch = [&](auto i) __attribute__((always_inline)) {  // of matrix instruction i
        constexpr int I = decltype(i)::value, PART = I / NS, N = I % NS, HALF = PART / 2;
        if constexpr (PART == 0 || PART == 2) ops[I % AHEAD] = k_operand(kt, HALF, N);
        else if constexpr (PART < 4) ops[I % AHEAD] = v_operand(vt, HALF, N / C::NJ, N % C::NJ);
      };
      times<AHEAD>(fetch);
      in_order();
      times<4 * NS>([&](auto i) __attribute__((always_inline)) {
        constexpr int I = decltype(i)::value, PART = I / NS, N = I % NS;
        const bf16x8 op = ops[I % AHEAD];
        if constexpr (PART == 0) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, q[N], N == 0 ? f32x16{} : z, 0, 0, 0);
        else if constexpr (PART == 2) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, q[N], N == 0 ? f32x16{} : x, 0, 0, 0);
        else acc[N % C::NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, w[PART / 2][N / C::NJ], acc[N % C::NJ], 0, 0, 0);
        fetch(std::integral_constant<int, I + AHEAD>{});
        // K of tile u + 2 takes the place of tile u's, V of tile u + 1 that of tile u - 1's; the next ones are asked for
        if constexpr (I == 1) stash_k(u & 1, kx);
        if constexpr (I == 3) stash_v(1 - (u & 1));
        if constexpr (I == 5) read(vx, p.c.v), locate(u + 3);
        if constexpr (I == 6) read(kx, p.c.k);
        if constexpr (I == 7) look(u + 4);
        // arguments of turn I, exponentials of turn I - 1, sums and roundings of turn I - 2 (a half's last ones are done in the next part's first turns)
        if constexpr (I >= 2 && I < 2 * NS + 2) {
          constexpr int B = (I - 2) % NS * EACH, W = (I - 2) / NS;
#pragma unroll
          for (int n = 0; n < EACH; ++n) l += e[I % 2][n], w[W][(B + n) / 8][(B + n) % 8] = (__bf16)e[I % 2][n];
        }
        if constexpr (I >= 1 && I < 2 * NS + 1) {
#pragma unroll
          for (int n = 0; n < EACH; ++n) e[(I - 1) % 2][n] = __builtin_amdgcn_exp2f(arg[(I - 1) % 2][n]);
        }
        if constexpr (I < 2 * NS) {
#pragma unroll
          for (int n = 0; n < EACH; ++n) arg[I % 2][n] = fmaf((PART == 0 ? x : y)[N * EACH + n], p.scale_log2, -ref);
        } else if constexpr (PART == 2) {
#pragma unroll
          for (int n = 0; n < EACH; ++n) top = fmaxf(top, z[N * EACH + n]);
        } else if constexpr (N >= NS / 4 && N < NS - 1) {  // (the last product is some turns old)
          constexpr int TURNS = NS - 1 - NS / 4, TURN = N - NS / 4;
#pragma unroll
          for (int n = TURN * 16 / TURNS; n < (TURN + 1) * 16 / TURNS; ++n) top = fmaxf(top, x[n]);
        }
        if constexpr (I == 4 * NS - 1) top = half_max(top) * p.scale_log2;
        in_order();
      });
      asm volatile("" : "+v"(top));
    };
    // behind tile u with ahead0 <= u < ahead1 there is nothing to look at
    const int ahead0 = max(quiet0, plain0) - 1, ahead1 = min(min(quiet1, plain1), u1) - 1;
    for (int u = u0; u < u1; ++u) {
      if (moves(top)) move_to(top);
      if (is_odd(u, u & 1)) add_odd(tiles.at(u) * C::KT), add_odd(tiles.at(u) * C::KT + 32);
      straight(u, s[0], s[1], next);  // (behind the last tile: its scores again, which nobody takes)
      s[1] = s[0], s[0] = next;
      if (u < ahead0 || u >= ahead1) {
        if (careful_with(u + 1)) look_through(1 - (u & 1));
        const int t = first_slot(u + 1);
        if (!all_seen(t, C::KT, low, high)) {
          mask(s[0], t), mask(s[1], t + 32);
          top = top_of(s[0], s[1]);
        }
      }
      __syncthreads();
    }
  }

  // ---- the key groups' results joined, and O^T turned over to rows ----
  l = half_sum(l);
  __syncthreads();
  float *patch = (float *)lds + wave * (32 * C::TP), *maxima = (float *)(lds + C::WAVES * C::PATCH), *sums = maxima + C::WAVES * 32;
  float top = m, sum = l;
  if constexpr (WK > 1) {
    if (half == 0) maxima[wave * 32 + l32] = m, sums[wave * 32 + l32] = l;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < WK; ++x) top = fmaxf(top, maxima[(x * WM + wm) * 32 + l32]);
    sum = 0.f;
#pragma unroll
    for (int x = 0; x < WK; ++x) {
      const float mx = maxima[(x * WM + wm) * 32 + l32], lx = sums[(x * WM + wm) * 32 + l32];
      sum += mx == -INFINITY ? lx : lx * __builtin_amdgcn_exp2f(mx - top);  // (0, or NaN)
    }
  }
  // what a row's O is multiplied by (NaN stays NaN), and where it goes
  const float f = (sum == 0.f ? 0.f : p.v_scale / sum) * (WK == 1 ? 1.f : m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top));
  const bool whole = parts == 1;
  const int64_t slot0 = (((int64_t)number * p.parts + part) * p.Hkv + g) * C::R;
  const int64_t to = whole ? (int64_t)(k.t0 + node) * p.Hq + head : slot0 + wm * 32 + l32;
  if (wk == 0 && half == 0 && wm * 32 + l32 < k.rows) {
    const float lse = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;  // (logf: base 2)
    if (!whole) p.part_lse[to] = lse;
    else if (p.lse) p.lse[to] = lse;
  }
#pragma unroll
  for (int j = 0; j < C::NJ; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = acc[j][i * 4 + e] * f;
      *(f32x4 *)(patch + l32 * C::TP + j * 32 + 8 * i + 4 * half) = x;
    }
  if constexpr (WK > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // a wave's rows are those of its row group; with several key groups each takes its share of them
  constexpr int LANES = D / 4, AT_ONCE = 64 / LANES, ROUNDS = 32 / WK / AT_ONCE, U = ROUNDS < 4 ? ROUNDS : 4;
  static_assert(ROUNDS % U == 0 && WK * ROUNDS * AT_ONCE == 32, "each row is joined and written by one wave");
  const int d = lane % LANES * 4;
#pragma unroll 1
  for (int n = 0; n < ROUNDS; n += U) {
    f32x4 o[U];
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = wk * (32 / WK) + (n + u) * AT_ONCE + lane / LANES;
      o[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < WK; ++x) o[u] += *(const f32x4 *)((const float *)lds + (x * WM + wm) * (32 * C::TP) + r * C::TP + d);
      at[u] = __shfl(to, r);
      if (wm * 32 + r >= k.rows) at[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at[u] < 0) continue;
      if (whole) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)o[u][e];
        *(bf16x4 *)(p.out + at[u] * D + d) = y;
      } else {
        *(f32x4 *)(p.part_out + at[u] * D + d) = o[u];
      }
    }
  }
}

// lse = log sum_s exp(lse_s), out = sum_s exp(lse_s - lse) out_s, D/4 lanes per row, eight parts in flight.
// Grid: KV head, rows of a block (1024 / D at a time), block.  (240 rows x 8 heads of 16 parts: 17 MB read, 5.7 us.)
template <int D, int R>
__global__ void __launch_bounds__(256) merge_kernel(const ChunkParams p, int KT) {
  constexpr int LPR = D / 4, U = 8, ROWS = 256 / LPR;
  const int g = blockIdx.x, r = blockIdx.y * ROWS + threadIdx.x / LPR, number = blockIdx.z;
  const Block k(p, R, number);
  const int S = Tiles(p, k, KT).parts(p, KT);
  if (S == 1 || r >= k.rows) return;
  const int64_t stride = (int64_t)p.Hkv * R, slot0 = ((int64_t)number * p.parts * p.Hkv + g) * R + r;
  const int d = (threadIdx.x % LPR) * 4;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;
  for (int s0 = 0; s0 < S; s0 += U) {
    float ls[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = slot0 + min(s0 + u, S - 1) * stride;
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
  o *= sum == 0.f ? 0.f : 1.f / sum;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)o[e];
  const int node = (k.row0 + r) / p.G, head = g * p.G + (k.row0 + r - node * p.G);
  const int64_t at = (int64_t)(k.t0 + node) * p.Hq + head;
  *(bf16x4 *)(p.out + at * D + d) = y;
  if (d == 0 && p.lse) p.lse[at] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum) * kLn2;
}

struct ChunkPlan {
  int rows, KT;    // of a workgroup, keys of its tiles
  bool by_keys;  // row blocks (Block)
  int blocks, each;
  int parts, part_keys;
};
// Rows of a workgroup.  Up to 32 rows of a sequence: 32.  More: 32 all the same where two rounds of workgroups hold them and a part has few keys
// (512 tokens alone 14.5 us, with 128 rows 21.6, behind 400 23.3 and 28.9; 256 behind 512 16.3 and 20.1; 30 behind 5000 18.7 and 20.6; but 128
// behind 1500 22.4 and 20.2, 60 behind 4096 25.7 and 23.3).  256 rows, which bring half as many tiles as 128, where 128 rows have twice the
// blocks, their keys are about as many and there are workgroups for every compute unit (2048 tokens behind 30000: 948 us, with 128 rows 1058;
// 8192 in a window of 4096 525 and 560) or 128 rows would have long parts (512 behind 16384 147 us, with 128 rows 161; 32 times 60 nodes behind
// 4096 166 and 185; but 60 behind 8192 32 and 29, 8 ragged ones of 10 to 100 119 and 90, one set of 16 ragged ones of 1 to 333 behind 100 to
// 8000 223 and 201, 70 of 1 to 30 behind up to 300 46 and 30), or where there are several rounds of blocks with many keys (4096 tokens 150 and 165; 10 times
// 2048 440 and 465; but 20 times 512 108 and 97, 70 ragged ones of 1 to 120 behind up to 3000 252 and 215).  A prompt's first chunk has row
// blocks of one tile to all, which two 128-row workgroups per CU level out (2048 tokens: 54 us, with 256 rows 63).  (A batch whose longest
// sequence is alone with its length waits for it: max_L says no more.)
// Parts: two launches cost 3 to 4 us more than one, and a partial row is written and read again.  One workgroup per CU, two where a part is long
// (32 rows, four waves to a workgroup, each with tiles of its own: one token behind 4096 in 32 parts 14.0 us, in 64 15.5; 32 sequences of 4096 in
// 2 parts 105, in 1 140.  128 rows: 60 nodes behind 4096 in 16 parts 23.3, in 32 26.5, behind 16384 39.3 and 41.4; 30 tokens behind 32768 in 32
// parts 41, in 64 46; four times 60 behind 16384 in 4 parts 112, in 8 101), of two tiles at least.  A join has to save its 32-row block some
// tiles: 16 tokens behind 600 in 2 parts 15.9 us, in one 14.1, twice 120 alone 11.5 and 7.7; one behind 512 in 8 parts 9.4, in one 12.9.
void plan_chunk(const tva_chunk_args *a, ChunkPlan *pl) {
  constexpr int kCUs = 256, kFewKeys = 768, kLongPart = 64, kLongPart128 = 24, kManyKeys = 768, kWorthAJoin = 14;
  const int G = a->Hq / a->Hkv;
  const int64_t rows = (int64_t)a->max_T * G;
  // row blocks of R rows: as many as the rows need (and one more for a sequence), or evenly as many as max_T tokens do
  auto by_rows = [&](int R) { return (int64_t)a->sum_T * G / R + a->B; };
  auto by_sequences = [&](int R) { return (int64_t)a->B * ((rows + R - 1) / R); };
  auto even = [&](int R) { return by_sequences(R) <= by_rows(R); };
  auto busy_with = [&](int R) { return std::max<int64_t>(1, std::min(by_rows(R), by_sequences(R))) * a->Hkv; };
  const int64_t all = (int64_t)a->max_L + a->max_T;
  // keys that a row sees, at the mean over a chunk
  const int64_t mean = a->window ? std::min<int64_t>(a->max_L + a->max_T / 2, (int64_t)a->window + a->n_first) : (int64_t)a->max_L + a->max_T / 2;
  auto seen_with = [&](int R, int KT) { return a->window ? std::min<int64_t>(all, (int64_t)a->window + a->n_first + R / G + 2 * KT) : all; };
  const bool long_with_128 = seen_with(128, 64) / 64 / std::max<int64_t>(1, kCUs / busy_with(128)) >= kLongPart128 && busy_with(128) <= 2 * kCUs;
  if (a->plan_rows) pl->rows = a->plan_rows;
  else if (rows <= 32 || (busy_with(32) <= 2 * kCUs && mean <= kFewKeys * std::max<int64_t>(1, kCUs / busy_with(32)))) pl->rows = 32;
  else if (rows >= 1024 && mean >= kManyKeys && busy_with(256) >= (even(256) ? 3 * kCUs / 2 : 4 * kCUs)) pl->rows = 256;
  else if (a->max_L >= a->max_T && 2 * busy_with(256) <= busy_with(128) && ((busy_with(256) >= kCUs && even(256)) || long_with_128)) pl->rows = 256;
  else pl->rows = 128;
  pl->KT = pl->rows == 32 ? 32 : 64;
  pl->each = even(pl->rows) ? (int)((rows + pl->rows - 1) / pl->rows) : 0;
  pl->blocks = (int)std::min<int64_t>(std::min(by_rows(pl->rows), by_sequences(pl->rows)), 0x7fffffff);
  const int64_t busy = busy_with(pl->rows), tiles = std::max<int64_t>(1, (seen_with(pl->rows, pl->KT) + pl->KT - 1) / pl->KT);
  int64_t parts = a->num_splits;
  if (parts == 0 && pl->rows == 32) {
    parts = std::max<int64_t>(1, kCUs / busy);
    if (tiles / parts >= kLongPart) parts = std::max<int64_t>(1, 2 * kCUs / busy);
    parts = std::min(parts, std::max<int64_t>(1, tiles / 2));
    if (tiles - tiles / parts < kWorthAJoin) parts = 1;
  } else if (parts == 0) {
    parts = std::max<int64_t>(1, kCUs / busy);
    if (pl->rows == 128 && tiles / parts >= kLongPart128) parts = std::max<int64_t>(1, 2 * kCUs / busy);
    parts = std::min(parts, std::max<int64_t>(1, tiles / 2));
  }
  parts = std::max<int64_t>(1, std::min<int64_t>(parts, tiles));
  pl->part_keys = (int)((tiles + parts - 1) / parts) * pl->KT;
  pl->parts = (int)parts;
  // (even batches gain nothing by the order and pay for it: 64 single tokens in a window of 1024 57 us, by their keys 62; lengths of 100 to 16000
  // 426 and 427)
  pl->by_keys = a->B > 1 && a->B <= 64 && !pl->each;
}

int check_chunk(const tva_chunk_args *a, bool shapes_only) {
  if (!a || a->B <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv) return TVA_INVALID_ARG;
  if (a->sum_T < 0 || a->max_T < 0 || a->max_L < 0 || a->num_splits < 0 || a->window < 0 || a->n_first < 0) return TVA_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return TVA_UNSUPPORTED;
  if (a->plan_rows != 0 && a->plan_rows != 32 && a->plan_rows != 128 && a->plan_rows != 256) return TVA_INVALID_ARG;
  if (a->max_L > 1 << 29 || a->max_T > 1 << 28 || (int64_t)a->max_T * (a->Hq / a->Hkv) > 1 << 30) return TVA_UNSUPPORTED;  // (positions below 2^30)
  if (a->anc_mask && (a->max_T > TVA_MAX_TREE || a->mask_words < 1 || a->mask_words > 2 || a->mask_words * 64 < a->max_T)) return TVA_UNSUPPORTED;
  if (shapes_only) return TVA_OK;
  if (!(a->scale > 0.f)) return TVA_INVALID_ARG;
  if (a->cache.kind < TVA_ROWS_BF16 || a->cache.kind > TVA_ROWS_E2M1) return TVA_INVALID_ARG;
  if (a->cache.kind == TVA_ROWS_E2M1) return TVA_UNSUPPORTED;
  if (a->q_stride && (a->q_stride % 8 || a->q_stride < (int64_t)a->Hq * a->D)) return TVA_INVALID_ARG;
  if (a->sum_T == 0) return TVA_OK;
  if (!a->cu_T || !a->L || !a->q || !a->out) return TVA_INVALID_ARG;
  if (((uintptr_t)a->q | (uintptr_t)a->out) & 15) return TVA_INVALID_ARG;
  return TVA_OK;
}

size_t chunk_bytes(const tva_chunk_args *a, const ChunkPlan &pl) {
  return pl.parts == 1 ? 0 : (size_t)pl.blocks * pl.parts * a->Hkv * pl.rows * (a->D + 1) * 4;
}

}  // namespace

extern "C" {

size_t tva_chunk_workspace_bytes(const tva_chunk_args *a) {
  ChunkPlan pl;
  if (check_chunk(a, true) != TVA_OK) return (size_t)-1;
  plan_chunk(a, &pl);
  return chunk_bytes(a, pl);
}

int32_t tva_chunk_plan_rows(const tva_chunk_args *a) {
  ChunkPlan pl;
  if (check_chunk(a, true) != TVA_OK) return -1;
  plan_chunk(a, &pl);
  return pl.rows;
}

int32_t tva_chunk_plan_splits(const tva_chunk_args *a) {
  ChunkPlan pl;
  if (check_chunk(a, true) != TVA_OK) return -1;
  plan_chunk(a, &pl);
  return pl.parts;
}

int tva_chunk_attn(const tva_chunk_args *a, void *stream) {
  int rc = check_chunk(a, false);
  if (rc != TVA_OK) return rc;
  ChunkParams p{};
  rc = view_of(a->cache, a->Hkv, a->D, true, &p.c);
  if (rc != TVA_OK) return rc;
  if (a->sum_T == 0 || a->max_T == 0) return TVA_OK;
  ChunkPlan pl;
  plan_chunk(a, &pl);
  const size_t need = chunk_bytes(a, pl);
  if (need && (!a->workspace || ((uintptr_t)a->workspace & 15))) return TVA_INVALID_ARG;
  if (a->workspace_bytes < need) return TVA_WORKSPACE_TOO_SMALL;
  if (pl.blocks > 65535 || pl.parts > 65535) return TVA_UNSUPPORTED;
  if (p.c.stride_tok >= 1 << 25) return TVA_UNSUPPORTED;  // (offsets among the rows that a wave brings at once)
  const bool eight = a->cache.kind == TVA_ROWS_E4M3;
  const float k_scale = !eight || a->cache.k_scale == 0.f ? 1.f : a->cache.k_scale;
  p.q = (const __bf16 *)a->q, p.cu_T = a->cu_T, p.L = a->L, p.mask = a->anc_mask;
  p.out = (__bf16 *)a->out, p.lse = a->lse;
  p.part_out = (float *)a->workspace, p.part_lse = p.part_out + (need ? need / 4 / (a->D + 1) * a->D : 0);
  p.q_stride = a->q_stride ? a->q_stride : (int64_t)a->Hq * a->D;
  p.B = a->B, p.Hq = a->Hq, p.Hkv = a->Hkv, p.G = a->Hq / a->Hkv, p.W = a->mask_words, p.blocks = pl.blocks, p.by_keys = pl.by_keys, p.each = pl.each, p.max_T = a->max_T;
  p.parts = pl.parts, p.part_keys = pl.part_keys;
  p.window = a->window ? std::min(a->window, 1 << 30) : 1 << 30, p.n_first = a->window ? a->n_first : 0;
  p.scale_log2 = a->scale * kLog2e * k_scale, p.v_scale = !eight || a->cache.v_scale == 0.f ? 1.f : a->cache.v_scale;
  const int first_round = 256 / a->Hkv;
  p.longest = pl.by_keys ? 0 : pl.rows == 128 && pl.parts == 1 && pl.blocks > first_round && pl.blocks <= 2 * first_round ? first_round : pl.blocks;
  const dim3 grid(a->Hkv, pl.parts, pl.blocks);
  const hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  auto launch = [&](auto d, auto wm, auto wk, auto kb) {
    constexpr int D = decltype(d)::value, WM = decltype(wm)::value, WK = decltype(wk)::value, KB = decltype(kb)::value, THREADS = 64 * WM * WK;
    auto form = [&](auto kind) {
      constexpr int KIND = decltype(kind)::value;
      typedef ChunkCfg<D, WM, WK, KB, KIND> C;
      static_assert(C::KT == (WM == 1 ? 32 : 64), "plan_chunk");
      auto go = [&](auto places) {
        constexpr int PLACES = decltype(places)::value;
        if (a->anc_mask) hipLaunchKernelGGL((chunk_kernel<D, WM, WK, KB, KIND, PLACES, true>), grid, dim3(THREADS), 0, st, p);
        else hipLaunchKernelGGL((chunk_kernel<D, WM, WK, KB, KIND, PLACES, false>), grid, dim3(THREADS), 0, st, p);
      };
      if (!a->cache.page_table) go(std::integral_constant<int, kDense>{});
      else if (a->cache.page_size % C::RPW == 0 && p.c.stride_page < 1ll << 31 && p.c.stride_tok * p.c.page_size < 1ll << 31) go(std::integral_constant<int, kPages>{});
      else go(std::integral_constant<int, kRows>{});
    };
    if (eight) form(std::integral_constant<int, TVA_ROWS_E4M3>{});
    else form(std::integral_constant<int, TVA_ROWS_BF16>{});
    if (pl.parts > 1 && hipPeekAtLastError() == hipSuccess)
      hipLaunchKernelGGL((merge_kernel<D, 32 * WM>), dim3(a->Hkv, 32 * WM / (1024 / D), pl.blocks), dim3(256), 0, st, p, pl.KT);
  };
  typedef std::integral_constant<int, 1> one;
  typedef std::integral_constant<int, 2> two;
  typedef std::integral_constant<int, 4> four;
  typedef std::integral_constant<int, 8> many;
  auto shapes = [&](auto d) {
    if (pl.rows == 32) launch(d, one{}, four{}, one{});
    else if (pl.rows == 128) launch(d, four{}, one{}, two{});
    else launch(d, many{}, one{}, two{});
  };
  if (a->D == 128) shapes(std::integral_constant<int, 128>{});
  else shapes(std::integral_constant<int, 64>{});
  return hipPeekAtLastError() == hipSuccess ? TVA_OK : TVA_HIP_ERROR;
}

size_t tva_sizeof_chunk_args(void) { return sizeof(tva_chunk_args); }

}  // extern "C"
