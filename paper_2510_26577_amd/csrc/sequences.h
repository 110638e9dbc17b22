// Which sequence a row (or a block of rows) of a ragged batch belongs to, found by a wave (gfx950).
#ifndef TVA_SEQUENCES_H
#define TVA_SEQUENCES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sequences {

struct Place {
  int b, t0, t1;  // the sequence, its first row and the row behind its last
  int L;          // its cached tokens (0 where no lengths are given)
};

// The largest b of 0 .. B-1 whose start(b, cu_T[b]) is at most x; start does not fall, and start of 0 is at most x.  All 64 lanes take part.
// Up to 64 sequences: one round of reads that do not wait for each other, whatever is found; beyond, 64 starts at a time, then its own.
template <class F>
__device__ __forceinline__ Place find(const int32_t *cu_T, const int32_t *L, int B, int64_t x, F start) {
  const int lane = threadIdx.x & 63;
  Place at;
  if (B <= 64) {
    const int n = min(lane, B - 1), from = cu_T[n], to = cu_T[n + 1], len = L ? L[n] : 0;
    at.b = max((int)__popcll(__ballot(lane < B && start(n, from) <= x)) - 1, 0);
    at.t0 = __builtin_amdgcn_readlane(from, at.b), at.t1 = __builtin_amdgcn_readlane(to, at.b), at.L = __builtin_amdgcn_readlane(len, at.b);
    return at;
  }
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lo + min(lane * step, n - 1);
    const int skip = max((int)__popcll(__ballot(lane * step < n && start(i, cu_T[i]) <= x)) - 1, 0) * step;
    lo += skip, n = min(step, n - skip);
  }
  at.b = lo, at.t0 = cu_T[lo], at.t1 = cu_T[lo + 1], at.L = L ? L[lo] : 0;
  return at;
}

}  // namespace sequences
#endif
