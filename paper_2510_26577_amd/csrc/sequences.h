// Which sequence a row (or a block of rows) of a ragged batch belongs to, found by a wave (gfx950).
#ifndef TVA_SEQUENCES_H
#define TVA_SEQUENCES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sequences {

// The largest b of 0 .. B-1 with start(b) <= x, start not falling and start(0) <= x; all 64 lanes take part.  64 starts at a time:
// one read for up to 64 sequences, two for up to 4096, none for one.
template <class F>
__device__ __forceinline__ int find(int B, F start_not_above) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const bool yes = lane * step < n && start_not_above(lo + min(lane * step, n - 1));
    const int skip = ((int)__popcll(__ballot(yes)) - 1) * step;
    if (skip < 0) break;
    lo += skip, n = min(step, n - skip);
  }
  return lo;
}

}  // namespace sequences
#endif
