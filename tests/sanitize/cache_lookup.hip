// The places of positions in a paged cache whose table has entries below 0 among those that are looked up (csrc/cache_rows.h), on the host:
// every place lies in the cache, and those of pages that are there are the right ones.
#include <climits>
#include <cstdio>
#include <random>
#include <vector>

#include "cache_rows.h"

using cache_rows::CacheView;
using cache_rows::Finder;

int main() {
  std::mt19937 rng(7);
  int failures = 0;
  long looked = 0, gone = 0;
  for (int page_size : {1, 4, 5, 16, 24, 48, 64})
    for (int kind : {TVA_ROWS_BF16, TVA_ROWS_E4M3})
      for (bool head_major : {false, true}) {
        const int B = 3, Hkv = 2, D = 64, pages = 7, max_pages = 11;
        std::vector<int32_t> table(B * max_pages);
        for (int32_t &x : table) {
          const int32_t none[4] = {-1, -7, INT_MIN, -(1 << 20)};
          x = rng() % 3 ? (int32_t)(rng() % pages) : none[rng() % 4];
        }
        tva_cache a{};
        a.kind = kind, a.page_size = page_size, a.max_pages = max_pages, a.page_table = table.data();
        a.k = a.v = (void *)64;  // (never read)
        if (head_major) a.stride_tok = D, a.stride_head = (int64_t)page_size * D, a.stride_page = (int64_t)Hkv * page_size * D;
        CacheView c;
        if (cache_rows::view_of(a, Hkv, D, true, &c) != TVA_OK) ++failures;
        const int64_t all = (int64_t)pages * page_size * Hkv * D;
        for (int b = 0; b < B; ++b)
          for (int g = 0; g < Hkv; ++g) {
            const Finder<true, true> find(c, b, g);
            for (int t = 0; t < max_pages * page_size; ++t, ++looked) {
              const int32_t page = table[b * max_pages + t / page_size];
              const int64_t at = find.at(c, t, find.entry(c, t));
              const int64_t want = head_major ? (((int64_t)(page < 0 ? 0 : page) * Hkv + g) * page_size + t % page_size) * D
                                              : (((int64_t)(page < 0 ? 0 : page) * page_size + t % page_size) * Hkv + g) * D;
              failures += at < 0 || at + D > all || at != want || find.entry_of(t / page_size) < 0;
              gone += page < 0;
            }
          }
      }
  printf("%ld positions, %ld of them in pages that are gone, %d failure(s)\n", looked, gone, failures);
  return failures != 0 || gone == 0;
}
