// Host-only check of a verification's lists of tiles, built by g++ under
// -fsanitize=address,undefined: prefixes of every length in a range, whose slots all see
// the cached keys t > prefix - window or t < sinks.  Key by key: what is seen is in
// exactly one tile, a tile loads only keys that are seen, and the pages staged for a part
// of the list are those of its keys and no others.  (A window of one key is the slot
// itself: of the prefix it holds nothing, so that there is no tile for it.)
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "simsd_span_list.h"

using namespace simsd;

static long g_fail = 0, g_checks = 0;
#define EXPECT(cond)                                                                    \
  do {                                                                                  \
    ++g_checks;                                                                         \
    if (!(cond)) {                                                                      \
      if (++g_fail < 20)                                                                \
        std::fprintf(stderr, "tile %d window %d sinks %d prefix %d page %d: %s\n", TK, window, sinks, kv, P, #cond); \
    }                                                                                   \
  } while (0)

static void one(int TK, int window, int sinks, int kv, int P) {
  auto seen = [&](int t) { return t < kv && (!window || t > kv - window || t < sinks); };
  const int first = window ? std::max(0, kv - window + 1) : 0;
  const Span s = span_of(sinks, first, kv, TK);
  std::vector<int> home(kv + 1, 0);
  bool some = true, kept = true, once = true;
  for (int L = 0; L < s.tiles; ++L) {
    const TileKeys k = tile_keys(s, L, TK);
    some &= k.beg < k.end && k.end <= kv && k.k0 < k.end && k.k0 + TK > k.beg;
    for (int j = 0; j < TK; ++j) kept &= seen(std::max(k.beg, std::min(k.k0 + j, k.end - 1)));
    for (int half = 0; half < TK / 32; ++half) {
      const uint32_t w = seen_word(s, k, k.k0 + 32 * half, kv, first);
      for (int j = 0; j < 32; ++j) {
        const int t = k.k0 + 32 * half + j;
        once &= (w >> j & 1) == row_sees(s, k, t, kv, first);
        if (!(w >> j & 1)) continue;
        once &= seen(t);
        if (t < kv) ++home[t];
      }
    }
  }
  for (int t = 0; t < kv; ++t) once &= home[t] == seen(t);
  EXPECT(some);
  EXPECT(kept);
  EXPECT(once);
  // Every part of the list.
  bool staged = true, used = true;
  for (int t0 = 0; t0 < s.tiles; ++t0)
    for (int t1 : {t0 + 1, t0 + 2, s.tiles, s.tiles + 1}) {
      const PageSpan g = pages_of(s, t0, t1, TK, P);
      for (int L = t0; L < std::min(t1, s.tiles); ++L) {
        const TileKeys k = tile_keys(s, L, TK);
        for (int j = 0; j < TK; ++j) {
          const int page = std::max(k.beg, std::min(k.k0 + j, k.end - 1)) / P;
          staged &= k.sink ? page >= g.first_sink && page < g.first_sink + g.sinks
                           : page >= g.first_win && page < g.first_win + g.wins;
        }
      }
      auto has = [&](int page) {
        for (int t = page * P; t < std::min(kv, (page + 1) * P); ++t)
          if (seen(t)) return true;
        return false;
      };
      for (int i = 0; i < g.sinks; ++i) used &= has(g.first_sink + i);
      for (int i = 0; i < g.wins; ++i) used &= has(g.first_win + i);
    }
  EXPECT(staged);
  EXPECT(used);
}

int main() {
  for (int kv = 0; kv <= 200; ++kv)
    for (int window : {0, 1, 2, 3, 31, 32, 33, 64, 65, 130, 300})
      for (int sinks : {0, 1, 4, 32, 64, 65, 90, 1000}) {
        if (!window && sinks) continue;
        for (int P : {1, 3, 16, 24, 64, 100})
          for (int TK : {32, 64}) one(TK, window, sinks, kv, P);
      }
  std::printf("%ld checks, %ld failed\n", g_checks, g_fail);
  return g_fail ? 1 : 0;
}
