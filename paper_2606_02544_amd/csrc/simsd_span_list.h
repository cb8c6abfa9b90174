// Which cached keys a row block sees under a sliding window with sinks, as a list of
// tiles.
//
// A row at position p, in the block of m positions that starts at p0 = p / m * m, sees
// the keys t < min(kv, p0 + m) with t > p0 - window or t < sinks.  Over the rows of a
// block that is [0, sinks) and [lo, hi), lo being the first row's first key and hi the
// last row's limit.  If the two meet, the list goes from key 0 (from lo without sinks)
// to hi; otherwise it has tiles for the sinks, which every row sees whole, and then
// those of [lo, hi), of which there are none if that is empty: a verification's slots see
// no cached key by a window of one, lo = hi being the prefix's length.  Keys outside both
// parts are never read, nor are their pages: a cache may have given them away, and the
// key at hi may lie behind its end.
#pragma once

#include <algorithm>
#include <cstdint>

#ifdef __HIP__
#define SIMSD_LIST __device__ __attribute__((always_inline)) inline
#else
#define SIMSD_LIST inline        // (a test goes through every list on the CPU)
#endif

namespace simsd {
namespace {

#ifndef __HIP__
using std::max;
using std::min;
#endif

struct Span {
  int lo, hi;                    // keys of the window's tiles
  int win0;                      // first key of the first of them
  int sink_end, sink_tiles;      // sinks in tiles of their own
  int tiles;                     // cached tiles in all
  int near;                      // one list: keys below this are seen whatever the window
};

// Keys that the token at `pos` of a sequence of kv sees without a window: those below
// this (m: positions of the mask's blocks; 0: one block).
SIMSD_LIST int limit_at(int m, int kv, int pos) {
  if (pos < 0) return 0;
  return m ? min(kv, (pos / m + 1) * m) : kv;
}
// First key of its window (0: no window, or no token).
SIMSD_LIST int first_at(int m, int window, int pos) {
  return window && pos >= 0 ? max(0, pos / m * m - window + 1) : 0;
}

// From the first row's first key and the last row's limit; TK keys to a tile.
SIMSD_LIST Span span_of(int all_sinks, int first, int hi, int TK) {
  Span s;
  const int sinks = min(all_sinks, hi);
  const bool apart = first > sinks;
  s.lo = apart ? first : 0;
  s.hi = hi;
  s.near = apart ? 0 : sinks;
  s.sink_end = apart ? sinks : 0;
  s.sink_tiles = (s.sink_end + TK - 1) / TK;
  s.win0 = s.lo / TK * TK;
  s.tiles = s.sink_tiles + (hi > s.lo ? (hi - s.win0 + TK - 1) / TK : 0);
  return s;
}

// Tile L of the list: its first key, and which of its keys there are.  (The pluses make
// the compiler choose between values, not between the members' addresses, which would
// put the structure in memory.)
struct TileKeys {
  int k0, beg, end;
  bool sink;
};
SIMSD_LIST TileKeys tile_keys(const Span& s, int L, int TK) {
  const bool sink = L < s.sink_tiles;
  return {sink ? L * TK : s.win0 + (L - s.sink_tiles) * TK, sink ? 0 : s.lo, sink ? +s.sink_end : +s.hi, sink};
}

// The pages that the tiles [t0, t1) of the list lie in: `sinks` of them from first_sink
// on, and `wins` from first_win on.
struct PageSpan {
  int first_sink, sinks, first_win, wins;
};
SIMSD_LIST PageSpan pages_of(const Span& s, int t0, int t1, int TK, int P) {
  PageSpan p = {0, 0, 0, 0};
  t1 = min(t1, s.tiles);
  const int sink1 = min(t1, s.sink_tiles), win0 = max(t0, s.sink_tiles);
  if (t0 < sink1) {
    p.first_sink = t0 * TK / P;
    p.sinks = (min(s.sink_end, sink1 * TK) - 1) / P - p.first_sink + 1;
  }
  if (win0 < t1) {
    const int k0 = s.win0 + (win0 - s.sink_tiles) * TK, k1 = s.win0 + (t1 - s.sink_tiles) * TK;
    p.first_win = max(s.lo, k0) / P;
    p.wins = (min(s.hi, k1) - 1) / P - p.first_win + 1;
  }
  return p;
}

// The keys [0, n) of 32 as a word.
SIMSD_LIST uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// What a row with this limit and first key sees of the 32 keys from k on, in a tile of
// the list.
SIMSD_LIST uint32_t seen_word(const Span& s, const TileKeys& t, int k, int limit, int first) {
  const int hi = t.sink ? min(limit, s.sink_end) : limit;
  return (low_bits(hi - k) & ~low_bits((t.sink ? 0 : first) - k)) | low_bits(min(s.near, limit) - k);
}
// The same of one key.
SIMSD_LIST bool row_sees(const Span& s, const TileKeys& t, int key, int limit, int first) {
  const int end = s.sink_end, near = s.near;
  const int hi = t.sink ? min(limit, end) : limit, lo = t.sink ? 0 : first;
  return key < hi && (key >= lo || key < near);
}

}  // namespace
}  // namespace simsd
