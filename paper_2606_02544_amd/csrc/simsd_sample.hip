// Sampling from filtered logits on gfx950: temperature, top-k, top-p, min-p and
// the draw from a given uniform number, one work-group per row.
//
// With the row's largest logit m, token i weighs w_i = exp((x_i - m) / T).  In
// the order of falling logits (the lowest index first among equal ones) every
// filter keeps a leading part: the first k; the fewest whose weights reach
// top_p of what top-k left; those with w_i >= min_p.  The token drawn is the
// first whose running weight exceeds u times the weight of the kept ones.  So a
// row needs no sort: each cut, and the draw, is a search in the running sums
// over the distinct logits from the top, and equal logits are told apart by
// counting.
//
// Weights are 64-bit fixed-point numbers with S = 62 - ceil(log2 V) binary
// places (exp in fp64, rounded once): their sums do not depend on the order of
// additions, so the token is the same on every run, and they are exact to
// V * 2^-(S+1) of the largest weight (V = 151936: 4e-9 at worst, 1e-11 as the
// roundings add up).  fp32 sums would move one boundary in a few hundred past a
// given u.
//
// bf16 rows: a logit is one of 65536 bit patterns, so one histogram of counts
// holds the row: 16-bit counters, two to an LDS word, 128 KB.  The row stays in
// registers (8 waves x 38 loads of 16 bytes a lane, up to 155648 entries; a longer
// row is read again), is read from memory once, and the weights are taken of the
// distinct values only (some 3000 of a row of 151936 logits N(0, 4)).  A counter that
// passes 65535 shows in the total and the histogram is built again, noting each wrap.
// What bounds a row is one work-group's LDS and issue, not memory: of a row of 151936
// (4 rows N(0, 4) without a filter: 42 us; 256: 52; 512: 95), a tenth is the read, nearly
// half the counting (2432 LDS atomics of a wave, 15 cycles each), a sixth the weights, the
// rest the cuts and the token's index.
// fp32 rows: the weights are added up in 8192 bins of the upper 13 bits of the
// ordered bit pattern; a search goes on in the bin it ends in, 10 and then 9
// bits further, over the row again, which the caches hold by then.
// What bounds them: two LDS atomics and an fp64 exp an entry, in one work-group a row (4
// rows of 151936: 156 us without a filter, 229 with top-p; 256 rows: 210 and 271).  A
// list of the bin's entries for the last 9 bits made rows with k = 1000 faster (by 15 %)
// and others, whose bins hold more than it, slower (by 8 %).
#include <type_traits>

#include "simsd_ops_kernels.h"

namespace simsd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int NT = 512;          // threads of a work-group
constexpr int NW = NT / 64;
constexpr int kRegs = 38;        // 16-byte loads of a bf16 row that a lane keeps; even
constexpr double kCut = 700.0;   // a token further below the maximum, in temperatures, is never kept

struct Params {
  double T, inv, top_p, min_p;   // inv = 1 / T
  uint32_t top_k;                // 0: off
  bool greedy;
};

// A logits value's place in the running sums.
struct Found {
  uint32_t key;                  // its key (bf16: place in the falling order; fp32: ordered pattern)
  uint32_t n_before, n;          // tokens above it, tokens equal to it
  uint64_t z_before, w;          // weight above it, weight of one such token
};

// Value of the lane that the DPP control names, 0 where there is none.
template <int CTRL, int ROWS>
__device__ inline uint32_t moved(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false));
}
__device__ inline uint64_t lane64(uint64_t v, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), l);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), l);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}

struct Sum {
  uint32_t n;
  uint64_t z;
};

template <int CTRL, int ROWS>
__device__ inline void add_moved(Sum& v) {
  const uint32_t n = moved<CTRL, ROWS>(v.n);
  const uint64_t lo = moved<CTRL, ROWS>(static_cast<uint32_t>(v.z));
  const uint64_t hi = moved<CTRL, ROWS>(static_cast<uint32_t>(v.z >> 32));
  v.n += n;
  v.z += hi << 32 | lo;
}
// Inclusive sums over the lanes: shifts by 1, 2, 4 and 8 within rows of 16, then
// the last lanes of rows into the rows after them.
__device__ inline Sum wave_scan(Sum v) {
  add_moved<0x111, 0xf>(v);
  add_moved<0x112, 0xf>(v);
  add_moved<0x114, 0xf>(v);
  add_moved<0x118, 0xf>(v);
  add_moved<0x142, 0xa>(v);
  add_moved<0x143, 0xc>(v);
  return v;
}

__device__ inline double weight(double gap, const Params& p) { return exp(gap * p.inv); }

// The row's segments: wave w holds the 16-byte vectors [w*seg, (w+1)*seg) of the
// row's aligned part, lane by lane; wave 0 also the entries before it (`extra`
// of lane i: entry i) and the last wave those behind it.
struct Segment {
  const u32x4* base;             // vector 0 of the row
  int first, count;              // of this wave's vectors
  int head;                      // entries before vector 0
  int extra;                     // this lane's entry outside the vectors, or -1
};

template <bool BF16>
__device__ inline Segment segment_of(const void* row, int V, int wave, int lane) {
  constexpr int VEC = BF16 ? 8 : 4;
  constexpr int ESZ = 16 / VEC;
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15u) / ESZ;
  Segment s;
  s.head = min(lead ? VEC - lead : 0, V);
  const int nvec = (V - s.head) / VEC, tail = V - s.head - nvec * VEC;
  s.base = reinterpret_cast<const u32x4*>(static_cast<const char*>(row) + s.head * ESZ);
  const int seg = ((nvec + NW - 1) / NW + 63) / 64 * 64;
  s.first = min(wave * seg, nvec);
  s.count = min(seg, nvec - s.first);
  s.extra = -1;
  if (wave == 0 && lane < s.head) s.extra = lane;
  if (wave == NW - 1 && lane < tail) s.extra = V - tail + lane;
  return s;
}

// Lanes past the end of a row hold the pattern of a NaN, which no filter keeps.
constexpr uint32_t kNone = 0xffffffffu;

// The wave's vectors in registers (rows of up to NW * 64 * kRegs vectors).
__device__ inline __attribute__((always_inline)) void load_row(u32x4 (&reg)[kRegs], const Segment& s, int lane) {
#pragma unroll
  for (int j = 0; j < kRegs; ++j) {
    reg[j] = u32x4{kNone, kNone, kNone, kNone};
    if (j * 64 + lane < s.count) reg[j] = s.base[s.first + j * 64 + lane];
  }
}

// f(j, vector) of the vectors in registers.  The code of f is there 38 times, so it
// is short, and what few vectors need is done by visit().  (Eight to a test of the
// count: a test each takes more scalar registers than there are; and vectors side by
// side take more vector registers.)
template <typename F>
__device__ inline __attribute__((always_inline)) void each_held(const u32x4 (&reg)[kRegs], const Segment& s, F f) {
#pragma unroll
  for (int b = 0; b < kRegs; b += 8)
    if (b * 64 < s.count) {
#pragma unroll
      for (int j = b; j < (b + 8 < kRegs ? b + 8 : kRegs); ++j) {
        f(j, reg[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
}

// f(j[], vector[]) of the wave's vectors as they lie in memory, four at a time: those
// of the bits of `hits` (j < 64), or, without HITS, all of them.  (Past the last
// one: vectors of NaN, j the last one's.)
constexpr int kBatch = 4;
template <bool HITS, typename F>
__device__ inline __attribute__((always_inline)) void visit_batches(const Segment& s, uint64_t hits, int lane, F f) {
  int next = 0;
  while (HITS ? hits != 0 : next * 64 < s.count) {
    int j[kBatch];
    u32x4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      bool is = true;
      if (HITS) {
        is = hits != 0;
        j[i] = is ? __builtin_ctzll(hits) : j[i ? i - 1 : 0];
        hits &= hits - 1;
      } else {
        j[i] = next++;
      }
      v[i] = u32x4{kNone, kNone, kNone, kNone};
      if (is && j[i] * 64 + lane < s.count) v[i] = s.base[s.first + j[i] * 64 + lane];
    }
    f(j, v);
  }
}
template <bool HITS, typename F>
__device__ inline __attribute__((always_inline)) void visit(const Segment& s, uint64_t hits, int lane, F f) {
  visit_batches<HITS>(s, hits, lane, [&](const int (&j)[kBatch], const u32x4 (&v)[kBatch]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) f(j[i], v[i]);
  });
}

__device__ inline Params params_of(const SampleArgs& a, int r) {
  Params p;
  // (An infinite temperature as the largest finite one: gap / T stays a number.)
  const float T = a.temperatures ? a.temperatures[r] : a.temperature;
  p.T = static_cast<double>(T > __FLT_MAX__ ? __FLT_MAX__ : T);
  const int k = a.top_ks ? a.top_ks[r] : a.top_k;
  p.top_p = static_cast<double>(a.top_ps ? a.top_ps[r] : a.top_p);
  p.min_p = static_cast<double>(a.min_ps ? a.min_ps[r] : a.min_p);
  p.greedy = !(p.T > 0.0);
  p.inv = 1.0 / p.T;
  p.top_k = k > 0 ? k : 0;
  return p;
}

// First token of the kept part's running sums past u * z.
__device__ inline uint64_t draw_target(float u, uint64_t z) {
  const double v = fmin(fmax(static_cast<double>(u), 0.0), 1.0);
  const uint64_t t = static_cast<uint64_t>(v * static_cast<double>(z));
  return t < z ? t : z - 1;
}

// Inclusive sum of a count over the lanes.
__device__ inline uint32_t count_scan(uint32_t v) {
  v += moved<0x111, 0xf>(v);
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);
  v += moved<0x143, 0xc>(v);
  return v;
}
__device__ inline uint32_t last_lane(uint32_t v) { return __builtin_amdgcn_readlane(v, 63); }

// The index of the rank-th entry (0-based, in vocabulary order) that matches, found
// by the wave that holds it, which writes the outputs.  `bits`: which entries of a
// vector match; `hits`: the vectors to look at, as in visit().
template <int VEC, bool HITS, typename Bits>
__device__ inline __attribute__((always_inline)) void find_and_write(
    const SampleArgs& a, int r, const Segment& s, uint64_t hits, uint32_t rank, float prob, uint32_t kept,
    int wave, int lane, uint32_t* s_count, bool extra_match, Bits bits) {
  uint32_t count = extra_match ? 1 : 0;
  visit<HITS>(s, hits, lane, [&](int, const u32x4& v) __attribute__((always_inline)) { count += __popc(bits(v)); });
  count = last_lane(count_scan(count));
  if (lane == 0) s_count[wave] = count;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += s_count[w];
  before = __builtin_amdgcn_readfirstlane(before);
  if (rank < before || rank >= before + count) return;   // uniform: another wave's
  uint32_t left = rank - before;
  int found = -1;
  // One step: lanes hold `own` matches each, in order; takes the left-th.
  auto take = [&](uint32_t b, int index) __attribute__((always_inline)) {   // b: matches, from index on
    const uint32_t own = __popc(b);
    const uint32_t incl = count_scan(own), total = last_lane(incl);
    if (found < 0 && left < total) {
      const bool mine = incl - own <= left && left < incl;
      uint32_t skip = left - (incl - own);
      int at = 0;
      if (mine) {
        while (skip--) b &= b - 1;
        at = __builtin_ctz(b);
      }
      found = __builtin_amdgcn_readlane(index + at, __builtin_ctzll(__ballot(mine)));
    }
    if (found < 0) left -= total;
  };
  if (wave == 0) take(extra_match && s.extra < s.head ? 1 : 0, s.extra);
  visit<HITS>(s, found >= 0 ? 0 : hits, lane, [&](int j, const u32x4& v) __attribute__((always_inline)) {
    take(bits(v), s.head + (s.first + j * 64 + lane) * VEC);
  });
  if (wave == NW - 1) take(extra_match && s.extra >= s.head ? 1 : 0, s.extra);
  if (lane == 0) {
    a.token[r] = found;
    if (a.prob) a.prob[r] = prob;
    if (a.kept) a.kept[r] = static_cast<int32_t>(kept);
  }
}

__device__ inline void write_none(const SampleArgs& a, int r) {
  if (threadIdx.x == 0) {
    a.token[r] = -1;
    if (a.prob) a.prob[r] = 0.f;
    if (a.kept) a.kept[r] = 0;
  }
}

// Sum over the work-group up to and including each thread; *total for all.
__device__ inline Sum block_scan(Sum v, int wave, int lane, Sum* s_wave, Sum* total) {
  v = wave_scan(v);
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  Sum all = {0, 0}, before = {0, 0};
  for (int w = 0; w < NW; ++w) {
    if (w == wave) before = all;
    all.n += s_wave[w].n;
    all.z += s_wave[w].z;
  }
  __syncthreads();
  v.n += before.n;
  v.z += before.z;
  *total = all;
  return v;
}

// What a search looks for: the first token at which the running count or weight
// reaches `target` (kCount, kReach) or passes it (kPass).
enum Kind { kCount, kReach, kPass };
__device__ inline bool reached(Kind k, const Sum& s, uint64_t target) {
  return k == kCount ? s.n >= target : k == kReach ? s.z >= target : s.z > target;
}

// What of a row's `all` tokens is kept, and the token drawn: up to three searches
// by `find`, in one loop so that its code exists once.  `min_p`: the part that
// min_p keeps.  Returns the draw's place; *rank among its equals; *kept the part.
template <typename Find>
__device__ inline __attribute__((always_inline)) Found cut_and_draw(const Params& p, Sum all, Sum min_p, float u,
                                                                   uint32_t* rank, Sum* kept, Find find) {
  Sum by_k = all, out = all;
  Found f = {};
  for (int stage = 0; stage < 3; ++stage) {
    Kind kind;
    uint64_t target;
    if (stage == 0) {
      if (!p.top_k || p.top_k >= all.n) continue;
      kind = kCount;
      target = p.top_k;
    } else if (stage == 1) {
      if (!(p.top_p < 1.0)) continue;
      kind = kReach;
      target = static_cast<uint64_t>(ceil(fmax(p.top_p, 0.0) * static_cast<double>(by_k.z)));
      target = min(max(target, uint64_t{1}), by_k.z);
    } else {
      if (min_p.n < out.n) out = min_p;
      kind = kPass;
      target = draw_target(u, out.z);
    }
    f = find(kind, target);
    if (stage == 0) {
      by_k = Sum{p.top_k, f.z_before + (p.top_k - f.n_before) * f.w};
      out = by_k;
    } else if (stage == 1) {
      uint64_t n = (target - f.z_before + f.w - 1) / f.w;
      n = min(max(n, uint64_t{1}), static_cast<uint64_t>(f.n));
      if (f.n_before + n < out.n) out = Sum{f.n_before + static_cast<uint32_t>(n), f.z_before + n * f.w};
    } else {
      *rank = static_cast<uint32_t>((target - f.z_before) / f.w);
    }
  }
  *kept = out;
  return f;
}

// ----------------------------------------------------------------------------
// The short way: where few tokens can be kept, they are sorted.
//
// A row's candidates are the entries not below a bound that no kept token is
// under: the maximum itself (T <= 0); the maximum less kCut T; m + T ln(min_p) where
// top_p is off; and the k-th largest of the maxima of the row's parts (k parts
// hold an entry not below it; a part is an eighth of a bf16 lane's entries, a quarter
// of an fp32 lane's).  Up to kCap of them are put in LDS in the order of falling
// logits and rising index, and every search is one in running sums over that list; a
// row with more goes the long way below.  Per call, long way -> short way: 4 bf16 rows
// of 151936 with k = 50, 57 -> 17 us; 61 fp32 rows of 50001 with min_p 0.02, 80 ->
// 22 us; 512 bf16 rows with settings of all kinds, 121 -> 90 us.
// ----------------------------------------------------------------------------
constexpr int kCap = 1024;

struct Small {                   // LDS beside the large arrays
  Sum wave[NW];
  uint32_t count[NW];
  float top[NW];
  uint32_t tally[2][NW];
  uint32_t listed;
  Found found;
};
struct List {
  uint64_t key[kCap];            // falling pattern << 32 | index
  uint64_t sorted[NT];
  uint32_t index[kCap];
  uint8_t mask[NW][kRegs][64];   // which of a lane's entries of a vector are candidates
};

// Bit patterns of fp32 in rising order; -0 as +0.
__device__ inline uint32_t ordered(uint32_t b) {
  if (b == 0x80000000u) b = 0;
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ inline float ordered_float(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Entry e of a vector, as fp32 bits.
template <bool BF16>
__device__ inline uint32_t entry(const u32x4& v, int e) {
  if constexpr (BF16) return e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16;
  else return v[e];
}

template <int CTRL, int ROWS>
__device__ inline float max_moved(float v) {
  const int b = __builtin_bit_cast(int, v);
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, ROWS, 0xf, false)));
}
// The largest of the lane's maxima over the wave, and over the work-group.
__device__ inline float wave_maximum(float m) {
  m = max_moved<0x111, 0xf>(m);
  m = max_moved<0x112, 0xf>(m);
  m = max_moved<0x114, 0xf>(m);
  m = max_moved<0x118, 0xf>(m);
  m = max_moved<0x142, 0xa>(m);
  m = max_moved<0x143, 0xc>(m);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), 63));
}
__device__ inline float block_maximum(float m, int wave, int lane, Small& sm) {
  m = wave_maximum(m);
  if (lane == 0) sm.top[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) m = fmaxf(m, sm.top[w]);
  return m;
}

// Maxima of this lane's parts of the row: key[i] the upper 16 bits of ordered(); and
// the row's largest entry (-inf where there is none that is a number).
constexpr uint32_t kNoKey = 0x7f;                // of -inf
template <bool BF16>
__device__ inline __attribute__((always_inline)) float part_maxima_read(const Segment& s, uint32_t xbits, int wave, int lane, Small& sm,
                                                                       uint32_t (&key)[4]) {
  constexpr int VEC = BF16 ? 8 : 4;
  float part[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) part[i] = -__builtin_huge_valf();
  part[0] = fmaxf(part[0], __uint_as_float(xbits));
  visit<false>(s, 0, lane, [&](int j, const u32x4& v) __attribute__((always_inline)) {
    float m = -__builtin_huge_valf();
#pragma unroll
    for (int e = 0; e < VEC; ++e) m = fmaxf(m, __uint_as_float(entry<BF16>(v, e)));
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i] = (j & 3) == i ? fmaxf(part[i], m) : part[i];
  });
#pragma unroll
  for (int i = 0; i < 4; ++i) key[i] = ordered(__float_as_uint(part[i])) >> 16;
  return block_maximum(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])), wave, lane, sm);
}
// bf16 in registers: two entries at a time as 16-bit integers in the order of their
// values; NaN of positive sign would be the largest, and sends the row to the other
// form (*odd).  `pair`: the maxima of two vectors each, even and odd entries apart.
constexpr int kPairs = kRegs / 2;
__device__ inline s16x2 rising(uint32_t w) {
  const s16x2 x = __builtin_bit_cast(s16x2, w);
  return x ^ ((x >> s16x2{15, 15}) & s16x2{0x7fff, 0x7fff});
}
// The row's largest entry from the lanes' largest.
__device__ inline float row_maximum(int best, int wave, int lane, Small& sm, bool* odd) {
  // Back to the pattern: non-negative ones are themselves.
  const uint32_t bits = static_cast<uint32_t>(best >= 0 ? best : best ^ 0x7fff) << 16;
  const float m = __uint_as_float(bits);
  const float top = block_maximum(m == m ? m : -__builtin_huge_valf(), wave, lane, sm);   // (nothing but NaN: -inf)
  *odd = __syncthreads_or(best > 0x7f80) != 0;
  return top;
}
__device__ inline __attribute__((always_inline)) float part_maxima_held(const u32x4 (&reg)[kRegs], const Segment& s, uint32_t xbits,
                                                                       int wave, int lane, Small& sm, uint32_t (&key)[8],
                                                                       s16x2 (&pair)[kPairs], bool* odd) {
  s16x2 part[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) part[i] = s16x2{-0x8000, -0x8000};
#pragma unroll
  for (int i = 0; i < kPairs; ++i) pair[i] = s16x2{-0x8000, -0x8000};
  // (The entry outside the vectors is of one half's part: in both, it would count as two of the k.)
  part[0] = rising(xbits >> 16 | 0xffff0000u);
  each_held(reg, s, [&](int j, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) pair[j / 2] = __builtin_elementwise_max(pair[j / 2], rising(v[q]));
    if (j % 2) part[j / 2 % 4] = __builtin_elementwise_max(part[j / 2 % 4], pair[j / 2]);
  });
  int best = -0x8000;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int x = part[i / 2][i % 2];
    best = max(best, x);
    key[i] = static_cast<uint32_t>(x + 0x8000);
  }
  return row_maximum(best, wave, lane, sm, odd);
}

// A bound that the k-th largest of the parts' maxima is not below, k <= N * NT: a
// search in the 4096 keys from the row's own down (32 octaves), a quarter of what is
// left a round (first 64, 256 and 1024 keys, where most rows' end); the lowest
// float if it is not among them.  A lane's counts of three thresholds add up in 10 bits
// each.  (A search by each wave for its share of k takes no barriers, but lets in twice
// the candidates: 4 rows of 151936, 17.4 -> 19.0 us.)
template <int N>
__device__ inline float kth_bound(const uint32_t (&key)[N], uint32_t top_key, uint32_t k, int wave, int lane, Small& sm) {
  static_assert(N * 64 < 1024, "counts of a wave in 10 bits");
  const uint32_t base = top_key > 4095 ? top_key - 4095 : 0;
  uint32_t lo = base, width = 4096;
  for (int round = 0; width > 1; ++round) {
    const uint32_t step = width / 4;
    const uint32_t t1 = round ? lo + step : base + 3072, t2 = round ? lo + 2 * step : base + 3840, t3 = round ? lo + 3 * step : base + 4032;
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += (key[i] >= t1 ? 1u : 0u) + (key[i] >= t2 ? 1u << 10 : 0u) + (key[i] >= t3 ? 1u << 20 : 0u);
    n = count_scan(n);
    if (lane == 63) sm.tally[round & 1][wave] = n;
    __syncthreads();                             // (the other buffer's readers are past it, too)
    uint32_t n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const uint32_t t = sm.tally[round & 1][w];
      n1 += t & 1023u;
      n2 += t >> 10 & 1023u;
      n3 += t >> 20;
    }
    if (round) {
      lo = n3 >= k ? t3 : n2 >= k ? t2 : n1 >= k ? t1 : lo;
      width = step;
    } else if (n1 >= k) {                        // (else all 4096 keys are left)
      lo = n3 >= k ? t3 : n2 >= k ? t2 : t1;
      width = n3 >= k ? 64 : n2 >= k ? 256 : 1024;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    width = __builtin_amdgcn_readfirstlane(width);
  }
  return lo == base || lo <= kNoKey ? -__FLT_MAX__ : ordered_float(lo << 16);
}

// Whether a bound worth the look at the parts' maxima is there.
__device__ inline bool bound_by_min(const Params& p) { return p.min_p > 0.0 && !(p.top_p < 1.0); }
__device__ inline bool bound_by_k(const Params& p) { return p.top_k && p.top_k <= kCap / 2; }
__device__ inline bool may_be_short(const Params& p, int V) {
  return p.greedy || bound_by_min(p) || bound_by_k(p) || V <= kCap || p.T < 0.05;
}

// Draws the row's token from the sorted list and writes it; false if there are too
// many candidates (nothing is written then).  N: parts of a lane.
template <bool BF16, bool REG, int N>
__device__ inline __attribute__((always_inline)) bool sample_short(
    const SampleArgs& a, int r, const u32x4 (&reg)[REG ? kRegs : 1], const Segment& s, uint32_t xbits, const Params& p,
    float u, float top, const uint32_t (&key)[N], const s16x2 (&pair)[REG ? kPairs : 1], int wave, int lane, Small& sm, List& list) {
  constexpr int VEC = BF16 ? 8 : 4;
  const int tid = threadIdx.x;
  const double m = static_cast<double>(top);
  // The bound, a little lower than it is (weights and cuts are looked at exactly
  // later on).
  auto below = [](double x) { return static_cast<float>(x - fabs(x) * 1e-6); };
  const bool by_min = bound_by_min(p), by_k = bound_by_k(p);
  if (!may_be_short(p, a.V)) return false;
  float bound = top;
  if (!p.greedy && top < __builtin_huge_valf()) {
    bound = fmaxf(below(m - kCut * p.T), -__FLT_MAX__);
    if (by_min) bound = fmaxf(bound, below(m + p.T * log(fmin(p.min_p, 1.0)) - 1e-6 * p.T));
    if (by_k) bound = fmaxf(bound, kth_bound(key, ordered(__float_as_uint(top)) >> 16, p.top_k, wave, lane, sm));
    bound = fminf(bound, top);
  }
  if (tid == 0) sm.listed = 0;
  __syncthreads();
  auto takes = [&](uint32_t bits) { return __uint_as_float(bits) >= bound; };   // (false for NaN)
  // Room for `own` entries of this lane, at the returned place.  (A place taken by
  // each lane from the counter, and its entries listed where they are found: 13 -> 17
  // thousand cycles for 60 candidates.)
  auto room = [&](uint32_t own) __attribute__((always_inline)) {
    const uint32_t incl = count_scan(own), total = last_lane(incl);
    uint32_t at = 0;
    if (total && lane == 0) at = atomicAdd(&sm.listed, total);
    return __builtin_amdgcn_readfirstlane(at) + incl - own;
  };
  auto put = [&](uint32_t at, int index) {
    if (at < kCap) list.index[at] = static_cast<uint32_t>(index);
  };
  auto mask_of = [&](const u32x4& v) __attribute__((always_inline)) {
    uint32_t b = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) b |= takes(entry<BF16>(v, e)) ? 1u << e : 0u;
    return b;
  };
  const bool extra = takes(xbits);
  if constexpr (REG) {
    // The masks of the wave's vectors with candidates, one after the other in LDS;
    // then their indices.  (One key lower than the bound's: -0 is not below 0.)
    const int low = static_cast<int>(ordered(__float_as_uint(bound)) >> 16) - 0x8000 - 2;
    const int16_t under = static_cast<int16_t>(max(low, -0x8000));
    const s16x2 none = {under, under};
    uint64_t hits = 0;
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const uint32_t over = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(pair[i], none));
      if (!__ballot(over != __builtin_bit_cast(uint32_t, none))) continue;
#pragma unroll
      for (int j = 2 * i; j < 2 * i + 2; ++j) {
        const uint32_t b = mask_of(reg[j]);
        if (!__ballot(b != 0)) continue;
        list.mask[wave][n++][lane] = static_cast<uint8_t>(b);
        hits |= uint64_t{1} << j;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    uint32_t own = extra ? 1 : 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) own += __popc(list.mask[wave][i][lane]);
    uint32_t at = room(own);
    if (extra) put(at++, s.extra);
#pragma unroll 4
    for (int i = 0; i < n; ++i, hits &= hits - 1) {
      const int index = s.head + (s.first + __builtin_ctzll(hits) * 64 + lane) * VEC;
      for (uint32_t b = list.mask[wave][i][lane]; b; b &= b - 1) put(at++, index + __builtin_ctz(b));
    }
  } else {
    const uint32_t first = room(extra ? 1 : 0);
    if (extra) put(first, s.extra);
    visit_batches<false>(s, 0, lane, [&](const int (&j)[kBatch], const u32x4 (&v)[kBatch]) __attribute__((always_inline)) {
      uint32_t b = 0;                            // which entries of the batch
#pragma unroll
      for (int i = 0; i < kBatch; ++i) b |= mask_of(v[i]) << (i * VEC);
      if (!__ballot(b != 0)) return;
      uint32_t at = room(__popc(b));
      for (; b; b &= b - 1) {
        const int i = __builtin_ctz(b);
        put(at++, s.head + (s.first + (j[0] + i / VEC) * 64 + lane) * VEC + i % VEC);
      }
    });
  }
  __syncthreads();
  const int n = static_cast<int>(__builtin_amdgcn_readfirstlane(sm.listed));
  if (n > kCap) return false;
  const char* row = reinterpret_cast<const char*>(s.base) - s.head * (16 / VEC);   // entry 0
  for (int i = tid; i < n; i += NT) {
    const uint32_t index = list.index[i];
    const uint32_t bits = BF16 ? static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[index]) << 16
                               : reinterpret_cast<const uint32_t*>(row)[index];
    list.key[i] = static_cast<uint64_t>(~ordered(bits)) << 32 | index;
  }
  __syncthreads();

  // In order: by rank where each thread has one candidate, else in pairs.
  const uint64_t* sorted = list.key;
  if (n <= NT) {
    const uint64_t mine = tid < n ? list.key[tid] : 0;
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += list.key[i] < mine ? 1 : 0;
    if (tid < n) list.sorted[rank] = mine;
    sorted = list.sorted;
    __syncthreads();
  } else {
    int size = 2 * NT;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) list.key[i] = ~uint64_t{0};
    for (int k = 2; k <= size; k *= 2)
      for (int d = k / 2; d >= 1; d /= 2) {
        __syncthreads();
        for (int t = tid; t < size / 2; t += NT) {
          const int i = (t & ~(d - 1)) * 2 + (t & (d - 1)), j = i + d;
          const uint64_t x = list.key[i], y = list.key[j];
          if ((x > y) == ((i & k) == 0)) {
            list.key[i] = y;
            list.key[j] = x;
          }
        }
      }
    __syncthreads();
  }

  if (p.greedy) {
    if (tid == 0) {
      a.token[r] = static_cast<int32_t>(sorted[0]);
      if (a.prob) a.prob[r] = 1.f;
      if (a.kept) a.kept[r] = 1;
    }
    return true;
  }
  // Thread t holds the candidates from t * per on.
  const int per = (n + NT - 1) / NT, first = tid * per;
  auto gap_at = [&](int i) {
    const float x = ordered_float(~static_cast<uint32_t>(sorted[i] >> 32));
    return x == top ? 0.0 : static_cast<double>(x) - m;
  };
  auto fixed_at = [&](int i, double* w) {        // 0 past the end and for what is never kept
    *w = -1.0;
    if (i >= n) return uint64_t{0};
    const double gap = gap_at(i);
    if (!(gap >= -kCut * p.T)) return uint64_t{0};
    *w = weight(gap, p);
    return static_cast<uint64_t>(rint(*w * a.one));
  };
  Sum mine = {0, 0}, by_min_mine = {0, 0}, all;
  for (int e = 0; e < per; ++e) {
    double w;
    const uint64_t z = fixed_at(first + e, &w);
    if (w >= 0.0) mine = Sum{mine.n + 1, mine.z + z};
    if (w >= fmin(p.min_p, 1.0)) by_min_mine = Sum{by_min_mine.n + 1, by_min_mine.z + z};
  }
  const Sum incl = block_scan(mine, wave, lane, sm.wave, &all);
  const Sum excl = {incl.n - mine.n, incl.z - mine.z};
  Sum by_min_all = all;
  if (p.min_p > 0.0) block_scan(by_min_mine, wave, lane, sm.wave, &by_min_all);
  auto find = [&](Kind kind, uint64_t target) __attribute__((always_inline)) {
    if (reached(kind, incl, target) && !reached(kind, excl, target)) {
      Sum before = excl;
      for (int e = 0; e < per; ++e) {
        double w;
        const uint64_t z = fixed_at(first + e, &w);
        const Sum next = {before.n + 1, before.z + z};
        if (reached(kind, next, target)) {
          sm.found = Found{static_cast<uint32_t>(first + e), before.n, 1, before.z, z};
          break;
        }
        before = next;
      }
    }
    __syncthreads();
    const Found f = sm.found;
    __syncthreads();
    return f;
  };
  uint32_t rank;
  Sum kept;
  const Found f = cut_and_draw(p, all, by_min_all, u, &rank, &kept, find);
  if (tid == 0) {
    a.token[r] = static_cast<int32_t>(sorted[f.key]);
    if (a.prob) a.prob[r] = static_cast<float>(weight(gap_at(f.key), p) * a.one / static_cast<double>(kept.z));
    if (a.kept) a.kept[r] = static_cast<int32_t>(kept.n);
  }
  return true;
}

// ----------------------------------------------------------------------------
// bf16
// ----------------------------------------------------------------------------
// Place of a bit pattern in the falling order: positive ones from the largest
// (+0 last), then negative ones from -0 on.  -0 counts as +0.
constexpr uint32_t kInfPlace = 0x7f, kZeroPlace = 0x7fff, kEndPlace = 0xff80;   // +inf; +0; -inf
constexpr int kMinusZero = 0x8000, kMinusInf = 0xff80;   // their patterns
__device__ inline uint32_t place_bits(uint32_t o) { return o < 0x8000u ? 0x7fffu - o : o; }
__device__ inline uint32_t place_of(uint32_t bits) { return bits < 0x8000u ? 0x7fffu - bits : bits; }
__device__ inline double place_value(uint32_t o) { return static_cast<double>(__uint_as_float(place_bits(o) << 16)); }

constexpr int kSteps = 512;      // 128 places each
constexpr int kWraps = 256;      // notes of wraps at most: 2^22 entries wrap 64 counters, with up to 3 notes each

struct Bf16Shared {
  union {
    uint32_t hist[32768];        // counts of patterns 2i (low half) and 2i + 1 (high half)
    List list;
  };
  uint32_t n[kSteps];            // tokens of the steps above (exclusive), after the scan
  uint64_t z[kSteps];
  Small small;
  uint64_t live[NW];             // steps with any count
  uint32_t total, wraps, step;
  uint8_t any[kSteps];
  int32_t wrap[kWraps];          // pattern whose count grew by 65536, or ~pattern: by one too many
};

template <bool REG>
__global__ void __launch_bounds__(NT) sample_bf16_kernel(SampleArgs a) {
  __shared__ Bf16Shared sh;
  const int r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const void* row = static_cast<const uint16_t*>(a.logits) + static_cast<int64_t>(r) * a.V;
  const Segment s = segment_of<true>(row, a.V, wave, lane);
  u32x4 reg[REG ? kRegs : 1];
  if constexpr (REG) load_row(reg, s, lane);
  uint32_t xbits = kNone;                        // this lane's entry outside the vectors, as fp32
  if (s.extra >= 0) xbits = static_cast<uint32_t>(static_cast<const uint16_t*>(row)[s.extra]) << 16;
  const Params p = params_of(a, r);
  const float u = a.uniforms[r];
  // The short way, where there may be one; other rows in registers are counted as
  // their loads arrive (512 rows with settings of all kinds: 94 -> 90 us).
  float best = -__builtin_huge_valf();
  const bool may = !REG || may_be_short(p, a.V);
  if (may) {
    if constexpr (REG) {
      uint32_t key[8];
      s16x2 pair[kPairs];
      bool odd;
      best = part_maxima_held(reg, s, xbits, wave, lane, sh.small, key, pair, &odd);
      if (odd) {                                 // (the pairs' maxima let every vector in that holds a NaN)
        uint32_t key4[4];
        best = part_maxima_read<true>(s, xbits, wave, lane, sh.small, key4);
#pragma unroll
        for (int i = 0; i < 8; ++i) key[i] = i < 4 ? key4[i] : kNoKey;
      }
      if (best > -__builtin_huge_valf() &&
          sample_short<true, true>(a, r, reg, s, xbits, p, u, best, key, pair, wave, lane, sh.small, sh.list))
        return;
    } else {
      uint32_t key[4];
      const s16x2 pair[1] = {};
      best = part_maxima_read<true>(s, xbits, wave, lane, sh.small, key);
      if (best > -__builtin_huge_valf() &&
          sample_short<true, false>(a, r, reg, s, xbits, p, u, best, key, pair, wave, lane, sh.small, sh.list))
        return;
    }
    if (best == -__builtin_huge_valf()) {
      write_none(a, r);
      return;
    }
    __syncthreads();                             // the list's LDS becomes the histogram's
  }

  // NaN of negative sign counts as -inf: neither is ever kept.
  auto counted = [](uint32_t w) __attribute__((always_inline)) {
    const u16x2 least = {kMinusInf, kMinusInf};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, w), least));
  };
  // One count of a pattern; NOTE: a counter that wraps is noted.
  auto add = [&](uint32_t twice, uint32_t one, auto note) __attribute__((always_inline)) {
    // twice: byte offset of the pattern's word; one: 1 in its half
    uint32_t* w = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(sh.hist) + twice);
    if constexpr (decltype(note)::value) {
      const uint32_t old = atomicAdd(w, one);
      const uint32_t even = twice >> 1;
      if (one == 1u && (old & 0xffffu) == 0xffffu) {
        // The carry went into the odd pattern's counter, and may wrap it too.
        const int i = atomicAdd(&sh.wraps, 2u);
        sh.wrap[i] = static_cast<int32_t>(even);
        sh.wrap[i + 1] = ~static_cast<int32_t>(even + 1);
        if (old == 0xffffffffu) sh.wrap[atomicAdd(&sh.wraps, 1u)] = static_cast<int32_t>(even + 1);
      } else if (one != 1u && (old >> 16) == 0xffffu) {
        sh.wrap[atomicAdd(&sh.wraps, 1u)] = static_cast<int32_t>(even + 1);
      }
    } else {
      atomicAdd(w, one);
    }
  };
  s16x2 most = {-0x8000, -0x8000};               // of this lane's entries in registers
  auto build = [&](auto note) __attribute__((always_inline)) {
    u32x4* h = reinterpret_cast<u32x4*>(sh.hist);
    for (int i = tid; i < 32768 / 4; i += NT) h[i] = u32x4{0, 0, 0, 0};
    if (tid == 0) {
      sh.total = 0;
      sh.wraps = 0;
    }
    __syncthreads();
    auto add_all = [&](int, const u32x4& v) __attribute__((always_inline)) {
      if ((v[0] & v[1] & v[2] & v[3]) != kNone) {   // (all NaN, or past the end)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t w = counted(v[q]);
          add((w << 1) & 0x1fffcu, 1u << ((w << 4) & 16u), note);
          add((w >> 15) & 0x1fffcu, 1u << ((w >> 12) & 16u), note);
        }
      }
    };
    if constexpr (REG && !decltype(note)::value)
      each_held(reg, s, [&](int j, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) most = __builtin_elementwise_max(most, rising(v[q]));
        add_all(j, v);
      });
    else visit<false>(s, 0, lane, add_all);
    if (s.extra >= 0) {
      const uint32_t w = counted(xbits);
      add((w >> 15) & 0x1fffcu, 1u << ((w >> 12) & 16u), note);
    }
    __syncthreads();
    // The sum of all counts, and which steps have any (a wave reads the words of
    // one step at a time).  (The odd pattern beside -inf, a NaN, is counted as -inf:
    // their word is one number, so masking with -inf wraps nothing.  Every count that
    // wraps lowers the sum and nothing raises it, so it is V only if none did.)
    uint32_t sum = 0;
#pragma unroll 8
    for (int i = 0; i < 32768 / NT; ++i) {
      const int at = i * NT + tid;
      const uint32_t w = sh.hist[at];
      sum += at == kEndPlace / 2 ? w : (w & 0xffffu) + (w >> 16);
      const int group = i * NW + wave;
      const bool live = __ballot(w != 0) != 0;
      if (lane == 0) sh.any[group < kSteps / 2 ? kSteps / 2 - 1 - group : group] = live;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) atomicAdd(&sh.total, sum);
    // -0 counts in +0's place, whose step is live with it.  (Thread 0 wrote that flag.)
    if (tid == 0 && (sh.hist[kMinusZero / 2] & 0xffffu)) sh.any[kZeroPlace / 128] = 1;
    __syncthreads();
    if constexpr (decltype(note)::value) {       // counts of 65536 read 0
      for (uint32_t i = tid; i < sh.wraps; i += NT)
        if (sh.wrap[i] >= 0) sh.any[sh.wrap[i] == kMinusZero ? kZeroPlace / 128 : place_of(sh.wrap[i]) / 128] = 1;
      __syncthreads();
    }
  };
  build(std::false_type{});
  if (sh.total != static_cast<uint32_t>(a.V)) {
    __syncthreads();
    build(std::true_type{});
  }
  if (!may) {
    most = __builtin_elementwise_max(most, rising(xbits >> 16 | xbits));
    bool odd;
    best = row_maximum(max(most[0], most[1]), wave, lane, sh.small, &odd);
    if (odd) {
      uint32_t key[4];
      best = part_maxima_read<true>(s, xbits, wave, lane, sh.small, key);
    }
    if (best == -__builtin_huge_valf()) {
      write_none(a, r);
      return;
    }
  }
  // The largest entry's place (-0 is +0).
  const uint32_t top = best == 0.f ? kZeroPlace : place_of(__float_as_uint(best) >> 16);
  const double m = place_value(top);
  const double scale = a.one;
  // Counts of the places 128 * step + 2 * lane and the next.
  auto counts = [&](uint32_t step, uint32_t (&c)[2]) __attribute__((always_inline)) {
    const uint32_t o = step * 128 + 2 * lane;
    const uint32_t w = sh.hist[place_bits(o) >> 1];
    c[0] = o < 0x8000u ? w >> 16 : w & 0xffffu;
    c[1] = o < 0x8000u ? w & 0xffffu : w >> 16;
    if (sh.wraps) {
      for (uint32_t i = 0; i < sh.wraps; ++i) {
        const int32_t k = sh.wrap[i];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (k == static_cast<int32_t>(place_bits(o + h))) c[h] += 65536;
          if (k == ~static_cast<int32_t>(place_bits(o + h))) c[h] -= 1;
        }
      }
    }
    if (o + 1 == kZeroPlace) {                   // -0 joins +0
      c[1] += sh.hist[kMinusZero / 2] & 0xffffu;
      for (uint32_t i = 0; i < sh.wraps; ++i) c[1] += sh.wrap[i] == kMinusZero ? 65536 : 0;
    }
    if (o == kZeroPlace + 1) c[0] = 0;
    if (o < kInfPlace) c[0] = 0;
    if (o + 1 < kInfPlace) c[1] = 0;
    if (o >= kEndPlace) c[0] = c[1] = 0;
  };
  // Count and weight of one place (0, 0 where it is too far below the top).
  // (Without a branch: the two places of a lane run side by side.)
  auto place_sum = [&](uint32_t o, uint32_t c, uint64_t* w) __attribute__((always_inline)) {
    const double gap = o == top ? 0.0 : place_value(o) - m;
    const bool in = c != 0 && gap >= -kCut * p.T;
    const double x = rint(weight(in ? gap : 0.0, p) * scale);
    *w = in ? static_cast<uint64_t>(x) : 0;
    return Sum{in ? c : 0, c * *w};
  };

  uint32_t place = top, rank = 0, kept = 1;
  float prob = 1.f;
  if (!p.greedy) {
    // Sums of the steps that have any count, dealt to the waves in turn (a row's
    // values lie close together in the order).
    sh.n[tid] = 0;
    sh.z[tid] = 0;
    const uint64_t live = __ballot(sh.any[tid] != 0);
    if (lane == 0) sh.live[wave] = live;
    __syncthreads();
    int turn = 0;
    for (int q = 0; q < NW; ++q) {
      uint64_t left = sh.live[q];
      left = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(left >> 32))) << 32 |
             static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(left)));
      for (; left; left &= left - 1) {
        if ((turn++ & (NW - 1)) != wave) continue;
        const uint32_t step = q * 64 + __builtin_ctzll(left);
        uint32_t c[2];
        counts(step, c);
        uint64_t w;
        Sum v = place_sum(step * 128 + 2 * lane, c[0], &w);
        const Sum v1 = place_sum(step * 128 + 2 * lane + 1, c[1], &w);
        v.n += v1.n;
        v.z += v1.z;
        v = wave_scan(v);
        if (lane == 63) {
          sh.n[step] = v.n;
          sh.z[step] = v.z;
        }
      }
    }
    __syncthreads();
    Sum mine = {0, 0}, all;
    mine = Sum{sh.n[tid], sh.z[tid]};
    static_assert(kSteps == NT, "one step a thread");
    const Sum incl = block_scan(mine, wave, lane, sh.small.wave, &all);
    const Sum excl = {incl.n - mine.n, incl.z - mine.z};
    sh.n[tid] = excl.n;
    sh.z[tid] = excl.z;
    __syncthreads();

    // Each wave looks at the step itself, so that all of them know the answer.
    auto in_step = [&](uint32_t step, Sum (&v)[2], uint64_t (&w)[2], uint32_t (&c)[2]) __attribute__((always_inline)) {
      counts(step, c);
      v[0] = place_sum(step * 128 + 2 * lane, c[0], &w[0]);
      v[1] = place_sum(step * 128 + 2 * lane + 1, c[1], &w[1]);
      const Sum own = {v[0].n + v[1].n, v[0].z + v[1].z};
      Sum sc = wave_scan(own);
      c[0] = v[0].n;
      c[1] = v[1].n;
      v[0] = Sum{sh.n[step] + sc.n - own.n, sh.z[step] + sc.z - own.z};   // before the first
      v[1] = Sum{v[0].n + c[0], v[0].z + c[0] * w[0]};                    // before the second
    };
    auto find = [&](Kind kind, uint64_t target) __attribute__((always_inline)) {
      if (reached(kind, incl, target) && !reached(kind, excl, target)) sh.step = tid;
      __syncthreads();
      const uint32_t step = __builtin_amdgcn_readfirstlane(sh.step);
      __syncthreads();
      Sum v[2];
      uint64_t w[2];
      uint32_t c[2];
      in_step(step, v, w, c);
      const Sum end = {v[1].n + c[1], v[1].z + c[1] * w[1]};
      const int h = reached(kind, v[1], target) ? 0 : 1;
      const int l = __builtin_ctzll(__ballot(reached(kind, end, target)));
      Found f;
      f.key = step * 128 + 2 * l + __builtin_amdgcn_readlane(h, l);
      f.n_before = __builtin_amdgcn_readlane(h ? v[1].n : v[0].n, l);
      f.n = __builtin_amdgcn_readlane(h ? c[1] : c[0], l);
      f.z_before = lane64(h ? v[1].z : v[0].z, l);
      f.w = lane64(h ? w[1] : w[0], l);
      return f;
    };
    Sum by_min = all;
    if (p.min_p > 0.0) {
      // The last place whose weight is not less: 64 places a round.
      uint32_t lo = top;
      for (int shift = 10; shift >= 0; shift -= 5) {
        const uint32_t o = min(lo + (static_cast<uint32_t>(lane) << shift), kEndPlace - 1);
        const double gap = o == top ? 0.0 : place_value(o) - m;
        const uint64_t b = __ballot(weight(gap, p) >= fmin(p.min_p, 1.0));
        lo = __builtin_amdgcn_readlane(o, 63 - __builtin_clzll(b));
      }
      Sum v[2];
      uint64_t w[2];
      uint32_t c[2];
      in_step(lo / 128, v, w, c);
      const int l = (lo % 128) / 2;
      Sum e = v[1];
      if (lo & 1) e = Sum{v[1].n + c[1], v[1].z + c[1] * w[1]};
      by_min = Sum{static_cast<uint32_t>(__builtin_amdgcn_readlane(e.n, l)), lane64(e.z, l)};
    }
    Sum part;
    const Found f = cut_and_draw(p, all, by_min, u, &rank, &part, find);
    place = f.key;
    kept = part.n;
    const double gap = place == top ? 0.0 : place_value(place) - m;
    prob = static_cast<float>(weight(gap, p) * scale / static_cast<double>(part.z));
  }

  // The rank-th entry with the drawn value, in vocabulary order.
  const uint32_t bits = place_bits(place), two = bits | bits << 16;
  const uint32_t mask = bits == 0 ? 0x7fff7fffu : 0xffffffffu;
  uint64_t hits = 0;                             // vectors that hold it
  if constexpr (REG)
    each_held(reg, s, [&](int j, const u32x4& v) __attribute__((always_inline)) {
      u16x2 x = {1, 1};                          // 0 in a half where an entry is equal
#pragma unroll
      for (int q = 0; q < 4; ++q) x = __builtin_elementwise_min(x, __builtin_bit_cast(u16x2, (v[q] ^ two) & mask));
      if (__ballot(x[0] == 0 || x[1] == 0)) hits |= uint64_t{1} << j;
    });
  auto equal = [&](const u32x4& v) __attribute__((always_inline)) {
    uint32_t b = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t x = (v[q] ^ two) & mask;
      b |= ((x & 0xffffu) == 0 ? 1u : 0u) << 2 * q | ((x >> 16) == 0 ? 2u : 0u) << 2 * q;
    }
    return b;
  };
  const bool extra_match = s.extra >= 0 && ((xbits >> 16 ^ bits) & mask & 0xffffu) == 0;
  find_and_write<8, REG>(a, r, s, hits, rank, prob, kept, wave, lane, sh.small.count, extra_match, equal);
}

// ----------------------------------------------------------------------------
// fp32
// ----------------------------------------------------------------------------
__device__ inline double ordered_value(uint32_t k) { return static_cast<double>(ordered_float(k)); }

constexpr int kBins = 8192, kMid = 1024;   // upper 13 bits; next 10 (and the last 9)
static_assert(kMid == 2 * NT, "two or one bins of the lower levels a thread");

struct F32Shared {
  union {
    struct {
      uint64_t z[kBins];
      uint32_t n[kBins];
      uint64_t z2[kMid];
      uint32_t n2[kMid];
    };
    List list;
  };
  Small small;
};

__global__ void __launch_bounds__(NT) sample_f32_kernel(SampleArgs a) {
  __shared__ F32Shared sh;
  const int r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const void* row = static_cast<const float*>(a.logits) + static_cast<int64_t>(r) * a.V;
  const Segment s = segment_of<false>(row, a.V, wave, lane);
  uint32_t xbits = kNone;
  if (s.extra >= 0) xbits = static_cast<const uint32_t*>(row)[s.extra];
  const Params p = params_of(a, r);
  const float u = a.uniforms[r];
  const u32x4 none[1] = {};                      // (the row is not kept in registers)
  uint32_t part[4];
  const s16x2 pair[1] = {};
  const float best = part_maxima_read<false>(s, xbits, wave, lane, sh.small, part);
  if (best == -__builtin_huge_valf()) {
    write_none(a, r);
    return;
  }
  if (sample_short<false, false>(a, r, none, s, xbits, p, u, best, part, pair, wave, lane, sh.small, sh.list)) return;
  __syncthreads();                               // the list's LDS becomes the bins'
  for (int i = tid; i < kBins; i += NT) {
    sh.z[i] = 0;
    sh.n[i] = 0;
  }
  __syncthreads();

  auto each = [&](auto f) __attribute__((always_inline)) {   // f(bits) of every entry (NaN past the end)
    visit<false>(s, 0, lane, [&](int, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f(v[q]);
        __builtin_amdgcn_sched_barrier(0);       // (exps side by side take more registers than there are)
      }
    });
    f(xbits);
  };
  const double m = static_cast<double>(best), scale = a.one;
  const uint32_t top = ordered(__float_as_uint(best));

  // The weight of a pattern, and whether it can be kept at all.
  auto gap_of = [&](uint32_t b) __attribute__((always_inline)) {
    return __uint_as_float(b) == best ? 0.0 : static_cast<double>(__uint_as_float(b)) - m;
  };
  auto fixed = [&](double gap) { return static_cast<uint64_t>(rint(weight(gap, p) * scale)); };
  const double least_gap = -kCut * p.T;

  uint32_t key = top, rank = 0, kept = 1;
  float prob = 1.f;
  if (!p.greedy) {
    each([&](uint32_t b) __attribute__((always_inline)) {
      const double gap = gap_of(b);
      if (gap >= least_gap) {                    // (false for NaN)
        const uint32_t bin = ordered(b) >> 19;
        atomicAdd(&sh.n[bin], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.z[bin]), static_cast<unsigned long long>(fixed(gap)));
      }
    });
    __syncthreads();
    // Thread t holds the bins 8191 - 16 t .. 8176 - 16 t, from the top.
    constexpr int PER = kBins / NT;
    Sum mine = {0, 0}, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      mine.n += sh.n[kBins - 1 - tid * PER - i];
      mine.z += sh.z[kBins - 1 - tid * PER - i];
    }
    const Sum incl = block_scan(mine, wave, lane, sh.small.wave, &all);
    const Sum excl = {incl.n - mine.n, incl.z - mine.z};

    // The pattern at which the running sums reach the target: its bin (the
    // thread that holds it looks), then the next bits within it, twice.
    auto find = [&](Kind kind, uint64_t target) __attribute__((always_inline)) {
      if (reached(kind, incl, target) && !reached(kind, excl, target)) {
        Sum at = excl;
        for (int i = 0; i < PER; ++i) {
          const int bin = kBins - 1 - tid * PER - i;
          const Sum next = {at.n + sh.n[bin], at.z + sh.z[bin]};
          if (reached(kind, next, target)) {
            sh.small.found = Found{static_cast<uint32_t>(bin), at.n, 0, at.z, 0};
            break;
          }
          at = next;
        }
      }
      __syncthreads();
      Found f = sh.small.found;
      for (int level = 0; level < 2; ++level) {
        const int bits = level ? 9 : 10, shift = level ? 0 : 9, width = 1 << bits;
        for (int i = tid; i < kMid; i += NT) {
          sh.n2[i] = 0;
          sh.z2[i] = 0;
        }
        __syncthreads();
        each([&](uint32_t b) __attribute__((always_inline)) {
          const uint32_t k = ordered(b);
          if (k >> (shift + bits) == f.key) {
            const double gap = gap_of(b);
            if (gap >= least_gap) {
              const uint32_t bin = (k >> shift) & (width - 1);
              atomicAdd(&sh.n2[bin], 1u);
              atomicAdd(reinterpret_cast<unsigned long long*>(&sh.z2[bin]), static_cast<unsigned long long>(fixed(gap)));
            }
          }
        });
        __syncthreads();
        // Thread t holds two bins (the upper bits) or one, from the top.
        Sum v[2] = {}, t;
        const int per = width / NT;
        for (int i = 0; i < 2; ++i)
          if (i < per) v[i] = Sum{sh.n2[width - 1 - tid * per - i], sh.z2[width - 1 - tid * per - i]};
        Sum in = block_scan(Sum{v[0].n + v[1].n, v[0].z + v[1].z}, wave, lane, sh.small.wave, &t);
        in.n += f.n_before;
        in.z += f.z_before;
        const Sum mid = {in.n - v[1].n, in.z - v[1].z}, ex = {mid.n - v[0].n, mid.z - v[0].z};
        if (reached(kind, in, target) && !reached(kind, ex, target)) {
          const int i = reached(kind, mid, target) ? 0 : 1;
          const Sum before = i ? mid : ex;
          sh.small.found = Found{f.key << bits | static_cast<uint32_t>(width - 1 - tid * per - i), before.n, v[i].n, before.z, v[i].z};
        }
        __syncthreads();
        f = sh.small.found;
      }
      __syncthreads();
      f.w = f.w / f.n;                           // equal patterns weigh the same
      return f;
    };
    Sum by_min = all;
    if (p.min_p > 0.0) {
      // The lowest pattern whose weight is not less: 64 patterns a round.
      const double least = fmin(p.min_p, 1.0);
      uint32_t hi = top;
      for (int shift = 26; shift >= 0; shift = shift > 2 ? shift - 6 : shift - 2) {
        const uint32_t d = static_cast<uint32_t>(lane) << shift;
        const uint32_t k = hi > d ? hi - d : 0u;
        const double gap = k == top ? 0.0 : ordered_value(k) - m;
        const uint64_t b = __ballot(weight(gap, p) >= least);   // (a NaN's pattern: false)
        hi = __builtin_amdgcn_readlane(k, 63 - __builtin_clzll(b));
      }
      // What the bins above its own hold, and its bin's share.
      const uint32_t bin = hi >> 19;
      Sum v = {0, 0};
      each([&](uint32_t b) __attribute__((always_inline)) {
        const uint32_t k = ordered(b);
        if (k >> 19 == bin && k >= hi) {
          const double gap = gap_of(b);
          if (gap >= least_gap) {
            v.n += 1;
            v.z += fixed(gap);
          }
        }
      });
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t q = kBins - 1 - tid * PER - i;
        if (q > bin) {
          v.n += sh.n[q];
          v.z += sh.z[q];
        }
      }
      block_scan(v, wave, lane, sh.small.wave, &by_min);
    }
    Sum part;
    const Found f = cut_and_draw(p, all, by_min, u, &rank, &part, find);
    key = f.key;
    kept = part.n;
    const double gap = key == top ? 0.0 : ordered_value(key) - m;
    prob = static_cast<float>(weight(gap, p) * scale / static_cast<double>(part.z));
  }

  const bool extra_match = s.extra >= 0 && ordered(xbits) == key;
  find_and_write<4, false>(a, r, s, 0, rank, prob, kept, wave, lane, sh.small.count, extra_match,
                           [&](const u32x4& v) __attribute__((always_inline)) {
                             uint32_t b = 0;
#pragma unroll
                             for (int e = 0; e < 4; ++e) b |= ordered(v[e]) == key ? 1u << e : 0u;
                             return b;
                           });
}

}  // namespace

hipError_t launch_sample(const simsd_sample_desc& d, const SampleArgs& a, hipStream_t st) {
  const dim3 grid(d.rows);
  if (d.dtype == SIMSD_F32) {
    hipLaunchKernelGGL(sample_f32_kernel, grid, dim3(NT), 0, st, a);
  } else {
    // Rows that fit the registers of a work-group: every wave's share of the
    // vectors, rounded up to whole loads.
    const int loads = ((a.V / 8 + NW - 1) / NW + 63) / 64;
    if (loads <= kRegs) hipLaunchKernelGGL((sample_bf16_kernel<true>), grid, dim3(NT), 0, st, a);
    else hipLaunchKernelGGL((sample_bf16_kernel<false>), grid, dim3(NT), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace simsd
