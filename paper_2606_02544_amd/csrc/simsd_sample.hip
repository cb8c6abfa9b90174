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
// row is read again), is read from memory once,
// and the weights are taken of the distinct values only (some 3000 of a row of
// 151936 logits N(0, 4)).  A counter that passes 65535 shows in the total and
// the histogram is built again, noting each wrap.
// fp32 rows: the weights are added up in 8192 bins of the upper 13 bits of the
// ordered bit pattern; a search goes on in the bin it ends in, 10 and then 9
// bits further, over the row again, which the caches hold by then.
#include <type_traits>

#include "simsd_ops_kernels.h"

namespace simsd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int NT = 512;          // threads of a work-group
constexpr int NW = NT / 64;
constexpr int kRegs = 38;        // 16-byte loads of a bf16 row that a lane keeps
constexpr double kCut = 700.0;   // a token further below the maximum, in temperatures, is never kept

struct Params {
  double T, top_p, min_p;
  uint32_t top_k;                // 0: off
  bool greedy;
};

// A logits value's place in the running sums.
struct Found {
  uint32_t key;                  // its key (bf16: place in the falling order; fp32: ordered pattern)
  uint32_t n_before, n;          // tokens above it, tokens equal to it
  uint64_t z_before, w;          // weight above it, weight of one such token
};

__device__ inline uint64_t shfl_up64(uint64_t v, int d) {
  const uint32_t lo = __shfl_up(static_cast<uint32_t>(v), d), hi = __shfl_up(static_cast<uint32_t>(v >> 32), d);
  return (static_cast<uint64_t>(hi) << 32) | lo;
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

__device__ inline Sum wave_scan(Sum v, int lane) {      // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t n = __shfl_up(v.n, d);
    const uint64_t z = shfl_up64(v.z, d);
    if (lane >= d) {
      v.n += n;
      v.z += z;
    }
  }
  return v;
}

__device__ inline double weight(double gap, double T) { return exp(gap / T); }

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

// f(j, vector) for this wave's vectors: from registers, or loaded.  Lanes past the
// end get the pattern of a NaN, which no filter keeps.
constexpr uint32_t kNone = 0xffffffffu;
template <bool REG, typename F>
__device__ inline __attribute__((always_inline)) void each_vector(const u32x4 (&reg)[kRegs], const Segment& s, int lane, F f) {
  if constexpr (REG) {
#pragma unroll
    for (int j = 0; j < kRegs; ++j)
      if (j * 64 < s.count) f(j, reg[j]);
  } else {
    for (int j = 0; j * 64 < s.count; ++j) {
      u32x4 v = {kNone, kNone, kNone, kNone};
      if (j * 64 + lane < s.count) v = s.base[s.first + j * 64 + lane];
      f(j, v);
    }
  }
}

template <bool REG>
__device__ inline __attribute__((always_inline)) void load_row(u32x4 (&reg)[kRegs], const Segment& s, int lane) {
  if constexpr (REG) {
#pragma unroll
    for (int j = 0; j < kRegs; ++j) {
      reg[j] = u32x4{kNone, kNone, kNone, kNone};
      if (j * 64 + lane < s.count) reg[j] = s.base[s.first + j * 64 + lane];
    }
  }
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
  p.top_k = k > 0 ? k : 0;
  return p;
}

// First token of the kept part's running sums past u * z.
__device__ inline uint64_t draw_target(float u, uint64_t z) {
  const double v = fmin(fmax(static_cast<double>(u), 0.0), 1.0);
  const uint64_t t = static_cast<uint64_t>(v * static_cast<double>(z));
  return t < z ? t : z - 1;
}

// The index of the rank-th entry (0-based, in vocabulary order) that `match`es,
// found by the wave that holds it, which writes the outputs.  `count` is this
// lane's number of matches.
template <bool BF16, bool REG, typename Match>
__device__ inline __attribute__((always_inline)) void find_and_write(
    const SampleArgs& a, int r, const u32x4 (&reg)[kRegs], const Segment& s, uint32_t count,
    uint32_t rank, float prob, uint32_t kept, int wave, int lane, uint32_t* s_count, bool extra_match, Match match) {
  constexpr int VEC = BF16 ? 8 : 4;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) count += __shfl_xor(count, d);
  if (lane == 0) s_count[wave] = count;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += s_count[w];
  if (rank < before || rank >= before + count) return;   // uniform: another wave's
  uint32_t left = rank - before;
  int found = -1;
  const uint64_t below = (uint64_t{1} << lane) - 1;
  auto take = [&](bool m, int index) {                   // one entry a lane, in lane order
    const uint64_t b = __ballot(m);
    const uint32_t n = __popcll(b);
    if (left < n && found < 0) {
      const bool mine = m && static_cast<uint32_t>(__popcll(b & below)) == left;
      const int l = __builtin_ctzll(__ballot(mine));
      found = __builtin_amdgcn_readlane(index, l);
    }
    left -= n;
  };
  if (wave == 0) take(extra_match && s.extra < s.head, s.extra);
  each_vector<REG>(reg, s, lane, [&](int j, const u32x4& v) __attribute__((always_inline)) {
    if (found >= 0) return;
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) bits |= match(v, e) ? 1u << e : 0u;
    if (!__ballot(bits != 0)) return;
    uint32_t incl = __popc(bits);
    const uint32_t own = incl;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    const uint32_t total = __builtin_amdgcn_readlane(incl, 63);
    if (left < total) {
      const uint32_t ex = incl - own;
      const bool mine = ex <= left && left < incl;
      int at = 0;
      uint32_t skip = left - ex, b = bits;
      if (mine) {
        while (skip--) b &= b - 1;
        at = __builtin_ctz(b);
      }
      const int index = s.head + (s.first + j * 64 + lane) * VEC + at;
      found = __builtin_amdgcn_readlane(index, __builtin_ctzll(__ballot(mine)));
    } else {
      left -= total;
    }
  });
  if (found < 0 && wave == NW - 1) take(extra_match && s.extra >= s.head, s.extra);
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
  v = wave_scan(v, lane);
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
// bf16
// ----------------------------------------------------------------------------
// Place of a bit pattern in the falling order: positive ones from the largest
// (+0 last), then negative ones from -0 on.  -0 counts as +0.
constexpr uint32_t kInfPlace = 0x7f, kZeroPlace = 0x7fff, kEndPlace = 0xff80;   // +inf; +0; -inf
__device__ inline uint32_t place_bits(uint32_t o) { return o < 0x8000u ? 0x7fffu - o : o; }
__device__ inline double place_value(uint32_t o) { return static_cast<double>(__uint_as_float(place_bits(o) << 16)); }

constexpr int kSteps = 512;      // 128 places each
constexpr int kWraps = 256;      // notes of wraps at most: 2^22 entries wrap 64 counters, with up to 3 notes each

struct Bf16Shared {
  uint32_t hist[32768];          // counts of patterns 2i (low half) and 2i + 1 (high half)
  uint32_t n[kSteps];            // tokens of the steps above (exclusive), after the scan
  uint64_t z[kSteps];
  Sum wave[NW];
  uint32_t count[NW];
  uint32_t top, total, wraps, step;
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
  u32x4 reg[kRegs];
  load_row<REG>(reg, s, lane);
  uint32_t xbits = kNone;                        // this lane's entry outside the vectors
  if (s.extra >= 0) xbits = static_cast<const uint16_t*>(row)[s.extra];
  const Params p = params_of(a, r);
  const float u = a.uniforms[r];

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
  auto build = [&](auto note) __attribute__((always_inline)) {
    u32x4* h = reinterpret_cast<u32x4*>(sh.hist);
    for (int i = tid; i < 32768 / 4; i += NT) h[i] = u32x4{0, 0, 0, 0};
    if (tid == 0) {
      sh.top = kEndPlace;
      sh.total = 0;
      sh.wraps = 0;
    }
    __syncthreads();
    each_vector<REG>(reg, s, lane, [&](int j, const u32x4& v) __attribute__((always_inline)) {
      if (j * 64 + lane < s.count) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          add((v[q] << 1) & 0x1fffcu, 1u << ((v[q] << 4) & 16u), note);
          add((v[q] >> 15) & 0x1fffcu, 1u << ((v[q] >> 12) & 16u), note);
        }
      }
    });
    if (s.extra >= 0) add((xbits << 1) & 0x1fffcu, 1u << ((xbits << 4) & 16u), note);
    __syncthreads();
    // The sum of all counts.  (-inf and the odd pattern beside it, a NaN, are
    // never kept: their word counts as one number, so masking with -inf wraps
    // nothing.)
    uint32_t sum = 0;
    for (int i = tid; i < 32768; i += NT) {
      const uint32_t w = sh.hist[i];
      sum += i == kEndPlace / 2 ? w : (w & 0xffffu) + (w >> 16);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) atomicAdd(&sh.total, sum);
    __syncthreads();
  };
  build(std::false_type{});
  if (sh.total != static_cast<uint32_t>(a.V)) {
    __syncthreads();
    build(std::true_type{});
  }
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
      c[1] += sh.hist[0x4000] & 0xffffu;
      for (uint32_t i = 0; i < sh.wraps; ++i) c[1] += sh.wrap[i] == 0x8000 ? 65536 : 0;
    }
    if (o == kZeroPlace + 1) c[0] = 0;
    if (o < kInfPlace) c[0] = 0;
    if (o + 1 < kInfPlace) c[1] = 0;
    if (o >= kEndPlace) c[0] = c[1] = 0;
  };
  uint32_t top = kEndPlace;                      // the row's largest entry
  for (uint32_t step = wave; step < kSteps && top == kEndPlace; step += NW) {
    uint32_t c[2];
    counts(step, c);
    const uint64_t b0 = __ballot(c[0] != 0), b1 = __ballot(c[1] != 0);
    if (b0 | b1) {
      const int l = __builtin_ctzll(b0 | b1);
      top = step * 128 + 2 * l + ((b0 >> l) & 1 ? 0 : 1);
    }
  }
  if (lane == 0) atomicMin(&sh.top, top);
  __syncthreads();
  top = __builtin_amdgcn_readfirstlane(sh.top);
  if (top == kEndPlace) {
    write_none(a, r);
    return;
  }
  const double m = place_value(top);
  const double scale = a.one;
  // Count and weight of one place (0, 0 where it is too far below the top).
  auto place_sum = [&](uint32_t o, uint32_t c, uint64_t* w) __attribute__((always_inline)) {
    Sum v = {0, 0};
    *w = 0;
    if (c) {
      const double gap = o == top ? 0.0 : place_value(o) - m;
      if (gap >= -kCut * p.T) {
        *w = static_cast<uint64_t>(rint(weight(gap, p.T) * scale));
        v.n = c;
        v.z = c * *w;
      }
    }
    return v;
  };

  uint32_t place = top, rank = 0, kept = 1;
  float prob = 1.f;
  if (!p.greedy) {
    // Sums of the steps, dealt to the waves in turn (a row's values lie close
    // together in the order).
    for (uint32_t step = wave; step < kSteps; step += NW) {
      uint32_t c[2];
      counts(step, c);
      Sum v = {0, 0};
      if (__ballot((c[0] | c[1]) != 0)) {
        uint64_t w;
        v = place_sum(step * 128 + 2 * lane, c[0], &w);
        const Sum v1 = place_sum(step * 128 + 2 * lane + 1, c[1], &w);
        v.n += v1.n;
        v.z += v1.z;
        v = wave_scan(v, lane);
      }
      if (lane == 63) {
        sh.n[step] = v.n;
        sh.z[step] = v.z;
      }
    }
    __syncthreads();
    Sum mine = {0, 0}, all;
    mine = Sum{sh.n[tid], sh.z[tid]};
    static_assert(kSteps == NT, "one step a thread");
    const Sum incl = block_scan(mine, wave, lane, sh.wave, &all);
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
      Sum sc = wave_scan(own, lane);
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
        const uint64_t b = __ballot(weight(gap, p.T) >= fmin(p.min_p, 1.0));
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
    prob = static_cast<float>(weight(gap, p.T) * scale / static_cast<double>(part.z));
  }

  // The rank-th entry with the drawn value, in vocabulary order.
  const uint32_t bits = place_bits(place), two = bits | bits << 16;
  const uint32_t mask = bits == 0 ? 0x7fff7fffu : 0xffffffffu;
  u16x2 other = {0, 0};                          // entries of this lane that differ
  uint32_t held = 0;
  each_vector<REG>(reg, s, lane, [&](int j, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      other += __builtin_elementwise_min(__builtin_bit_cast(u16x2, (v[q] ^ two) & mask), u16x2{1, 1});
    held += 8;
  });
  const bool extra_match = s.extra >= 0 && ((xbits ^ bits) & mask & 0xffffu) == 0;
  const uint32_t count = held - other[0] - other[1] + (extra_match ? 1 : 0);
  find_and_write<true, REG>(a, r, reg, s, count, rank, prob, kept, wave, lane, sh.count, extra_match,
                            [&](const u32x4& v, int e) __attribute__((always_inline)) {
                              return (((e & 1 ? v[e / 2] >> 16 : v[e / 2]) ^ bits) & mask & 0xffffu) == 0;
                            });
}

// ----------------------------------------------------------------------------
// fp32
// ----------------------------------------------------------------------------
// Bit patterns in rising order; -0 as +0.
__device__ inline uint32_t ordered(uint32_t b) {
  if (b == 0x80000000u) b = 0;
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ inline double ordered_value(uint32_t k) {
  return static_cast<double>(__uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k));
}

constexpr int kBins = 8192, kMid = 1024;   // upper 13 bits; next 10 (and the last 9)
static_assert(kMid == 2 * NT, "two or one bins of the lower levels a thread");

struct F32Shared {
  uint64_t z[kBins];
  uint32_t n[kBins];
  uint64_t z2[kMid];
  uint32_t n2[kMid];
  Sum wave[NW];
  uint32_t count[NW];
  float top[NW];
  Found found;
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
  for (int i = tid; i < kBins; i += NT) {
    sh.z[i] = 0;
    sh.n[i] = 0;
  }

  auto each = [&](auto f) __attribute__((always_inline)) {   // f(bits) of every entry (NaN past the end)
    constexpr int U = 4;                         // loads ahead
    for (int j = 0; j < s.count; j += 64 * U) {
      u32x4 v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        v[i] = u32x4{kNone, kNone, kNone, kNone};
        if (j + 64 * i + lane < s.count) v[i] = s.base[s.first + j + 64 * i + lane];
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f(v[i][q]);
          __builtin_amdgcn_sched_barrier(0);   // (sixteen exps side by side take more registers than there are)
        }
    }
    f(xbits);
  };
  float best = -__builtin_huge_valf();
  each([&](uint32_t b) __attribute__((always_inline)) { best = fmaxf(best, __uint_as_float(b)); });
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) best = fmaxf(best, __shfl_xor(best, d));
  if (lane == 0) sh.top[wave] = best;
  __syncthreads();
  for (int w = 0; w < NW; ++w) best = fmaxf(best, sh.top[w]);
  if (best == -__builtin_huge_valf()) {
    write_none(a, r);
    return;
  }
  const double m = static_cast<double>(best), scale = a.one;
  const uint32_t top = ordered(__float_as_uint(best));

  // The weight of a pattern, and whether it can be kept at all.
  auto gap_of = [&](uint32_t b) __attribute__((always_inline)) {
    return __uint_as_float(b) == best ? 0.0 : static_cast<double>(__uint_as_float(b)) - m;
  };
  auto fixed = [&](double gap) { return static_cast<uint64_t>(rint(weight(gap, p.T) * scale)); };
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
    const Sum incl = block_scan(mine, wave, lane, sh.wave, &all);
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
            sh.found = Found{static_cast<uint32_t>(bin), at.n, 0, at.z, 0};
            break;
          }
          at = next;
        }
      }
      __syncthreads();
      Found f = sh.found;
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
        Sum in = block_scan(Sum{v[0].n + v[1].n, v[0].z + v[1].z}, wave, lane, sh.wave, &t);
        in.n += f.n_before;
        in.z += f.z_before;
        const Sum mid = {in.n - v[1].n, in.z - v[1].z}, ex = {mid.n - v[0].n, mid.z - v[0].z};
        if (reached(kind, in, target) && !reached(kind, ex, target)) {
          const int i = reached(kind, mid, target) ? 0 : 1;
          const Sum before = i ? mid : ex;
          sh.found = Found{f.key << bits | static_cast<uint32_t>(width - 1 - tid * per - i), before.n, v[i].n, before.z, v[i].z};
        }
        __syncthreads();
        f = sh.found;
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
        const uint64_t b = __ballot(weight(gap, p.T) >= least);   // (a NaN's pattern: false)
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
      block_scan(v, wave, lane, sh.wave, &by_min);
    }
    Sum part;
    const Found f = cut_and_draw(p, all, by_min, u, &rank, &part, find);
    key = f.key;
    kept = part.n;
    const double gap = key == top ? 0.0 : ordered_value(key) - m;
    prob = static_cast<float>(weight(gap, p.T) * scale / static_cast<double>(part.z));
  }

  const u32x4 none[kRegs] = {};
  uint32_t count = 0;
  each([&](uint32_t b) __attribute__((always_inline)) { count += ordered(b) == key ? 1 : 0; });
  const bool extra_match = s.extra >= 0 && ordered(xbits) == key;
  find_and_write<false, false>(a, r, none, s, count, rank, prob, kept, wave, lane, sh.count, extra_match,
                             [&](const u32x4& v, int e) __attribute__((always_inline)) { return ordered(v[e]) == key; });
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
