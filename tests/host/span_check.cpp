// Host-only check of attention over a list of tiles, built by g++ under
// -fsanitize=address,undefined.  Every list of a small range, key by key: what each row
// sees is in exactly one tile, a tile loads only keys that some row sees, and the pages
// staged for a part of the list are those of its keys.  Then a seeded fuzz of
// descriptors with extreme values, whose plans hold what the kernels assume.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "simsd.h"
#include "simsd_ops_plan.h"
#include "simsd_plan.h"
#include "simsd_span_list.h"
#include "simsd_span_plan.h"

using namespace simsd;

static long g_fail = 0, g_checks = 0;
#define EXPECT(cond)                                                                    \
  do {                                                                                  \
    ++g_checks;                                                                         \
    if (!(cond)) {                                                                      \
      if (++g_fail < 50) std::fprintf(stderr, "%s:%d: expectation failed: %s\n", __FILE__, __LINE__, #cond); \
    }                                                                                   \
  } while (0)

static std::mt19937_64 rng(11);
template <typename T>
static T pick(std::initializer_list<T> v) { return *(v.begin() + rng() % v.size()); }

// The definition: does the token at position p of a sequence of kv see key t?
static bool defined(int m, int window, int sinks, int kv, int p, int t) {
  if (p < 0 || t >= kv) return false;
  if (m && t >= (p / m + 1) * m) return false;
  return !window || t > p / m * m - window || t < sinks;
}

// The rows at positions p0..p1 of a sequence of kv keys.
static void one_list(int TK, int m, int window, int sinks, int kv, int p0, int p1, int P) {
  const int hi = limit_at(m, kv, p1);
  const Span s = span_of(sinks, first_at(m, window, p0), hi, TK);
  std::vector<char> some(kv + 1, 0);
  for (int p = p0; p <= p1; ++p)
    for (int t = 0; t < kv; ++t) some[t] |= defined(m, window, sinks, kv, p, t);
  std::vector<int> home(kv + 1, 0);
  bool kept = true, once = true, word = true;
  for (int L = 0; L < s.tiles; ++L) {
    const TileKeys k = tile_keys(s, L, TK);
    kept &= k.k0 >= 0 && k.k0 % TK == 0 && k.beg < k.end && k.end <= kv;
    for (int j = 0; j < TK; ++j) {
      const int read = std::max(k.beg, std::min(k.k0 + j, k.end - 1));
      kept &= read >= 0 && read < kv && some[read];
    }
    for (int p = p0; p <= p1; ++p) {
      const int limit = limit_at(m, kv, p), first = first_at(m, window, p);
      for (int half = 0; half < TK / 32; ++half) {
        const uint32_t w = seen_word(s, k, k.k0 + 32 * half, limit, first);
        for (int j = 0; j < 32; ++j) {
          const int t = k.k0 + 32 * half + j;
          const bool sees = w >> j & 1;
          word &= sees == row_sees(s, k, t, limit, first);
          if (!sees) continue;
          once &= t < kv && defined(m, window, sinks, kv, p, t);
          if (t < kv) home[t] += p == p1;
        }
      }
    }
  }
  for (int t = 0; t < kv; ++t) once &= home[t] == defined(m, window, sinks, kv, p1, t);
  EXPECT(kept);
  EXPECT(once);
  EXPECT(word);
  // Any part of the list: the staged pages hold its keys' ones, and only such.
  for (int t0 = 0; t0 < s.tiles; t0 += 1 + rng() % 3) {
    const int t1 = std::min<int>(s.tiles, t0 + 1 + rng() % 4);
    const PageSpan g = pages_of(s, t0, t1, TK, P);
    bool in = g.sinks >= 0 && g.wins >= 0 && g.sinks + g.wins <= (t1 - t0) * TK / P + 4;
    for (int L = t0; L < t1; ++L) {
      const TileKeys k = tile_keys(s, L, TK);
      for (int j = 0; j < TK; ++j) {
        const int page = std::max(k.beg, std::min(k.k0 + j, k.end - 1)) / P;
        in &= k.sink ? page >= g.first_sink && page < g.first_sink + g.sinks
                     : page >= g.first_win && page < g.first_win + g.wins;
      }
    }
    auto used = [&](int page) {
      for (int t = page * P; t < std::min(kv, (page + 1) * P); ++t)
        if (some[t]) return true;
      return false;
    };
    for (int i = 0; i < g.sinks; ++i) in &= used(g.first_sink + i);
    for (int i = 0; i < g.wins; ++i) in &= used(g.first_win + i);
    EXPECT(in);
  }
}

static void lists() {
  for (int kv : {1, 2, 31, 63, 64, 65, 100, 128, 150, 200, 321})
    for (int m : {1, 2, 5, 8, 64, 100})
      for (int window : {0, 1, 2, 31, 63, 64, 65, 90, 130, 400})
        for (int sinks : {0, 1, 4, 63, 64, 65, 90, 1000}) {
          if (!window && sinks) continue;
          for (int i = 0; i < 3; ++i) {
            const int p1 = static_cast<int>(rng() % kv), p0 = std::max<int>(p1 - static_cast<int>(rng() % 40), -3);
            const int P = pick({1, 3, 16, 24, 64, 100, 256});
            one_list(64, m, window, sinks, kv, p0, p1, P);
            one_list(32, m, window, sinks, kv, p0, p1, P);
          }
          one_list(64, m, window, sinks, kv, kv - 1, kv - 1, 16);
        }
  for (int kv : {1, 64, 200}) one_list(64, 0, 0, 0, kv, 0, kv - 1, 16);
}

static int32_t some_int(std::initializer_list<int32_t> usual) {
  const int32_t odd[] = {INT32_MIN, -1, 0, 1, 2, 3, 7, 63, 64, 65, 1000, 65535, 65536, 1 << 20, INT32_MAX};
  return rng() % 6 ? pick(usual) : odd[rng() % (sizeof odd / sizeof *odd)];
}
static int64_t some_stride() {
  const int64_t odd[] = {INT64_MIN, -8, 0, 4, 8, 16, int64_t{1} << 40, int64_t{1} << 48, INT64_MAX};
  return rng() % 5 ? int64_t(rng() % 4096) * 16 : odd[rng() % (sizeof odd / sizeof *odd)];
}
static float some_float(std::initializer_list<float> usual) {
  const float odd[] = {-1.f, 0.f, 1e-30f, 3e38f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()};
  return rng() % 6 ? pick(usual) : odd[rng() % 6];
}
static void some_dtype(simsd_dtype* t) {
  const int v = rng() % 8 ? int(rng() % 2) : int(rng() % 100) - 50;
  std::memcpy(t, &v, sizeof *t);
}

// Blocks of the longest lists fit the ranges, whatever positions their rows have.
static void covered(const SpanPlan& p, int TK, int max_kv, int m, int window, int sinks, bool verify) {
  m = std::min(m, std::max(max_kv, 1));
  for (int i = 0; i < 6; ++i) {
    if (max_kv < 1) break;
    const int kv = i ? 1 + static_cast<int>(rng() % max_kv) : max_kv;
    const int span = verify ? 0 : (p.rows_pb - 1) / p.group + 1;
    const int p1 = i == 1 ? static_cast<int>(rng() % kv) : kv - 1;
    const int p0 = std::max(p1 - span, i == 2 ? -1 : 0);
    int first = first_at(m, window, p0), hi = limit_at(m, kv, p1);
    if (verify) {
      first = window ? std::max(0, kv - window + 1) : 0;
      hi = kv;
    }
    const Span s = span_of(sinks, first, hi, TK);
    const int64_t tiles = int64_t{s.tiles} + verify;
    EXPECT((tiles * TK + p.chunk - 1) / p.chunk <= p.splits);
  }
}

static void common(const SpanPlan& p, bool bf16, int page_size, int64_t tokens, int hq, int hkv, int d) {
  EXPECT(p.chunk >= 64 && p.chunk % 64 == 0);
  EXPECT(p.splits >= 1 && p.splits <= 65535);
  if (page_size > 0) EXPECT(int64_t{p.chunk} / page_size + 4 <= kMaxChunkPages || p.chunk == 64);
  if (page_size > 0) EXPECT(int64_t{p.chunk} / page_size + 4 <= kMaxChunkPages);
  EXPECT(int64_t{p.blocks} * hkv <= (1 << 22));
  EXPECT(p.fold == 0 || (p.splits == 1 && p.fold < p.blocks && p.blocks <= 2 * p.fold));
  EXPECT(p.tile == (bf16 && !p.few ? 64 : 32) && p.chunk % p.tile == 0);
  EXPECT(p.few    ? bf16 && p.rows_pb == 32 * p.few && p.few <= 2 && p.row_waves == 0
         : bf16   ? p.rows_pb == 32 * p.row_waves && (p.row_waves == 2 || p.row_waves == 4 || p.row_waves == 8)
              : p.rows_pb == 16 || p.rows_pb == 32 || p.rows_pb == 64 || p.rows_pb == 128);
  EXPECT(p.window >= 0 && p.sinks >= 0 && (p.window > 0 || p.sinks == 0));
  const size_t n = size_t(p.splits) * tokens * hq;
  EXPECT(p.workspace == (p.splits > 1 && tokens > 0 ? n * (d + 2) * 4 : 0));
  EXPECT(p.ml_off % 8 == 0);
}

static int fuzz_chunk() {
  simsd_chunk_desc d{};
  d.num_tokens = some_int({1, 8, 100, 4096});
  d.batch = some_int({1, 8, 64, 300});
  d.num_kv_heads = some_int({1, 2, 8});
  d.num_q_heads = rng() % 8 ? int32_t(std::min<int64_t>(int64_t{d.num_kv_heads} * (1 + rng() % 16), 1 << 20)) : some_int({32});
  d.head_dim = some_int({64, 128});
  d.max_q_len = some_int({1, 8, 300, 4096});
  d.max_kv_len = some_int({0, 100, 4000, 32768, 1000000, 1 << 30});
  d.mask_block = some_int({0, 1, 8, 32});
  d.page_size = some_int({0, 1, 16, 24, 64, 256});
  d.max_pages_per_seq = some_int({0, 4096, 1 << 20, 1 << 24});
  d.kv_chunk = rng() % 3 ? 0 : some_int({64, 128, 4096});
  d.cache_stride_seq = some_stride();
  d.cache_stride_token = some_stride();
  d.cache_stride_head = some_stride();
  d.scale = some_float({0.f, 0.1f});
  some_dtype(&d.dtype);
  const int window = some_int({0, 1, 100, 4096}), sinks = some_int({0, 0, 4, 100});
  const int cus = pick({1, 32, 256, 304});
  const bool fp4 = rng() % 2;
  SpanPlan p;
  const simsd_status st = fp4 ? plan_chunk_fp4(&d, window, sinks, cus, &p) : plan_window(&d, window, sinks, cus, &p);
  if (st != SIMSD_OK) return 0;
  EXPECT(window == 0 || d.mask_block >= 1);
  EXPECT(!fp4 || (d.dtype == SIMSD_BF16 && d.cache_stride_token % 16 == 0));
  const bool bf16 = d.dtype == SIMSD_BF16;
  common(p, bf16, d.page_size, d.num_tokens, d.num_q_heads, d.num_kv_heads, d.head_dim);
  EXPECT(p.blocks == std::max<int64_t>(int64_t{d.num_tokens} * p.group - 1, 0) / p.rows_pb + d.batch);
  EXPECT(fp4 ? p.row_waves != 2 : p.few == 0);
  covered(p, p.tile, d.max_kv_len, d.mask_block, p.window, p.sinks, false);
  return 1;
}

static int fuzz_verify() {
  simsd_attn_desc d{};
  d.batch = some_int({1, 8, 64, 300});
  d.num_kv_heads = some_int({1, 2, 8});
  d.num_q_heads = rng() % 8 ? int32_t(std::min<int64_t>(int64_t{d.num_kv_heads} * (1 + rng() % 16), 1 << 20)) : some_int({32});
  d.head_dim = some_int({64, 128});
  d.block_size = some_int({1, 4, 8, 32});
  d.max_ref = some_int({0, 1, 4, 8});
  d.max_prefix_len = some_int({0, 100, 4000, 32768, 1 << 30});
  d.page_size = some_int({0, 1, 16, 24, 256});
  d.max_pages_per_seq = some_int({0, 4096, 1 << 20, 1 << 24});
  d.kv_chunk = rng() % 3 ? 0 : some_int({64, 128, -1});
  d.cache_stride_seq = some_stride();
  d.cache_stride_token = some_stride();
  d.cache_stride_head = some_stride();
  d.scale = some_float({0.f, 0.1f});
  d.rope_theta = rng() % 4 ? 0.f : some_float({10000.f});
  some_dtype(&d.dtype);
  const int window = some_int({0, 1, 100, 4096}), sinks = some_int({0, 0, 4, 100});
  const int cus = pick({1, 32, 256, 304});
  SpanPlan p;
  if (plan_verify_span(&d, rng() % 2, window, sinks, cus, &p) != SIMSD_OK) return 0;
  EXPECT(d.dtype == SIMSD_BF16 && d.rope_theta == 0.f && d.kv_chunk >= 0);
  const int n = d.block_size + d.max_ref;
  common(p, true, d.page_size, int64_t{d.batch} * n, d.num_q_heads, d.num_kv_heads, d.head_dim);
  EXPECT(p.seq_blocks * p.rows_pb >= n * p.group && p.blocks == d.batch * p.seq_blocks);
  covered(p, p.tile, d.max_prefix_len, 1, p.window, p.sinks, true);
  return 1;
}

static void fuzz_append() {
  simsd_rotary_desc d{};
  d.num_tokens = some_int({1, 8, 4096});
  d.num_q_heads = some_int({0, 1, 8, 32});
  d.num_kv_heads = some_int({1, 2, 8});
  d.head_dim = some_int({64, 128});
  d.rotary_dim = some_int({2, 6, 32, 64, 128});
  d.batch = some_int({1, 8, 64});
  d.max_kv_len = some_int({0, 100, 32768});
  d.page_size = some_int({0, 16, 64});
  d.max_pages_per_seq = some_int({0, 10, 4096});
  d.num_pages = some_int({0, 100});
  d.attn_factor = some_float({1.f, 1.2f});
  int64_t* s[] = {&d.q_stride_token, &d.q_stride_head, &d.k_stride_token, &d.k_stride_head, &d.v_stride_token,
                  &d.v_stride_head, &d.cache_stride_seq, &d.cache_stride_token, &d.cache_stride_head};
  for (int64_t* x : s) *x = some_stride();
  d.q_out_stride_head = 512;
  d.q_out_stride_token = 65536;
  some_dtype(&d.dtype);
  simsd_fp4_cache c{};
  c.k = c.v = reinterpret_cast<void*>(uintptr_t{0x10000});
  c.k_scales = c.v_scales = reinterpret_cast<void*>(uintptr_t{0x10004});
  c.scale_stride_seq = some_stride();
  c.scale_stride_token = some_stride();
  c.scale_stride_head = some_stride();
  if (plan_fp4_append(&d, rng() % 8 ? &c : nullptr) == SIMSD_OK) EXPECT(d.dtype == SIMSD_BF16 && d.cache_stride_head % 16 == 0);
  simsd_fp4_values_desc v{};
  v.num = some_int({0, 1, 100});
  v.tokens = some_int({1, 16});
  v.num_kv_heads = some_int({1, 8});
  v.head_dim = some_int({32, 64, 96, 128, 512});
  v.cache_stride_seq = some_stride();
  v.cache_stride_token = some_stride();
  v.cache_stride_head = some_stride();
  if (check_fp4_values(&v, rng() % 8 ? &c : nullptr, c.k, rng() % 2 ? c.v : nullptr) == SIMSD_OK)
    EXPECT(v.num >= 0 && v.tokens >= 0 && v.num_kv_heads >= 0 && v.head_dim % 32 == 0 && v.head_dim <= 512);
}

int main() {
  lists();
  long good = 0;
  for (int i = 0; i < 200000; ++i) {
    good += fuzz_chunk() + fuzz_verify();
    fuzz_append();
  }
  EXPECT(good > 20000);
  std::printf("%ld checks, %ld plans, %ld failed\n", g_checks, good, g_fail);
  return g_fail ? 1 : 0;
}
