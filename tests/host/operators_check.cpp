// Host-only check of the planning and argument checks of rotary positions, chunk
// attention and sampling (simsd_ops_plan.cpp), built by g++ under
// -fsanitize=address,undefined: a seeded fuzz of descriptors with extreme values, whose
// plans hold what the kernels assume, and the frequencies' refusals.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "simsd.h"
#include "simsd_ops_plan.h"
#include "simsd_plan.h"

using namespace simsd;

static long g_fail = 0, g_checks = 0;
#define EXPECT(cond)                                                                    \
  do {                                                                                  \
    ++g_checks;                                                                         \
    if (!(cond)) {                                                                      \
      std::fprintf(stderr, "%s:%d: expectation failed: %s\n", __FILE__, __LINE__, #cond); \
      ++g_fail;                                                                         \
    }                                                                                   \
  } while (0)

static std::mt19937_64 rng(7);

template <typename T>
static T pick(std::initializer_list<T> v) { return *(v.begin() + rng() % v.size()); }

static int32_t some_int(std::initializer_list<int32_t> usual) {
  const int32_t odd[] = {INT32_MIN, -1, 0, 1, 2, 3, 7, 63, 64, 65, 1000, 65535, 65536, 1 << 20, INT32_MAX};
  return rng() % 6 ? pick(usual) : odd[rng() % (sizeof odd / sizeof *odd)];
}
static int64_t some_stride() {
  const int64_t odd[] = {INT64_MIN, -8, 0, 4, 7, 8, int64_t{1} << 40, (int64_t{1} << 40) + 8, int64_t{1} << 48, INT64_MAX};
  return rng() % 5 ? int64_t(rng() % 4096) * 8 : odd[rng() % (sizeof odd / sizeof *odd)];
}
static float some_float(std::initializer_list<float> usual) {
  const float odd[] = {-1.f, 0.f, 1e-30f, 3e38f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()};
  return rng() % 6 ? pick(usual) : odd[rng() % 6];
}
// (Through its bytes: a value outside the enumeration must not be read as one.)
static void some_dtype(simsd_dtype* t) {
  const int v = rng() % 8 ? int(rng() % 2) : int(rng() % 100) - 50;
  std::memcpy(t, &v, sizeof *t);
}

static const void* const P = reinterpret_cast<const void*>(uintptr_t{0x10000});
static const int32_t* const I = reinterpret_cast<const int32_t*>(uintptr_t{0x10000});
static const float* const F = reinterpret_cast<const float*>(uintptr_t{0x10000});
static const double* const D = reinterpret_cast<const double*>(uintptr_t{0x10000});

static int fuzz_rotary() {
  simsd_rotary_desc d{};
  d.num_tokens = some_int({1, 8, 100, 4096});
  d.num_q_heads = some_int({0, 1, 8, 32});
  d.num_kv_heads = some_int({1, 2, 8});
  d.head_dim = some_int({8, 64, 72, 128, 512});
  d.rotary_dim = some_int({2, 6, 32, 64, 128});
  d.interleaved = some_int({0, 1});
  d.batch = some_int({1, 8, 64});
  d.max_kv_len = some_int({0, 100, 32768});
  d.page_size = some_int({0, 16, 64});
  d.max_pages_per_seq = some_int({0, 10, 4096});
  d.num_pages = some_int({0, 100});
  d.attn_factor = some_float({1.f, 1.2f});
  int64_t* s[] = {&d.q_stride_token, &d.q_stride_head, &d.k_stride_token, &d.k_stride_head, &d.v_stride_token,
                  &d.v_stride_head, &d.cache_stride_seq, &d.cache_stride_token, &d.cache_stride_head};
  for (int64_t* x : s) *x = some_stride();
  d.q_out_stride_head = d.k_out_stride_head = rng() % 8 ? 512 : some_stride();
  d.q_out_stride_token = d.k_out_stride_token = rng() % 8 ? 65536 : some_stride();
  some_dtype(&d.dtype);
  const bool append = rng() % 2;
  RotaryPlan p;
  if (plan_rotary(&d, append, &p) != SIMSD_OK) return 0;
  const int w = d.dtype == SIMSD_F32 ? 4 : 8;
  EXPECT(p.vec == 1 || p.vec == w);
  // The units cover a head once: turning ones VEC pairs, the others VEC elements.
  const int turning = d.interleaved ? (p.vec == 1 ? d.rotary_dim / 2 : d.rotary_dim / p.vec) : d.rotary_dim / 2 / p.vec;
  const int per = d.interleaved && p.vec > 1 ? p.vec : 2 * p.vec;
  EXPECT(turning * per + (p.q_units - turning) * p.vec == d.head_dim);
  EXPECT(p.units == p.q_units * (d.num_q_heads + d.num_kv_heads) + p.v_units * d.num_kv_heads);
  EXPECT(p.units >= 0 && p.units <= (1 << 26));
  if (append) check_rotary_append_args(&d, P, P, P, I, D, P, P, P, I, I, I);
  else check_rotary_args(&d, P, P, I, D, P, P);
  return 1;
}

static int fuzz_chunk() {
  simsd_chunk_desc d{};
  d.num_tokens = some_int({1, 8, 100, 4096});
  d.batch = some_int({1, 8, 64, 300});
  d.num_kv_heads = some_int({1, 2, 8});
  d.num_q_heads = rng() % 8 ? int32_t(std::min<int64_t>(int64_t{d.num_kv_heads} * (1 + rng() % 16), 1 << 20)) : some_int({32});
  d.head_dim = some_int({64, 128});
  d.max_q_len = some_int({1, 8, 300, 4096});
  d.max_kv_len = some_int({0, 100, 4000, 32768, 1000000});
  d.mask_block = some_int({0, 1, 8, 32});
  d.page_size = some_int({0, 1, 16, 24, 64, 256});
  d.max_pages_per_seq = some_int({0, 4096, 1 << 20, 1 << 24});
  d.kv_chunk = rng() % 3 ? 0 : some_int({64, 128, 4096});
  d.cache_stride_seq = some_stride();
  d.cache_stride_token = some_stride();
  d.cache_stride_head = some_stride();
  d.scale = some_float({0.f, 0.1f});
  some_dtype(&d.dtype);
  const int cus = pick({1, 32, 256, 304});
  ChunkPlan p;
  if (plan_chunk(&d, cus, &p) != SIMSD_OK) return 0;
  EXPECT(p.chunk >= 64 && p.chunk % 64 == 0);
  EXPECT(p.splits >= 1 && p.splits <= 65535);
  EXPECT(int64_t{p.chunk} * p.splits >= d.max_kv_len);
  // A work-group's pages fit its LDS.
  if (d.page_size > 0) EXPECT((p.chunk - 1) / d.page_size + 2 <= kMaxChunkPages);
  // Every sequence's blocks have numbers, however the tokens are dealt out: b
  // sequences of x_i rows (X = T G in all) take sum ceil(x_i / R) <= floor((X - 1) / R) + b
  // blocks, as ceil(x / R) = floor((x - 1) / R) + 1.
  EXPECT(p.blocks == std::max<int64_t>(int64_t{d.num_tokens} * p.group - 1, 0) / p.rows_pb + d.batch);
  // A folded order is one of all blocks: every number once.
  EXPECT(p.fold == 0 || (p.splits == 1 && p.fold < p.blocks && p.blocks <= 2 * p.fold));
  EXPECT(int64_t{p.blocks} * d.num_kv_heads <= (1 << 22));
  EXPECT(d.dtype == SIMSD_BF16 ? p.rows_pb == 32 * p.row_waves && (p.row_waves == 2 || p.row_waves == 4 || p.row_waves == 8)
                               : p.rows_pb == 16 || p.rows_pb == 32 || p.rows_pb == 64 || p.rows_pb == 128);
  const size_t n = size_t(p.splits) * d.num_tokens * d.num_q_heads;
  EXPECT(p.workspace == (p.splits > 1 && d.num_tokens > 0 ? n * (d.head_dim + 2) * 4 : 0));
  EXPECT(p.ml_off % 8 == 0);
  check_chunk_args(&d, p, P, P, P, I, I, I, P, F, P, p.workspace);
  return 1;
}

static int fuzz_sample() {
  simsd_sample_desc d{};
  d.rows = some_int({1, 4, 512});
  d.vocab = some_int({1, 1000, 50001, 151936, 1 << 22});
  d.temperature = some_float({0.f, 1.f, 0.7f});
  d.top_k = some_int({0, 50});
  d.top_p = some_float({1.f, 0.9f});
  d.min_p = some_float({0.f, 0.1f});
  some_dtype(&d.dtype);
  double one;
  if (plan_sample(&d, &one) != SIMSD_OK) return 0;
  EXPECT(one * d.vocab <= 4.6116860184273879e18);   // 2^62: the weights' sum stays below 2^63
  EXPECT(one >= 1099511627776.0);
  check_sample_args(&d, P, F, F, I, F, F, I, F, I);
  return 1;
}

int main() {
  long good = 0;
  for (int i = 0; i < 200000; ++i) good += fuzz_rotary() + fuzz_chunk() + fuzz_sample();
  EXPECT(good > 60000);
  std::vector<double> f(256);
  // (As a C caller that passes any int for the enumeration.)
  const auto frequencies = reinterpret_cast<simsd_status (*)(int32_t, double, int, double, int32_t, double, double, double*, float*)>(
      &simsd_rope_frequencies);
  float extra;
  for (int rot : {0, 1, 2, 3, 64, 512, 514, INT32_MAX, INT32_MIN})
    for (double theta : {0.0, 1.0, 10000.0, 1e300, std::numeric_limits<double>::infinity()})
      for (int kind : {-1, 0, 1, 2, 3, 4})
        for (double factor : {0.0, 1.0, 16.0, 1e300})
          for (int context : {INT32_MIN, 0, 1, 4096, INT32_MAX}) {
            const simsd_status st = frequencies(rot, theta, kind, factor, context, 32.0, 1.0, f.data(), &extra);
            const bool fine = rot >= 2 && rot <= 512 && rot % 2 == 0 && theta > 1.0 && theta < 1e301 && kind >= 0 && kind <= 3 &&
                              (kind == 0 || factor >= 1.0) && (kind != 2 || rot >= 4) && (kind != 3 || context >= 1);
            EXPECT((st == SIMSD_OK) == fine);
          }
  std::printf("%ld checks, %ld failed\n", g_checks, g_fail);
  return g_fail ? 1 : 0;
}
