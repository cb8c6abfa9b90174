// Planning, argument checking and host helpers of the operators beside the
// verification step.  No HIP calls: this file is plain C++17.
#include "simsd_ops_plan.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "simsd_plan.h"

namespace simsd {

static simsd_status fail(simsd_status st, const std::string& msg) {
  set_error(msg);
  return st;
}

static bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A dtype field as the integer a C caller stored there.
static bool known_dtype(const simsd_dtype& field) {
  int v;
  std::memcpy(&v, &field, sizeof v);
  return v == SIMSD_F32 || v == SIMSD_BF16;
}

static simsd_status check_strides(const char* op, const int64_t* s, int n, int eb, int most_log2) {
  for (int i = 0; i < n; ++i) {
    if (s[i] < 0) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": negative stride");
    if (s[i] % (16 / eb) != 0)
      return fail(SIMSD_ERR_ALIGNMENT, std::string(op) + ": strides must be multiples of 16 bytes");
    if (s[i] > (int64_t{1} << most_log2))
      return fail(SIMSD_ERR_BAD_SHAPE,
                  std::string(op) + ": stride beyond 2^" + std::to_string(most_log2) + " elements");
  }
  return SIMSD_OK;
}

// Rows [tokens, heads] of d elements that do not overlap, whichever index is outer.
// (Strides up to 2^40 times counts up to 2^31: 128-bit products.)
static bool apart(__int128 tokens, __int128 heads, __int128 st, __int128 sh, __int128 d) {
  if (tokens < 1 || heads < 1) return true;
  const bool head_inner = (heads == 1 || sh >= d) && (tokens == 1 || st >= sh * (heads - 1) + d);
  const bool token_inner = (tokens == 1 || st >= d) && (heads == 1 || sh >= st * (tokens - 1) + d);
  return head_inner || token_inner;
}

simsd_status plan_rotary(const simsd_rotary_desc* d, bool append, RotaryPlan* p) {
  if (!d || !p) return fail(SIMSD_ERR_NULL_POINTER, "rotary: descriptor is NULL");
  if (!known_dtype(d->dtype))
    return fail(SIMSD_ERR_UNSUPPORTED, "rotary: dtype must be SIMSD_F32 or SIMSD_BF16");
  if (d->num_tokens < 0 || d->num_tokens > (1 << 24))
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: num_tokens must be in [0, 2^24]");
  if (d->num_q_heads < 0 || d->num_kv_heads < 0 || d->num_q_heads > 65535 || d->num_kv_heads > 65535 ||
      (append && d->num_kv_heads < 1))
    return fail(SIMSD_ERR_BAD_SHAPE, append ? "rotary: need num_q_heads in [0, 65535] and num_kv_heads in [1, 65535]"
                                            : "rotary: need num_q_heads and num_kv_heads in [0, 65535]");
  if (d->head_dim < 8 || d->head_dim > 512 || d->head_dim % 8 != 0)
    return fail(SIMSD_ERR_UNSUPPORTED, "rotary: head_dim must be a multiple of 8 in [8, 512]");
  if (d->rotary_dim < 2 || d->rotary_dim > d->head_dim || d->rotary_dim % 2 != 0)
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: rotary_dim must be even and in [2, head_dim]");
  if (d->interleaved != 0 && d->interleaved != 1)
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: interleaved must be 0 or 1");
  if (!(std::isfinite(d->attn_factor) && d->attn_factor > 0.f))
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: attn_factor must be finite and > 0");
  const int eb = d->dtype == SIMSD_F32 ? 4 : 2;
  const int64_t in[8] = {d->q_stride_token, d->q_stride_head, d->k_stride_token, d->k_stride_head,
                         d->q_out_stride_token, d->q_out_stride_head,
                         append ? d->v_stride_token : d->k_out_stride_token,
                         append ? d->v_stride_head : d->k_out_stride_head};
  simsd_status st = check_strides("rotary", in, 8, eb, 40);
  if (st != SIMSD_OK) return st;
  if (!apart(d->num_tokens, d->num_q_heads, d->q_out_stride_token, d->q_out_stride_head, d->head_dim) ||
      (!append && !apart(d->num_tokens, d->num_kv_heads, d->k_out_stride_token, d->k_out_stride_head, d->head_dim)))
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: rows of an output overlap");
  if (append) {
    if (d->batch < 1 || d->batch > 65535)
      return fail(SIMSD_ERR_BAD_SHAPE, "rotary: batch must be in [1, 65535]");
    if (d->max_kv_len < 0) return fail(SIMSD_ERR_BAD_SHAPE, "rotary: max_kv_len < 0");
    if (d->page_size < 0) return fail(SIMSD_ERR_BAD_SHAPE, "rotary: page_size < 0");
    if (d->page_size > 0 && (d->num_pages < 0 || d->max_pages_per_seq < ceil_div(d->max_kv_len, d->page_size)))
      return fail(SIMSD_ERR_BAD_SHAPE,
                  "rotary: need num_pages >= 0 and max_pages_per_seq >= ceil(max_kv_len / page_size)");
    const int64_t cache[3] = {d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head};
    st = check_strides("rotary", cache, 3, eb, 48);
    if (st != SIMSD_OK) return st;
  }
  RotaryPlan r;
  // Vectors of 16 bytes where both halves of the turning part (or, interleaved,
  // the part itself) are whole vectors; single elements else.
  const int w = 16 / eb, half = d->rotary_dim / 2;
  r.vec = (d->interleaved ? d->rotary_dim : half) % w == 0 ? w : 1;
  const int copy = (d->head_dim - d->rotary_dim) / r.vec;
  r.q_units = (d->interleaved ? (r.vec > 1 ? d->rotary_dim / r.vec : half) : half / r.vec) + copy;
  r.v_units = append ? d->head_dim / w : 0;
  const int64_t units = int64_t{r.q_units} * (int64_t{d->num_q_heads} + d->num_kv_heads) +
                        int64_t{r.v_units} * d->num_kv_heads;
  if (units > (int64_t{1} << 26)) return fail(SIMSD_ERR_BAD_SHAPE, "rotary: too many heads");
  r.units = static_cast<int>(units);
  *p = r;
  return SIMSD_OK;
}

simsd_status check_rotary_args(const simsd_rotary_desc* d, const void* q, const void* k,
                               const int32_t* positions, const double* freq, const void* q_out,
                               const void* k_out) {
  if (d->num_tokens == 0) return SIMSD_OK;
  if (!positions || !freq) return fail(SIMSD_ERR_NULL_POINTER, "rotary: positions and freq are required");
  if ((d->num_q_heads > 0 && (!q || !q_out)) || (d->num_kv_heads > 0 && (!k || !k_out)))
    return fail(SIMSD_ERR_NULL_POINTER, "rotary: q, q_out (Hq > 0) and k, k_out (Hkv > 0) are required");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16))
    return fail(SIMSD_ERR_ALIGNMENT, "rotary: q, k and the outputs must be 16-byte aligned");
  if (!aligned(positions, 4) || !aligned(freq, 8))
    return fail(SIMSD_ERR_ALIGNMENT, "rotary: positions must be 4-byte and freq 8-byte aligned");
  if ((d->num_q_heads > 0 && q == q_out && (d->q_stride_token != d->q_out_stride_token || d->q_stride_head != d->q_out_stride_head)) ||
      (d->num_kv_heads > 0 && k == k_out && (d->k_stride_token != d->k_out_stride_token || d->k_stride_head != d->k_out_stride_head)))
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: an output in place needs its input's strides");
  return SIMSD_OK;
}

simsd_status check_rotary_append_args(const simsd_rotary_desc* d, const void* q, const void* k,
                                      const void* v, const int32_t* positions,
                                      const double* freq, const void* q_out,
                                      const void* k_cache, const void* v_cache,
                                      const int32_t* block_table, const int32_t* q_starts,
                                      const int32_t* kv_lens) {
  if (d->num_tokens == 0) return SIMSD_OK;
  if (!k || !v || !freq || !q_starts || !kv_lens)
    return fail(SIMSD_ERR_NULL_POINTER, "rotary: k, v, freq, q_starts and kv_lens are required");
  if (d->num_q_heads > 0 && (!q || !q_out))
    return fail(SIMSD_ERR_NULL_POINTER, "rotary: q and q_out are required (Hq > 0)");
  if (d->max_kv_len > 0 && (!k_cache || !v_cache))
    return fail(SIMSD_ERR_NULL_POINTER, "rotary: k_cache and v_cache are required");
  if (d->page_size > 0 && d->max_kv_len > 0 && !block_table)
    return fail(SIMSD_ERR_NULL_POINTER, "rotary: block_table required for a paged cache");
  const void* data[] = {q, k, v, q_out, k_cache, v_cache};
  for (const void* a : data)
    if (!aligned(a, 16))
      return fail(SIMSD_ERR_ALIGNMENT, "rotary: q, k, v, q_out and the cache must be 16-byte aligned");
  const void* words[] = {positions, block_table, q_starts, kv_lens};
  for (const void* a : words)
    if (!aligned(a, 4)) return fail(SIMSD_ERR_ALIGNMENT, "rotary: int32 arrays must be 4-byte aligned");
  if (!aligned(freq, 8)) return fail(SIMSD_ERR_ALIGNMENT, "rotary: freq must be 8-byte aligned");
  if (d->num_q_heads > 0 && q == q_out &&
      (d->q_stride_token != d->q_out_stride_token || d->q_stride_head != d->q_out_stride_head))
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary: q_out in place needs the strides of q");
  return SIMSD_OK;
}

// Whether row blocks may be put on the CUs by their lengths where the chip holds them
// all at once, two to a CU: the second one of a CU is the shorter the longer its first
// (in the order of a longer grid the first half of the blocks, the long ones, all come
// before a second).  A prompt of 1000 in fp32, 64 rows: 122 -> 103 us; of 2000, 128 rows:
// 423 -> 335; in bf16, 128 rows: 116.6 -> 114.1.
static bool may_fold(const simsd_chunk_desc& d, int per_cu) { return per_cu == 2 && d.batch <= 64; }

simsd_status plan_chunk(const simsd_chunk_desc* d, int cus, ChunkPlan* p) {
  if (!d || !p) return fail(SIMSD_ERR_NULL_POINTER, "chunk_attention: descriptor is NULL");
  if (cus < 1) return fail(SIMSD_ERR_HIP, "chunk_attention: the device reports no compute units");
  if (!known_dtype(d->dtype))
    return fail(SIMSD_ERR_UNSUPPORTED, "chunk_attention: dtype must be SIMSD_F32 or SIMSD_BF16");
  if (d->num_tokens < 0 || d->num_tokens > (1 << 23))
    return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: num_tokens must be in [0, 2^23]");
  if (d->batch < 1 || d->batch > 65535)
    return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: batch must be in [1, 65535]");
  if (d->num_q_heads < 1 || d->num_kv_heads < 1 || d->num_q_heads % d->num_kv_heads != 0)
    return fail(SIMSD_ERR_BAD_SHAPE,
                "chunk_attention: need num_q_heads, num_kv_heads >= 1 and Hq % Hkv == 0");
  if (d->num_q_heads / d->num_kv_heads > kMaxGroup)
    return fail(SIMSD_ERR_UNSUPPORTED, "chunk_attention: Hq / Hkv must be <= 16");
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(SIMSD_ERR_UNSUPPORTED, "chunk_attention: head_dim must be 64 or 128");
  if (d->max_q_len < 0) return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: max_q_len < 0");
  if (d->max_kv_len < 0 || d->max_kv_len > (1 << 30))
    return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: max_kv_len must be in [0, 2^30]");
  if (d->mask_block < 0) return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: mask_block < 0");
  if (d->page_size < 0) return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: page_size < 0");
  if (d->page_size > 0 && d->max_pages_per_seq < ceil_div(d->max_kv_len, d->page_size))
    return fail(SIMSD_ERR_BAD_SHAPE,
                "chunk_attention: max_pages_per_seq < ceil(max_kv_len / page_size)");
  if (d->kv_chunk < 0 || d->kv_chunk % kTile != 0)
    return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: kv_chunk must be 0 (auto) or a multiple of 64");
  const int64_t strides[3] = {d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head};
  const int eb = d->dtype == SIMSD_F32 ? 4 : 2;
  const simsd_status st = check_strides("chunk_attention", strides, 3, eb, 48);
  if (st != SIMSD_OK) return st;
  if (!(std::isfinite(d->scale) && d->scale >= 0.f))
    return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: scale must be finite and >= 0");

  ChunkPlan r;
  r.group = d->num_q_heads / d->num_kv_heads;
  const int64_t rows = int64_t{std::min(d->max_q_len, d->num_tokens)} * r.group;   // of the longest sequence
  const int64_t tiles = std::max<int64_t>(ceil_div(d->max_kv_len, kTile), 1);
  int64_t most = tiles * kTile;
  if (d->page_size > 0)   // a work-group holds the ids of its pages in LDS
    most = std::min(most, std::max<int64_t>(int64_t{kMaxChunkPages - 1} * d->page_size / kTile * kTile, kTile));
  // Rows per work-group and key ranges per row: the cheapest by an estimate of the
  // call's time.  A shape's tile of 64 keys takes `alone` us where its CU has nothing
  // else, `full` where all slots are taken (D = 128), or what its keys take to come
  // from memory, which the blocks of a sequence share.  While all work-groups run at
  // once the slowest CU counts (see may_fold); else what a slot goes through (rows of a
  // chunk see half of it on average; and a guess, as the lengths are on the device, that
  // the sequences of a batch have 0.7 of the longest one's keys: ranges cost calls of equal
  // lengths 5 %, their lack others up to half) and a third of a work-group for the uneven
  // end.  Joining ranges costs a kernel and the partials' way to memory and back.
  //
  // Calls in us, 32/8 heads, by the shape taken and by others.  Single tokens, 64 rows: 64
  // over 512..32767 keys, ranges of 2048 820, whole 947; 16 over 512..32000, 24 ranges 226,
  // whole 630; 64 over 4000 each, 3 ranges 206, whole 196.  8 chunks of 32 over 4096, 64 rows
  // in 3 ranges 43, 128 rows 47 (whole: 68 and 95).  512 tokens over 16000, 128 rows in 4
  // ranges 158, whole 356, 64 rows 199.  24 of 1..351 over 101..6007, 128 rows 298, 256 rows
  // 301, 64 rows 370.  A prompt of 2048, 128 rows 56, 256 rows 67, 64 rows 62; 4 of 2048 over
  // 14336, 256 rows 1970, 128 rows 2050, 64 rows 2510.  fp32: a prompt of 1000, 64 rows 103,
  // 32 rows 118, 128 rows 138; of 512, 32 rows 36, 64 rows 52; 600 over 2000, 128 rows in 3
  // ranges 269, 32 rows 250.
  struct Shape { int row_waves, rows, per_cu; double alone, full; };
  constexpr Shape kBf16[] = {{2, 64, 2, 0.95, 1.35}, {4, 128, 2, 1.4, 2.2}, {8, 256, 1, 1.8, 2.1}};
  constexpr Shape kF32[] = {{4, 16, 2, 2.0, 3.25}, {4, 32, 2, 3.5, 5.1}, {4, 64, 2, 5.8, 8.2}, {4, 128, 2, 10.4, 17.4}};
  const bool bf16 = d->dtype == SIMSD_BF16;
  const Shape* shapes = bf16 ? kBf16 : kF32;
  const double scale_d = d->head_dim / 128.0;
  const double causal = d->mask_block > 0 && d->mask_block < d->max_q_len
                            ? 1.0 - 0.5 * std::min(d->max_q_len, d->max_kv_len) / std::max(d->max_kv_len, 1) : 1.0;
  const double even = (d->batch > 1 ? 0.7 : 1.0) * causal;
  const double least = std::max(2.0 * causal - 1.0, 0.0);   // the shortest block's keys, of the longest one's
  const double part_us = 8.0 * (d->head_dim + 2) * d->num_tokens * d->num_q_heads / 4e6;   // both ways at 4 TB/s
  int64_t chunk = most;
  int per_cu = 1;
  double best = -1.0;
  for (int i = 0; i < (bf16 ? 3 : 4); ++i) {
    const Shape& sh = shapes[i];
    if (i > 0 && shapes[i - 1].rows >= rows) break;   // no sequence fills more than the smaller one
    const double slots = static_cast<double>(sh.per_cu) * cus;
    // Blocks of a sequence: the last one is half full where the lengths differ.
    const double filled = static_cast<double>(d->num_tokens) * r.group / d->batch / sh.rows;
    const double blocks = d->batch > 1 ? std::max(filled + 0.5, 1.0) : std::ceil(filled);
    const double groups = blocks * d->batch * d->num_kv_heads;
    for (int64_t s = 1; s <= std::min<int64_t>(tiles, 64); s += s < 8 ? 1 : s < 16 ? 2 : s < 32 ? 4 : 8) {
      const int64_t t = ceil_div(tiles, s);
      const double x = groups * s / slots;
      const double cu = x <= 0.5 ? sh.alone : x <= 1.0 ? 0.5 * (sh.alone + sh.full) : sh.full;
      const double memory = kTile * 2.0 * d->head_dim * eb * std::min(x, 1.0) * slots / 5.5e6 / std::min(blocks, 8.0);
      double one = t * std::max(cu * scale_d, memory);
      if (s == 1 && x > 0.5 && x <= 1.0 && may_fold(*d, sh.per_cu)) {
        const double first = 1.0 - (1.0 / x - 1.0) * (1.0 - least);   // the longest with a second: `least`
        const double middle = 1.0 - 0.5 / x * (1.0 - least);          // the longest second: as long as its first
        const double slowest = std::max({sh.alone, sh.alone * (first - least) + sh.full * least, sh.full * middle});
        one = t * std::max(slowest * scale_d, memory);
      }
      double us = x <= 1.0 ? one + 7.0 : even * x * (one + 5.0) + 0.35 * (one + 7.0);
      if (s > 1) us += 5.0 + s * part_us;
      if (best < 0.0 || us < best) {
        best = us;
        chunk = t * kTile;
        r.row_waves = sh.row_waves;
        r.rows_pb = sh.rows;
        per_cu = sh.per_cu;
      }
    }
  }
  const int64_t blocks = std::max<int64_t>(int64_t{d->num_tokens} * r.group - 1, 0) / r.rows_pb + d->batch;
  if (blocks * d->num_kv_heads > (1 << 22))
    return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: too many tokens and sequences for one call");
  r.blocks = static_cast<int>(blocks);
  if (d->kv_chunk > 0) chunk = d->kv_chunk;
  chunk = std::min(chunk, most);
  r.chunk = static_cast<int>(chunk);
  r.splits = static_cast<int>(std::max<int64_t>(1, ceil_div(d->max_kv_len, chunk)));
  const int c = cus / d->num_kv_heads;
  if (r.splits == 1 && may_fold(*d, per_cu) && r.blocks > c && r.blocks <= 2 * c) r.fold = c;
  if (r.splits > 65535) return fail(SIMSD_ERR_BAD_SHAPE, "chunk_attention: too many key ranges");
  if (r.splits > 1 && d->num_tokens > 0) {
    const size_t n = static_cast<size_t>(r.splits) * d->num_tokens * d->num_q_heads;
    r.ml_off = n * d->head_dim * sizeof(float);
    r.workspace = r.ml_off + n * 2 * sizeof(float);
  }
  const float scale = d->scale > 0.f ? d->scale : 1.0f / std::sqrt(static_cast<float>(d->head_dim));
  r.scale_log2 = scale * 1.4426950408889634f;
  *p = r;
  return SIMSD_OK;
}

simsd_status check_chunk_args(const simsd_chunk_desc* d, const ChunkPlan& p, const void* q,
                              const void* k_cache, const void* v_cache, const int32_t* block_table,
                              const int32_t* q_starts, const int32_t* kv_lens, const void* out,
                              const float* lse, const void* workspace, size_t workspace_bytes) {
  if (d->num_tokens == 0) return SIMSD_OK;
  if (!q || !q_starts || !kv_lens || !out)
    return fail(SIMSD_ERR_NULL_POINTER, "chunk_attention: q, q_starts, kv_lens and out are required");
  if (d->max_kv_len > 0 && (!k_cache || !v_cache))
    return fail(SIMSD_ERR_NULL_POINTER, "chunk_attention: k_cache/v_cache required when max_kv_len > 0");
  if (d->page_size > 0 && d->max_kv_len > 0 && !block_table)
    return fail(SIMSD_ERR_NULL_POINTER, "chunk_attention: block_table required for a paged cache");
  const void* data[] = {q, k_cache, v_cache, out};
  for (const void* a : data)
    if (!aligned(a, 16))
      return fail(SIMSD_ERR_ALIGNMENT, "chunk_attention: q, the caches and out must be 16-byte aligned");
  const void* words[] = {block_table, q_starts, kv_lens, lse};
  for (const void* a : words)
    if (!aligned(a, 4)) return fail(SIMSD_ERR_ALIGNMENT, "chunk_attention: arrays must be 4-byte aligned");
  if (p.workspace > 0) {
    if (!workspace) return fail(SIMSD_ERR_WORKSPACE, "chunk_attention: workspace is NULL");
    if (!aligned(workspace, 16))
      return fail(SIMSD_ERR_ALIGNMENT, "chunk_attention: workspace must be 16-byte aligned");
    if (workspace_bytes < p.workspace)
      return fail(SIMSD_ERR_WORKSPACE,
                  "chunk_attention: workspace smaller than simsd_chunk_attention_workspace_size()");
  }
  return SIMSD_OK;
}

simsd_status plan_sample(const simsd_sample_desc* d, double* one) {
  if (!d || !one) return fail(SIMSD_ERR_NULL_POINTER, "sample: descriptor is NULL");
  if (!known_dtype(d->dtype))
    return fail(SIMSD_ERR_UNSUPPORTED, "sample: dtype must be SIMSD_F32 or SIMSD_BF16");
  if (d->rows < 0 || d->rows > (1 << 21)) return fail(SIMSD_ERR_BAD_SHAPE, "sample: rows must be in [0, 2^21]");
  if (d->vocab < 1 || d->vocab > (1 << 22)) return fail(SIMSD_ERR_BAD_SHAPE, "sample: vocab must be in [1, 2^22]");
  if (!(std::isfinite(d->temperature) && d->temperature >= 0.f))
    return fail(SIMSD_ERR_BAD_SHAPE, "sample: temperature must be finite and >= 0");
  if (d->top_k < 0) return fail(SIMSD_ERR_BAD_SHAPE, "sample: top_k must be >= 0");
  if (!(d->top_p >= 0.f && d->top_p <= 1.f) || !(d->min_p >= 0.f && d->min_p <= 1.f))
    return fail(SIMSD_ERR_BAD_SHAPE, "sample: top_p and min_p must be in [0, 1]");
  int bits = 0;                                  // ceil(log2 V): V weights of 2^(62 - bits) stay below 2^63
  while ((int64_t{1} << bits) < d->vocab) ++bits;
  *one = std::ldexp(1.0, 62 - bits);
  return SIMSD_OK;
}

simsd_status check_sample_args(const simsd_sample_desc* d, const void* logits, const float* uniforms,
                               const float* temperatures, const int32_t* top_ks, const float* top_ps,
                               const float* min_ps, const int32_t* token, const float* prob,
                               const int32_t* kept) {
  if (d->rows == 0) return SIMSD_OK;
  if (!logits || !uniforms || !token)
    return fail(SIMSD_ERR_NULL_POINTER, "sample: logits, uniforms and token are required");
  if (!aligned(logits, d->dtype == SIMSD_F32 ? 4 : 2))
    return fail(SIMSD_ERR_ALIGNMENT, "sample: logits must be aligned to their elements");
  const void* words[] = {uniforms, temperatures, top_ks, top_ps, min_ps, token, prob, kept};
  for (const void* w : words)
    if (!aligned(w, 4)) return fail(SIMSD_ERR_ALIGNMENT, "sample: arrays must be 4-byte aligned");
  return SIMSD_OK;
}

}  // namespace simsd

using namespace simsd;

static simsd_status rope_frequencies(int32_t rotary_dim, double theta, const simsd_rope_scaling& scaling,
                                     double factor, int32_t original_context, double beta_fast,
                                     double beta_slow, double* freq, float* attn_factor) {
  int kind;
  std::memcpy(&kind, &scaling, sizeof kind);
  if (!freq || !attn_factor) return fail(SIMSD_ERR_NULL_POINTER, "rope_frequencies: NULL output");
  if (kind < SIMSD_ROPE_NONE || kind > SIMSD_ROPE_YARN)
    return fail(SIMSD_ERR_UNSUPPORTED, "rope_frequencies: unknown scaling");
  if (rotary_dim < 2 || rotary_dim > 512 || rotary_dim % 2 != 0)
    return fail(SIMSD_ERR_BAD_SHAPE, "rope_frequencies: rotary_dim must be even and in [2, 512]");
  if (!(std::isfinite(theta) && theta > 1.0))
    return fail(SIMSD_ERR_BAD_SHAPE, "rope_frequencies: theta must be finite and > 1");
  if (kind != SIMSD_ROPE_NONE && !(std::isfinite(factor) && factor >= 1.0))
    return fail(SIMSD_ERR_BAD_SHAPE, "rope_frequencies: factor must be finite and >= 1");
  if (kind == SIMSD_ROPE_NTK && rotary_dim < 4)
    return fail(SIMSD_ERR_BAD_SHAPE, "rope_frequencies: NTK scaling needs rotary_dim >= 4");
  if (kind == SIMSD_ROPE_YARN &&
      !(original_context >= 1 && std::isfinite(beta_fast) && beta_slow > 0.0 && beta_fast >= beta_slow))
    return fail(SIMSD_ERR_BAD_SHAPE,
                "rope_frequencies: YARN needs original_context >= 1 and beta_fast >= beta_slow > 0");
  const int half = rotary_dim / 2;
  const double d = rotary_dim;
  const double base = kind == SIMSD_ROPE_NTK ? theta * std::pow(factor, d / (d - 2.0)) : theta;
  *attn_factor = 1.f;
  double low = 0.0, high = 0.0;
  if (kind == SIMSD_ROPE_YARN) {
    // Pair index whose pair turns `beta` times in the original context.
    const double two_pi = 6.283185307179586476925;
    auto index = [&](double beta) { return d * std::log(original_context / (beta * two_pi)) / (2.0 * std::log(theta)); };
    low = std::max(std::floor(index(beta_fast)), 0.0);
    high = std::min(std::ceil(index(beta_slow)), d - 1.0);
    if (high <= low) high = low + 0.001;   // a step instead of a ramp
    *attn_factor = static_cast<float>(0.1 * std::log(factor) + 1.0);
  }
  for (int i = 0; i < half; ++i) {
    const double f = std::pow(base, -2.0 * i / d);
    if (kind == SIMSD_ROPE_LINEAR) {
      freq[i] = f / factor;
    } else if (kind == SIMSD_ROPE_YARN) {
      const double slow = std::min(std::max((i - low) / (high - low), 0.0), 1.0);
      freq[i] = f / factor * slow + f * (1.0 - slow);
    } else {
      freq[i] = f;
    }
  }
  return SIMSD_OK;
}

extern "C" simsd_status simsd_rope_frequencies(int32_t rotary_dim, double theta,
                                               simsd_rope_scaling scaling, double factor,
                                               int32_t original_context, double beta_fast,
                                               double beta_slow, double* freq, float* attn_factor) {
  try {
    return rope_frequencies(rotary_dim, theta, scaling, factor, original_context, beta_fast, beta_slow, freq,
                            attn_factor);
  } catch (...) {                                // (no memory for the message)
    return SIMSD_ERR_HIP;
  }
}
