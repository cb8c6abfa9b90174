// Planning and argument checking of attention over a list of tiles and of the 4-bit
// cache's operators.  No HIP calls: this file is plain C++17.
#include "simsd_span_plan.h"

#include <algorithm>
#include <cmath>
#include <string>

#include "simsd_ops_plan.h"
#include "simsd_plan.h"

namespace simsd {

static simsd_status fail(simsd_status st, const std::string& msg) {
  set_error(msg);
  return st;
}

static bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A call, whichever entry it came by.
struct Problem {
  int tokens, batch, hq, hkv, d;
  int max_q, max_kv, mask_block, page_size, kv_chunk;
  int window, sinks;
  int n_new;                       // verification: B + L; else 0
  bool bf16, fp4;
  float scale;
};

// Tiles of a row block's list at most (TK keys each; see simsd_span.h): a row block of
// `rows` rows spans (rows - 1) / G + 2 positions, whose windows begin at their block of
// the mask and whose limits end with it.
static int64_t list_tiles(const Problem& c, int rows, int group, int64_t TK) {
  const int64_t whole = ceil_div(c.max_kv, TK);
  const int64_t fresh = c.n_new > 0 ? 1 : 0;
  if (c.window == 0) return whole + fresh;
  const int64_t between = c.n_new > 0 ? 0 : (rows - 1) / group + 1 + 2 * int64_t{c.mask_block};
  const int64_t list = ceil_div(std::min(c.sinks, c.max_kv), TK) + ceil_div(int64_t{c.window} + between, TK) + 1;
  return std::min(list, whole + (c.sinks > 0 ? 1 : 0)) + fresh;
}

static simsd_status plan(const char* op, Problem c, int cus, SpanPlan* p) {
  if (c.hq > 65535) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": num_q_heads must be <= 65535");
  SpanPlan r;
  r.group = c.hq / c.hkv;
  // A window past the longest cache is none (positions and windows add up in 32 bits).
  c.window = std::min(c.window, c.max_kv + 1);
  c.sinks = std::min(c.sinks, c.max_kv);
  c.mask_block = std::min(c.mask_block, std::max(c.max_kv, 1));
  if (c.window > c.max_kv) c.window = c.sinks = 0;
  r.window = c.window;
  r.sinks = c.sinks;
  int64_t most = int64_t{1} << 30;
  if (c.page_size > 0)   // a work-group holds the ids of its pages in LDS: two parts, each with an end page at either side
    most = std::max<int64_t>(int64_t{kMaxChunkPages - 4} * c.page_size / kTile * kTile, kTile);
  // Rows per work-group and key ranges per row: the cheapest by the estimate that the
  // chunk attention's plan makes (see there), over the tiles of a list.  alone, full: us of
  // a work-group for 64 keys (heads of 128) where it has a unit to itself and where the
  // units are full, from the difference of calls over 8192 and 16384 keys.
  // Both sides of what it chooses, us on the GPU (32 query and 8 KV heads of 128, 4 bits):
  //   verifications of 16 slots, prefixes of          planned  ranges of 16384  8192  4096
  //     64: 16640 each                                   395              380   388   412
  //     64: 512 to 32768, evenly                         402              409   420   436
  //     64: 4160, 12480, 20800 and 29120 in turn         409              385   396   432
  //     43: 24960 each                                   410              417   418   415
  //     16: 512 to 32768                                 147              211   163   160
  //   64 single tokens over 512 to 32768                 262              268   263   257
  //   one over 32768                                      26              143    78    46
  // and of the rows: 64 slots of 16 sequences over a window of 4096 in bf16, 256 rows in
  // two ranges 127, 128 rows in two 127, 128 rows in one 129.
  // The end of a call, when some units have run out of work, counts less where lists of
  // few rows start from the longest down: 0.1 of a work-group in place of 0.35 takes 8
  // ragged verifications from 103 to 65, 16 of up to 8192 from 66 to 52, 32 from 232 to 221,
  // and half of 8320 with half of 24960 from 403 to 437.
  // Chunks over 4 bits in blocks of 64, 128 and 256 rows: 11 prompts of up to 754 64, 45 and
  // 48, 7 of up to 1243 110, 83 and 90, 24 chunks of up to 469 past 3000 tokens 400, 388
  // and 407, 16 of 32 past 8000 103, 103 and 142, 42 verifications of 512 rows (heads of 64)
  // 73, 52 and 60.  The estimate takes 48, 91, 388, 106 and 60: between blocks this near it
  // errs both ways, and to make it prefer 128 throughout takes four prompts' last 2048 tokens
  // of 16384 from 1939 to 2081.
  // per_cu and the costs are those of heads of 128, the costs halved for heads of 64.  (Of
  // those three or four work-groups fit a unit where two or three are counted here, and two
  // of 256 rows; the estimate has not been fitted to them.)
  struct Shape { int row_waves, few, tile, rows, per_cu; double alone, full; };
  constexpr Shape kBf16[] = {{2, 0, 64, 64, 2, 0.95, 1.6}, {4, 0, 64, 128, 2, 1.4, 2.2}, {8, 0, 64, 256, 1, 1.8, 2.1}};
  constexpr Shape kFp4[] = {{0, 1, 32, 32, 3, 0.5, 1.2}, {0, 2, 32, 64, 2, 0.75, 1.3}, {4, 0, 64, 128, 2, 1.4, 2.2}, {8, 0, 64, 256, 1, 1.9, 2.1}};
  constexpr Shape kF32[] = {{4, 0, 32, 16, 2, 2.0, 2.8}, {4, 0, 32, 32, 2, 3.2, 4.2}, {4, 0, 32, 64, 2, 7.0, 10.0}, {4, 0, 32, 128, 2, 13.0, 21.0}};
  const Shape* shapes = c.fp4 ? kFp4 : c.bf16 ? kBf16 : kF32;
  const double scale_d = c.d / 128.0;
  const double key_bytes = 2.0 * (c.fp4 ? c.d * 17.0 / 32.0 : c.bf16 ? 2.0 * c.d : 4.0 * c.d);
  const bool open = c.window == 0 || c.window >= c.max_q;   // the lengths matter to the rows' keys
  const double causal = open && c.n_new == 0 && c.mask_block > 0 && c.mask_block < c.max_q
                            ? 1.0 - 0.5 * std::min(c.max_q, c.max_kv) / std::max(c.max_kv, 1) : 1.0;
  const double even = (c.batch > 1 && c.window == 0 ? 0.7 : 1.0) * causal;
  const double part_us = 8.0 * (c.d + 2) * c.tokens * c.hq / 4e6;   // both ways at 4 TB/s
  const int64_t rows = int64_t{std::min(c.max_q, c.tokens)} * r.group;   // of the longest sequence
  int64_t chunk = 0;
  int per_cu = 1;
  double best = -1.0;
  for (int i = 0; i < (c.bf16 && !c.fp4 ? 3 : 4); ++i) {
    const Shape& sh = shapes[i];
    if (i > 0 && shapes[i - 1].rows >= rows) break;   // no sequence fills more than the smaller one
    const int64_t tiles = std::max<int64_t>(ceil_div(list_tiles(c, sh.rows, r.group, sh.tile) * sh.tile, kTile), 1);
    const double slots = static_cast<double>(sh.per_cu) * cus;
    const double filled = static_cast<double>(c.tokens) * r.group / c.batch / sh.rows;
    const double blocks = c.n_new > 0 ? std::ceil(filled) : c.batch > 1 ? std::max(filled + 0.5, 1.0) : std::ceil(filled);
    const double groups = blocks * c.batch * c.hkv;
    for (int64_t s = 1; s <= std::min<int64_t>(tiles, 64); s += s < 8 ? 1 : s < 16 ? 2 : s < 32 ? 4 : 8) {
      const int64_t t = ceil_div(tiles, s);
      const double x = groups * s / slots;
      const double cu = x <= 0.5 ? sh.alone : x <= 1.0 ? sh.alone + (sh.full - sh.alone) * (2.0 * x - 1.0) : sh.full;
      const double memory = kTile * key_bytes * std::min(x, 1.0) * slots / 5.5e6 / std::min(blocks, 8.0);
      const double one = t * std::max(cu * scale_d, memory);
      const double end = sh.few > 0 && c.window == 0 && c.batch <= 64 ? 0.1 : 0.35;
      const double start = sh.few == 2 ? 7.0 : 5.0;
      double us = x <= 1.0 ? one + 7.0 : even * x * (one + start) + end * (one + 7.0);
      if (s > 1) us += 5.0 + s * part_us;
      if (best < 0.0 || us < best) {
        best = us;
        chunk = t * kTile;
        r.row_waves = sh.row_waves;
        r.few = sh.few;
        r.tile = sh.tile;
        r.rows_pb = sh.rows;
        per_cu = sh.per_cu;
      }
    }
  }
  if (c.kv_chunk > 0) chunk = c.kv_chunk;
  chunk = std::min(chunk, most);
  r.chunk = static_cast<int>(chunk);
  const int64_t splits = std::max<int64_t>(1, ceil_div(list_tiles(c, r.rows_pb, r.group, r.tile) * r.tile, chunk));
  if (splits > 65535) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": too many key ranges");
  r.splits = static_cast<int>(splits);
  int64_t blocks;
  if (c.n_new > 0) {
    r.seq_blocks = static_cast<int>(ceil_div(int64_t{c.n_new} * r.group, r.rows_pb));
    blocks = int64_t{c.batch} * r.seq_blocks;
  } else {
    blocks = std::max<int64_t>(int64_t{c.tokens} * r.group - 1, 0) / r.rows_pb + c.batch;
  }
  if (blocks * c.hkv > (1 << 22))
    return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": too many tokens and sequences for one call");
  r.blocks = static_cast<int>(blocks);
  const int units = cus / c.hkv;
  if (r.splits == 1 && per_cu == 2 && c.batch <= 64 && c.n_new == 0 && c.window == 0 && r.blocks > units && r.blocks <= 2 * units)
    r.fold = units;                // (as the chunk attention deals its blocks out)
  if (r.splits > 1 && c.tokens > 0) {
    const size_t n = static_cast<size_t>(r.splits) * c.tokens * c.hq;
    r.ml_off = n * c.d * sizeof(float);
    r.workspace = r.ml_off + n * 2 * sizeof(float);
  }
  const float scale = c.scale > 0.f ? c.scale : 1.0f / std::sqrt(static_cast<float>(c.d));
  r.scale_log2 = scale * 1.4426950408889634f;
  *p = r;
  return SIMSD_OK;
}

static simsd_status check_window(const char* op, int window, int sinks, bool may) {
  if (window < 0 || sinks < 0) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": need window >= 0 and sinks >= 0");
  if (window == 0 && sinks > 0) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": sinks need a window");
  if (window > 0 && !may) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": a window needs mask_block >= 1");
  return SIMSD_OK;
}

static simsd_status check_code_strides(const char* op, int64_t seq, int64_t tok, int64_t head) {
  for (int64_t s : {seq, tok, head})
    if (s % 16 != 0) return fail(SIMSD_ERR_ALIGNMENT, std::string(op) + ": strides of a 4-bit cache must be multiples of 16 bytes");
  return SIMSD_OK;
}

static simsd_status plan_chunk_span(const char* op, const simsd_chunk_desc* d, int window, int sinks, bool fp4, int cus,
                                    SpanPlan* p) {
  if (!p) return fail(SIMSD_ERR_NULL_POINTER, std::string(op) + ": plan is NULL");
  ChunkPlan whole;
  simsd_chunk_desc same{};
  if (d) same = *d;
  same.kv_chunk = d && d->kv_chunk > 0 && d->kv_chunk % kTile == 0 ? 0 : same.kv_chunk;   // (a list's ranges are counted below)
  simsd_status st = plan_chunk(d ? &same : nullptr, cus, &whole);
  if (st == SIMSD_OK) st = check_window(op, window, sinks, d->mask_block >= 1);
  if (st != SIMSD_OK) return st;
  if (fp4) {
    if (d->dtype != SIMSD_BF16) return fail(SIMSD_ERR_UNSUPPORTED, std::string(op) + ": dtype must be SIMSD_BF16");
    st = check_code_strides(op, d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head);
    if (st != SIMSD_OK) return st;
  }
  Problem c{};
  c.tokens = d->num_tokens;
  c.batch = d->batch;
  c.hq = d->num_q_heads;
  c.hkv = d->num_kv_heads;
  c.d = d->head_dim;
  c.max_q = d->max_q_len;
  c.max_kv = d->max_kv_len;
  c.mask_block = d->mask_block;
  c.page_size = d->page_size;
  c.kv_chunk = d->kv_chunk;
  c.window = window;
  c.sinks = sinks;
  c.bf16 = d->dtype == SIMSD_BF16;
  c.fp4 = fp4;
  c.scale = d->scale;
  return plan(op, c, cus, p);
}

simsd_status plan_window(const simsd_chunk_desc* d, int window, int sinks, int cus, SpanPlan* p) {
  return plan_chunk_span("chunk_attention", d, window, sinks, false, cus, p);
}

simsd_status plan_chunk_fp4(const simsd_chunk_desc* d, int window, int sinks, int cus, SpanPlan* p) {
  return plan_chunk_span("chunk_attention_fp4", d, window, sinks, true, cus, p);
}

simsd_status plan_verify_span(const simsd_attn_desc* d, bool fp4, int window, int sinks, int cus, SpanPlan* p) {
  const char* op = fp4 ? "verify_attention_fp4" : "verify_attention";
  if (!p) return fail(SIMSD_ERR_NULL_POINTER, std::string(op) + ": plan is NULL");
  AttnPlan whole;
  simsd_status st = plan_attention(d, cus, &whole);
  if (st == SIMSD_OK) st = check_window(op, window, sinks, true);
  if (st != SIMSD_OK) return st;
  if (d->dtype != SIMSD_BF16) return fail(SIMSD_ERR_UNSUPPORTED, std::string(op) + ": dtype must be SIMSD_BF16");
  if (d->rope_theta != 0.f)
    return fail(SIMSD_ERR_UNSUPPORTED, std::string(op) + ": rope_theta must be 0 (turn q and k_new before)");
  if (d->kv_chunk < 0) return fail(SIMSD_ERR_UNSUPPORTED, std::string(op) + ": no stream decomposition (kv_chunk -1)");
  if (d->max_prefix_len > (1 << 30))
    return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": max_prefix_len must be <= 2^30");
  const int n_new = d->block_size + d->max_ref;
  if (int64_t{d->batch} * n_new > (1 << 23))
    return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": too many sequences for one call");
  if (fp4) {
    st = check_code_strides(op, d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head);
    if (st != SIMSD_OK) return st;
  }
  Problem c{};
  c.tokens = d->batch * n_new;
  c.batch = d->batch;
  c.hq = d->num_q_heads;
  c.hkv = d->num_kv_heads;
  c.d = d->head_dim;
  c.max_q = n_new;
  c.max_kv = d->max_prefix_len;
  c.mask_block = 1;
  c.page_size = d->page_size;
  c.kv_chunk = d->kv_chunk;
  c.window = window;
  c.sinks = sinks;
  c.n_new = n_new;
  c.bf16 = true;
  c.fp4 = fp4;
  c.scale = d->scale;
  return plan(op, c, cus, p);
}

simsd_status check_span_workspace(const char* op, const SpanPlan& p, const void* workspace, size_t workspace_bytes) {
  if (p.workspace == 0) return SIMSD_OK;
  if (!workspace) return fail(SIMSD_ERR_WORKSPACE, std::string(op) + ": workspace is NULL");
  if (!aligned(workspace, 16)) return fail(SIMSD_ERR_ALIGNMENT, std::string(op) + ": workspace must be 16-byte aligned");
  if (workspace_bytes < p.workspace)
    return fail(SIMSD_ERR_WORKSPACE, std::string(op) + ": workspace smaller than its workspace_size()");
  return SIMSD_OK;
}

simsd_status check_fp4_cache(const char* op, const simsd_fp4_cache* c, int max_len, int scales_to) {
  if (!c) return fail(SIMSD_ERR_NULL_POINTER, std::string(op) + ": cache is NULL");
  if (max_len > 0 && (!c->k || !c->v || !c->k_scales || !c->v_scales))
    return fail(SIMSD_ERR_NULL_POINTER, std::string(op) + ": the cache's codes and scales are required");
  if (!aligned(c->k, 16) || !aligned(c->v, 16))
    return fail(SIMSD_ERR_ALIGNMENT, std::string(op) + ": the cache's codes must be 16-byte aligned");
  if (!aligned(c->k_scales, scales_to) || !aligned(c->v_scales, scales_to))
    return fail(SIMSD_ERR_ALIGNMENT, std::string(op) + ": the cache's scales must be aligned to head_dim / 32 bytes");
  for (int64_t s : {c->scale_stride_seq, c->scale_stride_token, c->scale_stride_head}) {
    if (s < 0) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": negative stride of the scales");
    if (s > (int64_t{1} << 48)) return fail(SIMSD_ERR_BAD_SHAPE, std::string(op) + ": stride of the scales beyond 2^48 bytes");
    if (s % scales_to != 0) return fail(SIMSD_ERR_ALIGNMENT, std::string(op) + ": strides of the scales must be multiples of head_dim / 32");
  }
  return SIMSD_OK;
}

// Rows [tokens, heads] of `n` bytes that do not overlap, whichever index is outer.
static bool apart(__int128 tokens, __int128 heads, __int128 st, __int128 sh, __int128 n) {
  if (tokens < 1 || heads < 1) return true;
  const bool head_inner = (heads == 1 || sh >= n) && (tokens == 1 || st >= sh * (heads - 1) + n);
  const bool token_inner = (tokens == 1 || st >= n) && (heads == 1 || sh >= st * (tokens - 1) + n);
  return head_inner || token_inner;
}

simsd_status plan_fp4_append(const simsd_rotary_desc* d, const simsd_fp4_cache* c) {
  RotaryPlan whole;
  simsd_status st = plan_rotary(d, true, &whole);
  if (st != SIMSD_OK) return st;
  if (d->dtype != SIMSD_BF16) return fail(SIMSD_ERR_UNSUPPORTED, "rotary_append_fp4: dtype must be SIMSD_BF16");
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(SIMSD_ERR_UNSUPPORTED, "rotary_append_fp4: head_dim must be 64 or 128");
  st = check_code_strides("rotary_append_fp4", d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head);
  if (st == SIMSD_OK) st = check_fp4_cache("rotary_append_fp4", c, d->num_tokens > 0 ? d->max_kv_len : 0, d->head_dim / 32);
  if (st != SIMSD_OK) return st;
  const int64_t tokens = d->page_size > 0 ? d->page_size : d->max_kv_len;
  if (!apart(tokens, d->num_kv_heads, d->cache_stride_token, d->cache_stride_head, d->head_dim / 2) ||
      !apart(tokens, d->num_kv_heads, c->scale_stride_token, c->scale_stride_head, d->head_dim / 32))
    return fail(SIMSD_ERR_BAD_SHAPE, "rotary_append_fp4: rows of the cache overlap");
  return SIMSD_OK;
}

simsd_status check_fp4_values(const simsd_fp4_values_desc* d, const simsd_fp4_cache* c, const void* k_out, const void* v_out) {
  if (!d) return fail(SIMSD_ERR_NULL_POINTER, "fp4_values: descriptor is NULL");
  if (d->num < 0 || d->tokens < 0 || d->num_kv_heads < 0)
    return fail(SIMSD_ERR_BAD_SHAPE, "fp4_values: need num, tokens and num_kv_heads >= 0");
  if (static_cast<__int128>(d->num) * d->tokens * d->num_kv_heads > (int64_t{1} << 36))
    return fail(SIMSD_ERR_BAD_SHAPE, "fp4_values: num * tokens * num_kv_heads must be <= 2^36");
  if (d->head_dim < 32 || d->head_dim > 512 || d->head_dim % 32 != 0)
    return fail(SIMSD_ERR_UNSUPPORTED, "fp4_values: head_dim must be a multiple of 32 in [32, 512]");
  // (A launch has fewer than 2^32 threads; 256 of them take 8192 elements.)
  if (int64_t{d->num} * d->tokens * d->num_kv_heads * d->head_dim > (int64_t{1} << 37) - 8192)
    return fail(SIMSD_ERR_BAD_SHAPE, "fp4_values: num * tokens * num_kv_heads * head_dim must be <= 2^37 - 8192");
  for (int64_t s : {d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head}) {
    if (s < 0) return fail(SIMSD_ERR_BAD_SHAPE, "fp4_values: negative stride");
    if (s > (int64_t{1} << 48)) return fail(SIMSD_ERR_BAD_SHAPE, "fp4_values: stride beyond 2^48 bytes");
  }
  simsd_status st = check_code_strides("fp4_values", d->cache_stride_seq, d->cache_stride_token, d->cache_stride_head);
  const bool some = d->num > 0 && d->tokens > 0 && d->num_kv_heads > 0;
  if (st == SIMSD_OK) st = check_fp4_cache("fp4_values", c, some, 1);
  if (st != SIMSD_OK || !some) return st;
  if (!k_out && !v_out) return fail(SIMSD_ERR_NULL_POINTER, "fp4_values: k_out or v_out is required");
  if (k_out == v_out) return fail(SIMSD_ERR_BAD_SHAPE, "fp4_values: k_out and v_out must not be the same");
  if (!aligned(k_out, 16) || !aligned(v_out, 16))
    return fail(SIMSD_ERR_ALIGNMENT, "fp4_values: k_out and v_out must be 16-byte aligned");
  return SIMSD_OK;
}

}  // namespace simsd
