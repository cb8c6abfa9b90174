// extern "C" entry points of attention over a list of tiles and of the 4-bit cache:
// check, plan, fill the argument block, launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "simsd.h"
#include "simsd_kernels.h"
#include "simsd_ops_kernels.h"
#include "simsd_span_plan.h"

using namespace simsd;

static simsd_status hip_fail(hipError_t e, const char* what) {
  set_error(std::string(what) + ": " + hipGetErrorString(e));
  return SIMSD_ERR_HIP;
}

// What an entry returns where an exception ends it (no memory for a message, say).
static simsd_status internal_error(const char* what) noexcept {
  try {
    set_error(std::string(what) + ": internal error");
  } catch (...) {
  }
  return SIMSD_ERR_HIP;
}

static void set_plan(const SpanPlan& p, int page_size, int max_pages, const int32_t* block_table, void* workspace,
                     SpanArgs* a) {
  a->block_table = page_size > 0 ? block_table : nullptr;
  a->page_size = std::max(page_size, 1);
  a->page_shift = (a->page_size & (a->page_size - 1)) == 0 ? __builtin_ctz(a->page_size) : -1;
  a->max_pages = max_pages;
  a->part = static_cast<float*>(workspace);
  a->part_ml = p.workspace ? reinterpret_cast<float2*>(static_cast<char*>(workspace) + p.ml_off) : nullptr;
  a->group = p.group;
  a->rows_pb = p.rows_pb;
  a->seq_blocks = p.seq_blocks;
  a->blocks = p.blocks;
  a->fold = p.fold;
  a->chunk = p.chunk;
  a->window = p.window;
  a->sinks = p.sinks;
  a->scale_log2 = p.scale_log2;
}

static void set_fp4(const simsd_fp4_cache* c, int64_t seq, int64_t tok, SpanArgs* a) {
  a->k_cache = c->k;
  a->v_cache = c->v;
  a->k_scales = static_cast<const uint8_t*>(c->k_scales);
  a->v_scales = static_cast<const uint8_t*>(c->v_scales);
  a->ss_seq = c->scale_stride_seq;
  a->ss_tok = c->scale_stride_token;
  a->ss_head = c->scale_stride_head;
  a->scales_alike = seq == 16 * c->scale_stride_seq && tok == 16 * c->scale_stride_token && seq < (int64_t{1} << 31) &&
                    tok < (int64_t{1} << 31);
}

// ----------------------------------------------------------------------------
// A chunk of new tokens
// ----------------------------------------------------------------------------
static size_t chunk_workspace(const simsd_chunk_desc* desc, int32_t window, int32_t sinks, bool fp4) {
  try {
    SpanPlan p;
    const int cus = current_cus();
    const simsd_status st = fp4 ? plan_chunk_fp4(desc, window, sinks, cus, &p) : plan_window(desc, window, sinks, cus, &p);
    if (st == SIMSD_OK && !fp4 && p.window == 0) return simsd_chunk_attention_workspace_size(desc);
    return st == SIMSD_OK ? p.workspace : 0;
  } catch (...) {
    return 0;
  }
}

static simsd_status chunk_span(const char* op, const simsd_chunk_desc* desc, int32_t window, int32_t sinks, const void* q,
                               const void* k_cache, const void* v_cache, const simsd_fp4_cache* cache, bool fp4,
                               const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, void* out,
                               float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int dev = 0, cus = 0;
  const hipError_t qe = stream_device(stream, &dev, &cus);
  SpanPlan p;
  simsd_status st = fp4 ? plan_chunk_fp4(desc, window, sinks, cus, &p) : plan_window(desc, window, sinks, cus, &p);
  if (st == SIMSD_OK && !fp4 && p.window == 0)   // (it reaches past every cache)
    return simsd_chunk_attention(desc, q, k_cache, v_cache, block_table, q_starts, kv_lens, out, lse, workspace,
                                 workspace_bytes, stream);
  if (st == SIMSD_OK && fp4) st = check_fp4_cache(op, cache, desc->num_tokens > 0 ? desc->max_kv_len : 0, desc->head_dim / 32);
  if (st == SIMSD_OK) {
    ChunkPlan none;                // (the workspace is this plan's)
    st = check_chunk_args(desc, none, q, fp4 ? cache->k : k_cache, fp4 ? cache->v : v_cache, block_table, q_starts, kv_lens,
                          out, lse, nullptr, 0);
  }
  if (st != SIMSD_OK || desc->num_tokens == 0) return st;
  st = check_span_workspace(op, p, workspace, workspace_bytes);
  if (st != SIMSD_OK) return st;
  if (qe != hipSuccess) return hip_fail(qe, op);
  SpanArgs a{};
  a.q = q;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  if (fp4) set_fp4(cache, desc->cache_stride_seq, desc->cache_stride_token, &a);
  a.q_starts = q_starts;
  a.kv_lens = kv_lens;
  a.out = out;
  a.lse = lse;
  a.cs_seq = desc->cache_stride_seq;
  a.cs_tok = desc->cache_stride_token;
  a.cs_head = desc->cache_stride_head;
  a.tokens = desc->num_tokens;
  a.batch = desc->batch;
  a.hq = desc->num_q_heads;
  a.hkv = desc->num_kv_heads;
  a.max_kv = desc->max_kv_len;
  a.mask_block = std::min(desc->mask_block, std::max(desc->max_kv_len, 1));
  set_plan(p, desc->page_size, desc->max_pages_per_seq, block_table, workspace, &a);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = fp4 ? launch_fp4(p, desc->head_dim, a, s) : launch_window(p, desc->dtype == SIMSD_BF16, desc->head_dim, a, s);
  return e == hipSuccess ? SIMSD_OK : hip_fail(e, op);
}

extern "C" size_t simsd_chunk_attention_window_workspace_size(const simsd_chunk_desc* desc, int32_t window, int32_t sinks) {
  return chunk_workspace(desc, window, sinks, false);
}

extern "C" simsd_status simsd_chunk_attention_window(const simsd_chunk_desc* desc, int32_t window, int32_t sinks,
                                                     const void* q, const void* k_cache, const void* v_cache,
                                                     const int32_t* block_table, const int32_t* q_starts,
                                                     const int32_t* kv_lens, void* out, float* lse, void* workspace,
                                                     size_t workspace_bytes, void* stream) {
  try {
    return chunk_span("simsd_chunk_attention_window", desc, window, sinks, q, k_cache, v_cache, nullptr, false, block_table,
                      q_starts, kv_lens, out, lse, workspace, workspace_bytes, stream);
  } catch (...) {
    return internal_error("simsd_chunk_attention_window");
  }
}

extern "C" size_t simsd_chunk_attention_fp4_workspace_size(const simsd_chunk_desc* desc, int32_t window, int32_t sinks) {
  return chunk_workspace(desc, window, sinks, true);
}

extern "C" simsd_status simsd_chunk_attention_fp4(const simsd_chunk_desc* desc, int32_t window, int32_t sinks, const void* q,
                                                  const simsd_fp4_cache* cache, const int32_t* block_table,
                                                  const int32_t* q_starts, const int32_t* kv_lens, void* out, float* lse,
                                                  void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return chunk_span("simsd_chunk_attention_fp4", desc, window, sinks, q, nullptr, nullptr, cache, true, block_table,
                      q_starts, kv_lens, out, lse, workspace, workspace_bytes, stream);
  } catch (...) {
    return internal_error("simsd_chunk_attention_fp4");
  }
}

// ----------------------------------------------------------------------------
// The verification step
// ----------------------------------------------------------------------------
static size_t verify_workspace(const simsd_attn_desc* desc, bool fp4, int32_t window, int32_t sinks) {
  try {
    SpanPlan p;
    return plan_verify_span(desc, fp4, window, sinks, current_cus(), &p) == SIMSD_OK ? p.workspace : 0;
  } catch (...) {
    return 0;
  }
}

static simsd_status verify_span(const char* op, const simsd_attn_desc* desc, int32_t window, int32_t sinks, const void* q,
                                const void* k_new, const void* v_new, const void* k_cache, const void* v_cache,
                                const simsd_fp4_cache* cache, bool fp4, const int32_t* block_table,
                                const int32_t* prefix_lens, const int32_t* step_map, const int32_t* num_ref, void* out,
                                float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int dev = 0, cus = 0;
  const hipError_t qe = stream_device(stream, &dev, &cus);
  SpanPlan p;
  simsd_status st = plan_verify_span(desc, fp4, window, sinks, cus, &p);
  if (st == SIMSD_OK && fp4) st = check_fp4_cache(op, cache, desc->max_prefix_len, desc->head_dim / 32);
  if (st == SIMSD_OK) {
    AttnPlan none;                 // (the workspace is this plan's)
    st = check_attention_args(desc, none, q, k_new, v_new, fp4 ? cache->k : k_cache, fp4 ? cache->v : v_cache, block_table,
                              prefix_lens, step_map, num_ref, out, lse, nullptr, 0);
  }
  for (const int32_t* words : {block_table, prefix_lens, step_map, num_ref})
    if (st == SIMSD_OK && (reinterpret_cast<uintptr_t>(words) & 3u)) {
      set_error(std::string(op) + ": int32 arrays must be 4-byte aligned");
      st = SIMSD_ERR_ALIGNMENT;
    }
  if (st == SIMSD_OK) st = check_span_workspace(op, p, workspace, workspace_bytes);
  if (st != SIMSD_OK) return st;
  if (qe != hipSuccess) return hip_fail(qe, op);
  SpanArgs a{};
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  if (fp4) set_fp4(cache, desc->cache_stride_seq, desc->cache_stride_token, &a);
  a.kv_lens = prefix_lens;
  a.step_map = step_map;
  a.num_ref = num_ref;
  a.out = out;
  a.lse = lse;
  a.cs_seq = desc->cache_stride_seq;
  a.cs_tok = desc->cache_stride_token;
  a.cs_head = desc->cache_stride_head;
  a.block = desc->block_size;
  a.n_new = desc->block_size + desc->max_ref;
  a.tokens = desc->batch * a.n_new;
  a.batch = desc->batch;
  a.hq = desc->num_q_heads;
  a.hkv = desc->num_kv_heads;
  a.max_kv = desc->max_prefix_len;
  a.mask_block = 1;
  set_plan(p, desc->page_size, desc->max_pages_per_seq, block_table, workspace, &a);
  const hipError_t e = launch_verify_span(p, fp4, desc->head_dim, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SIMSD_OK : hip_fail(e, op);
}

extern "C" size_t simsd_verify_attention_window_workspace_size(const simsd_attn_desc* desc, int32_t window, int32_t sinks) {
  return verify_workspace(desc, false, window, sinks);
}

extern "C" simsd_status simsd_verify_attention_window(const simsd_attn_desc* desc, int32_t window, int32_t sinks,
                                                      const void* q, const void* k_new, const void* v_new,
                                                      const void* k_cache, const void* v_cache,
                                                      const int32_t* block_table, const int32_t* prefix_lens,
                                                      const int32_t* step_map, const int32_t* num_ref, void* out,
                                                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return verify_span("simsd_verify_attention_window", desc, window, sinks, q, k_new, v_new, k_cache, v_cache, nullptr,
                       false, block_table, prefix_lens, step_map, num_ref, out, lse, workspace, workspace_bytes, stream);
  } catch (...) {
    return internal_error("simsd_verify_attention_window");
  }
}

extern "C" size_t simsd_verify_attention_fp4_workspace_size(const simsd_attn_desc* desc, int32_t window, int32_t sinks) {
  return verify_workspace(desc, true, window, sinks);
}

extern "C" simsd_status simsd_verify_attention_fp4(const simsd_attn_desc* desc, int32_t window, int32_t sinks, const void* q,
                                                   const void* k_new, const void* v_new, const simsd_fp4_cache* cache,
                                                   const int32_t* block_table, const int32_t* prefix_lens,
                                                   const int32_t* step_map, const int32_t* num_ref, void* out, float* lse,
                                                   void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return verify_span("simsd_verify_attention_fp4", desc, window, sinks, q, k_new, v_new, nullptr, nullptr, cache, true,
                       block_table, prefix_lens, step_map, num_ref, out, lse, workspace, workspace_bytes, stream);
  } catch (...) {
    return internal_error("simsd_verify_attention_fp4");
  }
}

// ----------------------------------------------------------------------------
// Filling a 4-bit cache, and reading it back
// ----------------------------------------------------------------------------
extern "C" simsd_status simsd_rotary_append_fp4(const simsd_rotary_desc* desc, const void* q, const void* k, const void* v,
                                                const int32_t* positions, const double* freq, void* q_out,
                                                const simsd_fp4_cache* cache, const int32_t* block_table,
                                                const int32_t* q_starts, const int32_t* kv_lens, void* stream) {
  try {
    simsd_status st = plan_fp4_append(desc, cache);
    if (st == SIMSD_OK)
      st = check_rotary_append_args(desc, q, k, v, positions, freq, q_out, cache->k, cache->v, block_table, q_starts, kv_lens);
    if (st != SIMSD_OK || desc->num_tokens == 0) return st;
    int dev = 0, cus = 0;
    const hipError_t qe = stream_device(stream, &dev, &cus);
    if (qe != hipSuccess) return hip_fail(qe, "simsd_rotary_append_fp4: device query");
    // The queries' part: the append without keys.
    simsd_rotary_desc queries = *desc;
    queries.num_kv_heads = 0;
    queries.k_out_stride_token = queries.k_out_stride_head = 0;
    RotaryPlan p;
    st = plan_rotary(&queries, false, &p);
    if (st != SIMSD_OK) return st;
    Fp4AppendArgs f{};
    f.r.tokens = desc->num_tokens;
    f.r.hq = desc->num_q_heads;
    f.r.d = desc->head_dim;
    f.r.rot = desc->rotary_dim;
    f.r.q_tok = desc->q_stride_token;
    f.r.q_head = desc->q_stride_head;
    f.r.k_tok = desc->k_stride_token;
    f.r.k_head = desc->k_stride_head;
    f.r.v_tok = desc->v_stride_token;
    f.r.v_head = desc->v_stride_head;
    f.r.qo_tok = desc->q_out_stride_token;
    f.r.qo_head = desc->q_out_stride_head;
    f.r.cs_seq = desc->cache_stride_seq;
    f.r.cs_tok = desc->cache_stride_token;
    f.r.cs_head = desc->cache_stride_head;
    f.r.batch = desc->batch;
    f.r.page_size = desc->page_size;
    f.r.max_pages = desc->max_pages_per_seq;
    f.r.num_pages = desc->num_pages;
    f.r.max_kv = desc->max_kv_len;
    f.r.q_units = p.q_units;
    f.r.units = p.units;
    f.r.factor = desc->attn_factor;
    f.r.q = q;
    f.r.k = k;
    f.r.v = v;
    f.r.positions = positions;
    f.r.freq = freq;
    f.r.q_out = q_out;
    f.r.k_out = cache->k;
    f.r.v_out = cache->v;
    f.r.block_table = block_table;
    f.r.q_starts = q_starts;
    f.r.kv_lens = kv_lens;
    f.hkv = desc->num_kv_heads;
    f.k_scales = static_cast<uint8_t*>(cache->k_scales);
    f.v_scales = static_cast<uint8_t*>(cache->v_scales);
    f.ss_seq = cache->scale_stride_seq;
    f.ss_tok = cache->scale_stride_token;
    f.ss_head = cache->scale_stride_head;
    const hipError_t e = launch_fp4_append(f, desc->interleaved != 0, cus, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SIMSD_OK : hip_fail(e, "simsd_rotary_append_fp4 launch");
  } catch (...) {
    return internal_error("simsd_rotary_append_fp4");
  }
}

extern "C" simsd_status simsd_fp4_values(const simsd_fp4_values_desc* desc, const simsd_fp4_cache* cache, void* k_out,
                                         void* v_out, void* stream) {
  try {
    const simsd_status st = check_fp4_values(desc, cache, k_out, v_out);
    if (st != SIMSD_OK) return st;
    Fp4Args a{};
    a.rows = int64_t{desc->num} * desc->tokens * desc->num_kv_heads;
    if (a.rows == 0) return SIMSD_OK;
    int dev = 0, cus = 0;
    const hipError_t qe = stream_device(stream, &dev, &cus);
    if (qe != hipSuccess) return hip_fail(qe, "simsd_fp4_values: device query");
    a.k = cache->k;
    a.v = cache->v;
    a.k_scales = static_cast<const uint8_t*>(cache->k_scales);
    a.v_scales = static_cast<const uint8_t*>(cache->v_scales);
    a.k_out = k_out;
    a.v_out = v_out;
    a.c0 = desc->cache_stride_seq;
    a.c1 = desc->cache_stride_token;
    a.c2 = desc->cache_stride_head;
    a.s0 = cache->scale_stride_seq;
    a.s1 = cache->scale_stride_token;
    a.s2 = cache->scale_stride_head;
    a.n1 = desc->tokens;
    a.n2 = desc->num_kv_heads;
    a.groups = desc->head_dim / 32;
    const hipError_t e = launch_fp4_values(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SIMSD_OK : hip_fail(e, "simsd_fp4_values launch");
  } catch (...) {
    return internal_error("simsd_fp4_values");
  }
}
