// extern "C" entry points of the operators beside the verification step:
// check, plan, fill the argument block, launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "simsd.h"
#include "simsd_kernels.h"
#include "simsd_ops_kernels.h"
#include "simsd_ops_plan.h"

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

static RotaryArgs rotary_args(const simsd_rotary_desc* d, const RotaryPlan& p) {
  RotaryArgs a{};
  a.tokens = d->num_tokens;
  a.hq = d->num_q_heads;
  a.hkv = d->num_kv_heads;
  a.d = d->head_dim;
  a.rot = d->rotary_dim;
  a.q_tok = d->q_stride_token;
  a.q_head = d->q_stride_head;
  a.k_tok = d->k_stride_token;
  a.k_head = d->k_stride_head;
  a.v_tok = d->v_stride_token;
  a.v_head = d->v_stride_head;
  a.qo_tok = d->q_out_stride_token;
  a.qo_head = d->q_out_stride_head;
  a.ko_tok = d->k_out_stride_token;
  a.ko_head = d->k_out_stride_head;
  a.cs_seq = d->cache_stride_seq;
  a.cs_tok = d->cache_stride_token;
  a.cs_head = d->cache_stride_head;
  a.batch = d->batch;
  a.page_size = d->page_size;
  a.max_pages = d->max_pages_per_seq;
  a.num_pages = d->num_pages;
  a.max_kv = d->max_kv_len;
  a.q_units = p.q_units;
  a.v_units = p.v_units;
  a.units = p.units;
  a.factor = d->attn_factor;
  return a;
}

extern "C" simsd_status simsd_rotary(const simsd_rotary_desc* desc, const void* q, const void* k,
                                     const int32_t* positions, const double* freq, void* q_out,
                                     void* k_out, void* stream) {
  try {
    RotaryPlan p;
    simsd_status st = plan_rotary(desc, false, &p);
    if (st == SIMSD_OK) st = check_rotary_args(desc, q, k, positions, freq, q_out, k_out);
    if (st != SIMSD_OK || desc->num_tokens == 0) return st;
    int dev = 0, cus = 0;
    const hipError_t qe = stream_device(stream, &dev, &cus);
    if (qe != hipSuccess) return hip_fail(qe, "simsd_rotary: device query");
    RotaryArgs a = rotary_args(desc, p);
    a.q = q;
    a.k = k;
    a.positions = positions;
    a.freq = freq;
    a.q_out = q_out;
    a.k_out = k_out;
    const hipError_t e = launch_rotary(*desc, p, a, false, cus, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "simsd_rotary launch");
    return SIMSD_OK;
  } catch (...) {
    return internal_error("simsd_rotary");
  }
}

extern "C" simsd_status simsd_rotary_append(const simsd_rotary_desc* desc, const void* q,
                                            const void* k, const void* v, const int32_t* positions,
                                            const double* freq, void* q_out, void* k_cache,
                                            void* v_cache, const int32_t* block_table,
                                            const int32_t* q_starts, const int32_t* kv_lens,
                                            void* stream) {
  try {
    RotaryPlan p;
    simsd_status st = plan_rotary(desc, true, &p);
    if (st == SIMSD_OK)
      st = check_rotary_append_args(desc, q, k, v, positions, freq, q_out, k_cache, v_cache, block_table,
                                    q_starts, kv_lens);
    if (st != SIMSD_OK || desc->num_tokens == 0) return st;
    int dev = 0, cus = 0;
    const hipError_t qe = stream_device(stream, &dev, &cus);
    if (qe != hipSuccess) return hip_fail(qe, "simsd_rotary_append: device query");
    RotaryArgs a = rotary_args(desc, p);
    a.q = q;
    a.k = k;
    a.v = v;
    a.positions = positions;
    a.freq = freq;
    a.q_out = q_out;
    a.k_out = k_cache;
    a.v_out = v_cache;
    a.block_table = block_table;
    a.q_starts = q_starts;
    a.kv_lens = kv_lens;
    const hipError_t e = launch_rotary(*desc, p, a, true, cus, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "simsd_rotary_append launch");
    return SIMSD_OK;
  } catch (...) {
    return internal_error("simsd_rotary_append");
  }
}

extern "C" size_t simsd_chunk_attention_workspace_size(const simsd_chunk_desc* desc) {
  try {
    ChunkPlan p;
    return plan_chunk(desc, current_cus(), &p) == SIMSD_OK ? p.workspace : 0;
  } catch (...) {
    return 0;
  }
}

extern "C" simsd_status simsd_chunk_attention(const simsd_chunk_desc* desc, const void* q,
                                              const void* k_cache, const void* v_cache,
                                              const int32_t* block_table, const int32_t* q_starts,
                                              const int32_t* kv_lens, void* out, float* lse,
                                              void* workspace, size_t workspace_bytes, void* stream) {
  try {
    int dev = 0, cus = 0;
    const hipError_t qe = stream_device(stream, &dev, &cus);
    ChunkPlan p;
    simsd_status st = plan_chunk(desc, cus, &p);
    if (st == SIMSD_OK)
      st = check_chunk_args(desc, p, q, k_cache, v_cache, block_table, q_starts, kv_lens, out, lse,
                            workspace, workspace_bytes);
    if (st != SIMSD_OK || desc->num_tokens == 0) return st;
    if (qe != hipSuccess) return hip_fail(qe, "simsd_chunk_attention: device query");
    ChunkArgs a{};
    a.q = q;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.block_table = desc->page_size > 0 ? block_table : nullptr;
    a.q_starts = q_starts;
    a.kv_lens = kv_lens;
    a.out = out;
    a.lse = lse;
    a.part = static_cast<float*>(workspace);
    a.part_ml = p.workspace ? reinterpret_cast<float2*>(static_cast<char*>(workspace) + p.ml_off) : nullptr;
    a.cs_seq = desc->cache_stride_seq;
    a.cs_tok = desc->cache_stride_token;
    a.cs_head = desc->cache_stride_head;
    a.tokens = desc->num_tokens;
    a.batch = desc->batch;
    a.hq = desc->num_q_heads;
    a.hkv = desc->num_kv_heads;
    a.group = p.group;
    a.max_kv = desc->max_kv_len;
    // (A block past the longest cache is the whole cache; sums of it and a position
    // stay in 32 bits.)
    a.mask_block = std::min(desc->mask_block, std::max(desc->max_kv_len, 1));
    a.page_size = std::max(desc->page_size, 1);
    a.page_shift = (a.page_size & (a.page_size - 1)) == 0 ? __builtin_ctz(a.page_size) : -1;
    a.max_pages = desc->max_pages_per_seq;
    a.rows_pb = p.rows_pb;
    a.blocks = p.blocks;
    a.fold = p.fold;
    a.chunk = p.chunk;
    a.scale_log2 = p.scale_log2;
    const hipError_t e = launch_chunk(*desc, p, a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "simsd_chunk_attention launch");
    return SIMSD_OK;
  } catch (...) {
    return internal_error("simsd_chunk_attention");
  }
}

extern "C" simsd_status simsd_sample(const simsd_sample_desc* desc, const void* logits,
                                     const float* uniforms, const float* temperatures,
                                     const int32_t* top_ks, const float* top_ps, const float* min_ps,
                                     int32_t* token, float* prob, int32_t* kept, void* stream) {
  try {
    SampleArgs a{};
    simsd_status st = plan_sample(desc, &a.one);
    if (st == SIMSD_OK)
      st = check_sample_args(desc, logits, uniforms, temperatures, top_ks, top_ps, min_ps, token, prob, kept);
    if (st != SIMSD_OK || desc->rows == 0) return st;
    a.logits = logits;
    a.uniforms = uniforms;
    a.temperatures = temperatures;
    a.top_ks = top_ks;
    a.top_ps = top_ps;
    a.min_ps = min_ps;
    a.token = token;
    a.prob = prob;
    a.kept = kept;
    a.V = desc->vocab;
    a.temperature = desc->temperature;
    a.top_p = desc->top_p;
    a.min_p = desc->min_p;
    a.top_k = desc->top_k;
    const hipError_t e = launch_sample(*desc, a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "simsd_sample launch");
    return SIMSD_OK;
  } catch (...) {
    return internal_error("simsd_sample");
  }
}
