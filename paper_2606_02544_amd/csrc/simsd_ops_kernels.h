// Argument blocks and launch entry points of the operators beside the
// verification step.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "simsd_ops_plan.h"

namespace simsd {

struct RotaryArgs {
  const void* q;
  const void* k;
  const void* v;            // append only
  const int32_t* positions; // may be null (append: the cache index)
  const double* freq;
  void* q_out;
  void* k_out;              // rotary: the turned keys; append: the key cache
  void* v_out;              // append: the value cache
  const int32_t* block_table;
  const int32_t* q_starts;  // append only
  const int32_t* kv_lens;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, qo_tok, qo_head, ko_tok, ko_head;
  int64_t cs_seq, cs_tok, cs_head;
  int tokens, hq, hkv, d, rot, batch, page_size, max_pages, num_pages, max_kv;
  int q_units, v_units, units;
  float factor;
};

struct ChunkArgs {
  const void* q;
  const void* k_cache;
  const void* v_cache;
  const int32_t* block_table;   // null: contiguous
  const int32_t* q_starts;
  const int32_t* kv_lens;
  void* out;
  float* lse;
  float* part;                  // split partials (workspace)
  float2* part_ml;
  int64_t cs_seq, cs_tok, cs_head;
  int tokens, batch, hq, hkv, group, mask_block, max_kv, page_size, page_shift, max_pages;
  int rows_pb, blocks, fold, chunk;
  float scale_log2;
};

hipError_t launch_chunk(const simsd_chunk_desc& d, const ChunkPlan& p, const ChunkArgs& a,
                        hipStream_t stream);

struct SampleArgs {
  const void* logits;
  const float* uniforms;
  const float* temperatures;   // per-row parameters, or null
  const int32_t* top_ks;
  const float* top_ps;
  const float* min_ps;
  int32_t* token;
  float* prob;
  int32_t* kept;
  int V;
  float temperature, top_p, min_p;
  int top_k;
  double one;                  // the fixed-point unit of the weights
};

hipError_t launch_sample(const simsd_sample_desc& d, const SampleArgs& a, hipStream_t stream);
hipError_t launch_rotary(const simsd_rotary_desc& d, const RotaryPlan& p, const RotaryArgs& a,
                         bool append, int cus, hipStream_t stream);

}  // namespace simsd
