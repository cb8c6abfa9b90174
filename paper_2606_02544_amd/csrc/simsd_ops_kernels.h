// Argument blocks and launch entry points of the operators beside the
// verification step.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "simsd_ops_plan.h"
#include "simsd_span_plan.h"

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

// Attention over the cache under a sliding window with sinks, over a 4-bit cache, and
// of the verification step's new slots.  `chunk` is a multiple of a tile's keys.
struct SpanArgs : ChunkArgs {
  int window, sinks;            // window 0: none
  const uint8_t* k_scales;      // 4-bit cache
  const uint8_t* v_scales;
  int64_t ss_seq, ss_tok, ss_head;
  int scales_alike;             // strides of the codes: 16 times the scales', below 2^31
  const void* k_new;            // verification: kv_lens counts the cached prefix alone
  const void* v_new;
  const int32_t* step_map;
  const int32_t* num_ref;
  int block, n_new, seq_blocks; // B, B + L, row blocks of a sequence
};

hipError_t launch_window(const SpanPlan& p, bool bf16, int d, const SpanArgs& a, hipStream_t stream);
hipError_t launch_fp4(const SpanPlan& p, int d, const SpanArgs& a, hipStream_t stream);
hipError_t launch_verify_span(const SpanPlan& p, bool fp4, int d, const SpanArgs& a, hipStream_t stream);

struct Fp4Args {
  const void* k;                // codes [n0, n1, n2, d / 2]
  const void* v;
  const uint8_t* k_scales;      // [n0, n1, n2, d / 32]
  const uint8_t* v_scales;
  void* k_out;                  // each may be null
  void* v_out;
  int64_t c0, c1, c2, s0, s1, s2;
  int64_t rows;                 // n0 * n1 * n2
  int n1, n2, groups;
};
hipError_t launch_fp4_values(const Fp4Args& a, hipStream_t stream);

// The append to a 4-bit cache.  `r` is the append of the queries alone (no KV heads), with
// the keys and values and, in k_out and v_out, the cache's codes.
struct Fp4AppendArgs {
  RotaryArgs r;
  int hkv;
  uint8_t* k_scales;
  uint8_t* v_scales;
  int64_t ss_seq, ss_tok, ss_head;
};
hipError_t launch_fp4_append(const Fp4AppendArgs& a, bool interleaved, int cus, hipStream_t stream);

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
