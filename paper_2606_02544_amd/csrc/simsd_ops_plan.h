// Planning and argument checking of the operators beside the verification step
// (rotary positions, chunk attention, sampling).  Pure host C++ (no HIP).
#pragma once

#include <cstddef>
#include <cstdint>

#include "simsd.h"

namespace simsd {

// Rotary: how a call's kernel walks its rows.
struct RotaryPlan {
  int vec = 1;        // elements a load: 16 bytes, or 1 where the pairs' halves are no whole vectors
  int q_units = 0;    // loads (or pairs of loads) of one query or key head
  int v_units = 0;    // loads of one value head
  int units = 0;      // of one token
};

simsd_status plan_rotary(const simsd_rotary_desc* d, bool append, RotaryPlan* p);
simsd_status check_rotary_args(const simsd_rotary_desc* d, const void* q, const void* k,
                               const int32_t* positions, const double* freq, const void* q_out,
                               const void* k_out);
simsd_status check_rotary_append_args(const simsd_rotary_desc* d, const void* q, const void* k,
                                      const void* v, const int32_t* positions,
                                      const double* freq, const void* q_out,
                                      const void* k_cache, const void* v_cache,
                                      const int32_t* block_table, const int32_t* q_starts,
                                      const int32_t* kv_lens);

// Chunk attention.
struct ChunkPlan {
  int group = 0;        // Hq / Hkv
  int row_waves = 0;    // bf16: waves that own distinct rows (32 each)
  int rows_pb = 0;      // rows per work-group
  int blocks = 0;       // row-block numbers: floor((num_tokens * group - 1) / rows_pb) + batch
  int fold = 0;         // blocks that start first where the others share their CUs; 0: all the same
  int chunk = 0;        // keys per work-group
  int splits = 0;       // ceil(max_kv_len / chunk), >= 1
  size_t ml_off = 0;    // workspace offset (bytes) of the partial maxima and sums
  size_t workspace = 0;
  float scale_log2 = 0.f;
};

// `cus`: compute units of the device the call runs on, >= 1.
simsd_status plan_chunk(const simsd_chunk_desc* d, int cus, ChunkPlan* p);
simsd_status check_chunk_args(const simsd_chunk_desc* d, const ChunkPlan& p, const void* q,
                              const void* k_cache, const void* v_cache, const int32_t* block_table,
                              const int32_t* q_starts, const int32_t* kv_lens, const void* out,
                              const float* lse, const void* workspace, size_t workspace_bytes);

// Sampling: the fixed-point weights' unit (2^S).
simsd_status plan_sample(const simsd_sample_desc* d, double* one);
simsd_status check_sample_args(const simsd_sample_desc* d, const void* logits, const float* uniforms,
                               const float* temperatures, const int32_t* top_ks, const float* top_ps,
                               const float* min_ps, const int32_t* token, const float* prob,
                               const int32_t* kept);

}  // namespace simsd
