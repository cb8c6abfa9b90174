// Planning and argument checking of attention over a list of tiles (a sliding window
// with sinks, a 4-bit cache, the verification step over either) and of the 4-bit cache's
// own operators.  Pure host C++ (no HIP).
#pragma once

#include <cstddef>
#include <cstdint>

#include "simsd.h"

namespace simsd {

struct SpanPlan {
  int group = 0;        // Hq / Hkv
  int row_waves = 0;    // bf16: waves that own distinct rows (32 each)
  int few = 0;          // 4 bits, few rows: 32-row blocks that every wave holds (then no row waves)
  int tile = 0;         // keys of a tile of the list
  int rows_pb = 0;      // rows per work-group
  int seq_blocks = 0;   // verification: row blocks of a sequence
  int blocks = 0;       // row-block numbers
  int fold = 0;         // as in ChunkPlan
  int chunk = 0;        // keys (of the list's tiles) per work-group
  int splits = 0;       // key ranges of a row block at most, >= 1
  int window = 0, sinks = 0;   // as the kernels take them
  size_t ml_off = 0;    // workspace offset (bytes) of the partial maxima and sums
  size_t workspace = 0;
  float scale_log2 = 0.f;
};

// `cus`: compute units of the device the call runs on, >= 1.  `cache`: the 4-bit
// cache, or null.
simsd_status plan_window(const simsd_chunk_desc* d, int window, int sinks, int cus, SpanPlan* p);
simsd_status plan_chunk_fp4(const simsd_chunk_desc* d, int window, int sinks, int cus, SpanPlan* p);
simsd_status plan_verify_span(const simsd_attn_desc* d, bool fp4, int window, int sinks, int cus, SpanPlan* p);

// The workspace of a call with this plan.
simsd_status check_span_workspace(const char* op, const SpanPlan& p, const void* workspace, size_t workspace_bytes);
// The pointers and strides of a 4-bit cache of `max_len` tokens at most (whose codes'
// strides are the descriptor's).  Scales lie at multiples of `scales_to` bytes, a power of
// two: a head's scales where they are read as a word, a byte where one by one.
simsd_status check_fp4_cache(const char* op, const simsd_fp4_cache* c, int max_len, int scales_to);

simsd_status plan_fp4_append(const simsd_rotary_desc* d, const simsd_fp4_cache* c);
simsd_status check_fp4_values(const simsd_fp4_values_desc* d, const simsd_fp4_cache* c, const void* k_out, const void* v_out);

}  // namespace simsd
