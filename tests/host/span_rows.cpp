// Rows of a work-group that the plans of windowed and 4-bit attention choose, on 256
// compute units.  A line a call on standard input:
//   c form tokens batch hq hkv d max_q max_kv mask_block window sinks
//   v form batch hq hkv d block refs max_prefix window sinks
// (form 0: bf16, 1: 4 bits, 2: fp32), a line with the rows of each on standard output.
#include <cstdio>

#include "simsd.h"
#include "simsd_ops_plan.h"
#include "simsd_span_plan.h"

using namespace simsd;

int main() {
  char kind;
  int form;
  while (std::scanf(" %c %d", &kind, &form) == 2) {
    SpanPlan p;
    simsd_status st;
    int window, sinks;
    if (kind == 'c') {
      simsd_chunk_desc d{};
      if (std::scanf("%d %d %d %d %d %d %d %d %d %d", &d.num_tokens, &d.batch, &d.num_q_heads, &d.num_kv_heads, &d.head_dim,
                     &d.max_q_len, &d.max_kv_len, &d.mask_block, &window, &sinks) != 10)
        return 1;
      d.dtype = form == 2 ? SIMSD_F32 : SIMSD_BF16;
      st = form == 1 ? plan_chunk_fp4(&d, window, sinks, 256, &p) : plan_window(&d, window, sinks, 256, &p);
    } else {
      simsd_attn_desc d{};
      if (std::scanf("%d %d %d %d %d %d %d %d %d", &d.batch, &d.num_q_heads, &d.num_kv_heads, &d.head_dim, &d.block_size,
                     &d.max_ref, &d.max_prefix_len, &window, &sinks) != 9)
        return 1;
      d.dtype = SIMSD_BF16;
      st = plan_verify_span(&d, form == 1, window, sinks, 256, &p);
    }
    std::printf("%d\n", st == SIMSD_OK ? p.rows_pb : -1);
  }
}
