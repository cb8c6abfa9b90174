// Chunk attention over a cache held in 4 bits.
#include "simsd_span_kernel.h"

namespace simsd {

hipError_t launch_fp4(const SpanPlan& p, int d, const SpanArgs& a, hipStream_t st) {
  if (d == 128) launch_span_d<128, true, false>(p, a, st);
  else launch_span_d<64, true, false>(p, a, st);
  return hipGetLastError();
}

}  // namespace simsd
