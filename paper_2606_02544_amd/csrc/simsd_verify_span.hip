// The verification step's attention under a sliding window with sinks, and over a cache
// held in 4 bits: the cached prefix as a list of tiles, the new slots as its last tile.
#include "simsd_span_kernel.h"

namespace simsd {

hipError_t launch_verify_span(const SpanPlan& p, bool fp4, int d, const SpanArgs& a, hipStream_t st) {
  if (fp4) {
    if (d == 128) launch_span_d<128, true, true>(p, a, st);
    else launch_span_d<64, true, true>(p, a, st);
  } else {
    if (d == 128) launch_span_d<128, false, true>(p, a, st);
    else launch_span_d<64, false, true>(p, a, st);
  }
  return hipGetLastError();
}

}  // namespace simsd
