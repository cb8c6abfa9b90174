// The verification step's attention under a sliding window with sinks, and over a cache
// held in 4 bits: the cached prefix as a list of tiles, the new slots as its last tile.
#include "simsd_fp4_rows.h"
#include "simsd_span_kernel.h"

namespace simsd {
namespace {

template <int D>
void launch_d(const SpanPlan& p, const SpanArgs& a, hipStream_t st) {
  if (p.few == 1) launch_fp4_rows<D, 1, true>(p, a, st);
  else if (p.few == 2) launch_fp4_rows<D, 2, true>(p, a, st);
  else launch_span_d<D, true, true>(p, a, st);
}

}  // namespace

hipError_t launch_verify_span(const SpanPlan& p, bool fp4, int d, const SpanArgs& a, hipStream_t st) {
  if (fp4) {
    if (d == 128) launch_d<128>(p, a, st);
    else launch_d<64>(p, a, st);
  } else {
    if (d == 128) launch_span_d<128, false, true>(p, a, st);
    else launch_span_d<64, false, true>(p, a, st);
  }
  return hipGetLastError();
}

}  // namespace simsd
