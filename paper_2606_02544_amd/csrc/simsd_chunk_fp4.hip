// Chunk attention over a cache held in 4 bits.
#include "simsd_fp4_rows.h"
#include "simsd_span_kernel.h"

namespace simsd {
namespace {

template <int D>
void launch_d(const SpanPlan& p, const SpanArgs& a, hipStream_t st) {
  if (p.few == 1) launch_fp4_rows<D, 1, false>(p, a, st);
  else if (p.few == 2) launch_fp4_rows<D, 2, false>(p, a, st);
  else launch_span_d<D, true, false>(p, a, st);
}

}  // namespace

hipError_t launch_fp4(const SpanPlan& p, int d, const SpanArgs& a, hipStream_t st) {
  if (d == 128) launch_d<128>(p, a, st);
  else launch_d<64>(p, a, st);
  return hipGetLastError();
}

}  // namespace simsd
