// Chunk attention under a sliding window with sinks.
//
// fp32 takes the chunk attention's kernels over the list of tiles: six sequences of 1 to
// 501 new tokens under a window of 511 over pages of 24 (16 query and 4 KV heads of 64) in
// 54 us, of which the products are 21 at the rate of a large one (3.2 GFLOP).  One round
// of work-groups of 32 rows, each a chain of 18 tiles with its start and end.  In ranges
// of 512 or 256 keys the pass took 63 and 65 us, with whole lists 50.
#include "simsd_chunk_f32.h"
#include "simsd_span_kernel.h"

namespace simsd {
namespace {

template <int D, bool PAGED>
void launch_window_f32(const SpanPlan& p, dim3 grid, const SpanArgs& a, hipStream_t st) {
  switch (p.rows_pb) {
    case 16: hipLaunchKernelGGL((chunk_f32_kernel<D, 1, PAGED, true>), grid, dim3(256), 0, st, a); break;
    case 32: hipLaunchKernelGGL((chunk_f32_kernel<D, 2, PAGED, true>), grid, dim3(256), 0, st, a); break;
    case 64: hipLaunchKernelGGL((chunk_f32_rows_kernel<D, 1, PAGED, true>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((chunk_f32_rows_kernel<D, 2, PAGED, true>), grid, dim3(256), 0, st, a); break;
  }
}

template <int D>
void launch_window_d(const SpanPlan& p, bool bf16, const SpanArgs& a, hipStream_t st) {
  if (bf16) {
    launch_span_d<D, false, false>(p, a, st);
    return;
  }
  const dim3 grid(p.blocks * a.hkv, p.splits);
  if (a.block_table) launch_window_f32<D, true>(p, grid, a, st);
  else launch_window_f32<D, false>(p, grid, a, st);
  launch_span_merge<D, false, false>(p, a, kF32Tile, st);
}

}  // namespace

hipError_t launch_window(const SpanPlan& p, bool bf16, int d, const SpanArgs& a, hipStream_t st) {
  if (d == 128) launch_window_d<128>(p, bf16, a, st);
  else launch_window_d<64>(p, bf16, a, st);
  return hipGetLastError();
}

}  // namespace simsd
