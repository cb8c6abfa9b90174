// Rotary positions on gfx950, and the write of keys and values to the cache.
//
// Pair (x1, x2) of a head turns by a = position * freq[i]:
//   y1 = m (x1 cos a - x2 sin a),  y2 = m (x2 cos a + x1 sin a),
// the pairs being dims (i, i + rot/2) or (2i, 2i + 1) of the leading rot dims;
// the other dims are copied.
//
// What bounds it: memory.  Every value is read once and written once, so a
// work-group takes whole tokens: the angles of a token are formed once, in LDS,
// for all of its heads (rot/2 of them: fp64 products, whole turns dropped in
// fp64, sine and cosine in fp32), and the heads of queries, keys and values are
// dealt to the threads in 16-byte loads.  A thread's first loads go out before
// the angles and the cache row are known, so that the round trips overlap.
// (32/8 heads of 128, bf16: 32768 tokens into a contiguous cache 157 us, 5.1 TB/s; 4224
// into pages of 16, 21 us, 4.9 TB/s; 8 tokens 3.2 us.)
#include "simsd_rotary_device.h"

namespace simsd {
namespace {

template <bool BF16, int VEC, bool INTER, bool APPEND, int TOKENS>
__global__ void __launch_bounds__(NT) rotary_kernel(RotaryArgs a) {
  rotary_tokens<BF16, VEC, INTER, APPEND, TOKENS>(a, blockIdx.x);
}

template <bool BF16, int VEC, bool INTER, bool APPEND>
void launch_tokens(const RotaryArgs& a, int cus, hipStream_t st) {
  constexpr int kMany = 4;
  if (a.tokens >= 8 * kMany * cus)
    hipLaunchKernelGGL((rotary_kernel<BF16, VEC, INTER, APPEND, kMany>), dim3((a.tokens + kMany - 1) / kMany), dim3(NT), 0, st, a);
  else
    hipLaunchKernelGGL((rotary_kernel<BF16, VEC, INTER, APPEND, 1>), dim3(a.tokens), dim3(NT), 0, st, a);
}

template <bool BF16, int VEC, bool INTER>
void launch_kind(const RotaryArgs& a, bool append, int cus, hipStream_t st) {
  if (append) launch_tokens<BF16, VEC, INTER, true>(a, cus, st);
  else launch_tokens<BF16, VEC, INTER, false>(a, cus, st);
}

template <bool BF16, int W>
void launch_layout(const RotaryPlan& p, const RotaryArgs& a, bool inter, bool append, int cus, hipStream_t st) {
  if (p.vec == 1) {
    if (inter) launch_kind<BF16, 1, true>(a, append, cus, st);
    else launch_kind<BF16, 1, false>(a, append, cus, st);
  } else {
    if (inter) launch_kind<BF16, W, true>(a, append, cus, st);
    else launch_kind<BF16, W, false>(a, append, cus, st);
  }
}

}  // namespace

hipError_t launch_rotary(const simsd_rotary_desc& d, const RotaryPlan& p, const RotaryArgs& a,
                         bool append, int cus, hipStream_t st) {
  if (a.tokens == 0 || a.units == 0) return hipSuccess;
  if (d.dtype == SIMSD_BF16) launch_layout<true, 8>(p, a, d.interleaved != 0, append, cus, st);
  else launch_layout<false, 4>(p, a, d.interleaved != 0, append, cus, st);
  return hipGetLastError();
}

}  // namespace simsd
