// The temporal mask over the new slots, as the verification attentions form it.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace simsd {
namespace {

// ----------------------------------------------------------------------------
// Temporal mask (Sec. 3.1, eq. 1).  Section 0 = block slot (mask section),
// 1 = reference slot (data section), -1 = padding.  Committed block slots
// (label 0) are visible to every non-padded row; undrafted ones carry label
// gamma + 1.
// ----------------------------------------------------------------------------
struct SlotLabel {
  int sec;
  int tau;
};

// Label of new slot `slot` given its block-slot step (ignored for reference
// slots).
__device__ inline SlotLabel slot_label(int slot, int step, int gamma, int B) {
  if (slot < B) {
    if (step < 0) return {-1, -1};
    return {0, step > gamma ? gamma + 1 : step};
  }
  const int r = slot - B;
  if (r >= gamma) return {-1, -1};
  return {1, r + 1};
}

// Whether a non-padded row with label li may attend to new slot lj.
__device__ inline bool slot_visible(SlotLabel li, SlotLabel lj) {
  if (lj.sec < 0) return false;
  if (lj.sec == 0 && lj.tau == 0) return true;
  if (li.sec == 1) return lj.sec == 1 ? lj.tau <= li.tau : lj.tau > li.tau;
  return lj.sec == 1 ? lj.tau < li.tau : lj.tau >= li.tau;
}

// Visibility words of the new slots, one 64-bit word per row (bit j: the row
// may attend to slot j; zero for padding rows), written to vis[0, n_new).
// Lane j holds slot j's label; row i's word is one ballot against the label
// of lane i.  `step` is lane j's block-slot step (any value for j >= B).
template <int NW>
__device__ inline void build_visibility(uint64_t* vis, int step, int gamma, int B, int n_new,
                                        int wave, int lane) {
  const SlotLabel lj = slot_label(lane, step, gamma, B);
  for (int i = wave; i < n_new; i += NW) {
    const SlotLabel li = {__builtin_amdgcn_readlane(lj.sec, i), __builtin_amdgcn_readlane(lj.tau, i)};
    const bool v = lane < n_new && li.sec >= 0 && slot_visible(li, lj);
    const uint64_t word = __ballot(v);
    if (lane == 0) vis[i] = word;
  }
}

}  // namespace
}  // namespace simsd
