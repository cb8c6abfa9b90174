// The row blocks and key ranges of attention over a list of tiles, and the kernel that
// joins the ranges.
#pragma once

#include "simsd_chunk_device.h"
#include "simsd_mask.h"
#include "simsd_span_list.h"

namespace simsd {
namespace {

// What the rows [row0, last] of a sequence see, over all of them and at the least.
// (Rows' first keys and limits rise with the row.)
struct Bounds {
  int first, hi;                 // lowest first key, highest limit
  int first_last, limit_first;   // highest first key, lowest limit
};
template <bool VERIFY>
__device__ __attribute__((always_inline)) inline Bounds bounds_of(const SpanArgs& a, int kv, int n, int row0, int last) {
  if constexpr (VERIFY) {        // the cached prefix: the same for every row
    const int first = a.window ? max(0, kv - a.window + 1) : 0;
    return {first, kv, first, kv};
  } else {
    const int p0 = kv - n + row0 / a.group, p1 = kv - n + last / a.group;
    return {first_at(a.mask_block, a.window, p0), limit_at(a.mask_block, kv, p1), first_at(a.mask_block, a.window, p1),
            limit_at(a.mask_block, kv, p0)};
  }
}

struct SpanBlock : Block {
  Span s;
  Bounds lim;
  int t0, nt;                    // tiles [t0, t0 + nt) of the list are this work-group's
};

// How many key ranges a list is divided into.  VERIFY: the tile of the new slots is the
// last of the list.
template <bool VERIFY>
__device__ __attribute__((always_inline)) inline int ranges_of(const SpanArgs& a, int tiles, int TK) {
  const int c = a.chunk / TK;
  return max(1, (tiles + (VERIFY ? 1 : 0) + c - 1) / c);
}

template <bool VERIFY>
__device__ __attribute__((always_inline)) inline bool setup_span(const SpanArgs& a, SpanBlock& w, int TK) {
  w.kvh = blockIdx.x % a.hkv;
  w.split = blockIdx.y;
  w.kbeg = w.kend = w.full = 0;                // (of one range of keys, not a list)
  int rb, rank = static_cast<int>(blockIdx.x) / a.hkv;
  if constexpr (VERIFY) {
    w.b = rank / a.seq_blocks;
    rb = rank % a.seq_blocks;
    // From the longest prefix down, so that the last to start are short (64 of 4160, 12480,
    // 20800 and 29120 in turn: 506 -> 412 us; the longest met on one unit before).
    if (a.batch <= 64 && a.window == 0) {
      const int lane = threadIdx.x & 63, kv = a.kv_lens[min(lane, a.batch - 1)];
      int place = 0;
      for (int i = 0; i < a.batch; ++i) {
        const int k = __builtin_amdgcn_readlane(kv, i);
        place += k > kv || (k == kv && i < lane) ? 1 : 0;
      }
      w.b = __builtin_ctzll(__ballot(lane < a.batch && place == w.b));
    }
    w.q0 = w.b * a.n_new;
    w.n = a.n_new;
    w.kv = min(max(a.kv_lens[w.b], 0), a.max_kv);
  } else {
    if (a.fold) {
      const int place = rank, twice = a.blocks - a.fold;
      rank = place >= a.fold ? a.blocks - 1 - (place - a.fold) : place < twice ? a.fold - twice + place : place - twice;
    }
    if (!find_block(a, rank, threadIdx.x & 63, w, &rb)) return false;
  }
  w.rows = w.n * a.group;
  w.row0 = rb * a.rows_pb;
  if (w.row0 >= w.rows) return false;
  w.lim = bounds_of<VERIFY>(a, w.kv, w.n, w.row0, min(w.row0 + a.rows_pb, w.rows) - 1);
  w.s = span_of(a.sinks, w.lim.first, w.lim.hi, TK);
  w.nsplit = ranges_of<VERIFY>(a, w.s.tiles, TK);
  if (w.split >= w.nsplit) return false;
  const int c = a.chunk / TK;
  w.t0 = w.split * c;
  w.nt = min(w.s.tiles + (VERIFY ? 1 : 0) - w.t0, c);
  return true;
}

// The ids of the pages that a work-group's tiles lie in, those of the sinks' tiles
// first: page g of tile kind x is entry g - first[x].
struct PageIds {
  int first_sink, first_win;
  __device__ inline void stage(const SpanArgs& a, const SpanBlock& w, int TK, int tid, int nthreads, SIMSD_LDS int* s_pg) {
    const PageSpan p = pages_of(w.s, w.t0, w.t0 + w.nt, TK, a.page_size);
    const int32_t* bt = a.block_table + static_cast<int64_t>(w.b) * a.max_pages;
    for (int j = tid; j < p.sinks; j += nthreads) s_pg[j] = bt[p.first_sink + j];
    for (int j = tid; j < p.wins; j += nthreads) s_pg[p.sinks + j] = bt[p.first_win + j];
    first_sink = p.first_sink;
    first_win = p.first_win - p.sinks;
  }
};

// Where a row's log-sum-exp goes: [Hq, tokens], or the verification's [batch, Hq, B + L].
template <bool VERIFY>
__device__ inline int64_t lse_at(const SpanArgs& a, int token, int head) {
  if (!VERIFY) return static_cast<int64_t>(head) * a.tokens + token;
  return (static_cast<int64_t>(token / a.n_new) * a.hq + head) * a.n_new + token % a.n_new;
}

// ----------------------------------------------------------------------------
// Joins the key ranges of a token's rows, as the chunk attention's second kernel does:
// D / 4 lanes hold a row, four dims each; WIDE: the four waves of a work-group share
// the ranges of one wave's rows.  A range in which a row sees nothing has weight 0.
// ----------------------------------------------------------------------------
template <int D, bool BF16, bool VERIFY, bool WIDE>
__global__ void __launch_bounds__(256) span_merge_kernel(SpanArgs a, int TK) {
  constexpr int LPR = D / 4;                   // lanes per row
  constexpr int RPW = 64 / LPR;                // rows per wave
  constexpr int U = 4;                         // ranges loaded at a time
  __shared__ f32x4 xo[WIDE ? 256 : 1];
  __shared__ float2 xml[WIDE ? 256 : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int token = blockIdx.x;
  int b, q0, n;
  if constexpr (VERIFY) {
    b = token / a.n_new;
    q0 = b * a.n_new;
    n = a.n_new;
  } else {
    b = __builtin_amdgcn_readfirstlane(leading(a.batch, lane, [&](int i) { return a.q_starts[i + 1] <= token; }));
    if (b >= a.batch || token < a.q_starts[0]) return;
    q0 = a.q_starts[b];
    n = min(a.q_starts[b + 1], a.tokens) - q0;
  }
  const int kv = min(max(a.kv_lens[b], 0), a.max_kv);
  const int head = blockIdx.y * (WIDE ? RPW : 4 * RPW) + (WIDE ? 0 : wave * RPW) + lane / LPR;
  const int d0 = 4 * (lane % LPR);
  const int i = token - q0;
  // The ranges of the row's block.
  const int hc = min(head, a.hq - 1);
  const int row0 = (i * a.group + hc % a.group) / a.rows_pb * a.rows_pb;
  const Bounds lim = bounds_of<VERIFY>(a, kv, n, row0, min(row0 + a.rows_pb, n * a.group) - 1);
  const int ranges = ranges_of<VERIFY>(a, span_of(a.sinks, lim.first, lim.hi, TK).tiles, TK);
  const bool joined = ranges > 1;
  const int most = joined ? ranges : 0;
  bool valid;
  if constexpr (VERIFY)
    valid = slot_label(i, i < a.block ? a.step_map[b * a.block + i] : 0, a.num_ref[b], a.block).sec >= 0;
  else
    valid = visible_keys(a, kv, n, i) > 0;
  float m = kNegInf, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int STEP = WIDE ? 4 : 1;
  for (int s = WIDE ? wave : 0; s < most; s += STEP * U) {
    float2 ml[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = partial_row(a, min(s + u * STEP, most - 1), token, hc);
      ml[u] = a.part_ml[r];
      x[u] = *reinterpret_cast<const f32x4*>(a.part + r * D + d0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u * STEP >= most) continue;
      const float mm = fmaxf(m, ml[u].x);
      const float ref = mm == kNegInf ? 0.f : mm;
      const float c0 = __builtin_amdgcn_exp2f(m - ref), c1 = __builtin_amdgcn_exp2f(ml[u].x - ref);
      o = o * c0 + x[u] * c1;
      l = l * c0 + ml[u].y * c1;
      m = mm;
    }
  }
  if constexpr (WIDE) {
    xo[tid] = o;
    xml[tid] = float2{m, l};
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int g = 1; g < 4; ++g) {
      const float2 ml = xml[g * 64 + lane];
      const float mm = fmaxf(m, ml.x);
      const float ref = mm == kNegInf ? 0.f : mm;
      const float c0 = __builtin_amdgcn_exp2f(m - ref), c1 = __builtin_amdgcn_exp2f(ml.x - ref);
      o = o * c0 + xo[g * 64 + lane] * c1;
      l = l * c0 + ml.y * c1;
      m = mm;
    }
  }
  if (!joined || head >= a.hq) return;
  o = valid ? o * (1.f / l) : f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t at = (static_cast<int64_t>(token) * a.hq + head) * D + d0;
  if constexpr (BF16)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = u32x2{pack2(o[0], o[1]), pack2(o[2], o[3])};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = o;
  if (a.lse && d0 == 0) a.lse[lse_at<VERIFY>(a, token, head)] = valid ? log_sum(m, l) : kNegInf;
}

template <int D, bool BF16, bool VERIFY>
void launch_span_merge(const SpanPlan& p, const SpanArgs& a, int TK, hipStream_t st) {
  if (p.splits == 1) return;
  constexpr int RPW = 64 / (D / 4);
  // WIDE where the chip holds all its work-groups at once (eight to a unit): in rounds of
  // them their chains of loads add up (1024 rows of 32 heads: 28 us, with two rows to each wave 14).
  const bool wide = p.splits > 4 && int64_t{a.tokens} * ((a.hq + RPW - 1) / RPW) <= 2048;
  const int per = wide ? RPW : 4 * RPW;
  const dim3 grid(a.tokens, (a.hq + per - 1) / per);
  if (wide) hipLaunchKernelGGL((span_merge_kernel<D, BF16, VERIFY, true>), grid, dim3(256), 0, st, a, TK);
  else hipLaunchKernelGGL((span_merge_kernel<D, BF16, VERIFY, false>), grid, dim3(256), 0, st, a, TK);
}

}  // namespace
}  // namespace simsd
