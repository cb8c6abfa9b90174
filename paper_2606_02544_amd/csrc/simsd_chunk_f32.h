// Chunk attention in float32: the kernels of few rows and of many rows.
#pragma once

#include <type_traits>

#include "simsd_span.h"

namespace simsd {
namespace {

// SPAN: the keys are a list of tiles (a sliding window with sinks), of this many each.
constexpr int kF32Tile = 32;
template <bool SPAN>
using F32Args = std::conditional_t<SPAN, SpanArgs, ChunkArgs>;
template <bool SPAN>
using F32Block = std::conditional_t<SPAN, SpanBlock, Block>;
template <bool SPAN>
__device__ inline bool setup_f32(const F32Args<SPAN>& a, F32Block<SPAN>& w) {
  if constexpr (SPAN) return setup_span<false>(a, w, kF32Tile);
  else return setup_block(a, w);
}

// ----------------------------------------------------------------------------
// float32 kernel (fp32 matrix cores), laid out as the verification attention's: a
// work-group of four waves owns RB 16-row blocks; each wave takes every fourth
// 16-key sub-tile of the range on its own, with its own running output, maximum and
// sum, K and V loading straight into the registers that feed the products; the four
// states merge in LDS at the end.  v_mfma_f32_16x16x4_f32 takes one float a lane:
//   S^T = K Q^T: lane (n = lane % 16, q = lane / 16) holds dims 16 i + 4 q + e
//     of key n (register e of load i), and of query row n.
//   O^T += V^T P^T: MFMA j contracts keys 4 {0..3} + j.  Register j of the
//     scores is key 4 q + j of row n already; the V^T operand is key 4 q + j, dim
//     64 u + 4 n + e, register e of the 16-byte load (j, u).
// It serves few rows (single tokens over 4000 keys, 32/8 heads: 8 of them 51 us, 5.2 TB/s,
// 64 of them 364 us, 5.8 TB/s; a prompt of 512: 36 us, of 1000: 118, where the kernel below
// takes 103).
// ----------------------------------------------------------------------------
template <int D, int RB, bool PAGED, bool SPAN = false>
__global__ void __launch_bounds__(256, 2) chunk_f32_kernel(F32Args<SPAN> a) {
  constexpr int NW = 4, SUB = 16;              // waves; keys per sub-tile
  constexpr int KI = D / 16;                   // 16-byte loads per lane of a K (or Q) row
  constexpr int VU = D / 64;                   // 16-byte loads per lane of a V key
  constexpr int ROWS = 16 * RB;
  constexpr int XROW = D + 4;                  // LDS row stride of the merge (floats)
  __shared__ __attribute__((aligned(16))) float xs[NW * ROWS * XROW];
  __shared__ float s_m[NW][ROWS], s_l[NW][ROWS];

  F32Block<SPAN> w;
  if (!setup_f32<SPAN>(a, w)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q = lane >> 4;
  int nsub = 0;
  if constexpr (SPAN) {
    nsub = w.nt * (kF32Tile / SUB);
    if (w.t0 + w.nt == w.s.tiles && w.nt > 0)  // (sub-tiles behind the last key)
      nsub -= (kF32Tile - 1 - (w.s.hi - 1) % kF32Tile) / SUB;
  } else {
    nsub = w.kend > w.kbeg ? (w.kend - w.kbeg + SUB - 1) / SUB : 0;
  }
  const int items = nsub > wave ? (nsub - wave + NW - 1) / NW : 0;
  const int64_t head0 = (PAGED ? 0 : w.b * a.cs_seq) + w.kvh * a.cs_head;
  const float* kc = static_cast<const float*>(a.k_cache) + head0;
  const float* vc = static_cast<const float*>(a.v_cache) + head0;
  const int32_t* pages = a.block_table + static_cast<int64_t>(w.b) * a.max_pages;
  auto list = [&](int i) __attribute__((always_inline)) {   // SPAN: the tile of this wave's sub-tile i
    if constexpr (SPAN) return tile_keys(w.s, w.t0 + (wave + NW * i) / (kF32Tile / SUB), kF32Tile);
    else return 0;
  };
  auto key0 = [&](int i) __attribute__((always_inline)) {
    if constexpr (SPAN) return list(i).k0 + SUB * ((wave + NW * i) % (kF32Tile / SUB));
    else return w.kbeg + SUB * (wave + NW * i);
  };
  // The key that is read for key `key` of sub-tile i.
  auto held = [&](int i, int key) __attribute__((always_inline)) {
    if constexpr (SPAN) {
      const TileKeys k = list(i);
      return max(k.beg, min(key, k.end - 1));
    } else {
      return min(key, w.kend - 1);
    }
  };
  // Keys past the range's last one read that one (their scores are masked).
  auto key_at = [&](const float* base, int i, int key, int page) __attribute__((always_inline)) {
    key = held(i, key);
    if (!PAGED) return base + key * a.cs_tok;
    return base + (page * a.cs_seq + (key % a.page_size) * a.cs_tok);
  };
  f32x4 kx[KI], vx[SUB / 4][VU];
  int page = 0, page_v = 0;                    // of key n: of the K loads ahead, of the V loads ahead
  auto next_page = [&](int i) __attribute__((always_inline)) {
    if (PAGED && i < items) page = pages[held(i, key0(i) + n) / a.page_size];
  };
  auto load_k = [&](int i) __attribute__((always_inline)) {
    const f32x4* kr = reinterpret_cast<const f32x4*>(key_at(kc, i, key0(i) + n, page));
#pragma unroll
    for (int c = 0; c < KI; ++c) kx[c] = kr[4 * c + q];
    page_v = page;
    next_page(i + 1);
  };
  auto load_v = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < SUB / 4; ++j) {
      const int pj = PAGED ? __shfl(page_v, 4 * q + j) : 0;
      const f32x4* vr = reinterpret_cast<const f32x4*>(key_at(vc, i, key0(i) + 4 * q + j, pj));
#pragma unroll
      for (int u = 0; u < VU; ++u) vx[j][u] = vr[16 * u + n];
    }
  };
  if (items > 0) {
    next_page(0);
    load_k(0);
    load_v(0);
  }

  // Query operands: row 16 r + n of the block, dims 16 i + 4 q + e; and its limit.
  f32x4 qop[RB][KI];
  int limit[RB], first[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int m = w.row0 + 16 * r + n;
    const int mc = min(m, w.rows - 1), t = mc / a.group;
    const f32x4* qr = reinterpret_cast<const f32x4*>(
        static_cast<const float*>(a.q) + (static_cast<int64_t>(w.q0 + t) * a.hq + w.kvh * a.group + mc % a.group) * D);
#pragma unroll
    for (int i = 0; i < KI; ++i) qop[r][i] = qr[4 * i + q];
    limit[r] = m < w.rows ? visible_keys(a, w.kv, w.n, t) : 0;
    if constexpr (SPAN) first[r] = m < w.rows ? first_at(a.mask_block, a.window, w.kv - w.n + t) : 0;
  }

  f32x4 o[RB][D / 16];
  // Whether row r sees key `key` of sub-tile i.
  auto sees = [&](int r, int i, int key) __attribute__((always_inline)) {
    if constexpr (SPAN) {
      return row_sees(w.s, list(i), key, limit[r], first[r]);
    } else {
      return key < limit[r];
    }
  };
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[r] = kNegInf;
    l_run[r] = 0.f;
  }
  const float sl2 = a.scale_log2;
  // m_run is the running maximum (log2 units) rounded up to a whole number: the
  // state is rescaled by exact powers of two, only when the maximum passes one, and
  // no weight exceeds 1.  The scale goes into the exponent's FMA, except past 2^24,
  // where the exact product differs from the rounded maximum by more than 1: there
  // it rounds first, as the maximum did.
  int bad_first = 0x7fffffff, bad_last = -1;   // items with values that are not finite
  for (int it = 0; it < items; ++it) {
    const int k0 = key0(it);
    // Four partial sums of D / 4 dims each, added up as they end: shorter
    // rounding chains than one sum over all D.
    f32x4 s[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      f32x4 sp[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) sp[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = c * KI / 4; i < (c + 1) * KI / 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < RB; ++r)
            sp[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[i][e], qop[r][i][e], sp[r], 0, 0, 0);
#pragma unroll
      for (int r = 0; r < RB; ++r) s[r] += sp[r];
    }
    __builtin_amdgcn_sched_barrier(0);
    if (it + 1 < items) load_k(it + 1);
    bool masked;                               // some row does not see all of it
    if constexpr (SPAN) masked = list(it).sink || k0 + SUB > w.lim.limit_first || k0 < w.lim.first_last;
    else masked = k0 + SUB > w.full;
    if (masked) {
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!sees(r, it, k0 + 4 * q + j)) s[r][j] = kNegInf;
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const float mx = quad_max(fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3])));
      const float m_new = mx * sl2;
      if (m_new > m_run[r]) {
        const float up = ceilf(m_new);
        const float alpha = __builtin_amdgcn_exp2f(m_run[r] - up);
        l_run[r] *= alpha;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[r][c] *= alpha;
        m_run[r] = up;
      }
      const float moff = m_run[r] == kNegInf ? 0.f : m_run[r];
      if (__builtin_expect(__any(fabsf(moff) > 0x1p24f), 0)) {
#pragma clang fp contract(off)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[r][j] = s[r][j] * sl2 - moff;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[r][j] = fmaf(s[r][j], sl2, -moff);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[r][j] = __builtin_amdgcn_exp2f(s[r][j]);
        l_run[r] += s[r][j];
      }
    }
    if (masked) {
      bool mine = false;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(fabsf(vx[j][u][e]) < __builtin_huge_valf())) {
              vx[j][u][e] = 0.f;
              mine = true;
            }
      if (__any(mine)) {
        bad_first = min(bad_first, it);
        bad_last = it;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int u = 0; u < VU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < RB; ++r)
            o[r][4 * u + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[j][u][e], s[r][j], o[r][4 * u + e], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (it + 1 < items) load_v(it + 1);
  }
  // The sub-tiles with values that are not finite, again (as in the bf16 kernel).
  for (int it = bad_first; it <= bad_last; ++it) {
    const int k0 = key0(it);
    if constexpr (SPAN)                        // (a sub-tile between them that all rows see whole)
      if (!list(it).sink && k0 + SUB <= w.lim.limit_first && k0 >= w.lim.first_last) continue;
    next_page(it);
    page_v = page;
    load_v(it);
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = vx[j][u][e];
            const float code = fabsf(x) < __builtin_huge_valf() ? 0.f : x > 0.f ? 1.f : x < 0.f ? float(kCode1) : float(kCode2);
            sum = __builtin_amdgcn_mfma_f32_16x16x4f32(code, sees(r, it, k0 + 4 * q + j) ? 1.f : 0.f, sum, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (sum[i] != 0.f) o[r][4 * u + e][i] += code_value(sum[i]);
          __builtin_amdgcn_sched_barrier(0);
        }
  }

  // Merge of the four waves' states.
#pragma unroll
  for (int r = 0; r < RB; ++r) l_run[r] = quad_sum(l_run[r]);
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int row = 16 * r + n;
    // Register t of o[r][4 u + e] holds dim 64 u + 16 q + 4 t + e of this row.
    float* x = &xs[(wave * ROWS + row) * XROW + 16 * q];
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        *reinterpret_cast<f32x4*>(x + 64 * u + 4 * t) =
            f32x4{o[r][4 * u][t], o[r][4 * u + 1][t], o[r][4 * u + 2][t], o[r][4 * u + 3][t]};
    if (q == 0) {
      s_m[wave][row] = m_run[r];
      s_l[wave][row] = l_run[r];
    }
  }
  __syncthreads();
  for (int idx = tid; idx < ROWS * (D / 4); idx += NW * 64) {
    const int row = idx / (D / 4), d0 = 4 * (idx % (D / 4));
    const int m = w.row0 + row;
    if (m >= w.rows) continue;
    float mt = kNegInf;
#pragma unroll
    for (int g = 0; g < NW; ++g) mt = fmaxf(mt, s_m[g][row]);
    const float mref = mt == kNegInf ? 0.f : mt;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int g = 0; g < NW; ++g) {
      const float wt = __builtin_amdgcn_exp2f(s_m[g][row] - mref);
      acc += wt * *reinterpret_cast<const f32x4*>(&xs[(g * ROWS + row) * XROW + d0]);
      l += wt * s_l[g][row];
    }
    const int t = m / a.group, hq = w.kvh * a.group + m % a.group, token = w.q0 + t;
    if (w.nsplit == 1) {
      const bool valid = visible_keys(a, w.kv, w.n, t) > 0;
      const float inv = valid ? 1.f / l : 0.f;
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + (static_cast<int64_t>(token) * a.hq + hq) * D + d0) = acc * inv;
      if (a.lse && d0 == 0)
        a.lse[static_cast<int64_t>(hq) * a.tokens + token] = valid ? log_sum(mt, l) : kNegInf;
    } else {
      const int64_t r = partial_row(a, w.split, token, hq);
      *reinterpret_cast<f32x4*>(a.part + r * D + d0) = acc;
      if (d0 == 0) a.part_ml[r] = float2{mt, l};
    }
  }
}

// ----------------------------------------------------------------------------
// float32, many rows: four waves of RB 16-row blocks each share tiles of 32 keys in an
// LDS ring of two slots, two work-groups a CU.  The kernel above reads K and V once
// per 32 rows from the L2, at 19 TB/s for the chip were its products at their full
// rate; here it is once per 64 or 128 rows.  What bounds it: the fp32 products.  4 sequences of
// 512 tokens over 4000 keys, 32/8 heads: 1379 us with the kernel above, 1240 here
// (floor 928); a prompt of 4096: 1335 above, 1224 here (64 rows; floor 894).
// Operands are as above, read from LDS.
// ----------------------------------------------------------------------------
template <int D, int RB, bool PAGED, bool SPAN = false>
__global__ void __launch_bounds__(256, 2) chunk_f32_rows_kernel(F32Args<SPAN> a) {
  constexpr int NW = 4, SUB = 16, NBUF = 2;
  constexpr int KI = D / 16, VU = D / 64;
  using Ring = ChunkRing<F32Tile<D>, NW, PAGED, SPAN>;
  constexpr int ROWB = Ring::ROWB, TILEB = Ring::TILEB, KEYS = Ring::KEYS;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NBUF][2][TILEB];   // [slot][K, V]
  __shared__ int s_pg_arr[PAGED ? kMaxChunkPages : 1];
  __shared__ int s_bad[2];                     // first and last tile with values that are not finite
  __shared__ int s_first[SPAN ? 64 * RB : 1];  // the rows' first keys (for the tiles that need them)
  SIMSD_LDS int* s_pg = (SIMSD_LDS int*)(&s_pg_arr[0]);

  F32Block<SPAN> w;
  if (!setup_f32<SPAN>(a, w)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q = lane >> 4;
  if (tid == 0) {
    s_bad[0] = 0x7fffffff;
    s_bad[1] = -1;
  }
  const int wrow = w.row0 + wave * 16 * RB;    // this wave's first row
  const int wave_last = min(wrow + 16 * RB, w.rows) - 1;
  const int wave_end = wrow < w.rows ? visible_keys(a, w.kv, w.n, wave_last / a.group) : 0;

  f32x4 qop[RB][KI];
  int limit[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int m = wrow + 16 * r + n;
    const int mc = min(m, w.rows - 1), t = mc / a.group;
    const f32x4* qr = reinterpret_cast<const f32x4*>(
        static_cast<const float*>(a.q) + (static_cast<int64_t>(w.q0 + t) * a.hq + w.kvh * a.group + mc % a.group) * D);
#pragma unroll
    for (int i = 0; i < KI; ++i) qop[r][i] = qr[4 * i + q];
    limit[r] = m < w.rows ? visible_keys(a, w.kv, w.n, t) : 0;
    if constexpr (SPAN)
      if (q == 0) s_first[16 * (wave * RB + r) + n] = first_at(a.mask_block, a.window, w.kv - w.n + t);
  }
  Ring kv;
  kv.init(a, w, wave, lane, s_pg);
  PageIds pages = {0, 0};
  if constexpr (SPAN && PAGED) pages.stage(a, w, KEYS, tid, NW * 64, s_pg);
  __builtin_amdgcn_s_waitcnt(0);               // (as in the bf16 kernel)
  __syncthreads();                             // staged page ids, s_bad
  static_assert(!SPAN || KEYS == kF32Tile, "tiles of the list");
  int nt = 0;
  if constexpr (SPAN) nt = w.nt;
  else nt = w.kend > w.kbeg ? (w.kend - w.kbeg + KEYS - 1) / KEYS : 0;
  auto list = [&](int it) __attribute__((always_inline)) {
    if constexpr (SPAN) return tile_keys(w.s, w.t0 + it, KEYS);
    else return 0;
  };
  auto key0 = [&](int it) __attribute__((always_inline)) {
    if constexpr (SPAN) return list(it).k0;
    else return w.kbeg + it * KEYS;
  };
  auto issue = [&](uint32_t slot, int it) __attribute__((always_inline)) {
    if constexpr (SPAN) {
      const TileKeys k = list(it);
      kv.pg_first = k.sink ? +pages.first_sink : +pages.first_win;
      kv.issue(slot, k.k0, k.end, s_pg, k.beg);
    } else {
      kv.issue(slot, w.kbeg + it * KEYS, w.kend, s_pg);
    }
  };
  auto sees = [&](int r, int it, int key) __attribute__((always_inline)) {
    if constexpr (SPAN) {
      return row_sees(w.s, list(it), key, limit[r], s_first[16 * (wave * RB + r) + n]);
    } else {
      return key < limit[r];
    }
  };
  // Whether some row of the block does not see all of the tile at k0.
  auto open = [&](int it, int k0) __attribute__((always_inline)) {
    if constexpr (SPAN) return list(it).sink | (k0 + KEYS > w.lim.limit_first) | (k0 < w.lim.first_last);
    else return k0 + KEYS > w.full;
  };
  const uint32_t ring0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((SIMSD_LDS void*)(&smem[0][0][0])));
  constexpr uint32_t kSlotBytes = 2 * TILEB;
#pragma unroll
  for (int j = 0; j < NBUF; ++j)
    if (j < nt) issue(ring0 + j * kSlotBytes, j);

  f32x4 o[RB][D / 16];
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[r] = kNegInf;
    l_run[r] = 0.f;
  }
  const float sl2 = a.scale_log2;
  // LDS offsets: K chunk 4 i + q of key n; V chunk 16 u + n of key 4 q + j.
  auto k_at = [&](const SIMSD_LDS uint8_t* sk, int i) {
    return *reinterpret_cast<const SIMSD_LDS f32x4*>(sk + n * ROWB + 16 * ((4 * i + q) ^ (n & 7)));
  };
  auto v_at = [&](const SIMSD_LDS uint8_t* sv, int j, int u) {
    const int key = 4 * q + j;
    return *reinterpret_cast<const SIMSD_LDS f32x4*>(sv + key * ROWB + 16 * ((16 * u + n) ^ (key & 7)));
  };

#pragma unroll 1
  for (int it = 0; it < nt; ++it) {
    const int k0 = key0(it);
    if (it == 0 && nt > 1) wait_vm<Ring::PERW>();
    else wait_vm<0>();
    lds_barrier();                             // all of tile `it` is in; the other slot is free
    if (it >= 1 && it + 1 < nt) issue(ring0 + ((it + 1) & 1) * kSlotBytes, it + 1);
    const SIMSD_LDS uint8_t* sk = reinterpret_cast<const SIMSD_LDS uint8_t*>(ring0) + (it & 1) * kSlotBytes;
    const SIMSD_LDS uint8_t* sv = sk + TILEB;
    const bool masked = open(it, k0);
    if (masked) {
      bool mine = false;
#pragma unroll
      for (int i = 0; i < TILEB / (NW * 64 * 16); ++i) {
        SIMSD_LDS f32x4* at = (SIMSD_LDS f32x4*)(sv + (i * NW * 64 + tid) * 16);
        f32x4 x = *at;
        bool wild = false;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!(fabsf(x[e]) < __builtin_huge_valf())) {
            x[e] = 0.f;
            wild = true;
          }
        if (wild) {
          *at = x;
          mine = true;
        }
      }
      if (__ballot(mine) && lane == 0) {
        atomicMin(&s_bad[0], it);
        atomicMax(&s_bad[1], it);
      }
      lds_barrier();
    }
#pragma unroll 1
    for (int sub = 0; sub < KEYS / SUB; ++sub) {
      const int ks = k0 + SUB * sub;
      if (ks >= wave_end) break;               // no row of this wave sees a key of it
      const SIMSD_LDS uint8_t* skb = sk + SUB * sub * ROWB;
      const SIMSD_LDS uint8_t* svb = sv + SUB * sub * ROWB;
      f32x4 s[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 4; ++c) {            // four partial sums: shorter rounding chains
        f32x4 sp[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) sp[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = c * KI / 4; i < (c + 1) * KI / 4; ++i) {
          const f32x4 kx = k_at(skb, i);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < RB; ++r)
              sp[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[e], qop[r][i][e], sp[r], 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) s[r] += sp[r];
      }
      if (masked) {
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (!sees(r, it, ks + 4 * q + j)) s[r][j] = kNegInf;
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const float mx = quad_max(fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3])));
        const float m_new = mx * sl2;
        if (m_new > m_run[r]) {
          const float up = ceilf(m_new);
          const float alpha = __builtin_amdgcn_exp2f(m_run[r] - up);
          l_run[r] *= alpha;
#pragma unroll
          for (int c = 0; c < D / 16; ++c) o[r][c] *= alpha;
          m_run[r] = up;
        }
        const float moff = m_run[r] == kNegInf ? 0.f : m_run[r];
        if (__builtin_expect(__any(fabsf(moff) > 0x1p24f), 0)) {
#pragma clang fp contract(off)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[r][j] = s[r][j] * sl2 - moff;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[r][j] = fmaf(s[r][j], sl2, -moff);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[r][j] = __builtin_amdgcn_exp2f(s[r][j]);
          l_run[r] += s[r][j];
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < VU; ++u) {
          const f32x4 vx = v_at(svb, j, u);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < RB; ++r)
              o[r][4 * u + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[e], s[r][j], o[r][4 * u + e], 0, 0, 0);
        }
    }
  }
  // The tiles with values that are not finite, again.
  lds_barrier();                               // the ring is free (no load is pending)
  const int last = __builtin_amdgcn_readfirstlane(s_bad[1]);
#pragma unroll 1
  for (int it = __builtin_amdgcn_readfirstlane(s_bad[0]); it <= last; ++it) {
    if constexpr (SPAN)
      if (!open(it, key0(it))) continue;
    issue(ring0, it);
    wait_vm<0>();
    lds_barrier();
    const SIMSD_LDS uint8_t* sv = reinterpret_cast<const SIMSD_LDS uint8_t*>(ring0) + TILEB;
#pragma unroll 1
    for (int sub = 0; sub < KEYS / SUB; ++sub) {
      const int ks = key0(it) + SUB * sub;
#pragma unroll
      for (int u = 0; u < VU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = v_at(sv + SUB * sub * ROWB, j, u)[e];
              const float code = fabsf(x) < __builtin_huge_valf() ? 0.f : x > 0.f ? 1.f : x < 0.f ? float(kCode1) : float(kCode2);
              sum = __builtin_amdgcn_mfma_f32_16x16x4f32(code, sees(r, it, ks + 4 * q + j) ? 1.f : 0.f, sum, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (sum[i] != 0.f) o[r][4 * u + e][i] += code_value(sum[i]);
            __builtin_amdgcn_sched_barrier(0);
          }
    }
    lds_barrier();
  }

#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const float l = quad_sum(l_run[r]);
    const int m = wrow + 16 * r + n;
    if (m >= w.rows) continue;
    const int t = m / a.group, hq = w.kvh * a.group + m % a.group, token = w.q0 + t;
    const bool whole = w.nsplit == 1;
    const int64_t at = whole ? static_cast<int64_t>(token) * a.hq + hq : partial_row(a, w.split, token, hq);
    const float by = !whole ? 1.f : limit[r] > 0 ? 1.f / l : 0.f;
    // Register t of o[r][4 u + e] holds dim 64 u + 16 q + 4 t + e of this row.
    float* x = (whole ? static_cast<float*>(a.out) : a.part) + at * D + 16 * q;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(x + 64 * u + 4 * i) =
            f32x4{o[r][4 * u][i], o[r][4 * u + 1][i], o[r][4 * u + 2][i], o[r][4 * u + 3][i]} * by;
    if (q == 0) {
      if (!whole) a.part_ml[at] = float2{m_run[r], l};
      else if (a.lse) a.lse[static_cast<int64_t>(hq) * a.tokens + token] = limit[r] > 0 ? log_sum(m_run[r], l) : kNegInf;
    }
  }
}

}  // namespace
}  // namespace simsd
