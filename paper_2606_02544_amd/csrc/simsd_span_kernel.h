// bf16 attention over a list of tiles (see simsd_span.h): a chunk of new tokens under a
// sliding window with sinks, or over a cache held in 4 bits, or the verification step's
// new slots over either.
//
// The products are the chunk attention's (S^T = K Q^T and O^T = V^T P^T on
// v_mfma_f32_32x32x16_bf16, tiles of 64 keys in a swizzled LDS ring, RW row waves of 32
// rows, KW = 2: a second wave for the other 32 keys of each).  Tiles that some row does
// not see whole take a word of visible keys a row and 32 keys: from its limit and first
// key, or, for the tile of the new slots, the temporal mask's word.
//
// 4 bits: a tile's codes and scales are loaded into registers a tile ahead, and made bf16
// on the way into LDS once for all row waves: four instructions a word of eight codes
// (v_cvt_scalef32_pk_bf16_fp4), which is why this kernel takes 128 or 256 rows and
// fewer go to simsd_fp4_rows.h.
//
// What bounds it: matrix cores and softmax in one chain.  32 query and 8 KV heads of 128:
// two prompts of 8192 under a window of 2048 588 us (826 TFLOP/s; 410 at the rate of a
// large product), the last 2048 tokens of four 16384 over 4 bits 1880 us (1098 TFLOP/s),
// 64 slots of 16 sequences over a window of 4096 95 to 116 us (69 GFLOP, 290 MB) and 12 for
// the join of its two ranges.  Single tokens are bound by HBM: 64 over a window of 4096
// 188 us, 5.4 TB/s.
#pragma once

#include <type_traits>

#include "simsd_fp4.h"
#include "simsd_span.h"

namespace simsd {
namespace {

// One tile of the new slots' keys and values, bf16 [batch, n_new, Hkv, D], into a ring
// slot by direct loads; slots from n_new on read the last one.
template <int D, int NW>
__device__ inline void issue_new(const SpanArgs& a, const SpanBlock& w, uint32_t slot, int wave, int lane) {
  constexpr int ROWB = TileGeom<D>::ROWB, TILEB = TileGeom<D>::TILEB;
  constexpr int CPR = ROWB / 16, RPI = 1024 / ROWB, IPT = kTile / RPI, PERW = 2 * IPT / NW;
#pragma unroll
  for (int i = 0; i < PERW; ++i) {
    const int g = wave * PERW + i;
    const int row = (g % IPT) * RPI + lane / CPR;
    const int chunk = (lane % CPR) ^ swz<D>(row);
    const int64_t at = (static_cast<int64_t>(w.q0 + min(row, a.n_new - 1)) * a.hkv + w.kvh) * ROWB + chunk * 16;
    dma16(static_cast<const char*>(g < IPT ? a.k_new : a.v_new) + at, slot + (g / IPT) * TILEB + (g % IPT) * 1024);
  }
}

template <int D, int RW, int KW, bool PAGED, bool FP4, bool VERIFY>
__global__ void __launch_bounds__(RW * KW * 64, 2) span_bf16_kernel(SpanArgs a) {
  constexpr int NW = RW * KW;
  constexpr int NBUF = !FP4 && NW >= 8 ? 4 : 2;
  constexpr int NB = D / 32;                   // 32-dim output blocks
  constexpr int KS = D / 16;                   // k-steps of QK^T
  constexpr int ROWB = TileGeom<D>::ROWB;
  constexpr int TILEB = TileGeom<D>::TILEB;
  using Dma = ChunkRing<Bf16Tile<D>, NW, PAGED, true>;
  using Ring = std::conditional_t<FP4, Fp4Tiles<D, NW, PAGED>, Dma>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NBUF][2][TILEB];   // [slot][K, V]
  __shared__ int s_pg_arr[PAGED ? kMaxChunkPages : 1];
  __shared__ int s_bad[2];                     // first and last tile with values that are not finite
  __shared__ uint64_t s_vis[VERIFY ? kMaxNew : 1];
  SIMSD_LDS int* s_pg = (SIMSD_LDS int*)(&s_pg_arr[0]);

  SpanBlock w;
  if (!setup_span<VERIFY>(a, w, kTile)) return;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int rw = wave % RW, kw = wave / RW;    // row wave, key half
  if (tid == 0) {
    s_bad[0] = 0x7fffffff;
    s_bad[1] = -1;
  }

  const int m = w.row0 + rw * 32 + n;
  const bool row_in = m < w.rows;
  const int t = row_in ? m / a.group : 0;
  const int hq = w.kvh * a.group + (row_in ? m % a.group : 0);
  const int limit = !row_in ? 0 : VERIFY ? w.kv : visible_keys(a, w.kv, w.n, t);
  const int first = VERIFY ? w.lim.first : row_in ? first_at(a.mask_block, a.window, w.kv - w.n + t) : 0;
  // Keys past which no row of this wave sees anything, and before which none does by
  // its window.
  const bool wave_in = w.row0 + rw * 32 < w.rows;
  const int wave_last = min(w.row0 + rw * 32 + 31, w.rows - 1);
  int wave_end = 0, wave_first = 0;
  if (wave_in) {
    const Bounds b = bounds_of<VERIFY>(a, w.kv, w.n, w.row0 + rw * 32, wave_last);
    wave_end = b.hi;
    wave_first = b.first;
  }

  // Q^T operands of this lane's row (dims 16*ks + 8*h + [0, 8)), loaded first
  // so that they have landed before the tile loop starts.
  bf16x8 qop[KS];
  {
    const bf16x8* qrow = reinterpret_cast<const bf16x8*>(
        static_cast<const uint16_t*>(a.q) + (static_cast<int64_t>(w.q0 + t) * a.hq + hq) * D);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (row_in) {
        qop[ks] = qrow[2 * ks + h];
      } else {
        const u32x4 z = {0u, 0u, 0u, 0u};
        qop[ks] = __builtin_bit_cast(bf16x8, z);
      }
    }
  }
  Ring kv;
  kv.init(a, w, wave, lane, s_pg);
  PageIds pages = {0, 0};
  if constexpr (PAGED) pages.stage(a, w, kTile, tid, NW * 64, s_pg);
  if constexpr (VERIFY) {
    const int step = lane < a.block ? a.step_map[w.b * a.block + lane] : 0;
    build_visibility<NW>(s_vis, step, a.num_ref[w.b], a.block, a.n_new, wave, lane);
  }
  // Every load the compiler knows of completes before the tile loads start (it
  // cannot see those, and a wait of its own would wait for the whole ring).
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();                             // staged page ids, s_bad, the masks' words
  uint64_t vis = 0;
  if constexpr (VERIFY) vis = row_in ? s_vis[t] : 0;

  const int nt = w.nt;
  const uint32_t ring0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
      (SIMSD_LDS void*)(&smem[0][0][0])));      // LDS byte address of slot 0
  constexpr uint32_t kSlotBytes = 2 * TILEB;
  auto is_new = [&](int it) __attribute__((always_inline)) { return VERIFY && w.t0 + it == w.s.tiles; };
  // Loads of tile `it` on their way: into its slot (bf16), or into registers (4 bits).
  auto fetch = [&](int it, uint32_t slot) __attribute__((always_inline)) {
    if (is_new(it)) {
      if constexpr (!FP4) issue_new<D, NW>(a, w, slot, wave, lane);
      return;
    }
    const TileKeys k = tile_keys(w.s, w.t0 + it, kTile);
    const int first_page = k.sink ? +pages.first_sink : +pages.first_win;
    if constexpr (FP4) {
      kv.load(k.k0, k.beg, k.end, first_page, s_pg);
    } else {
      kv.pg_first = first_page;
      kv.issue(slot, k.k0, k.end, s_pg, k.beg);
    }
  };
  // 4 bits: the fetched tile's values into its slot.
  auto unpack = [&](int it, uint32_t slot) __attribute__((always_inline)) {
    if constexpr (FP4) {
      if (is_new(it)) issue_new<D, NW>(a, w, slot, wave, lane);
      else kv.store(slot);
    }
  };
  if constexpr (FP4) {
    if (nt > 0) {
      fetch(0, ring0);
      unpack(0, ring0);
    }
    if (nt > 1) fetch(1, ring0 + kSlotBytes);
  } else {
#pragma unroll
    for (int j = 0; j < NBUF; ++j)
      if (j < nt) fetch(j, ring0 + j * kSlotBytes);
  }

  f32x16 o[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[c][j] = 0.f;
  float m_run = kNegInf, l_run = 0.f;
  const float sl2 = a.scale_log2;

  // Per-lane LDS read offsets (swizzled), as in the chunk attention.
  int koff[KS], voff[NB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) koff[ks] = n * ROWB + 16 * ((2 * ks + h) ^ swz<D>(n));
  {
    const int k = (lane & 15) >> 2, q = lane & 3, gg = (lane >> 4) & 1;
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int hl = 0; hl < 2; ++hl) {
        const int r = 8 * hl + 4 * h + k;
        const int L = 4 * c + 2 * gg + (q >> 1);
        voff[c][hl] = r * ROWB + 16 * (L ^ swz<D>(r)) + 8 * (q & 1);
      }
  }
  auto v_operand = [&](const SIMSD_LDS uint8_t* vblk, int c) __attribute__((always_inline)) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SIMSD_LDS s16x4*)(vblk + voff[c][0]));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SIMSD_LDS s16x4*)(vblk + voff[c][1]));
    const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
    return __builtin_bit_cast(bf16x8, (u32x4{l2[0], l2[1], h2[0], h2[1]}));
  };
  // Which of the 32 keys of half kb of tile `it` this lane's row sees.
  auto word = [&](int it, int kb) __attribute__((always_inline)) {
    if (is_new(it)) return static_cast<uint32_t>(vis >> (32 * kb));
    const TileKeys k = tile_keys(w.s, w.t0 + it, kTile);
    return seen_word(w.s, k, k.k0 + 32 * kb, limit, first);
  };

  // One tile: wait for it, free the slot of the previous tile for the next load (4
  // bits: put the next tile there), then its key blocks.
  auto tile = [&](auto masked, int it, int sl) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    if constexpr (FP4) {
      if (MASKED && is_new(it)) wait_vm<0>();
      lds_barrier();                           // all of tile `it` is in; the other slot is free
      if (it + 1 < nt) {
        unpack(it + 1, ring0 + (sl ^ 1) * kSlotBytes);
        if (it + 2 < nt) fetch(it + 2, ring0);
      }
    } else {
      // This wave's share of tile `it` has landed once at most the loads of the
      // younger tiles remain (vector memory completes in issue order).
      const int younger = min(nt - 1, max(NBUF - 1, it + NBUF - 2)) - it;
      if (NBUF >= 4 && younger >= 3) wait_vm<3 * Dma::PERW>();
      else if (NBUF >= 3 && younger >= 2) wait_vm<2 * Dma::PERW>();
      else if (younger >= 1) wait_vm<Dma::PERW>();
      else wait_vm<0>();
      lds_barrier();                           // all of tile `it` is in; slot of tile it-1 is free
      if (it >= 1 && it + NBUF - 1 < nt) fetch(it + NBUF - 1, ring0 + ((sl + NBUF - 1) % NBUF) * kSlotBytes);
    }
    const SIMSD_LDS uint8_t* sk = reinterpret_cast<const SIMSD_LDS uint8_t*>(ring0) + sl * kSlotBytes;
    const SIMSD_LDS uint8_t* sv = sk + TILEB;
    if constexpr (MASKED) {
      bool mine = false;
#pragma unroll
      for (int i = 0; i < TILEB / (NW * 64 * 16); ++i) {
        SIMSD_LDS u32x4* at = (SIMSD_LDS u32x4*)(sv + (i * NW * 64 + tid) * 16);
        u32x4 x = *at;
        if (wild(x[0]) || wild(x[1]) || wild(x[2]) || wild(x[3])) {
#pragma unroll
          for (int q = 0; q < 4; ++q) x[q] = tamed(x[q]);
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
    // No row of this wave sees a key of the tile (or it has no rows).
    if (MASKED && is_new(it)) {
      if (!wave_in) return;
    } else {
      const TileKeys k = tile_keys(w.s, w.t0 + it, kTile);
      if (k.k0 >= wave_end || (!k.sink && k.k0 + kTile <= wave_first && k.k0 >= w.s.near)) return;
    }

#pragma unroll
    for (int kb1 = 0; kb1 < 2 / KW; ++kb1) {
      const int kb = KW == 1 ? kb1 : kw;
      f32x16 s;
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = 0.f;
      // S^T = K Q^T.  Register j of s holds key 32*kb + 8*(j/4) + 4*h + j%4
      // of this lane's row.
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 ka = *reinterpret_cast<const SIMSD_LDS bf16x8*>(sk + 32 * kb * ROWB + koff[ks]);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qop[ks], s, 0, 0, 0);
      }
      if constexpr (MASKED) {
        const uint32_t seen = word(it, kb) >> (4 * h);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!(seen >> (8 * (j >> 2) + (j & 3)) & 1)) s[j] = kNegInf;
      }

      float mx = kNegInf;
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[j]);
      mx = xhalf_max(mx);
      const float m_new = fmaxf(m_run, mx * sl2);
      if (m_new > m_run + kLazy) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int c = 0; c < NB; ++c) o[c] *= alpha;
        m_run = m_new;
      }
      const float moff = m_run == kNegInf ? 0.f : m_run;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[j], sl2, -moff));
        s[j] = p;
        l_run += p;
      }

      // O^T += V^T P^T, two 16-key chunks per block.  (The weights go in as bf16, the
      // type of the other operand: half a step, 2^-8 of each at most, as the output's own
      // rounding is.  l_run adds them up in fp32.)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        u32x4 pw;
#pragma unroll
        for (int p = 0; p < 4; ++p) pw[p] = pack2(s[8 * hf + 2 * p], s[8 * hf + 2 * p + 1]);
        const bf16x8 pb = __builtin_bit_cast(bf16x8, pw);
        const SIMSD_LDS uint8_t* vblk = sv + (32 * kb + 16 * hf) * ROWB;
#pragma unroll
        for (int c = 0; c < NB; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(vblk, c), pb, o[c], 0, 0, 0);
      }
    }
  };

  // Tiles that every row sees whole, [full0, full1) of this work-group's, unrolled by
  // NBUF from a multiple of it so that ring slots are compile-time offsets; before and
  // after them the others.
  const int open0 = w.s.sink_tiles + max(0, (w.lim.first_last - w.s.win0 + kTile - 1) / kTile) - w.t0;
  const int open1 = w.s.sink_tiles + max(0, min(w.lim.limit_first, w.s.hi) - w.s.win0) / kTile - w.t0;
  const int full0 = min(max(open0, 0) + NBUF - 1, nt + NBUF - 1) / NBUF * NBUF;
  const int full1 = max(full0, min(open1, nt));
  for (int it = 0; it < min(full0, nt); ++it) tile(std::true_type{}, it, it % NBUF);
  for (int it0 = full0; it0 < full1; it0 += NBUF) {
#pragma unroll
    for (int u = 0; u < NBUF; ++u) {
      if (it0 + u >= full1) break;
      tile(std::false_type{}, it0 + u, u);
    }
  }
  for (int it = full1; it < nt; ++it) tile(std::true_type{}, it, it % NBUF);
  // The masked tiles with values that are not finite, again.
  {
    lds_barrier();                             // the ring is free (no load is pending)
    const int last = __builtin_amdgcn_readfirstlane(s_bad[1]);
    for (int it = __builtin_amdgcn_readfirstlane(s_bad[0]); it <= last; ++it) {
      if (it >= full0 && it < full1) continue;
      fetch(it, ring0);
      unpack(it, ring0);
      wait_vm<0>();
      lds_barrier();
      SIMSD_LDS uint8_t* sv = reinterpret_cast<SIMSD_LDS uint8_t*>(ring0) + TILEB;
      for (int i = tid; i < TILEB / 16; i += NW * 64) {
        SIMSD_LDS u32x4* at = (SIMSD_LDS u32x4*)(sv + i * 16);
        u32x4 x = *at;
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = code_of(x[q] & 0xffffu) | code_of(x[q] >> 16) << 16;
        *at = x;
      }
      lds_barrier();
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        f32x16 sum;
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[j] = 0.f;
        for (int ch = KW == 1 ? 0 : 2 * kw; ch < (KW == 1 ? 4 : 2 * kw + 2); ++ch) {   // 16-key chunks
          const uint32_t seen = word(it, ch >> 1) >> (16 * (ch & 1) + 4 * h);
          u32x4 sees;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const int key = 8 * (p >> 1) + 2 * (p & 1);
            sees[p] = (seen >> key & 1 ? 0x3f80u : 0u) | (seen >> key & 2 ? 0x3f800000u : 0u);
          }
          sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(sv + 16 * ch * ROWB, c),
                                                        __builtin_bit_cast(bf16x8, sees), sum, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (sum[j] != 0.f) o[c][j] += code_value(sum[j]);
      }
      lds_barrier();
    }
  }
  if constexpr (KW == 2) {
    __syncthreads();                           // the ring is free (no load is pending)
    // Merge the two key halves of each row through LDS (the tiles are free).
    constexpr int SLOT = NB * 16 + 2;
    SIMSD_LDS float* xs = reinterpret_cast<SIMSD_LDS float*>(ring0) + (rw * 64 + lane) * SLOT;
    if (kw == 1) {
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) xs[c * 16 + j] = o[c][j];
      xs[NB * 16] = m_run;
      xs[NB * 16 + 1] = l_run;
    }
    __syncthreads();
    if (kw == 0) {
      const float m1 = xs[NB * 16], l1 = xs[NB * 16 + 1];
      const float mm = fmaxf(m_run, m1);
      const float mref = mm == kNegInf ? 0.f : mm;
      const float a0 = __builtin_amdgcn_exp2f(m_run - mref), a1 = __builtin_amdgcn_exp2f(m1 - mref);
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] = o[c][j] * a0 + xs[c * 16 + j] * a1;
      l_run = l_run * a0 + l1 * a1;
      m_run = mm;
    }
  }
  const float l_tot = xhalf_sum(l_run);
  // Register j of o[c] holds dim 32*c + 8*(j/4) + 4*h + j%4 of this row.
  if (row_in && (KW == 1 || kw == 0)) {
    const int token = w.q0 + t;
    if (w.nsplit == 1) {
      const bool valid = VERIFY ? vis != 0 : limit > 0;   // (a slot sees itself, a padded one nothing)
      const float inv = valid ? 1.f / l_tot : 0.f;
      uint16_t* orow = static_cast<uint16_t*>(a.out) + (static_cast<int64_t>(token) * a.hq + hq) * D;
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          u32x2 v = {pack2(o[c][4 * q] * inv, o[c][4 * q + 1] * inv),
                     pack2(o[c][4 * q + 2] * inv, o[c][4 * q + 3] * inv)};
          if (VERIFY && !valid) v = u32x2{0u, 0u};
          *reinterpret_cast<u32x2*>(orow + 32 * c + 8 * q + 4 * h) = v;
        }
      if (a.lse && h == 0) a.lse[lse_at<VERIFY>(a, token, hq)] = valid ? log_sum(m_run, l_tot) : kNegInf;
    } else {
      const int64_t r = partial_row(a, w.split, token, hq);
      float* part = a.part + r * D;
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(part + 32 * c + 8 * q + 4 * h) =
              f32x4{o[c][4 * q], o[c][4 * q + 1], o[c][4 * q + 2], o[c][4 * q + 3]};
      if (h == 0) a.part_ml[r] = float2{m_run, l_tot};
    }
  }
}

template <int D, bool PAGED, bool FP4, bool VERIFY>
void launch_span_bf16(const SpanPlan& p, dim3 grid, const SpanArgs& a, hipStream_t st) {
  if (p.row_waves == 4) {
    hipLaunchKernelGGL((span_bf16_kernel<D, 4, 1, PAGED, FP4, VERIFY>), grid, dim3(256), 0, st, a);
  } else if (p.row_waves == 8) {
    hipLaunchKernelGGL((span_bf16_kernel<D, 8, 1, PAGED, FP4, VERIFY>), grid, dim3(512), 0, st, a);
  } else if constexpr (!FP4) {                 // (4 bits: fp4_rows_kernel)
    hipLaunchKernelGGL((span_bf16_kernel<D, 2, 2, PAGED, FP4, VERIFY>), grid, dim3(256), 0, st, a);
  }
}

template <int D, bool FP4, bool VERIFY>
void launch_span_d(const SpanPlan& p, const SpanArgs& a, hipStream_t st) {
  const dim3 grid(p.blocks * a.hkv, p.splits);
  if (a.block_table) launch_span_bf16<D, true, FP4, VERIFY>(p, grid, a, st);
  else launch_span_bf16<D, false, FP4, VERIFY>(p, grid, a, st);
  launch_span_merge<D, true, VERIFY>(p, a, kTile, st);
}

}  // namespace
}  // namespace simsd
