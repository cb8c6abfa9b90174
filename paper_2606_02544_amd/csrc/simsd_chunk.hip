// Attention of a ragged batch of new tokens over the cache on gfx950, under the
// block-causal mask of a block-diffusion model.
//
// Token i of a sequence's n new ones sits at position p = kv_len - n + i and sees
// the cached keys t < limit(p) = min(kv_len, (p / m + 1) * m), m the mask's block
// (1: causal; 0: all kv_len keys).  The new tokens' own keys are in the cache.
//
// Work decomposition: one work-group per (row block, KV head, key range).  The G
// query heads of a KV head and the tokens of a sequence are packed into rows
// (row = token * G + head), a row block takes up to 256 of them, and a key range is
// the whole of what the block's last row sees, or a chunk of it when there are too
// few blocks to fill the chip: then every range writes its unnormalised fp32 output
// with the running maximum and sum, and a second kernel joins them.  Row blocks are
// numbered without knowing the lengths on the host: sequence b's first block is
// floor(q_starts[b] * G / R) + b, which leaves room for every sequence's own blocks
// and at most one unused number a sequence (batches of up to 64 are counted on the
// device).  KV heads run fastest over the grid, so
// that the work-groups of one head land on the same XCDs and share their L2; blocks
// run from the last to the first, the ones with the most keys first.
//
// bf16 path: as the verification attention's (S^T = K Q^T and O^T = V^T P^T on
// v_mfma_f32_32x32x16_bf16, K and V tiles of 64 keys in a swizzled LDS ring filled
// by direct loads), with the rows' limits in place of its visibility words.  Tiles
// that every row of the block sees whole run a copy of the code without the mask.
#include <algorithm>
#include <type_traits>

#include "simsd_chunk_device.h"
#include "simsd_chunk_f32.h"

namespace simsd {
namespace {

// RW row waves of 32 rows each; KW = 2 pairs every row wave with a second wave that
// takes the other 32-key half of each tile.  The ring holds NBUF tiles.  (Group
// shapes and ring depths are the verification attention's, measured there.)
// What bounds it: with many rows the matrix cores and the softmax between them (4
// sequences of 2048 tokens over 14336 keys, 32/8 heads of 128: 1970 us, 1050 TFLOP/s; a
// large matrix product reaches 1133); with few, memory (64 single tokens over 512..32767
// keys: 812 us, 5.4 TB/s; one block of 4 over 1024 keys: 7 us of round trips).
template <int D, int RW, int KW, bool PAGED>
__global__ void __launch_bounds__(RW * KW * 64, 2) chunk_bf16_kernel(ChunkArgs a) {
  constexpr int NW = RW * KW;
  constexpr int NBUF = NW >= 8 ? 4 : 2;
  constexpr int NB = D / 32;                   // 32-dim output blocks
  constexpr int KS = D / 16;                   // k-steps of QK^T
  constexpr int ROWB = TileGeom<D>::ROWB;
  constexpr int TILEB = TileGeom<D>::TILEB;
  using Ring = ChunkRing<Bf16Tile<D>, NW, PAGED>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NBUF][2][TILEB];   // [slot][K, V]
  __shared__ int s_pg_arr[PAGED ? kMaxChunkPages : 1];
  __shared__ int s_bad[2];                     // first and last tile with values that are not finite
  SIMSD_LDS int* s_pg = (SIMSD_LDS int*)(&s_pg_arr[0]);

  Block w;
  if (!setup_block(a, w)) return;
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
  const int limit = row_in ? visible_keys(a, w.kv, w.n, t) : 0;
  // Keys past which no row of this wave sees anything: its last row's limit.
  const int wave_last = min(w.row0 + rw * 32 + 31, w.rows - 1);
  const int wave_end = w.row0 + rw * 32 < w.rows ? visible_keys(a, w.kv, w.n, wave_last / a.group) : 0;

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
  // Every load the compiler knows of completes before the tile loads start (it
  // cannot see those, and a wait of its own would wait for the whole ring).
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();                             // staged page ids, s_bad

  const int nt = w.kend > w.kbeg ? (w.kend - w.kbeg + kTile - 1) / kTile : 0;
  const uint32_t ring0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
      (SIMSD_LDS void*)(&smem[0][0][0])));      // LDS byte address of slot 0
  constexpr uint32_t kSlotBytes = 2 * TILEB;
#pragma unroll
  for (int j = 0; j < NBUF; ++j)
    if (j < nt) kv.issue(ring0 + j * kSlotBytes, w.kbeg + j * kTile, w.kend, s_pg);

  f32x16 o[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[c][j] = 0.f;
  float m_run = kNegInf, l_run = 0.f;
  const float sl2 = a.scale_log2;

  // Per-lane LDS read offsets (swizzled).  K operand of k-step ks: row n of a
  // 32-key block, chunk 2*ks + h.  V transpose reads: lane (g = lane/16,
  // k = (lane%16)/4, q = lane%4) reads 4 dims at column 32*c + 16*(g%2) + 4*q
  // of key row 4*h + k (lo) or 8 + 4*h + k (hi) of a 16-key chunk.
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

  // One tile: wait for it, free the slot of the previous tile for the next
  // load, then its key blocks.  `masked` tiles are those that some row of the
  // block does not see whole.
  auto tile = [&](auto masked, int it, int sl) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int k0 = w.kbeg + it * kTile;
    // This wave's share of tile `it` has landed once at most the loads of the
    // younger tiles remain (vector memory completes in issue order).
    const int younger = min(nt - 1, max(NBUF - 1, it + NBUF - 2)) - it;
    if (NBUF >= 4 && younger >= 3) wait_vm<3 * Ring::PERW>();
    else if (NBUF >= 3 && younger >= 2) wait_vm<2 * Ring::PERW>();
    else if (younger >= 1) wait_vm<Ring::PERW>();
    else wait_vm<0>();
    lds_barrier();                             // all of tile `it` is in; slot of tile it-1 is free
    if (it >= 1 && it + NBUF - 1 < nt) {
      const int nx = it + NBUF - 1;
      kv.issue(ring0 + ((sl + NBUF - 1) % NBUF) * kSlotBytes, w.kbeg + nx * kTile, w.kend, s_pg);
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
    if (k0 >= wave_end) return;

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
        const int seen = limit - k0 - 32 * kb - 4 * h;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (8 * (j >> 2) + (j & 3) >= seen) s[j] = kNegInf;
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

      // O^T += V^T P^T, two 16-key chunks per block.  Chunk hf of block kb
      // covers keys 32*kb + 16*hf + kappa(h, i), kappa(h, i) = 8*(i/4) + 4*h + i%4.
      // (The weights go in as bf16, the type of the other operand: half a step, 2^-8
      // of each at most, as the output's own rounding is.  l_run adds them up in fp32.)
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

  // Tiles that every row sees whole, unrolled by NBUF so that ring slots are
  // compile-time offsets; then the others.
  const int nfull = max(0, min(w.full, w.kend) - w.kbeg) / kTile;
  for (int it0 = 0; it0 < nfull; it0 += NBUF) {
#pragma unroll
    for (int u = 0; u < NBUF; ++u) {
      if (it0 + u >= nfull) break;
      tile(std::false_type{}, it0 + u, u);
    }
  }
  for (int it = nfull; it < nt; ++it) tile(std::true_type{}, it, it % NBUF);
  if (nfull < nt) {
    lds_barrier();                             // the ring is free (no load is pending)
    const int last = __builtin_amdgcn_readfirstlane(s_bad[1]);
    for (int it = __builtin_amdgcn_readfirstlane(s_bad[0]); it <= last; ++it) {
      kv.issue(ring0, w.kbeg + it * kTile, w.kend, s_pg);
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
          const int seen = limit - w.kbeg - it * kTile - 16 * ch - 4 * h;
          u32x4 sees;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const int key = 8 * (p >> 1) + 2 * (p & 1);
            sees[p] = (key < seen ? 0x3f80u : 0u) | (key + 1 < seen ? 0x3f800000u : 0u);
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
      const float inv = limit > 0 ? 1.f / l_tot : 0.f;
      uint16_t* orow = static_cast<uint16_t*>(a.out) + (static_cast<int64_t>(token) * a.hq + hq) * D;
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const u32x2 v = {pack2(o[c][4 * q] * inv, o[c][4 * q + 1] * inv),
                           pack2(o[c][4 * q + 2] * inv, o[c][4 * q + 3] * inv)};
          *reinterpret_cast<u32x2*>(orow + 32 * c + 8 * q + 4 * h) = v;
        }
      if (a.lse && h == 0)
        a.lse[static_cast<int64_t>(hq) * a.tokens + token] = limit > 0 ? log_sum(m_run, l_tot) : kNegInf;
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

// ----------------------------------------------------------------------------
// Joins the key ranges of a token's rows.  Grid: (token, groups of heads).  D / 4
// lanes hold a row, four dims each; WIDE: the four waves of a work-group share the
// ranges of one wave's rows (many ranges), else each has rows of its own.  Round trips
// bound it: 4 tokens in 9 ranges 3.8 us, 64 in 16 ranges 6.
// ----------------------------------------------------------------------------
template <int D, bool BF16, bool WIDE>
__global__ void __launch_bounds__(256) chunk_merge_kernel(ChunkArgs a) {
  constexpr int LPR = D / 4;                   // lanes per row
  constexpr int RPW = 64 / LPR;                // rows per wave
  constexpr int U = 4;                         // ranges loaded at a time
  __shared__ f32x4 xo[WIDE ? 256 : 1];
  __shared__ float2 xml[WIDE ? 256 : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int token = blockIdx.x;
  const int b = __builtin_amdgcn_readfirstlane(leading(a.batch, lane, [&](int i) { return a.q_starts[i + 1] <= token; }));
  if (b >= a.batch || token < a.q_starts[0]) return;
  const int q0 = a.q_starts[b], n = min(a.q_starts[b + 1], a.tokens) - q0;
  const int kv = min(max(a.kv_lens[b], 0), a.max_kv);
  const int head = blockIdx.y * (WIDE ? RPW : 4 * RPW) + (WIDE ? 0 : wave * RPW) + lane / LPR;
  const int d0 = 4 * (lane % LPR);
  const int i = token - q0;
  // The row's block is joined if its last row needed more than one range.
  const int hc = min(head, a.hq - 1);
  const int row = i * a.group + hc % a.group;
  const int last = min((row / a.rows_pb + 1) * a.rows_pb, n * a.group) - 1;
  const bool joined = visible_keys(a, kv, n, last / a.group) > a.chunk;
  const int limit = visible_keys(a, kv, n, i);
  const int ranges = (limit + a.chunk - 1) / a.chunk;
  const int most = joined ? ranges : 0;
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
  const float inv = limit > 0 ? 1.f / l : 0.f;
  const int64_t at = (static_cast<int64_t>(token) * a.hq + head) * D + d0;
  if constexpr (BF16)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) =
        u32x2{pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = o * inv;
  if (a.lse && d0 == 0)
    a.lse[static_cast<int64_t>(head) * a.tokens + token] = limit > 0 ? log_sum(m, l) : kNegInf;
}

template <int D, bool PAGED>
void launch_bf16(const ChunkPlan& p, dim3 grid, const ChunkArgs& a, hipStream_t st) {
  switch (p.row_waves) {
    case 2: hipLaunchKernelGGL((chunk_bf16_kernel<D, 2, 2, PAGED>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((chunk_bf16_kernel<D, 4, 1, PAGED>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((chunk_bf16_kernel<D, 8, 1, PAGED>), grid, dim3(512), 0, st, a); break;
  }
}

template <int D, bool PAGED>
void launch_f32(const ChunkPlan& p, dim3 grid, const ChunkArgs& a, hipStream_t st) {
  switch (p.rows_pb) {
    case 16: hipLaunchKernelGGL((chunk_f32_kernel<D, 1, PAGED>), grid, dim3(256), 0, st, a); break;
    case 32: hipLaunchKernelGGL((chunk_f32_kernel<D, 2, PAGED>), grid, dim3(256), 0, st, a); break;
    case 64: hipLaunchKernelGGL((chunk_f32_rows_kernel<D, 1, PAGED>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((chunk_f32_rows_kernel<D, 2, PAGED>), grid, dim3(256), 0, st, a); break;
  }
}

template <int D>
void launch_chunk_d(const ChunkPlan& p, bool bf16, const ChunkArgs& a, hipStream_t st) {
  const dim3 grid(p.blocks * a.hkv, p.splits);
  if (bf16) {
    if (a.block_table) launch_bf16<D, true>(p, grid, a, st);
    else launch_bf16<D, false>(p, grid, a, st);
  } else {
    if (a.block_table) launch_f32<D, true>(p, grid, a, st);
    else launch_f32<D, false>(p, grid, a, st);
  }
  if (p.splits == 1) return;
  constexpr int RPW = 64 / (D / 4);
  const bool wide = p.splits > 4;
  const int per = wide ? RPW : 4 * RPW;
  const dim3 mgrid(a.tokens, (a.hq + per - 1) / per);
  if (bf16) {
    if (wide) hipLaunchKernelGGL((chunk_merge_kernel<D, true, true>), mgrid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((chunk_merge_kernel<D, true, false>), mgrid, dim3(256), 0, st, a);
  } else {
    if (wide) hipLaunchKernelGGL((chunk_merge_kernel<D, false, true>), mgrid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((chunk_merge_kernel<D, false, false>), mgrid, dim3(256), 0, st, a);
  }
}

}  // namespace

hipError_t launch_chunk(const simsd_chunk_desc& d, const ChunkPlan& p, const ChunkArgs& a, hipStream_t st) {
  if (d.head_dim == 128) launch_chunk_d<128>(p, d.dtype == SIMSD_BF16, a, st);
  else launch_chunk_d<64>(p, d.dtype == SIMSD_BF16, a, st);
  return hipGetLastError();
}

}  // namespace simsd
