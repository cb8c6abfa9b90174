// Attention of few rows (up to 64) over a cache held in 4 bits.
//
// Four waves share a row block of RB * 32 rows, and each takes every fourth 32-key tile
// of the list on its own, with a running output, maximum and sum of its own; the four
// states merge at the end.  No wave waits for another before that: the codes go straight
// into the registers that feed the first product, and the values through an LDS tile of
// the wave's own (LDS works a wave's accesses off in their order).
//
//   S^T = K Q^T on v_mfma_f32_32x32x16_bf16: lane (n = lane % 32, h = lane / 32) holds
//     dims 8 ks + [0, 8) of its half of key n's dims in step ks: the half is 16 bytes of
//     codes and a scale for each 32 dims, and step ks is one word of them.  The queries'
//     operands take their dims in the same order (from LDS for RB = 2).
//   O^T += V^T P^T as in the chunk attention: the values in bf16 in a swizzled LDS tile,
//     read back transposed.
// Codes are loaded a tile (a wave's, four in all) ahead.
//
// Why waves on their own: with one tile of 64 keys shared by the row waves, as in
// simsd_span_kernel.h, a tile's bytes are a quarter of bf16's and its two barriers are
// not: 64 single tokens of uneven length (1.06 M keys, 8 KV heads of 128) took 421 us and
// 64 verifications over as many 621; this kernel takes 256 to 288 and 400 to 453.
//
// What bounds it.  32 rows (12 waves a CU): HBM, 397 ns for 64 keys a CU, 5.4 TB/s; of
// 262 us of a pass there 232 are that and the rest uneven ends and the start of a work-group (8 to
// 12 us: lengths, page ids, codes, one after the other).  64 rows (8 waves a CU, 250
// registers): 650 ns for 64 keys, 300 vector instructions and 32 products a wave and
// tile; without the loads it takes 474.  Priorities of waves, other orders of products
// and conversions and loads two tiles ahead gave nothing.
#pragma once

#include "simsd_fp4.h"
#include "simsd_span.h"

namespace simsd {
namespace {

constexpr int kFewTile = 32;     // keys of a tile

template <int D, int RB, bool PAGED, bool VERIFY>
__global__ void __launch_bounds__(256, RB == 1 ? 3 : 2) fp4_rows_kernel(SpanArgs a) {
  constexpr int NW = 4, TK = kFewTile;
  constexpr int NB = D / 32;                   // 32-dim output blocks
  constexpr int KS = D / 16;                   // k-steps of the scores
  constexpr int CH = D / 64;                   // 16-byte chunks of codes (and scales) of a lane's half
  constexpr int ROWB = TileGeom<D>::ROWB;
  constexpr int VB = TK * ROWB;                // a wave's tile of values
  constexpr bool QLDS = RB > 1;
  constexpr int XB = NB * 16 * 64 * 4 + 2 * 64 * 4;     // one state of a 32-row block
  constexpr int kBytes = NW * VB > 2 * XB ? NW * VB : 2 * XB;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t s_q[QLDS ? RB * 32 * ROWB : 16];
  __shared__ int s_pg_arr[PAGED ? kMaxChunkPages : 1];
  __shared__ uint64_t s_vis[VERIFY ? kMaxNew : 1];
  SIMSD_LDS int* s_pg = (SIMSD_LDS int*)(&s_pg_arr[0]);

  SpanBlock w;
  if (!setup_span<VERIFY>(a, w, TK)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const SIMSD_LDS uint8_t* sq = (const SIMSD_LDS uint8_t*)(&s_q[0]);
  const uint32_t vt0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((SIMSD_LDS void*)(&smem[0]))) + wave * VB;
  SIMSD_LDS uint8_t* vt = reinterpret_cast<SIMSD_LDS uint8_t*>(vt0);

  // The rows of this lane: 32 rb + n of the block.
  int limit[RB], first[RB];
  uint64_t vis[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int m = w.row0 + 32 * rb + n;
    const bool in = m < w.rows;
    const int t = in ? m / a.group : 0;
    limit[rb] = VERIFY ? w.kv : in ? visible_keys(a, w.kv, w.n, t) : 0;
    first[rb] = VERIFY ? w.lim.first : in ? first_at(a.mask_block, a.window, w.kv - w.n + t) : 0;
    vis[rb] = 0;
  }
  // Queries: chunk c (8 dims) of a row, in order.  Step ks of lane half h is chunk h * KS + ks.
  bf16x8 qop[QLDS ? 1 : KS];
  auto q_chunk = [&](int row, int c) __attribute__((always_inline)) {
    const int m = w.row0 + row;
    if (m >= w.rows) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      return __builtin_bit_cast(bf16x8, z);
    }
    const int64_t at = static_cast<int64_t>(w.q0 + m / a.group) * a.hq + w.kvh * a.group + m % a.group;
    return reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(a.q) + at * D)[c];
  };
  if constexpr (QLDS) {
    for (int i = tid; i < RB * 32 * (D / 8); i += NW * 64) {
      const int row = i / (D / 8), c = i % (D / 8);
      *(SIMSD_LDS bf16x8*)((SIMSD_LDS uint8_t*)sq + row * ROWB + 16 * (c ^ swz<D>(row))) = q_chunk(row, c);
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qop[ks] = q_chunk(n, h * KS + ks);
  }

  PageIds pages = {0, 0};
  if constexpr (PAGED) pages.stage(a, w, TK, tid, NW * 64, s_pg);
  if constexpr (VERIFY) {
    const int step = lane < a.block ? a.step_map[w.b * a.block + lane] : 0;
    build_visibility<NW>(s_vis, step, a.num_ref[w.b], a.block, a.n_new, wave, lane);
  }
  __syncthreads();                             // page ids, queries, the masks' words
  if constexpr (VERIFY) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      if (w.row0 + 32 * rb + n < w.rows) vis[rb] = s_vis[(w.row0 + 32 * rb + n) / a.group];
  }

  // This lane's half of a cached key's codes and scales.
  const int64_t seq = PAGED ? 0 : w.b;
  const uint8_t* kc = static_cast<const uint8_t*>(a.k_cache) + seq * a.cs_seq + w.kvh * a.cs_head;
  const uint8_t* vc = static_cast<const uint8_t*>(a.v_cache) + seq * a.cs_seq + w.kvh * a.cs_head;
  const uint8_t* ksc = a.k_scales + seq * a.ss_seq + w.kvh * a.ss_head;
  const uint8_t* vsc = a.v_scales + seq * a.ss_seq + w.kvh * a.ss_head;
  const int cached = min(w.t0 + w.nt, w.s.tiles) - w.t0;    // cached tiles of this work-group
  const int items = cached > wave ? (cached - wave + NW - 1) / NW : 0;
  auto list = [&](int it) __attribute__((always_inline)) { return tile_keys(w.s, w.t0 + wave + NW * it, TK); };

  // A tile's codes and scales in registers: lane (n, h) holds its half of key n's codes and
  // of its value's, and all the scales of the key (h = 0) or of the value (h = 1).  Scales
  // that lie as the codes do, a sixteenth of their strides, of which none needs more than
  // 32 bits, take the fewest products of 64 bits.
  u32x4 kx[CH], vx[CH];
  uint32_t scale = 0;
  auto load = [&](int it) __attribute__((always_inline)) {
    const TileKeys k = list(it);
    const int key = max(k.beg, min(k.k0 + n, k.end - 1));
    int id = 0, in = key;
    if (PAGED) {
      const int pg = a.page_shift >= 0 ? key >> a.page_shift : key / a.page_size;
      id = s_pg[pg - (k.sink ? +pages.first_sink : +pages.first_win)];
      in = a.page_shift >= 0 ? key - (pg << a.page_shift) : key - pg * a.page_size;
    }
    int64_t c, s;
    if (a.scales_alike) {
      c = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(in)) * static_cast<uint32_t>(a.cs_tok));
      if (PAGED) c += static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(id)) * static_cast<uint32_t>(a.cs_seq));
      s = c >> 4;
    } else {
      c = in * a.cs_tok;
      s = in * a.ss_tok;
      if (PAGED) {
        c += id * a.cs_seq;
        s += id * a.ss_seq;
      }
    }
    const uint8_t* sc = (h ? vsc : ksc) + s;
    c += h * (D / 4);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      kx[i] = *reinterpret_cast<const u32x4*>(kc + c + 16 * i);
      vx[i] = *reinterpret_cast<const u32x4*>(vc + c + 16 * i);
    }
    if constexpr (CH == 2) scale = *reinterpret_cast<const uint32_t*>(sc);
    else scale = *reinterpret_cast<const uint16_t*>(sc);
  };
  // Scale byte i (of CH) of this lane's half of the key, of the value.
  auto split_scales = [&](uint32_t (&ks)[CH], uint32_t (&vs)[CH]) __attribute__((always_inline)) {
    const auto both = __builtin_amdgcn_permlane32_swap(scale, scale, false, false);   // the keys', in both halves; the values'
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      ks[i] = both[0] >> (8 * (h * CH + i)) & 0xff;
      vs[i] = both[1] >> (8 * (h * CH + i)) & 0xff;
    }
  };
  if (items > 0) load(0);

  f32x16 o[RB][NB];
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[rb][c][j] = 0.f;
    m_run[rb] = kNegInf;
    l_run[rb] = 0.f;
  }
  const float sl2 = a.scale_log2;

  // LDS offsets.  Chunk c (8 dims) of row r lies at chunk c ^ swz(r), so the chunks of a
  // lane are its first one's place with their number's bits turned: one register, which
  // is hidden from the compiler in every tile, or it would hold every offset.
  uint32_t put = n * ROWB + 16 * ((h * KS) ^ swz<D>(n));      // this lane's half of key n (or of query n)
  uint32_t get[2];                             // transpose reads (as in the chunk attention)
  {
    const int k = (lane & 15) >> 2, q = lane & 3, gg = (lane >> 4) & 1;
#pragma unroll
    for (int hl = 0; hl < 2; ++hl) {
      const int r = 8 * hl + 4 * h + k;
      get[hl] = r * ROWB + 16 * ((2 * gg + (q >> 1)) ^ swz<D>(r)) + 8 * (q & 1);
    }
  }
  auto put_v = [&](int c, u32x4 x) __attribute__((always_inline)) { *(SIMSD_LDS u32x4*)(vt + (put ^ (16 * c))) = x; };
  auto v_operand = [&](int hf, int c) __attribute__((always_inline)) {
    const SIMSD_LDS uint8_t* at = vt + 16 * hf * ROWB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SIMSD_LDS s16x4*)(at + (get[0] ^ (64 * c))));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SIMSD_LDS s16x4*)(at + (get[1] ^ (64 * c))));
    const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
    return __builtin_bit_cast(bf16x8, (u32x4{l2[0], l2[1], h2[0], h2[1]}));
  };
  // The scores of a tile whose keys are in kop.
  auto scores = [&](const bf16x8 (&kop)[KS], f32x16 (&s)[RB]) __attribute__((always_inline)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int j = 0; j < 16; ++j) s[rb][j] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        bf16x8 qx;
        if constexpr (QLDS)
          qx = *reinterpret_cast<const SIMSD_LDS bf16x8*>(sq + 32 * rb * ROWB + (put ^ (16 * ks)));
        else
          qx = qop[ks];
        s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[ks], qx, s[rb], 0, 0, 0);
      }
  };
  // Their softmax, and the product with the values in the wave's LDS tile.  seen(rb): the
  // word of keys that this lane's row sees, where `masked`.
  auto products = [&](f32x16 (&s)[RB], bool masked, auto seen) __attribute__((always_inline)) {
    if (masked) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const uint32_t see = seen(rb) >> (4 * h);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!(see >> (8 * (j >> 2) + (j & 3)) & 1)) s[rb][j] = kNegInf;
      }
    }
    float m_new[RB];
    bool grown = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float mx = kNegInf;
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[rb][j]);
      m_new[rb] = fmaxf(m_run[rb], xhalf_max(mx) * sl2);
      grown |= m_new[rb] > m_run[rb] + kLazy;
    }
    if (__any(grown)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        if (m_new[rb] > m_run[rb] + kLazy) {
          const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - m_new[rb]);
          l_run[rb] *= alpha;
#pragma unroll
          for (int c = 0; c < NB; ++c) o[rb][c] *= alpha;
          m_run[rb] = m_new[rb];
        }
    }
    float moff[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) moff[rb] = m_run[rb] == kNegInf ? 0.f : m_run[rb];
    // Sixteen keys at a time: their weights (in bf16, as in the chunk attention), and while
    // the matrix cores take them the next ones'.
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      bf16x8 pb[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        u32x4 pw;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          float x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[e] = __builtin_amdgcn_exp2f(fmaf(s[rb][8 * hf + 2 * p + e], sl2, -moff[rb]));
            l_run[rb] += x[e];
          }
          pw[p] = pack2(x[0], x[1]);
        }
        pb[rb] = __builtin_bit_cast(bf16x8, pw);
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const bf16x8 vx = v_operand(hf, c);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          o[rb][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vx, pb[rb], o[rb][c], 0, 0, 0);
      }
    }
  };
  // The codes of values in the LDS tile, added to the rows that see them (see code_value).
  auto add_codes = [&](auto seen) __attribute__((always_inline)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        f32x16 sum;
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[j] = 0.f;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const uint32_t see = seen(rb) >> (16 * hf + 4 * h);
          u32x4 ones;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const int key = 8 * (p >> 1) + 2 * (p & 1);
            ones[p] = (see >> key & 1 ? 0x3f80u : 0u) | (see >> key & 2 ? 0x3f800000u : 0u);
          }
          sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(hf, c), __builtin_bit_cast(bf16x8, ones), sum, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (sum[j] != 0.f) o[rb][c][j] += code_value(sum[j]);
      }
  };

  int bad_first = 0x7fffffff, bad_last = -1;   // masked tiles with values that are not finite
  for (int it = 0; it < items; ++it) {
    asm volatile("" : "+v"(put), "+v"(get[0]), "+v"(get[1]) :: "memory");
    const TileKeys k = list(it);
    const bool masked = k.sink | (k.k0 + TK > w.lim.limit_first) | (k.k0 < w.lim.first_last);
    uint32_t ks[CH], vs[CH];
    split_scales(ks, vs);
    if (masked) {
      bool mine = false;                       // (253 and 254 hold values past bf16's range, and others)
#pragma unroll
      for (int i = 0; i < CH; ++i) mine |= vs[i] >= 253u;
      if (__any(mine)) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (vs[i] >= 253u) {
#pragma unroll
            for (int j = 0; j < 4; ++j) vx[i][j] = fp4_finite(vx[i][j], vs[i] == 253u ? 1u : 0u);
            if (vs[i] == 255u) vs[i] = 0u;
          }
        bad_first = min(bad_first, it);
        bad_last = it;
      }
    }
    // The keys' products, and between them the values' way into LDS and the next loads.
    f32x16 s[RB];
    bf16x8 kop[KS];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kop[4 * i + j] = __builtin_bit_cast(bf16x8, fp4_values(kx[i][j], ks[i]));
    u32x4 v[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) v[i] = vx[i];
    load(min(it + 1, items - 1));
    scores(kop, s);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) put_v(4 * i + j, fp4_values(v[i][j], vs[i]));
#pragma unroll
    for (int i = 0; i < KS * RB; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a product
      __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);   // vector instructions
    }
    asm volatile("" ::: "memory");             // (written before it is read back)
    products(s, masked, [&](int rb) __attribute__((always_inline)) { return seen_word(w.s, k, k.k0, limit[rb], first[rb]); });
  }
  // The masked tiles with such values, again.
  for (int it = bad_first; it <= bad_last; ++it) {
    const TileKeys k = list(it);
    if (!(k.sink | (k.k0 + TK > w.lim.limit_first) | (k.k0 < w.lim.first_last))) continue;
    load(it);
    uint32_t ks[CH], vs[CH];
    split_scales(ks, vs);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 x = fp4_values(vx[i][j], vs[i]);
#pragma unroll
        for (int p = 0; p < 4; ++p) x[p] = code_of(x[p] & 0xffffu) | code_of(x[p] >> 16) << 16;
        put_v(4 * i + j, x);
      }
    }
    asm volatile("" ::: "memory");
    add_codes([&](int rb) __attribute__((always_inline)) { return seen_word(w.s, k, k.k0, limit[rb], first[rb]); });
  }
  if constexpr (VERIFY) {
    // The new slots (the list's last tile, of 64): 32 of them a wave, bf16.
    const int half = wave == NW - 1 ? 0 : wave == NW - 2 ? 1 : 2;
    if (w.t0 + w.nt > w.s.tiles && 32 * half < a.n_new) {
      const int64_t at = (static_cast<int64_t>(w.q0 + min(32 * half + n, a.n_new - 1)) * a.hkv + w.kvh) * D + h * (D / 2);
      const u32x4* kr = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.k_new) + at);
      const u32x4* vr = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.v_new) + at);
      bf16x8 kop[KS];
      bool mine = false;
      asm volatile("" ::: "memory");
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        kop[c] = __builtin_bit_cast(bf16x8, kr[c]);
        u32x4 x = vr[c];
        if (wild(x[0]) || wild(x[1]) || wild(x[2]) || wild(x[3])) {
#pragma unroll
          for (int p = 0; p < 4; ++p) x[p] = tamed(x[p]);
          mine = true;
        }
        put_v(c, x);
      }
      asm volatile("" ::: "memory");
      auto seen = [&](int rb) __attribute__((always_inline)) { return static_cast<uint32_t>(vis[rb] >> (32 * half)); };
      f32x16 s[RB];
      scores(kop, s);
      products(s, true, seen);
      if (__any(mine)) {
#pragma unroll
        for (int c = 0; c < KS; ++c) {
          u32x4 x = vr[c];
#pragma unroll
          for (int p = 0; p < 4; ++p) x[p] = code_of(x[p] & 0xffffu) | code_of(x[p] >> 16) << 16;
          put_v(c, x);
        }
        asm volatile("" ::: "memory");
        add_codes(seen);
      }
    }
  }

  // Merge of the four waves' states, two by two, one 32-row block at a time.
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int step = 2; step >= 1; --step) {
      __syncthreads();                         // the tiles, or the last states, have been read
      SIMSD_LDS float* xs = (SIMSD_LDS float*)(&smem[0]) + (wave & 1) * (XB / 4);
      if (step == 2 ? wave >= 2 : wave == 1) {
        if (step == 1) xs = (SIMSD_LDS float*)(&smem[0]);
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int j = 0; j < 16; ++j) xs[(c * 16 + j) * 64 + lane] = o[rb][c][j];
        xs[NB * 16 * 64 + lane] = m_run[rb];
        xs[NB * 16 * 64 + 64 + lane] = l_run[rb];
      }
      __syncthreads();
      if (step == 2 ? wave < 2 : wave == 0) {
        const float m1 = xs[NB * 16 * 64 + lane], l1 = xs[NB * 16 * 64 + 64 + lane];
        const float mm = fmaxf(m_run[rb], m1);
        const float mref = mm == kNegInf ? 0.f : mm;
        const float a0 = __builtin_amdgcn_exp2f(m_run[rb] - mref), a1 = __builtin_amdgcn_exp2f(m1 - mref);
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[rb][c][j] = o[rb][c][j] * a0 + xs[(c * 16 + j) * 64 + lane] * a1;
        l_run[rb] = l_run[rb] * a0 + l1 * a1;
        m_run[rb] = mm;
      }
    }
  }
  if (wave != 0) return;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l_tot = xhalf_sum(l_run[rb]);
    const int m = w.row0 + 32 * rb + n;
    if (m >= w.rows) continue;
    // Register j of o[rb][c] holds dim 32*c + 8*(j/4) + 4*h + j%4 of this row.
    const int token = w.q0 + m / a.group, hq = w.kvh * a.group + m % a.group;
    if (w.nsplit == 1) {
      const bool valid = VERIFY ? vis[rb] != 0 : limit[rb] > 0;
      const float inv = valid ? 1.f / l_tot : 0.f;
      uint16_t* orow = static_cast<uint16_t*>(a.out) + (static_cast<int64_t>(token) * a.hq + hq) * D;
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          u32x2 v = {pack2(o[rb][c][4 * q] * inv, o[rb][c][4 * q + 1] * inv),
                     pack2(o[rb][c][4 * q + 2] * inv, o[rb][c][4 * q + 3] * inv)};
          if (VERIFY && !valid) v = u32x2{0u, 0u};
          *reinterpret_cast<u32x2*>(orow + 32 * c + 8 * q + 4 * h) = v;
        }
      if (a.lse && h == 0) a.lse[lse_at<VERIFY>(a, token, hq)] = valid ? log_sum(m_run[rb], l_tot) : kNegInf;
    } else {
      const int64_t r = partial_row(a, w.split, token, hq);
      float* part = a.part + r * D;
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(part + 32 * c + 8 * q + 4 * h) =
              f32x4{o[rb][c][4 * q], o[rb][c][4 * q + 1], o[rb][c][4 * q + 2], o[rb][c][4 * q + 3]};
      if (h == 0) a.part_ml[r] = float2{m_run[rb], l_tot};
    }
  }
}

template <int D, int RB, bool VERIFY>
void launch_fp4_rows(const SpanPlan& p, const SpanArgs& a, hipStream_t st) {
  const dim3 grid(p.blocks * a.hkv, p.splits);
  if (a.block_table) hipLaunchKernelGGL((fp4_rows_kernel<D, RB, true, VERIFY>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((fp4_rows_kernel<D, RB, false, VERIFY>), grid, dim3(256), 0, st, a);
  launch_span_merge<D, true, VERIFY>(p, a, kFewTile, st);
}

}  // namespace
}  // namespace simsd
