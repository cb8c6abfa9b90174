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

#include "simsd_device.h"
#include "simsd_ops_kernels.h"
#include "simsd_search.h"

namespace simsd {
namespace {

constexpr int kCode1 = 256, kCode2 = 65536;   // see code_value

// Where a work-group's rows and keys are.
struct Block {
  int b, q0, n;                  // sequence, its first token, its new tokens
  int row0, rows;                // first row of the block in the sequence; rows of the sequence
  int kv;                        // cached length
  int kvh, split, nsplit;        // KV head; this key range of how many
  int kbeg, kend;                // keys of this range that some row sees
  int full;                      // keys every row of the block sees
};

// Keys that token i of the sequence sees.
__device__ inline int visible_keys(const ChunkArgs& a, int kv, int n, int i) {
  const int pos = kv - n + i;
  if (pos < 0) return 0;
  return a.mask_block ? min(kv, (pos / a.mask_block + 1) * a.mask_block) : kv;
}

// Number of the first row block of the sequence that starts at token q0, in
// batches of more than 64.
__device__ inline int first_block(const ChunkArgs& a, int q0, int b) { return q0 * a.group / a.rows_pb + b; }

// The sequence and row block of number `blk`; false if there is none.
//
// Up to 64 sequences: a lane each; blocks are numbered from the sequence with the
// most keys down, and from the last rows of each, so that the work-groups with the
// most work start first and the last ones to start are short.  (24 sequences of 1..351
// new tokens over 101..6007 keys, 256-row blocks: 360 us in the order of the batch, 304
// in this one.)  More sequences: in the order of the batch from its end, each starting
// at first_block(), whose numbers rise by one a sequence at least.
__device__ inline bool find_block(const ChunkArgs& a, int blk, int lane, Block& w, int* rb) {
  if (a.batch <= 64) {
    const int j = min(lane, a.batch - 1);
    const int q0 = a.q_starts[j], q1 = min(a.q_starts[j + 1], a.tokens), kv = min(max(a.kv_lens[j], 0), a.max_kv);
    const int nb = lane < a.batch && q1 > q0 ? ((q1 - q0) * a.group + a.rows_pb - 1) / a.rows_pb : 0;
    int first = 0;                               // blocks of the sequences before this one
    for (int i = 0; i < a.batch; ++i) {
      const int k = __builtin_amdgcn_readlane(kv, i), n = __builtin_amdgcn_readlane(nb, i);
      first += k > kv || (k == kv && i < lane) ? n : 0;
    }
    const uint64_t in = __ballot(blk >= first && blk < first + nb);
    if (!in) return false;
    const int l = __builtin_ctzll(in);
    w.b = l;
    w.q0 = __builtin_amdgcn_readlane(q0, l);
    w.n = __builtin_amdgcn_readlane(q1, l) - w.q0;
    w.kv = __builtin_amdgcn_readlane(kv, l);
    *rb = __builtin_amdgcn_readlane(nb - 1 + first, l) - blk;
    return w.q0 >= 0;
  }
  blk = a.blocks - 1 - blk;
  const int n = leading(a.batch, lane, [&](int b) { return first_block(a, a.q_starts[b], b) <= blk; });
  if (n == 0) return false;
  w.b = __builtin_amdgcn_readfirstlane(n - 1);
  w.q0 = a.q_starts[w.b];
  w.n = min(a.q_starts[w.b + 1], a.tokens) - w.q0;
  w.kv = min(max(a.kv_lens[w.b], 0), a.max_kv);
  *rb = blk - first_block(a, w.q0, w.b);
  return w.q0 >= 0;
}

__device__ inline bool setup_block(const ChunkArgs& a, Block& w) {
  w.kvh = blockIdx.x % a.hkv;
  w.split = blockIdx.y;
  int rb, rank = static_cast<int>(blockIdx.x) / a.hkv;
  if (a.fold) {
    const int place = rank, twice = a.blocks - a.fold;   // of the first `fold`, the first `twice` get a second
    rank = place >= a.fold ? a.blocks - 1 - (place - a.fold) : place < twice ? a.fold - twice + place : place - twice;
  }
  if (!find_block(a, rank, threadIdx.x & 63, w, &rb)) return false;
  w.rows = w.n * a.group;
  w.row0 = rb * a.rows_pb;
  if (w.row0 >= w.rows) return false;
  const int last = min(w.row0 + a.rows_pb, w.rows) - 1;
  const int seen = visible_keys(a, w.kv, w.n, last / a.group);
  w.nsplit = max(1, (seen + a.chunk - 1) / a.chunk);
  if (w.split >= w.nsplit) return false;
  w.kbeg = w.split * a.chunk;
  w.kend = min(seen, w.kbeg + a.chunk);
  w.full = visible_keys(a, w.kv, w.n, w.row0 / a.group);
  return true;
}

// Log-sum-exp of a row from its maximum (log2 units) and sum.  (The hardware's
// logarithm: 2^-22 off, what an fp32 log-sum-exp of 4 or more is rounded by anyway.)
__device__ inline float log_sum(float m, float l) { return (m + __log2f(l)) * kLn2; }

// Partials: O[split][token][head][D] fp32, then (max, sum)[split][token][head].
__device__ inline int64_t partial_row(const ChunkArgs& a, int split, int token, int head) {
  return (static_cast<int64_t>(split) * a.tokens + token) * a.hq + head;
}

// ----------------------------------------------------------------------------
// bf16 MFMA kernel
// ----------------------------------------------------------------------------
// Tiles in LDS: bf16, 64 keys, swizzled for the transpose reads; fp32, 32 keys, chunk
// c of row r at c ^ (r mod 8), so that the eight rows that eight lanes read at one
// chunk lie in different banks.
template <int D>
struct Bf16Tile {
  static constexpr int KEYS = kTile, ROWB = TileGeom<D>::ROWB, ELEM = 2;
  static __device__ inline int swizzle(int r) { return swz<D>(r); }
};
template <int D>
struct F32Tile {
  static constexpr int KEYS = 32, ROWB = 4 * D, ELEM = 4;
  static __device__ inline int swizzle(int r) { return r & 7; }
};

// Streams K/V tiles of a key range into a ring of LDS tile slots with direct
// loads, split between the waves by instruction.  One instruction covers RPI key
// rows of one tensor; lane i writes chunk position i % CPR of row i / CPR of its
// block and so fetches logical chunk (i % CPR) ^ swz(row).  Full tiles take a
// wave-uniform base an instruction plus a fixed lane offset (paged: an instruction's
// rows lie in one page when RPI divides the page size); other tiles, and rows past
// the range's last key, which read that key instead, an address a lane.
template <typename Tile, int NW, bool PAGED>
struct ChunkRing {
  static constexpr int ROWB = Tile::ROWB, KEYS = Tile::KEYS, TILEB = KEYS * ROWB;
  static constexpr int CPR = ROWB / 16;        // 16-byte chunks per key row
  static constexpr int RPI = 1024 / ROWB;      // key rows per instruction
  static constexpr int IPT = KEYS / RPI;       // instructions per tensor per tile
  static constexpr int PERW = 2 * IPT / NW;    // instructions per wave per tile
  static_assert(PERW >= 1 && (2 * IPT) % NW == 0, "tile instructions split evenly over the waves");

  const char* kc;         // caches, offset to this KV head
  const char* vc;
  int64_t seqoff;         // contiguous: this sequence's cache offset (bytes)
  int64_t tokb, pageb;    // bytes per token, per page
  uint32_t voff[PERW];    // lane offset of instruction i (bytes)
  int row[PERW], chunk[PERW];
  int wave, lane, P, lgP, pg_first;
  bool fast;              // full tiles take the uniform-base path

  __device__ __attribute__((always_inline)) void init(const ChunkArgs& a, const Block& w, int wave_, int lane_, SIMSD_LDS int* s_pg) {
    wave = wave_;
    lane = lane_;
    const int64_t hoff = static_cast<int64_t>(w.kvh) * a.cs_head * Tile::ELEM;
    kc = static_cast<const char*>(a.k_cache) + hoff;
    vc = static_cast<const char*>(a.v_cache) + hoff;
    tokb = a.cs_tok * Tile::ELEM;
    // Lane offsets of an instruction must fit 32 bits: RPI rows of tokb bytes.
    fast = tokb < (int64_t{1} << 25);
    if (PAGED) {
      P = a.page_size;
      lgP = a.page_shift;
      pageb = a.cs_seq * Tile::ELEM;
      pg_first = w.kbeg / P;
      const int npg = w.kend > w.kbeg ? (w.kend - 1) / P - pg_first + 1 : 0;   // the plan's chunks: <= kMaxChunkPages
      const int32_t* bt = a.block_table + static_cast<int64_t>(w.b) * a.max_pages + pg_first;
      for (int j = wave * 64 + lane; j < npg; j += NW * 64) s_pg[j] = bt[j];
      fast = fast && P % RPI == 0;
    } else {
      seqoff = static_cast<int64_t>(w.b) * a.cs_seq * Tile::ELEM;
    }
#pragma unroll
    for (int i = 0; i < PERW; ++i) {
      const int g = wave * PERW + i;
      row[i] = (g % IPT) * RPI + lane / CPR;
      chunk[i] = (lane % CPR) ^ Tile::swizzle(row[i]);
      voff[i] = static_cast<uint32_t>(static_cast<int64_t>(lane / CPR) * tokb + chunk[i] * 16);
    }
  }

  // Byte offset of (key, element 0) from this head's cache base.
  __device__ __attribute__((always_inline)) int64_t key_offset(int key, const SIMSD_LDS int* s_pg) const {
    if (!PAGED) return seqoff + static_cast<int64_t>(key) * tokb;
    const int pg = lgP >= 0 ? key >> lgP : key / P;
    return s_pg[pg - pg_first] * pageb + static_cast<int64_t>(key - pg * P) * tokb;
  }

  // Issue this wave's share of the tile starting at key k0 into the ring slot at
  // LDS byte address `slot`.
  __device__ __attribute__((always_inline)) void issue(uint32_t slot, int k0, int kend, const SIMSD_LDS int* s_pg) const {
    if (k0 + KEYS <= kend && fast) {
      // Lane j holds the offset of the rows of instruction j of a tensor.
      int64_t at = 0;
      if (PAGED) at = key_offset(k0 + (lane % IPT) * RPI, s_pg);
#pragma unroll
      for (int i = 0; i < PERW; ++i) {
        const int g = wave * PERW + i;
        int64_t base;
        if (PAGED) {
          const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(at), g % IPT);
          const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(at >> 32), g % IPT);
          base = static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
        } else {
          base = seqoff + static_cast<int64_t>(k0 + (g % IPT) * RPI) * tokb;
        }
        dma16s((g < IPT ? kc : vc) + base, voff[i], slot + (g / IPT) * TILEB + (g % IPT) * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < PERW; ++i) {
        const int g = wave * PERW + i;
        const int64_t off = key_offset(min(k0 + row[i], kend - 1), s_pg) + chunk[i] * 16;
        dma16((g < IPT ? kc : vc) + off, slot + (g / IPT) * TILEB + (g % IPT) * 1024);
      }
    }
  }
};

// Values that are not finite, in tiles whose keys some rows do not see: a masked
// key weighs 0, and 0 * inf would be NaN in rows that must not know of it.  Such a
// tile's product takes 0 in place of them, and when the range is done those tiles
// are gone through again with a code of each value (1: +inf, 256: -inf, 65536: NaN;
// at most 64 of each in a tile, exact in fp32) added up over the keys each row sees,
// from which the sums inf, -inf or NaN are put in.
__device__ inline float code_value(float code) {
  const uint32_t c = static_cast<uint32_t>(code);
  float v = 0.f;
  if (c % kCode1) v += __builtin_huge_valf();
  if (c / kCode1 % (kCode2 / kCode1)) v -= __builtin_huge_valf();
  if (c / kCode2) v = __builtin_nanf("");
  return v;
}
__device__ inline bool wild(uint32_t w) {          // either bf16 of a word
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ inline uint32_t tamed(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
__device__ inline uint32_t code_of(uint32_t x) {   // one bf16 -> the bf16 code of it
  if ((x & 0x7f80u) != 0x7f80u) return 0;
  return x == 0x7f80u ? 0x3f80u : x == 0xff80u ? 0x4380u : 0x4780u;
}

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
template <int D, int RB, bool PAGED>
__global__ void __launch_bounds__(256, 2) chunk_f32_kernel(ChunkArgs a) {
  constexpr int NW = 4, SUB = 16;              // waves; keys per sub-tile
  constexpr int KI = D / 16;                   // 16-byte loads per lane of a K (or Q) row
  constexpr int VU = D / 64;                   // 16-byte loads per lane of a V key
  constexpr int ROWS = 16 * RB;
  constexpr int XROW = D + 4;                  // LDS row stride of the merge (floats)
  __shared__ __attribute__((aligned(16))) float xs[NW * ROWS * XROW];
  __shared__ float s_m[NW][ROWS], s_l[NW][ROWS];

  Block w;
  if (!setup_block(a, w)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q = lane >> 4;
  const int nsub = w.kend > w.kbeg ? (w.kend - w.kbeg + SUB - 1) / SUB : 0;
  const int items = nsub > wave ? (nsub - wave + NW - 1) / NW : 0;
  const int64_t head0 = (PAGED ? 0 : w.b * a.cs_seq) + w.kvh * a.cs_head;
  const float* kc = static_cast<const float*>(a.k_cache) + head0;
  const float* vc = static_cast<const float*>(a.v_cache) + head0;
  const int32_t* pages = a.block_table + static_cast<int64_t>(w.b) * a.max_pages;
  auto key0 = [&](int i) { return w.kbeg + SUB * (wave + NW * i); };
  // Keys past the range's last one read that one (their scores are masked).
  auto key_at = [&](const float* base, int key, int page) __attribute__((always_inline)) {
    key = min(key, w.kend - 1);
    if (!PAGED) return base + key * a.cs_tok;
    return base + (page * a.cs_seq + (key % a.page_size) * a.cs_tok);
  };
  f32x4 kx[KI], vx[SUB / 4][VU];
  int page = 0, page_v = 0;                    // of key n: of the K loads ahead, of the V loads ahead
  auto next_page = [&](int i) __attribute__((always_inline)) {
    if (PAGED && i < items) page = pages[min(key0(i) + n, w.kend - 1) / a.page_size];
  };
  auto load_k = [&](int i) __attribute__((always_inline)) {
    const f32x4* kr = reinterpret_cast<const f32x4*>(key_at(kc, key0(i) + n, page));
#pragma unroll
    for (int c = 0; c < KI; ++c) kx[c] = kr[4 * c + q];
    page_v = page;
    next_page(i + 1);
  };
  auto load_v = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < SUB / 4; ++j) {
      const int pj = PAGED ? __shfl(page_v, 4 * q + j) : 0;
      const f32x4* vr = reinterpret_cast<const f32x4*>(key_at(vc, key0(i) + 4 * q + j, pj));
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
  int limit[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int m = w.row0 + 16 * r + n;
    const int mc = min(m, w.rows - 1), t = mc / a.group;
    const f32x4* qr = reinterpret_cast<const f32x4*>(
        static_cast<const float*>(a.q) + (static_cast<int64_t>(w.q0 + t) * a.hq + w.kvh * a.group + mc % a.group) * D);
#pragma unroll
    for (int i = 0; i < KI; ++i) qop[r][i] = qr[4 * i + q];
    limit[r] = m < w.rows ? visible_keys(a, w.kv, w.n, t) : 0;
  }

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
    const bool masked = k0 + SUB > w.full;     // some row does not see all of it
    if (masked) {
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k0 + 4 * q + j >= limit[r]) s[r][j] = kNegInf;
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
    next_page(it);
    page_v = page;
    load_v(it);
    const int k0 = key0(it);
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
            sum = __builtin_amdgcn_mfma_f32_16x16x4f32(code, k0 + 4 * q + j < limit[r] ? 1.f : 0.f, sum, 0, 0, 0);
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
template <int D, int RB, bool PAGED>
__global__ void __launch_bounds__(256, 2) chunk_f32_rows_kernel(ChunkArgs a) {
  constexpr int NW = 4, SUB = 16, NBUF = 2;
  constexpr int KI = D / 16, VU = D / 64;
  using Ring = ChunkRing<F32Tile<D>, NW, PAGED>;
  constexpr int ROWB = Ring::ROWB, TILEB = Ring::TILEB, KEYS = Ring::KEYS;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NBUF][2][TILEB];   // [slot][K, V]
  __shared__ int s_pg_arr[PAGED ? kMaxChunkPages : 1];
  __shared__ int s_bad[2];                     // first and last tile with values that are not finite
  SIMSD_LDS int* s_pg = (SIMSD_LDS int*)(&s_pg_arr[0]);

  Block w;
  if (!setup_block(a, w)) return;
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
  }
  Ring kv;
  kv.init(a, w, wave, lane, s_pg);
  __builtin_amdgcn_s_waitcnt(0);               // (as in the bf16 kernel)
  __syncthreads();                             // staged page ids, s_bad
  const int nt = w.kend > w.kbeg ? (w.kend - w.kbeg + KEYS - 1) / KEYS : 0;
  const uint32_t ring0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((SIMSD_LDS void*)(&smem[0][0][0])));
  constexpr uint32_t kSlotBytes = 2 * TILEB;
#pragma unroll
  for (int j = 0; j < NBUF; ++j)
    if (j < nt) kv.issue(ring0 + j * kSlotBytes, w.kbeg + j * KEYS, w.kend, s_pg);

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
    const int k0 = w.kbeg + it * KEYS;
    if (it == 0 && nt > 1) wait_vm<Ring::PERW>();
    else wait_vm<0>();
    lds_barrier();                             // all of tile `it` is in; the other slot is free
    if (it >= 1 && it + 1 < nt) kv.issue(ring0 + ((it + 1) & 1) * kSlotBytes, k0 + KEYS, w.kend, s_pg);
    const SIMSD_LDS uint8_t* sk = reinterpret_cast<const SIMSD_LDS uint8_t*>(ring0) + (it & 1) * kSlotBytes;
    const SIMSD_LDS uint8_t* sv = sk + TILEB;
    const bool masked = k0 + KEYS > w.full;    // some row of the block does not see all of it
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
            if (ks + 4 * q + j >= limit[r]) s[r][j] = kNegInf;
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
    kv.issue(ring0, w.kbeg + it * KEYS, w.kend, s_pg);
    wait_vm<0>();
    lds_barrier();
    const SIMSD_LDS uint8_t* sv = reinterpret_cast<const SIMSD_LDS uint8_t*>(ring0) + TILEB;
#pragma unroll 1
    for (int sub = 0; sub < KEYS / SUB; ++sub) {
      const int ks = w.kbeg + it * KEYS + SUB * sub;
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
              sum = __builtin_amdgcn_mfma_f32_16x16x4f32(code, ks + 4 * q + j < limit[r] ? 1.f : 0.f, sum, 0, 0, 0);
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
