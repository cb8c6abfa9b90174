// Device pieces that the chunk attention's kernels share: which rows and keys a
// work-group has, tiles in LDS and the ring that streams them, and the code of values
// that are not finite.
#pragma once

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
// the range's last key, which read that key instead, an address a lane.  SPAN: the
// range is a list of tiles (see Span), whose issue says which keys of a tile there are.
template <typename Tile, int NW, bool PAGED, bool SPAN = false>
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
      if constexpr (!SPAN)
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
  // (SPAN: keys below kbeg are read as that one too.)
  __device__ __attribute__((always_inline)) void issue(uint32_t slot, int k0, int kend, const SIMSD_LDS int* s_pg, int kbeg = 0) const {
    if (k0 + KEYS <= kend && fast && (!SPAN || k0 >= kbeg)) {
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
        const int key = SPAN ? max(kbeg, min(k0 + row[i], kend - 1)) : min(k0 + row[i], kend - 1);
        const int64_t off = key_offset(key, s_pg) + chunk[i] * 16;
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

}  // namespace
}  // namespace simsd
