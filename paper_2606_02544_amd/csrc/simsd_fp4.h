// The cache's 4-bit form, and its tiles on their way into LDS.
//
// 32 dims of a head share a power of two, held as its exponent + 127 in a byte, and each
// is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it with a sign, two a byte (the even dim in
// the low half).  The conversions are the hardware's: to 4 bits it rounds to the nearest,
// ties to the even code, past 6 to 6; from 4 bits every value is exact in bf16, and a
// scale byte of 255 gives NaN.
#pragma once

#include "simsd_chunk_device.h"

namespace simsd {
namespace {

constexpr int kFp4Group = 32;    // dims that share a scale

// Eight codes of a word with this scale byte, in bf16.
__device__ inline u32x4 fp4_values(uint32_t w, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
}

// Eight codes without those that are past bf16's range at a scale of 254 (`shift` 0: from
// 2 on at 2^127, the codes' bit 2) or 253 (1: 4 and 6 at 2^126, their bits 2 and 1).
__device__ inline uint32_t fp4_finite(uint32_t w, uint32_t shift) {
  const uint32_t past = w & (w << shift) & 0x44444444u;
  return w & ~(past | (past - (past >> 2)));
}

// The scale byte of 32 values whose largest magnitude has these fp32 bits: the least
// exponent at which it is below 7, which rounds to 6.  (Adding a quarter of the mantissa's
// range carries into the exponent from 1.75 * 2^x = 7 * 2^(x - 2) on.)  255: one of them is
// infinite or NaN, and all are held as NaN.
__device__ inline uint32_t fp4_scale(uint32_t largest) {
  if (largest >= 0x7f800000u) return 255u;
  return min(max(static_cast<int>((largest + 0x200000u) >> 23) - 2, 2), 252);
}

// A tile of 64 keys of a 4-bit cache: a unit is 16 bytes, the 32 dims of one scale, of
// one key and tensor; every thread loads its units of a tile into registers, and turns
// them into bf16 in the tile's layout in LDS a tile later.
template <int D, int NW, bool PAGED>
struct Fp4Tiles {
  static constexpr int ROWB = TileGeom<D>::ROWB, TILEB = TileGeom<D>::TILEB;
  static constexpr int GROUPS = D / kFp4Group;
  static constexpr int UNITS = kTile * GROUPS;              // of a tensor
  static constexpr int PER = (2 * UNITS + NW * 64 - 1) / (NW * 64);
  static_assert(UNITS % 64 == 0, "a wave's units are of one tensor");

  const uint8_t* codes[PER];    // of the unit's tensor, offset to this head and group
  const uint8_t* scales[PER];
  int64_t tokb, pageb, tok_s, page_s;   // bytes per token and page, of codes and of scales
  int row, P, lgP;              // key of this thread's units in the tile
  int at;                       // LDS offset of the key's row
  int chunk[4];                 // LDS offsets of the unit's four 16-byte chunks in it
  int tensor0;
  bool live;
  u32x4 data[PER];
  uint32_t scale[PER];

  __device__ __attribute__((always_inline)) void init(const SpanArgs& a, const Block& w, int wave, int lane, SIMSD_LDS int*) {
    const int u0 = wave * 64;                               // (wave-uniform: which tensor)
    tensor0 = u0 / UNITS;
    live = u0 < 2 * UNITS;
    const int idx = u0 % UNITS + lane;
    const int g = idx % GROUPS, k = idx / GROUPS;
    // The eight lanes that write at a time take keys 0 and 2 (1 and 3, ...): their
    // swizzles differ in the chunk's low bits, so that they write different banks.
    row = D == 128 ? (k & ~3) | (k & 1) << 1 | (k >> 1 & 1) : k;
    at = row * ROWB;
#pragma unroll
    for (int j = 0; j < 4; ++j) chunk[j] = 16 * ((4 * g + j) ^ swz<D>(row));
    const int64_t seq = PAGED ? 0 : w.b;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool v = tensor0 + i > 0;
      codes[i] = static_cast<const uint8_t*>(v ? a.v_cache : a.k_cache) + seq * a.cs_seq + w.kvh * a.cs_head + g * 16;
      scales[i] = (v ? a.v_scales : a.k_scales) + seq * a.ss_seq + w.kvh * a.ss_head + g;
    }
    tokb = a.cs_tok;
    pageb = a.cs_seq;
    tok_s = a.ss_tok;
    page_s = a.ss_seq;
    P = a.page_size;
    lgP = a.page_shift;
  }

  // Keys outside [beg, end) are read as the nearest one inside.
  __device__ __attribute__((always_inline)) void load(int k0, int beg, int end, int first_page, const SIMSD_LDS int* s_pg) {
    if (!live) return;
    const int key = max(beg, min(k0 + row, end - 1));
    int64_t c, s;
    if (PAGED) {
      const int pg = lgP >= 0 ? key >> lgP : key / P;
      const int id = s_pg[pg - first_page], in = key - pg * P;
      c = id * pageb + in * tokb;
      s = id * page_s + in * tok_s;
    } else {
      c = key * tokb;
      s = key * tok_s;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      data[i] = *reinterpret_cast<const u32x4*>(codes[i] + c);
      scale[i] = scales[i][s];
    }
  }

  __device__ __attribute__((always_inline)) void store(uint32_t slot) const {
    if (!live) return;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      SIMSD_LDS uint8_t* to = reinterpret_cast<SIMSD_LDS uint8_t*>(slot) + (tensor0 + i) * TILEB + at;
#pragma unroll
      for (int j = 0; j < 4; ++j) *(SIMSD_LDS u32x4*)(to + chunk[j]) = fp4_values(data[i][j], scale[i]);
    }
  }
};

}  // namespace
}  // namespace simsd
