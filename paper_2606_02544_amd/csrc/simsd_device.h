// Device pieces that the attention kernels share: matrix-core operand types,
// lane exchanges, the LDS tile layout and the direct global -> LDS loads.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "simsd_plan.h"

namespace simsd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#define SIMSD_LDS __attribute__((address_space(3)))

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLazy = 8.0f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two floats -> two bf16 (round to nearest even) in one instruction.
__device__ inline uint32_t pack2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Combine a value across lanes l and l ^ 32 (the two halves of an MFMA
// column) with one VALU lane swap instead of an LDS permute.  Both halves
// get the same bits (low half's value first).
__device__ inline float xhalf_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float xhalf_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Over lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ inline float quad_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return xhalf_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float quad_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return xhalf_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

template <int D>
struct TileGeom {
  static constexpr int CH = D / 8;             // 16-byte chunks per key row
  static constexpr int ROWB = 2 * D;           // LDS bytes per key row (unpadded)
  static constexpr int TILEB = kTile * ROWB;   // one tensor (K or V) of one tile
};

// LDS swizzle: 16-byte chunk L of key row r is stored at chunk L ^ swz(r).  The
// XOR masks were chosen (by exhaustive search over linear maps of r mod 16) so
// that the K operand reads (32 rows, one chunk) and the transpose reads of V
// (4 rows x 4 chunks per 32 lanes) hit distinct banks with 32 or 64 LDS banks.
template <int D>
__device__ inline int swz(int r) {
  if constexpr (D == 128)
    return ((r & 1) ? 4 : 0) ^ ((r & 2) ? 10 : 0) ^ ((r & 4) ? 1 : 0) ^ ((r & 8) ? 2 : 0);
  else
    return ((r & 1) ? 2 : 0) ^ ((r & 2) ? 4 : 0) ^ ((r & 4) ? 1 : 0) ^ ((r & 8) ? 2 : 0);
}

// Direct global -> LDS copy of 16 bytes per lane (global_load_lds_dwordx4):
// lane i's bytes land at LDS byte lds + 16 * i, so one instruction moves 1 KB.
// It counts in vmcnt like any vector load but the compiler does not track it:
// readers wait with wait_vm and then pass a barrier.  M0 (the LDS base) is a
// reserved register that the compiler does not allocate to values, so setting
// it here disturbs nothing.  dma16s takes a wave-uniform 64-bit base and a
// 32-bit per-lane offset (no per-lane address arithmetic).
__device__ inline void dma16(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off"
               :: "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}
__device__ inline void dma16s(const void* base, uint32_t voff, uint32_t lds) {
  // readfirstlane works on (signed) int: each half goes through uint32_t
  // before widening so that the low half is not sign-extended.
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32)));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b & 0xffffffffu)));
  const uint64_t bu = (static_cast<uint64_t>(hi) << 32) | lo;
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(voff), "s"(bu), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}
template <int N>
__device__ inline void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
// This wave's LDS accesses complete, then a work-group barrier.  Unlike
// __syncthreads it does not wait for vector memory, so tiles still loading
// stay in flight.
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

}  // namespace
}  // namespace simsd
