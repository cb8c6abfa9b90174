// Filling a cache held in 4 bits, and reading it back.
#include <hip/hip_runtime.h>

#include "simsd_fp4.h"
#include "simsd_rotary_device.h"

namespace simsd {
namespace {

// ----------------------------------------------------------------------------
// The append: queries turned as simsd_rotary_append turns them (the first q_blocks
// work-groups), keys turned and rounded to 4 bits, values rounded to 4 bits (the others:
// TOKENS tokens each, a thread per eight dims of a key or value head, four threads a
// scale).
//
// Keys are turned in fp64 and rounded once: their fp32 value on the way is rounded to
// odd, so that the code is the nearest to the turned key, as if it had not been there.
// (The angle, position * freq in turns, is three roundings off: 3.4e-16 of itself.)
// (An fp32 rotation is off by 1e-7, which moves one key in ten million to the
// next code: a step of up to a third.  The fp64 products hide behind the loads.)
//
// What bounds it: memory.  A head of 128 is read as 256 bytes and written as 68.  Of
// 32768 tokens (32 query heads and 8 KV heads of 128, 709 MB) it reaches 3.8 TB/s in
// 188 us, where a copy of as many bytes takes 146: the queries' part goes at 5, the keys'
// and values' at about half of that, whose loads wait for the token's angles and cache
// row and whose stores are 4 bytes a thread.  (The two parts in turn, eight work-groups
// of each, so that one fills the other's waits: 0 to 3 % less there, 2 % more for 4200
// ragged tokens.)
// ----------------------------------------------------------------------------
constexpr int kMaxHalf = 64;     // pairs of the largest head

// y in fp32, with the last place odd where that is not exact; past fp32's range, its end.
__device__ inline uint32_t rounded_to_odd(double y) {
  const float f = static_cast<float>(y);
  uint32_t bits = __float_as_uint(f);
  const double back = static_cast<double>(f);
  if (back != y) bits = (bits - (fabs(back) > fabs(y) ? 1u : 0u)) | 1u;
  return bits;
}

template <int VEC, bool INTER, int TOKENS>
__device__ __attribute__((always_inline)) inline void fp4_tokens(const Fp4AppendArgs& f, int block) {
  const RotaryArgs& a = f.r;
  __shared__ double2 cs[TOKENS][kMaxHalf];
  __shared__ int64_t s_row[TOKENS][2];         // offsets of the token's codes and scales, or -1
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = block * TOKENS;
  const int half = a.rot / 2;
  const int per_head = a.d / 8;
  const int per_tensor = f.hkv * per_head, per_token = 2 * per_tensor;
  const int total = per_token * min(TOKENS, a.tokens - t0);

  struct Unit {
    int tok, head, at;           // at: first of its eight dims
    bool value;
  };
  auto unit = [&](int i) {
    Unit u;
    u.tok = TOKENS == 1 ? 0 : i / per_token;
    int r = TOKENS == 1 ? i : i % per_token;
    u.value = r >= per_tensor;
    if (u.value) r -= per_tensor;
    u.head = r / per_head;
    u.at = r % per_head * 8;
    return u;
  };
  u32x4 x1[kDepth], x2[kDepth];
  auto load = [&](int i, int s) __attribute__((always_inline)) {
    if (i >= total) return;
    const Unit u = unit(i);
    const int64_t t = t0 + u.tok;
    if (u.value) {
      x1[s] = load_raw<true, 8>(a.v, t * a.v_tok + u.head * a.v_head + u.at);
      return;
    }
    const int64_t row = t * a.k_tok + u.head * a.k_head;
    x1[s] = load_raw<true, 8>(a.k, row + u.at);
    // The other halves of the eight dims' pairs, where those are eight dims too.
    if (!INTER && VEC > 1 && u.at < a.rot)
      x2[s] = load_raw<true, 8>(a.k, row + (u.at < half ? u.at + half : u.at - half));
  };
#pragma unroll
  for (int s = 0; s < kDepth; ++s) load(tid + s * NT, s);

  for (int j = wave; j < TOKENS; j += NT / 64) {
    const int t = t0 + j;
    int pos = 0;
    int64_t row = -1, srow = -1;
    if (t < a.tokens) {
      const int b = sequence_of(a.q_starts, a.batch, t, lane);
      if (b < a.batch && t >= a.q_starts[0]) {
        const int at = a.kv_lens[b] - (a.q_starts[b + 1] - t);
        pos = a.positions ? a.positions[t] : at;
        if (at >= 0 && at < a.max_kv) {
          if (a.page_size > 0) {
            const int page = a.block_table[static_cast<int64_t>(b) * a.max_pages + at / a.page_size];
            if (page >= 0 && page < a.num_pages) {
              row = page * a.cs_seq + (at % a.page_size) * a.cs_tok;
              srow = page * f.ss_seq + (at % a.page_size) * f.ss_tok;
            }
          } else {
            row = b * a.cs_seq + at * a.cs_tok;
            srow = b * f.ss_seq + at * f.ss_tok;
          }
        }
      }
    }
    if (lane == 0) {
      s_row[j][0] = row;
      s_row[j][1] = srow;
    }
    for (int i = lane; i < half; i += 64) {
      constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)
      const double rev = static_cast<double>(pos) * a.freq[i] * kTurn;
      double sn, c;
      sincospi(2.0 * (rev - rint(rev)), &sn, &c);
      cs[j][i] = double2{c * a.factor, sn * a.factor};
    }
  }
  __syncthreads();

  for (int base = 0; base < total; base += kDepth * NT) {
#pragma unroll
    for (int s = 0; s < kDepth; ++s) {
      const int i = base + tid + s * NT;
      if (i >= total) continue;                // (four threads of a scale together)
      const Unit u = unit(i);
      if (s_row[u.tok][0] < 0) continue;       // (likewise)
      uint32_t y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = e & 1 ? x1[s][e / 2] & 0xffff0000u : x1[s][e / 2] << 16;
      if (!u.value && u.at < a.rot) {
        if constexpr (VEC == 1) {              // (rotary dims that end inside eight dims)
          const uint16_t* k = static_cast<const uint16_t*>(a.k) + (t0 + u.tok) * a.k_tok + u.head * a.k_head;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int j = u.at + e;
            if (j >= a.rot) continue;
            const bool second = INTER ? j & 1 : j >= half;
            const int other = INTER ? j ^ 1 : second ? j - half : j + half;
            const double2 r = cs[u.tok][INTER ? j / 2 : second ? other : j];
            const double v = __uint_as_float(y[e]), o = __uint_as_float(static_cast<uint32_t>(k[other]) << 16);
            y[e] = rounded_to_odd(second ? v * r.x + o * r.y : v * r.x - o * r.y);
          }
        } else if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const double2 r = cs[u.tok][(u.at + e) / 2];
            const double v = __uint_as_float(y[e]), o = __uint_as_float(y[e + 1]);
            y[e] = rounded_to_odd(v * r.x - o * r.y);
            y[e + 1] = rounded_to_odd(o * r.x + v * r.y);
          }
        } else {
          const bool second = u.at >= half;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const double2 r = cs[u.tok][(second ? u.at - half : u.at) + e];
            const double v = __uint_as_float(y[e]);
            const double o = __uint_as_float(e & 1 ? x2[s][e / 2] & 0xffff0000u : x2[s][e / 2] << 16);
            y[e] = rounded_to_odd(v * r.x + (second ? o : -o) * r.y);
          }
        }
      }
      uint32_t largest = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) largest = max(largest, y[e] & 0x7fffffffu);
      largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 1)));
      largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 2)));
      const uint32_t scale = fp4_scale(largest);
      const float by = __uint_as_float(scale << 23);
      uint32_t codes = 0;
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(y[0]), __uint_as_float(y[1]), by, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(y[2]), __uint_as_float(y[3]), by, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(y[4]), __uint_as_float(y[5]), by, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(y[6]), __uint_as_float(y[7]), by, 3);
      if (scale == 255u) codes = 0;
      uint8_t* to = static_cast<uint8_t*>(u.value ? a.v_out : a.k_out) + s_row[u.tok][0] + u.head * a.cs_head;
      *reinterpret_cast<uint32_t*>(to + u.at / 2) = codes;
      if (u.at % kFp4Group == 0)
        (u.value ? f.v_scales : f.k_scales)[s_row[u.tok][1] + u.head * f.ss_head + u.at / kFp4Group] = static_cast<uint8_t>(scale);
    }
    if (base + kDepth * NT < total) {
#pragma unroll
      for (int s = 0; s < kDepth; ++s) load(base + kDepth * NT + tid + s * NT, s);
    }
  }
}

template <int VEC, bool INTER, int TOKENS>
__global__ void __launch_bounds__(NT) fp4_append_kernel(Fp4AppendArgs f, int q_blocks) {
  const int block = blockIdx.x;
  if (block < q_blocks) rotary_tokens<true, VEC, INTER, true, TOKENS>(f.r, block);
  else fp4_tokens<VEC, INTER, TOKENS>(f, block - q_blocks);
}

template <int VEC, bool INTER>
void launch_append(const Fp4AppendArgs& f, int cus, hipStream_t st) {
  constexpr int kMany = 4;
  const bool many = f.r.tokens >= 8 * kMany * cus;
  const int blocks = many ? (f.r.tokens + kMany - 1) / kMany : f.r.tokens;
  const int q_blocks = f.r.hq > 0 ? blocks : 0;
  const dim3 grid(q_blocks + blocks);
  if (many) hipLaunchKernelGGL((fp4_append_kernel<VEC, INTER, kMany>), grid, dim3(NT), 0, st, f, q_blocks);
  else hipLaunchKernelGGL((fp4_append_kernel<VEC, INTER, 1>), grid, dim3(NT), 0, st, f, q_blocks);
}

// ----------------------------------------------------------------------------
// The values of codes in bf16: a thread takes eight dims (4 bytes in, 16 out), and
// several of them a work-group's width apart.  Memory bounds it: 408 MB in 69 us, 6 TB/s
// (the codes partly from the last-level cache, as written just before).
// ----------------------------------------------------------------------------
constexpr int kUnits = 4;        // of a thread

template <typename Index>
__global__ void __launch_bounds__(256) fp4_values_kernel(Fp4Args a) {
  // Keys, then values (those that are wanted).
  const bool value = !a.k_out || blockIdx.y == 1;
  const uint8_t* codes = static_cast<const uint8_t*>(value ? a.v : a.k);
  const uint8_t* scales = value ? a.v_scales : a.k_scales;
  char* out = static_cast<char*>(value ? a.v_out : a.k_out);
  const Index per_row = a.groups * 4;
  const Index total = static_cast<Index>(a.rows) * per_row;
  const Index first = static_cast<Index>(blockIdx.x) * (256 * kUnits) + threadIdx.x;
  uint32_t w[kUnits], s[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const Index u = first + i * 256;
    if (u >= total) break;
    const Index row = u / per_row;
    const int at = static_cast<int>(u - row * per_row);
    const Index r1 = row / a.n2;
    const int64_t i2 = row - r1 * a.n2, i0 = r1 / a.n1, i1 = r1 - i0 * a.n1;
    w[i] = *reinterpret_cast<const uint32_t*>(codes + i0 * a.c0 + i1 * a.c1 + i2 * a.c2 + at * 4);
    s[i] = scales[i0 * a.s0 + i1 * a.s1 + i2 * a.s2 + at / 4];
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const Index u = first + i * 256;
    if (u >= total) break;
    *reinterpret_cast<u32x4*>(out + static_cast<int64_t>(u) * 16) = fp4_values(w[i], s[i]);
  }
}

}  // namespace

hipError_t launch_fp4_append(const Fp4AppendArgs& f, bool interleaved, int cus, hipStream_t st) {
  const bool whole = (interleaved ? f.r.rot : f.r.rot / 2) % 8 == 0;
  if (interleaved) {
    if (whole) launch_append<8, true>(f, cus, st);
    else launch_append<1, true>(f, cus, st);
  } else {
    if (whole) launch_append<8, false>(f, cus, st);
    else launch_append<1, false>(f, cus, st);
  }
  return hipGetLastError();
}

hipError_t launch_fp4_values(const Fp4Args& a, hipStream_t st) {
  const int64_t units = a.rows * a.groups * 4;
  const dim3 grid(static_cast<uint32_t>((units + 256 * kUnits - 1) / (256 * kUnits)), a.k_out && a.v_out ? 2 : 1);
  if (units < (int64_t{1} << 31) - 256 * kUnits) hipLaunchKernelGGL((fp4_values_kernel<int32_t>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((fp4_values_kernel<int64_t>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace simsd
