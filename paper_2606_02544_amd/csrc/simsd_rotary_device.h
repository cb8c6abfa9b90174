// Rotary positions of a work-group's tokens, and where a token goes in the cache.
#pragma once

#include "simsd_ops_kernels.h"
#include "simsd_search.h"

namespace simsd {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int NT = 256;        // threads of a work-group
constexpr int kDepth = 4;      // units a thread loads before it writes the first
constexpr int kMaxRot = 512;   // largest rotary_dim

// 16 bytes, or one element in the first word, as they lie in memory.
template <bool BF16, int VEC>
__device__ inline u32x4 load_raw(const void* base, int64_t at) {
  if constexpr (VEC > 1) {
    return *reinterpret_cast<const u32x4*>(static_cast<const char*>(base) + at * (BF16 ? 2 : 4));
  } else {
    u32x4 w = {0, 0, 0, 0};
    if constexpr (BF16) w[0] = static_cast<const uint16_t*>(base)[at];
    else w[0] = static_cast<const uint32_t*>(base)[at];
    return w;
  }
}
template <bool BF16, int VEC>
__device__ inline void store_raw(void* base, int64_t at, u32x4 w) {
  if constexpr (VEC > 1) *reinterpret_cast<u32x4*>(static_cast<char*>(base) + at * (BF16 ? 2 : 4)) = w;
  else if constexpr (BF16) static_cast<uint16_t*>(base)[at] = static_cast<uint16_t>(w[0]);
  else static_cast<uint32_t*>(base)[at] = w[0];
}
// The two values of word i (fp32: one).
template <bool BF16>
__device__ inline f32x2 values(uint32_t w) {
  if constexpr (BF16) return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  else return f32x2{__uint_as_float(w), 0.f};
}
template <bool BF16>
__device__ inline uint32_t packed(float lo, float hi) {
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
  else return __float_as_uint(lo);
}

// What a work-group knows of one of its tokens.
struct Token {
  int live;          // belongs to a sequence (append), or always
  int pos;
  int64_t row;       // append: element offset of its cache row, or -1
};

// Sequence of token t: the number of sequences that end at or before it (one
// wave; starts do not fall).
__device__ inline int sequence_of(const int32_t* q_starts, int batch, int t, int lane) {
  return leading(batch, lane, [&](int b) { return q_starts[b + 1] <= t; });
}

// Unit u of a token, in order: queries, keys, values.  A turning unit holds VEC
// pairs (half: VEC elements of either half; interleaved: VEC elements, or one
// pair where VEC is 1); a copying unit holds VEC elements of the rest.  Values
// are always whole vectors.
template <bool BF16, int VEC, bool INTER, bool APPEND, int TOKENS>
__device__ __attribute__((always_inline)) inline void rotary_tokens(RotaryArgs a, int block) {
  constexpr int W = BF16 ? 8 : 4;              // elements of 16 bytes
  constexpr bool PAIR = !INTER || VEC == 1;    // a turning unit loads from two places
  __shared__ float2 cs[TOKENS][kMaxRot / 2];
  __shared__ Token tk[TOKENS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = block * TOKENS;
  const int half = a.rot / 2;
  const int turning = INTER ? (VEC == 1 ? half : a.rot / VEC) : half / VEC;
  const int qk = a.q_units * (a.hq + a.hkv);   // units of the queries and keys of a token
  const int total = a.units * min(TOKENS, a.tokens - t0);

  struct Unit {
    int tok, kind, head, at;                   // kind 0: query, 1: key, 2: value; at: first element
    bool turns;
  };
  auto unit = [&](int i) {
    Unit u;
    u.tok = TOKENS == 1 ? 0 : i / a.units;
    const int r = TOKENS == 1 ? i : i % a.units;
    if (r < qk) {
      const int h = r / a.q_units, e = r % a.q_units;
      u.kind = h < a.hq ? 0 : 1;
      u.head = h < a.hq ? h : h - a.hq;
      u.turns = e < turning;
      u.at = u.turns ? (INTER && VEC == 1 ? 2 * e : e * VEC) : a.rot + (e - turning) * VEC;
    } else {
      u.kind = 2;
      u.head = (r - qk) / a.v_units;
      u.at = (r - qk) % a.v_units * W;
      u.turns = false;
    }
    return u;
  };
  auto second = [&](const Unit& u) { return INTER ? u.at + 1 : u.at + half; };

  u32x4 x1[kDepth], x2[kDepth];
  auto load = [&](int i, int s) __attribute__((always_inline)) {
    if (i >= total) return;
    const Unit u = unit(i);
    const int64_t t = t0 + u.tok;
    if (APPEND && u.kind == 2) {
      x1[s] = load_raw<BF16, W>(a.v, t * a.v_tok + u.head * a.v_head + u.at);
      return;
    }
    const void* base = u.kind == 0 ? a.q : a.k;
    const int64_t row = u.kind == 0 ? t * a.q_tok + u.head * a.q_head : t * a.k_tok + u.head * a.k_head;
    x1[s] = load_raw<BF16, VEC>(base, row + u.at);
    if (PAIR && u.turns) x2[s] = load_raw<BF16, VEC>(base, row + second(u));
  };
#pragma unroll
  for (int s = 0; s < kDepth; ++s) load(tid + s * NT, s);

  // Where each token goes, and its angles.
  for (int j = wave; j < TOKENS; j += NT / 64) {
    const int t = t0 + j;
    Token k = {0, 0, -1};
    if (t < a.tokens) {
      k.live = 1;
      if constexpr (APPEND) {
        const int b = sequence_of(a.q_starts, a.batch, t, lane);
        k.live = b < a.batch && t >= a.q_starts[0];
        if (k.live) {
          const int at = a.kv_lens[b] - (a.q_starts[b + 1] - t);
          k.pos = at;
          if (at >= 0 && at < a.max_kv) {
            if (a.page_size > 0) {
              const int page = a.block_table[static_cast<int64_t>(b) * a.max_pages + at / a.page_size];
              if (page >= 0 && page < a.num_pages)
                k.row = page * a.cs_seq + (at % a.page_size) * a.cs_tok;
            } else {
              k.row = b * a.cs_seq + at * a.cs_tok;
            }
          }
        }
      }
      if (a.positions && k.live) k.pos = a.positions[t];
    }
    if (lane == 0) tk[j] = k;
    for (int i = lane; i < half; i += 64) {
      constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)
      const double rev = static_cast<double>(k.pos) * a.freq[i] * kTurn;
      // (Half a turn at most: in fp32 it is off by pi 2^-24 radians, and the sine and
      // cosine by two roundings, as the rotation after them is by its own.)
      const float f = static_cast<float>(rev - rint(rev));
      float sn, c;
      sincospif(2.f * f, &sn, &c);
      cs[j][i] = float2{c * a.factor, sn * a.factor};
    }
  }
  __syncthreads();

  for (int base = 0; base < total; base += kDepth * NT) {
#pragma unroll
    for (int s = 0; s < kDepth; ++s) {
      const int i = base + tid + s * NT;
      if (i >= total) continue;
      const Unit u = unit(i);
      const Token k = tk[u.tok];
      const int64_t t = t0 + u.tok;
      if (APPEND && u.kind == 2) {
        if (k.row >= 0) store_raw<BF16, W>(a.v_out, k.row + u.head * a.cs_head + u.at, x1[s]);
        continue;
      }
      if (u.turns) {
        constexpr int PW = BF16 ? 2 : 1;         // values of a word
        constexpr int WORDS = VEC == 1 ? 1 : 4;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          if constexpr (PAIR) {
            const f32x2 v1 = values<BF16>(x1[s][w]), v2 = values<BF16>(x2[s][w]);
            float y1[2] = {0.f, 0.f}, y2[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < (VEC == 1 ? 1 : PW); ++e) {
              const float2 r = cs[u.tok][INTER ? u.at / 2 : u.at + w * PW + e];
              y1[e] = v1[e] * r.x - v2[e] * r.y;
              y2[e] = v2[e] * r.x + v1[e] * r.y;
            }
            x1[s][w] = packed<BF16>(y1[0], y1[1]);
            x2[s][w] = packed<BF16>(y2[0], y2[1]);
          } else if constexpr (BF16) {
            const float2 r = cs[u.tok][u.at / 2 + w];
            const f32x2 v = values<BF16>(x1[s][w]);
            x1[s][w] = packed<BF16>(v[0] * r.x - v[1] * r.y, v[1] * r.x + v[0] * r.y);
          } else if (w % 2 == 0) {
            const float2 r = cs[u.tok][(u.at + w) / 2];
            const float y1 = __uint_as_float(x1[s][w]), y2 = __uint_as_float(x1[s][w + 1]);
            x1[s][w] = __float_as_uint(y1 * r.x - y2 * r.y);
            x1[s][w + 1] = __float_as_uint(y2 * r.x + y1 * r.y);
          }
        }
      }
      void* out;
      int64_t row;
      if (u.kind == 0) {
        if (APPEND && !k.live) continue;
        out = a.q_out;
        row = t * a.qo_tok + u.head * a.qo_head;
      } else if (APPEND) {
        if (k.row < 0) continue;
        out = a.k_out;
        row = k.row + u.head * a.cs_head;
      } else {
        out = a.k_out;
        row = t * a.ko_tok + u.head * a.ko_head;
      }
      store_raw<BF16, VEC>(out, row + u.at, x1[s]);
      if (PAIR && u.turns) store_raw<BF16, VEC>(out, row + second(u), x2[s]);
    }
    if (base + kDepth * NT < total) {
#pragma unroll
      for (int s = 0; s < kDepth; ++s) load(base + kDepth * NT + tid + s * NT, s);
    }
  }
}

}  // namespace
}  // namespace simsd
