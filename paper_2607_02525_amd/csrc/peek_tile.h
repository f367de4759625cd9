// Rows of attention over tiles of 64 keys in LDS: what the prefill and the
// prefix that a group of sequences shares have in common.
//
// A wavefront has 32 rows. K times Q^T leaves lane l with keys of row l % 32
// alone: its maximum and sum need one exchange with the lane 32 away,
// and its weights are already the operand of V^T times weights (peek_mfma.h).
// K and V tiles lie in LDS as 16-bit rows; 16-byte pieces of a row are permuted
// by the row's number so that reads down a column of rows spread over the banks.
// V is read by transposing loads.
#pragma once

#include <hip/hip_runtime.h>

#include "peek_mfma.h"

namespace peek {
namespace mm {

constexpr int kKeys = 64;             // keys of a tile

// Where the 16-byte piece c of row t lies in a tile of D / 8 pieces a row.
template <int D>
__device__ __forceinline__ uint32_t k_piece(uint32_t t, uint32_t c) {
  return t * (D / 8) + (c ^ (t & (D / 8 - 1)));
}
// V is read by 32 lanes at a time, from four adjacent pieces of four rows: all
// of the 64 banks, once these lie in different quarters (halves, where two rows fill the banks).
__device__ __forceinline__ uint32_t v_turn(uint32_t t, int dim) { return dim == 128 ? (t << 2) & 12 : (t << 1) & 4; }
template <int D>
__device__ __forceinline__ uint32_t v_piece(uint32_t t, uint32_t c) {
  return t * (D / 8) + (c ^ v_turn(t, D));
}

typedef __attribute__((address_space(3))) s4 lds_s4;
typedef __attribute__((address_space(3))) u4 lds_u4;
typedef __attribute__((address_space(3))) uint8_t lds_byte;

// What sched_group_barrier calls them.
constexpr int kProducts = 0x8, kLdsReads = 0x100;

// A wavefront's 32 rows, of WAVES wavefronts that share the tiles of keys.
template <int TYPE, int FMT, int D, int WAVES>
struct Tile {
  static constexpr int kPieces = D / 8;                      // of a row
  static constexpr int kBytes = kKeys * D * 2;
  static constexpr int kSteps = D / 16;                      // k steps of K Q^T
  static constexpr int kParts = D / 32;                      // 32-wide parts of the output
  static constexpr int kUnits = 2 * kKeys * (D / 16);        // 16-code units of a cached tile, K and V
  static constexpr int kUnitsEach = kUnits / (64 * WAVES);

  u4 q[kSteps];
  f16 acc[kParts];
  float top, peak, sum;
  uint64_t far;        // of the wavefront: lanes whose row's top is beyond kFar

  // Where lane l begins to read a tile of K, and of V, at `tile` of LDS. From
  // there, k step i is at ^ 32 i and part p of the output at ^ 64 p: addresses
  // that are made anew for every tile take fewer registers than those kept.
  static __device__ __forceinline__ uint32_t k_lane(uint32_t tile, int lane) {
    uint32_t at = tile + 16 * k_piece<D>(lane & 31, lane >> 5);
    asm volatile("" : "+v"(at));
    return at;
  }
  static __device__ __forceinline__ uint32_t v_lane(uint32_t tile, int lane) {
    // lane l reads, for the 16 lanes of its group, four tokens of 16 columns
    const uint32_t i16 = lane & 15, t = 4 * (lane >> 5) + (i16 >> 2), piece = 2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1);
    uint32_t at = tile + 16 * v_piece<D>(t, piece) + 8 * (i16 & 1);
    asm volatile("" : "+v"(at));
    return at;
  }

  // weights of 64 keys and what they add; K and V at these places of LDS
  template <bool CACHED>
  __device__ __forceinline__ void step(uint32_t ks, uint32_t vs, const f4* scales, int lane, float scale, bool masked,
                                       int32_t seen) {
    const int half = lane >> 5;
    const uint32_t at_k = k_lane(ks, lane);
    f16 s[2] = {};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u4 a = *(const lds_u4*)(uintptr_t)((at_k ^ (32 * i)) + 32 * j * D * 2);
        s[j] = mul32<TYPE>(a, q[i], s[j]);
      }
    }
    // LDS reads three products ahead
    __builtin_amdgcn_sched_group_barrier(kLdsReads, 6, 0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      __builtin_amdgcn_sched_group_barrier(kProducts, 2, 0);
      __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 0);
    }
    if constexpr (CACHED) __builtin_amdgcn_sched_barrier(0);      // the scales are read after them
    auto mask = [&]() {
      const int32_t left = seen - 4 * half;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[j][e] = 32 * j + 8 * (e >> 2) + (e & 3) < left ? s[j][e] : -__builtin_inff();
    };
    auto largest = [&]() {
      float most = s[0][0];
#pragma unroll
      for (int e = 1; e < 32; ++e) most = fmaxf(most, s[e >> 4][e & 15]);
      return max_halves(most);
    };
    auto move = [&](float most) {
      const float by = move_top<TYPE>(most, top, peak);
      sum *= by;
#pragma unroll
      for (int p = 0; p < kParts; ++p) acc[p] *= by;
      far = __ballot(fabsf(top) > kFar);
    };
    if constexpr (CACHED) {
      f4 by[8];                  // of keys 4 g .. 4 g + 3: the logits' scale, the values' logarithm and reciprocal
#pragma unroll
      for (int g = 0; g < 8; ++g) by[g] = scales[2 * g + half];
      auto scaled = [&](const f16* from, f16* to, float less) {
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const float add = by[g][1] - less;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            to[g >> 2][(g & 3) * 4 + e] = fmaf(from[g >> 2][(g & 3) * 4 + e], by[g][0], add);
        }
      };
      const f16 raw[2] = {s[0], s[1]};
      scaled(raw, s, top);       // most often that is all
      if ((int)masked | (int)(far != 0) | __any(moves<TYPE>(largest(), 0.0f))) {
        scaled(raw, s, 0.0f);
        move(largest());
#pragma unroll
        for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] -= top;
        // keys past the end are the last one again, so the maximum was right; a key's scale may be 0, so the mask
        // comes after it
        if (masked) mask();
      }
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        s[e >> 4][e & 15] = exp2_fast(s[e >> 4][e & 15]);
        sum = fmaf(s[e >> 4][e & 15], by[e >> 2][2], sum);
      }
    } else {
      if (masked) mask();        // (the call's scale is not 0: -infinity stays)
      const float most = largest() * scale;
      if (__any(moves<TYPE>(most, top))) move(most);
      float by = scale;
      if (far != 0) {
#pragma clang fp contract(off)
        by = 1.0f;
#pragma unroll
        for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] *= scale;
      }
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        s[e >> 4][e & 15] = exp2_fast(fmaf(s[e >> 4][e & 15], by, -top));
        sum += s[e >> 4][e & 15];
      }
    }
    auto weights = [&](int i) {
      const f16& w = s[i >> 1];
      const int o = (i & 1) * 8;
      return (u4){pack2<TYPE>(w[o], w[o + 1]), pack2<TYPE>(w[o + 2], w[o + 3]), pack2<TYPE>(w[o + 4], w[o + 5]),
                  pack2<TYPE>(w[o + 6], w[o + 7])};
    };
    const uint32_t at_v = v_lane(vs, lane);
    auto values = [&](int i, int p) {
      u2 part[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        part[h] = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (lds_s4*)(uintptr_t)((at_v ^ (64 * p)) + (16 * i + 8 * h) * D * 2)));
      return (u4){part[0][0], part[0][1], part[1][0], part[1][1]};
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u4 w = weights(i);
#pragma unroll
      for (int p = 0; p < kParts; ++p) acc[p] = mul32<TYPE>(values(i, p), w, acc[p]);
    }
  }

  // A product's logit, less top.
  __device__ __forceinline__ float logit(float dot, float scale) const {
#pragma clang fp contract(off)
    const float rounded = dot * scale;
    return far != 0 ? rounded - top : fmaf(dot, scale, -top);
  }

  // An element that is infinite or NaN, and eight of them with only those or without.
  static __device__ __forceinline__ bool odd(uint32_t x) {
    return (x & 0x7fffu) >= (TYPE == PEEK_TYPE_BF16 ? 0x7f80u : 0x7c00u);
  }
  static __device__ __forceinline__ uint32_t only(uint32_t w, bool odds) {
    return (odd(w) == odds ? w & 0xffffu : 0u) | (odd(w >> 16) == odds ? w & 0xffff0000u : 0u);
  }

  // Puts zeros for what is infinite or NaN in this wavefront's share of a tile; whether there was any.
  static __device__ __forceinline__ bool clean(uint8_t* tile, int wave, int lane) {
    bool found = false;
#pragma unroll
    for (int i = 0; i < kBytes / 1024 / WAVES; ++i) {
      u4* at = (u4*)(tile + ((i * WAVES + wave) * 64 + lane) * 16);
      const u4 x = *at;
      u4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = only(x[e], false);
      const bool differs = x[0] != y[0] || x[1] != y[1] || x[2] != y[2] || x[3] != y[3];
      if (differs) *at = y;
      found = found || differs;
    }
    return __any(found);
  }

  // Adds the infinite and NaN values of own keys [t0, end) to the rows, of which
  // each sees the first `seen`: one key at a time, so that a row takes only what
  // it sees. With the final maximum; the sum has their weights already.
  __device__ __forceinline__ void add_seen(const uint16_t* k, int64_t k_token, const uint16_t* v, int64_t v_token,
                                           int32_t t0, int32_t end, int half, float scale, int32_t seen) {
    for (int32_t t = t0; t < end; ++t) {
      float dot = 0.0f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const u4 x = *(const u4*)(k + t * k_token + 16 * i + 8 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t a = x[e], b = q[i][e];
          dot = fmaf(kv::to_float<TYPE>((uint16_t)a), kv::to_float<TYPE>((uint16_t)b), dot);
          dot = fmaf(kv::to_float<TYPE>((uint16_t)(a >> 16)), kv::to_float<TYPE>((uint16_t)(b >> 16)), dot);
        }
      }
      const float w = exp2_fast(logit(sum_halves(dot), scale));
      if (t >= seen) continue;
#pragma unroll
      for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const u2 x = *(const u2*)(v + t * v_token + 32 * p + 8 * e + 4 * half);
          const uint32_t a = only(x[0], true), b = only(x[1], true);
          acc[p][4 * e] = fmaf(w, kv::to_float<TYPE>((uint16_t)a), acc[p][4 * e]);
          acc[p][4 * e + 1] = fmaf(w, kv::to_float<TYPE>((uint16_t)(a >> 16)), acc[p][4 * e + 1]);
          acc[p][4 * e + 2] = fmaf(w, kv::to_float<TYPE>((uint16_t)b), acc[p][4 * e + 2]);
          acc[p][4 * e + 3] = fmaf(w, kv::to_float<TYPE>((uint16_t)(b >> 16)), acc[p][4 * e + 3]);
        }
    }
  }
};

}  // namespace mm
}  // namespace peek
