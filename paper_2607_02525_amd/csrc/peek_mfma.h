// Matrix-core products and 8-bit conversions for the attention kernels.
//
// Lane layouts on gfx950 (64 lanes, l the lane):
//   32x32x16: A lane l holds row l % 32, k = 8 (l / 32) .. + 7; B the same of column l % 32;
//             C register v of lane l is row 8 (v / 4) + 4 (l / 32) + v % 4, column l % 32
//   16x16x32: A lane l holds row l % 16, k = 8 (l / 16) .. + 7; B the same of column l % 16;
//             C register v of lane l is row 4 (l / 16) + v, column l % 16
// k is summed over, so any order of it serves that A and B share. That is what
// keeps weights in registers: keys times queries leaves a lane with four
// (or 16) keys of one query, which is one lane's share of the B operand of
// values times weights, once the values' tokens are taken in the same order.
#pragma once

#include <hip/hip_runtime.h>

#include "peek_kv.h"

namespace peek {
namespace mm {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

template <int TYPE>
__device__ __forceinline__ f16 mul32(u4 a, u4 b, f16 c) {
  if constexpr (TYPE == PEEK_TYPE_BF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
}
template <int TYPE>
__device__ __forceinline__ f4 mul16(u4 a, u4 b, f4 c) {
  if constexpr (TYPE == PEEK_TYPE_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
}

// Two floats to a pair of 16-bit elements, to nearest, ties to even.
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (TYPE == PEEK_TYPE_BF16) {
    return __builtin_bit_cast(uint32_t, (b2){(__bf16)a, (__bf16)b});
  } else {
    return __builtin_bit_cast(uint32_t, (h2){(_Float16)a, (_Float16)b});
  }
}

// Four codes to 16-bit elements: exact, both formats' values have at most
// eight significant bits and lie within float16's range.
template <int TYPE, int FMT>
__device__ __forceinline__ u2 widen4(uint32_t w) {
  u2 r;
  if constexpr (FMT == PEEK_TYPE_F8E4M3 && TYPE == PEEK_TYPE_BF16) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  } else if constexpr (FMT == PEEK_TYPE_F8E4M3) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  } else {
    r[0] = pack2<TYPE>((float)(int8_t)w, (float)(int8_t)(w >> 8));
    r[1] = pack2<TYPE>((float)(int8_t)(w >> 16), (float)((int32_t)w >> 24));
  }
  return r;
}

// The larger, or the sum, of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float max_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// Over the lanes that hold the same row: l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float swap16_max(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float swap16_sum(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// Four tokens of four bytes each -> four bytes' worth of four tokens.
__device__ __forceinline__ void turn4(const uint32_t a, const uint32_t b, const uint32_t c, const uint32_t d,
                                      uint32_t* r) {
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602);
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602);
  r[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100);
  r[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302);
  r[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100);
  r[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302);
}

// ------------------------------------------- running softmax, parts of a row
// A row's weights are 2^(x - top), of 16 bits where they meet the values. Where a
// tile's largest x lies too far from `top`, top moves and what the row has
// summed is scaled along; most tiles move nothing.
//
// bfloat16 has float32's range: top is the largest x, or one up to 2^8 smaller.
//
// float16 ends at 2^16 and loses bits below 2^-14, nearly all of them at 2^-24.
// Small weights are often many, and together as much as the largest: all that
// lies 14 nats below one key is a tenth of the sum from 130000 keys on, more
// than that of the numerator where its V scale is smaller. So a
// move puts a tile's largest weight at 2^7, up to 2^15 are let pass, and
// top also moves down, when a tile's largest falls below 2^-8: rounding takes
// from a weight 2^-11 of itself or 2^-17 of its own tile's largest at most, down
// to kDeep + 15 below the row's (no further: the sum must stay within float32,
// weights being divided by scales of 2^-60 and more). top is a whole number,
// and every move exact. (Moves below 2^-2 came often where keys' scales differ by
// 4 from block to block: 64 prompts over such a cache 1.25 ms, 1.18 with 2^-8, 1.15 where top only rises.)
constexpr float kSlack = 8.0f;
constexpr float kLeast = -8.0f, kMost = 15.0f, kMiddle = 7.0f, kDeep = 24.0f;
constexpr float kNone = -3.402823466e38f;      // a maximum of nothing: no logit is lower, and differences are numbers
// Beyond this, x - top is a difference of numbers rounded alike, not the rounded difference of x's product: that may be
// off by half a unit of top's, and 2^ that out of any range.
constexpr float kFar = 0x1p22f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// top + log2(sum), the sum's power of two taken out first: the logarithm of a number near 2^7, where a float16 row's
// largest weight lies, has a unit many times as large as its fraction's. (A block's weight and its row's sum take the
// same one: beside a top of 1e9 other sums of the same parts differ by whole powers of two.)
__device__ __forceinline__ float log2_sum(float top, float sum) {
  return top + (float)__builtin_amdgcn_frexp_expf(sum) + log2_fast(__builtin_amdgcn_frexp_mantf(sum));
}

// Whether a tile whose largest x is `most` moves top.
template <int TYPE>
__device__ __forceinline__ bool moves(float most, float top) {
  if constexpr (TYPE == PEEK_TYPE_BF16) return most > top + kSlack;
  else return fabsf(most - top - (kMost + kLeast) / 2) > (kMost - kLeast) / 2;
}

// Moves top for such a tile (or leaves it, for another); what to scale sums by. `peak` is the highest top so far.
template <int TYPE>
__device__ __forceinline__ float move_top(float most, float& top, float& peak) {
  float next = top;
  if constexpr (TYPE == PEEK_TYPE_BF16) {
    if (most > top + kSlack) next = most;
    const float by = exp2_fast(top - next);
    top = next;
    return by;
  } else {
    const float here = floorf(most) - kMiddle;
    if (most > top + kMost) next = here;
    else if (most < top + kLeast && most > -__builtin_inff()) next = fminf(top, fmaxf(here, peak - kDeep));
    const float by = __builtin_ldexpf(1.0f, (int)fmaxf(top - next, -1000.0f));
    top = next;
    peak = fmaxf(peak, top);
    return by;
  }
}

// Base-2 logarithm of a row's sum of weights from its parts' (-infinity: none), by a whole wavefront.
__device__ __forceinline__ float row_log_sum(const float* __restrict__ p, int32_t parts, int lane) {
  float top = kNone, sum = 0.0f;
  for (int32_t s = lane; s < parts; s += 64) {
    const float x = p[s], next = fmaxf(top, x);
    sum = sum * exp2_fast(top - next) + exp2_fast(x - next);
    top = next;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float x = __shfl_xor(top, d), y = __shfl_xor(sum, d), next = fmaxf(top, x);
    sum = sum * exp2_fast(top - next) + y * exp2_fast(x - next);
    top = next;
  }
  return log2_sum(top, sum);
}

// A row's parts [parts][D] joined by WAVES wavefronts of a workgroup, this one
// the wave-th with its share of them: a lane to each part for its weight and to
// D / 64 elements for the sum. `out` is the row's; s_sum, for WAVES > 1, has
// WAVES * D floats.
template <int TYPE, int D, int WAVES>
__device__ __forceinline__ void join_parts(const float* __restrict__ part_out, const float* __restrict__ lse,
                                           int32_t parts, int wave, int lane, float* s_sum, uint16_t* out,
                                           float* log_sum) {
  constexpr int kEach = D / 64;
  const float l2 = row_log_sum(lse, parts, lane);
  float o[kEach] = {};
  const float* from = part_out + lane * kEach;
  const int32_t share = (parts + WAVES - 1) / WAVES, end = min(parts, (wave + 1) * share);
  for (int32_t s0 = wave * share; s0 < end; s0 += 64) {
    const int32_t count = min(64, end - s0);
    const float mine = lane < count ? exp2_fast(lse[s0 + lane] - l2) : 0.0f;
    for (int32_t s1 = 0; s1 < count; s1 += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {      // those past the last read the last again, as 0 (it may be infinite)
        const int32_t s = s1 + i;
        const float part = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, mine), s));
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const float x = from[(int64_t)(s0 + min(s, count - 1)) * D + e];
          o[e] = fmaf(part, s < count ? x : 0.0f, o[e]);
        }
      }
    }
  }
  *log_sum = l2;
  if constexpr (WAVES == 1) {
    if constexpr (kEach == 2) *(uint32_t*)(out + 2 * lane) = pack2<TYPE>(o[0], o[1]);
    else out[lane] = kv::from_float<TYPE>(o[0]);
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e) s_sum[wave * D + lane * kEach + e] = o[e];
    __syncthreads();
    const int d = wave * 64 + lane;
    if (d < D) {
      float x = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) x += s_sum[w * D + d];
      out[d] = kv::from_float<TYPE>(x);
    }
  }
}

}  // namespace mm
}  // namespace peek
