// Rounding rows of 16-bit elements to 8-bit codes with a scale: what the calls
// that write pages share.
#pragma once

#include <hip/hip_runtime.h>

#include "peek_kv.h"

namespace peek {
namespace quant {

__device__ __forceinline__ float wave_max(float x) {
  for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// The scale of a block whose largest finite magnitude is `most`.
template <int FMT>
__device__ __forceinline__ float scale_of(float most) {
  if constexpr (FMT == PEEK_TYPE_F8E4M3) {
    // most = m * 2^e with m in [1, 2); 448 = 1.75 * 2^8
    const uint32_t bits = __builtin_bit_cast(uint32_t, most);
    int32_t e = (int32_t)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = max(-60, min(60, e));
    return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
  } else {
    return fminf(fmaxf(most * (1.0f / 127.0f), kv::kScaleMin), kv::kScaleMax);
  }
}

// x / scale, correctly rounded where it is below 512 (beyond, any value there
// is as good): the product with the rounded reciprocal is at most two units off,
// its remainder is exact, and the quotient corrected by that is the nearest.
__device__ __forceinline__ float quotient(float x, float scale, float inv) {
  const float y = x * inv;
  return fabsf(y) < 512.0f ? fmaf(fmaf(-y, scale, x), inv, y) : y;
}

// Whether values that are `plain` to their own scale (below) are so to the one that their block holds. Float8's scales
// are powers of two where an append made them, but older tokens may have come with any other: a product with its
// rounded reciprocal can fall on the wrong side of a tie between two codes (29 of float16's numbers at a scale of 7).
template <int FMT>
__device__ __forceinline__ bool plain_scale(float scale) {
  return FMT != PEEK_TYPE_F8E4M3 || (__builtin_bit_cast(uint32_t, scale) & 0x7fffffu) == 0;
}

// Four values' codes. `plain`: all are finite and below a code beyond the largest, and a float8 scale is a power of two:
// then that one needs no correction, and the other format's no look at the quotient's size.
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(const float* x, float scale, float inv, bool plain) {
  float y[4];
  if (plain) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = x[i] * inv;
      if constexpr (FMT == PEEK_TYPE_I8) y[i] = fmaf(fmaf(-y[i], scale, x[i]), inv, y[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = quotient(x[i], scale, inv);
      if constexpr (FMT == PEEK_TYPE_F8E4M3) y[i] = y[i] < -448.0f ? -448.0f : y[i] > 448.0f ? 448.0f : y[i];
      else y[i] = y[i] != y[i] ? 0.0f : y[i] < -127.0f ? -127.0f : y[i] > 127.0f ? 127.0f : y[i];
    }
  }
  if constexpr (FMT == PEEK_TYPE_F8E4M3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  } else {
    // 1.5 * 2^23 + y has y, rounded to nearest even, in its low byte
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_bit_cast(uint32_t, y[i] + 12582912.0f);
    return __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400) | __builtin_amdgcn_perm(u[3], u[2], 0x04000c0c);
  }
}

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef unsigned short p2u __attribute__((ext_vector_type(2)));

template <int TYPE>
__device__ __forceinline__ void spread8(const u4 w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = w[i];
    x[2 * i] = kv::to_float<TYPE>((uint16_t)u);
    x[2 * i + 1] = kv::to_float<TYPE>((uint16_t)(u >> 16));
  }
}

// Magnitudes of 16-bit elements are in the order of their bits without the sign: the largest of eight and of those in
// `most`, two side by side. (Infinities and NaN are above every number: kInfinity and more.)
template <int TYPE>
constexpr uint32_t kInfinity = TYPE == PEEK_TYPE_BF16 ? 0x7f80u : 0x7c00u;
__device__ __forceinline__ uint32_t largest8(const u4 w, uint32_t most) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(p2u, most),
                                                                  __builtin_bit_cast(p2u, w[i] & 0x7fff7fffu)));
  return most;
}
// Of a wavefront.
__device__ __forceinline__ uint32_t wave_largest(uint32_t most) {
  most = max(most & 0xffffu, most >> 16);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) most = max(most, (uint32_t)__shfl_xor(most, d));
  return __builtin_amdgcn_readfirstlane(most);
}
// The largest finite magnitude of eight elements and of `most`.
template <int TYPE>
__device__ __forceinline__ float finite8(const u4 w, float most) {
  float x[8];
  spread8<TYPE>(w, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float m = fabsf(x[e]);
    most = fmaxf(most, m < __builtin_inff() ? m : 0.0f);
  }
  return most;
}

// `count` codes (a multiple of 8) of a scale rounded again to a larger one, by a wavefront. Values are at most the
// largest code times the smaller scale; NaN codes stay NaN.
template <int FMT>
__device__ __forceinline__ void rescale(uint8_t* codes, int32_t count, float held, float scale, float inv, int lane) {
  for (int32_t p = lane; p < count / 8; p += 64) {
    u2 c = *(const u2*)(codes + p * 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float y[4];
      const uint32_t word = c[h];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = kv::code_value<FMT>((uint8_t)(word >> (8 * e))) * held;
      c[h] = codes_of<FMT>(y, scale, inv, false);
    }
    *(u2*)(codes + p * 8) = c;
  }
}

}  // namespace quant
}  // namespace peek
