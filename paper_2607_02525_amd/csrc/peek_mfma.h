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

}  // namespace mm
}  // namespace peek
