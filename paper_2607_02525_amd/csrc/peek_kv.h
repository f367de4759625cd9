// Types and device helpers shared by the calls on the cache's contents
// (append, attention, eviction by attention weight).
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../../include/peek.h"

namespace peek {
namespace kv {

// Scales stay within 2^-60 .. 2^60: their reciprocals and logarithms are then
// ordinary floats, and a weight times a scale cannot leave float32's range. A
// pool may come with others. V's scales of 0, and those that a logarithm or a
// reciprocal might not have, count as 2^-60, or 2^100 where they are larger;
// between these they are as they are, and so is NaN.
constexpr float kScaleMin = 0x1p-60f;
constexpr float kScaleMax = 0x1p60f;
__device__ __forceinline__ float value_scale(float s) {
  return s < 0x1p-100f ? kScaleMin : s > 0x1p100f ? 0x1p100f : s;
}

// A pool as kernels see it.
struct Pool {
  uint8_t* pages;
  float* scales;
  uint32_t num_pages;
  int32_t heads;
  int32_t log_block;   // block_size = 1 << log_block
};

// Rows of heads in 16-bit elements; strides in elements.
struct Rows {
  const void* data;
  int64_t token;
  int64_t head;
};

struct Table {
  const int32_t* ids;
  int64_t stride;
  int32_t width;       // max_blocks
};

// Page of block b of sequence r; a page outside the pool reads as page 0
// (the header's promise: such an id never leads outside the pool's memory).
__device__ __forceinline__ uint32_t page_of(const Table& t, const Pool& p, int32_t r, int32_t b) {
  const uint32_t id = (uint32_t)t.ids[(int64_t)r * t.stride + b];
  return id < p.num_pages ? id : 0u;
}

// Tokens of a sequence as the table can hold them.
__device__ __forceinline__ int32_t clip_tokens(int32_t tokens, int32_t width, int32_t log_block) {
  const int64_t most = (int64_t)width << log_block;
  return tokens < 0 ? 0 : (int64_t)tokens > most ? (int32_t)most : tokens;
}

// A 16-bit element's value and its rounding to nearest, ties to even.
template <int TYPE>
__device__ __forceinline__ float to_float(uint16_t x) {
  if constexpr (TYPE == PEEK_TYPE_BF16) {
    return __builtin_bit_cast(float, (uint32_t)x << 16);
  } else {
    return (float)__builtin_bit_cast(_Float16, x);
  }
}
template <int TYPE>
__device__ __forceinline__ uint16_t from_float(float x) {
  if constexpr (TYPE == PEEK_TYPE_BF16) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
  } else {
    return __builtin_bit_cast(uint16_t, (_Float16)x);
  }
}

// The value of an 8-bit code before its scale.
template <int FMT>
__device__ __forceinline__ float code_value(uint8_t c) {
  if constexpr (FMT == PEEK_TYPE_F8E4M3) {
    return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
  } else {
    return (float)(int8_t)c;
  }
}

// What PEEK_VALIDATE finds.
constexpr int32_t kBadOffsets = 1, kBadLength = 2, kBadPage = 4, kBadScale = 8;

// Of block b of sequence r: its page, and where the pool has scales and the block `holds` tokens these (of one that an
// append adds to: what that asks for).
__device__ __forceinline__ int32_t block_faults(const Table& table, const Pool& pool, int32_t r, int32_t b, bool holds,
                                                bool appends) {
  const int32_t id = table.ids[(int64_t)r * table.stride + b];
  if (id < 0 || (uint32_t)id >= pool.num_pages) return kBadPage;
  if (pool.scales == nullptr || !holds) return 0;
  const float* x = pool.scales + (int64_t)id * 2 * pool.heads;
  int32_t bad = 0;
  for (int32_t h = 0; h < pool.heads; ++h) {
    const bool k_fits = appends ? x[h] >= 0 && x[h] <= kScaleMax : fabsf(x[h]) < __builtin_inff();
    const float v = x[pool.heads + h];
    if (!k_fits || !(v >= 0 && v <= kScaleMax)) bad = kBadScale;
  }
  return bad;
}

// The last r in [0, n) with at(r) <= x, for at() that does not decrease (0 if
// there is none). A wavefront looks at 64 places at a time: one load's
// wait up to 64 sequences, two up to 4096.
template <typename F>
__device__ __forceinline__ int32_t last_at_most(int32_t n, int64_t x, int lane, F&& at) {
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + 63) / 64;
    const int64_t place = lo + (int64_t)lane * step;
    const uint64_t below = __ballot(place < hi && at((int32_t)(place < hi ? place : lo)) <= x);
    const int32_t count = __popcll(below);      // the places are in order, so these are the first
    lo += (count > 0 ? count - 1 : 0) * step;
    hi = count > 0 ? min(hi, lo + step) : lo + 1;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace kv

// Argument checks shared by the entry points (peek_kv.hip).
peek_status check_pool(const peek_kv_pool* pool, kv::Pool* out);
peek_status check_rows(const char* what, const void* data, int64_t token_stride, int64_t head_stride);
// The same for rows that a call writes: no two of them share an element.
peek_status check_out_rows(const char* what, const void* data, int64_t token_stride, int64_t head_stride,
                           int64_t tokens, int32_t heads, int32_t dim);
peek_status check_table(const int32_t* table, int32_t max_blocks, int64_t stride, int32_t block_size);

peek_status check_heads(int32_t type, int32_t q_heads, int32_t kv_heads, float scale);
peek_status check_workspace(const void* d_workspace, size_t bytes, size_t need);

// A caller's scale as the kernels take it: a factor > 0 of base-2 logits, and
// what to do to q's bits so that it is one (a masked logit of -infinity stays one).
inline void set_scale(float scale, float* factor, uint32_t* q_flip, uint32_t* q_mask) {
  const float f = std::fabs(scale) * 1.44269504088896341f;
  const bool none = f == 0.0f;
  *factor = none ? 1.0f : std::fmin(f, 3e38f);
  *q_flip = !none && scale < 0 ? 0x80008000u : 0u;
  *q_mask = none ? 0u : 0xffffffffu;
}

// Calls f with the element type, the cache format and the head's width as constants.
template <typename F>
void with_types(int32_t type, int32_t format, int32_t dim, F&& f) {
  auto by_dim = [&](auto t, auto m) {
    if (dim == 64) f(t, m, std::integral_constant<int, 64>{});
    else f(t, m, std::integral_constant<int, 128>{});
  };
  auto by_format = [&](auto t) {
    if (format == PEEK_TYPE_F8E4M3) by_dim(t, std::integral_constant<int, PEEK_TYPE_F8E4M3>{});
    else by_dim(t, std::integral_constant<int, PEEK_TYPE_I8>{});
  };
  if (type == PEEK_TYPE_BF16) by_format(std::integral_constant<int, PEEK_TYPE_BF16>{});
  else by_format(std::integral_constant<int, PEEK_TYPE_F16>{});
}

// With PEEK_VALIDATE: offsets (nullable) non-decreasing within num_tokens,
// lengths within the table, the pages that they reach (with the new tokens,
// where `appends`) inside the pool, and where `pool` is given the scales of the
// blocks that hold tokens within their range. Waits for `st`. PEEK_OK when off.
peek_status validate_kv(int32_t n, const int64_t* d_offsets, int64_t num_tokens, const int32_t* d_len, bool appends,
                        const int32_t* d_table, int32_t max_blocks, int64_t table_stride, int32_t block_size,
                        const kv::Pool* pool, hipStream_t st);
// These faults as a status, with its message.
peek_status kv_status(int32_t bad);

}  // namespace peek
