// The cache's contents on gfx950: quantising new tokens into 8-bit pages, and
// the checks that the calls on pages share.
#include "peek_internal.h"
#include "peek_kv.h"
#include "peek_validate.h"

namespace peek {

using kv::Pool;
using kv::Rows;
using kv::Table;

namespace {

constexpr int kWave = 64;

// ------------------------------------------------------------------ append
//
// A wavefront owns one (block, K or V, head): it alone writes that block's
// codes and scale. Which block: sequence r's first is given the slot
// offsets[r] / B + 2 r, which leaves every sequence room for the blocks it
// can touch (new tokens / B + 2 at most), so slots need no counting; a slot past its
// sequence's last block has nothing to do.
//
// Bound by memory: 16-byte loads of eight elements, which stay in registers
// from the maximum to the rounding up to HELD of them a lane, as many as a block has,
// 16 at most; larger blocks are read again, from L2. Measured, 72000 tokens of 8 heads
// of 128, 439 MB: 91 to 98 us, 4.5 to 4.8 TB/s, in blocks of 16 tokens (a large copy
// reaches 4.95); of 32 87 us (104 with four a lane), of 64 99 (116), of 256 137 (158);
// blocks of 16 with eight a lane 107. 64 single tokens 5.3 us: the waits for
// offsets, page id, old scale and codes, one after the other.

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

// Four values' codes. `plain`: none is NaN or above the largest code.
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(const float* x, float scale, float inv, bool plain) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = quotient(x[i], scale, inv);
    if (!plain) {
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

template <int TYPE>
__device__ __forceinline__ void spread8(const u4 w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = w[i];
    x[2 * i] = kv::to_float<TYPE>((uint16_t)u);
    x[2 * i + 1] = kv::to_float<TYPE>((uint16_t)(u >> 16));
  }
}

template <int TYPE, int FMT, int D, int HELD>
__global__ __launch_bounds__(256) void k_kv_append(Pool pool, Rows k, Rows v, int32_t n, int64_t num_tokens,
                                                   const int64_t* __restrict__ offsets,
                                                   const int32_t* __restrict__ context, Table table, int64_t slots) {
  constexpr int kPieces = D / 8;       // of a token
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t parts = 2 * pool.heads;
  const int64_t slot = unit / parts;
  if (slot >= slots) return;
  const int32_t part = (int32_t)(unit % parts), is_v = part / pool.heads, head = part % pool.heads;
  const int32_t lb = pool.log_block;
  const int32_t r =
      kv::last_at_most(n, slot, lane, [&](int32_t i) { return (offsets[i] >> lb) + 2 * (int64_t)i; });
  const int64_t start = offsets[r], first = max((int64_t)0, start), end = min(num_tokens, offsets[r + 1]);
  const int64_t ctx = max(0, context[r]);
  const int64_t b = (ctx >> lb) + slot - ((start >> lb) + 2 * (int64_t)r);
  // positions of the block's new tokens
  const int64_t from = max(ctx, b << lb), to = min(ctx + (end - first), (b + 1) << lb);
  if (b < 0 || b >= table.width || from >= to) return;
  const uint32_t page = (uint32_t)table.ids[(int64_t)r * table.stride + b];
  if (page >= pool.num_pages) return;
  const int32_t old = (int32_t)(from - (b << lb)), pieces = (int32_t)(to - from) * kPieces;

  const Rows src = is_v ? v : k;
  const uint16_t* x = (const uint16_t*)src.data + (first + from - ctx) * src.token + head * src.head;
  const int64_t at = ((int64_t)page * 2 + is_v) * pool.heads + head;
  uint8_t* codes = pool.pages + (at << lb) * D;
  const float held = old > 0 ? pool.scales[at] : 0.0f;

  u4 w[HELD];
  auto load = [&](int32_t p0) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int32_t p = p0 + i * kWave + lane;
      w[i] = p < pieces ? *(const u4*)(x + (int64_t)(p / kPieces) * src.token + p % kPieces * 8) : (u4){};
    }
  };
  float most = 0.0f;
  bool plain = true;
  for (int32_t p0 = 0; p0 < pieces; p0 += HELD * kWave) {
    load(p0);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      float y[8];
      spread8<TYPE>(w[i], y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = fabsf(y[e]);
        plain = plain && m < __builtin_inff();
        most = fmaxf(most, m < __builtin_inff() ? m : 0.0f);
      }
    }
  }
  float scale = scale_of<FMT>(wave_max(most));
  plain = __all(plain) && scale < kv::kScaleMax;
  if (old > 0 && !(scale > held)) scale = held;
  const float inv = 1.0f / scale;
  if (old > 0 && scale > held) {
    // older values are at most the largest code times a smaller scale; NaN codes stay NaN
    for (int32_t p = lane; p < old * kPieces; p += kWave) {
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
  for (int32_t p0 = 0; p0 < pieces; p0 += HELD * kWave) {
    if (pieces > HELD * kWave) load(p0);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int32_t p = p0 + i * kWave + lane;
      if (p < pieces) {
        float y[8];
        spread8<TYPE>(w[i], y);
        *(u2*)(codes + old * D + p * 8) =
            (u2){codes_of<FMT>(y, scale, inv, plain), codes_of<FMT>(y + 4, scale, inv, plain)};
      }
    }
  }
  if (lane == 0) pool.scales[at] = scale;
}

// -------------------------------------------------------------- validation
__global__ void k_validate_kv(int32_t n, const int64_t* __restrict__ offsets, int64_t num_tokens,
                              const int32_t* __restrict__ len, bool appends, Table table, int32_t log_block,
                              Pool pool, int32_t* __restrict__ bad) {
  const int32_t r = blockIdx.x;
  int32_t f = 0;
  int64_t fresh = 0;
  if (offsets != nullptr) {
    const int64_t a = offsets[r], b = offsets[r + 1];
    if (a < 0 || b < a || b > num_tokens) f |= 1;
    else fresh = b - a;
  }
  if (len != nullptr) {
    const int64_t held = len[r], all = held + (appends ? fresh : 0);
    if (held < 0 || all > ((int64_t)table.width << log_block)) {
      f |= 2;
    } else {
      const int32_t from = appends ? (int32_t)(held >> log_block) : 0;
      const int32_t to = (int32_t)((all + (1 << log_block) - 1) >> log_block);
      for (int32_t b = from + (int32_t)threadIdx.x; b < to; b += (int32_t)blockDim.x) {
        const int32_t id = table.ids[(int64_t)r * table.stride + b];
        if (id < 0 || (uint32_t)id >= pool.num_pages) {
          f |= 4;
        } else if (pool.scales != nullptr && (int64_t)b << log_block < held) {       // the block holds tokens
          const float* x = pool.scales + (int64_t)id * 2 * pool.heads;
          for (int32_t h = 0; h < pool.heads; ++h) {
            const bool k_fits = appends ? x[h] >= 0 && x[h] <= kv::kScaleMax : fabsf(x[h]) < __builtin_inff();
            const float v = x[pool.heads + h];
            if (!k_fits || !(v >= 0 && v <= kv::kScaleMax)) f |= 8;
          }
        }
      }
    }
  }
  if (f) atomicOr(bad, f);
}

__global__ void k_clear_flag(int32_t* flag) { *flag = 0; }

}  // namespace

peek_status validate_kv(int32_t n, const int64_t* d_offsets, int64_t num_tokens, const int32_t* d_len, bool appends,
                        const int32_t* d_table, int32_t max_blocks, int64_t table_stride, int32_t block_size,
                        const Pool* pool, hipStream_t st) {
  if (!validation_enabled() || n <= 0) return PEEK_OK;
  int32_t* d_bad = nullptr;
  PEEK_HIP_TRY(hipMalloc((void**)&d_bad, sizeof(int32_t)));
  int32_t bad = 0;
  hipLaunchKernelGGL(k_clear_flag, dim3(1), dim3(1), 0, st, d_bad);
  const Pool any{nullptr, nullptr, INT32_MAX, 0, 0};
  hipLaunchKernelGGL(k_validate_kv, dim3((unsigned)n), dim3(64), 0, st, n, d_offsets, num_tokens, d_len, appends,
                     Table{d_table, table_stride, max_blocks}, __builtin_ctz((unsigned)block_size), pool ? *pool : any,
                     d_bad);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = hipMemcpyAsync(&bad, d_bad, sizeof(int32_t), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  (void)hipFree(d_bad);
  if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "input validation failed to run: %s", hipGetErrorString(e));
  if (bad & 1)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "d_offsets must be non-decreasing from 0 or more and end within num_tokens");
  if (bad & 2) return fail(PEEK_ERR_INVALID_ARGUMENT, "a sequence has fewer than 0 tokens or more than its table holds");
  if (bad & 4) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_block_table names pages outside the pool");
  if (bad & 8)
    return fail(PEEK_ERR_INVALID_ARGUMENT,
                "a block's scales are out of range (keys: finite; values, and what an append adds to: 0 to 2^60)");
  return PEEK_OK;
}

peek_status check_pool(const peek_kv_pool* p, Pool* out) {
  if (!p) return fail(PEEK_ERR_INVALID_ARGUMENT, "pool is NULL");
  if (!p->d_pages || !p->d_scales)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "the pool's d_pages and d_scales must not be NULL");
  if ((reinterpret_cast<uintptr_t>(p->d_pages) & 15) != 0)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "the pool's d_pages must be 16-byte aligned");
  if (p->num_pages < 1 || p->num_pages > INT32_MAX)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "num_pages must be in [1, 2^31) (got %lld)", (long long)p->num_pages);
  if (p->kv_heads < 1 || p->kv_heads > 1024)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "kv_heads must be in [1, 1024] (got %d)", p->kv_heads);
  if (p->block_size < 4 || p->block_size > 256 || (p->block_size & (p->block_size - 1)) != 0)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "block_size must be a power of two in [4, 256] (got %d)", p->block_size);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "head_dim must be 64 or 128 (got %d)", p->head_dim);
  if (p->type != PEEK_TYPE_F8E4M3 && p->type != PEEK_TYPE_I8)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "the pool's type must be PEEK_TYPE_F8E4M3 or PEEK_TYPE_I8 (got %d)", p->type);
  *out = Pool{(uint8_t*)p->d_pages, p->d_scales, (uint32_t)p->num_pages, p->kv_heads,
              __builtin_ctz((unsigned)p->block_size)};
  return PEEK_OK;
}

peek_status check_rows(const char* what, const void* data, int64_t token_stride, int64_t head_stride) {
  if (!data) return fail(PEEK_ERR_INVALID_ARGUMENT, "%s must not be NULL", what);
  if ((reinterpret_cast<uintptr_t>(data) & 15) != 0)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned", what);
  if (token_stride < 0 || head_stride < 0 || ((token_stride | head_stride) & 7) != 0)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "%s: strides must be multiples of 8 from 0 on (got %lld, %lld)", what,
                (long long)token_stride, (long long)head_stride);
  return PEEK_OK;
}

peek_status check_out_rows(const char* what, const void* data, int64_t token_stride, int64_t head_stride,
                           int64_t tokens, int32_t heads, int32_t dim) {
  const peek_status s = check_rows(what, data, token_stride, head_stride);
  if (s != PEEK_OK) return s;
  typedef __int128 wide;
  const wide t = token_stride, h = head_stride;
  bool overlap = (tokens > 1 && t < dim) || (heads > 1 && h < dim);
  // tokens whole one after the other, or heads: most layouts. Otherwise head j of a
  // token must not meet the first of one nearby.
  if (!overlap && tokens > 1 && heads > 1 && (heads - 1) * h + dim > t && (tokens - 1) * t + dim > h) {
    for (int32_t j = 1; j < heads && !overlap; ++j) {
      const wide below = j * h / t, off = j * h - below * t;
      overlap = (below >= 1 && below < tokens && off < dim) || (below + 1 < tokens && t - off < dim);
    }
  }
  if (overlap)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "%s: rows of %d elements overlap at strides %lld (tokens) and %lld (heads)",
                what, dim, (long long)token_stride, (long long)head_stride);
  return PEEK_OK;
}

peek_status check_table(const int32_t* table, int32_t max_blocks, int64_t stride, int32_t block_size) {
  if (max_blocks < 0 || stride < max_blocks)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "max_blocks must be >= 0 and table_stride at least that (got %d, %lld)",
                max_blocks, (long long)stride);
  if ((int64_t)max_blocks * block_size > INT32_MAX)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "max_blocks * block_size must be below 2^31 (got %d * %d)", max_blocks,
                block_size);
  if (!table && max_blocks > 0) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_block_table must not be NULL");
  return PEEK_OK;
}

peek_status check_heads(int32_t type, int32_t q_heads, int32_t kv_heads, float scale) {
  if (type != PEEK_TYPE_BF16 && type != PEEK_TYPE_F16)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "type must be PEEK_TYPE_BF16 or PEEK_TYPE_F16 (got %d)", type);
  if (q_heads < 1 || q_heads > 65536 || q_heads % kv_heads != 0)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "q_heads must be a multiple of kv_heads in [1, 65536] (got %d and %d)",
                q_heads, kv_heads);
  if (!std::isfinite(scale)) return fail(PEEK_ERR_INVALID_ARGUMENT, "scale must be finite");
  return PEEK_OK;
}

peek_status check_workspace(const void* d_workspace, size_t bytes, size_t need) {
  if (need == 0) return PEEK_OK;
  if (!d_workspace) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_workspace is NULL");
  if (bytes < need) return fail(PEEK_ERR_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes, got %zu", need, bytes);
  if ((reinterpret_cast<uintptr_t>(d_workspace) & 255) != 0)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "d_workspace must be 256-byte aligned");
  return PEEK_OK;
}

}  // namespace peek

using namespace peek;

extern "C" {

peek_status peek_kv_append(const peek_kv_pool* pool, int32_t n, int64_t num_tokens, int32_t type, const void* d_k,
                           int64_t k_token_stride, int64_t k_head_stride, const void* d_v, int64_t v_token_stride,
                           int64_t v_head_stride, const int64_t* d_offsets, const int32_t* d_context,
                           const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Pool p;
    peek_status s = check_pool(pool, &p);
    if (s != PEEK_OK) return s;
    if (n < 0 || num_tokens < 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "n and num_tokens must be >= 0 (got %d, %lld)", n, (long long)num_tokens);
    if (type != PEEK_TYPE_BF16 && type != PEEK_TYPE_F16)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "type must be PEEK_TYPE_BF16 or PEEK_TYPE_F16 (got %d)", type);
    s = check_table(d_block_table, max_blocks, table_stride, pool->block_size);
    if (s != PEEK_OK) return s;
    if (n == 0 || num_tokens == 0) return PEEK_OK;
    s = check_rows("d_k", d_k, k_token_stride, k_head_stride);
    if (s != PEEK_OK) return s;
    s = check_rows("d_v", d_v, v_token_stride, v_head_stride);
    if (s != PEEK_OK) return s;
    if (!d_offsets || !d_context)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_offsets and d_context must not be NULL");
    const int64_t slots = (num_tokens >> p.log_block) + 2 * (int64_t)n;
    const int64_t groups = (slots * 2 * p.heads + 3) / 4;
    if (groups >= (1 << 24))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many tokens for one call (%lld)", (long long)num_tokens);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, d_offsets, num_tokens, d_context, true, d_block_table, max_blocks, table_stride,
                    pool->block_size, &p, st);
    if (s != PEEK_OK) return s;
    const Rows k{d_k, k_token_stride, k_head_stride}, v{d_v, v_token_stride, v_head_stride};
    const Table t{d_block_table, table_stride, max_blocks};
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, st, p, k, v, n, num_tokens, d_offsets, d_context,
                         t, slots);
    };
    with_types(type, pool->type, pool->head_dim, [&](auto e, auto f, auto d) {
      const int32_t pieces = pool->block_size * d() / 8;      // of a block, K or V
      if (pieces <= 4 * kWave) go(k_kv_append<e(), f(), d(), 4>);
      else if (pieces <= 8 * kWave) go(k_kv_append<e(), f(), d(), 8>);
      else go(k_kv_append<e(), f(), d(), 16>);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "append launch failed: %s", hipGetErrorString(e));
    return PEEK_OK;
  });
}

}  // extern "C"
