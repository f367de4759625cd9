// Attention over the paged 8-bit cache on gfx950: packed prompts after their
// cached prefix, and single tokens.
#include <cmath>

#include "peek_internal.h"
#include "peek_kv.h"
#include "peek_validate.h"

namespace peek {

using kv::Pool;
using kv::Rows;
using kv::Table;

namespace {

constexpr int kWave = 64;

__device__ __forceinline__ float wave_sum(float x) {
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// One row of one query head, spread over a wavefront: lane l has elements
// E l .. E l + E - 1. The running maximum, sum and weighted values of its softmax.
template <int E>
struct Row {
  float q[E], acc[E], top, sum;

  __device__ __forceinline__ float logit(const float* k, float scale) const {
    float s = 0.0f;
    for (int e = 0; e < E; ++e) s += q[e] * k[e];
    return wave_sum(s) * scale;
  }
  __device__ __forceinline__ void add(float x, const float* v) {
    const float next = fmaxf(top, x), old = expf(top - next), w = expf(x - next);
    for (int e = 0; e < E; ++e) acc[e] = acc[e] * old + w * v[e];
    sum = sum * old + w;
    top = next;
  }
};

template <int TYPE, int E>
__device__ __forceinline__ void load_row(const Rows& rows, int64_t token, int32_t head, int lane, float* x) {
  const uint16_t* p = (const uint16_t*)rows.data + token * rows.token + head * rows.head + lane * E;
  for (int e = 0; e < E; ++e) x[e] = kv::to_float<TYPE>(p[e]);
}

template <int FMT, int E>
__device__ __forceinline__ void load_cached(const Pool& pool, const Table& table, int32_t r, int32_t t, int32_t is_v,
                                            int32_t head, int lane, float* x) {
  const uint32_t page = kv::page_of(table, pool, r, t >> pool.log_block);
  const int64_t at = ((int64_t)page * 2 + is_v) * pool.heads + head;
  const uint8_t* p = pool.pages + ((at << pool.log_block) + (t & ((1 << pool.log_block) - 1))) * (E * kWave) + lane * E;
  const float scale = pool.scales[at];
  for (int e = 0; e < E; ++e) x[e] = kv::code_value<FMT>(p[e]) * scale;
}

// A wavefront per row and query head.
template <int TYPE, int FMT, int E>
__global__ __launch_bounds__(256) void k_prefill(Pool pool, Rows q, Rows k, Rows v, int32_t n, int64_t num_tokens,
                                                 int32_t group, const int64_t* __restrict__ offsets,
                                                 const int32_t* __restrict__ prefix, Table table, float scale,
                                                 uint16_t* __restrict__ out, int64_t out_token, int64_t out_head,
                                                 float* __restrict__ lse, int32_t q_heads) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int64_t token = unit / q_heads;
  const int32_t head = (int32_t)(unit % q_heads);
  if (token >= num_tokens) return;
  const int32_t r = kv::sequence_of(offsets, n, token);
  const int64_t first = offsets[r];
  if (first < 0 || token < first || token >= offsets[r + 1]) return;
  const int32_t held = prefix ? kv::clip_tokens(prefix[r], table.width, pool.log_block) : 0;
  Row<E> row;
  load_row<TYPE, E>(q, token, head, lane, row.q);
  for (int e = 0; e < E; ++e) row.acc[e] = 0.0f;
  row.top = -__builtin_inff();
  row.sum = 0.0f;
  float a[E], b[E];
  for (int32_t j = 0; j < held; ++j) {
    load_cached<FMT, E>(pool, table, r, j, 0, head / group, lane, a);
    load_cached<FMT, E>(pool, table, r, j, 1, head / group, lane, b);
    row.add(row.logit(a, scale), b);
  }
  for (int64_t j = first; j <= token; ++j) {
    load_row<TYPE, E>(k, j, head / group, lane, a);
    load_row<TYPE, E>(v, j, head / group, lane, b);
    row.add(row.logit(a, scale), b);
  }
  for (int e = 0; e < E; ++e)
    out[token * out_token + head * out_head + lane * E + e] = kv::from_float<TYPE>(row.acc[e] / row.sum);
  if (lse && lane == 0) lse[token * q_heads + head] = row.top + logf(row.sum);
}

// A wavefront per sequence and kv head; the group's heads one after the other.
template <int TYPE, int FMT, int E>
__global__ __launch_bounds__(kWave) void k_decode(Pool pool, Rows q, int32_t group, const int32_t* __restrict__ context,
                                                  Table table, float scale, uint16_t* __restrict__ out,
                                                  int64_t out_token, int64_t out_head, float* __restrict__ lse,
                                                  const float* mass_in, float* mass, float* __restrict__ row_lse) {
  const int lane = threadIdx.x;
  const int32_t r = blockIdx.x / pool.heads, h = blockIdx.x % pool.heads;
  const int32_t held = kv::clip_tokens(context[r], table.width, pool.log_block);
  const int32_t q_heads = group * pool.heads;
  Row<E> row;
  float a[E], b[E];
  for (int32_t g = 0; g < group; ++g) {
    const int32_t head = h * group + g;
    load_row<TYPE, E>(q, r, head, lane, row.q);
    for (int e = 0; e < E; ++e) row.acc[e] = 0.0f;
    row.top = -__builtin_inff();
    row.sum = 0.0f;
    for (int32_t j = 0; j < held; ++j) {
      load_cached<FMT, E>(pool, table, r, j, 0, h, lane, a);
      load_cached<FMT, E>(pool, table, r, j, 1, h, lane, b);
      row.add(row.logit(a, scale), b);
    }
    const float whole = held > 0 ? row.top + logf(row.sum) : -__builtin_inff();
    for (int e = 0; e < E; ++e)
      out[(int64_t)r * out_token + head * out_head + lane * E + e] =
          kv::from_float<TYPE>(held > 0 ? row.acc[e] / row.sum : 0.0f);
    if (lane == 0) {
      if (lse) lse[(int64_t)r * q_heads + head] = whole;
      row_lse[(int64_t)r * q_heads + head] = whole;
    }
  }
  if (!mass) return;
  __syncthreads();
  const int32_t block = 1 << pool.log_block;
  for (int32_t blk = 0; blk < table.width; ++blk) {
    float w = 0.0f;
    for (int32_t g = 0; g < group && (blk << pool.log_block) < held; ++g) {
      load_row<TYPE, E>(q, r, h * group + g, lane, row.q);
      const float whole = row_lse[(int64_t)r * q_heads + h * group + g];
      for (int32_t j = blk << pool.log_block; j < min(held, (blk << pool.log_block) + block); ++j) {
        load_cached<FMT, E>(pool, table, r, j, 0, h, lane, a);
        w += expf(row.logit(a, scale) - whole);
      }
    }
    const int64_t at = ((int64_t)r * pool.heads + h) * table.width + blk;
    if (lane == 0) mass[at] = (mass_in ? mass_in[at] : 0.0f) + w;
  }
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

// Calls f with the element type, cache format and elements per lane as constants.
template <typename F>
void with_types(int32_t type, int32_t format, int32_t dim, F&& f) {
  auto by_dim = [&](auto t, auto m) {
    if (dim == 64) f(t, m, std::integral_constant<int, 1>{});
    else f(t, m, std::integral_constant<int, 2>{});
  };
  auto by_format = [&](auto t) {
    if (format == PEEK_TYPE_F8E4M3) by_dim(t, std::integral_constant<int, PEEK_TYPE_F8E4M3>{});
    else by_dim(t, std::integral_constant<int, PEEK_TYPE_I8>{});
  };
  if (type == PEEK_TYPE_BF16) by_format(std::integral_constant<int, PEEK_TYPE_BF16>{});
  else by_format(std::integral_constant<int, PEEK_TYPE_F16>{});
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

size_t peek_prefill_attention_workspace(int32_t n, int64_t num_tokens, int32_t q_heads, int32_t kv_heads,
                                        int32_t head_dim, int64_t max_context) {
  return 0;
}

peek_status peek_prefill_attention(const peek_kv_pool* pool, int32_t n, int64_t num_tokens, int32_t type,
                                   int32_t q_heads, int32_t kv_heads, int32_t head_dim, const void* d_q,
                                   int64_t q_token_stride, int64_t q_head_stride, const void* d_k,
                                   int64_t k_token_stride, int64_t k_head_stride, const void* d_v,
                                   int64_t v_token_stride, int64_t v_head_stride, const int64_t* d_offsets,
                                   const int32_t* d_prefix, const int32_t* d_block_table, int32_t max_blocks,
                                   int64_t table_stride, float scale, void* d_out, int64_t out_token_stride,
                                   int64_t out_head_stride, float* d_lse, void* d_workspace, size_t workspace_bytes,
                                   void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    if (n < 0 || num_tokens < 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "n and num_tokens must be >= 0 (got %d, %lld)", n, (long long)num_tokens);
    if (kv_heads < 1 || kv_heads > 1024)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "kv_heads must be in [1, 1024] (got %d)", kv_heads);
    if (head_dim != 64 && head_dim != 128)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "head_dim must be 64 or 128 (got %d)", head_dim);
    peek_status s = check_heads(type, q_heads, kv_heads, scale);
    if (s != PEEK_OK) return s;
    Pool p{};
    if ((pool != nullptr) != (d_prefix != nullptr))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "pool and d_prefix must be given together");
    if (pool) {
      s = check_pool(pool, &p);
      if (s != PEEK_OK) return s;
      if (pool->kv_heads != kv_heads || pool->head_dim != head_dim)
        return fail(PEEK_ERR_INVALID_ARGUMENT, "the pool has %d heads of %d, the rows %d of %d", pool->kv_heads,
                    pool->head_dim, kv_heads, head_dim);
      s = check_table(d_block_table, max_blocks, table_stride, pool->block_size);
      if (s != PEEK_OK) return s;
    }
    if (n == 0 || num_tokens == 0) return PEEK_OK;
    if ((s = check_rows("d_q", d_q, q_token_stride, q_head_stride)) != PEEK_OK) return s;
    if ((s = check_rows("d_k", d_k, k_token_stride, k_head_stride)) != PEEK_OK) return s;
    if ((s = check_rows("d_v", d_v, v_token_stride, v_head_stride)) != PEEK_OK) return s;
    if ((s = check_rows("d_out", d_out, out_token_stride, out_head_stride)) != PEEK_OK) return s;
    if (!d_offsets) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_offsets must not be NULL");
    const int64_t context = pool ? (int64_t)max_blocks * pool->block_size : 0;
    s = check_workspace(d_workspace, workspace_bytes,
                        peek_prefill_attention_workspace(n, num_tokens, q_heads, kv_heads, head_dim, context));
    if (s != PEEK_OK) return s;
    const int64_t groups = (num_tokens * q_heads + 3) / 4;
    if (groups >= (1 << 24)) return fail(PEEK_ERR_INVALID_ARGUMENT, "too many rows for one call (%lld)", (long long)num_tokens);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, d_offsets, num_tokens, d_prefix, false, d_block_table, max_blocks, table_stride,
                    pool ? pool->block_size : 4, pool ? pool->num_pages : 0, st);
    if (s != PEEK_OK) return s;
    with_types(type, pool ? pool->type : PEEK_TYPE_F8E4M3, head_dim, [&](auto t, auto m, auto e) {
      hipLaunchKernelGGL((k_prefill<t(), m(), e()>), dim3((unsigned)groups), dim3(256), 0, st, p,
                         Rows{d_q, q_token_stride, q_head_stride}, Rows{d_k, k_token_stride, k_head_stride},
                         Rows{d_v, v_token_stride, v_head_stride}, n, num_tokens, q_heads / kv_heads, d_offsets,
                         d_prefix, Table{d_block_table, table_stride, max_blocks}, scale, (uint16_t*)d_out,
                         out_token_stride, out_head_stride, d_lse, q_heads);
    });
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(PEEK_ERR_DEVICE, "prefill launch failed: %s", hipGetErrorString(err));
    return PEEK_OK;
  });
}

size_t peek_decode_attention_workspace(const peek_kv_pool* pool, int32_t n, int32_t q_heads, int32_t max_blocks,
                                       int32_t with_mass) {
  if (!pool || n < 0 || q_heads < 1 || max_blocks < 0) return 0;
  return ((size_t)n * q_heads * sizeof(float) + 255) & ~(size_t)255;
}

peek_status peek_decode_attention(const peek_kv_pool* pool, int32_t n, int32_t type, int32_t q_heads, const void* d_q,
                                  int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_context,
                                  const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, float scale,
                                  void* d_out, int64_t out_token_stride, int64_t out_head_stride, float* d_lse,
                                  const float* d_mass_in, float* d_mass, void* d_workspace, size_t workspace_bytes,
                                  void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Pool p;
    peek_status s = check_pool(pool, &p);
    if (s != PEEK_OK) return s;
    if (n < 0) return fail(PEEK_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
    s = check_heads(type, q_heads, p.heads, scale);
    if (s != PEEK_OK) return s;
    s = check_table(d_block_table, max_blocks, table_stride, pool->block_size);
    if (s != PEEK_OK) return s;
    if (d_mass_in && !d_mass) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_mass_in needs d_mass");
    if (n == 0) return PEEK_OK;
    if ((s = check_rows("d_q", d_q, q_token_stride, q_head_stride)) != PEEK_OK) return s;
    if ((s = check_rows("d_out", d_out, out_token_stride, out_head_stride)) != PEEK_OK) return s;
    if (!d_context) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_context must not be NULL");
    s = check_workspace(d_workspace, workspace_bytes,
                        peek_decode_attention_workspace(pool, n, q_heads, max_blocks, d_mass != nullptr));
    if (s != PEEK_OK) return s;
    if ((int64_t)n * p.heads >= (1 << 24)) return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, pool->block_size,
                    pool->num_pages, st);
    if (s != PEEK_OK) return s;
    with_types(type, pool->type, pool->head_dim, [&](auto t, auto m, auto e) {
      hipLaunchKernelGGL((k_decode<t(), m(), e()>), dim3((unsigned)(n * p.heads)), dim3(kWave), 0, st, p,
                         Rows{d_q, q_token_stride, q_head_stride}, q_heads / p.heads, d_context,
                         Table{d_block_table, table_stride, max_blocks}, scale, (uint16_t*)d_out, out_token_stride,
                         out_head_stride, d_lse, d_mass_in, d_mass, (float*)d_workspace);
    });
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(PEEK_ERR_DEVICE, "decode launch failed: %s", hipGetErrorString(err));
    return PEEK_OK;
  });
}

}  // extern "C"
