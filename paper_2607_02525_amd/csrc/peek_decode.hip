// Attention of single tokens over the paged 8-bit cache on gfx950.
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

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

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
    with_types(type, pool->type, pool->head_dim, [&](auto t, auto m, auto d) {
      hipLaunchKernelGGL((k_decode<t(), m(), d() / kWave>), dim3((unsigned)(n * p.heads)), dim3(kWave), 0, st, p,
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
