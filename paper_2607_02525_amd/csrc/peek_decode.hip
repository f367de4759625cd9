// Attention of single tokens over the paged 8-bit cache, on gfx950.
//
// Bound by reading the pages once: a kv head's keys and values serve the
// group's query heads together, as 16 rows of the matrix products. A
// workgroup of four wavefronts takes one chunk of one sequence's tokens for one
// kv head and 16 of its rows; a wavefront takes every fourth tile of 32
// tokens, on its own, with a running maximum and sum. Long sequences are split
// into chunks so that a few of them still fill the device; the chunks'
// results are joined by a second kernel, in a fixed order.
//
// Nothing but the final join of the wavefronts goes through LDS: the order in
// which k is summed is free (peek_mfma.h), so
//   keys:    lane l loads D/4 adjacent bytes of token l % 16, which are its
//            parts of D/32 products, and q is laid out to match;
//   weights: keys times queries leaves lane l with tokens 4 (l / 16) .. + 3 of
//            both 16-token halves, for row l % 16: eight of 32, the
//            operand of the second product;
//   values:  lane l loads D/16 adjacent bytes of those eight tokens and turns
//            them round in registers, four tokens by four bytes at a time.
// Scales never touch the codes, as in the prefill: K's multiplies the logit,
// V's is added to it as an exponent, and the sum divides by it again.
//
// With weights wanted, every row's weight of every 16 tokens (of a block, where
// that is smaller) is kept as a logarithm, which needs no maximum to go with
// it; the second kernel sums them over the rows once the rows' sums are known.
#include <algorithm>

#include "peek_internal.h"
#include "peek_kv.h"
#include "peek_mfma.h"
#include "peek_validate.h"

namespace peek {

using kv::Pool;
using kv::Rows;
using kv::Table;
using namespace mm;

namespace {

constexpr int kWave = 64;
constexpr int kWaves = 4;
constexpr int kThreads = kWave * kWaves;
constexpr int kRows = 16;
constexpr int kTile = 32;                        // tokens of a wavefront's step
constexpr int kMaxChunk = 2048;                  // tokens of a workgroup, at most
constexpr float kSlack = 8.0f;                   // see peek_prefill.hip
constexpr float kNone = -1e30f;

struct Decode {
  Pool pool;
  Rows q;
  const int32_t* context;
  Table table;
  uint16_t* out;
  int64_t out_token, out_head;
  float* lse;
  const float* mass_in;
  float* mass;
  float* part_out;       // [n][splits][q_heads][D]: a chunk's sum of weight * value / its sum of weights
  float* part_lse;       // [n][splits][q_heads]: base-2 logarithm of its sum of weights
  float* weights;        // [n][q_heads][grains]: base-2 logarithm of the weight on every grain of tokens
  int64_t grains;
  int32_t log_grain;
  int32_t n, group, row_tiles, chunk, splits;
  float scale;
  uint32_t q_flip, q_mask;
};

// What the products need of a block: its logits' scale, the logarithm and the
// reciprocal of its values' scale, and where it lies.
struct alignas(16) Block {
  float scale, log_v, inv_v;
  uint32_t page;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

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

template <int TYPE, int FMT, int D, bool MASS>
__global__ __launch_bounds__(kThreads) void k_decode(Decode a) {
  constexpr int kSteps = D / 32;        // products of keys and queries a 16-token half
  constexpr int kParts = D / 16;        // 16-wide parts of the output; also bytes of a token's values in a lane
  constexpr int kKeyWords = D / 16;     // words of a token's key in a lane
  __shared__ Block s_block[kMaxChunk / 4 + 1];           // of the chunk's blocks
  __shared__ float s_out[kWaves][kRows][D + 4];
  __shared__ float s_top[kWaves][kRows], s_sum[kWaves][kRows];

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  uint32_t unit = blockIdx.x;
  const int32_t head = unit % a.pool.heads;
  unit /= a.pool.heads;
  const int32_t row_tile = unit % a.row_tiles;
  unit /= a.row_tiles;
  const int32_t split = unit % a.splits, r = unit / a.splits;
  const int32_t q_heads = a.group * a.pool.heads, lb = a.pool.log_block;
  const int32_t held = kv::clip_tokens(a.context[r], a.table.width, lb);
  const int32_t from = split * a.chunk, to = min(held, from + a.chunk);
  const int32_t row = row_tile * kRows + (lane & 15), rows = min(kRows, a.group - row_tile * kRows);
  if (from >= to) {
    if (split == 0) {        // no tokens at all
      for (int32_t i = tid; i < rows * D; i += kThreads)
        a.out[(int64_t)r * a.out_token + (head * a.group + row_tile * kRows + i / D) * a.out_head + i % D] = 0;
      if (a.lse && tid < rows)
        a.lse[(int64_t)r * q_heads + head * a.group + row_tile * kRows + tid] = -__builtin_inff();
    }
    return;
  }

  const int32_t block0 = from >> lb, blocks = ((to - 1) >> lb) - block0 + 1;
  for (int32_t i = tid; i < blocks; i += kThreads) {
    const uint32_t page = kv::page_of(a.table, a.pool, r, block0 + i);
    const int64_t at = (int64_t)page * 2 * a.pool.heads + head;
    const float k = a.pool.scales[at], v = a.pool.scales[at + a.pool.heads];
    s_block[i] = Block{k * a.scale, log2_fast(v), 1.0f / v, page};
  }

  const int32_t grp = lane >> 4, col = lane & 15;
  u4 q[kSteps];
  {
    const int32_t q_head = head * a.group + min(row, a.group - 1);
    const uint16_t* p = (const uint16_t*)a.q.data + (int64_t)r * a.q.token + q_head * a.q.head + grp * (D / 4);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      q[i] = *(const u4*)(p + 8 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) q[i][e] = (q[i][e] ^ a.q_flip) & a.q_mask;
    }
  }
  __syncthreads();

  f4 acc[kParts] = {};
  float top = kNone, sum = 0.0f;

  struct Raw {
    uint32_t k[2][kKeyWords];
    uint32_t v[8][kParts / 4];
  };
  const int64_t half_page = (int64_t)a.pool.heads << lb;      // tokens from a page's keys to its values
  auto token_at = [&](int32_t t) {                            // of the pool's rows of D bytes
    const uint32_t page = s_block[(t >> lb) - block0].page;
    return (((int64_t)page * 2 * a.pool.heads + head) << lb) + (t & ((1 << lb) - 1));
  };
  auto load = [&](int32_t t0, Raw& x) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = a.pool.pages + token_at(min(t0 + 16 * h + col, to - 1)) * D + grp * (D / 4);
#pragma unroll
      for (int i = 0; i < kKeyWords / 4; ++i) {
        const u4 w = *(const u4*)(p + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) x.k[h][4 * i + e] = w[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint8_t* pv = a.pool.pages + (token_at(min(t0 + 16 * h + 4 * grp + e, to - 1)) + half_page) * D + col * kParts;
        if constexpr (kParts == 8) {
          const u2 w = *(const u2*)pv;
          x.v[4 * h + e][0] = w[0];
          x.v[4 * h + e][1] = w[1];
        } else {
          x.v[4 * h + e][0] = *(const uint32_t*)pv;
        }
      }
    }
  };
  auto step = [&](int32_t t0, const Raw& x) {
    f4 s[2];
    float inv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = (f4){};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const u2 lo = widen4<TYPE, FMT>(x.k[h][2 * i]), hi = widen4<TYPE, FMT>(x.k[h][2 * i + 1]);
        s[h] = mul16<TYPE>((u4){lo[0], lo[1], hi[0], hi[1]}, q[i], s[h]);
      }
      const int32_t t = t0 + 16 * h + 4 * grp;
      const Block c = s_block[(min(t, to - 1) >> lb) - block0];
      inv[h] = c.inv_v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = fmaf(s[h][e], c.scale, c.log_v);
        s[h][e] = t + e < to ? y : -__builtin_inff();
      }
    }
    float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                       fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    most = max_halves(swap16_max(most));
    if (__any(most > top + kSlack)) {
      const float next = most > top + kSlack ? most : top;
      const float fall = exp2_fast(top - next);
      top = next;
      sum *= fall;
#pragma unroll
      for (int p = 0; p < kParts; ++p) acc[p] *= fall;
    }
    u4 w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[h][e] = exp2_fast(s[h][e] - top);
      float add = ((s[h][0] + s[h][1]) + (s[h][2] + s[h][3])) * inv[h];
      sum += add;
      w[2 * h] = pack2<TYPE>(s[h][0], s[h][1]);
      w[2 * h + 1] = pack2<TYPE>(s[h][2], s[h][3]);
      if constexpr (MASS) {
        if (a.log_grain >= 3) add = swap16_sum(add);
        if (a.log_grain >= 4) add = sum_halves(add);
        const int32_t t = t0 + 16 * h + 4 * grp;
        if (t < to && (t & ((1 << a.log_grain) - 1)) == 0 && row < a.group)
          a.weights[((int64_t)r * q_heads + head * a.group + row) * a.grains + (t >> a.log_grain)] = log2_fast(add) + top;
      }
    }
#pragma unroll
    for (int p = 0; p < kParts / 4; ++p) {
      uint32_t lo[4], hi[4];
      turn4(x.v[0][p], x.v[1][p], x.v[2][p], x.v[3][p], lo);
      turn4(x.v[4][p], x.v[5][p], x.v[6][p], x.v[7][p], hi);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u2 y = widen4<TYPE, FMT>(lo[e]), z = widen4<TYPE, FMT>(hi[e]);
        acc[4 * p + e] = mul16<TYPE>((u4){y[0], y[1], z[0], z[1]}, w, acc[4 * p + e]);
      }
    }
  };

  {
    Raw x, y;
    int32_t t = from + wave * kTile;
    if (t < to) load(t, x);
    while (t < to) {
      const int32_t next = t + kWaves * kTile;
      if (next < to) load(next, y);
      step(t, x);
      x = y;
      t = next;
    }
  }

  // the wavefronts' results, joined: acc register v of part p is row col, element (4 grp + v) kParts + p
  sum = sum_halves(swap16_sum(sum));
  if (grp == 0) {
    s_top[wave][col] = top;
    s_sum[wave][col] = sum;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int p = 0; p < kParts; ++p) s_out[wave][col][(4 * grp + e) * kParts + p] = acc[p][e];
  __syncthreads();
  const bool whole = held <= a.chunk;       // the only chunk: this is the answer
  for (int32_t i = tid; i < rows * (D / 8); i += kThreads) {
    const int32_t g = i / (D / 8), d = i % (D / 8) * 8, q_head = head * a.group + row_tile * kRows + g;
    float highest = s_top[0][g];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) highest = fmaxf(highest, s_top[w][g]);
    float total = 0.0f, o[8] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float part = exp2_fast(s_top[w][g] - highest);
      total += part * s_sum[w][g];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += part * s_out[w][g][d + e];
    }
    const float over = 1.0f / total, l2 = highest + log2_fast(total);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= over;
    if (whole) {
      *(u4*)(a.out + (int64_t)r * a.out_token + q_head * a.out_head + d) =
          (u4){pack2<TYPE>(o[0], o[1]), pack2<TYPE>(o[2], o[3]), pack2<TYPE>(o[4], o[5]), pack2<TYPE>(o[6], o[7])};
      if (a.lse && d == 0) a.lse[(int64_t)r * q_heads + q_head] = l2 * 0.69314718055994531f;
    } else {
      f4* p = (f4*)(a.part_out + (((int64_t)r * a.splits + split) * q_heads + q_head) * D + d);
      p[0] = (f4){o[0], o[1], o[2], o[3]};
      p[1] = (f4){o[4], o[5], o[6], o[7]};
    }
    if (d == 0 && (MASS || !whole)) a.part_lse[((int64_t)r * a.splits + split) * q_heads + q_head] = l2;
  }
}

// ------------------------------------------------------------------- join
// Workgroups below `outs` join the chunks of 256 / (D / 8) rows each; the
// others turn kept logarithms into the weights of 1024 blocks of a (sequence, kv head).
constexpr int kMassBlocks = 1024;

__device__ __forceinline__ float row_log_sum(const Decode& a, int32_t r, int32_t q_head, int32_t parts, int32_t q_heads) {
  const float* p = a.part_lse + (int64_t)r * a.splits * q_heads + q_head;
  float highest = p[0];
  for (int32_t s = 1; s < parts; ++s) highest = fmaxf(highest, p[(int64_t)s * q_heads]);
  float total = 0.0f;
  for (int32_t s = 0; s < parts; ++s) total += exp2_fast(p[(int64_t)s * q_heads] - highest);
  return highest + log2_fast(total);
}

template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void k_decode_join(Decode a, uint32_t outs) {
  const int32_t tid = threadIdx.x, q_heads = a.group * a.pool.heads, lb = a.pool.log_block;
  if (blockIdx.x < outs) {
    constexpr int kPerGroup = kThreads / (D / 8);
    const int64_t at = (int64_t)blockIdx.x * kPerGroup + tid / (D / 8);
    const int32_t d = tid % (D / 8) * 8;
    if (at >= (int64_t)a.n * q_heads) return;
    const int32_t r = (int32_t)(at / q_heads), q_head = (int32_t)(at % q_heads);
    const int32_t held = kv::clip_tokens(a.context[r], a.table.width, lb), parts = (held + a.chunk - 1) / a.chunk;
    if (parts < 2) return;
    const float l2 = row_log_sum(a, r, q_head, parts, q_heads);
    float o[8] = {};
    for (int32_t s = 0; s < parts; ++s) {
      const int64_t from = ((int64_t)r * a.splits + s) * q_heads + q_head;
      const float part = exp2_fast(a.part_lse[from] - l2);
      const f4 x = *(const f4*)(a.part_out + from * D + d), y = *(const f4*)(a.part_out + from * D + d + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e] = fmaf(part, x[e], o[e]);
        o[4 + e] = fmaf(part, y[e], o[4 + e]);
      }
    }
    *(u4*)(a.out + (int64_t)r * a.out_token + q_head * a.out_head + d) =
        (u4){pack2<TYPE>(o[0], o[1]), pack2<TYPE>(o[2], o[3]), pack2<TYPE>(o[4], o[5]), pack2<TYPE>(o[6], o[7])};
    if (a.lse && d == 0) a.lse[at] = l2 * 0.69314718055994531f;
    return;
  }
  __shared__ float s_lse[kThreads];
  const int32_t width = a.table.width, spans = (width + kMassBlocks - 1) / kMassBlocks;
  const uint32_t unit = blockIdx.x - outs;
  const int32_t span = unit % spans, head = unit / spans % a.pool.heads, r = unit / spans / a.pool.heads;
  const int32_t held = kv::clip_tokens(a.context[r], width, lb), parts = (held + a.chunk - 1) / a.chunk;
  const int32_t live = (held + (1 << lb) - 1) >> lb, sub = 1 << (lb - a.log_grain);
  const int64_t mass_at = ((int64_t)r * a.pool.heads + head) * width;
  constexpr int kEach = kMassBlocks / kThreads;
  float w[kEach] = {};
  for (int32_t g0 = 0; g0 < a.group; g0 += kThreads) {
    __syncthreads();
    if (parts > 0 && g0 + tid < a.group) s_lse[tid] = row_log_sum(a, r, head * a.group + g0 + tid, parts, q_heads);
    __syncthreads();
    for (int i = 0; i < kEach; ++i) {
      const int32_t b = span * kMassBlocks + i * kThreads + tid;
      if (b >= live) continue;
      const int32_t grains = min(sub, (int32_t)(((int64_t)held + (1 << a.log_grain) - 1) >> a.log_grain) - b * sub);
      for (int32_t g = 0; g < min(kThreads, a.group - g0); ++g) {
        const float* p = a.weights + ((int64_t)r * q_heads + head * a.group + g0 + g) * a.grains + (int64_t)b * sub;
        for (int32_t e = 0; e < grains; ++e) w[i] += exp2_fast(p[e] - s_lse[g]);
      }
    }
  }
  for (int i = 0; i < kEach; ++i) {
    const int32_t b = span * kMassBlocks + i * kThreads + tid;
    if (b < width) a.mass[mass_at + b] = (a.mass_in ? a.mass_in[mass_at + b] : 0.0f) + w[i];
  }
}

// -------------------------------------------------------------------- plan
struct Plan {
  int32_t chunk, splits, log_grain;
  int64_t grains;
  size_t part_out, part_lse, weights, bytes;    // offsets into the workspace, and its size
};

// Tokens of a chunk: as many as leave about kGroups workgroups, from 256 on.
constexpr int64_t kGroups = 2048;

Plan plan_for(const peek_kv_pool& pool, int32_t n, int32_t q_heads, int32_t max_blocks, bool with_mass) {
  Plan p{};
  const int32_t row_tiles = (q_heads / pool.kv_heads + kRows - 1) / kRows;
  const int64_t tokens = std::max<int64_t>(1, (int64_t)max_blocks * pool.block_size);
  const int64_t units = std::max<int64_t>(1, (int64_t)n * pool.kv_heads * row_tiles);
  int64_t chunk = 256;
  while (chunk < kMaxChunk && units * ((tokens + chunk - 1) / chunk) > kGroups) chunk *= 2;
  p.chunk = (int32_t)chunk;
  p.splits = (int32_t)((tokens + chunk - 1) / chunk);
  const int32_t lb = __builtin_ctz((unsigned)pool.block_size);
  p.log_grain = std::min(4, lb);
  p.grains = tokens >> p.log_grain;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t rows = (size_t)n * q_heads;
  size_t at = 0;
  p.part_out = at;
  if (p.splits > 1) at = up(at + rows * p.splits * pool.head_dim * sizeof(float));
  p.part_lse = at;
  if (p.splits > 1 || with_mass) at = up(at + rows * p.splits * sizeof(float));
  p.weights = at;
  if (with_mass) at = up(at + rows * (size_t)p.grains * sizeof(float));
  p.bytes = at;
  return p;
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

size_t peek_decode_attention_workspace(const peek_kv_pool* pool, int32_t n, int32_t q_heads, int32_t max_blocks,
                                       int32_t with_mass) {
  Pool p;
  if (n < 0 || q_heads < 1 || max_blocks < 0 || check_pool(pool, &p) != PEEK_OK || q_heads % p.heads != 0) return 0;
  return plan_for(*pool, n, q_heads, max_blocks, with_mass != 0).bytes;
}

peek_status peek_decode_attention(const peek_kv_pool* pool, int32_t n, int32_t type, int32_t q_heads, const void* d_q,
                                  int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_context,
                                  const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, float scale,
                                  void* d_out, int64_t out_token_stride, int64_t out_head_stride, float* d_lse,
                                  const float* d_mass_in, float* d_mass, void* d_workspace, size_t workspace_bytes,
                                  void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Decode a{};
    peek_status s = check_pool(pool, &a.pool);
    if (s != PEEK_OK) return s;
    if (n < 0) return fail(PEEK_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
    s = check_heads(type, q_heads, a.pool.heads, scale);
    if (s != PEEK_OK) return s;
    s = check_table(d_block_table, max_blocks, table_stride, pool->block_size);
    if (s != PEEK_OK) return s;
    if (d_mass_in && !d_mass) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_mass_in needs d_mass");
    if (n == 0) return PEEK_OK;
    if ((s = check_rows("d_q", d_q, q_token_stride, q_head_stride)) != PEEK_OK) return s;
    if ((s = check_rows("d_out", d_out, out_token_stride, out_head_stride)) != PEEK_OK) return s;
    if (!d_context) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_context must not be NULL");
    const Plan p = plan_for(*pool, n, q_heads, max_blocks, d_mass != nullptr);
    s = check_workspace(d_workspace, workspace_bytes, p.bytes);
    if (s != PEEK_OK) return s;
    a.n = n;
    a.group = q_heads / a.pool.heads;
    a.row_tiles = (a.group + kRows - 1) / kRows;
    const int64_t groups = (int64_t)n * a.pool.heads * a.row_tiles * p.splits;
    const int32_t per_group = kThreads / (pool->head_dim / 8);
    const int64_t outs = p.splits > 1 ? ((int64_t)n * q_heads + per_group - 1) / per_group : 0;
    const int64_t masses = d_mass ? (int64_t)n * a.pool.heads * ((max_blocks + kMassBlocks - 1) / kMassBlocks) : 0;
    if (groups >= (1 << 24) || outs + masses >= (1 << 24))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, pool->block_size,
                    pool->num_pages, st);
    if (s != PEEK_OK) return s;
    char* ws = (char*)d_workspace;
    a.q = Rows{d_q, q_token_stride, q_head_stride};
    a.context = d_context;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.out = (uint16_t*)d_out;
    a.out_token = out_token_stride;
    a.out_head = out_head_stride;
    a.lse = d_lse;
    a.mass_in = d_mass_in;
    a.mass = d_mass;
    a.part_out = (float*)(ws + p.part_out);
    a.part_lse = (float*)(ws + p.part_lse);
    a.weights = (float*)(ws + p.weights);
    a.grains = p.grains;
    a.log_grain = p.log_grain;
    a.chunk = p.chunk;
    a.splits = p.splits;
    set_scale(scale, &a.scale, &a.q_flip, &a.q_mask);
    with_types(type, pool->type, pool->head_dim, [&](auto t, auto m, auto d) {
      if (d_mass) {
        hipLaunchKernelGGL((k_decode<t(), m(), d(), true>), dim3((unsigned)groups), dim3(kThreads), 0, st, a);
      } else {
        hipLaunchKernelGGL((k_decode<t(), m(), d(), false>), dim3((unsigned)groups), dim3(kThreads), 0, st, a);
      }
    });
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && outs + masses > 0) {
      with_types(type, PEEK_TYPE_I8, pool->head_dim, [&](auto t, auto, auto d) {
        hipLaunchKernelGGL((k_decode_join<t(), d()>), dim3((unsigned)(outs + masses)), dim3(kThreads), 0, st, a,
                           (uint32_t)outs);
      });
      err = hipGetLastError();
    }
    if (err != hipSuccess) return fail(PEEK_ERR_DEVICE, "decode launch failed: %s", hipGetErrorString(err));
    return PEEK_OK;
  });
}

}  // extern "C"
