// Attention of single tokens over the paged 8-bit cache, on gfx950.
//
// Bound by reading the pages once: a kv head's keys and values serve the
// group's query heads together, as 16 rows of the matrix products. A
// workgroup of four wavefronts takes one chunk of one sequence's tokens for one
// kv head and 16 of its rows; a wavefront takes every fourth tile of 32
// tokens, on its own, with a running reference and sum. Long sequences are split
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
// They take 4 bytes a row and 16 tokens, of the 4 KB that the tokens take.
//
// Measured: 192 sequences of 2000 to 24000 tokens, 8 kv heads of 128, int8, 5.5 GB:
// 0.95 to 0.99 ms, 5.6 to 5.8 TB/s (a streaming read of memory reaches 6.3);
// 64 sequences of up to 7400 tokens with weights, 0.56 GB: 115 us and 9 for the
// second kernel; one of 5117 tokens: 5.4 us and 4.2, its page ids', scales' and
// pages' waits one after the other.
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
constexpr int kMaxChunk = 4096;                  // tokens of a workgroup, at most

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
  float* part_out;       // [n][q_heads][splits][D]: a chunk's sum of weight * value / its sum of weights
  float* part_lse;       // [n][q_heads][splits]: base-2 logarithm of its sum of weights
  float* weights;        // [n][kv_heads][row_tiles][grains][16]: base-2 logarithm of the weight on a grain of tokens
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

// Chunks of a sequence (lengths up to 2^31 - 1).
__device__ __forceinline__ int32_t parts_of(int32_t tokens, int32_t chunk) {
  return tokens > 0 ? (tokens - 1) / chunk + 1 : 0;
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

// WIDE: blocks of 16 tokens or more. Sixteen tokens that start at a multiple
// of 16 then lie in one block, whose page and scales are the same for the whole
// wavefront and come by scalar loads; smaller blocks are looked up by every
// lane in LDS. (Blocks of 16 looked up in LDS: 64 sequences of 4000 tokens 112 us
// where these take 106, one of 130000 24.0 where these take 21.7.)
template <int TYPE, int FMT, int D, bool MASS, bool WIDE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(WIDE ? 4 : 3))) void k_decode(Decode a) {
  constexpr int kSteps = D / 32;        // products of keys and queries a 16-token half
  constexpr int kParts = D / 16;        // 16-wide parts of the output; also bytes of a token's values in a lane
  constexpr int kKeyWords = D / 16;     // words of a token's key in a lane
  __shared__ Block s_block[WIDE ? 1 : kMaxChunk / 4 + 1];           // of the chunk's blocks
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
  const int32_t from = split * a.chunk, to = from + min(a.chunk, held - from);   // (no sum passes `held`, nor 2^31)
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

  const int32_t block0 = from >> lb;
  if constexpr (!WIDE) {
    const int32_t blocks = ((to - 1) >> lb) - block0 + 1;
    for (int32_t i = tid; i < blocks; i += kThreads) {
      const uint32_t page = kv::page_of(a.table, a.pool, r, block0 + i);
      const int64_t at = (int64_t)page * 2 * a.pool.heads + head;
      const float k = a.pool.scales[at], v = kv::value_scale(a.pool.scales[at + a.pool.heads]);
      s_block[i] = Block{k * a.scale, log2_fast(v), __builtin_amdgcn_rcpf(v), page};
    }
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
  if constexpr (!WIDE) __syncthreads();

  f4 acc[kParts] = {};
  float top = kNone, peak = kNone, sum = 0.0f;
  uint32_t kw[2][kKeyWords];        // keys, and values, of the tile at hand, then of the next
  uint32_t vw[8][kParts / 4];
  float scale[2], log_v[2], inv_v[2];
  const int64_t half_page = ((int64_t)a.pool.heads << lb) * D;      // bytes from a page's keys to its values

  // Where the 16 tokens from t on (WIDE), or this lane's token t, begin.
  typedef const __attribute__((address_space(4))) int32_t* const_ints;
  typedef const __attribute__((address_space(4))) float* const_floats;
  const const_ints ids = (const_ints)(a.table.ids + (int64_t)r * a.table.stride);
  const const_floats scales = (const_floats)a.pool.scales;
  const uint8_t* base[2];           // WIDE: of the next tile's halves
  int32_t limit[2];                 // and the last of their 16 tokens that there is
  auto place = [&](int32_t t0) {    // pages and scales of the tile at t0 (its halves past the end: of the last tokens)
    if constexpr (WIDE) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int32_t t = min(t0 + 16 * h, (to - 1) & ~15);
        const uint32_t id = (uint32_t)ids[t >> lb], page = id < a.pool.num_pages ? id : 0u;
        const int64_t at = (int64_t)page * 2 * a.pool.heads + head;
        base[h] = a.pool.pages + ((at << lb) + (t & ((1 << lb) - 1))) * D;
        limit[h] = to - 1 - t;
        const float v = kv::value_scale(scales[at + a.pool.heads]);
        scale[h] = scales[at] * a.scale;
        log_v[h] = log2_fast(v);
        inv_v[h] = __builtin_amdgcn_rcpf(v);
      }
    }
  };
  auto row_at = [&](int32_t t) {    // !WIDE: this lane's token
    const uint32_t page = s_block[(t >> lb) - block0].page;
    return a.pool.pages + ((((int64_t)page * 2 * a.pool.heads + head) << lb) + (t & ((1 << lb) - 1))) * D;
  };
  auto load_keys = [&](int32_t t0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p;
      if constexpr (WIDE) p = base[h] + (uint32_t)(min(col, limit[h]) * D + grp * (D / 4));
      else p = row_at(min(t0 + 16 * h + col, to - 1)) + grp * (D / 4);
#pragma unroll
      for (int i = 0; i < kKeyWords / 4; ++i) {
        const u4 w = *(const u4*)(p + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) kw[h][4 * i + e] = w[e];
      }
    }
  };
  auto load_values = [&](int32_t t0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t t = min(t0 + 16 * h + 4 * grp, (to - 1) & ~3);      // !WIDE: four tokens of one block
      const uint8_t* p = WIDE ? base[h] : row_at(t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int32_t at = WIDE ? min(4 * grp + e, limit[h]) : min(e, to - 1 - t);
        const uint8_t* pv = p + half_page + (uint32_t)(at * D + col * kParts);
        if constexpr (kParts == 8) {
          const u2 w = *(const u2*)pv;
          vw[4 * h + e][0] = w[0];
          vw[4 * h + e][1] = w[1];
        } else {
          vw[4 * h + e][0] = *(const uint32_t*)pv;
        }
      }
    }
  };
  // One tile; the next one's keys are fetched as soon as this one's are used, then its values.
  auto step = [&](int32_t t0) {
    const bool more = to - t0 > kWaves * kTile;
    const int32_t next = more ? t0 + kWaves * kTile : 0;
    f4 s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = (f4){};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const u2 lo = widen4<TYPE, FMT>(kw[h][2 * i]), hi = widen4<TYPE, FMT>(kw[h][2 * i + 1]);
        s[h] = mul16<TYPE>((u4){lo[0], lo[1], hi[0], hi[1]}, q[i], s[h]);
      }
      if constexpr (!WIDE) {
        const Block c = s_block[(min(t0 + 16 * h + 4 * grp, to - 1) >> lb) - block0];
        scale[h] = c.scale;
        log_v[h] = c.log_v;
        inv_v[h] = c.inv_v;
      }
    }
    const float inv[2] = {inv_v[0], inv_v[1]};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[h][e] = fmaf(s[h][e], scale[h], log_v[h]);
    if (more) {
      place(next);
      load_keys(next);
    }
    if (to - t0 < kTile) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[h][e] = t0 + 16 * h + 4 * grp + e < to ? s[h][e] : -__builtin_inff();
    }
    float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                       fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    most = max_halves(swap16_max(most));
    if (__any(moves<TYPE>(most, top))) {
      const float by = move_top<TYPE>(most, top, peak);
      sum *= by;
#pragma unroll
      for (int p = 0; p < kParts; ++p) acc[p] *= by;
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
        if (WIDE || a.log_grain >= 3) add = swap16_sum(add);
        if (WIDE || a.log_grain >= 4) add = sum_halves(add);
        const int32_t t = t0 + 16 * h + 4 * grp;
        if (t < to && (t & ((1 << a.log_grain) - 1)) == 0)
          a.weights[((((int64_t)r * a.pool.heads + head) * a.row_tiles + row_tile) * a.grains + (t >> a.log_grain)) * kRows +
                    col] = log2_sum(top, add);
      }
    }
#pragma unroll
    for (int p = 0; p < kParts / 4; ++p) {
      uint32_t lo[4], hi[4];
      turn4(vw[0][p], vw[1][p], vw[2][p], vw[3][p], lo);
      turn4(vw[4][p], vw[5][p], vw[6][p], vw[7][p], hi);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u2 y = widen4<TYPE, FMT>(lo[e]), z = widen4<TYPE, FMT>(hi[e]);
        acc[4 * p + e] = mul16<TYPE>((u4){y[0], y[1], z[0], z[1]}, w, acc[4 * p + e]);
      }
    }
    if (more) load_values(next);
  };

  {
    const int32_t mine = to - from - wave * kTile;      // tokens from this wavefront's first one on
    if (mine > 0) {
      place(to - mine);
      load_keys(to - mine);
      load_values(to - mine);
    }
    for (int32_t left = mine; left > 0; left -= kWaves * kTile) step(to - left);
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
    const float over = 1.0f / total, l2 = log2_sum(highest, total);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= over;
    if (whole) {
      *(u4*)(a.out + (int64_t)r * a.out_token + q_head * a.out_head + d) =
          (u4){pack2<TYPE>(o[0], o[1]), pack2<TYPE>(o[2], o[3]), pack2<TYPE>(o[4], o[5]), pack2<TYPE>(o[6], o[7])};
      if (a.lse && d == 0) a.lse[(int64_t)r * q_heads + q_head] = l2 * 0.69314718055994531f;
    } else {
      f4* p = (f4*)(a.part_out + (((int64_t)r * q_heads + q_head) * a.splits + split) * D + d);
      p[0] = (f4){o[0], o[1], o[2], o[3]};
      p[1] = (f4){o[4], o[5], o[6], o[7]};
    }
    if (d == 0 && (MASS || !whole)) a.part_lse[((int64_t)r * q_heads + q_head) * a.splits + split] = l2;
  }
}

// ------------------------------------------------------------------- join
// Workgroups below `outs` join the chunks of rows, WAVES wavefronts to a row
// (THREADS / 64 to all of them); the others turn kept logarithms into the weights
// of THREADS blocks of a (sequence, kv head). Bound by its waits: 4.2 us for one
// sequence's 40 rows of 20 parts, 11 us for 192 sequences of 64 rows. A row of kManyParts
// parts or more has 16 wavefronts: 390 parts of 96 rows 127 us for both kernels
// instead of 140, 508 of 8 rows 22 instead of 46; of few parts they cost more
// than they save (64 sequences of 8 parts 119 us instead of 106).

template <int TYPE, int D, int THREADS, int WAVES>
__global__ __launch_bounds__(THREADS) void k_decode_join(Decode a, uint32_t outs) {
  constexpr int kWaves = THREADS / kWave;
  __shared__ float s_sum[WAVES > 1 ? WAVES * D : 1];
  const int32_t tid = threadIdx.x, q_heads = a.group * a.pool.heads, lb = a.pool.log_block;
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  if (blockIdx.x < outs) {
    const int64_t at = (int64_t)blockIdx.x * (kWaves / WAVES) + wave / WAVES;
    if (at >= (int64_t)a.n * q_heads) return;
    const int32_t r = (int32_t)(at / q_heads), q_head = (int32_t)(at % q_heads);
    const int32_t held = kv::clip_tokens(a.context[r], a.table.width, lb), parts = parts_of(held, a.chunk);
    if (parts < 2) return;
    float l2;
    join_parts<TYPE, D, WAVES>(a.part_out + at * a.splits * D, a.part_lse + at * a.splits, parts, wave % WAVES, lane,
                               s_sum, a.out + (int64_t)r * a.out_token + q_head * a.out_head, &l2);
    if (a.lse && lane == 0 && wave % WAVES == 0) a.lse[at] = l2 * 0.69314718055994531f;
    return;
  }
  __shared__ float s_lse[kRows];
  const int32_t width = a.table.width, spans = (width + THREADS - 1) / THREADS;
  const uint32_t unit = blockIdx.x - outs;
  const int32_t span = unit % spans, head = unit / spans % a.pool.heads, r = unit / spans / a.pool.heads;
  const int32_t held = kv::clip_tokens(a.context[r], width, lb), parts = parts_of(held, a.chunk);
  const int32_t sub = 1 << (lb - a.log_grain), b = span * THREADS + tid;
  const int64_t mass_at = ((int64_t)r * a.pool.heads + head) * width + b;
  const int32_t grains = min(sub, (int32_t)(((int64_t)held + (1 << a.log_grain) - 1) >> a.log_grain) - b * sub);
  float w = 0.0f;
  if (span * THREADS * (int64_t)sub << a.log_grain < held) {
    for (int32_t tile = 0; tile < a.row_tiles; ++tile) {
      const int32_t rows = min(kRows, a.group - tile * kRows);
      __syncthreads();
      for (int32_t g = wave; g < rows; g += kWaves) {
        const float l2 =
            row_log_sum(a.part_lse + ((int64_t)r * q_heads + head * a.group + tile * kRows + g) * a.splits, parts, lane);
        if (lane == 0) s_lse[g] = l2;
      }
      __syncthreads();
      const float* p = a.weights +
          ((((int64_t)r * a.pool.heads + head) * a.row_tiles + tile) * a.grains + (int64_t)b * sub) * kRows;
      for (int32_t e = 0; e < grains; ++e)
        for (int32_t g = 0; g < rows; ++g) w += exp2_fast(p[e * kRows + g] - s_lse[g]);
    }
  }
  if (b < width) a.mass[mass_at] = (a.mass_in ? a.mass_in[mass_at] : 0.0f) + w;
}

// -------------------------------------------------------------------- plan
struct Plan {
  int32_t chunk, splits, log_grain;
  int64_t grains;
  size_t part_out, part_lse, weights, bytes;    // offsets into the workspace, and its size
};

// Tokens of a chunk: as many as leave about kGroups workgroups, from 256 on up to
// kMaxChunk. Fewer workgroups leave compute units idle at the end where lengths differ
// (64 sequences of 1100 to 7400 tokens with weights: 8192 124 us, 4096 135, 2048
// 152), more have more parts to join (three sequences of 100000: 16384 137 us, 8192
// 127, 4096 123). Chunks of 1024 at most cost the largest batches 7% (192 sequences of up
// to 24000 tokens 1.06 ms instead of 0.99).
constexpr int64_t kGroups = 8192;
constexpr int32_t kManyParts = 32;

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
  if (with_mass) at = up(at + (size_t)n * pool.kv_heads * row_tiles * (size_t)p.grains * kRows * sizeof(float));
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
    s = check_out_rows("d_out", d_out, out_token_stride, out_head_stride, n, q_heads, pool->head_dim);
    if (s != PEEK_OK) return s;
    if (!d_context) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_context must not be NULL");
    const Plan p = plan_for(*pool, n, q_heads, max_blocks, d_mass != nullptr);
    s = check_workspace(d_workspace, workspace_bytes, p.bytes);
    if (s != PEEK_OK) return s;
    a.n = n;
    a.group = q_heads / a.pool.heads;
    a.row_tiles = (a.group + kRows - 1) / kRows;
    const int64_t groups = (int64_t)n * a.pool.heads * a.row_tiles * p.splits;
    const bool many = p.splits >= kManyParts;
    const int32_t threads = many ? 1024 : kThreads, rows = many ? 1 : kWaves;      // of a joining workgroup
    const int64_t outs = p.splits > 1 ? ((int64_t)n * q_heads + rows - 1) / rows : 0;
    const int64_t masses = d_mass ? (int64_t)n * a.pool.heads * ((max_blocks + threads - 1) / threads) : 0;
    if (groups >= (1 << 24) || outs + masses >= (1 << 24))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, pool->block_size,
                    &a.pool, st);
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
      auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kThreads), 0, st, a); };
      if (a.pool.log_block >= 4) {
        d_mass ? go(k_decode<t(), m(), d(), true, true>) : go(k_decode<t(), m(), d(), false, true>);
      } else {
        d_mass ? go(k_decode<t(), m(), d(), true, false>) : go(k_decode<t(), m(), d(), false, false>);
      }
    });
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && outs + masses > 0) {
      with_types(type, PEEK_TYPE_I8, pool->head_dim, [&](auto t, auto, auto d) {
        auto go = [&](auto kernel) {
          hipLaunchKernelGGL(kernel, dim3((unsigned)(outs + masses)), dim3(threads), 0, st, a, (uint32_t)outs);
        };
        many ? go(k_decode_join<t(), d(), 1024, 16>) : go(k_decode_join<t(), d(), kThreads, 1>);
      });
      err = hipGetLastError();
    }
    if (err != hipSuccess) return fail(PEEK_ERR_DEVICE, "decode launch failed: %s", hipGetErrorString(err));
    return PEEK_OK;
  });
}

}  // extern "C"
