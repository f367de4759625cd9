// Which blocks of a long context a query should look at, on gfx950: the largest
// and the smallest key of every block, element by element, and from these the
// blocks that promise the largest logits.
//
// With hi and lo a block's bounds, no key of it has a product with q above
//   sum_d max(q_d hi_d, q_d lo_d) = max(q, 0) . hi + min(q, 0) . lo,
// one product of 2 D elements a (query, block). Bounds are 8-bit whole numbers:
// int8 codes as they are, float8 values in steps of 4 (448 / 4 = 112), rounded outwards; the
// block's scale goes with them. Queries are rounded to 8 bits by a power of two.
// Products and sums are then whole numbers below 2^22, so scores are the same
// in any order of summation, and so is the choice.
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

// ------------------------------------------------------------------ bounds
// A wavefront takes every splits-th block of a sequence for one head. Maxima and
// minima are taken of 16-bit halves, two at a time, and joined over the lanes so that
// every step leaves half of the words (145 us with all words joined over all lanes).
// Bound by memory: 64 sequences of 3200 to 7168 tokens, 369 MB: 86 us, 4.3 TB/s; the
// newest block of 64 sequences 5 us, of one 2.7.

constexpr int64_t kBoundsWaves = 8192;      // wavefronts of a call, where the sequences are fewer

struct Bounds {
  Pool pool;
  const int32_t* first;       // null: from the first token on
  const int32_t* context;
  Table table;
  int8_t* out;                // [num_pages][kv_heads][2][D]
  int32_t n, splits;
};

// float8 codes (sign and magnitude) to bytes in the order of their values, and back.
template <int FMT>
__device__ __forceinline__ uint32_t ordered4(uint32_t w) {
  if constexpr (FMT == PEEK_TYPE_F8E4M3) return w ^ ((w >> 7) & 0x01010101u) * 0x7fu;
  return w;
}

typedef short p2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(p2, a), __builtin_bit_cast(p2, b)));
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(p2, a), __builtin_bit_cast(p2, b)));
}

// An ordered byte's bound: in units of the scale (int8), or of four of it, upwards or downwards.
template <int FMT>
__device__ __forceinline__ int32_t bound_of(uint8_t o, bool up) {
  if constexpr (FMT == PEEK_TYPE_F8E4M3) {
    const uint8_t c = o & 0x80 ? o ^ 0x7f : o;
    if ((c & 0x7f) == 0x7f) return c & 0x80 ? -127 : 127;        // NaN: beyond every number of its sign
    const float x = kv::code_value<FMT>(c) * 0.25f;
    return (int32_t)(up ? ceilf(x) : floorf(x));
  } else {
    return max(-127, (int32_t)(int8_t)o);
  }
}

// What the lane 4, or 8, places round the 16 has.
__device__ __forceinline__ uint32_t round4(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t round8(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true); }

// Two words of every lane to one: joined over the lanes 32 (or 16) apart, the first word in the lower of them and the
// second in the upper.
template <typename F>
__device__ __forceinline__ uint32_t fold32(uint32_t a, uint32_t b, F&& join) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return join((uint32_t)r[0], (uint32_t)r[1]);
}
template <typename F>
__device__ __forceinline__ uint32_t fold16(uint32_t a, uint32_t b, F&& join) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return join((uint32_t)r[0], (uint32_t)r[1]);
}

template <int FMT, int D>
__global__ __launch_bounds__(kThreads) void k_kv_bounds(Bounds a) {
  constexpr int kLanes = D / 16;              // of a token, 16 codes to a lane
  constexpr int kStep = kWave / kLanes;       // tokens a load
  const int lane = threadIdx.x & (kWave - 1);
  uint32_t unit = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t heads = a.pool.heads, lb = a.pool.log_block;
  const int32_t head = unit % heads;
  unit /= heads;
  const int32_t split = unit % a.splits, r = unit / a.splits;
  if (r >= a.n) return;
  const int32_t held = kv::clip_tokens(a.context[r], a.table.width, lb);
  const int32_t first = a.first ? max(0, a.first[r]) : 0;
  const int32_t blocks = (int32_t)(((int64_t)held + (1 << lb) - 1) >> lb);
  const int32_t at = lane % kLanes, sub = lane / kLanes;
  const bool upper32 = lane >= 32, upper16 = lane & 16, upper8 = lane & 8;
  for (int64_t b = (first >> lb) + split; b < blocks; b += a.splits) {
    const uint32_t id = (uint32_t)a.table.ids[(int64_t)r * a.table.stride + b], page = id < a.pool.num_pages ? id : 0u;
    const int32_t tokens = min(1 << lb, held - ((int32_t)b << lb));
    const uint8_t* codes = a.pool.pages + (((int64_t)page * 2 * heads + head) << lb) * D + at * 16;
    const bool turned = a.pool.scales[(int64_t)page * 2 * heads + head] < 0.0f;
    uint32_t hi[8], lo[8];        // of word e bytes 1 and 3, in the upper halves of 16 bits, at 2 e; bytes 0 and 2 after it
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = 0x80008000u;
      lo[e] = 0x7fff7fffu;
    }
    for (int32_t t0 = 0; t0 < tokens; t0 += 2 * kStep) {
      u4 w[2];                    // tokens past the end: the last again
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = *(const u4*)(codes + min(t0 + i * kStep + sub, tokens - 1) * D);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t o = ordered4<FMT>(w[i][e]), odd = o & 0xff00ff00u, even = (o << 8) & 0xff00ff00u;
          hi[2 * e] = max2(hi[2 * e], odd);
          lo[2 * e] = min2(lo[2 * e], odd);
          hi[2 * e + 1] = max2(hi[2 * e + 1], even);
          lo[2 * e + 1] = min2(lo[2 * e + 1], even);
        }
    }
    // Over the lanes of the same codes, half of the words going with each step: a lane ends with one of
    // the eight, of word 2 upper8 + upper16 the bytes 1 and 3 (or 0 and 2, upper32).
    auto over_lanes = [&](const uint32_t* x, auto join) {
      uint32_t y[4], z[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fold32(x[2 * e], x[2 * e + 1], join);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        z[e] = fold16(y[2 * e], y[2 * e + 1], join);
        if constexpr (kLanes == 4) z[e] = join(z[e], round4(z[e]));
      }
      return join(upper8 ? z[1] : z[0], round8(upper8 ? z[0] : z[1]));
    };
    const uint32_t top = over_lanes(hi, [](uint32_t x, uint32_t y) { return max2(x, y); });
    const uint32_t bottom = over_lanes(lo, [](uint32_t x, uint32_t y) { return min2(x, y); });
    int32_t up[2], down[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      up[i] = bound_of<FMT>((uint8_t)(top >> (16 * i + 8)), true);
      down[i] = bound_of<FMT>((uint8_t)(bottom >> (16 * i + 8)), false);
      if (turned) {
        const int32_t x = up[i];
        up[i] = -down[i];
        down[i] = -x;
      }
    }
    auto word = [&](const int32_t* x) {        // bytes 0 and 2, or 1 and 3
      const uint32_t w = (uint32_t)(uint8_t)x[0] | (uint32_t)(uint8_t)x[1] << 16;
      return upper32 ? w : w << 8;
    };
    // the lower lanes write the largest, the upper ones the smallest
    const uint32_t out = fold32(word(up), word(down), [](uint32_t x, uint32_t y) { return x | y; });
    const int32_t e = 2 * upper8 + upper16;
    if (id < a.pool.num_pages)       // (no page, no bounds: page 0 is another block's)
      *(uint32_t*)(a.out + (((int64_t)page * heads + head) * 2 + upper32) * D + at * 16 + e * 4) = out;
  }
}

// ------------------------------------------------------------------ scores
// A wavefront takes 64 blocks at a time of one (sequence, kv head): queries times
// bounds, 16 queries by 16 blocks by 64 elements a matrix instruction. Bound by
// reading the bounds, 2 D bytes a block and head in pages of any order: 64 sequences of up to
// 1500 blocks 30 to 34 us, 3.4 TB/s; 16 of up to 4063 22 us, 5.9 TB/s; one of 1472 6 us.
// With four wavefronts to a SIMD instead of three, and registers for as many, the 64 sequences
// took 1.5 us more, with six 38 more; bounds of the next blocks fetched before these are used: 1 to 8 more.

struct Select {
  Pool pool;
  Rows q;
  const int8_t* bounds;
  const int32_t* context;
  Table table;
  float* scores;              // [n][kv_heads][width]
  int32_t* context_out;       // [n][kv_heads]
  int32_t* table_out;         // [n][kv_heads][keep]
  int32_t n, group, keep, sink, recent;
};

constexpr int kSpan = 64;     // blocks of a wavefront

typedef int32_t i4 __attribute__((ext_vector_type(4)));

constexpr int64_t kScoreWaves = 16384;      // wavefronts of a call, where these have 64 blocks each or more

// Queries as whole numbers: lane l has row row0 + l % 16 (past the last: the last again), elements 16 (l / 16) .. + 15
// of every 64; positive ones in `up`, negative ones in `down`.
template <int TYPE, int D>
struct Query {
  static constexpr int kSteps = D / 64;
  u4 up[kSteps], down[kSteps];
  float of_row[4];            // the units of the rows that this lane's products belong to

  __device__ __forceinline__ void take(const uint16_t* q, int lane) {
    float x[kSteps][16];
    float most = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const u4 w[2] = {*(const u4*)(q + s * 64), *(const u4*)(q + s * 64 + 8)};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t u = w[e >> 3][(e >> 1) & 3];
        x[s][e] = kv::to_float<TYPE>((uint16_t)(u >> (16 * (e & 1))));
        const float m = fabsf(x[s][e]);
        most = fmaxf(most, m < __builtin_inff() ? m : 0.0f);
      }
    }
    most = max_halves(swap16_max(most));
    const int32_t e = __builtin_amdgcn_frexp_expf(most) - 7;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t u = 0, v = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = __builtin_ldexpf(x[s][4 * w + i], -e);
          const int32_t c = y != y ? 0 : (int32_t)__builtin_rintf(fminf(fmaxf(y, -127.0f), 127.0f));
          u |= (uint32_t)(uint8_t)max(c, 0) << (8 * i);
          v |= (uint32_t)(uint8_t)min(c, 0) << (8 * i);
        }
        up[s][w] = u;
        down[s][w] = v;
      }
    const float unit = __builtin_ldexpf(1.0f, e);       // 2^-139 to 2^121
#pragma unroll
    for (int v = 0; v < 4; ++v) of_row[v] = __shfl(unit, 4 * (lane >> 4) + v);
  }
};

template <int TYPE, int FMT, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void k_block_scores(Select a, int32_t waves) {
  constexpr int kSteps = D / 64;
  const int lane = threadIdx.x & (kWave - 1), col = lane & 15, grp = lane >> 4;
  uint32_t unit = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t heads = a.pool.heads, lb = a.pool.log_block;
  const int32_t head = unit % heads;
  unit /= heads;
  const int32_t wave = unit % waves, r = unit / waves;
  if (r >= a.n) return;
  const uint16_t* q = (const uint16_t*)a.q.data + (int64_t)r * a.q.token + grp * 16;
  auto q_row = [&](int32_t row0) { return q + (int64_t)(head * a.group + min(row0 + col, a.group - 1)) * a.q.head; };
  const int32_t held = kv::clip_tokens(a.context[r], a.table.width, lb);
  const int32_t blocks = (int32_t)(((int64_t)held + (1 << lb) - 1) >> lb);
  if (blocks <= a.keep) return;        // (all of them are kept)
  Query<TYPE, D> query;
  int32_t row_at = -1;                 // whose rows `query` has
  auto entry = [&](int64_t b0) { return a.table.ids[(int64_t)r * a.table.stride + min(b0 + lane, (int64_t)blocks - 1)]; };
  uint32_t next = (uint32_t)entry((int64_t)wave * kSpan);
  for (int64_t b0 = (int64_t)wave * kSpan; b0 < blocks; b0 += (int64_t)waves * kSpan) {
    const uint32_t page = next < a.pool.num_pages ? next : 0u;
    next = (uint32_t)entry(b0 + (int64_t)waves * kSpan);
    u4 bounds[4][2 * kSteps];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t p = __shfl(page, 16 * i + col);
      const int8_t* from = a.bounds + ((int64_t)p * heads + head) * 2 * D + grp * 16;
#pragma unroll
      for (int s = 0; s < 2 * kSteps; ++s) bounds[i][s] = *(const u4*)(from + s * 64);
    }
    const float step = fabsf(a.pool.scales[(int64_t)page * 2 * heads + head]) * (FMT == PEEK_TYPE_F8E4M3 ? 4.0f : 1.0f);
    float best[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
    for (int32_t row0 = 0; row0 < a.group; row0 += 16) {
      if (row_at != row0) {
        query.take(q_row(row0), lane);
        row_at = row0;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        i4 dot = {};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, query.up[s]),
                                                      __builtin_bit_cast(i4, bounds[i][s]), dot, 0, 0, 0);
          dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, query.down[s]),
                                                      __builtin_bit_cast(i4, bounds[i][kSteps + s]), dot, 0, 0, 0);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) best[i] = fmaxf(best[i], (float)dot[v] * query.of_row[v]);
      }
    }
    // block 16 i + col of every i, for all rows; lane l keeps that of block l
    float score = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float top = max_halves(swap16_max(best[i]));
      score = grp == i ? top : score;
    }
    if (b0 + lane < blocks)
      a.scores[((int64_t)r * heads + head) * a.table.width + b0 + lane] = score * step;
  }
}

// ------------------------------------------------------------------ choice
// A workgroup takes one (sequence, kv head). The candidates' scores, as whole
// numbers in their order, are counted by digits of 8 bits from the first bit in
// which they differ: after three or four passes the least score to stay and how
// many of that score are known. One barrier a pass: every wavefront sums the
// counts for itself, and clears the other pass's while this one's are made.
//
// Bound by its waits: 9 us for 8 rows of 1472 blocks, 10 us for 512 of up to 1500, 12 us
// for 128 of up to 4063. In one kernel with the scores, which then come at the rate
// of a compute unit: 22 us, 45, 46 where the two take 15, 45, 36.

// NaN above all. (-0, of a product too small for 32 bits, becomes 0 by adding 0 here, where that cannot be made one
// operation with the product, rounded once and -0 again.)
__device__ __forceinline__ uint32_t rank_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return x != x ? 0xffffffffu : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The sum of the lanes up to this one.
__device__ __forceinline__ uint32_t sum_to(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // within 16 lanes: from 1, 2, 4, 8 lanes below
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // lane 15 to the next 16, 47 too
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // lane 31 to the upper 32
  return x;
}

constexpr int kHeld = 8;      // scores of a thread that stay in registers; where there are more, they are read again

template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_block_select(Select a) {
  constexpr int kWaves = THREADS / kWave;
  __shared__ uint32_t s_count[2][kWaves][256];
  __shared__ uint32_t s_more[kWaves], s_equal[kWaves];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t heads = a.pool.heads, lb = a.pool.log_block;
  const int32_t head = blockIdx.x % heads, r = blockIdx.x / heads;
  const int32_t held = kv::clip_tokens(a.context[r], a.table.width, lb);
  const int32_t blocks = (int32_t)(((int64_t)held + (1 << lb) - 1) >> lb);
  const int64_t unit = (int64_t)r * heads + head;
  const int32_t* ids = a.table.ids + (int64_t)r * a.table.stride;
  int32_t* out = a.table_out + unit * a.keep;
  const int32_t kept = min(blocks, a.keep);
  // the last block stays, so only that one can be part full
  if (tid == 0) a.context_out[unit] = held - ((blocks - kept) << lb);
  for (int32_t i = kept + tid; i < a.keep; i += THREADS) out[i] = -1;
  if (blocks <= a.keep) {
    for (int32_t i = tid; i < blocks; i += THREADS) out[i] = ids[i];
    return;
  }
  const float* scores = a.scores + unit * a.table.width;
  const int32_t lo = a.sink, hi = blocks - a.recent;          // candidates (blocks > keep >= sink + recent)
  // A wavefront has blocks in order, 64 after 64; block b is a candidate's rank, or must stay.
  const int32_t share = (int32_t)(((int64_t)blocks + THREADS - 1) / THREADS) * kWave;
  const int32_t from = (int32_t)min((int64_t)wave * share, (int64_t)blocks), to = min(blocks - from, share) + from;
  const bool fits = share <= kHeld * kWave;
  auto read = [&](int32_t b) { return b < to && b >= lo && b < hi ? rank_of(scores[b]) : 0u; };
  uint32_t x[kHeld];
  int32_t entry[kHeld];
  if (fits) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int32_t b = from + i * kWave + lane;
      x[i] = read(b);
      entry[i] = b < to ? ids[b] : 0;
    }
  }
  auto each = [&](auto f) {          // f(block, rank, held entry) of this lane's blocks, up to the end of the share and beyond
    if (fits) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (from + i * kWave < to) f(from + i * kWave + lane, x[i], entry[i]);
    } else {
      for (int32_t b = from; b < to; b += kWave) f(b + lane, read(b + lane), 0);
    }
  };
  uint32_t prefix = 0, left = (uint32_t)(a.keep - a.sink - a.recent);      // so many of the candidates stay
  const bool any = left > 0;
  if (any) {
    // the bits in which candidates differ: scores of one call begin alike
    const uint32_t alike = rank_of(scores[lo]);
    uint32_t differ = 0;
    each([&](int32_t b, uint32_t rank, int32_t) { differ |= b < to && b >= lo && b < hi ? rank ^ alike : 0u; });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) differ |= __shfl_xor(differ, d);
    if (lane == 0) s_more[wave] = differ;
#pragma unroll
    for (int e = 0; e < 4; ++e) s_count[0][wave][4 * lane + e] = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) differ |= s_more[w];
    differ = __builtin_amdgcn_readfirstlane(differ);
    int open = differ != 0 ? 32 - __builtin_clz(differ) : 0;      // low bits of the least rank to stay that are not known
    prefix = open == 32 ? 0u : alike >> open << open;
    for (int pass = 0; open > 0; ++pass) {
      const int shift = max(0, open - 8);
      const uint32_t digits = (1u << (open - shift)) - 1;
      uint32_t(*count)[256] = s_count[pass & 1];
      // (lanes of one digit counted as one, by ballots, took 1.5 to 2.5 us more than these)
      each([&](int32_t b, uint32_t rank, int32_t) {
        if (b < to && b >= lo && b < hi && (pass == 0 || (rank ^ prefix) >> open == 0))
          atomicAdd(&count[wave][(rank >> shift) & digits], 1u);
      });
      __syncthreads();
      // (a wavefront clears its own counts for the next pass: they were last read before this barrier)
#pragma unroll
      for (int e = 0; e < 4; ++e) s_count[(pass + 1) & 1][wave][4 * lane + e] = 0;
      uint32_t c[4] = {}, sum = 0;      // lane l: digits 255 - 4 l .. 252 - 4 l
      for (int w = 0; w < kWaves; ++w) {
        const u4 v = *(const u4*)&count[w][252 - 4 * lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] += v[3 - e];
      }
      sum = c[0] + c[1] + c[2] + c[3];
      uint32_t before = sum_to(sum) - sum;
      uint32_t digit = 0, rest = 0;
      bool here = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (before < left && left <= before + c[e]) {
          digit = 255 - 4 * lane - e;
          rest = left - before;
          here = true;
        }
        before += c[e];
      }
      const int from_lane = __builtin_ctzll(__ballot(here) | 1ull << 63);
      prefix |= (uint32_t)__builtin_amdgcn_readlane(digit, from_lane) << shift;
      left = __builtin_amdgcn_readlane(rest, from_lane);
      open = shift;
    }
    __syncthreads();        // (s_more is written again)
  }
  // counted, then placed
  auto look = [&](int32_t b, uint32_t rank, bool* more, bool* equal) {
    const bool in = b < to, must = b < lo || b >= hi;
    *more = in && (must || (any && rank > prefix));
    *equal = in && !must && any && rank == prefix;
  };
  uint32_t more = 0, equal = 0;
  each([&](int32_t b, uint32_t rank, int32_t) {
    bool m, e;
    look(b, rank, &m, &e);
    more += __popcll(__ballot(m));
    equal += __popcll(__ballot(e));
  });
  if (lane == 0) {
    s_more[wave] = more;
    s_equal[wave] = equal;
  }
  __syncthreads();
  uint32_t place = 0, ties = 0;        // of what comes before: places taken, and equal ones
  for (int w = 0; w < wave; ++w) {
    place += s_more[w];
    ties += s_equal[w];
  }
  place += min(ties, left);
  const uint64_t below = (1ull << lane) - 1;
  each([&](int32_t b, uint32_t rank, int32_t held_entry) {
    bool m, e;
    look(b, rank, &m, &e);
    const uint64_t equals = __ballot(e);
    const bool stays = m || (e && ties + (uint32_t)__popcll(equals & below) < left);
    const uint64_t all = __ballot(stays);
    if (stays) out[place + __popcll(all & below)] = fits ? held_entry : ids[b];
    place += __popcll(all);
    ties += __popcll(equals);
  });
}

int64_t score_bytes(int32_t n, int32_t heads, int32_t width) {
  return ((int64_t)n * heads * width * (int64_t)sizeof(float) + 255) & ~(int64_t)255;
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

peek_status peek_kv_bounds(const peek_kv_pool* pool, int32_t n, const int32_t* d_first, const int32_t* d_context,
                           const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, int8_t* d_bounds,
                           void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Bounds a{};
    peek_status s = check_pool(pool, &a.pool);
    if (s != PEEK_OK) return s;
    if (n < 0) return fail(PEEK_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
    if ((s = check_table(d_block_table, max_blocks, table_stride, pool->block_size)) != PEEK_OK) return s;
    if (n == 0 || max_blocks == 0) return PEEK_OK;
    if (!d_context || !d_bounds) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_context and d_bounds must not be NULL");
    if ((reinterpret_cast<uintptr_t>(d_bounds) & 15) != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_bounds must be 16-byte aligned");
    const int64_t units = (int64_t)n * a.pool.heads;
    a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(max_blocks, kBoundsWaves / units));
    const int64_t groups = (units * a.splits + kWaves - 1) / kWaves;
    if (groups >= (1 << 24)) return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, pool->block_size, &a.pool,
                    st);
    if (s != PEEK_OK) return s;
    a.first = d_first;
    a.context = d_context;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.out = d_bounds;
    a.n = n;
    with_types(PEEK_TYPE_BF16, pool->type, pool->head_dim, [&](auto, auto f, auto d) {
      hipLaunchKernelGGL((k_kv_bounds<f(), d()>), dim3((unsigned)groups), dim3(kThreads), 0, st, a);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "bounds launch failed: %s", hipGetErrorString(e));
    return PEEK_OK;
  });
}

size_t peek_block_select_workspace(const peek_kv_pool* pool, int32_t n, int32_t max_blocks) {
  Pool p;
  if (n < 0 || max_blocks < 0 || check_pool(pool, &p) != PEEK_OK) return 0;
  return (size_t)score_bytes(n, p.heads, max_blocks);
}

peek_status peek_block_select(const peek_kv_pool* pool, const int8_t* d_bounds, int32_t n, int32_t type,
                              int32_t q_heads, const void* d_q, int64_t q_token_stride, int64_t q_head_stride,
                              const int32_t* d_context, const int32_t* d_block_table, int32_t max_blocks,
                              int64_t table_stride, int32_t keep, int32_t sink, int32_t recent, int32_t* d_context_out,
                              int32_t* d_table_out, void* d_workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Select a{};
    peek_status s = check_pool(pool, &a.pool);
    if (s != PEEK_OK) return s;
    if (n < 0) return fail(PEEK_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
    if ((s = check_heads(type, q_heads, a.pool.heads, 1.0f)) != PEEK_OK) return s;
    if ((s = check_table(d_block_table, max_blocks, table_stride, pool->block_size)) != PEEK_OK) return s;
    if (sink < 0 || recent < 1 || keep < 1 || (int64_t)sink + recent > keep)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "sink >= 0, recent >= 1 and sink + recent <= keep (got %d, %d, %d)", sink,
                  recent, keep);
    if ((int64_t)keep * pool->block_size > INT32_MAX)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "keep * block_size must be below 2^31 (got %d * %d)", keep,
                  pool->block_size);
    if (n == 0) return PEEK_OK;
    if ((s = check_rows("d_q", d_q, q_token_stride, q_head_stride)) != PEEK_OK) return s;
    if (!d_bounds || !d_context || !d_context_out || !d_table_out)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_bounds, d_context, d_context_out and d_table_out must not be NULL");
    if ((reinterpret_cast<uintptr_t>(d_bounds) & 15) != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_bounds must be 16-byte aligned");
    s = check_workspace(d_workspace, workspace_bytes, (size_t)score_bytes(n, a.pool.heads, max_blocks));
    if (s != PEEK_OK) return s;
    const int64_t units = (int64_t)n * a.pool.heads;
    const int32_t spans = (max_blocks + kSpan - 1) / kSpan;
    const int32_t waves = (int32_t)std::max<int64_t>(1, std::min<int64_t>(spans, kScoreWaves / units));
    const int64_t groups = (units * waves + kWaves - 1) / kWaves;
    const int threads = max_blocks <= kHeld * 256 ? 256 : max_blocks <= kHeld * 512 ? 512 : 1024;      // of a choice
    if (groups >= (1 << 24) || units * threads >= (int64_t)1 << 32)      // (launches have fewer than 2^32 threads)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, pool->block_size, &a.pool,
                    st);
    if (s != PEEK_OK) return s;
    a.q = Rows{d_q, q_token_stride, q_head_stride};
    a.bounds = d_bounds;
    a.context = d_context;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.scores = (float*)d_workspace;
    a.context_out = d_context_out;
    a.table_out = d_table_out;
    a.n = n;
    a.group = q_heads / a.pool.heads;
    a.keep = keep;
    a.sink = sink;
    a.recent = recent;
    if (max_blocks > keep) {        // (otherwise all blocks are kept)
      with_types(type, pool->type, pool->head_dim, [&](auto t, auto f, auto d) {
        hipLaunchKernelGGL((k_block_scores<t(), f(), d()>), dim3((unsigned)groups), dim3(kThreads), 0, st, a, waves);
      });
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) {
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)units), dim3((unsigned)threads), 0, st, a);
      };
      if (threads == 256) go(k_block_select<256>);
      else if (threads == 512) go(k_block_select<512>);
      else go(k_block_select<1024>);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "selection launch failed: %s", hipGetErrorString(e));
    return PEEK_OK;
  });
}

}  // extern "C"
