// Heads of queries and keys normed and rotated by their tokens' positions, keys
// and values quantised into pages in the same pass, on gfx950.
//
//   y = x / sqrt(mean(x^2) + eps) * w          (of a head, where norms are given)
//   (a, b) -> (a c - b s, b c + a s)           c, s = magnitude * cos, sin(position * freq_i)
//
// on pairs (i, i + rot / 2), or (2i, 2i + 1); the rest of a head past rot passes.
// The angle is a product in 64 bits, taken to a turn's fraction there, so that
// positions of millions keep the precision of small ones; what follows is in 32.
// Rows are rounded to their 16 bits once, and it is those that the pages get:
// a cache holds the same codes whether a row came through here or through
// k_out and an append (the step of the codes is 2^4 times coarser or more).
//
// A lane's unit of work is 16 elements of a head, two 16-byte pieces that hold
// both halves of eight pairs: no lane needs another's elements to turn its own,
// and what it overwrites in place is what it has read. Angles are computed once
// for the heads of a workgroup and shared through LDS.
//
// Bound by memory: 72000 tokens of 32 query and 8 kv heads of 128, half of each head
// turned in pairs, into int8 blocks of 16 and k_out, 1.77 GB: 355 us, 5.0 TB/s (a large copy
// 4.95); 84000 of 64 and 8 heads, normed, 3.07 GB: 680 us, 4.5 TB/s. Rows alone run at 5.1 to 5.5 TB/s;
// blocks alone at 2.9 to 3.3, by their vector instructions (19 an element of a
// plain append before its maximum and quotients were shortened, now 7), beside rows they
// cost what their bytes do. Blocks of 64 tokens 399 us, of 256 444. 64 single tokens 6.5 us.
// Fewer registers for more wavefronts spill: limits of 4 and 5 to a SIMD 425 and 660 us instead of 389.
#include <cmath>

#include "peek_internal.h"
#include "peek_kv.h"
#include "peek_quant.h"
#include "peek_validate.h"

namespace peek {

using kv::Pool;
using kv::Rows;
using kv::Table;
using namespace quant;

namespace {

constexpr int kWave = 64;
constexpr int kWaves = 4;
constexpr int kThreads = kWave * kWaves;
constexpr int kTokens = 16;        // whose angles a workgroup holds at a time
constexpr int kRowTokens = 4;      // of a workgroup over rows, where there are many
constexpr int64_t kManyBlocks = 1024;   // all heads of a block to a workgroup: 4500 blocks 421 us instead of 453; few
                                        // blocks have more workgroups with four heads each

struct OutRows {
  uint16_t* data;
  int64_t token;
  int64_t head;
};

struct Rotate {
  Pool pool;                       // pages: null without a cache
  Rows q, k, v;
  OutRows q_out, k_out;            // k_out: data may be null
  const int64_t* offsets;
  const int32_t* context;
  Table table;
  const double* freq;
  const uint16_t* q_norm;
  const uint16_t* k_norm;
  int64_t num_tokens, slots;
  uint32_t page_groups;            // workgroups of blocks, before those of rows
  int32_t n, q_heads, kv_heads, rot, inter, row_tokens;
  int32_t share;                   // heads of a workgroup of blocks
  float eps, magnitude;
};

// Cosines and sines of a workgroup's tokens, times the magnitude.
struct Turns {
  float c[kTokens][64], s[kTokens][64];
};

// The angle as a fraction of a turn, from a product in 64 bits; its nearest quarter and what is left of it, x, of
// pi / 4 at most, whose sine and cosine are their series up to x^9 and x^10 (what is left out is below 2^-28).
__device__ __forceinline__ void turn(const Rotate& a, int64_t position, int pair, float* c, float* s) {
  constexpr double kTurn = 0.15915494309189533577;        // 1 / (2 pi)
  const double angle = (double)position * a.freq[pair] * kTurn;
  const float part = (float)(angle - __builtin_rint(angle)), quarter = __builtin_rintf(4.0f * part);
  const float x = fmaf(quarter, -0.25f, part) * 6.28318530717958648f, y = x * x;
  float sn = fmaf(y, 1.0f / 362880, -1.0f / 5040);
  sn = fmaf(y, sn, 1.0f / 120);
  sn = fmaf(y, sn, -1.0f / 6);
  sn = fmaf(x * y, sn, x);
  float cs = fmaf(y, -1.0f / 3628800, 1.0f / 40320);
  cs = fmaf(y, cs, -1.0f / 720);
  cs = fmaf(y, cs, 1.0f / 24);
  cs = fmaf(y, cs, -0.5f);
  cs = fmaf(y, cs, 1.0f);
  // cos, sin of x + q pi / 2: q = 0 (c, s), 1 (-s, c), 2 (-c, -s), 3 (s, -c)
  const int q = (int)quarter & 3;
  const float c0 = q & 1 ? sn : cs, s0 = q & 1 ? cs : sn;
  *c = (q == 1 || q == 2 ? -c0 : c0) * a.magnitude;
  *s = (q >= 2 ? -s0 : s0) * a.magnitude;
}

// The two pieces (of eight elements) of a head that are item j of D / 16: both halves of eight pairs, or, where there
// are none of these (interleaved pairs lie in one piece), pieces of either half of the head.
template <int D>
__device__ __forceinline__ void pieces_of(const Rotate& a, int rot, int j, int* p0, int* p1) {
  const bool halves = j < rot / 16;
  if (a.inter || rot == 0) {
    *p0 = j;
    *p1 = j + D / 16;
  } else {
    *p0 = halves ? j : 2 * j;
    *p1 = halves ? j + rot / 16 : 2 * j + 1;
  }
}

template <int TYPE>
__device__ __forceinline__ u4 pack8(const float* x) {
  u4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (uint32_t)kv::from_float<TYPE>(x[2 * i]) | (uint32_t)kv::from_float<TYPE>(x[2 * i + 1]) << 16;
  return w;
}

// An item normed and turned. All lanes of a head (D / 16 adjacent ones) take part; `c` and `s` are its token's.
template <int TYPE, int D>
__device__ __forceinline__ void rotate_item(const Rotate& a, const uint16_t* norm, int rot, int j, int p0, int p1,
                                            const float* c, const float* s, u4* lo, u4* hi) {
  float x[16];
  spread8<TYPE>(*lo, x);
  spread8<TYPE>(*hi, x + 8);
  if (norm != nullptr) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
    for (int d = 1; d < D / 16; d <<= 1) sum += __shfl_xor(sum, d);
    const float by = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
    float w[16];
    spread8<TYPE>(*(const u4*)(norm + 8 * p0), w);
    spread8<TYPE>(*(const u4*)(norm + 8 * p1), w + 8);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = x[e] * by * w[e];
  }
  if (a.inter) {
    // (the pieces of an item are eight or more apart: a part of the head may end between them)
    const bool turns[2] = {p0 < rot / 8, p1 < rot / 8};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!turns[h]) continue;
      const int pair = 4 * (h == 0 ? p0 : p1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = x[8 * h + 2 * e], w = x[8 * h + 2 * e + 1], cs = c[pair + e], sn = s[pair + e];
        x[8 * h + 2 * e] = fmaf(u, cs, -w * sn);
        x[8 * h + 2 * e + 1] = fmaf(w, cs, u * sn);
      }
    }
  } else if (j < rot / 16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = x[e], w = x[e + 8], cs = c[8 * j + e], sn = s[8 * j + e];
      x[e] = fmaf(u, cs, -w * sn);
      x[e + 8] = fmaf(w, cs, u * sn);
    }
  }
  if (norm != nullptr || rot > 0) {       // (what passes is rounded to what it was)
    *lo = pack8<TYPE>(x);
    *hi = pack8<TYPE>(x + 8);
  }
}

// ------------------------------------------------------------------- rows
// Rows of q, and of k where there is no cache: TOKENS tokens' heads a workgroup, four where there are
// thousands of them (one search for their sequence each, and four times the angles to a barrier), else one.
// A thread has four items on their way at a time, the first of them before the
// positions are known (of rows that are in no sequence they are not stored).
constexpr int kBatch = 4;

template <int TYPE, int D, int TOKENS>
__device__ __forceinline__ void rotate_rows(const Rotate& a, uint32_t group, Turns& turns, int64_t* s_at) {
  constexpr int kItems = D / 16;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int64_t t0 = (int64_t)group * TOKENS;
  const int32_t heads = a.q_heads + (a.pool.pages == nullptr && a.k_out.data != nullptr ? a.kv_heads : 0);
  const uint32_t each = (uint32_t)heads * kItems, all = each * (uint32_t)min((int64_t)TOKENS, a.num_tokens - t0);
  u4 lo[kBatch], hi[kBatch];
  // an item's token, head and place in it
  auto item = [&](uint32_t u, int* i, int32_t* h, int* j) {
    *i = 0;
#pragma unroll
    for (int t = 1; t < TOKENS; ++t) *i += u >= t * each;
    const uint32_t rest = u - *i * each;
    *h = rest / kItems;
    *j = rest % kItems;
  };
  auto load = [&](uint32_t u0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t u = u0 + b * kThreads;
      if (u >= all) continue;
      int i, j, p0, p1;
      int32_t h;
      item(u, &i, &h, &j);
      pieces_of<D>(a, a.rot, j, &p0, &p1);
      const bool is_q = h < a.q_heads;
      const Rows& from = is_q ? a.q : a.k;
      const uint16_t* x = (const uint16_t*)from.data + (t0 + i) * from.token + (is_q ? h : h - a.q_heads) * from.head;
      lo[b] = *(const u4*)(x + 8 * p0);
      hi[b] = *(const u4*)(x + 8 * p1);
    }
  };
  load(tid);
  for (int32_t i = wave; i < TOKENS; i += kWaves) {
    const int64_t t = t0 + i;
    int64_t position = -1;
    if (t < a.num_tokens) {
      const int32_t r = kv::last_at_most(a.n, t, lane, [&](int32_t s) { return a.offsets[s]; });
      const int64_t first = a.offsets[r];
      if (first <= t && t < a.offsets[r + 1]) position = (int64_t)max(0, a.context[r]) + (t - first);
    }
    if (lane == 0) s_at[i] = position;
    if (position >= 0 && lane < a.rot / 2) turn(a, position, lane, &turns.c[i][lane], &turns.s[i][lane]);
  }
  __syncthreads();
  for (uint32_t u0 = tid; u0 < all; u0 += kBatch * kThreads) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t u = u0 + b * kThreads;
      if (u >= all) continue;
      int i, j, p0, p1;
      int32_t h;
      item(u, &i, &h, &j);
      if (s_at[i] < 0) continue;
      pieces_of<D>(a, a.rot, j, &p0, &p1);
      const bool is_q = h < a.q_heads;
      const OutRows& to = is_q ? a.q_out : a.k_out;
      rotate_item<TYPE, D>(a, is_q ? a.q_norm : a.k_norm, a.rot, j, p0, p1, turns.c[i], turns.s[i], &lo[b], &hi[b]);
      uint16_t* y = to.data + (t0 + i) * to.token + (is_q ? h : h - a.q_heads) * to.head;
      *(u4*)(y + 8 * p0) = lo[b];
      *(u4*)(y + 8 * p1) = hi[b];
    }
    load(u0 + kBatch * kThreads);
  }
}

// ------------------------------------------------------------------ blocks
// A workgroup takes K or V of one block, a wavefront to every fourth head of its
// share of them (all, where there are blocks enough: their angles are computed
// once); blocks are found as an append finds them. HELD chunks of 16 tokens stay in
// registers from the maximum to the rounding; those of larger blocks are taken again.
template <int TYPE, int FMT, int D, int HELD>
__device__ __forceinline__ void rotate_block(const Rotate& a, uint32_t group, Turns& turns) {
  constexpr int kItems = D / 16;
  constexpr int kEach = kTokens * kItems / kWave;        // items of a chunk and lane: 2 (D = 128) or 1
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t shares = (a.pool.heads + a.share - 1) / a.share;
  const int64_t slot = group / (2 * shares);
  const int32_t part = group % (2 * shares), is_v = part / shares;
  const int32_t head0 = part % shares * a.share, heads = min(a.share, a.pool.heads - head0);
  const int32_t lb = a.pool.log_block;
  const int32_t r = kv::last_at_most(a.n, slot, lane, [&](int32_t i) { return (a.offsets[i] >> lb) + 2 * (int64_t)i; });
  const int64_t start = a.offsets[r], first = max((int64_t)0, start), end = min(a.num_tokens, a.offsets[r + 1]);
  const int64_t ctx = max(0, a.context[r]);
  const int64_t b = (ctx >> lb) + slot - ((start >> lb) + 2 * (int64_t)r);
  const int64_t from = max(ctx, b << lb), to = min(ctx + (end - first), (b + 1) << lb);
  if (b < 0 || from >= to) return;
  bool stored = b < a.table.width;
  uint32_t page = 0;
  if (stored) {
    page = (uint32_t)a.table.ids[(int64_t)r * a.table.stride + b];
    stored = page < a.pool.num_pages;
  }
  uint16_t* const k_out = is_v ? nullptr : a.k_out.data;
  if (!stored && k_out == nullptr) return;
  const int32_t old = (int32_t)(from - (b << lb)), tokens = (int32_t)(to - from);
  const int32_t rot = is_v ? 0 : a.rot;
  const uint16_t* const norm = is_v ? nullptr : a.k_norm;

  const Rows src = is_v ? a.v : a.k;
  const int64_t row0 = first + from - ctx;
  for (int32_t of = 0; of < heads; of += kWaves) {
    const int32_t head = head0 + of + wave;
    const bool active = of + wave < heads;        // (the others stay for the barriers)
    const uint16_t* x = (const uint16_t*)src.data + row0 * src.token + head * src.head;
    uint16_t* y = k_out != nullptr ? k_out + row0 * a.k_out.token + head * a.k_out.head : nullptr;
    const int64_t at = ((int64_t)page * 2 + is_v) * a.pool.heads + head;
    uint8_t* codes = a.pool.pages + (at << lb) * D;
    const float held = active && stored && old > 0 ? a.pool.scales[at] : 0.0f;

    u4 w[HELD][kEach][2];
    // chunk c's rows as they go into the cache; `again`: those in k_out are ready. The rows are on their way while
    // the angles are computed.
    auto load = [&](int32_t c, u4 (*z)[2], bool again) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int32_t u = i * kWave + lane, t = c * kTokens + u / kItems, j = u % kItems;
        z[i][0] = z[i][1] = (u4){};
        if (!active || t >= tokens) continue;
        int p0, p1;
        pieces_of<D>(a, rot, j, &p0, &p1);
        const uint16_t* p = again ? y + t * a.k_out.token : x + t * src.token;
        z[i][0] = *(const u4*)(p + 8 * p0);
        z[i][1] = *(const u4*)(p + 8 * p1);
      }
      if (again) return;
      if (rot > 0 && (of == 0 || tokens > kTokens)) {      // (else they are there)
        __syncthreads();
        const int32_t pairs = rot / 2;
        for (int32_t i = tid; i < kTokens * pairs; i += kThreads) {
          const int32_t t = i / pairs, p = i - t * pairs;
          if (c * kTokens + t < tokens) turn(a, from + c * kTokens + t, p, &turns.c[t][p], &turns.s[t][p]);
        }
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int32_t u = i * kWave + lane, t = c * kTokens + u / kItems, j = u % kItems;
        if (!active || t >= tokens) continue;
        int p0, p1;
        pieces_of<D>(a, rot, j, &p0, &p1);
        rotate_item<TYPE, D>(a, norm, rot, j, p0, p1, turns.c[u / kItems], turns.s[u / kItems], &z[i][0], &z[i][1]);
        if (y != nullptr) {
          *(u4*)(y + t * a.k_out.token + 8 * p0) = z[i][0];
          *(u4*)(y + t * a.k_out.token + 8 * p1) = z[i][1];
        }
      }
    };
    const int32_t chunks = (tokens + kTokens - 1) / kTokens;
    const bool kept = chunks <= HELD;
    uint32_t bits = 0;
    float most = 0.0f;                // finite magnitudes of chunks that are not held
#pragma unroll
    for (int c = 0; c < HELD; ++c) {
      if (c < chunks) {
        load(c, w[c], false);
#pragma unroll
        for (int i = 0; i < 2 * kEach; ++i) bits = largest8(w[c][i / 2][i % 2], bits);
      }
    }
    for (int32_t c = HELD; c < chunks; ++c) {
      u4 z[kEach][2];
      load(c, z, false);
#pragma unroll
      for (int i = 0; i < 2 * kEach; ++i) {
        bits = largest8(z[i / 2][i % 2], bits);
        most = finite8<TYPE>(z[i / 2][i % 2], most);
      }
    }
    if (!stored) continue;
    bits = wave_largest(bits);
    bool plain = bits < kInfinity<TYPE>;
    if (plain) {
      most = kv::to_float<TYPE>((uint16_t)bits);
    } else {
#pragma unroll
      for (int c = 0; c < HELD; ++c) {
        if (c < chunks) {
#pragma unroll
          for (int i = 0; i < 2 * kEach; ++i) most = finite8<TYPE>(w[c][i / 2][i % 2], most);
        }
      }
      most = wave_max(most);
    }
    float scale = scale_of<FMT>(most);
    plain = plain && scale < kv::kScaleMax;
    if (old > 0 && !(scale > held)) {
      scale = held;
      plain = plain && plain_scale<FMT>(held);
    }
    const float inv = 1.0f / scale;
    if (active && old > 0 && scale > held) rescale<FMT>(codes, old * D, held, scale, inv, lane);
    auto store = [&](int32_t c, const u4 (*z)[2]) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int32_t u = i * kWave + lane, t = c * kTokens + u / kItems, j = u % kItems;
        if (!active || t >= tokens) continue;
        int p[2];
        pieces_of<D>(a, rot, j, &p[0], &p[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float f[8];
          spread8<TYPE>(z[i][h], f);
          *(u2*)(codes + (old + t) * D + p[h] * 8) =
              (u2){codes_of<FMT>(f, scale, inv, plain), codes_of<FMT>(f + 4, scale, inv, plain)};
        }
      }
    };
    if (kept) {
#pragma unroll
      for (int c = 0; c < HELD; ++c)
        if (c < chunks) store(c, w[c]);
    } else {
      for (int32_t c = 0; c < chunks; ++c) {
        u4 z[kEach][2];
        load(c, z, y != nullptr);
        store(c, z);
      }
    }
    if (active && lane == 0) a.pool.scales[at] = scale;
  }
}

template <int TYPE, int FMT, int D, int HELD>
__global__ __launch_bounds__(kThreads) void k_rotate_append(Rotate a) {
  __shared__ Turns s_turns;
  __shared__ int64_t s_at[kTokens];
  if (blockIdx.x < a.page_groups) rotate_block<TYPE, FMT, D, HELD>(a, blockIdx.x, s_turns);
  else if (a.row_tokens == 1) rotate_rows<TYPE, D, 1>(a, blockIdx.x - a.page_groups, s_turns, s_at);
  else rotate_rows<TYPE, D, kRowTokens>(a, blockIdx.x - a.page_groups, s_turns, s_at);
}

// -------------------------------------------------------------------- read
// A wavefront takes the tokens of one (block, K or V, head), found as an append
// finds them. Bound by memory: 64 sequences of 3200 to 7168 tokens, 2 GB: 394 us, 5.0 TB/s;
// one of 5117: 9 us, its waits and 31 MB.
template <int TYPE, int FMT, int D>
__global__ __launch_bounds__(kThreads) void k_kv_read(Pool pool, OutRows k, OutRows v, int32_t n, int64_t num_tokens,
                                                      const int64_t* __restrict__ offsets,
                                                      const int32_t* __restrict__ begin, Table table, int64_t slots) {
  constexpr int kItems = D / 16;        // of 16 codes
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t parts = 2 * pool.heads, lb = pool.log_block;
  const int64_t slot = unit / parts;
  if (slot >= slots) return;
  const int32_t part = (int32_t)(unit % parts), is_v = part / pool.heads, head = part % pool.heads;
  const int32_t r = kv::last_at_most(n, slot, lane, [&](int32_t i) { return (offsets[i] >> lb) + 2 * (int64_t)i; });
  const int64_t start = offsets[r], first = max((int64_t)0, start), end = min(num_tokens, offsets[r + 1]);
  const int64_t ctx = max(0, begin[r]);
  const int64_t b = (ctx >> lb) + slot - ((start >> lb) + 2 * (int64_t)r);
  const int64_t from = max(ctx, b << lb), to = min(ctx + (end - first), (b + 1) << lb);
  if (b < 0 || b >= table.width || from >= to) return;
  const uint32_t page = kv::page_of(table, pool, r, (int32_t)b);
  const int64_t at = ((int64_t)page * 2 + is_v) * pool.heads + head;
  const float scale = pool.scales[at];
  const uint8_t* codes = pool.pages + ((at << lb) + (from - (b << lb))) * D;
  const OutRows out = is_v ? v : k;
  uint16_t* y = out.data + (first + from - ctx) * out.token + head * out.head;
  const int32_t items = (int32_t)(to - from) * kItems;
  for (int32_t i = lane; i < items; i += kWave) {
    const u4 w = *(const u4*)(codes + i * 16);
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t word = w[e >> 2];
      x[e] = kv::code_value<FMT>((uint8_t)(word >> (8 * (e & 3)))) * scale;
    }
    uint16_t* to_row = y + (int64_t)(i / kItems) * out.token + i % kItems * 16;
    *(u4*)to_row = pack8<TYPE>(x);
    *(u4*)(to_row + 8) = pack8<TYPE>(x + 8);
  }
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

peek_status peek_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double trained,
                                    double low, double high, double* out) {
  return guarded([&]() -> peek_status {
    clear_error();
    if (rot_dim < 2 || rot_dim > 128 || rot_dim % 2 != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "rot_dim must be even, in [2, 128] (got %d)", rot_dim);
    if (!(base > 0) || !std::isfinite(base)) return fail(PEEK_ERR_INVALID_ARGUMENT, "base must be above 0 and finite");
    if (scaling < PEEK_ROTARY_PLAIN || scaling > PEEK_ROTARY_RAMP)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "scaling must be one of peek_rotary_scaling (got %d)", scaling);
    if (!out) return fail(PEEK_ERR_INVALID_ARGUMENT, "out must not be NULL");
    if (scaling != PEEK_ROTARY_PLAIN && (!(factor > 0) || !std::isfinite(factor)))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "factor must be above 0 and finite");
    if (scaling == PEEK_ROTARY_BASE && rot_dim < 4)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "PEEK_ROTARY_BASE needs a rot_dim of 4 at least (got %d)", rot_dim);
    const bool blends = scaling == PEEK_ROTARY_TURNS || scaling == PEEK_ROTARY_RAMP;
    if (blends && (!(trained > 0) || !std::isfinite(trained) || !(low > 0) || !(high > low) || !std::isfinite(high)))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "trained must be above 0 and finite, and 0 < low < high");
    if (scaling == PEEK_ROTARY_RAMP && base == 1.0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "PEEK_ROTARY_RAMP needs a base other than 1");
    if (scaling == PEEK_ROTARY_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    constexpr double kTwoPi = 6.283185307179586476925;
    // the pair, as a real number, that makes so many turns over the trained length
    auto pair_of = [&](double turns) { return rot_dim * std::log(trained / (turns * kTwoPi)) / (2 * std::log(base)); };
    for (int32_t i = 0; i < rot_dim / 2; ++i) {
      const double f = std::pow(base, -2.0 * i / rot_dim);
      double keep = 1.0;                               // the share of f that stays as it is
      if (scaling == PEEK_ROTARY_LINEAR) {
        keep = 0.0;
      } else if (scaling == PEEK_ROTARY_TURNS) {
        keep = (trained * f / kTwoPi - low) / (high - low);
      } else if (scaling == PEEK_ROTARY_RAMP) {
        const double a = std::fmax(std::floor(pair_of(high)), 0.0);
        const double b = std::fmin(std::ceil(pair_of(low)), rot_dim - 1.0);
        keep = 1.0 - (i - a) / std::fmax(b - a, 0.001);
      }
      keep = std::fmin(std::fmax(keep, 0.0), 1.0);
      out[i] = scaling == PEEK_ROTARY_BASE ? f : f * keep + f / (scaling == PEEK_ROTARY_PLAIN ? 1.0 : factor) * (1.0 - keep);
    }
    return PEEK_OK;
  });
}

peek_status peek_rotate_append(const peek_kv_pool* pool, int32_t n, int64_t num_tokens, int32_t type, int32_t q_heads,
                               int32_t kv_heads, int32_t head_dim, const peek_rotary* rotary, const void* d_q,
                               int64_t q_token_stride, int64_t q_head_stride, const void* d_k, int64_t k_token_stride,
                               int64_t k_head_stride, const void* d_v, int64_t v_token_stride, int64_t v_head_stride,
                               const int64_t* d_offsets, const int32_t* d_context, const int32_t* d_block_table,
                               int32_t max_blocks, int64_t table_stride, void* d_q_out, int64_t q_out_token_stride,
                               int64_t q_out_head_stride, void* d_k_out, int64_t k_out_token_stride,
                               int64_t k_out_head_stride, void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    if (n < 0 || num_tokens < 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "n and num_tokens must be >= 0 (got %d, %lld)", n, (long long)num_tokens);
    if (type != PEEK_TYPE_BF16 && type != PEEK_TYPE_F16)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "type must be PEEK_TYPE_BF16 or PEEK_TYPE_F16 (got %d)", type);
    if (kv_heads < 1 || kv_heads > 1024)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "kv_heads must be in [1, 1024] (got %d)", kv_heads);
    if (q_heads < 0 || q_heads > 65536)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "q_heads must be in [0, 65536] (got %d)", q_heads);
    if (head_dim != 64 && head_dim != 128)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "head_dim must be 64 or 128 (got %d)", head_dim);
    if (!rotary) return fail(PEEK_ERR_INVALID_ARGUMENT, "rotary is NULL");
    if (rotary->rot_dim < 0 || rotary->rot_dim > head_dim || rotary->rot_dim % 16 != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "rot_dim must be a multiple of 16 in [0, head_dim] (got %d)",
                  rotary->rot_dim);
    if (rotary->rot_dim > 0 && !rotary->d_freq) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_freq must not be NULL");
    if ((reinterpret_cast<uintptr_t>(rotary->d_freq) & 7) != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_freq must be 8-byte aligned");
    if (!std::isfinite(rotary->magnitude)) return fail(PEEK_ERR_INVALID_ARGUMENT, "magnitude must be finite");
    if (!(rotary->eps >= 0) || !std::isfinite(rotary->eps))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "eps must be 0 or more and finite");
    if (((reinterpret_cast<uintptr_t>(rotary->d_q_norm) | reinterpret_cast<uintptr_t>(rotary->d_k_norm)) & 15) != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_q_norm and d_k_norm must be 16-byte aligned");
    Rotate a{};
    peek_status s;
    if (pool) {
      if ((s = check_pool(pool, &a.pool)) != PEEK_OK) return s;
      if (pool->kv_heads != kv_heads || pool->head_dim != head_dim)
        return fail(PEEK_ERR_INVALID_ARGUMENT, "the pool has %d heads of %d, the rows %d of %d", pool->kv_heads,
                    pool->head_dim, kv_heads, head_dim);
      if ((s = check_table(d_block_table, max_blocks, table_stride, pool->block_size)) != PEEK_OK) return s;
    } else if (d_v || d_block_table) {
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_v and d_block_table need a pool");
    }
    if (!pool && !d_k_out && d_k) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_k needs a pool or d_k_out");
    if (n == 0 || num_tokens == 0) return PEEK_OK;
    if (q_heads > 0) {
      if ((s = check_rows("d_q", d_q, q_token_stride, q_head_stride)) != PEEK_OK) return s;
      s = check_out_rows("d_q_out", d_q_out, q_out_token_stride, q_out_head_stride, num_tokens, q_heads, head_dim);
      if (s != PEEK_OK) return s;
    }
    if (pool || d_k_out) {
      if ((s = check_rows("d_k", d_k, k_token_stride, k_head_stride)) != PEEK_OK) return s;
    }
    if (pool) {
      if ((s = check_rows("d_v", d_v, v_token_stride, v_head_stride)) != PEEK_OK) return s;
    }
    if (d_k_out) {
      s = check_out_rows("d_k_out", d_k_out, k_out_token_stride, k_out_head_stride, num_tokens, kv_heads, head_dim);
      if (s != PEEK_OK) return s;
    }
    if (!d_offsets || !d_context)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_offsets and d_context must not be NULL");
    a.slots = pool ? (num_tokens >> a.pool.log_block) + 2 * (int64_t)n : 0;
    a.share = a.slots >= kManyBlocks ? kv_heads : kWaves;
    const int64_t pages = a.slots * 2 * ((kv_heads + a.share - 1) / a.share);
    const int32_t row_heads = q_heads + (!pool && d_k_out ? kv_heads : 0);
    a.row_tokens = num_tokens >= 4096 ? kRowTokens : 1;
    const int64_t rows = row_heads > 0 ? (num_tokens + a.row_tokens - 1) / a.row_tokens : 0;
    if (pages + rows >= (1 << 24))        // (a launch has fewer than 2^32 threads)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many tokens for one call (%lld)", (long long)num_tokens);
    if (pages + rows == 0) return PEEK_OK;
    hipStream_t st = (hipStream_t)stream;
    // (without a cache there is no table to check lengths against)
    s = validate_kv(n, d_offsets, num_tokens, pool ? d_context : nullptr, true, d_block_table, max_blocks, table_stride,
                    pool ? pool->block_size : 4, pool ? &a.pool : nullptr, st);
    if (s != PEEK_OK) return s;
    a.q = Rows{d_q, q_token_stride, q_head_stride};
    a.k = Rows{d_k, k_token_stride, k_head_stride};
    a.v = Rows{d_v, v_token_stride, v_head_stride};
    a.q_out = OutRows{(uint16_t*)d_q_out, q_out_token_stride, q_out_head_stride};
    a.k_out = OutRows{(uint16_t*)d_k_out, k_out_token_stride, k_out_head_stride};
    a.offsets = d_offsets;
    a.context = d_context;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.freq = rotary->d_freq;
    a.q_norm = (const uint16_t*)rotary->d_q_norm;
    a.k_norm = (const uint16_t*)rotary->d_k_norm;
    a.num_tokens = num_tokens;
    a.page_groups = (uint32_t)pages;
    a.n = n;
    a.q_heads = q_heads;
    a.kv_heads = kv_heads;
    a.rot = rotary->rot_dim;
    a.inter = rotary->interleaved != 0;
    a.eps = rotary->eps;
    a.magnitude = rotary->magnitude;
    with_types(type, pool ? pool->type : PEEK_TYPE_F8E4M3, head_dim, [&](auto e, auto f, auto d) {
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(pages + rows)), dim3(kThreads), 0, st, a);
      };
      const int32_t block = pool ? pool->block_size : 4;
      if (block <= kTokens) go(k_rotate_append<e(), f(), d(), 1>);
      else if (block <= 2 * kTokens) go(k_rotate_append<e(), f(), d(), 2>);
      else go(k_rotate_append<e(), f(), d(), 4>);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "rotation launch failed: %s", hipGetErrorString(e));
    return PEEK_OK;
  });
}

peek_status peek_kv_read(const peek_kv_pool* pool, int32_t n, int64_t num_tokens, int32_t type,
                         const int64_t* d_offsets, const int32_t* d_first, const int32_t* d_block_table,
                         int32_t max_blocks, int64_t table_stride, void* d_k_out, int64_t k_token_stride,
                         int64_t k_head_stride, void* d_v_out, int64_t v_token_stride, int64_t v_head_stride,
                         void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Pool p;
    peek_status s = check_pool(pool, &p);
    if (s != PEEK_OK) return s;
    if (n < 0 || num_tokens < 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "n and num_tokens must be >= 0 (got %d, %lld)", n, (long long)num_tokens);
    if (type != PEEK_TYPE_BF16 && type != PEEK_TYPE_F16)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "type must be PEEK_TYPE_BF16 or PEEK_TYPE_F16 (got %d)", type);
    if ((s = check_table(d_block_table, max_blocks, table_stride, pool->block_size)) != PEEK_OK) return s;
    if (n == 0 || num_tokens == 0) return PEEK_OK;
    s = check_out_rows("d_k_out", d_k_out, k_token_stride, k_head_stride, num_tokens, p.heads, pool->head_dim);
    if (s != PEEK_OK) return s;
    s = check_out_rows("d_v_out", d_v_out, v_token_stride, v_head_stride, num_tokens, p.heads, pool->head_dim);
    if (s != PEEK_OK) return s;
    if (!d_offsets || !d_first)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_offsets and d_first must not be NULL");
    const int64_t slots = (num_tokens >> p.log_block) + 2 * (int64_t)n;
    const int64_t groups = (slots * 2 * p.heads + kWaves - 1) / kWaves;
    if (groups >= (1 << 24))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many tokens for one call (%lld)", (long long)num_tokens);
    hipStream_t st = (hipStream_t)stream;
    // (as of an append: the pages that these tokens reach; scales may be any)
    Pool any = p;
    any.scales = nullptr;
    s = validate_kv(n, d_offsets, num_tokens, d_first, true, d_block_table, max_blocks, table_stride, pool->block_size,
                    &any, st);
    if (s != PEEK_OK) return s;
    const OutRows k{(uint16_t*)d_k_out, k_token_stride, k_head_stride};
    const OutRows v{(uint16_t*)d_v_out, v_token_stride, v_head_stride};
    with_types(type, pool->type, pool->head_dim, [&](auto e, auto f, auto d) {
      hipLaunchKernelGGL((k_kv_read<e(), f(), d()>), dim3((unsigned)groups), dim3(kThreads), 0, st, p, k, v, n,
                         num_tokens, d_offsets, d_first, Table{d_block_table, table_stride, max_blocks}, slots);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "read launch failed: %s", hipGetErrorString(e));
    return PEEK_OK;
  });
}

}  // extern "C"
