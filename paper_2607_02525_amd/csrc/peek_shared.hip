// Attention of single tokens where groups of sequences share their first pages,
// on gfx950.
//
// A row (one query head of one sequence) is a softmax over two spans of keys:
// the group's, whose pages are those of its first member, and its own. Each
// span is split into chunks, every chunk leaves a row with sum of weight * value / sum
// of weights and the logarithm of that sum, and a last kernel joins a row's
// parts in a fixed order.
//
// Over a group's span the rows of all members stand side by side, (member,
// query head of the kv head) in that order, in tiles of 16 ROWS; over its own a
// sequence has a tile to itself. A workgroup of four wavefronts takes one chunk of
// keys for one such tile; a wavefront takes every fourth 32 keys of it, alone.
// Keys and values are loaded, widened to 16 bits and turned round in
// registers as in the decode of single sequences, once for all ROWS tiles of
// 16, which then take only their products and exponentials.
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
constexpr int kTile = 32;             // keys of a wavefront's step
constexpr int kMaxChunk = 4096;       // keys of a workgroup, at most

struct Shared {
  Pool pool;
  Rows q;
  const int32_t* context;
  Table table;
  const int32_t* members;             // null: 0, 1, ...
  const int32_t* group_offsets;
  const int32_t* shared;
  uint16_t* out;
  int64_t out_token, out_head;
  float* lse;
  float* part_out;                    // [n][q_heads][splits][D], n in the order of members
  float* part_lse;                    // [n][q_heads][splits]
  int32_t n, groups, group;           // `group`: query heads to a kv head
  int32_t prefix_chunk, own_chunk, splits;
  float scale;
  uint32_t q_flip, q_mask;
};

__device__ __forceinline__ int32_t parts_of(int32_t tokens, int32_t chunk) {
  return tokens > 0 ? (tokens - 1) / chunk + 1 : 0;
}

// The sequence at a position of the members, or -1.
__device__ __forceinline__ int32_t member_at(const Shared& a, int32_t position) {
  const int32_t r = a.members ? a.members[position] : position;
  return (uint32_t)r < (uint32_t)a.n ? r : -1;
}

__device__ __forceinline__ int32_t held_by(const Shared& a, int32_t r) {
  return kv::clip_tokens(a.context[r], a.table.width, a.pool.log_block);
}

// Group g: its positions, its first member and the tokens that it shares.
struct Group {
  int32_t lo, hi, leader, tokens;
};
__device__ __forceinline__ Group group_at(const Shared& a, int32_t g) {
  Group x;
  x.lo = min(max(a.group_offsets[g], 0), a.n);
  x.hi = min(max(a.group_offsets[g + 1], x.lo), a.n);
  x.leader = x.lo < x.hi ? member_at(a, x.lo) : -1;
  const int32_t lb = a.pool.log_block;
  x.tokens = x.leader < 0 ? 0 : kv::clip_tokens(a.shared[g], a.table.width, lb) >> lb << lb;
  return x;
}

// What a sequence of `held` tokens shares of its group's: all of it, or nothing.
__device__ __forceinline__ int32_t shares(const Group& g, int32_t held) { return held >= g.tokens ? g.tokens : 0; }

// The group of a position: nothing shared where there is none.
__device__ __forceinline__ Group group_of(const Shared& a, int32_t position, int lane) {
  Group none{0, 0, -1, 0};
  if (a.groups == 0) return none;
  const int32_t g = kv::last_at_most(a.groups, position, lane, [&](int32_t i) { return (int64_t)a.group_offsets[i]; });
  const Group x = group_at(a, g);
  return x.lo <= position && position < x.hi ? x : none;
}

struct alignas(16) Block {
  float scale, log_v, inv_v;
  uint32_t page;
};

// PREFIX: a tile of rows of a group over a chunk of what it shares; else rows
// of one sequence over a chunk of its own. WIDE: blocks of 16 tokens or more, whose
// page and scales come by scalar loads; smaller ones are looked up in LDS.
template <int TYPE, int FMT, int D, int ROWS, bool PREFIX, bool WIDE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(ROWS == 1 ? (WIDE ? 4 : 3) : ROWS == 2 ? 2 : 1)))
void k_shared(Shared a, int32_t tiles) {
  constexpr int kSteps = D / 32;        // products of keys and queries a 16-token half
  constexpr int kParts = D / 16;        // 16-wide parts of the output; also bytes of a token's values in a lane
  constexpr int kKeyWords = D / 16;     // words of a token's key in a lane
  __shared__ Block s_block[WIDE ? 1 : kMaxChunk / 4 + 1];
  __shared__ float s_out[kWaves][16][D + 4];
  __shared__ float s_top[kWaves][16], s_sum[kWaves][16];
  __shared__ int64_t s_row[16 * ROWS];       // position * q_heads + query head, -1 for none

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t q_heads = a.group * a.pool.heads, lb = a.pool.log_block;
  uint32_t unit = blockIdx.x;
  const int32_t head = unit % a.pool.heads;
  unit /= a.pool.heads;
  const int32_t tile = unit % tiles, split = unit / tiles;

  // the span: `from` to `to` of the sequence `owner`, which is part `part` of each row
  int32_t owner, from, to, part;
  int32_t position = 0, row0, rows;          // the tile's rows: row0 .. of `rows` from `position` on
  bool whole = false;
  Group g;
  if constexpr (PREFIX) {
    const int32_t each = 16 * ROWS;
    const int32_t at = kv::last_at_most(a.groups, tile, lane, [&](int32_t i) {
      return (int64_t)min(max(a.group_offsets[i], 0), a.n) * a.group / each + i;
    });
    g = group_at(a, at);
    const int64_t first = (int64_t)g.lo * a.group / each + at;
    const int64_t row = ((int64_t)tile - first) * each, all = (int64_t)(g.hi - g.lo) * a.group;
    if (row < 0 || row >= all) return;
    position = g.lo;
    row0 = (int32_t)row;
    rows = (int32_t)all;
    owner = g.leader;
    from = split * a.prefix_chunk;
    if (from >= g.tokens) return;
    to = from + min(a.prefix_chunk, g.tokens - from);
    part = split;
  } else {
    const int32_t row_tiles = (a.group + 15) / 16;
    position = tile / row_tiles;
    row0 = tile % row_tiles * 16;
    rows = a.group;
    owner = member_at(a, position);
    if (owner < 0) return;
    g = group_of(a, position, lane);
    const int32_t held = held_by(a, owner), begin = shares(g, held);
    if (held == 0) {
      if (split == 0) {
        const int32_t here = min(16, rows - row0);
        for (int32_t i = tid; i < here * D; i += kThreads)
          a.out[(int64_t)owner * a.out_token + (head * a.group + row0 + i / D) * a.out_head + i % D] = 0;
        if (a.lse && tid < here)
          a.lse[(int64_t)owner * q_heads + head * a.group + row0 + tid] = -__builtin_inff();
      }
      return;
    }
    if ((int64_t)split * a.own_chunk >= held - begin) return;
    from = begin + split * a.own_chunk;
    to = from + min(a.own_chunk, held - from);
    part = parts_of(begin, a.prefix_chunk) + split;
    whole = begin == 0 && held <= a.own_chunk;
  }

  const int32_t block0 = from >> lb;
  const int32_t* const row_ids = a.table.ids + owner * a.table.stride;
  if constexpr (!WIDE) {
    const int32_t blocks = ((to - 1) >> lb) - block0 + 1;
    for (int32_t i = tid; i < blocks; i += kThreads) {
      const uint32_t id = (uint32_t)row_ids[block0 + i], page = id < a.pool.num_pages ? id : 0u;
      const int64_t at = (int64_t)page * 2 * a.pool.heads + head;
      const float k = a.pool.scales[at], v = kv::value_scale(a.pool.scales[at + a.pool.heads]);
      s_block[i] = Block{k * a.scale, log2_fast(v), __builtin_amdgcn_rcpf(v), page};
    }
  }
  const int32_t grp = lane >> 4, col = lane & 15;
  u4 q[ROWS][kSteps];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    // rows that share nothing, or that there are not, are computed as another's and not stored
    const int32_t row = min(row0 + 16 * i + col, rows - 1), of = PREFIX ? row / a.group : 0;
    const int32_t q_head = head * a.group + row - of * a.group, at = position + of;
    const int32_t r = PREFIX ? member_at(a, at) : owner;
    bool live = row0 + 16 * i + col < rows && r >= 0;
    if (PREFIX && live) live = held_by(a, r) >= g.tokens;
    if (grp == 0 && wave == 0) s_row[16 * i + col] = live ? (int64_t)at * q_heads + q_head : -1;
    const uint16_t* p =
        (const uint16_t*)a.q.data + (int64_t)(r >= 0 ? r : owner) * a.q.token + q_head * a.q.head + grp * (D / 4);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      q[i][s] = *(const u4*)(p + 8 * s);
#pragma unroll
      for (int e = 0; e < 4; ++e) q[i][s][e] = (q[i][s][e] ^ a.q_flip) & a.q_mask;
    }
  }
  __syncthreads();

  f4 acc[ROWS][kParts] = {};
  float top[ROWS], peak[ROWS], sum[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    top[i] = peak[i] = kNone;
    sum[i] = 0.0f;
  }
  uint32_t kw[2][kKeyWords];        // keys, and values, of the tile at hand, then of the next
  uint32_t vw[8][kParts / 4];
  float scale[2], log_v[2], inv_v[2];
  const int64_t half_page = ((int64_t)a.pool.heads << lb) * D;      // bytes from a page's keys to its values

  typedef const __attribute__((address_space(4))) int32_t* const_ints;
  typedef const __attribute__((address_space(4))) float* const_floats;
  const const_ints ids = (const_ints)row_ids;
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
    f4 s[ROWS][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) s[i][h] = (f4){};
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const u2 lo = widen4<TYPE, FMT>(kw[h][2 * k]), hi = widen4<TYPE, FMT>(kw[h][2 * k + 1]);
        const u4 key = (u4){lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) s[i][h] = mul16<TYPE>(key, q[i][k], s[i][h]);
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
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][h][e] = fmaf(s[i][h][e], scale[h], log_v[h]);
    if (more) {
      place(next);
      load_keys(next);
    }
    if (to - t0 < kTile) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[i][h][e] = t0 + 16 * h + 4 * grp + e < to ? s[i][h][e] : -__builtin_inff();
    }
    u4 w[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      float most = fmaxf(fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3])),
                         fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3])));
      most = max_halves(swap16_max(most));
      if (__any(moves<TYPE>(most, top[i]))) {
        const float by = move_top<TYPE>(most, top[i], peak[i]);
        sum[i] *= by;
#pragma unroll
        for (int p = 0; p < kParts; ++p) acc[i][p] *= by;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][h][e] = exp2_fast(s[i][h][e] - top[i]);
        sum[i] += ((s[i][h][0] + s[i][h][1]) + (s[i][h][2] + s[i][h][3])) * inv[h];
        w[i][2 * h] = pack2<TYPE>(s[i][h][0], s[i][h][1]);
        w[i][2 * h + 1] = pack2<TYPE>(s[i][h][2], s[i][h][3]);
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
        const u4 value = (u4){y[0], y[1], z[0], z[1]};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) acc[i][4 * p + e] = mul16<TYPE>(value, w[i], acc[i][4 * p + e]);
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
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const float total_here = sum_halves(swap16_sum(sum[i]));
    if (i > 0) __syncthreads();
    if (grp == 0) {
      s_top[wave][col] = top[i];
      s_sum[wave][col] = total_here;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int p = 0; p < kParts; ++p) s_out[wave][col][(4 * grp + e) * kParts + p] = acc[i][p][e];
    __syncthreads();
    for (int32_t u = tid; u < 16 * (D / 8); u += kThreads) {
      const int32_t c = u / (D / 8), d = u % (D / 8) * 8;
      const int64_t row = s_row[16 * i + c];
      if (row < 0) continue;
      float highest = s_top[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) highest = fmaxf(highest, s_top[w][c]);
      float total = 0.0f, o[8] = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float by = exp2_fast(s_top[w][c] - highest);
        total += by * s_sum[w][c];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += by * s_out[w][c][d + e];
      }
      const float over = 1.0f / total, l2 = log2_sum(highest, total);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= over;
      if (whole) {
        const int32_t q_head = head * a.group + row0 + c;
        *(u4*)(a.out + (int64_t)owner * a.out_token + q_head * a.out_head + d) =
            (u4){pack2<TYPE>(o[0], o[1]), pack2<TYPE>(o[2], o[3]), pack2<TYPE>(o[4], o[5]), pack2<TYPE>(o[6], o[7])};
        if (a.lse && d == 0) a.lse[(int64_t)owner * q_heads + q_head] = l2 * 0.69314718055994531f;
      } else {
        f4* p = (f4*)(a.part_out + (row * a.splits + part) * D + d);
        p[0] = (f4){o[0], o[1], o[2], o[3]};
        p[1] = (f4){o[4], o[5], o[6], o[7]};
        if (d == 0) a.part_lse[row * a.splits + part] = l2;
      }
    }
  }
}

// ------------------------------------------------------------------- join
// A wavefront (WAVES of them) to a row.
template <int TYPE, int D, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : kWave * WAVES) void k_shared_join(Shared a) {
  constexpr int kRowsHere = WAVES == 1 ? kWaves : 1;
  __shared__ float s_sum[WAVES > 1 ? WAVES * D : 1];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t q_heads = a.group * a.pool.heads;
  const int64_t row = (int64_t)blockIdx.x * kRowsHere + wave / WAVES;
  if (row >= (int64_t)a.n * q_heads) return;
  const int32_t position = (int32_t)(row / q_heads), q_head = (int32_t)(row % q_heads), r = member_at(a, position);
  if (r < 0) return;
  const int32_t held = held_by(a, r);
  if (held == 0) return;
  const Group g = group_of(a, position, lane);
  const int32_t begin = shares(g, held);
  if (begin == 0 && held <= a.own_chunk) return;       // the answer is there
  const int32_t parts = parts_of(begin, a.prefix_chunk) + parts_of(held - begin, a.own_chunk);
  float l2;
  join_parts<TYPE, D, WAVES>(a.part_out + row * a.splits * D, a.part_lse + row * a.splits, parts, wave % WAVES, lane,
                             s_sum, a.out + (int64_t)r * a.out_token + q_head * a.out_head, &l2);
  if (a.lse && lane == 0 && wave % WAVES == 0) a.lse[(int64_t)r * q_heads + q_head] = l2 * 0.69314718055994531f;
}

// -------------------------------------------------------------------- plan
struct Plan {
  int32_t rows;                       // tiles of 16 rows a workgroup, over what a group shares
  int32_t prefix_chunk, own_chunk;
  int32_t prefix_splits, own_splits;
  int64_t tiles;                      // of rows, over what groups share: room for them
  size_t part_lse, bytes;
};

constexpr int64_t kPrefixGroups = 2048, kOwnGroups = 8192;
constexpr int32_t kManyParts = 32;

Plan plan_for(const peek_kv_pool& pool, int32_t n, int32_t q_heads, int32_t max_blocks, int32_t groups) {
  Plan p{};
  const int32_t group = q_heads / pool.kv_heads;
  const int64_t tokens = std::max<int64_t>(1, (int64_t)max_blocks * pool.block_size);
  const int64_t each = groups > 0 ? (int64_t)n * group / groups : 0;        // rows of a group and kv head
  p.rows = each > 32 ? 4 : each > 16 ? 2 : 1;
  p.tiles = groups > 0 ? (int64_t)n * group / (16 * p.rows) + groups : 0;
  auto chunk_for = [&](int64_t units, int64_t most) {
    int64_t chunk = 256;
    while (chunk < kMaxChunk && units * ((tokens + chunk - 1) / chunk) > most) chunk *= 2;
    return (int32_t)chunk;
  };
  p.prefix_chunk = chunk_for(std::max<int64_t>(1, p.tiles * pool.kv_heads), kPrefixGroups);
  p.own_chunk = chunk_for((int64_t)n * pool.kv_heads * ((group + 15) / 16), kOwnGroups);
  p.prefix_splits = groups > 0 ? (int32_t)((tokens + p.prefix_chunk - 1) / p.prefix_chunk) : 0;
  p.own_splits = (int32_t)((tokens + p.own_chunk - 1) / p.own_chunk);
  const size_t rows = (size_t)n * q_heads, splits = (size_t)p.prefix_splits + p.own_splits;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.part_lse = up(rows * splits * pool.head_dim * sizeof(float));
  p.bytes = p.part_lse + up(rows * splits * sizeof(float));
  return p;
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

size_t peek_shared_decode_attention_workspace(const peek_kv_pool* pool, int32_t n, int32_t q_heads, int32_t max_blocks,
                                              int32_t groups) {
  Pool p;
  if (n < 0 || groups < 0 || q_heads < 1 || max_blocks < 0 || check_pool(pool, &p) != PEEK_OK || q_heads % p.heads != 0)
    return 0;
  return plan_for(*pool, n, q_heads, max_blocks, groups).bytes;
}

peek_status peek_shared_decode_attention(const peek_kv_pool* pool, int32_t n, int32_t type, int32_t q_heads,
                                         const void* d_q, int64_t q_token_stride, int64_t q_head_stride,
                                         const int32_t* d_context, const int32_t* d_block_table, int32_t max_blocks,
                                         int64_t table_stride, int32_t groups, const int32_t* d_members,
                                         const int32_t* d_group_offsets, const int32_t* d_shared, float scale,
                                         void* d_out, int64_t out_token_stride, int64_t out_head_stride, float* d_lse,
                                         void* d_workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    Shared a{};
    peek_status s = check_pool(pool, &a.pool);
    if (s != PEEK_OK) return s;
    if (n < 0 || groups < 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "n and groups must be >= 0 (got %d, %d)", n, groups);
    if ((s = check_heads(type, q_heads, a.pool.heads, scale)) != PEEK_OK) return s;
    if ((s = check_table(d_block_table, max_blocks, table_stride, pool->block_size)) != PEEK_OK) return s;
    if (n == 0) return PEEK_OK;
    if ((s = check_rows("d_q", d_q, q_token_stride, q_head_stride)) != PEEK_OK) return s;
    s = check_out_rows("d_out", d_out, out_token_stride, out_head_stride, n, q_heads, pool->head_dim);
    if (s != PEEK_OK) return s;
    if (!d_context) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_context must not be NULL");
    if (groups > 0 && (!d_group_offsets || !d_shared))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_group_offsets and d_shared must not be NULL");
    const Plan p = plan_for(*pool, n, q_heads, max_blocks, groups);
    if ((s = check_workspace(d_workspace, workspace_bytes, p.bytes)) != PEEK_OK) return s;
    a.n = n;
    a.groups = groups;
    a.group = q_heads / a.pool.heads;
    const int64_t own_tiles = (int64_t)n * ((a.group + 15) / 16);
    const int64_t prefix_groups = p.tiles * a.pool.heads * p.prefix_splits;
    const int64_t own_groups = own_tiles * a.pool.heads * p.own_splits;
    const bool many = p.prefix_splits + p.own_splits >= kManyParts;
    const int64_t joins = ((int64_t)n * q_heads + (many ? 0 : kWaves - 1)) / (many ? 1 : kWaves);
    if (prefix_groups >= (1 << 24) || own_groups >= (1 << 24) || joins >= (1 << 24))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, pool->block_size, &a.pool,
                    st);
    if (s != PEEK_OK) return s;
    a.q = Rows{d_q, q_token_stride, q_head_stride};
    a.context = d_context;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.members = d_members;
    a.group_offsets = d_group_offsets;
    a.shared = d_shared;
    a.out = (uint16_t*)d_out;
    a.out_token = out_token_stride;
    a.out_head = out_head_stride;
    a.lse = d_lse;
    a.part_out = (float*)d_workspace;
    a.part_lse = (float*)((char*)d_workspace + p.part_lse);
    a.prefix_chunk = p.prefix_chunk;
    a.own_chunk = p.own_chunk;
    a.splits = p.prefix_splits + p.own_splits;
    set_scale(scale, &a.scale, &a.q_flip, &a.q_mask);
    with_types(type, pool->type, pool->head_dim, [&](auto t, auto m, auto d) {
      auto go = [&](auto kernel, int64_t count, int64_t tiles) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(kThreads), 0, st, a, (int32_t)tiles);
      };
      auto all = [&](auto wide) {
        if (prefix_groups > 0) {
          if (p.rows == 4) go(k_shared<t(), m(), d(), 4, true, wide()>, prefix_groups, p.tiles);
          else if (p.rows == 2) go(k_shared<t(), m(), d(), 2, true, wide()>, prefix_groups, p.tiles);
          else go(k_shared<t(), m(), d(), 1, true, wide()>, prefix_groups, p.tiles);
        }
        go(k_shared<t(), m(), d(), 1, false, wide()>, own_groups, own_tiles);
      };
      if (a.pool.log_block >= 4) all(std::true_type{});
      else all(std::false_type{});
    });
    hipError_t err = hipGetLastError();
    if (err == hipSuccess) {
      with_types(type, PEEK_TYPE_I8, pool->head_dim, [&](auto t, auto, auto d) {
        if (many) hipLaunchKernelGGL((k_shared_join<t(), d(), 16>), dim3((unsigned)joins), dim3(1024), 0, st, a);
        else hipLaunchKernelGGL((k_shared_join<t(), d(), 1>), dim3((unsigned)joins), dim3(kThreads), 0, st, a);
      });
      err = hipGetLastError();
    }
    if (err != hipSuccess) return fail(PEEK_ERR_DEVICE, "decode launch failed: %s", hipGetErrorString(err));
    return PEEK_OK;
  });
}

}  // extern "C"
