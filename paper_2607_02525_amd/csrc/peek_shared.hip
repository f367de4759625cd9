// Attention of single tokens where groups of sequences share their first pages,
// on gfx950.
//
// A row (one query head of one sequence) is a softmax over two spans of keys:
// the group's, whose pages are those of its first member, and its own. Each
// span is cut into parts, every part leaves a row with sum of weight * value / sum
// of weights and the logarithm of that sum, and a last kernel joins a row's
// parts in a fixed order.
//
// Over a group's span the rows of all members stand side by side, (member,
// query head of the kv head) in that order, 32 to a wavefront, against tiles of
// 64 keys that the workgroup widens to 16 bits in LDS (peek_tile.h). Lengths
// and sizes of groups are on the device and as uneven as a queue is, so
// the work is one line of steps, (tile of rows, tile of keys) after each other
// through all groups, that is cut into equal pieces, one to a workgroup of as many as
// the device holds at once. A piece may end within a tile of rows and begin the
// next: what it leaves of each goes to a place of its own.
//
// Groups of few rows take tiles of 16 or 32 rows instead, and their keys to the
// products without LDS between wavefronts: they are bound by reading them. So
// is a sequence's own span, for which they serve too, in the same launch: what
// waits for memory runs beside what waits for the matrix cores.
#include <algorithm>

#include "peek_internal.h"
#include "peek_kv.h"
#include "peek_mfma.h"
#include "peek_tile.h"
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
constexpr int kTile = 32;             // own keys of a wavefront's step
constexpr int kMaxChunk = 4096;       // own keys of a workgroup, at most
constexpr int64_t kLeastSteps = 2;    // tiles of shared keys of a workgroup
constexpr int kFewKeys = kWaves * kTile;      // keys of a step of stream_keys

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
  float* part_out;                    // own keys: [n][q_heads][splits][D], n in the order of members
  float* part_lse;                    // [n][q_heads][splits]
  float* prefix_out;                  // shared keys: [kv_heads][slots][slot_rows][D]
  float* prefix_lse;                  // [kv_heads][slots][slot_rows]
  int64_t* first_step;                // [groups + 1]: steps before each group; then those of a piece
  int32_t* first_tile;                // [groups]: tiles of rows before it
  int32_t n, groups, group;           // `group`: query heads to a kv head
  int32_t own_chunk, splits;
  int32_t pieces, slots, slot_rows;   // of a kv head; piece w's part of tile u of rows is in slot w + u
  int32_t tile_rows, step_keys;       // of a step
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

// Group g: its positions, and the tokens that its members share with the first of them.
struct Group {
  int32_t index, lo, hi, tokens;
};
__device__ __forceinline__ Group group_at(const Shared& a, int32_t g) {
  Group x;
  x.index = g;
  x.lo = min(max(a.group_offsets[g], 0), a.n);
  x.hi = min(max(a.group_offsets[g + 1], x.lo), a.n);
  const int32_t lb = a.pool.log_block;
  x.tokens = x.lo < x.hi ? kv::clip_tokens(a.shared[g], a.table.width, lb) >> lb << lb : 0;
  return x;
}

// What a sequence of `held` tokens shares of its group's: all of it, or nothing.
__device__ __forceinline__ int32_t shares(const Group& g, int32_t held) { return held >= g.tokens ? g.tokens : 0; }

// The group of a position: nothing shared where there is none.
__device__ __forceinline__ Group group_of(const Shared& a, int32_t position, int lane) {
  const Group none{0, 0, 0, 0};
  if (a.groups == 0) return none;
  const int32_t g = kv::last_at_most(a.groups, position, lane, [&](int32_t i) { return (int64_t)a.group_offsets[i]; });
  const Group x = group_at(a, g);
  return x.lo <= position && position < x.hi ? x : none;
}

// The answer where there are no keys: 0, and -infinity.
template <int D>
__device__ __forceinline__ void no_keys(const Shared& a, int32_t r, int32_t q_head, int32_t rows) {
  for (int32_t i = threadIdx.x; i < rows * D; i += kThreads)
    a.out[(int64_t)r * a.out_token + (q_head + i / D) * a.out_head + i % D] = 0;
  if (a.lse && threadIdx.x < rows)
    a.lse[(int64_t)r * a.group * a.pool.heads + q_head + threadIdx.x] = -__builtin_inff();
}

struct alignas(16) Block {
  float scale, log_v, inv_v;
  uint32_t page;
};

// Each lane's 16 bytes at `base` + its offset to LDS at `to` + 16 * lane, base
// and `to` the same for the wavefront; done when vmcnt says so. No vector
// register is written. (m0 is reserved: the compiler keeps nothing there.)
__device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base)
               : "memory");
}

// Waits until no more than LEFT of this wavefront's loads are on their way: the
// builtin, so that the compiler knows it and waits for none of these again.
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (LEFT & 15) | (LEFT >> 4 << 14));      // vmcnt(LEFT), the other counters as they are
  asm volatile("" ::: "memory");
}

// ------------------------------------------------------------- shared keys
// A step is a tile of rows (32 to a wavefront) against a tile of keys.

// The sum of the lanes up to this one.
__device__ __forceinline__ int64_t sum_to(int64_t x) {
  auto add = [&](auto move, auto rows) {        // what another lane has, 0 where there is none
    constexpr int kMove = move(), kRows = rows();
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, kMove, kRows, 0xf, kRows == 0xf);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), kMove, kRows, 0xf, kRows == 0xf);
    x += (int64_t)((uint64_t)hi << 32 | lo);
  };
  const std::integral_constant<int, 0xf> all{};
  add(std::integral_constant<int, 0x111>{}, all);        // within 16 lanes: from 1, 2, 4, 8 lanes below
  add(std::integral_constant<int, 0x112>{}, all);
  add(std::integral_constant<int, 0x114>{}, all);
  add(std::integral_constant<int, 0x118>{}, all);
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});      // lane 15 to the next 16, 47 too
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});      // lane 31 to the upper 32
  return x;
}
__device__ __forceinline__ int64_t lane_of(int64_t x, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// x / y of numbers from 0 on: nearly always of 32 bits, where it takes a tenth of the time.
__device__ __forceinline__ int64_t over(int64_t x, int64_t y) {
  return ((uint64_t)x | (uint64_t)y) >> 32 == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// A piece of one group's line of steps: its rows row0 .. of `rows` (row r is head r % group of member r / group from
// position lo on) against its tiles of keys first .. last - 1, of `tokens` keys in all.
struct Run {
  int32_t lo, rows, row0, first, last, tokens, leader, slot;
};

// The line of steps. A lane has the sums up to its group of the 64 groups at hand; up to 64 are looked at once.
template <int ROWS, int KEYS>
struct Line {
  int32_t g0, rows, keys;             // tiles of this lane's group
  Group group;
  int64_t steps, tiles;               // up to and with it
  int64_t steps0, tiles0;             // before the groups at hand
  int64_t all, each;                  // steps of all groups, and of a piece

  __device__ __forceinline__ void look(const Shared& a, int32_t from, int64_t steps_before, int64_t tiles_before, int lane) {
    g0 = from;
    steps0 = steps_before;
    tiles0 = tiles_before;
    rows = keys = 0;
    group = Group{0, 0, 0, 0};
    if (g0 + lane < a.groups) {
      group = group_at(a, g0 + lane);
      keys = (int32_t)(((int64_t)group.tokens + KEYS - 1) / KEYS);
      rows = group.tokens > 0 ? (int32_t)(((int64_t)(group.hi - group.lo) * a.group + ROWS - 1) / ROWS) : 0;
    }
    steps = steps_before + sum_to((int64_t)rows * keys);
    tiles = tiles_before + sum_to(rows);
  }

  // With `write`, where each group begins and what a piece has is written down for the join.
  __device__ __forceinline__ void count(const Shared& a, int64_t least, int lane, bool write) {
    int64_t s = 0, t = 0;
    for (int32_t g = 0; g < a.groups; g += kWave) {
      look(a, g, s, t, lane);
      if (write && g + lane < a.groups) {
        a.first_step[g + lane] = steps - (int64_t)rows * keys;
        a.first_tile[g + lane] = (int32_t)(tiles - rows);
      }
      s = lane_of(steps, kWave - 1);
      t = lane_of(tiles, kWave - 1);
    }
    all = s;
    each = max(least, over(all + a.pieces - 1, a.pieces));
    if (write && lane == 0) a.first_step[a.groups] = each;
  }

  // The run of piece `piece` that begins with step `at` (of those that there are) and ends before `end`.
  __device__ __forceinline__ Run find(const Shared& a, int32_t piece, int64_t at, int64_t end, int lane) {
    if (at < steps0) look(a, 0, 0, 0, lane);        // (counting ends with the last groups; runs come in order)
    uint64_t past = __ballot(steps > at);
    while (past == 0 && g0 + kWave < a.groups) {
      look(a, g0 + kWave, lane_of(steps, kWave - 1), lane_of(tiles, kWave - 1), lane);
      past = __ballot(steps > at);
    }
    const int l = __builtin_ctzll(past);
    Run x;
    const int32_t key_tiles = __builtin_amdgcn_readlane(keys, l);
    const int64_t in_group = at - lane_of(steps - (int64_t)rows * keys, l);
    const int32_t tile = __builtin_amdgcn_readfirstlane((int32_t)over(in_group, key_tiles));
    x.first = __builtin_amdgcn_readfirstlane((int32_t)(in_group - (int64_t)tile * key_tiles));
    x.last = __builtin_amdgcn_readfirstlane((int32_t)min((int64_t)key_tiles, x.first + (end - at)));
    x.lo = __builtin_amdgcn_readlane(group.lo, l);
    x.rows = (__builtin_amdgcn_readlane(group.hi, l) - x.lo) * a.group;
    x.row0 = tile * ROWS;
    x.tokens = __builtin_amdgcn_readlane(group.tokens, l);
    x.leader = __builtin_amdgcn_readfirstlane(max(0, member_at(a, x.lo)));        // (none: any pages)
    x.slot = piece + __builtin_amdgcn_readlane((int32_t)(tiles - rows), l) + tile;
    return x;
  }
};

// LDS of a workgroup of either kind: two buffers of K and V tiles and their scales, or the wavefronts' rings and their
// references and sums.
template <int D>
constexpr int kMemory = 4 * kKeys * D * 2 + 512;

template <int TYPE, int FMT, int D>
__device__ __forceinline__ void shared_tiles(const Shared& a, uint32_t block, uint8_t* memory) {
  using T = Tile<TYPE, FMT, D, kWaves>;
  constexpr int kRows = 32 * kWaves;
  constexpr int kEach = T::kUnitsEach;                        // 16-code units of a tile and thread
  constexpr int kMine = kEach / 2;                            // keys that they are of, K and V of each
  constexpr int kStride = kThreads / (D / 16);                // from one of these to the next
  uint8_t(*const s_k)[T::kBytes] = (uint8_t(*)[T::kBytes])memory;
  uint8_t(*const s_v)[T::kBytes] = s_k + 2;
  f4(*const s_scale)[kKeys / 4] = (f4(*)[kKeys / 4])(s_v + 2);

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // kv heads side by side: each on XCDs of its own where there are eight
  const int32_t head = block % a.pool.heads, piece = block / a.pool.heads, lb = a.pool.log_block;
  Line<kRows, kKeys> line;
  line.count(a, kLeastSteps, lane, block == 0 && wave == 0);
  const int64_t end = min(line.all, (piece + 1) * line.each);

  const int col = lane & 31, half = lane >> 5;
  const uint32_t lds_k = (uint32_t)(uintptr_t)(lds_byte*)s_k, lds_v = (uint32_t)(uintptr_t)(lds_byte*)s_v;
  const uint32_t half_bytes = ((uint32_t)a.pool.heads << lb) * D;         // a page's keys, or values
  const uint8_t* head_pages = a.pool.pages + ((int64_t)head << lb) * D;
  const int32_t unit_key = tid / (D / 16) % kKeys, unit_at = tid % (D / 16);
  const bool leads = unit_at == 0 && (unit_key & 3) == 0;       // fetches four keys' scales

  for (int64_t at = piece * line.each; at < end;) {
    const Run run = line.find(a, piece, at, end, lane);
    const int32_t first = run.first, last = run.last, held = run.tokens, rows = run.rows, row0 = run.row0;
    const int32_t slot = run.slot;
    at += last - first;

    // this lane's row; those past the last, of no sequence or of one that shares nothing are computed as any
    const bool active = row0 + wave * 32 < rows;
    const int32_t row = min(row0 + wave * 32 + col, rows - 1), member = row / a.group;
    const int32_t q_head = head * a.group + row - member * a.group;
    int32_t r = member_at(a, run.lo + member);
    if (r < 0) r = run.leader;
    T tile;
    {
      const uint16_t* q = (const uint16_t*)a.q.data + (int64_t)r * a.q.token + q_head * a.q.head + half * 8;
#pragma unroll
      for (int s = 0; s < T::kSteps; ++s) {
        tile.q[s] = *(const u4*)(q + 16 * s);
#pragma unroll
        for (int e = 0; e < 4; ++e) tile.q[s][e] = (tile.q[s][e] ^ a.q_flip) & a.q_mask;
      }
#pragma unroll
      for (int p = 0; p < T::kParts; ++p) tile.acc[p] = (f16){};
      tile.top = tile.peak = kNone;
      tile.far = ~0ull;
      tile.sum = 0.0f;
    }

    const int32_t* ids = a.table.ids + (int64_t)run.leader * a.table.stride;
    u4 codes[kEach];
    float scale_k[kMine], scale_v[kMine];
    int32_t page[kMine];      // as the table has it: looked at only when it is used, a tile later
    auto key_of = [&](int32_t j, int k) { return min(j * kKeys + unit_key + k * kStride, held - 1); };
    auto find_page = [&](int32_t j) {
#pragma unroll
      for (int k = 0; k < kMine; ++k) page[k] = ids[key_of(j, k) >> lb];
    };
    auto fetch = [&](int32_t j) {
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        const uint32_t id = (uint32_t)page[k] < a.pool.num_pages ? (uint32_t)page[k] : 0u;
        const uint32_t in_block = key_of(j, k) & ((1 << lb) - 1);
        const uint8_t* p = head_pages + (uint64_t)id * (2 * half_bytes) + in_block * D + unit_at * 16;
        codes[k] = *(const u4*)p;
        codes[kMine + k] = *(const u4*)(p + half_bytes);
        if (leads) {
          const float* x = a.pool.scales + head + (uint64_t)id * (uint32_t)(2 * a.pool.heads);
          scale_k[k] = x[0];
          scale_v[k] = x[a.pool.heads];
        }
      }
    };
    auto store = [&](int buf) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const bool is_v = i >= kMine;
        const int32_t key = unit_key + i % kMine * kStride;
        const u2 x0 = widen4<TYPE, FMT>(codes[i][0]), x1 = widen4<TYPE, FMT>(codes[i][1]);
        const u2 x2 = widen4<TYPE, FMT>(codes[i][2]), x3 = widen4<TYPE, FMT>(codes[i][3]);
        uint8_t* to = is_v ? s_v[buf] : s_k[buf];
        const uint32_t c = 2 * unit_at;
        const uint32_t p0 = is_v ? v_piece<D>(key, c) : k_piece<D>(key, c);
        const uint32_t p1 = is_v ? v_piece<D>(key, c + 1) : k_piece<D>(key, c + 1);
        *(u4*)(to + 16 * p0) = (u4){x0[0], x0[1], x1[0], x1[1]};
        *(u4*)(to + 16 * p1) = (u4){x2[0], x2[1], x3[0], x3[1]};
      }
      if (leads) {
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          const float v = kv::value_scale(scale_v[k]);
          s_scale[buf][(unit_key + k * kStride) / 4] =
              (f4){scale_k[k] * a.scale, log2_fast(v), __builtin_amdgcn_rcpf(v), 0.0f};
        }
      }
    };

    find_page(first);
    fetch(first);
    if (first + 1 < last) find_page(first + 1);
    __syncthreads();                       // (a piece's tile of rows before this one is done with)
    store(first & 1);
    __syncthreads();
    for (int32_t j = first; j < last; ++j) {
      const int buf = j & 1;
      if (j + 1 < last) {
        fetch(j + 1);
        if (j + 2 < last) find_page(j + 2);
      }
      const int32_t left = held - j * kKeys;
      if (active)
        tile.template step<true>(lds_k + buf * T::kBytes, lds_v + buf * T::kBytes, s_scale[buf], lane, a.scale,
                                 left < kKeys, left);
      if (j + 1 < last) store(buf ^ 1);
      __syncthreads();
    }
    // (groups that overlap have more tiles than there is room for)
    if (active && row0 + wave * 32 + col < rows && (uint32_t)slot < (uint32_t)a.slots) {
      const float sum = sum_halves(tile.sum), over = 1.0f / sum;
      const int64_t place = ((int64_t)head * a.slots + slot) * a.slot_rows + wave * 32 + col;
      float* out = a.prefix_out + place * D + half * 4;
#pragma unroll
      for (int p = 0; p < T::kParts; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f16& x = tile.acc[p];
          *(f4*)(out + 32 * p + 8 * e) =
              (f4){x[4 * e] * over, x[4 * e + 1] * over, x[4 * e + 2] * over, x[4 * e + 3] * over};
        }
      if (half == 0) a.prefix_lse[place] = log2_sum(tile.top, sum);
    }
  }
}

// The same for few rows to a group, 16 ROWS to a tile, which are bound by the
// reading, and after it in one launch the sequences' own keys: workgroups past
// `shared_groups` take a tile of one sequence's rows and a chunk of its keys each.
// A wavefront takes every fourth 32 keys, all by itself, and
// keeps two of them on their way in a ring of its own in LDS. What a lane puts there
// is what it reads again, so no other lane waits for it; the slot of the keys at
// hand is asked to be filled again as soon as they are in registers. Blocks of 16
// tokens or more: 16 keys lie in one page, which scalar loads find.
//
// Bound by memory: 16 documents of 3200 to 7168 tokens in blocks of 16, 8 kv heads of 128,
// with 128 users and their own 32 to 700 tokens, 260 MB: 76 us. Own keys alone, 192 times 500 to 8000
// in blocks of 64, 1.67 GB: 312 us, 5.4 TB/s. With one slot and twice the workgroups these
// took 336 (256 sequences of 16 own tokens: 93 us instead of 101), from registers
// without a ring 338. Tiles of 48 rows took 66 us where these take 54 for the shared
// keys of the documents, tiles of 64 rows 83: more vector instructions to a
// wavefront, whose keys still come at the rate of memory.
template <int TYPE, int FMT, int D, int ROWS>
__device__ __forceinline__ void stream_keys(const Shared& a, uint32_t block, uint32_t shared_groups, uint8_t* memory) {
  constexpr int kSteps = D / 32, kParts = D / 16;
  constexpr int kRows = 16 * ROWS;
  constexpr int kLoads = D / 16;                  // of a tile: 1 KB each, keys and then values
  constexpr int kSlot = kLoads * 1024;
  constexpr int kTurn = kWaves * kTile;
  constexpr int kJoin = kWaves * 16 * (D + 4) * (int)sizeof(float);
  constexpr int kRing = kWaves * 2 * kSlot;
  static_assert(kRing + 512 <= kMemory<D> && kJoin + 512 <= kMemory<D>, "the rings and what is joined fit");
  uint8_t* const s_ring = memory;
  float(*const s_top)[16] = (float(*)[16])(memory + kMemory<D> - 512);
  float(*const s_sum)[16] = s_top + kWaves;

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const bool own = block >= shared_groups;
  const uint32_t unit = own ? block - shared_groups : block;
  const int32_t head = unit % a.pool.heads, lb = a.pool.log_block, q_heads = a.group * a.pool.heads;
  const int32_t piece = unit / a.pool.heads;
  Line<kRows, kFewKeys> line;
  int64_t at = 0, end = 1;
  Run run;
  int32_t from = 0, split = 0;
  bool whole = false;
  if (own) {
    const int32_t row_tiles = (a.group + kRows - 1) / kRows, position = piece / row_tiles % a.n;
    split = piece / row_tiles / a.n;
    // (the group is looked for while the member is on its way, and read while its context is)
    const int32_t r = member_at(a, position);
    const Group g = group_of(a, position, lane);
    const int32_t held = held_by(a, max(0, r));
    run = Run{position, a.group, piece % row_tiles * kRows, 0, 0, held, r, 0};
    if (r < 0) return;
    if (held == 0) {
      if (split == 0) no_keys<D>(a, r, head * a.group + run.row0, min(kRows, a.group - run.row0));
      return;
    }
    const int32_t begin = shares(g, held);
    if ((int64_t)split * a.own_chunk >= held - begin) return;
    from = begin + split * a.own_chunk;
    whole = begin == 0 && held <= a.own_chunk;      // the only part: this is the answer
  } else {
    line.count(a, 1, lane, block == 0 && wave == 0);
    at = piece * line.each;
    end = min(line.all, at + line.each);
  }
  const int grp = lane >> 4, col = lane & 15;
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_byte*)s_ring + wave * 2 * kSlot;
  const uint8_t* const here = s_ring + wave * 2 * kSlot;
  const uint32_t half_page = ((uint32_t)a.pool.heads << lb) * D;      // bytes from a page's keys to its values
  typedef const __attribute__((address_space(4))) int32_t* const_ints;
  typedef const __attribute__((address_space(4))) float* const_floats;
  const const_floats scales = (const_floats)a.pool.scales;
  // values: 16-byte piece `v_piece` of token v_token[k], so that the tokens 4 g + e of every e lie side by side
  int32_t v_token[D / 64];
#pragma unroll
  for (int k = 0; k < D / 64; ++k) {
    const int row = (k * kWave + lane) / (D / 16);
    v_token[k] = 4 * (row & 3) + (row >> 2);
  }
  const uint32_t v_at = half_page + lane % (D / 16) * 16;

  while (at < end) {
    int32_t count;
    if (own) {
      count = min(a.own_chunk, run.tokens - from);
      at = end;
    } else {
      run = line.find(a, piece, at, end, lane);
      from = run.first * kFewKeys;
      count = (int32_t)min((int64_t)(run.tokens - from), (int64_t)(run.last - run.first) * kFewKeys);
      at += run.last - run.first;
    }
    const int32_t rows = run.rows, row0 = run.row0, slot = run.slot;
    // `count` keys from `from` on, `mine` of them from this wavefront's first one
    const int32_t to = from + count, mine = count - wave * kTile;

    u4 q[ROWS][kSteps];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      // rows past the last, of no sequence or of one that shares nothing are computed as any
      const int32_t row = min(row0 + 16 * i + col, rows - 1), member = row / a.group;
      const int32_t q_head = head * a.group + row - member * a.group;
      int32_t r = member_at(a, run.lo + member);
      if (r < 0) r = run.leader;
      const uint16_t* p = (const uint16_t*)a.q.data + (int64_t)r * a.q.token + q_head * a.q.head + grp * (D / 4);
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        q[i][k] = *(const u4*)(p + 8 * k);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[i][k][e] = (q[i][k][e] ^ a.q_flip) & a.q_mask;
      }
    }
    f4 acc[ROWS][kParts] = {};
    float top[ROWS], peak[ROWS], sum[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      top[i] = peak[i] = kNone;
      sum[i] = 0.0f;
    }
    const const_ints ids = (const_ints)(a.table.ids + (int64_t)run.leader * a.table.stride);
    uint32_t found[2];                // entries of the table, asked for a tile before they are used
    float raw_k[2][2], raw_v[2][2];   // scales of the tiles in either slot
    // A tile is named by the keys that are left from its first one on (none: the last 16 again); no sum passes `to`.
    auto half_at = [&](int32_t left, int h) { return left > 16 * h ? to - (left - 16 * h) : (to - 1) & ~15; };
    auto find = [&](int32_t left) {
#pragma unroll
      for (int h = 0; h < 2; ++h) found[h] = (uint32_t)ids[half_at(left, h) >> lb];
    };
    auto load = [&](int32_t left, auto slot_of) {
      constexpr int o = slot_of();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int32_t t = half_at(left, h), limit = to - 1 - t;
        const uint32_t page = found[h] < a.pool.num_pages ? found[h] : 0u;
        const int64_t place = (int64_t)page * 2 * a.pool.heads + head;
        const uint8_t* base = a.pool.pages + ((place << lb) + (t & ((1 << lb) - 1))) * D;
        raw_k[o][h] = scales[place];
        raw_v[o][h] = scales[place + a.pool.heads];
        const uint32_t k_at = min(col, limit) * D + grp * (D / 4);
#pragma unroll
        for (int k = 0; k < D / 64; ++k) {
          to_lds(base, k_at + 16 * k, ring + o * kSlot + (h * (D / 64) + k) * 1024);
          to_lds(base, v_at + min(v_token[k], limit) * D, ring + o * kSlot + kSlot / 2 + (h * (D / 64) + k) * 1024);
        }
      }
    };
    auto step = [&](int32_t left, auto slot_of) {
      constexpr int o = slot_of();
      // (those of the next tile may be on their way)
      if (left > kTurn) wait_loads<kLoads>();
      else wait_loads<0>();
      const uint8_t* in = here + o * kSlot;
      u4 kw[2][D / 64];
      uint32_t vw[8][kParts / 4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int k = 0; k < D / 64; ++k) kw[h][k] = *(const u4*)(in + (h * (D / 64) + k) * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint8_t* pv = in + kSlot / 2 + h * (D * 16) + (e * 4 + grp) * D + col * kParts;
          if constexpr (kParts == 8) {
            const u2 w = *(const u2*)pv;
            vw[4 * h + e][0] = w[0];
            vw[4 * h + e][1] = w[1];
          } else {
            vw[4 * h + e][0] = *(const uint32_t*)pv;
          }
        }
      }
      float scale[2], log_v[2], inv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float v = kv::value_scale(raw_v[o][h]);
        scale[h] = raw_k[o][h] * a.scale;
        log_v[h] = log2_fast(v);
        inv[h] = __builtin_amdgcn_rcpf(v);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the slot has been read
      if (left > 2 * kTurn) {
        load(left - 2 * kTurn, slot_of);
        find(left - 3 * kTurn);
      }
      f4 s[ROWS][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) s[i][h] = (f4){};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const u2 lo = widen4<TYPE, FMT>(kw[h][k / 2][2 * (k & 1)]), hi = widen4<TYPE, FMT>(kw[h][k / 2][2 * (k & 1) + 1]);
          const u4 key = (u4){lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
          for (int i = 0; i < ROWS; ++i) s[i][h] = mul16<TYPE>(key, q[i][k], s[i][h]);
        }
      }
      u4 w[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][h][e] = fmaf(s[i][h][e], scale[h], log_v[h]);
        if (left < kTile) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[i][h][e] = 16 * h + 4 * grp + e < left ? s[i][h][e] : -__builtin_inff();
        }
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
    };
    const std::integral_constant<int, 0> s0{};
    const std::integral_constant<int, 1> s1{};
    if (mine > 0) {
      find(mine);
      wait_loads<0>();                // q is there: from here on the loads in flight are the ring's
      load(mine, s0);
      find(mine - kTurn);
      if (mine > kTurn) load(mine - kTurn, s1);
      find(mine - 2 * kTurn);
      for (int32_t left = mine;; left -= 2 * kTurn) {
        step(left, s0);
        if (left <= kTurn) break;
        step(left - kTurn, s1);
        if (left <= 2 * kTurn) break;
      }
    }

    // the wavefronts' results, joined: acc register v of part p is row col, element (4 grp + v) kParts + p
    float(*s_out)[16][D + 4] = (float(*)[16][D + 4])s_ring;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float here_sum = sum_halves(swap16_sum(sum[i]));
      __syncthreads();                // the rings, or what was joined before, are done with
      if (grp == 0) {
        s_top[wave][col] = top[i];
        s_sum[wave][col] = here_sum;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int p = 0; p < kParts; ++p) s_out[wave][col][(4 * grp + e) * kParts + p] = acc[i][p][e];
      __syncthreads();
      for (int32_t u = tid; u < 16 * (D / 8); u += kThreads) {
        const int32_t c = u / (D / 8), d = u % (D / 8) * 8;
        // (groups that overlap have more tiles than there is room for)
        if (row0 + 16 * i + c >= rows || (uint32_t)slot >= (uint32_t)a.slots) continue;
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
        const float by = 1.0f / total, l2 = log2_sum(highest, total);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= by;
        const int32_t q_head = head * a.group + row0 + 16 * i + c;        // (of own keys)
        if (whole) {
          *(u4*)(a.out + (int64_t)run.leader * a.out_token + q_head * a.out_head + d) =
              (u4){pack2<TYPE>(o[0], o[1]), pack2<TYPE>(o[2], o[3]), pack2<TYPE>(o[4], o[5]), pack2<TYPE>(o[6], o[7])};
          if (a.lse && d == 0) a.lse[(int64_t)run.leader * q_heads + q_head] = l2 * 0.69314718055994531f;
          continue;
        }
        const int64_t place = own ? ((int64_t)run.lo * q_heads + q_head) * a.splits + split
                                  : ((int64_t)head * a.slots + slot) * a.slot_rows + 16 * i + c;
        f4* p = (f4*)((own ? a.part_out : a.prefix_out) + place * D + d);
        p[0] = (f4){o[0], o[1], o[2], o[3]};
        p[1] = (f4){o[4], o[5], o[6], o[7]};
        if (d == 0) (own ? a.part_lse : a.prefix_lse)[place] = l2;
      }
    }
    __syncthreads();
  }
}

// ----------------------------------------------------------------- kernels
template <int TYPE, int FMT, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_shared_tiles(Shared a) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_memory[kMemory<D>];
  shared_tiles<TYPE, FMT, D>(a, blockIdx.x, s_memory);
}
template <int TYPE, int FMT, int D, int ROWS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_shared_stream(Shared a, uint32_t shared_groups) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_memory[kMemory<D>];
  stream_keys<TYPE, FMT, D, ROWS>(a, blockIdx.x, shared_groups, s_memory);
}
// Workgroups below `shared_groups` take tiles of 128 rows over shared keys, the others own keys, beside them.
template <int TYPE, int FMT, int D, int ROWS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_shared_both(Shared a, uint32_t shared_groups) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_memory[kMemory<D>];
  if (blockIdx.x < shared_groups) shared_tiles<TYPE, FMT, D>(a, blockIdx.x, s_memory);
  else stream_keys<TYPE, FMT, D, ROWS>(a, blockIdx.x - shared_groups, 0, s_memory);
}

// ------------------------------------------- own keys in blocks of 4 or 8
// 16 rows of one sequence over a chunk of its own keys, as
// in the decode of single sequences. Blocks are looked up in LDS.
template <int TYPE, int FMT, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void k_shared_own(Shared a) {
  constexpr int kSteps = D / 32;        // products of keys and queries a 16-token half
  constexpr int kParts = D / 16;        // 16-wide parts of the output; also bytes of a token's values in a lane
  constexpr int kKeyWords = D / 16;     // words of a token's key in a lane
  __shared__ Block s_block[kMaxChunk / 4 + 1];
  __shared__ float s_out[kWaves][16][D + 4];
  __shared__ float s_top[kWaves][16], s_sum[kWaves][16];

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t q_heads = a.group * a.pool.heads, lb = a.pool.log_block;
  uint32_t unit = blockIdx.x;
  const int32_t head = unit % a.pool.heads;
  unit /= a.pool.heads;
  const int32_t row_tiles = (a.group + 15) / 16;
  const int32_t row0 = unit % row_tiles * 16;
  unit /= row_tiles;
  const int32_t position = unit % a.n, split = unit / a.n;
  // (the group is looked for while the member is on its way, and read while its context is)
  const int32_t r = member_at(a, position);
  const Group g = group_of(a, position, lane);
  const int32_t held = held_by(a, max(0, r));
  const int32_t rows = min(16, a.group - row0);
  if (r < 0) return;
  if (held == 0) {
    if (split == 0) no_keys<D>(a, r, head * a.group + row0, rows);
    return;
  }
  const int32_t begin = shares(g, held);
  if ((int64_t)split * a.own_chunk >= held - begin) return;
  // tokens from here on are counted from `from`, a block's first: no sum of them comes near 2^31
  const int32_t from = begin + split * a.own_chunk, to = min(a.own_chunk, held - from);
  const bool whole = begin == 0 && held <= a.own_chunk;      // the only part: this is the answer

  const int32_t* const row_ids = a.table.ids + r * a.table.stride + (from >> lb);
  const int32_t blocks = ((to - 1) >> lb) + 1;
  for (int32_t i = tid; i < blocks; i += kThreads) {
    const uint32_t id = (uint32_t)row_ids[i], page = id < a.pool.num_pages ? id : 0u;
    const int64_t at = (int64_t)page * 2 * a.pool.heads + head;
    const float k = a.pool.scales[at], v = kv::value_scale(a.pool.scales[at + a.pool.heads]);
    s_block[i] = Block{k * a.scale, log2_fast(v), __builtin_amdgcn_rcpf(v), page};
  }
  const int32_t grp = lane >> 4, col = lane & 15;
  u4 q[kSteps];
  {
    const int32_t q_head = head * a.group + min(row0 + col, a.group - 1);
    const uint16_t* p = (const uint16_t*)a.q.data + (int64_t)r * a.q.token + q_head * a.q.head + grp * (D / 4);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      q[s] = *(const u4*)(p + 8 * s);
#pragma unroll
      for (int e = 0; e < 4; ++e) q[s][e] = (q[s][e] ^ a.q_flip) & a.q_mask;
    }
  }
  __syncthreads();

  f4 acc[kParts] = {};
  float top = kNone, peak = kNone, sum = 0.0f;
  uint32_t kw[2][kKeyWords];        // keys, and values, of the tile at hand, then of the next
  uint32_t vw[8][kParts / 4];
  float scale[2], log_v[2], inv_v[2];
  const int64_t half_page = ((int64_t)a.pool.heads << lb) * D;      // bytes from a page's keys to its values

  auto row_at = [&](int32_t t) {
    const uint32_t page = s_block[t >> lb].page;
    return a.pool.pages + ((((int64_t)page * 2 * a.pool.heads + head) << lb) + (t & ((1 << lb) - 1))) * D;
  };
  auto load_keys = [&](int32_t t0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* p = row_at(min(t0 + 16 * h + col, to - 1)) + grp * (D / 4);
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
      const int32_t t = min(t0 + 16 * h + 4 * grp, (to - 1) & ~3);      // four tokens of one block
      const uint8_t* p = row_at(t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint8_t* pv = p + half_page + (uint32_t)(min(e, to - 1 - t) * D + col * kParts);
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
      for (int k = 0; k < kSteps; ++k) {
        const u2 lo = widen4<TYPE, FMT>(kw[h][2 * k]), hi = widen4<TYPE, FMT>(kw[h][2 * k + 1]);
        s[h] = mul16<TYPE>((u4){lo[0], lo[1], hi[0], hi[1]}, q[k], s[h]);
      }
      const Block c = s_block[min(t0 + 16 * h + 4 * grp, to - 1) >> lb];
      scale[h] = c.scale;
      log_v[h] = c.log_v;
      inv_v[h] = c.inv_v;
    }
    const float inv[2] = {inv_v[0], inv_v[1]};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[h][e] = fmaf(s[h][e], scale[h], log_v[h]);
    if (more) {
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
      sum += ((s[h][0] + s[h][1]) + (s[h][2] + s[h][3])) * inv[h];
      w[2 * h] = pack2<TYPE>(s[h][0], s[h][1]);
      w[2 * h + 1] = pack2<TYPE>(s[h][2], s[h][3]);
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
    const int32_t mine = to - wave * kTile;      // tokens from this wavefront's first one on
    if (mine > 0) {
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
  for (int32_t i = tid; i < rows * (D / 8); i += kThreads) {
    const int32_t g = i / (D / 8), d = i % (D / 8) * 8, q_head = head * a.group + row0 + g;
    float highest = s_top[0][g];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) highest = fmaxf(highest, s_top[w][g]);
    float total = 0.0f, o[8] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = exp2_fast(s_top[w][g] - highest);
      total += by * s_sum[w][g];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += by * s_out[w][g][d + e];
    }
    const float over = 1.0f / total, l2 = log2_sum(highest, total);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= over;
    if (whole) {
      *(u4*)(a.out + (int64_t)r * a.out_token + q_head * a.out_head + d) =
          (u4){pack2<TYPE>(o[0], o[1]), pack2<TYPE>(o[2], o[3]), pack2<TYPE>(o[4], o[5]), pack2<TYPE>(o[6], o[7])};
      if (a.lse && d == 0) a.lse[(int64_t)r * q_heads + q_head] = l2 * 0.69314718055994531f;
    } else {
      const int64_t at = ((int64_t)position * q_heads + q_head) * a.splits + split;
      f4* p = (f4*)(a.part_out + at * D + d);
      p[0] = (f4){o[0], o[1], o[2], o[3]};
      p[1] = (f4){o[4], o[5], o[6], o[7]};
      if (d == 0) a.part_lse[at] = l2;
    }
  }
}

// ------------------------------------------------------------------- join
// WAVES wavefronts to a row; its parts of shared keys first, then those of its own.
template <int TYPE, int D, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : kWave * WAVES) void k_shared_join(Shared a) {
  constexpr int kRowsHere = WAVES == 1 ? kWaves : 1, kLanes = D / 64;      // floats of a lane
  __shared__ float s_sum[WAVES > 1 ? WAVES * D : 1];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t q_heads = a.group * a.pool.heads;
  const int64_t row = (int64_t)blockIdx.x * kRowsHere + wave / WAVES;
  if (row >= (int64_t)a.n * q_heads) return;
  const int32_t position = (int32_t)(row / q_heads), q_head = (int32_t)(row % q_heads), r = member_at(a, position);
  const Group g = group_of(a, position, lane);
  const int32_t held = held_by(a, max(0, r));
  if (r < 0 || held == 0) return;
  const int32_t begin = shares(g, held);
  if (begin == 0 && held <= a.own_chunk) return;       // the answer is there
  // the pieces that the row's tile was in
  int64_t place = 0;
  int32_t shared_parts = 0;
  const int64_t stride = a.slot_rows;
  if (begin > 0) {
    const int32_t head = q_head / a.group, rows = a.tile_rows;
    const int32_t in_group = (position - g.lo) * a.group + q_head - head * a.group, tile = in_group / rows;
    const int32_t keys = (int32_t)(((int64_t)g.tokens + a.step_keys - 1) / a.step_keys);
    const int64_t each = a.first_step[a.groups], from = a.first_step[g.index] + (int64_t)tile * keys;
    const int64_t piece = over(from, each);
    shared_parts = (int32_t)(over(from + keys - 1, each) - piece) + 1;
    const int64_t slot = piece + a.first_tile[g.index] + tile;
    if (slot < 0 || slot + shared_parts > a.slots) return;
    place = ((int64_t)head * a.slots + slot) * stride + in_group - tile * rows;
  }
  const int32_t parts = shared_parts + parts_of(held - begin, a.own_chunk);
  auto lse_of = [&](int32_t s) {
    return s < shared_parts ? a.prefix_lse[place + s * stride] : a.part_lse[row * a.splits + s - shared_parts];
  };
  auto out_of = [&](int32_t s) {
    return s < shared_parts ? a.prefix_out + (place + s * stride) * D : a.part_out + (row * a.splits + s - shared_parts) * D;
  };
  float top = kNone, sum = 0.0f;
  for (int32_t s = lane; s < parts; s += kWave) {
    const float x = lse_of(s), next = fmaxf(top, x);
    sum = sum * exp2_fast(top - next) + exp2_fast(x - next);
    top = next;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float x = __shfl_xor(top, d), y = __shfl_xor(sum, d), next = fmaxf(top, x);
    sum = sum * exp2_fast(top - next) + y * exp2_fast(x - next);
    top = next;
  }
  const float l2 = log2_sum(top, sum);
  const int mine = wave % WAVES;
  float o[kLanes] = {};
  const int32_t share = (parts + WAVES - 1) / WAVES, end = min(parts, (mine + 1) * share);
  for (int32_t s0 = mine * share; s0 < end; s0 += kWave) {
    const int32_t count = min(kWave, end - s0);
    const float weight = lane < count ? exp2_fast(lse_of(s0 + lane) - l2) : 0.0f;
    for (int32_t s1 = 0; s1 < count; s1 += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {      // those past the last read the last again, as 0 (it may be infinite)
        const int32_t s = s1 + i;
        const float by = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), s));
        const float* from = out_of(s0 + min(s, count - 1)) + lane * kLanes;
#pragma unroll
        for (int e = 0; e < kLanes; ++e) {
          const float x = from[e];
          o[e] = fmaf(by, s < count ? x : 0.0f, o[e]);
        }
      }
    }
  }
  uint16_t* out = a.out + (int64_t)r * a.out_token + q_head * a.out_head;
  if (a.lse && lane == 0 && mine == 0) a.lse[(int64_t)r * q_heads + q_head] = l2 * 0.69314718055994531f;
  if constexpr (WAVES == 1) {
    if constexpr (kLanes == 2) *(uint32_t*)(out + 2 * lane) = pack2<TYPE>(o[0], o[1]);
    else out[lane] = kv::from_float<TYPE>(o[0]);
  } else {
#pragma unroll
    for (int e = 0; e < kLanes; ++e) s_sum[mine * D + lane * kLanes + e] = o[e];
    __syncthreads();
    const int d = threadIdx.x;
    if (d < D) {
      float x = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) x += s_sum[w * D + d];
      out[d] = kv::from_float<TYPE>(x);
    }
  }
}

// -------------------------------------------------------------- validation
// What the call reads: a group's shared blocks in its first member's row (where a member shares them), a member's own
// ones in its own.
constexpr int32_t kBadMember = 16, kMemberTwice = 32, kBadGroups = 64, kBadShared = 128;

__global__ __launch_bounds__(kWave) void k_validate_shared(Shared a, int32_t* __restrict__ bad, int32_t* __restrict__ seen) {
  const int lane = threadIdx.x, lb = a.pool.log_block;
  const int64_t most = (int64_t)a.table.width << lb;
  int32_t f = 0;
  if ((int32_t)blockIdx.x < a.groups) {
    const int32_t g = blockIdx.x, from = a.group_offsets[g], to = a.group_offsets[g + 1];
    if (from < 0 || to < from || to > a.n || (g == 0 && from != 0)) f |= kBadGroups;
    const Group x = group_at(a, g);
    if (x.lo < x.hi && (a.shared[g] < 0 || a.shared[g] > most)) f |= kBadShared;
    bool read = false;
    for (int32_t i = x.lo + lane; i < x.hi && x.tokens > 0; i += kWave) {
      const int32_t r = member_at(a, i);
      read = read || (r >= 0 && shares(x, held_by(a, r)) > 0);
    }
    if (__any(read)) {
      const int32_t r = max(0, member_at(a, x.lo));
      for (int32_t b = lane; b < x.tokens >> lb; b += kWave) f |= kv::block_faults(a.table, a.pool, r, b, true, false);
    }
  } else {
    const int32_t position = blockIdx.x - a.groups, r = member_at(a, position);
    const Group g = group_of(a, position, lane);
    if (r < 0) {
      f |= kBadMember;
    } else {
      if (lane == 0 && atomicAdd(&seen[r], 1) > 0) f |= kMemberTwice;
      const int32_t held = a.context[r];
      if (held < 0 || held > most) {
        f |= kv::kBadLength;
      } else {
        const int32_t blocks = (int32_t)(((int64_t)held + (1 << lb) - 1) >> lb);
        for (int32_t b = (shares(g, held) >> lb) + lane; b < blocks; b += kWave)
          f |= kv::block_faults(a.table, a.pool, r, b, true, false);
      }
    }
  }
  if (f) atomicOr(bad, f);
}
__global__ void k_clear(int32_t* p, int32_t count) {
  const int32_t i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < count) p[i] = 0;
}

// With PEEK_VALIDATE: group offsets from 0, non-decreasing, within 0 .. n, members within the batch and each once,
// lengths within the table, pages and scales of what is read. Waits for `st`.
peek_status validate_shared(const Shared& a, hipStream_t st) {
  if (!validation_enabled()) return PEEK_OK;
  int32_t* d_bad = nullptr;
  PEEK_HIP_TRY(hipMalloc((void**)&d_bad, ((size_t)a.n + 1) * sizeof(int32_t)));
  int32_t bad = 0;
  hipLaunchKernelGGL(k_clear, dim3((unsigned)(a.n / 256 + 1)), dim3(256), 0, st, d_bad, a.n + 1);
  hipLaunchKernelGGL(k_validate_shared, dim3((unsigned)(a.groups + a.n)), dim3(kWave), 0, st, a, d_bad, d_bad + 1);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = hipMemcpyAsync(&bad, d_bad, sizeof(int32_t), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  (void)hipFree(d_bad);
  if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "input validation failed to run: %s", hipGetErrorString(e));
  if (bad & kBadGroups)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "d_group_offsets must be non-decreasing offsets from 0, within 0 .. n");
  if (bad & kBadMember) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_members names sequences outside the batch");
  if (bad & kMemberTwice) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_members names a sequence twice");
  if (bad & kBadShared)
    return fail(PEEK_ERR_INVALID_ARGUMENT, "a group shares fewer than 0 tokens or more than the table holds");
  return kv_status(bad);
}

// -------------------------------------------------------------------- plan
struct Plan {
  bool few;                           // shared keys by stream_keys
  int32_t own_rows;                   // of a tile of own keys
  int32_t tile_rows;
  int32_t pieces, slots, slot_rows;
  int32_t own_chunk, own_splits;
  size_t part_lse, prefix_out, prefix_lse, first_step, first_tile, bytes;
};

// Own keys are cut into chunks, of 256 to kMaxChunk, that leave no more workgroups than this where tables are full: empty
// ones wait for a sequence's length and group before they end (with 8192 the 128 document chats take 81 us instead of
// 77, with 1024 the same).
constexpr int64_t kOwnGroups = 2048;
// Rows of a group and kv head, on average, up to which the reading is what bounds it: 64 to each of 4 groups over 8192
// tokens 43 us either way, 32 to each 32 instead of 39 by tiles of 128, 128 to each 62 instead of 56.
constexpr int64_t kFewRows = 64;
constexpr int32_t kMostGroups = 1 << 24;
// Workgroups over shared keys beside those over own ones, of the 512 that the device holds at once: 192 agents with 500 to
// 8000 own tokens 452, 460, 461, 478 us with 256, 320, 384, 512 of them (492 one after the other, tiles of 256 rows first);
// 256 sequences in 4 groups with 16 own tokens 95, 99, 90, 87 (103).
constexpr int64_t kBothGroups = 384;
// A row is joined by a workgroup of 16 wavefronts where it may have this many parts of its own, or where rows are this few
// (two sequences of 40 heads, 40 parts to a row: 6.3 us, with a wavefront to a row 8.7), else by one wavefront.
constexpr int32_t kManyParts = 32;
constexpr int64_t kFewJoins = 512;

Plan plan_for(const peek_kv_pool& pool, int32_t n, int32_t q_heads, int32_t max_blocks, int32_t groups) {
  Plan p{};
  const int32_t group = q_heads / pool.kv_heads;
  const int64_t tokens = std::max<int64_t>(1, (int64_t)max_blocks * pool.block_size);
  const int64_t all_rows = (int64_t)n * group;                              // of a kv head
  const int64_t rows_each = groups > 0 ? all_rows / groups : 0;
  p.few = groups > 0 && pool.block_size >= 16 && rows_each <= kFewRows;
  // (tiles of 16 rows where groups have 8 or fewer on average and are as uneven as queues are, or where only own keys
  // go this way: two users of 4 heads each 17.9 us instead of 20.9 by tiles of 32)
  p.own_rows = pool.block_size >= 16 && ((p.few && rows_each > 8) || group > 16) ? 32 : 16;
  p.tile_rows = p.few ? p.own_rows : 32 * kWaves;
  const int64_t tiles = all_rows / p.tile_rows + groups;                    // no more than these
  p.pieces = (int32_t)std::max<int64_t>(1, (!p.few && pool.block_size >= 16 ? kBothGroups : 512) / pool.kv_heads);
  p.slots = (int32_t)(p.pieces + tiles);
  p.slot_rows = (int32_t)std::min<int64_t>(p.tile_rows, all_rows);
  int64_t chunk = 256;
  const int64_t units = (int64_t)n * pool.kv_heads * ((group + p.own_rows - 1) / p.own_rows);
  while (chunk < kMaxChunk && units * ((tokens + chunk - 1) / chunk) > kOwnGroups) chunk *= 2;
  p.own_chunk = (int32_t)chunk;
  p.own_splits = (int32_t)((tokens + chunk - 1) / chunk);
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t parts = (size_t)n * q_heads * p.own_splits;
  size_t at = up(parts * pool.head_dim * sizeof(float));
  p.part_lse = at;
  at = up(at + parts * sizeof(float));
  if (groups > 0) {
    const size_t rows = (size_t)pool.kv_heads * p.slots * p.slot_rows;
    p.prefix_out = at;
    at = up(at + rows * pool.head_dim * sizeof(float));
    p.prefix_lse = at;
    at = up(at + rows * sizeof(float));
    p.first_step = at;
    at = up(at + ((size_t)groups + 1) * sizeof(int64_t));
    p.first_tile = at;
    at = up(at + (size_t)groups * sizeof(int32_t));
  }
  p.bytes = at;
  return p;
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

size_t peek_shared_decode_attention_workspace(const peek_kv_pool* pool, int32_t n, int32_t q_heads, int32_t max_blocks,
                                              int32_t groups) {
  Pool p;
  if (n < 0 || groups < 0 || groups >= kMostGroups || q_heads < 1 || max_blocks < 0 || check_pool(pool, &p) != PEEK_OK || q_heads % p.heads != 0)
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
    if (groups >= kMostGroups) return fail(PEEK_ERR_INVALID_ARGUMENT, "too many groups for one call (%d)", groups);
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
    const int64_t prefix_groups = groups > 0 ? (int64_t)p.pieces * a.pool.heads : 0;
    const int32_t own_rows = p.own_rows;
    const int64_t own_groups = (int64_t)n * ((a.group + own_rows - 1) / own_rows) * a.pool.heads * p.own_splits;
    // a workgroup to a row where rows are few or may have many parts of their own
    const bool many = p.own_splits >= kManyParts || (groups > 0 && (int64_t)n * q_heads <= kFewJoins);
    const int64_t joins = ((int64_t)n * q_heads + (many ? 0 : kWaves - 1)) / (many ? 1 : kWaves);
    // (launches have fewer than 2^32 threads; blocks of 16 or more: shared keys' workgroups are beside the own ones)
    const int64_t beside = pool->block_size >= 16 ? prefix_groups : 0;
    if (own_groups + beside >= (1 << 24) || joins * (many ? 1024 : kThreads) >= (int64_t)1 << 32)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many sequences for one call (%d)", n);
    hipStream_t st = (hipStream_t)stream;
    a.q = Rows{d_q, q_token_stride, q_head_stride};
    a.context = d_context;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.members = d_members;
    a.group_offsets = d_group_offsets;
    a.shared = d_shared;
    if ((s = validate_shared(a, st)) != PEEK_OK) return s;
    a.out = (uint16_t*)d_out;
    a.out_token = out_token_stride;
    a.out_head = out_head_stride;
    a.lse = d_lse;
    char* ws = (char*)d_workspace;
    a.part_out = (float*)ws;
    a.part_lse = (float*)(ws + p.part_lse);
    a.prefix_out = (float*)(ws + p.prefix_out);
    a.prefix_lse = (float*)(ws + p.prefix_lse);
    a.first_step = (int64_t*)(ws + p.first_step);
    a.first_tile = (int32_t*)(ws + p.first_tile);
    a.own_chunk = p.own_chunk;
    a.splits = p.own_splits;
    a.pieces = p.pieces;
    a.slots = p.slots;
    a.slot_rows = p.slot_rows;
    a.tile_rows = p.tile_rows;
    a.step_keys = p.few ? kFewKeys : kKeys;
    set_scale(scale, &a.scale, &a.q_flip, &a.q_mask);
    with_types(type, pool->type, pool->head_dim, [&](auto t, auto m, auto d) {
      const bool both = prefix_groups > 0 && !p.few && a.pool.log_block >= 4;
      if (prefix_groups > 0 && !p.few && !both)
        hipLaunchKernelGGL((k_shared_tiles<t(), m(), d()>), dim3((unsigned)prefix_groups), dim3(kThreads), 0, st, a);
      const uint32_t first = p.few || both ? (uint32_t)prefix_groups : 0u;
      auto go = [&](auto kernel, auto... more) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)own_groups + first), dim3(kThreads), 0, st, a, more...);
      };
      if (a.pool.log_block < 4) go(k_shared_own<t(), m(), d()>);
      else if (both && own_rows == 32) go(k_shared_both<t(), m(), d(), 2>, first);
      else if (both) go(k_shared_both<t(), m(), d(), 1>, first);
      else if (own_rows == 32) go(k_shared_stream<t(), m(), d(), 2>, first);
      else go(k_shared_stream<t(), m(), d(), 1>, first);
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
