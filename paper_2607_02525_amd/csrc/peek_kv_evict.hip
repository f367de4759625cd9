// Evicting the blocks of a sequence that attention hardly reads, on gfx950.
//
// A block's score is the sum of its masses over the kv heads. Scores become
// keys whose unsigned order is theirs; three counting passes of 11, 11 and 10 bits
// find the key of the last block to go. The blocks below it go, and the first
// `equal` of those that equal it, so the number gone before a block is (lower
// keys before it) + min(equal keys before it, equal): one sum over the blocks in
// order places them all, without a sort.
//
// Bound by the longest table's one workgroup, which scores, selects and moves all of
// it: 192 tables of 250 to 8125 blocks of 8 heads, 59 MB, 42 us, 32 where the masses
// are in the cache already (a copy of as much memory takes 12); by the passes' waits
// where tables are short: 64 of up to 463 blocks 8.6 us.
#include <algorithm>

#include "peek_internal.h"
#include "peek_kv.h"

namespace peek {

using kv::Table;

namespace {

constexpr int kWave = 64;
constexpr int32_t kMaxGridY = 65535;
constexpr int kBins = 2048;
// A table of up to kLdsTable blocks has one workgroup, its keys in LDS: 256 threads
// up to kSmallTable (1500 tables of up to 500 blocks 17 us, with 1024 threads 41; 64
// of up to 1875 blocks 16.5 us, with 1024 threads 11). A wider one is spread
// over workgroups, with one for the passes between scores and move (three tables of up
// to 32500 blocks 37 us, with a workgroup each 112; of up to 8000 blocks 22 either
// way, of up to 4000 14 with one workgroup and 20 spread).
constexpr int32_t kSmallTable = 1024;
constexpr int32_t kLdsTable = 8192;
constexpr int kPart = 1024;                 // blocks of a workgroup that scores or moves
constexpr int kPartThreads = kPart / 4;
constexpr int32_t kPartHeads = 8;           // heads of a workgroup that moves
constexpr int kSelectThreads = 1024;

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f4_unaligned __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

struct Evict {
  Table table;
  const int32_t* context;
  const float* mass;
  const int32_t* keep;
  int32_t* context_out;
  int32_t* table_out;
  float* mass_out;
  int32_t* freed;
  int32_t* num_freed;
  int32_t heads, log_block, sink, recent;
  // wide tables: keys [n][stride], counts of lower and equal keys before every
  // part [n][parts], and what the passes found [n]
  uint32_t* keys;
  int2* before;
  struct Found* found;
  int64_t stride;
  int32_t parts, head_groups, n;
};

// The candidates [lo, hi) of a sequence and how many of them go.
struct Range {
  int32_t lo, hi, drop;
};

// What the passes over the keys find: the key of the last block to go and how
// many of that key go. (The context may be overwritten by the kernel that
// moves, so the range is kept with it.)
struct Found {
  Range range;
  uint32_t last;
  int32_t equal;
};
__device__ __forceinline__ Range range_of(const Evict& a, int32_t r) {
  const int32_t tokens = kv::clip_tokens(a.context[r], a.table.width, a.log_block);
  const int32_t nb = (int32_t)(((int64_t)tokens + (1 << a.log_block) - 1) >> a.log_block);
  const int32_t lo = min(a.sink, nb), hi = (int32_t)max((int64_t)lo, (int64_t)nb - a.recent);
  return Range{lo, hi, (int32_t)min((int64_t)(hi - lo), max((int64_t)0, (int64_t)nb - max(0, a.keep[r])))};
}

__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);   // -0 counts as 0
  return (u >> 31) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kZeroKey = 0x80000000u;

// Four masses; a row of them begins at any multiple of 4 bytes.
__device__ __forceinline__ f4 load4(const float* __restrict__ p, int32_t at, int32_t end) {
  if (at + 4 <= end) return *(const f4_unaligned*)(p + at);
  f4 x = {};
  for (int i = 0; i < 3; ++i)
    if (at + i < end) x[i] = p[at + i];
  return x;
}

// Scores of blocks b .. b + 3: heads in ascending order, eight loads at a time.
__device__ __forceinline__ f4 scores(const float* __restrict__ m, int32_t heads, int32_t width, int32_t b) {
  f4 s = load4(m, b, width);
  int32_t h = 1;
  for (; h + 8 <= heads; h += 8) {
    f4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = load4(m + (int64_t)(h + i) * width, b, width);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i];
  }
#pragma unroll 7
  for (; h < heads; ++h) s += load4(m + (int64_t)h * width, b, width);
  return s;
}

// Exclusive sum over the workgroup of two counts at once; *total gets the wholes.
template <int THREADS>
__device__ __forceinline__ int2 group_sum(int2 x, int2* s_part, int2* total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int2 inc = x;
  for (int d = 1; d < kWave; d <<= 1) {
    const int a = __shfl_up(inc.x, d), b = __shfl_up(inc.y, d);
    if (lane >= d) {
      inc.x += a;
      inc.y += b;
    }
  }
  if (lane == kWave - 1) s_part[wave] = inc;
  __syncthreads();
  int2 before{0, 0}, all{0, 0};
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) {
    const int2 p = s_part[w];
    if (w < wave) {
      before.x += p.x;
      before.y += p.y;
    }
    all.x += p.x;
    all.y += p.y;
  }
  __syncthreads();
  *total = all;
  return int2{before.x + inc.x - x.x, before.y + inc.y - x.y};
}

template <int THREADS>
struct Select {
  int32_t count[kBins];
  int2 part[THREADS / kWave];
  uint32_t prefix;
  int32_t left;
};

// The key of the last of `drop` (> 0) blocks to go and how many of that key
// go. each(f) calls f with every candidate's key of this thread; keys of 0, which
// blocks that nothing has looked at share, are counted by the wavefront.
template <int THREADS, typename EACH>
__device__ __forceinline__ void select(Select<THREADS>& s, int32_t drop, EACH&& each, uint32_t* last, int32_t* equal) {
  const int t = threadIdx.x, lane = t & (kWave - 1);
  if (t == 0) {
    s.prefix = 0;
    s.left = drop;
  }
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int32_t i = t; i < kBins; i += THREADS) s.count[i] = 0;
    __syncthreads();
    const uint32_t prefix = s.prefix, above = pass == 0 ? 0u : 0xffffffffu << (shift + bits);
    const int32_t left = s.left;
    each([&](uint32_t k) {
      const bool here = (k & above) == prefix;
      if (here && k != kZeroKey) atomicAdd(&s.count[(k >> shift) & ((1 << bits) - 1)], 1);
      const uint64_t zeros = __ballot(here && k == kZeroKey);
      if (zeros != 0 && lane == __ffsll((unsigned long long)zeros) - 1)
        atomicAdd(&s.count[(kZeroKey >> shift) & ((1 << bits) - 1)], __popcll(zeros));
    });
    __syncthreads();
    constexpr int kEach = kBins / THREADS;
    int32_t c[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += c[i] = s.count[t * kEach + i];
    int2 all;
    int32_t before = group_sum<THREADS>(int2{sum, 0}, s.part, &all).x;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (before < left && left <= before + c[i]) {
        s.prefix = prefix | ((uint32_t)(t * kEach + i) << shift);
        s.left = left - before;
      }
      before += c[i];
    }
    __syncthreads();
  }
  *last = s.prefix;
  *equal = s.left;
}

__device__ __forceinline__ int2 votes(const Range& g, int32_t b, uint32_t k, uint32_t last) {
  const bool able = g.drop > 0 && b >= g.lo && b < g.hi;
  return int2{(int)__popcll(__ballot(able && k < last)), (int)__popcll(__ballot(able && k == last))};
}

// This wavefront's run of 64-block segments from block b0 on: place[i] of block
// b0 + i becomes where it moves to, -1 if it goes (then its page is listed
// in `freed`, unless another workgroup does that). `mine` counts the lower and the
// equal keys before b0.
template <typename KEY>
__device__ __forceinline__ void find_places(const Evict& a, int32_t r, int32_t b0, int32_t segments, const Range& g,
                                            uint32_t last, int32_t equal, int2 mine, bool list, KEY&& key,
                                            int32_t* place) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int32_t seg = 0; seg < segments; ++seg) {
    const int32_t i = seg * kWave + lane, b = b0 + i;
    const bool able = g.drop > 0 && b >= g.lo && b < g.hi;
    const uint32_t k = able ? key(b) : 0xffffffffu;
    const uint64_t lower = __ballot(able && k < last), same = __ballot(able && k == last);
    const uint64_t under = ((uint64_t)1 << lane) - 1;
    const int32_t ties = mine.y + __popcll(same & under);
    const int32_t gone = mine.x + __popcll(lower & under) + min(ties, equal);
    const bool goes = ((lower >> lane) & 1) || (((same >> lane) & 1) && ties < equal);
    if (b < a.table.width) {
      if (goes && list) a.freed[(int64_t)r * a.table.width + gone] = a.table.ids[(int64_t)r * a.table.stride + b];
      place[i] = goes ? -1 : b - gone;
    }
    mine.x += __popcll(lower);
    mine.y += __popcll(same);
  }
}

// Blocks [b0, b1) of a sequence to their places, place[b - b0]: the table's entries
// (`ids`) and the masses of heads [h0, h1). What is left of a row past what stays
// (the last `drop` columns), and of the list past what went, is filled.
template <int THREADS>
__device__ __forceinline__ void move(const Evict& a, int32_t r, int32_t b0, int32_t b1, int32_t h0, int32_t h1,
                                     bool ids, int32_t drop, const int32_t* place) {
  const int32_t width = a.table.width;
  const float* m = a.mass + (int64_t)r * a.heads * width;
  float* out_mass = a.mass_out + (int64_t)r * a.heads * width;
  int32_t* out_ids = a.table_out + (int64_t)r * width;
  for (int32_t b = b0 + (int32_t)threadIdx.x; b < b1; b += THREADS) {
    const int32_t to = place[b - b0];
    if (to >= 0) {
      if (ids) out_ids[to] = a.table.ids[(int64_t)r * a.table.stride + b];
      int32_t h = h0;
      for (; h + 8 <= h1; h += 8) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = m[(int64_t)(h + i) * width + b];
#pragma unroll
        for (int i = 0; i < 8; ++i) out_mass[(int64_t)(h + i) * width + to] = x[i];
      }
      for (; h < h1; ++h) out_mass[(int64_t)h * width + to] = m[(int64_t)h * width + b];
    }
    if (ids && b >= drop) a.freed[(int64_t)r * width + b] = -1;
    if (b >= width - drop) {
      if (ids) out_ids[b] = -1;
      for (int32_t h = h0; h < h1; ++h) out_mass[(int64_t)h * width + b] = 0.0f;
    }
  }
}

// ------------------------------------------------------- one workgroup each
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_evict_one(Evict a) {
  constexpr int kWaves = THREADS / kWave;
  extern __shared__ uint32_t s_key[];        // a multiple of 64 of them; places later
  __shared__ Select<THREADS> s_select;
  __shared__ int2 s_wave[kWaves];
  const int32_t r = blockIdx.x, t = threadIdx.x, width = a.table.width;
  const int lane = t & (kWave - 1), wave = t / kWave;
  const int32_t ctx = kv::clip_tokens(a.context[r], width, a.log_block);
  const Range g = range_of(a, r);
  uint32_t last = 0;
  int32_t equal = 0;
  if (g.drop > 0) {
    for (int32_t b = (g.lo & ~3) + 4 * t; b < g.hi; b += 4 * THREADS) {
      const f4 s = scores(a.mass + (int64_t)r * a.heads * width, a.heads, width, b);
      *(u4*)(s_key + b) = (u4){score_key(s[0]), score_key(s[1]), score_key(s[2]), score_key(s[3])};
    }
    __syncthreads();
    select<THREADS>(s_select, g.drop, [&](auto f) {
      for (int32_t b = g.lo + t; b < g.hi; b += THREADS) f(s_key[b]);
    }, &last, &equal);
  }
  const int32_t segments = (width + kWave - 1) / kWave, each = (segments + kWaves - 1) / kWaves;
  const int32_t seg0 = min(segments, wave * each), seg1 = min(segments, seg0 + each);
  int2 mine{0, 0};
  for (int32_t seg = seg0; seg < seg1; ++seg) {
    const int32_t b = seg * kWave + lane;
    const int2 v = votes(g, b, s_key[b], last);
    mine.x += v.x;
    mine.y += v.y;
  }
  if (lane == 0) s_wave[wave] = mine;
  __syncthreads();
  mine = int2{0, 0};
  for (int w = 0; w < wave; ++w) {
    mine.x += s_wave[w].x;
    mine.y += s_wave[w].y;
  }
  find_places(a, r, seg0 * kWave, seg1 - seg0, g, last, equal, mine, true, [&](int32_t b) { return s_key[b]; },
              (int32_t*)s_key + seg0 * kWave);
  __syncthreads();
  move<THREADS>(a, r, 0, width, 0, a.heads, true, g.drop, (const int32_t*)s_key);
  if (t == 0) {
    a.num_freed[r] = g.drop;
    a.context_out[r] = ctx - (g.drop << a.log_block);
  }
}

// ------------------------------------------------------------- wide tables
__global__ __launch_bounds__(kPartThreads) void k_evict_score(Evict a) {
  const int32_t b = (int32_t)blockIdx.x * kPart + 4 * (int32_t)threadIdx.x;
  for (int32_t r = blockIdx.y; r < a.n; r += (int32_t)gridDim.y) {
    const Range g = range_of(a, r);
    if (g.drop == 0 || b >= g.hi || b + 3 < g.lo) continue;
    const f4 s = scores(a.mass + (int64_t)r * a.heads * a.table.width, a.heads, a.table.width, b);
    *(u4*)(a.keys + r * a.stride + b) = (u4){score_key(s[0]), score_key(s[1]), score_key(s[2]), score_key(s[3])};
  }
}

__global__ __launch_bounds__(kSelectThreads) void k_evict_select(Evict a) {
  constexpr int kWaves = kSelectThreads / kWave;
  __shared__ Select<kSelectThreads> s_select;
  const int32_t r = blockIdx.x, t = threadIdx.x, lane = t & (kWave - 1), wave = t / kWave;
  const Range g = range_of(a, r);
  uint32_t last = 0;
  int32_t equal = 0;
  if (g.drop > 0) {
    const uint32_t* keys = a.keys + r * a.stride;
    select<kSelectThreads>(s_select, g.drop, [&](auto f) {
      for (int32_t b = (g.lo & ~3) + 4 * t; b < g.hi; b += 4 * kSelectThreads) {
        const u4 k = *(const u4*)(keys + b);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (b + i >= g.lo && b + i < g.hi) f(k[i]);
      }
    }, &last, &equal);
    // counts of every part, a wavefront to a part, and their sums in order
    int2* before = a.before + (int64_t)r * a.parts;
    int2 carry{0, 0};
    for (int32_t p0 = 0; p0 < a.parts; p0 += kSelectThreads) {
      for (int32_t p = p0 + wave; p < min(a.parts, p0 + kSelectThreads); p += kWaves) {
        u4 k[kPart / kWave / 4];
#pragma unroll
        for (int i = 0; i < kPart / kWave / 4; ++i) {
          const int32_t b = p * kPart + 4 * (i * kWave + lane);
          k[i] = b < g.hi && b + 3 >= g.lo ? *(const u4*)(keys + b) : (u4){};
        }
        int2 mine{0, 0};
#pragma unroll
        for (int i = 0; i < kPart / kWave / 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int2 v = votes(g, p * kPart + 4 * (i * kWave + lane) + e, k[i][e], last);
            mine.x += v.x;
            mine.y += v.y;
          }
        if (lane == 0) before[p] = mine;
      }
      __syncthreads();
      const int2 mine = p0 + t < a.parts ? before[p0 + t] : int2{0, 0};
      int2 all;
      const int2 sum = group_sum<kSelectThreads>(mine, s_select.part, &all);
      if (p0 + t < a.parts) before[p0 + t] = int2{carry.x + sum.x, carry.y + sum.y};
      carry.x += all.x;
      carry.y += all.y;
    }
  }
  if (t == 0) a.found[r] = Found{g, last, equal};
}

// A workgroup moves one part of a row for kPartHeads heads.
__global__ __launch_bounds__(kPartThreads) void k_evict_move(Evict a) {
  constexpr int kWaves = kPartThreads / kWave, kSegments = kPart / kWave / kWaves;
  __shared__ int2 s_wave[kWaves];
  __shared__ int32_t s_place[kPart];
  const int32_t part = (int32_t)blockIdx.x / a.head_groups, group = (int32_t)blockIdx.x % a.head_groups;
  const int32_t t = threadIdx.x, lane = t & (kWave - 1), wave = t / kWave;
  const int32_t b0 = part * kPart, mine0 = wave * kSegments * kWave;
  const int32_t h0 = group * kPartHeads, h1 = min(a.heads, h0 + kPartHeads);
  for (int32_t r = blockIdx.y; r < a.n; r += (int32_t)gridDim.y) {
    const Found found = a.found[r];
    const Range g = found.range;
    const uint32_t* keys = a.keys + r * a.stride;
    int2 mine = g.drop > 0 ? a.before[(int64_t)r * a.parts + part] : int2{0, 0};
    int2 own{0, 0};
#pragma unroll
    for (int i = 0; i < kSegments; ++i) {
      const int32_t b = b0 + mine0 + i * kWave + lane;
      const int2 v = votes(g, b, g.drop > 0 && b >= g.lo && b < g.hi ? keys[b] : 0u, found.last);
      own.x += v.x;
      own.y += v.y;
    }
    if (lane == 0) s_wave[wave] = own;
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
      mine.x += s_wave[w].x;
      mine.y += s_wave[w].y;
    }
    find_places(a, r, b0 + mine0, kSegments, g, found.last, found.equal, mine, group == 0,
                [&](int32_t b) { return keys[b]; }, s_place + mine0);
    __syncthreads();
    move<kPartThreads>(a, r, b0, min(a.table.width, b0 + kPart), h0, h1, group == 0, g.drop, s_place);
    __syncthreads();
    if (blockIdx.x == 0 && t == 0) {
      a.num_freed[r] = g.drop;
      a.context_out[r] = kv::clip_tokens(a.context[r], a.table.width, a.log_block) - (g.drop << a.log_block);
    }
  }
}

// Scratch of a call on wide tables, in bytes from its beginning.
struct Scratch {
  size_t before, found, total;
  int64_t stride;
  int32_t parts;
};
Scratch scratch_of(int32_t n, int32_t max_blocks) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  Scratch s;
  s.stride = ((int64_t)max_blocks + 3) & ~(int64_t)3;
  s.parts = (max_blocks + kPart - 1) / kPart;
  s.before = up((size_t)n * s.stride * sizeof(uint32_t));
  s.found = s.before + up((size_t)n * s.parts * sizeof(int2));
  s.total = s.found + up((size_t)n * sizeof(Found));
  return s;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na > 0 && nb > 0 && x < y + nb && y < x + na;
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

size_t peek_kv_evict_workspace(int32_t n, int32_t kv_heads, int32_t max_blocks) {
  if (n < 0 || kv_heads < 1 || max_blocks <= kLdsTable) return 0;
  return scratch_of(n, max_blocks).total;
}

peek_status peek_kv_evict(int32_t n, int32_t kv_heads, int32_t block_size, const int32_t* d_context,
                          const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, const float* d_mass,
                          const int32_t* d_keep, int32_t sink, int32_t recent, int32_t* d_context_out,
                          int32_t* d_table_out, float* d_mass_out, int32_t* d_freed, int32_t* d_num_freed,
                          void* d_workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> peek_status {
    clear_error();
    if (n < 0 || n >= (1 << 22)) return fail(PEEK_ERR_INVALID_ARGUMENT, "n must be in [0, 2^22) (got %d)", n);
    if (kv_heads < 1 || kv_heads > 1024)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "kv_heads must be in [1, 1024] (got %d)", kv_heads);
    if (block_size < 4 || block_size > 256 || (block_size & (block_size - 1)) != 0)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "block_size must be a power of two in [4, 256] (got %d)", block_size);
    if (sink < 0 || recent < 1)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "sink must be >= 0 and recent >= 1 (got %d, %d)", sink, recent);
    peek_status s = check_table(d_block_table, max_blocks, table_stride, block_size);
    if (s != PEEK_OK) return s;
    if (n == 0) return PEEK_OK;
    if (!d_context || !d_keep || !d_context_out || !d_num_freed)
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_context, d_keep, d_context_out and d_num_freed must not be NULL");
    if (max_blocks > 0 && (!d_mass || !d_table_out || !d_mass_out || !d_freed))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "d_mass, d_table_out, d_mass_out and d_freed must not be NULL");
    const size_t row = (size_t)n * max_blocks * 4, in_row = ((size_t)(n - 1) * table_stride + max_blocks) * 4;
    if (overlap(d_table_out, row, d_block_table, in_row) || overlap(d_freed, row, d_block_table, in_row) ||
        overlap(d_mass_out, row * kv_heads, d_mass, row * kv_heads))
      return fail(PEEK_ERR_INVALID_ARGUMENT,
                  "the outputs must not overlap the table and the masses they are made from");
    const size_t need = peek_kv_evict_workspace(n, kv_heads, max_blocks);
    s = check_workspace(d_workspace, workspace_bytes, need);
    if (s != PEEK_OK) return s;
    // every array that is written against every other, in place of which only the context may be
    const struct {
      const void* at;
      size_t bytes;
    } arrays[] = {{d_context_out, (size_t)n * 4}, {d_table_out, row}, {d_mass_out, row * kv_heads}, {d_freed, row},
                  {d_num_freed, (size_t)n * 4}, {d_workspace, need},
                  {d_context, (size_t)n * 4}, {d_block_table, in_row}, {d_mass, row * kv_heads}, {d_keep, (size_t)n * 4}};
    constexpr int kWritten = 6, kContextOut = 0, kContext = 6;
    for (int i = 0; i < kWritten; ++i)
      for (int j = i + 1; j < (int)(sizeof(arrays) / sizeof(arrays[0])); ++j)
        if (!(i == kContextOut && j == kContext && d_context_out == d_context) &&
            overlap(arrays[i].at, arrays[i].bytes, arrays[j].at, arrays[j].bytes))
          return fail(PEEK_ERR_INVALID_ARGUMENT, "the outputs must not overlap each other, the inputs or the workspace");
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, nullptr, 0, d_context, false, d_block_table, max_blocks, table_stride, block_size, nullptr, st);
    if (s != PEEK_OK) return s;
    Evict a{Table{d_block_table, table_stride, max_blocks}, d_context, d_mass, d_keep, d_context_out, d_table_out,
            d_mass_out, d_freed, d_num_freed, kv_heads, __builtin_ctz((unsigned)block_size), sink, recent};
    a.n = n;
    if (max_blocks <= kLdsTable) {
      auto go = [&](auto kernel, int threads) {
        const size_t lds = (((size_t)max_blocks + kWave - 1) & ~(size_t)(kWave - 1)) * sizeof(uint32_t);
        hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(threads), lds, st, a);
      };
      if (max_blocks <= kSmallTable) go(k_evict_one<256>, 256);
      else go(k_evict_one<1024>, 1024);
    } else {
      const Scratch w = scratch_of(n, max_blocks);
      char* base = (char*)d_workspace;
      a.keys = (uint32_t*)base;
      a.before = (int2*)(base + w.before);
      a.found = (Found*)(base + w.found);
      a.stride = w.stride;
      a.parts = w.parts;
      a.head_groups = (kv_heads + kPartHeads - 1) / kPartHeads;
      const unsigned rows = (unsigned)std::min(n, kMaxGridY);
      hipLaunchKernelGGL(k_evict_score, dim3((unsigned)w.parts, rows), dim3(kPartThreads), 0, st, a);
      hipLaunchKernelGGL(k_evict_select, dim3((unsigned)n), dim3(kSelectThreads), 0, st, a);
      hipLaunchKernelGGL(k_evict_move, dim3((unsigned)(w.parts * a.head_groups), rows), dim3(kPartThreads), 0, st, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(PEEK_ERR_DEVICE, "eviction launch failed: %s", hipGetErrorString(e));
    return PEEK_OK;
  });
}

}  // extern "C"
