// Attention of packed prompts after their cached prefixes, on gfx950.
//
// One workgroup of eight wavefronts takes 256 rows of one kv head of one
// sequence, a row being a (token, query head of the group) pair in that
// order, so that a few new tokens of a wide group still fill a tile and every
// row of it shares the keys. It goes over the keys in tiles of 64, first the
// cached prefix, then the sequence's own tokens up to its last row, and keeps a
// running reference and sum of every row's softmax (one pass over the keys).
//
// A wavefront has 32 rows. K times Q^T leaves lane l with keys of row l % 32
// alone: its maximum and sum need one exchange with the lane 32 away,
// and its weights are already the operand of V^T times weights (peek_mfma.h).
// K and V tiles lie in LDS as 16-bit rows, two buffers of each; 16-byte
// pieces of a row are permuted by the row's number so that reads down a
// column of rows spread over the banks. V is read by transposing loads.
//
// Own tokens go from memory to LDS directly. Cached codes are widened to 16
// bits on the way, which is exact, and their scales never touch them: K's
// multiplies the logit, and V's goes into the weight as an exponent,
//   w_j s_j = 2^(x_j + log2 s_j - m),   sum of weights = sum_j (w_j s_j) / s_j,
// with m near the maximum of x_j + log2 s_j so far, or here (peek_mfma.h), so weights times
// scales stay within the range of either 16-bit type.
//
// Rows and keys past the end: rows are clamped to the last one and not
// stored; keys are clamped to the last one and masked, so nothing outside the
// sequence is read.
//
// Bound, over own tokens, by the power that the products draw: 5 prompts of
// up to 24000 tokens, 32 query heads of 128, 4.98 TFLOP: 4.35 to 4.55 ms, 1.1
// PFLOP/s (a library product of 8192^3 reaches 1.24), the clock held at 1.8 to
// 1.9 of 2.4 GHz, the matrix cores busy 55% of the cycles.
// Over cached tokens by the vector instructions, which widen the codes too (8.7 to each
// matrix instruction, four cycles each to its 32), and by the last workgroups:
// 64 queries of up to 256 tokens after up to 7168, 40 query heads, 1.07 TFLOP:
// 1.38 to 1.42 ms, 760 TFLOP/s. Few rows by the 2 us that 64 keys take a workgroup.
// With 128 rows to a workgroup, two to a compute unit, tiles are loaded twice as
// often (467 TFLOP/s where 256 rows had 716); two groups of wavefronts a phase
// apart gained 3% on the first and lost 9% on the second.
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
constexpr int kWaves = 8;
constexpr int kThreads = kWave * kWaves;
constexpr int kRows = 32 * kWaves;    // rows of a tile
constexpr int64_t kTargetGroups = 256;   // of tiles in parts: 128 take 81 us where 256 take 50, 512 the same
constexpr int32_t kCounted = kWave;   // sequences, at most, whose tiles are counted

struct Prefill {
  Pool pool;
  Rows q, k, v;
  const int64_t* offsets;
  const int32_t* prefix;
  Table table;
  uint16_t* out;
  int64_t out_token, out_head;
  float* lse;
  float* part_out;                    // [rows][splits][D]: a part's sum of weight * value / its sum of weights
  float* part_lse;                    // [rows][splits]: base-2 logarithm of its sum of weights, -infinity for none
  int64_t num_tokens;
  int32_t n, group, kv_heads;
  int32_t splits;                     // room for parts of a row
  float scale;                        // of logits, in powers of two: >= 0
  uint32_t q_flip;                    // sign bits to flip in q, where the caller's scale is negative
  uint32_t q_mask;                    // 0 where the caller's scale is 0
};

// Each lane's 16 bytes at `base` + its offset to LDS at `to` + 16 * lane, base
// and `to` the same for the wavefront. Written out because the builtin makes
// every later LDS read wait for the load, the reads of the other buffer
// included. Done when vmcnt says so; no vector register is written. (m0 is
// reserved: the compiler keeps nothing there.)
__device__ __forceinline__ void to_lds(const uint16_t* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base)
               : "memory");
}

// Waits for them, and for this wavefront's other loads: the builtin, so that the
// compiler knows it and waits for none of these again in a loop.
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0), the other counters as they are
  asm volatile("" ::: "memory");
}

// Tiles of sequence i's rows; 0 where its offsets are none.
__device__ __forceinline__ uint32_t tiles_of(const Prefill& a, int32_t i) {
  const int64_t first = a.offsets[i], end = min(a.num_tokens, a.offsets[i + 1]);
  return first < 0 || end <= first ? 0u : (uint32_t)(((end - first) * a.group + kRows - 1) / kRows);
}

// Parts that every tile's keys are split into: as many as leave a workgroup to a compute unit.
__device__ __forceinline__ int32_t parts_for(const Prefill& a, uint32_t tiles) {
  const uint32_t groups = min(tiles, (uint32_t)kTargetGroups) * (uint32_t)a.kv_heads;
  return max(1, min(a.splits, (int32_t)((uint32_t)kTargetGroups / max(1u, groups))));
}

// A workgroup's tile: of sequence r, from row row0 on, its part of the keys.
struct Work {
  int32_t r, split, parts;
  int64_t row0;
};

// Tiles of up to kCounted sequences: *mine is lane i's sequence's, the result those of the first to the i-th.
__device__ __forceinline__ uint32_t count_tiles(const Prefill& a, int lane, uint32_t* mine) {
  uint32_t sum = *mine = lane < a.n ? tiles_of(a, lane) : 0u;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint32_t x = __shfl_up(sum, d);
    if (lane >= d) sum += x;
  }
  return sum;
}

// Work `unit` from the end: the last rows of the last sequences come first, they
// have the most keys. Up to kCounted sequences the tiles are counted, so that
// workgroups without work are the last ones: among the others, dealt out in turn over the
// shader engines, they left some of these with twice the work of others (16
// prompts of one tile each after 8000 tokens 259 -> 186 us, 64 chats 364 -> 353).
// More sequences would cost each workgroup more than that saves (250 short prompts 230
// -> 241 us, 1000 0.90 -> 1.28 ms): they have a slot for each tile and one
// more, numbered without counting, sequence r's from offsets[r] * group / kRows + r on.
__device__ __forceinline__ bool find_work(const Prefill& a, uint32_t unit, uint32_t units, int lane, Work* w) {
  if (a.n > kCounted) {
    const int64_t slot = units - 1 - unit;
    w->r = kv::last_at_most(a.n, slot, lane, [&](int32_t i) { return a.offsets[i] * a.group / kRows + i; });
    w->row0 = (slot - (a.offsets[w->r] * a.group / kRows + w->r)) * kRows;
    w->split = 0;
    w->parts = 1;
    return true;
  }
  uint32_t mine;
  const uint32_t sum = count_tiles(a, lane, &mine), tiles = __builtin_amdgcn_readlane(sum, kWave - 1);
  w->parts = parts_for(a, tiles);
  if (unit >= tiles * (uint32_t)w->parts) return false;
  const uint32_t from_first = tiles * w->parts - 1 - unit, slot = from_first / w->parts;
  w->split = from_first % w->parts;
  const uint64_t past = __ballot(sum > slot);
  if (past == 0) return false;
  w->r = __builtin_ctzll(past);
  w->row0 = (int64_t)(slot - (uint32_t)__builtin_amdgcn_readlane(sum - mine, w->r)) * kRows;
  return true;
}

template <int TYPE, int FMT, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_prefill(Prefill a) {
  using T = Tile<TYPE, FMT, D, kWaves>;
  __shared__ __attribute__((aligned(1024))) uint8_t s_k[2][T::kBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t s_v[2][T::kBytes];
  __shared__ f4 s_scale[2][kKeys / 4];
  __shared__ uint32_t s_odd;

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // kv heads side by side: each on XCDs of its own where there are eight
  const int32_t head = blockIdx.x % a.kv_heads;
  Work w;
  if (!find_work(a, blockIdx.x / a.kv_heads, gridDim.x / a.kv_heads, lane, &w)) return;
  const int32_t r = __builtin_amdgcn_readfirstlane(w.r), split = w.split;
  const int64_t row0 = w.row0, first = a.offsets[r], end = min(a.num_tokens, a.offsets[r + 1]);
  if (first < 0 || end <= first || row0 < 0 || row0 >= (end - first) * a.group) return;
  const int64_t rows = (end - first) * a.group;
  const int32_t held = a.prefix ? kv::clip_tokens(a.prefix[r], a.table.width, a.pool.log_block) : 0;
  const int32_t cached = (int32_t)(((uint32_t)held + kKeys - 1) / kKeys);
  const int32_t last_row_token = (int32_t)((min(row0 + kRows, rows) - 1) / a.group);
  // this part's tiles of all (the cached ones, then the sequence's own)
  const int32_t all_tiles = cached + last_row_token / kKeys + 1, each = (all_tiles + w.parts - 1) / w.parts;
  const int32_t tile0 = min(split * each, all_tiles), tiles = min(tile0 + each, all_tiles);

  // this lane's row
  const int col = lane & 31, half = lane >> 5;
  const int64_t wave_row = row0 + wave * 32;
  const bool active = wave_row < rows;
  const int64_t row = min(wave_row + col, rows - 1);
  const int32_t token = (int32_t)(row / a.group);
  const int32_t q_head = head * a.group + (int32_t)(row - (int64_t)token * a.group);
  // own tokens that all, and that any, of the wavefront's rows see
  const int32_t least = (int32_t)(min(wave_row, rows - 1) / a.group) + 1;
  const int32_t most = (int32_t)(min(wave_row + 31, rows - 1) / a.group) + 1;

  T tile;
  {
    const uint16_t* q = (const uint16_t*)a.q.data + (first + token) * a.q.token + q_head * a.q.head + half * 8;
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) {
      tile.q[i] = *(const u4*)(q + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) tile.q[i][e] = (tile.q[i][e] ^ a.q_flip) & a.q_mask;
    }
#pragma unroll
    for (int p = 0; p < T::kParts; ++p) tile.acc[p] = (f16){};
    tile.top = tile.peak = kNone;
    tile.far = ~0ull;
    tile.sum = 0.0f;
  }

  // ---- bringing tiles in
  const uint16_t* own_k = (const uint16_t*)a.k.data + first * a.k.token + head * a.k.head;
  const uint16_t* own_v = (const uint16_t*)a.v.data + first * a.v.token + head * a.v.head;
  const int32_t own = (int32_t)(end - first);
  const uint32_t lds_k = (uint32_t)(uintptr_t)(lds_byte*)s_k, lds_v = (uint32_t)(uintptr_t)(lds_byte*)s_v;
  constexpr int kLoads = T::kBytes / 1024 / kWaves;      // of each of K and V, a wavefront and tile
  uint32_t from_k[kLoads], from_v[kLoads];               // bytes from a tile's first token to what this lane loads
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const uint32_t piece = (i * kWaves + wave) * kWave + lane, t = piece / T::kPieces, at = piece % T::kPieces;
    from_k[i] = t * (uint32_t)a.k.token * 2 + (at ^ (t & (T::kPieces - 1))) * 16;
    from_v[i] = t * (uint32_t)a.v.token * 2 + (at ^ v_turn(t, D)) * 16;
  }
  auto load_own = [&](int32_t t0, int buf) {
    const uint16_t* k0 = own_k + t0 * a.k.token;
    const uint16_t* v0 = own_v + t0 * a.v.token;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t base = (i * kWaves + wave) * kWave;
      uint32_t back = 0;
      if (t0 + kKeys > own)                              // past the end: the last token again
        back = max(0, t0 + (int32_t)((base + lane) / T::kPieces) - (own - 1));
      to_lds(k0, from_k[i] - back * (uint32_t)a.k.token * 2, lds_k + buf * T::kBytes + base * 16);
      to_lds(v0, from_v[i] - back * (uint32_t)a.v.token * 2, lds_v + buf * T::kBytes + base * 16);
    }
  };
  // a cached tile's 16-code units of this thread: unit u of K (then of V) is
  // codes 16 (u % (D / 16)) of key u / (D / 16)
  u4 codes[T::kUnitsEach];
  float scale_k = 1.0f, scale_v = 1.0f;
  int32_t page = 0;      // as the table has it: looked at only when it is used, a tile later
  const int32_t unit_key = (tid % (kKeys * (D / 16))) / (D / 16), unit_at = tid % (D / 16);
  const bool leads = tid < kKeys * (D / 16) && unit_at == 0 && (unit_key & 3) == 0;   // fetches four keys' scales
  const uint32_t half_bytes = ((uint32_t)a.pool.heads << a.pool.log_block) * D;         // a page's keys, or values
  const uint8_t* head_pages = a.pool.pages + ((int64_t)head << a.pool.log_block) * D;
  const int32_t* ids = a.table.ids + (int64_t)r * a.table.stride;
  auto key_of = [&](int32_t j) { return min(j * kKeys + unit_key, held - 1); };
  auto find_page = [&](int32_t j) { page = ids[key_of(j) >> a.pool.log_block]; };
  auto fetch = [&](int32_t j) {
    const uint32_t id = (uint32_t)page < a.pool.num_pages ? (uint32_t)page : 0u;
    const uint32_t in_block = key_of(j) & ((1 << a.pool.log_block) - 1);
    const uint8_t* p = head_pages + (uint64_t)id * (2 * half_bytes) + in_block * D + unit_at * 16;
#pragma unroll
    for (int i = 0; i < T::kUnitsEach; ++i) {
      const int is_v = T::kUnitsEach == 2 ? i : tid >= kThreads / 2;
      codes[i] = *(const u4*)(p + (is_v ? half_bytes : 0u));
    }
    if (leads) {
      const float* x = a.pool.scales + head + (uint64_t)id * (uint32_t)(2 * a.pool.heads);
      scale_k = x[0];
      scale_v = x[a.pool.heads];
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < T::kUnitsEach; ++i) {
      const bool is_v = T::kUnitsEach == 2 ? i == 1 : tid >= kThreads / 2;
      const u2 x0 = widen4<TYPE, FMT>(codes[i][0]), x1 = widen4<TYPE, FMT>(codes[i][1]);
      const u2 x2 = widen4<TYPE, FMT>(codes[i][2]), x3 = widen4<TYPE, FMT>(codes[i][3]);
      uint8_t* to = is_v ? s_v[buf] : s_k[buf];
      const uint32_t c = 2 * unit_at;
      const uint32_t p0 = is_v ? v_piece<D>(unit_key, c) : k_piece<D>(unit_key, c);
      const uint32_t p1 = is_v ? v_piece<D>(unit_key, c + 1) : k_piece<D>(unit_key, c + 1);
      *(u4*)(to + 16 * p0) = (u4){x0[0], x0[1], x1[0], x1[1]};
      *(u4*)(to + 16 * p1) = (u4){x2[0], x2[1], x3[0], x3[1]};
    }
    if (leads) {
      const float v = kv::value_scale(scale_v);
      s_scale[buf][unit_key / 4] = (f4){scale_k * a.scale, log2_fast(v), __builtin_amdgcn_rcpf(v), 0.0f};
    }
  };

  if (tid == 0) s_odd = 0;
  const int32_t cached_end = min(cached, tiles);
  if (tile0 < cached_end) {
    find_page(tile0);
    fetch(tile0);
    if (tile0 + 1 < cached_end) find_page(tile0 + 1);
    store(tile0 & 1);
  } else if (tile0 < tiles) {
    load_own((tile0 - cached) * kKeys, tile0 & 1);
  }
  wait_loads();
  __syncthreads();

  // a loop for the cached tiles and one for the sequence's own, so that each
  // keeps the accumulators where they are
  for (int32_t j = tile0; j < cached_end; ++j) {
    const int buf = j & 1;
    if (j + 1 < cached_end) {
      fetch(j + 1);
      if (j + 2 < cached_end) find_page(j + 2);
    } else if (j + 1 < tiles) {
      load_own(0, buf ^ 1);
    }
    const int32_t left = held - j * kKeys;
    if (active)
      tile.template step<true>(lds_k + buf * T::kBytes, lds_v + buf * T::kBytes, s_scale[buf], lane, a.scale,
                               left < kKeys, left);
    if (j + 1 < cached_end) store(buf ^ 1);
    wait_loads();
    __syncthreads();
  }
  // from here on, some row must not see all of a tile, and 0 times a NaN or an
  // infinity is no 0: such values are taken out of it, and given to the rows that see them at the end
  const int32_t whole = cached + (int32_t)(row0 / a.group + 1) / kKeys;
  for (int32_t j = max(cached, tile0); j < tiles; ++j) {
    const int buf = j & 1;
    const int32_t t0 = (j - cached) * kKeys;
    if (j + 1 < tiles) load_own(t0 + kKeys, buf ^ 1);
    if (j >= whole) {
      if (T::clean(s_v[buf], wave, lane) && lane == 0) atomicOr(&s_odd, 1u << (j - whole));
      __syncthreads();
    }
    if (active && t0 < most)
      tile.template step<false>(lds_k + buf * T::kBytes, lds_v + buf * T::kBytes, nullptr, lane, a.scale,
                                t0 + kKeys > least, token + 1 - t0);
    wait_loads();
    __syncthreads();
  }
  // (a tile of rows spans 256 tokens at most: five tiles of keys)
  for (uint32_t odd = active ? s_odd : 0; odd != 0; odd &= odd - 1) {
    const int32_t t0 = (whole - cached + (int32_t)__builtin_ctz(odd)) * kKeys;
    tile.add_seen(own_k, a.k.token, own_v, a.v.token, t0, min(t0 + kKeys, most), half, a.scale, token + 1);
  }
  if (!active || wave_row + col >= rows) return;
  const float sum = sum_halves(tile.sum);
  const int64_t out_row = (first + token) * a.kv_heads * a.group + q_head;
  if (w.parts > 1) {
    const bool none = sum == 0.0f;      // this part has no key that the row sees
    const float over = none ? 0.0f : 1.0f / sum;
    float* out = a.part_out + (out_row * a.splits + split) * D + half * 4;
#pragma unroll
    for (int p = 0; p < T::kParts; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f16& x = tile.acc[p];
        *(f4*)(out + 32 * p + 8 * e) =
            (f4){x[4 * e] * over, x[4 * e + 1] * over, x[4 * e + 2] * over, x[4 * e + 3] * over};
      }
    if (half == 0) a.part_lse[out_row * a.splits + split] = none ? -__builtin_inff() : log2_sum(tile.top, sum);
    return;
  }
  const float over = 1.0f / sum;
  uint16_t* out = a.out + (first + token) * a.out_token + q_head * a.out_head + half * 4;
#pragma unroll
  for (int p = 0; p < T::kParts; ++p)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f16& x = tile.acc[p];
      *(u2*)(out + 32 * p + 8 * e) = (u2){pack2<TYPE>(x[4 * e] * over, x[4 * e + 1] * over),
                                          pack2<TYPE>(x[4 * e + 2] * over, x[4 * e + 3] * over)};
    }
  if (a.lse && half == 0) a.lse[out_row] = log2_sum(tile.top, sum) * 0.69314718055994531f;
}

// Joins the parts of four rows, a wavefront to a row: 5 us for 37 tokens of 64
// heads in 16 parts, most of it waits (four wavefronts to a row take as long).
// Rows of no sequence are left alone.
template <int TYPE, int D>
__global__ __launch_bounds__(256) void k_prefill_join(Prefill a) {
  const int lane = threadIdx.x & (kWave - 1), q_heads = a.kv_heads * a.group;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t token = row / q_heads;
  if (token >= a.num_tokens) return;
  uint32_t mine;
  const uint32_t tiles = __builtin_amdgcn_readlane(count_tiles(a, lane, &mine), kWave - 1);
  const int32_t parts = parts_for(a, tiles);
  if (parts < 2) return;
  const int32_t q_head = (int32_t)(row - token * q_heads);
  const int32_t r = kv::last_at_most(a.n, token, lane, [&](int32_t i) { return a.offsets[i]; });
  if (a.offsets[r] > token || token >= a.offsets[r + 1]) return;
  float l2;
  join_parts<TYPE, D, 1>(a.part_out + row * a.splits * D, a.part_lse + row * a.splits, parts, 0, lane, nullptr,
                         a.out + token * a.out_token + q_head * a.out_head, &l2);
  if (a.lse && lane == 0) a.lse[row] = l2 * 0.69314718055994531f;
}

// Tiles of rows, for all kv heads: no fewer and no more than these.
int64_t least_groups(int64_t num_tokens, int32_t q_heads, int32_t kv_heads) {
  return (num_tokens * (q_heads / kv_heads) + kRows - 1) / kRows * kv_heads;
}
int64_t most_groups(int32_t n, int64_t num_tokens, int32_t q_heads, int32_t kv_heads) {
  return (num_tokens * (q_heads / kv_heads) / kRows + n) * kv_heads;
}

// Room for parts of a tile's keys, where there may be fewer tiles than the
// device's 256 compute units (one agent's turn of 37 tokens after 23552: 49 us, with
// no parts 490). A part has two tiles of the longest prefix at least (a turn after 800
// tokens 15.5 us, with eight tiles a part 27), or eight of own tokens, of which
// a row sees half (700 tokens alone 25 us, in parts of two 27.5).
int32_t splits_for(int32_t n, int64_t num_tokens, int32_t q_heads, int32_t kv_heads, int64_t max_context) {
  if (n > kCounted) return 1;
  const int64_t groups = std::max<int64_t>(1, least_groups(num_tokens, q_heads, kv_heads));
  const int64_t parts = max_context / (2 * kKeys) + num_tokens / (8 * kKeys);
  return (int32_t)std::max<int64_t>(1, std::min(kTargetGroups / groups, parts));
}

}  // namespace
}  // namespace peek

using namespace peek;

extern "C" {

size_t peek_prefill_attention_workspace(int32_t n, int64_t num_tokens, int32_t q_heads, int32_t kv_heads,
                                        int32_t head_dim, int64_t max_context) {
  if (n < 1 || num_tokens < 1 || kv_heads < 1 || q_heads < kv_heads || (head_dim != 64 && head_dim != 128) ||
      max_context < 0 || num_tokens >= ((int64_t)1 << 40))
    return 0;
  const int32_t splits = splits_for(n, num_tokens, q_heads, kv_heads, max_context);
  if (splits < 2) return 0;
  return ((size_t)num_tokens * q_heads * splits * (head_dim + 1) * sizeof(float) + 255) & ~(size_t)255;
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
    Prefill a{};
    if ((pool != nullptr) != (d_prefix != nullptr))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "pool and d_prefix must be given together");
    if (pool) {
      s = check_pool(pool, &a.pool);
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
    s = check_out_rows("d_out", d_out, out_token_stride, out_head_stride, num_tokens, q_heads, head_dim);
    if (s != PEEK_OK) return s;
    if (k_token_stride >= (1 << 23) || v_token_stride >= (1 << 23))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "the token strides of d_k and d_v must be below 2^23 (got %lld, %lld)",
                  (long long)k_token_stride, (long long)v_token_stride);
    if (!d_offsets) return fail(PEEK_ERR_INVALID_ARGUMENT, "d_offsets must not be NULL");
    const int64_t context = pool ? (int64_t)max_blocks * pool->block_size : 0;
    s = check_workspace(d_workspace, workspace_bytes,
                        peek_prefill_attention_workspace(n, num_tokens, q_heads, kv_heads, head_dim, context));
    if (s != PEEK_OK) return s;
    const int32_t group = q_heads / kv_heads;
    const int64_t tiles = num_tokens < ((int64_t)1 << 40) ? most_groups(n, num_tokens, q_heads, kv_heads) : INT64_MAX;
    if (tiles >= (1 << 22))
      return fail(PEEK_ERR_INVALID_ARGUMENT, "too many rows for one call (%lld)", (long long)num_tokens);
    a.splits = splits_for(n, num_tokens, q_heads, kv_heads, context);
    // in parts there are kTargetGroups workgroups at most
    const int64_t groups = std::max(tiles, std::min(tiles * a.splits, kTargetGroups));
    hipStream_t st = (hipStream_t)stream;
    s = validate_kv(n, d_offsets, num_tokens, d_prefix, false, d_block_table, max_blocks, table_stride,
                    pool ? pool->block_size : 4, pool ? &a.pool : nullptr, st);
    if (s != PEEK_OK) return s;
    a.q = Rows{d_q, q_token_stride, q_head_stride};
    a.k = Rows{d_k, k_token_stride, k_head_stride};
    a.v = Rows{d_v, v_token_stride, v_head_stride};
    a.offsets = d_offsets;
    a.prefix = d_prefix;
    a.table = Table{d_block_table, table_stride, max_blocks};
    a.out = (uint16_t*)d_out;
    a.out_token = out_token_stride;
    a.out_head = out_head_stride;
    a.lse = d_lse;
    a.num_tokens = num_tokens;
    a.n = n;
    a.group = group;
    a.kv_heads = kv_heads;
    set_scale(scale, &a.scale, &a.q_flip, &a.q_mask);
    a.part_out = (float*)d_workspace;
    a.part_lse = a.part_out + num_tokens * q_heads * a.splits * head_dim;
    with_types(type, pool ? pool->type : PEEK_TYPE_F8E4M3, head_dim, [&](auto t, auto m, auto d) {
      hipLaunchKernelGGL((k_prefill<t(), m(), d()>), dim3((unsigned)groups), dim3(kThreads), 0, st, a);
      if (a.splits > 1)
        hipLaunchKernelGGL((k_prefill_join<t(), d()>), dim3((unsigned)((num_tokens * q_heads + 3) / 4)), dim3(256), 0,
                           st, a);
    });
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(PEEK_ERR_DEVICE, "prefill launch failed: %s", hipGetErrorString(err));
    return PEEK_OK;
  });
}

}  // extern "C"
