// The attention of a batch of new tokens: arguments, a workgroup's place in the plan, its query tile and what the tile's rows see.
// attn_chunk.hip has the overview; chunk_wide.h and chunk_narrow.h have the two ways through a tile's keys.
#pragma once

#include "kv16_cache.h"
#include "chunk_plan.h"
#include "kv4_cache.h"
#include "mfma_tile.h"

#include <type_traits>

namespace rtp {

constexpr int kCkWaves = 8;                     // of the workgroups that take wide tiles
constexpr int kCkThreads = kCkWaves * 64;
constexpr int kCkSmallWaves = 4;                // of those that take narrow ones alone, two to a compute unit
constexpr int kCkK = 64;                       // keys per tile
constexpr int kCkPart = kHeadDim + 4;          // floats per partial row: reference, sum, sum of unrounded probabilities, pad, outputs
constexpr int kCkTileBytes = 2 * kCkK * kHeadDim * 2;

struct ChunkArgs {
  ChunkShape shape;
  int32_t n_q_heads, f16;
  float scale, scale_log2;
  const uint16_t* q;
  int64_t q_stride;
  const int32_t* q_offset;
  const int32_t* ctx_len;
  uint16_t* out;
  float* lse;
  float* part;                 // [units of cut tiles, part_rows, kCkPart]
  int32_t part_rows;           // rows of a partial result: what a tile can have
  struct ChunkMerge* merge;    // [n_merge]: the tiles, for the merge launch (NULL: nothing is cut)
  int32_t n_merge;
  int32_t* plan;               // B > 64: what chunk_plan_kernel leaves, kPlanHead ints and three lists of B + 1
  int32_t* again;              // [workgroups]: 1 = its unit has to be taken again
  Kv16Cache c16;
  Kv4Cache c4;
};
// A query tile as the merge launch needs it; rows = 0: its results are complete.
struct ChunkMerge {
  int32_t rows, splits, part, step;      // ranges: partial results part, part + step ...
  int32_t heads, members, kvh, q0;
};
enum { kPlanCandidate = 0, kPlanLongest = 1, kPlanHead = 4 };

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x));
}
struct ChunkLane {
  int n, q0, ctx;              // new tokens, their first row, context
  int tiles, key_tiles;
};
__device__ __forceinline__ ChunkLane chunk_lane(const ChunkArgs& a, int b) {
  ChunkLane s = {0, 0, 0, 0, 1};
  if (b < a.shape.B) {
    const NewTokens nt = new_tokens(a.q_offset, b, a.shape.total_q, a.shape.max_q);
    s.n = nt.n;
    s.q0 = nt.q0;
    s.ctx = min(max(a.ctx_len[b], 0), kMostContext);
    s.tiles = chunk_tiles(a.shape, nt.n);
    s.key_tiles = nt.n > 0 ? chunk_key_tiles(a.shape, nt.n, s.ctx) : 1;
  }
  return s;
}
// Lane i adds up candidate i over the sequences that the wave's lanes hold.
__device__ __forceinline__ void chunk_add_up(const ChunkShape& shape, const ChunkLane& s, int lanes, int longest, uint32_t magic, ChunkSums* sums) {
  const int candidate = chunk_candidate(threadIdx.x & 63);
  const int tiles = __float_as_int((float)s.tiles), rows = __float_as_int((float)(s.n * shape.n_served));
  const float per_place = chunk_over(1.f, shape.places);
#pragma unroll 1
  for (int k = 0; k < lanes; ++k) {
    const int kt = __builtin_amdgcn_readlane(s.key_tiles, k);
    chunk_sum(sums, __int_as_float(__builtin_amdgcn_readlane(tiles, k)), __int_as_float(__builtin_amdgcn_readlane(rows, k)), (float)kt,
              chunk_splits(kt, longest, candidate, magic), per_place);
  }
}
// The best candidate of the lanes': the least cost, to within 2^-17.
__device__ __forceinline__ int chunk_best(const ChunkShape& s, int longest, float work, const ChunkSums& sums) {
  const float cost = chunk_cost(work, sums, longest, chunk_candidate(threadIdx.x & 63), s.places);
  const bool fits = sums.cut_units <= (float)s.cap && cost < __builtin_huge_valf();
  int key = fits ? -(int)((__float_as_uint(cost) & ~63u) | (threadIdx.x & 63)) : -0x7fffffff;         // (negative: the largest is wanted)
#define RTP_STEP(CTRL, MASK) key = max(key, __builtin_amdgcn_update_dpp(-0x7fffffff, key, CTRL, MASK, 0xf, false));
  RTP_WAVE_SCAN_STEPS(RTP_STEP)
#undef RTP_STEP
  key = -wave_last(key);
  return chunk_candidate(key == 0x7fffffff ? 0 : key & 63);
}
__device__ __forceinline__ float wave_sum_f32(float x) {
#define RTP_STEP(CTRL, MASK) x += __int_as_float(dpp_or_zero<CTRL, MASK>(__float_as_int(x)));
  RTP_WAVE_SCAN_STEPS(RTP_STEP)
#undef RTP_STEP
  return __int_as_float(wave_last(__float_as_int(x)));
}

// The plan as a wave has it: of up to 64 sequences one to a lane (scans inclusive), of more in memory.
struct ChunkPlan {
  ChunkLane seq;
  int splits, units, unit_last, part_last, tile_last;
};
__device__ __forceinline__ ChunkPlan chunk_plan(const ChunkArgs& a) {
  const ChunkShape& s = a.shape;
  ChunkPlan p = {};
  if (__builtin_expect(s.B > 64, 0)) return p;
  p.seq = chunk_lane(a, threadIdx.x & 63);
  const int longest = max(wave_max_ge_m1(p.seq.n > 0 ? p.seq.key_tiles : 1), 1);
  const uint32_t magic = chunk_magic(longest);
  int candidate = 1;
  if (s.cap > 0) {
    ChunkSums sums = {};
    chunk_add_up(s, p.seq, s.B, longest, magic, &sums);
    const float work = wave_sum_f32((float)p.seq.tiles * (float)p.seq.key_tiles);
    candidate = chunk_best(s, longest, work, sums);
  }
  p.splits = chunk_splits(p.seq.key_tiles, longest, candidate, magic);
  p.units = p.seq.tiles * p.splits;
  p.unit_last = wave_incl_scan(p.units);
  p.part_last = wave_incl_scan(p.splits > 1 ? p.units : 0);
  p.tile_last = wave_incl_scan(p.seq.tiles);
  return p;
}

// A unit's sequence: the unit's number in it, what it has, and the numbers of its first partial result and its first tile.  b = -1: the unit is `rel`
// behind the last one, and there are `tile0` tiles.
struct ChunkSpot {
  int b, rel, n, q0, ctx, splits, part0, tile0;
};
__device__ __forceinline__ ChunkSpot chunk_find(const ChunkArgs& a, int at) {
  const ChunkShape& s = a.shape;
  ChunkSpot spot = {};
  spot.b = -1;
  if (__builtin_expect(s.B <= 64, 1)) {
    const ChunkPlan p = chunk_plan(a);
    const int b = __popcll(__ballot(p.unit_last <= at));
    if (b >= 64) {
      spot.rel = at - wave_last(p.unit_last);
      spot.tile0 = wave_last(p.tile_last);
      return spot;
    }
    spot.b = b;
    spot.rel = at - __builtin_amdgcn_readlane(p.unit_last - p.units, b);
    spot.n = __builtin_amdgcn_readlane(p.seq.n, b);
    spot.q0 = __builtin_amdgcn_readlane(p.seq.q0, b);
    spot.ctx = __builtin_amdgcn_readlane(p.seq.ctx, b);
    spot.splits = __builtin_amdgcn_readlane(p.splits, b);
    spot.part0 = __builtin_amdgcn_readlane(p.part_last - (p.splits > 1 ? p.units : 0), b);
    spot.tile0 = __builtin_amdgcn_readlane(p.tile_last - p.seq.tiles, b);
    return spot;
  }
  const int32_t* unit_first = a.plan + kPlanHead;
  const int32_t* part_first = unit_first + s.B + 1;
  const int32_t* tile_first = part_first + s.B + 1;
  if (at >= unit_first[s.B]) {
    spot.rel = at - unit_first[s.B];
    spot.tile0 = tile_first[s.B];
    return spot;
  }
  const int b = wave_last_at_most(unit_first, s.B, at);
  const ChunkLane mine = chunk_lane(a, b);
  const int longest = a.plan[kPlanLongest];
  spot.b = b;
  spot.rel = at - unit_first[b];
  spot.n = mine.n;
  spot.q0 = mine.q0;
  spot.ctx = mine.ctx;
  spot.splits = chunk_splits(mine.key_tiles, longest, a.plan[kPlanCandidate], chunk_magic(longest));
  spot.part0 = part_first[b];
  spot.tile0 = tile_first[b];
  return spot;
}

// A workgroup's unit: a query tile of one KV head, and the range of its key tiles [it_lo, it_hi).
struct ChunkTile {
  int nh, over;                // heads per token; row / nh = row * over >> 16 (exact for rows below 256, nh up to 8)
  int kvh, members;            // KV head; its served heads, as bits
  int rows;                    // (token, head) pairs of the tile
  int64_t q0;                  // its first token's row of q
  int m_lo, m_hi;              // its first and last position; may be negative, where ctx_len says so
  int kend;                    // keys that some row may see
  int sink_tiles, gap;         // 64-key tiles of the sink; tiles between those and the band
  int it_lo, it_hi;
  int splits, part;            // ranges of the tile; where this one's partial result lies
  const int32_t* pt;           // the sequence's row of the page table
};

__device__ __forceinline__ int chunk_tile_n0(const ChunkTile& t, int it) { return (it + (it >= t.sink_tiles ? t.gap : 0)) * kCkK; }
__device__ __forceinline__ int chunk_row_factor(int h) { return (int)(65536.f * __builtin_amdgcn_rcpf((float)h)) + 1; }     // 65536 / h + 1
// Query head of a row, whose token is the rt-th.
__device__ __forceinline__ int chunk_head(const ChunkArgs& a, const ChunkTile& t, int row, int rt) {
  const int k = row - rt * t.nh;
  return t.kvh * a.shape.group + (t.nh == a.shape.group ? k : chunk_nth((uint32_t)t.members, k));
}
__device__ __forceinline__ int chunk_row_pos(const ChunkTile& t, int row) { return t.m_lo + ((row * t.over) >> 16); }

// A workgroup's unit (false: there is none).  Workgroups are dealt to the eight dies in turn; 2^run_shift units in a row go to one die, and every
// other deal goes the other way round, since what comes first is longer.
template <bool LOCAL, bool KV4>
__device__ __forceinline__ bool chunk_tile(const ChunkArgs& a, int workgroup, ChunkTile* t) {
  const ChunkShape& s = a.shape;
  const int k8 = workgroup >> 3, in_run = k8 & ((1 << s.run_shift) - 1), deal = k8 >> s.run_shift, die = (workgroup & 7) ^ ((deal & 1) * 7);
  const ChunkSpot spot = chunk_find(a, ((deal * 8 + die) << s.run_shift) + in_run);
  if (spot.b < 0) {
    // (there are as many workgroups without a unit as there may be tiles that are not there)
    if (a.merge && threadIdx.x == 0 && spot.tile0 + spot.rel < a.n_merge) a.merge[spot.tile0 + spot.rel].rows = 0;
    return false;
  }
  const ChunkUnit u = chunk_unit(s, spot.n, spot.splits, spot.rel);
  if (u.kv >= s.n_kv) return false;                                    // (offsets that do not ascend)
  t->nh = u.heads;
  t->over = chunk_row_factor(u.heads);
  t->kvh = u.kv;
  t->members = (int)chunk_members(s, u.kv);
  const int most = ((kChunkRows >> s.fine) * t->over) >> 16, t0 = u.tile * most, tokens = min(most, spot.n - t0);
  t->rows = tokens * t->nh;
  t->q0 = spot.q0 + t0;
  t->m_lo = spot.ctx - spot.n + t0;
  t->m_hi = t->m_lo + tokens - 1;
  const int64_t pt_stride = KV4 ? a.c4.pt_stride : a.c16.pt_stride;
  t->pt = (KV4 ? a.c4.page_table : a.c16.page_table) + spot.b * pt_stride;
  const int shift = KV4 ? a.c4.page_shift : a.c16.page_shift;          // (kend: not behind the table, in 32 bits)
  t->kend = max(t->m_hi + 1, 0);
  if (pt_stride <= 0x7fffffff >> shift) t->kend = min(t->kend, (int)pt_stride << shift);
  const int all = (t->kend + kCkK - 1) / kCkK;
  t->sink_tiles = t->gap = 0;
  if (LOCAL) {
    t->sink_tiles = (min(s.sink, t->kend) + kCkK - 1) / kCkK;
    t->gap = max((s.window > 0 ? min(max(t->m_lo - s.window + 1, 0) / kCkK, all) : all) - t->sink_tiles, 0);      // (kend may end before the band)
  }
  const int n_tiles = all - t->gap;
  chunk_range(n_tiles, u.split, spot.splits, &t->it_lo, &t->it_hi);
  t->splits = spot.splits;
  t->part = spot.part0 + spot.rel;
  const int number = spot.tile0 + u.before + u.tiles - 1 - u.tile;
  if (a.merge && u.split == 0 && threadIdx.x == 0 && number < a.n_merge)
    a.merge[number] =
        ChunkMerge{spot.splits > 1 ? t->rows : 0, spot.splits, t->part, u.step, u.heads, t->members, u.kv, (int)t->q0};
  // (the same in every lane, which the compiler does not see everywhere)
  int* const whole[] = {&t->nh, &t->over, &t->kvh, &t->members, &t->rows, &t->m_lo, &t->m_hi, &t->kend, &t->sink_tiles, &t->gap, &t->it_lo, &t->it_hi,
                        &t->splits, &t->part};
#pragma unroll
  for (int* w : whole) *w = __builtin_amdgcn_readfirstlane(*w);
  t->q0 = uniform64(t->q0);
  t->pt = reinterpret_cast<const int32_t*>(uniform64((int64_t)(uintptr_t)t->pt));
  return true;
}

template <bool KV4>
__device__ __forceinline__ int chunk_page(const ChunkArgs& a, const ChunkTile& t, int n) {       // 0 <= n < kend; -1: a page that is not there
  const int page = t.pt[n >> (KV4 ? a.c4.page_shift : a.c16.page_shift)];
  return (uint32_t)page < (uint32_t)(KV4 ? a.c4.n_pages : a.c16.n_pages) ? page : -1;
}

// What one row sees: the tokens n <= hi that are below the sink or above lo.
struct ChunkSight {
  int hi, lo, sink;
};
__device__ __forceinline__ ChunkSight chunk_sight(const ChunkShape& s, const ChunkTile& t, int row) {
  const int m = chunk_row_pos(t, row);
  return ChunkSight{row < t.rows ? min(m, t.kend - 1) : -1, m - s.window, s.sink};
}
// Bit i: the row sees key n + 8 (i / 4) + i % 4, the lane's i-th of a block if n is the block's first plus 4 g.
template <bool LOCAL>
__device__ __forceinline__ bool chunk_sees(const ChunkSight& e, int off) { return off <= e.hi && (!LOCAL || off < e.sink || off > e.lo); }
template <bool LOCAL>
__device__ __forceinline__ void chunk_mask(const ChunkSight& sight, int n, f32x16& S) {
  const ChunkSight e = {sight.hi - n, sight.lo - n, sight.sink - n};
#pragma unroll
  for (int i = 0; i < 16; ++i) S[i] = chunk_sees<LOCAL>(e, 8 * (i >> 2) + (i & 3)) ? S[i] : -__builtin_huge_valf();
}
// The same as bits, of keys whose pages are there.
template <bool LOCAL, bool KV4>
__device__ __forceinline__ uint32_t chunk_seen(const ChunkArgs& a, const ChunkTile& t, const ChunkSight& sight, int n) {
  const ChunkSight e = {sight.hi - n, sight.lo - n, sight.sink - n};
  uint32_t seen = 0;
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) {
    const int n4 = n + i4 * 8;                                              // (four neighbours share their page)
    const bool there = n4 < t.kend && chunk_page<KV4>(a, t, min(n4, t.kend - 1)) >= 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) seen |= there && chunk_sees<LOCAL>(e, i4 * 8 + j) ? 1u << (i4 * 4 + j) : 0u;
  }
  return seen;
}
// Rows at the positions [lo, hi] (hi < 0: no rows) and keys [n, n + len): does some row see one of them; does some row not see all of them.
template <bool LOCAL>
__device__ __forceinline__ bool chunk_any_seen(const ChunkShape& s, const ChunkTile& t, int lo, int hi, int n, int len) {
  return n <= hi && n < t.kend && (!LOCAL || n < s.sink || n + len - 1 > lo - s.window);
}
template <bool LOCAL>
__device__ __forceinline__ bool chunk_all_seen(const ChunkShape& s, const ChunkTile& t, int lo, int hi, int n, int len) {
  return n + len - 1 <= lo && n + len <= t.kend && (!LOCAL || n + len <= s.sink || n > hi - s.window);
}
// The reference that goes with a sum: none for a range without keys; a sum that is not a number has one that the merge does not take for that.
__device__ __forceinline__ float chunk_reference(float m, float l) {
  const float ninf = -__builtin_huge_valf();
  return l == 0.f ? ninf : l != l && m == ninf ? 0.f : m;
}
// Four neighbouring outputs of a row, normalised (L == 0: the row sees nothing), or of a range's partial result; the row's sums with its first four.
// F: the sum of the probabilities before their rounding to 16 bits, which the log-sum is of.
template <bool F16>
__device__ __forceinline__ void chunk_store4(const ChunkArgs& a, const ChunkTile& t, int row, int dim, float m, float l, float F, const float (&o)[4]) {
  if (t.splits > 1) {
    if (row >= a.part_rows) return;
    float* const p = a.part + ((int64_t)t.part * a.part_rows + row) * kCkPart;
    if (dim == 0) *reinterpret_cast<float4*>(p) = make_float4(chunk_reference(m, l), l, F, 0.f);
    *reinterpret_cast<float4*>(p + 4 + dim) = make_float4(o[0], o[1], o[2], o[3]);
    return;
  }
  const int rt = (row * t.over) >> 16;
  const int64_t at = (t.q0 + rt) * a.n_q_heads + chunk_head(a, t, row, rt);
  const bool none = l == 0.f;
  const float inv = none ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2*>(a.out + at * kHeadDim + dim) =
      none ? (u32x2){0u, 0u} : (u32x2){pack16<F16>(o[0] * inv, o[1] * inv), pack16<F16>(o[2] * inv, o[3] * inv)};
  if (a.lse && dim == 0) a.lse[at] = none ? -__builtin_huge_valf() : m * a.scale + logf(F);
}

// ---- products of a wave over 32 keys in LDS: K rows then, V_AT bytes further, V rows, of 256 bytes each.  K row n keeps its 16-byte chunk c at
// position c ^ (n % 16), V row n its 32-byte unit u at position u ^ 2 (n % 4): the operand reads below are then spread over the banks. ----
struct ChunkReads {
  int k, kx, v, vx;
};
__device__ __forceinline__ ChunkReads chunk_reads() {
  const int lane = threadIdx.x & 63, g = lane >> 5, r = lane & 31, j = lane & 15;
  return ChunkReads{r * 256, (g ^ (r & 15)) << 4, (4 * g + (j >> 2)) * 256 + 8 * (j & 3), (((lane >> 4) & 1) ^ (2 * (j >> 2))) << 5};
}
__device__ __forceinline__ u32x4 chunk_read_k(const unsigned char* rows, const ChunkReads& d, int kk) {
  return *reinterpret_cast<const u32x4*>(rows + d.k + ((kk << 5) ^ d.kx));
}
// 8 keys x 1 dim of V^T: two transposing reads of 4 keys each
__device__ __forceinline__ u32x4 chunk_read_v(const unsigned char* rows, const ChunkReads& d, int tt, int db) {
  const unsigned char* p0 = rows + d.v + 16 * tt * 256 + ((db << 6) ^ d.vx);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p0));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p0 + 8 * 256));
  return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <bool F16>
__device__ __forceinline__ uint32_t chunk_not_finite(const u32x4 v) {      // not 0 iff one of eight values is not finite
  constexpr uint32_t kExp = F16 ? 0x7c007c00u : 0x7f807f80u, kOne = F16 ? 0x04000400u : 0x00800080u;
  uint32_t any = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) any |= ((v[w] & kExp) + kOne) & 0x80008000u;
  return any;
}
// A lane's i-th probability of a block: its rounding P, and the rounding of the rest R.
template <bool F16>
__device__ __forceinline__ float chunk_probability(const uint32_t (&P)[8], const uint32_t (&R)[8], int i) {      // the lane's i-th
  uint32_t w = P[0], x = R[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    w = e == (i >> 1) ? P[e] : w;
    x = e == (i >> 1) ? R[e] : x;
  }
  return (i & 1) ? hi16<F16>(w) + hi16<F16>(x) : lo16<F16>(w) + lo16<F16>(x);
}
// O^T += V^T (P + R)^T over the seen keys alone, one by one: a key that a row does not see has probability 0, and 0 times a value that is not
// finite would not be 0; nor would R, which is 0 where P is exact.  seen: bit i = the lane's i-th key, 8 (i / 4) + 4 g + i % 4.
template <bool F16>
__device__ __forceinline__ void chunk_pv_seen(const unsigned char* v_rows, uint32_t seen, const uint32_t (&P)[8], const uint32_t (&R)[8], f32x16 (&O)[4]) {
  const int g = (threadIdx.x & 63) >> 5;
  const uint32_t seen_other = (uint32_t)__shfl_xor((int)seen, 32);
#pragma unroll
  for (int db = 0; db < 4; ++db) {
#pragma unroll 1
    for (int k = 0; k < 32; ++k) {                                         // key 8 (i / 4) + 4 half + i % 4
      const int i = k >> 1, half = k & 1, n = 8 * (i >> 2) + 4 * half + (i & 3);
      const float p_own = chunk_probability<F16>(P, R, i), p_other = __shfl_xor(p_own, 32), p = half == g ? p_own : p_other;
      const bool ok = ((half == g ? seen : seen_other) >> i) & 1u;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int d = db * 32 + i4 * 8 + g * 4;
        const u32x2 v = *reinterpret_cast<const u32x2*>(v_rows + n * 256 + ((d >> 4) ^ (2 * (n & 3))) * 32 + (d & 15) * 2);
        const float x[4] = {lo16<F16>(v[0]), hi16<F16>(v[0]), lo16<F16>(v[1]), hi16<F16>(v[1])};
#pragma unroll
        for (int j = 0; j < 4; ++j) O[db][i4 * 4 + j] = ok ? fmaf(p, x[j], O[db][i4 * 4 + j]) : O[db][i4 * 4 + j];
      }
    }
  }
}

// LDS words that only the own wave writes and reads.
__device__ __forceinline__ void chunk_wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// 16 bytes per lane from global memory to LDS, 1 KiB per wave.  (Assembly, since through the compiler's intrinsic every later LDS read waits for
// all outstanding loads; whoever reads the rows waits for them itself.)
__device__ __forceinline__ void chunk_load_lds(uint32_t dst, const uint8_t* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(dst)), "v"(offset),
               "s"(uniform64((int64_t)(uintptr_t)base)) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void chunk_wait_loads() {          // all but the last N of the wave's loads have landed
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

}  // namespace rtp
