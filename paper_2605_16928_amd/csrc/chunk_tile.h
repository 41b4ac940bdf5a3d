// The attention of a batch of new tokens: arguments, a workgroup's place in the plan, its query tile and what the tile's rows see.
// attn_chunk.hip has the overview; chunk_wide.h and chunk_narrow.h have the two ways through a tile's keys.
#pragma once

#include "kv16_cache.h"
#include "chunk_plan.h"
#include "kv4_cache.h"
#include "mfma_tile.h"

#include <type_traits>

namespace rtp {

constexpr int kCkThreads = 512;
constexpr int kCkWaves = kCkThreads / 64;
constexpr int kCkK = 64;                       // keys per tile
constexpr int kCkPart = kHeadDim + 4;          // floats per partial row: reference, sum, sum of unrounded probabilities, pad, outputs
constexpr int kCkTileBytes = 2 * kCkK * kHeadDim * 2;

struct ChunkArgs {
  ChunkShape shape;
  const uint16_t* q;
  int64_t q_stride;
  Kv16Cache c16;
  Kv4Cache c4;
  const int32_t* q_offset;
  const int32_t* ctx_len;
  int32_t n_q_heads, n_served;
  float scale, scale_log2;
  uint16_t* out;
  float* lse;
  float* part;                 // [units of cut tiles, part_rows, kCkPart]
  int32_t part_rows;           // rows of a partial result: what a tile can have
  int32_t* plan;               // B > 64: what chunk_plan_kernel leaves, kPlanHead ints and three lists of B + 1
  int32_t run;                 // units in a row that go to one die
  int32_t f16;
};
enum { kPlanCandidate = 0, kPlanLongest = 1, kPlanHead = 4 };

// The plan of a batch of up to 64 sequences, a sequence to a lane, or of a longer one, from memory.
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
    s.ctx = max(a.ctx_len[b], 0);
    s.tiles = chunk_tiles(a.shape, nt.n);
    s.key_tiles = nt.n > 0 ? chunk_key_tiles(a.shape, nt.n, s.ctx) : 1;
  }
  return s;
}
// Lane i adds up candidate i over the sequences that the wave's lanes hold.
__device__ __forceinline__ void chunk_add_up(const ChunkLane& s, int lanes, int longest, uint32_t magic, uint64_t* units, uint64_t* split_units) {
  const int candidate = chunk_candidate(threadIdx.x & 63);
  for (int k = 0; k < lanes; ++k) {
    const int tiles = __builtin_amdgcn_readlane(s.tiles, k), kt = __builtin_amdgcn_readlane(s.key_tiles, k);
    const int S = chunk_splits(kt, longest, candidate, magic);
    *units += (uint64_t)tiles * (uint32_t)S;
    *split_units += S > 1 ? (uint64_t)tiles * (uint32_t)S : 0;
  }
}
// The best candidate of the lanes'.
__device__ __forceinline__ int chunk_best(const ChunkShape& s, uint64_t work, uint64_t units, uint64_t split_units) {
  uint32_t key = split_units > (uint64_t)s.cap ? 0xffffffffu : (chunk_cost(work, units, split_units, s.n_cu) << 6) | (threadIdx.x & 63);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) key = min(key, (uint32_t)__shfl_xor((int)key, o));
  return chunk_candidate(key == 0xffffffffu ? 0 : (int)(key & 63u));
}

// One sequence's place in the plan.
struct ChunkSpot {
  int b, rel;                  // rel: unit (or row of cut sequences) inside the sequence; b = -1: there is none
  int n, q0, ctx, splits, part0;
};
// The sequence of unit `at` (ROWS: of the at-th row of a sequence whose tiles are cut), found by the whole wave.
template <bool ROWS>
__device__ __forceinline__ ChunkSpot chunk_find(const ChunkArgs& a, int at) {
  const ChunkShape& s = a.shape;
  const int lane = threadIdx.x & 63;
  ChunkSpot spot = {};
  spot.b = -1;
  if (s.B <= 64) {
    const ChunkLane mine = chunk_lane(a, lane);
    const int longest = max(wave_max_ge_m1(mine.n > 0 ? mine.key_tiles : 1), 1);
    const uint32_t magic = chunk_magic(longest);
    uint64_t units = 0, split_units = 0;
    chunk_add_up(mine, s.B, longest, magic, &units, &split_units);
    uint64_t work = (uint64_t)(uint32_t)mine.tiles * (uint32_t)mine.key_tiles;
    work = wave_incl_scan(work);
    work = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(work >> 32), 63) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)work, 63);
    const int S = chunk_splits(mine.key_tiles, longest, chunk_best(s, work, units, split_units), magic);
    const int own = mine.tiles * S, own_rows = S > 1 ? mine.n * a.n_served : 0;
    const int last = wave_incl_scan(ROWS ? own_rows : own);
    const int part_last = wave_incl_scan(S > 1 ? own : 0);
    const int b = __popcll(__ballot(last <= at));
    if (b >= 64) return spot;
    spot.b = b;
    spot.rel = at - (__builtin_amdgcn_readlane(last, b) - __builtin_amdgcn_readlane(ROWS ? own_rows : own, b));
    spot.n = __builtin_amdgcn_readlane(mine.n, b);
    spot.q0 = __builtin_amdgcn_readlane(mine.q0, b);
    spot.ctx = __builtin_amdgcn_readlane(mine.ctx, b);
    spot.splits = __builtin_amdgcn_readlane(S, b);
    spot.part0 = __builtin_amdgcn_readlane(part_last - (S > 1 ? own : 0), b);
    return spot;
  }
  const int32_t* unit_first = a.plan + kPlanHead;
  const int32_t* part_first = unit_first + s.B + 1;
  const int32_t* row_first = part_first + s.B + 1;
  const int32_t* list = ROWS ? row_first : unit_first;
  if (at >= list[s.B]) return spot;
  const int b = wave_last_at_most(list, s.B, at);
  const ChunkLane mine = chunk_lane(a, b);
  const int longest = a.plan[kPlanLongest];
  spot.b = b;
  spot.rel = at - list[b];
  spot.n = mine.n;
  spot.q0 = mine.q0;
  spot.ctx = mine.ctx;
  spot.splits = chunk_splits(mine.key_tiles, longest, a.plan[kPlanCandidate], chunk_magic(longest));
  spot.part0 = part_first[b];
  return spot;
}

// A workgroup's unit: a query tile of one KV head, and the range of its key tiles [it_lo, it_hi).
struct ChunkTile {
  int nh, over;                // heads per token; row / nh = row * over >> 16 (exact for rows below 256, nh up to 8)
  int kvh, head0;              // KV head; its first served head's place in ChunkShape::heads
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
__device__ __forceinline__ int chunk_row_pos(const ChunkTile& t, int row) { return t.m_lo + ((row * t.over) >> 16); }

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x));
}
// The workgroup's unit (false: there is none).  Workgroups are dealt to the eight dies in turn; `run` units in a row go to one die.
template <bool LOCAL, bool KV4>
__device__ __forceinline__ bool chunk_tile(const ChunkArgs& a, ChunkTile* t) {
  const ChunkShape& s = a.shape;
  const int k8 = (int)blockIdx.x >> 3;
  const ChunkSpot spot = chunk_find<false>(a, (k8 / a.run * 8 + ((int)blockIdx.x & 7)) * a.run + k8 % a.run);
  if (spot.b < 0) return false;
  const ChunkUnit u = chunk_unit(s, spot.n, spot.splits, spot.rel);
  t->nh = s.slot_n[u.slot];
  t->over = 65536 / t->nh + 1;
  t->kvh = s.slot_kv[u.slot];
  t->head0 = s.slot_first[u.slot];
  const int t0 = u.tile * s.tok[t->nh], tokens = min((int)s.tok[t->nh], spot.n - t0);
  t->rows = tokens * t->nh;
  t->q0 = spot.q0 + t0;
  t->m_lo = spot.ctx - spot.n + t0;
  t->m_hi = t->m_lo + tokens - 1;
  const int64_t pt_stride = KV4 ? a.c4.pt_stride : a.c16.pt_stride;
  t->pt = (KV4 ? a.c4.page_table : a.c16.page_table) + spot.b * pt_stride;
  t->kend = (int)min((int64_t)max(t->m_hi + 1, 0), pt_stride << (KV4 ? a.c4.page_shift : a.c16.page_shift));
  const int all = (t->kend + kCkK - 1) / kCkK;
  t->sink_tiles = t->gap = 0;
  if (LOCAL) {
    t->sink_tiles = (min(s.sink, t->kend) + kCkK - 1) / kCkK;
    t->gap = max((s.window > 0 ? max(t->m_lo - s.window + 1, 0) / kCkK : all) - t->sink_tiles, 0);
  }
  const int n_tiles = all - t->gap;
  t->it_lo = (int)((int64_t)n_tiles * u.split / spot.splits);
  t->it_hi = (int)((int64_t)n_tiles * (u.split + 1) / spot.splits);
  t->splits = spot.splits;
  t->part = spot.part0 + spot.rel;
  // (the same in every lane, which the compiler does not see everywhere)
  int* const whole[] = {&t->nh, &t->over, &t->kvh, &t->head0, &t->rows, &t->m_lo, &t->m_hi, &t->kend, &t->sink_tiles, &t->gap, &t->it_lo, &t->it_hi,
                        &t->splits, &t->part};
#pragma unroll
  for (int* w : whole) *w = __builtin_amdgcn_readfirstlane(*w);
  t->q0 = uniform64(t->q0);
  t->pt = reinterpret_cast<const int32_t*>(uniform64((int64_t)(uintptr_t)t->pt));
  return true;
}

// What one row sees: the tokens n <= hi that are below the sink or above lo.
struct ChunkSight {
  int hi, lo;
};
__device__ __forceinline__ ChunkSight chunk_sight(const ChunkShape& s, const ChunkTile& t, int row) {
  const int m = chunk_row_pos(t, row);
  return ChunkSight{row < t.rows ? min(m, t.kend - 1) : -1, m - s.window};
}
template <bool LOCAL>
__device__ __forceinline__ bool chunk_sees(const ChunkShape& s, const ChunkSight& e, int n) {
  return n <= e.hi && (!LOCAL || n < s.sink || n > e.lo);
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
template <bool KV4>
__device__ __forceinline__ int chunk_page(const ChunkArgs& a, const ChunkTile& t, int n) {       // 0 <= n < kend; -1: a page that is not there
  const int page = t.pt[n >> (KV4 ? a.c4.page_shift : a.c16.page_shift)];
  return (uint32_t)page < (uint32_t)(KV4 ? a.c4.n_pages : a.c16.n_pages) ? page : -1;
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
  const int64_t at = (t.q0 + rt) * a.n_q_heads + a.shape.heads[t.head0 + row - rt * t.nh];
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
// O^T += V^T P^T over the seen keys alone, one by one: a key that a row does not see has probability 0, and 0 times a value that is not
// finite would not be 0.  seen: bit i = the lane's i-th key, 8 (i / 4) + 4 g + i % 4.
template <bool F16>
__device__ __forceinline__ void chunk_pv_seen(const unsigned char* v_rows, uint32_t seen, const uint32_t (&P)[8], f32x16 (&O)[4]) {
  const int g = (threadIdx.x & 63) >> 5;
  const uint32_t seen_other = (uint32_t)__shfl_xor((int)seen, 32);
  for (int i = 0; i < 16; ++i) {
    float p_own = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) p_own = e == (i >> 1) ? ((i & 1) ? hi16<F16>(P[e]) : lo16<F16>(P[e])) : p_own;
    const float p_other = __shfl_xor(p_own, 32);
    for (int half = 0; half < 2; ++half) {
      const int n = 8 * (i >> 2) + 4 * half + (i & 3);
      const bool ok = ((half == g ? seen : seen_other) >> i) & 1u;
      const float p = half == g ? p_own : p_other;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int d = db * 32 + i4 * 8 + g * 4;
          const u32x2 w = *reinterpret_cast<const u32x2*>(v_rows + n * 256 + ((d >> 4) ^ (2 * (n & 3))) * 32 + (d & 15) * 2);
          const float v[4] = {lo16<F16>(w[0]), hi16<F16>(w[0]), lo16<F16>(w[1]), hi16<F16>(w[1])};
#pragma unroll
          for (int j = 0; j < 4; ++j) O[db][i4 * 4 + j] = ok ? fmaf(p, v[j], O[db][i4 * 4 + j]) : O[db][i4 * 4 + j];
        }
    }
  }
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
