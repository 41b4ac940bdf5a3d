// Causal attention of a batch of new tokens over a cache in pages: rtp_dense_attn_chunk (every token) and rtp_local_attn_chunk (sink +
// window), from 16-bit pages or from the 4-bit cache.
//
//   out_m = sum_n p_n v_n / sum_n p_n,   p_n = 2^(c <q_m, k_n> - r_m),   c = softmax scale * log2(e)
// over the tokens n that position m sees; r_m is a reference that cancels.
//
// Work: a KV head's served query heads share its rows, so a query tile is 256 (token, head) pairs of one KV head -- 64 tokens of a group of
// four, one token's eight heads where there is one -- and eight waves of 32 rows share every staged tile of 64 keys.  Tiles and the ranges of
// their keys are numbered by chunk_plan.h from the lengths on the device: every workgroup finds its own, the host sees bounds only.  Where a
// tile's keys are cut into ranges, the workgroups leave (maximum, sums, unnormalised outputs) per row to a merge launch.
//
// A wave computes the transposed scores S^T = K Q^T of 32 keys (v_mfma_f32_32x32x16): lane (g, r) then holds 16 keys of ONE row, the softmax is
// per lane, and the probabilities, rounded to 16 bits, are in place as the B operand of O^T = V^T P^T.
#include "kv16_cache.h"
#include "chunk_plan.h"
#include "kv4_cache.h"
#include "mfma_tile.h"

#include <algorithm>
#include <type_traits>

namespace rtp {

constexpr int kCkThreads = 512;
constexpr int kCkWaves = kCkThreads / 64;
constexpr int kCkK = 64;                       // keys per tile
constexpr int kCkPart = kHeadDim + 4;          // floats per partial row: reference, sum, sum of unrounded probabilities, pad, outputs
constexpr int kCkTileBytes = 2 * kCkK * kHeadDim * 2;
constexpr int kCkStages = 3;

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

// B > 64: the same by one workgroup, once for the launches behind it.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void chunk_plan_kernel(const ChunkArgs a) {
  constexpr int NW = kPlanThreads / 64;
  __shared__ uint64_t sh_units[NW][64], sh_split[NW][64], sh_work[NW];
  __shared__ int sh_longest[NW], sh_candidate, sh_sum[3][NW];
  const ChunkShape& s = a.shape;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int longest = 1;
  for (int b0 = wave * 64; b0 < s.B; b0 += kPlanThreads) {
    const ChunkLane mine = chunk_lane(a, b0 + lane);
    longest = max(longest, wave_max_ge_m1(mine.n > 0 ? mine.key_tiles : 1));
  }
  if (lane == 0) sh_longest[wave] = longest;
  __syncthreads();
  for (int w = 0; w < NW; ++w) longest = max(longest, sh_longest[w]);
  const uint32_t magic = chunk_magic(longest);
  uint64_t units = 0, split_units = 0, work = 0;
  for (int b0 = wave * 64; b0 < s.B; b0 += kPlanThreads) {
    const ChunkLane mine = chunk_lane(a, b0 + lane);
    chunk_add_up(mine, min(64, s.B - b0), longest, magic, &units, &split_units);
    work += (uint64_t)(uint32_t)mine.tiles * (uint32_t)mine.key_tiles;
  }
  work = wave_incl_scan(work);
  sh_units[wave][lane] = units;
  sh_split[wave][lane] = split_units;
  if (lane == 63) sh_work[wave] = work;
  __syncthreads();
  if (wave == 0) {
    units = split_units = work = 0;
    for (int w = 0; w < NW; ++w) {
      units += sh_units[w][lane];
      split_units += sh_split[w][lane];
      work += sh_work[w];
    }
    const int best = chunk_best(s, work, units, split_units);
    if (lane == 0) {
      sh_candidate = best;
      a.plan[kPlanCandidate] = best;
      a.plan[kPlanLongest] = longest;
    }
  }
  __syncthreads();
  int32_t* const lists[3] = {a.plan + kPlanHead, a.plan + kPlanHead + s.B + 1, a.plan + kPlanHead + 2 * (s.B + 1)};
  int before[3] = {0, 0, 0};
  for (int b0 = 0; b0 < s.B; b0 += kPlanThreads) {
    const ChunkLane mine = chunk_lane(a, b0 + tid);
    const int S = chunk_splits(mine.key_tiles, longest, sh_candidate, magic), own = mine.tiles * S;
    const int add[3] = {own, S > 1 ? own : 0, S > 1 ? mine.n * a.n_served : 0};
    int last[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      last[k] = wave_incl_scan(add[k]);
      if (lane == 63) sh_sum[k][wave] = last[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      int first = before[k], all = 0;
      for (int w = 0; w < NW; ++w) {
        if (w < wave) first += sh_sum[k][w];
        all += sh_sum[k][w];
      }
      if (b0 + tid < s.B) lists[k][b0 + tid] = first + last[k] - add[k];
      before[k] += all;
    }
    __syncthreads();
  }
  if (tid < 3) lists[tid][s.B] = before[tid];
}

// What a row sees, as bounds: the tokens n <= hi that are below `sink` or above `lo`.
struct RowSight {
  int hi, lo;
};

template <bool F16, bool LOCAL, bool KV4>
__global__ __launch_bounds__(kCkThreads, 2) void chunk_attn_kernel(const ChunkArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[kCkTileBytes * kCkStages];
  const ChunkShape& sh = a.shape;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const float ninf = -__builtin_huge_valf();

  // ---- the unit: workgroups are dealt to the eight dies in turn, `run` units in a row go to one of them ----
  const int k8 = (int)blockIdx.x >> 3;
  const int unit = (k8 / a.run * 8 + ((int)blockIdx.x & 7)) * a.run + k8 % a.run;
  const ChunkSpot spot = chunk_find<false>(a, unit);
  if (spot.b < 0) return;
  const ChunkUnit u = chunk_unit(sh, spot.n, spot.splits, spot.rel);
  const int nh = sh.slot_n[u.slot], tok = sh.tok[nh], kvh = sh.slot_kv[u.slot];
  const int t0 = u.tile * tok, rows = min(tok, spot.n - t0) * nh;
  const int pos0 = spot.ctx - spot.n + t0;                          // the first row's position; may be negative, where ctx_len says so
  const int page_shift = KV4 ? a.c4.page_shift : a.c16.page_shift, n_pages = KV4 ? a.c4.n_pages : a.c16.n_pages;
  const int64_t pt_stride = KV4 ? a.c4.pt_stride : a.c16.pt_stride;
  const int32_t* const pt = (KV4 ? a.c4.page_table : a.c16.page_table) + spot.b * pt_stride;
  const int64_t held = pt_stride << page_shift;                     // positions that the table has entries for
  auto page_of = [&](int n) __attribute__((always_inline)) {        // 0 <= n < held
    const int page = pt[n >> page_shift];
    return (uint32_t)page < (uint32_t)n_pages ? page : -1;
  };

  // ---- rows ----
  const int over = 65536 / nh + 1;                                  // row / nh by a product: exact for rows below 256, nh up to 8
  const int row = wave * 32 + r, row_t = (row * over) >> 16;
  const bool qok = row < rows;
  const int head = qok ? sh.heads[sh.slot_first[u.slot] + row - row_t * nh] : 0;
  const int64_t qi = spot.q0 + t0 + row_t;
  u32x4 qreg[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
    qreg[kk] = qok ? *reinterpret_cast<const u32x4*>(a.q + qi * a.q_stride + head * kHeadDim + kk * 16 + g * 8) : (u32x4){0u, 0u, 0u, 0u};
  const int m_lo = pos0, m_hi = pos0 + (rows - 1) / nh;             // the tile's first and last position
  const int kend = (int)min((int64_t)max(m_hi + 1, 0), held);       // keys that some row may see
  const int mq = pos0 + row_t;
  const RowSight sight = {qok ? min(mq, kend - 1) : -1, LOCAL ? mq - sh.window : -1};
  auto sees = [&](int n) __attribute__((always_inline)) { return n <= sight.hi && (!LOCAL || n < sh.sink || n > sight.lo); };
  // the wave's rows: positions of the first and the last, -1 and less for a wave without rows
  const int w_lo = wave * 32 < rows ? pos0 + ((wave * 32 * over) >> 16) : -1;
  const int w_hi = wave * 32 < rows ? pos0 + ((min(wave * 32 + 31, rows - 1) * over) >> 16) : -1;

  // ---- the tile's key tiles: those of the sink, then those of the band ----
  const int all_tiles = (kend + kCkK - 1) / kCkK;
  int sink_tiles = 0, gap = 0;
  if (LOCAL) {
    sink_tiles = (min(sh.sink, kend) + kCkK - 1) / kCkK;
    const int band = sh.window > 0 ? max(m_lo - sh.window + 1, 0) / kCkK : all_tiles;
    gap = max(band - sink_tiles, 0);
  }
  const int n_tiles = all_tiles - gap;
  auto tile_n0 = [&](int it) __attribute__((always_inline)) { return (it + (it >= sink_tiles ? gap : 0)) * kCkK; };
  const int it_lo = (int)((int64_t)n_tiles * u.split / spot.splits), it_hi = (int)((int64_t)n_tiles * (u.split + 1) / spot.splits);

  // ---- staging: K rows then V rows of 256 bytes; K row n keeps 16-byte chunk c at position c ^ (n % 16), V row n 32-byte unit u
  // at position u ^ 2 (n % 4), which spreads the operand reads below over the banks ----
  const uint32_t lds_base = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int ld_sub = lane >> 4, ld_pos = lane & 15;
  const int ld_ck = ld_pos ^ ((4 * wave + ld_sub) & 15);
  const int ld_cv = ((((ld_pos >> 1) ^ (2 * (ld_sub & 3))) << 1) | (ld_pos & 1));
  const uint8_t* const Kh = KV4 ? nullptr : a.c16.K + (int64_t)kvh * a.c16.head_bytes;
  const uint8_t* const Vh = KV4 ? nullptr : a.c16.V + (int64_t)kvh * a.c16.head_bytes;
  // 16-bit rows go to LDS directly: four neighbouring rows (of one page) per wave and instruction.  Rows behind the last key repeat it, rows of a
  // page that the pool does not have are the pool's first: masked all the same.
  auto load_rows = [&](int n0, int slot, int jj) __attribute__((always_inline)) {
    const int nb = min(n0 + 32 * jj + 4 * wave, (kend - 1) & ~3), n = min(nb + ld_sub, kend - 1);
    const int64_t at = (int64_t)max(page_of(n), 0) * a.c16.page_bytes + (int64_t)(n & ((1 << page_shift) - 1)) * a.c16.row_bytes;
    const uint32_t dst = lds_base + slot * kCkTileBytes + (jj * kCkWaves + wave) * 1024;
    // (assembly, since through the compiler's intrinsic every later LDS read waits for all outstanding loads)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(Kh + at + ld_ck * 16) : "memory", "m0");
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst + kCkTileBytes / 2), "v"(Vh + at + ld_cv * 16) : "memory", "m0");
  };
  // A 4-bit row is 16 bytes for each of eight lanes: four blocks of K, four of V, each with its scale.
  auto load_codes = [&](int n0, u32x4& codes, uint32_t& scale) __attribute__((always_inline)) {
    const int n = min(n0 + 8 * wave + (lane >> 3), kend - 1), piece = lane & 7, slot = n & ((1 << page_shift) - 1);
    const int64_t page = max(page_of(n), 0);
    codes = *reinterpret_cast<const u32x4*>(a.c4.codes + page * a.c4.code_page16 * 16 + (int64_t)kvh * a.c4.code_head_stride + (int64_t)slot * kKv4Row + piece * 16);
    scale = a.c4.scales[page * a.c4.scale_page16 * 16 + (int64_t)kvh * a.c4.scale_head_stride + (int64_t)(slot >> 2) * kKv4Group + piece * 4 + (slot & 3)];
  };
  auto put_codes = [&](int slot, const u32x4 codes, uint32_t scale) __attribute__((always_inline)) {
    const int n = 8 * wave + (lane >> 3), piece = lane & 7, blk = piece & 3;
    const float f = __uint_as_float(scale << 23);
    unsigned char* const dst = smem + slot * kCkTileBytes + (piece < 4 ? 0 : kCkTileBytes / 2) + n * 256;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ck = (4 * blk + i) ^ (n & 15), cv = ((2 * blk + (i >> 1)) ^ (2 * (n & 3))) * 2 + (i & 1);
      *reinterpret_cast<u32x4*>(dst + (piece < 4 ? ck : cv) * 16) = decode8<F16>(codes[i], f);
    }
  };
  auto loads_landed = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

  // ---- operand reads ----
  const int rd_k = r * 256, rd_kx = (g ^ (r & 15)) << 4;
  const int rd_j = lane & 15, rd_G = (lane >> 4) & 1;
  const int rd_v = kCkTileBytes / 2 + (4 * g + (rd_j >> 2)) * 256 + 8 * (rd_j & 3);
  const int rd_vx = (rd_G ^ (2 * (rd_j >> 2))) << 5;
  auto read_k = [&](const unsigned char* tile, int kb, int kk) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4*>(tile + kb * 8192 + rd_k + ((kk << 5) ^ rd_kx));
  };
  // 8 keys x 1 dim of V^T: two transposing reads of 4 keys each
  auto read_v = [&](const unsigned char* tile, int kb, int tt, int db) __attribute__((always_inline)) {
    const unsigned char* p0 = tile + rd_v + (kb * 32 + 16 * tt) * 256 + ((db << 6) ^ rd_vx);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p0));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p0 + 8 * 256));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  f32x16 O[4];
  float mrow = ninf, lrow = 0.f, lsum_full = 0.f;
  const float c = a.scale_log2;
  auto mfma_S = [&](const unsigned char* tile, int kb, f32x16& S) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) S = mfma32<F16>(read_k(tile, kb, kk), qreg[kk], S);
  };
  auto mfma_PV = [&](const unsigned char* tile, int kb, const uint32_t (&P)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int db = 0; db < 4; ++db)
        O[db] = mfma32<F16>(read_v(tile, kb, tt, db), (u32x4){P[4 * tt], P[4 * tt + 1], P[4 * tt + 2], P[4 * tt + 3]}, O[db]);
  };

  // ---- running maximum, accumulators rescaled in place; the next tile's rows are on their way ----
  auto exact_pass = [&]() __attribute__((always_inline)) {
    f32x16 S;
    uint32_t P[8];
    u32x4 codes;
    uint32_t scale = 0;
    mrow = ninf;
    lrow = lsum_full = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
    __syncthreads();
    if (it_lo >= it_hi) return;
    if constexpr (KV4) load_codes(tile_n0(it_lo), codes, scale);
    else {
      load_rows(tile_n0(it_lo), 0, 0);
      load_rows(tile_n0(it_lo), 0, 1);
    }
    for (int it = it_lo; it < it_hi; ++it) {
      const int buf = (it - it_lo) & 1, n0 = tile_n0(it);
      const unsigned char* const tile = smem + buf * kCkTileBytes;
      if constexpr (KV4) put_codes(buf, codes, scale);
      else loads_landed();
      __syncthreads();
      if (it + 1 < it_hi) {
        if constexpr (KV4) load_codes(tile_n0(it + 1), codes, scale);
        else {
          load_rows(tile_n0(it + 1), buf ^ 1, 0);
          load_rows(tile_n0(it + 1), buf ^ 1, 1);
        }
      }
      for (int kb = 0; kb < 2; ++kb) {
        const int nb0 = n0 + kb * 32;
        if (nb0 > w_hi || nb0 >= kend) continue;                     // (the same for the whole wave)
        if (LOCAL && nb0 >= sh.sink && nb0 + 31 <= w_lo - sh.window) continue;
        mfma_S(tile, kb, S);
        uint32_t seen = 0;                                           // bit i: the lane's i-th key, nb0 + 8 (i / 4) + 4 g + i % 4, is seen
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int n4 = nb0 + i4 * 8 + g * 4;
          const bool there = n4 < kend && page_of(min(n4, kend - 1)) >= 0;       // (four neighbours share their page)
#pragma unroll
          for (int j = 0; j < 4; ++j) seen |= there && sees(n4 + j) ? 1u << (i4 * 4 + j) : 0u;
        }
        const bool masked = __ballot(seen != 0xffffu) != 0ull;
        float mx = ninf;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          S[i] = (seen >> i) & 1u ? S[i] : ninf;
          mx = fmaxf(mx, S[i]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mnew = fmaxf(mrow, mx), msafe = mnew == ninf ? 0.f : mnew, mc = msafe * c;
        float lsum = 0.f, lfull = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = fast_exp2(fmaf(S[i], c, -mc)), p1 = fast_exp2(fmaf(S[i + 1], c, -mc));
          P[i >> 1] = pack16<F16>(p0, p1);
          lfull += p0 + p1;
          lsum += lo16<F16>(P[i >> 1]) + hi16<F16>(P[i >> 1]);
        }
        const float corr = fast_exp2((mrow - msafe) * c);
        lrow = lrow * corr + lsum;
        lsum_full = lsum_full * corr + lfull;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[db][i] *= corr;
        mrow = mnew;
        // A key that a row does not see has probability 0, and 0 times a value that is not finite would not be 0: such a block's
        // products are taken one by one, over the seen keys alone.
        bool odd = false;
        if (masked) {
          uint32_t any = 0;
          constexpr uint32_t kExp = F16 ? 0x7c007c00u : 0x7f807f80u, kOne = F16 ? 0x04000400u : 0x00800080u;
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
              const u32x4 v = read_v(tile, kb, tt, db);
#pragma unroll
              for (int w = 0; w < 4; ++w) any |= ((v[w] & kExp) + kOne) & 0x80008000u;
            }
          odd = __ballot(any != 0u) != 0ull;
        }
        if (!odd) {
          mfma_PV(tile, kb, P);
        } else {
          for (int i = 0; i < 16; ++i) {
            float p_own = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) p_own = e == (i >> 1) ? ((i & 1) ? hi16<F16>(P[e]) : lo16<F16>(P[e])) : p_own;
            const uint32_t seen_other = (uint32_t)__shfl_xor((int)seen, 32);
            const float p_other = __shfl_xor(p_own, 32);
            for (int half = 0; half < 2; ++half) {
              const int n = kb * 32 + 8 * (i >> 2) + 4 * half + (i & 3);                    // row of the tile
              const bool ok = ((half == g ? seen : seen_other) >> i) & 1u;
              const float p = half == g ? p_own : p_other;
              const unsigned char* vrow = tile + kCkTileBytes / 2 + n * 256;
#pragma unroll
              for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                  const int d = db * 32 + i4 * 8 + g * 4;
                  const u32x2 w = *reinterpret_cast<const u32x2*>(vrow + ((d >> 4) ^ (2 * (n & 3))) * 32 + (d & 15) * 2);
                  const float v[4] = {lo16<F16>(w[0]), hi16<F16>(w[0]), lo16<F16>(w[1]), hi16<F16>(w[1])};
#pragma unroll
                  for (int j = 0; j < 4; ++j) O[db][i4 * 4 + j] = ok ? fmaf(p, v[j], O[db][i4 * 4 + j]) : O[db][i4 * 4 + j];
                }
            }
          }
        }
      }
      __syncthreads();
    }
  };
  exact_pass();

  // ---- normalise and store, or leave the range's partial result ----
  const float l = lrow + __shfl_xor(lrow, 32), l_full = lsum_full + __shfl_xor(lsum_full, 32);
  if (!qok) return;
  if (spot.splits > 1) {
    if (row >= a.part_rows) return;
    float* prow = a.part + ((int64_t)(spot.part0 + spot.rel) * a.part_rows + row) * kCkPart;
    // (a sum that is not a number comes with a reference that the merge does not take for a range without keys)
    if (g == 0) *reinterpret_cast<float4*>(prow) = make_float4(l != l && mrow == ninf ? 0.f : mrow, l, l_full, 0.f);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
        *reinterpret_cast<float4*>(prow + 4 + db * 32 + i4 * 8 + g * 4) =
            make_float4(O[db][i4 * 4], O[db][i4 * 4 + 1], O[db][i4 * 4 + 2], O[db][i4 * 4 + 3]);
    return;
  }
  const bool none = l == 0.f;
  const float inv = none ? 0.f : 1.f / l;
  uint16_t* const orow = a.out + (qi * a.n_q_heads + head) * kHeadDim;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
      *reinterpret_cast<u32x2*>(orow + db * 32 + i4 * 8 + g * 4) =
          none ? (u32x2){0u, 0u} : (u32x2){pack16<F16>(O[db][i4 * 4] * inv, O[db][i4 * 4 + 1] * inv), pack16<F16>(O[db][i4 * 4 + 2] * inv, O[db][i4 * 4 + 3] * inv)};
  if (a.lse && g == 0) a.lse[qi * a.n_q_heads + head] = none ? ninf : mrow * a.scale + logf(l_full);
}

// Merges the ranges of the rows whose tiles were cut: SLICES groups of 32 lanes per row take the ranges in turn, a lane 4 of the 128 dims.
template <int SLICES>
__global__ __launch_bounds__(256) void chunk_merge_kernel(const ChunkArgs a) {
  __shared__ float sh_h[8][3];
  __shared__ __attribute__((aligned(16))) float sh_acc[8][kHeadDim];
  constexpr int kRows = 8 / SLICES;
  const ChunkShape& sh = a.shape;
  const int tid = threadIdx.x, d4 = tid & 31, grp = tid >> 5, slice = grp % SLICES;
  const float ninf = -__builtin_huge_valf();
  for (int at0 = blockIdx.x * kRows;; at0 += (int)gridDim.x * kRows) {
    const ChunkSpot spot = chunk_find<true>(a, at0);                 // (the rows of a workgroup: those of one sequence, or the next ones' too)
    if (spot.b < 0) return;
    // row -> (token, served head)
    const int at = at0 + grp / SLICES;
    ChunkSpot mine = spot;
    if (spot.rel + kRows > spot.n * a.n_served) {                     // (the same for the whole workgroup)
      for (int k = 0; k < kRows; ++k) {
        const ChunkSpot other = chunk_find<true>(a, at0 + k);
        if (grp / SLICES == k) mine = other;
      }
    } else {
      mine.rel += at - at0;
    }
    const bool have = mine.b >= 0;
    float M = ninf, L = 0.f, F = 0.f;
    float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
    int64_t o = 0;
    if (have) {
      const int t = mine.rel / a.n_served, hs = mine.rel - t * a.n_served;
      int slot = 0;
      while (hs >= sh.slot_first[slot] + sh.slot_n[slot]) ++slot;
      const int nh = sh.slot_n[slot], tile = t / sh.tok[nh];
      const int row = (t - tile * sh.tok[nh]) * nh + hs - sh.slot_first[slot];
      int step;
      const int first = chunk_unit_of(sh, mine.n, mine.splits, slot, tile, &step);
      o = (int64_t)(mine.q0 + t) * a.n_q_heads + sh.heads[hs];
      const float* p = a.part + ((int64_t)(mine.part0 + first) * a.part_rows + row) * kCkPart;
      const int64_t pstep = (int64_t)step * a.part_rows * kCkPart;
      for (int s0 = slice; s0 < mine.splits; s0 += 4 * SLICES) {
        float4 h[4], v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int s = s0 + k * SLICES;
          h[k] = make_float4(ninf, 0.f, 0.f, 0.f);
          v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (s < mine.splits) {
            h[k] = *reinterpret_cast<const float4*>(p + s * pstep);
            v[k] = *reinterpret_cast<const float4*>(p + s * pstep + 4 + d4 * 4);
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float Mn = fmaxf(M, h[k].x);
          if (Mn == ninf) continue;
          const float c0 = fast_exp2((M - Mn) * a.scale_log2), c1 = fast_exp2((h[k].x - Mn) * a.scale_log2);
          L = L * c0 + h[k].y * c1;
          F = F * c0 + h[k].z * c1;
          A.x = A.x * c0 + v[k].x * c1; A.y = A.y * c0 + v[k].y * c1;
          A.z = A.z * c0 + v[k].z * c1; A.w = A.w * c0 + v[k].w * c1;
          M = Mn;
        }
      }
    }
    if (d4 == 0) { sh_h[grp][0] = M; sh_h[grp][1] = L; sh_h[grp][2] = F; }
    *reinterpret_cast<float4*>(&sh_acc[grp][d4 * 4]) = A;
    __syncthreads();
    if (slice == 0 && have) {
      float Mt = ninf, Lt = 0.f, Ft = 0.f;
      float4 At = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < SLICES; ++k) Mt = fmaxf(Mt, sh_h[grp + k][0]);
      if (Mt != ninf) {
#pragma unroll
        for (int k = 0; k < SLICES; ++k) {
          const float cw = fast_exp2((sh_h[grp + k][0] - Mt) * a.scale_log2);
          const float4 v = *reinterpret_cast<const float4*>(&sh_acc[grp + k][d4 * 4]);
          Lt += sh_h[grp + k][1] * cw;
          Ft += sh_h[grp + k][2] * cw;
          At.x += v.x * cw; At.y += v.y * cw; At.z += v.z * cw; At.w += v.w * cw;
        }
      }
      const bool none = Lt == 0.f;
      const float inv = none ? 0.f : 1.f / Lt;
      const u32x2 w = a.f16 ? (u32x2){pack16<true>(At.x * inv, At.y * inv), pack16<true>(At.z * inv, At.w * inv)}
                            : (u32x2){pack16<false>(At.x * inv, At.y * inv), pack16<false>(At.z * inv, At.w * inv)};
      *reinterpret_cast<u32x2*>(a.out + o * kHeadDim + d4 * 4) = none ? (u32x2){0u, 0u} : w;
      if (a.lse && d4 == 0) a.lse[o] = none ? ninf : Mt * a.scale + logf(Ft);
    }
    __syncthreads();
  }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------------
namespace {
int compute_units() {
  static const int n = [] {
    int dev = 0, cu = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cu <= 0) cu = 256;
    (void)hipGetLastError();
    return cu;
  }();
  return n;
}

enum { kServeAll = 0, kServeRet = 1, kServeLocal = 2 };

// The heads that a call serves, by KV head.
void serve(const rtp_layer_desc* L, const HeadTable& ht, int which, ChunkShape* s, int32_t* n_served) {
  const int group = L->n_q_heads / L->n_kv_heads;
  int n = 0;
  for (int kv = 0; kv < L->n_kv_heads; ++kv) {
    const int first = n;
    for (int h = kv * group; h < (kv + 1) * group; ++h)
      if (which == kServeAll || (ht.is_ret[h] != 0) == (which == kServeRet)) s->heads[n++] = (uint8_t)h;
    if (n == first) continue;
    s->slot_kv[s->n_slots] = (uint8_t)kv;
    s->slot_first[s->n_slots] = (uint8_t)first;
    s->slot_n[s->n_slots] = (uint8_t)(n - first);
    ++s->cnt[n - first];
    ++s->n_slots;
  }
  for (int k = 1; k <= 8; ++k) s->tok[k] = (uint16_t)(kChunkRows / k);
  *n_served = n;
}

struct ChunkSizes {
  int64_t tiles;               // query tiles that the bounds allow
  int64_t cap;                 // units of cut tiles
  int32_t part_rows;
  size_t plan_bytes, part_bytes;
  size_t total() const { return plan_bytes + part_bytes; }
};
ChunkSizes chunk_sizes(const ChunkShape& s, int32_t B, int64_t total_q, int64_t max_q, int64_t max_ctx) {
  ChunkSizes z = {};
  int widest = 1;
  max_q = std::max<int64_t>(1, std::min(max_q, total_q));
  for (int h = 1; h <= 8; ++h) {
    if (!s.cnt[h]) continue;
    widest = h;
    // a sequence of n tokens has ceil(n / tok) tiles: at most n of them, at most one more than its share
    const int64_t per_seq = (max_q + s.tok[h] - 1) / s.tok[h];
    z.tiles += s.cnt[h] * std::min(std::min(total_q, total_q / s.tok[h] + B), per_seq * B);
  }
  // ranges of two key tiles and more, about two units to a compute unit
  int64_t keys = max_ctx;
  if (s.local) keys = std::min<int64_t>(keys, (int64_t)s.sink + s.window + 64);
  const int64_t ranges = std::max<int64_t>(1, std::min<int64_t>((keys + 2 * kCkK - 1) / (2 * kCkK), 289));
  z.cap = ranges > 1 ? std::min<int64_t>(z.tiles * ranges, 4 * (int64_t)compute_units()) : 0;
  z.part_rows = (int32_t)std::min<int64_t>(kChunkRows, max_q * widest);
  z.plan_bytes = B > 64 ? align_up((size_t)(kPlanHead + 3 * ((int64_t)B + 1)) * sizeof(int32_t), 256) : 0;
  z.part_bytes = align_up((size_t)z.cap * z.part_rows * kCkPart * sizeof(float), 256);
  return z;
}

size_t chunk_workspace(const rtp_layer_desc* layer, int which, int32_t B, int32_t total_q, int32_t max_q, int64_t max_ctx) {
  HeadTable ht;
  if (fill_head_table(layer, &ht, "workspace") != RTP_OK || B <= 0 || B > kMaxSeqs || total_q <= 0 || total_q > (1 << 24) || max_q <= 0 ||
      max_ctx <= 0 || max_ctx > ((int64_t)1 << 30))
    return 256;
  ChunkShape s = {};
  int32_t served = 0;
  serve(layer, ht, which, &s, &served);
  s.local = which == kServeLocal;
  s.sink = layer->sink;
  s.window = layer->window;
  return std::max<size_t>(256, chunk_sizes(s, B, total_q, max_q, max_ctx).total());
}

int32_t chunk_call(const char* who, int which, const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv_cache* c16,
                   const rtp_kv4_cache* c4, bool kv4, const rtp_chunk* chunk, void* out, float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  HeadTable ht;
  int32_t rc = fill_head_table(layer, &ht, who);
  if (rc != RTP_OK) return rc;
  rc = check_chunk(who, chunk);
  if (rc != RTP_OK) return rc;
  ChunkArgs a = {};
  rc = kv4 ? check_kv4_cache(who, layer, c4, chunk->max_ctx, &a.c4) : check_kv16_cache(who, layer, c16, chunk->max_ctx, &a.c16);
  if (rc != RTP_OK) return rc;
  if (!q || !out) return fail(RTP_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  if (((uintptr_t)q & 15) || ((uintptr_t)out & 15) || ((uintptr_t)lse & 3))
    return fail(RTP_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned, lse 4-byte aligned", who);
  const int64_t width = (int64_t)layer->n_q_heads * kHeadDim;
  if ((q_stride & 7) || q_stride < width || q_stride > ((int64_t)1 << 40))
    return fail(RTP_ERR_INVALID_ARG, "%s: q_stride must be a multiple of 8 elements that holds a token's rows", who);
  if (chunk->total_q > 0 && rows_overlap(q, q_stride, width, out, width, width, chunk->total_q))
    return fail(RTP_ERR_INVALID_ARG, "%s: out overlaps q", who);
  serve(layer, ht, which, &a.shape, &a.n_served);
  a.shape.local = which == kServeLocal;
  a.shape.sink = layer->sink;
  a.shape.window = layer->window;
  if (a.n_served == 0 || chunk->total_q == 0) {
    clear_error();
    return RTP_OK;
  }
  const ChunkSizes z = chunk_sizes(a.shape, chunk->B, chunk->total_q, chunk->max_q, chunk->max_ctx);
  if (z.total() > 0 && (!ws || ((uintptr_t)ws & 255) || ws_bytes < z.total()))
    return fail(RTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, 256-byte aligned, needed", who, z.total());
  const int64_t run = std::min<int64_t>(32, (std::min(chunk->max_q, chunk->total_q) + kChunkRows / 8 - 1) / (kChunkRows / 8));
  a.run = 1;
  while (a.run * 2 <= run) a.run *= 2;
  const int64_t deal = 8 * (int64_t)a.run, grid = (z.tiles + z.cap + deal - 1) / deal * deal;
  if (grid > 0x7fffffff / kCkThreads) return fail(RTP_ERR_UNSUPPORTED, "%s: too many query tiles for one call", who);
  clear_error();
  a.shape.B = chunk->B;
  a.shape.total_q = chunk->total_q;
  a.shape.max_q = chunk->max_q;
  a.shape.cap = (int32_t)z.cap;
  a.shape.n_cu = compute_units();
  a.q = (const uint16_t*)q;
  a.q_stride = q_stride;
  a.q_offset = chunk->q_offset;
  a.ctx_len = chunk->ctx_len;
  a.n_q_heads = layer->n_q_heads;
  a.scale = softmax_scale_of(layer);
  a.scale_log2 = a.scale * 1.4426950408889634f;
  a.out = (uint16_t*)out;
  a.lse = lse;
  a.plan = (int32_t*)ws;
  a.part = (float*)((uint8_t*)ws + z.plan_bytes);
  a.part_rows = z.part_rows;
  a.f16 = layer->kv_dtype == RTP_DTYPE_FP16;
  if (chunk->B > 64) RTP_LAUNCH(chunk_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
  const bool local = a.shape.local != 0;
#define RTP_CHUNK(F16, LOCAL, KV4)                                                                          \
  if ((a.f16 != 0) == F16 && local == LOCAL && kv4 == KV4)                                                  \
    RTP_LAUNCH((chunk_attn_kernel<F16, LOCAL, KV4>), dim3((unsigned)grid), dim3(kCkThreads), 0, stream, a);
  RTP_CHUNK(false, false, false)
  RTP_CHUNK(true, false, false)
  RTP_CHUNK(false, true, false)
  RTP_CHUNK(true, true, false)
  RTP_CHUNK(false, false, true)
  RTP_CHUNK(true, false, true)
  RTP_CHUNK(false, true, true)
  RTP_CHUNK(true, true, true)
#undef RTP_CHUNK
  if (z.cap > 0) {
    const int64_t rows = (int64_t)chunk->total_q * a.n_served;
    if (rows <= 2048) RTP_LAUNCH(chunk_merge_kernel<8>, dim3((unsigned)rows), dim3(256), 0, stream, a);
    else RTP_LAUNCH(chunk_merge_kernel<2>, dim3((unsigned)std::min<int64_t>((rows + 3) / 4, 8192)), dim3(256), 0, stream, a);
  }
  return check_launch(who);
}
}  // namespace

}  // namespace rtp

using namespace rtp;

extern "C" size_t rtp_dense_attn_chunk_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int32_t total_q, int32_t max_q, int64_t max_ctx,
                                                       int32_t heads) {
  return chunk_workspace(layer, heads == RTP_HEADS_RETRIEVAL ? kServeRet : kServeAll, B, total_q, max_q, max_ctx);
}
extern "C" size_t rtp_local_attn_chunk_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int32_t total_q, int32_t max_q, int64_t max_ctx) {
  return chunk_workspace(layer, kServeLocal, B, total_q, max_q, max_ctx);
}

static int32_t dense_which(const char* who, int32_t heads, int* which) {
  if (heads != RTP_HEADS_ALL && heads != RTP_HEADS_RETRIEVAL)
    return fail(RTP_ERR_INVALID_ARG, "%s: heads must be RTP_HEADS_ALL or RTP_HEADS_RETRIEVAL", who);
  *which = heads == RTP_HEADS_ALL ? kServeAll : kServeRet;
  return RTP_OK;
}

extern "C" int32_t rtp_dense_attn_chunk(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv_cache* cache,
                                        const rtp_chunk* chunk, int32_t heads, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  int which = 0;
  const int32_t rc = dense_which("rtp_dense_attn_chunk", heads, &which);
  return rc != RTP_OK ? rc : chunk_call("rtp_dense_attn_chunk", which, layer, q, q_stride, cache, nullptr, false, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_dense_attn_chunk_kv4(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv4_cache* cache,
                                            const rtp_chunk* chunk, int32_t heads, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  int which = 0;
  const int32_t rc = dense_which("rtp_dense_attn_chunk_kv4", heads, &which);
  return rc != RTP_OK ? rc : chunk_call("rtp_dense_attn_chunk_kv4", which, layer, q, q_stride, nullptr, cache, true, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_local_attn_chunk(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv_cache* cache,
                                        const rtp_chunk* chunk, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return chunk_call("rtp_local_attn_chunk", kServeLocal, layer, q, q_stride, cache, nullptr, false, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_local_attn_chunk_kv4(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv4_cache* cache,
                                            const rtp_chunk* chunk, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return chunk_call("rtp_local_attn_chunk_kv4", kServeLocal, layer, q, q_stride, nullptr, cache, true, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
