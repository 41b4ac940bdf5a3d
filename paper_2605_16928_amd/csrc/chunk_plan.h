// How the attention of a batch of new tokens (attn_chunk.hip) is cut into units of work, from the lengths that only the device knows.
// Apart from the kernels so that it also compiles for the host.
//
// A KV head with h served query heads takes 256 / h tokens per query tile (an eighth of the rows where all sequences have few: `fine`); a tile's rows
// are (token, head) pairs, the heads of a token side by side.  A tile's keys are cut into as many ranges as its sequence has splits; a unit is one
// range of one tile.  Units that read the same keys are neighbours, and long ones come before short ones: a sequence's units are numbered (group of
// 2^run_shift tiles from the last to the first, KV head, range, tile from the last to the first), as far as every KV head has whole groups, and then
// (KV head, range, tile) over the tiles that are left.
//
// One number, the candidate, fixes all splits: sequence b has ceil(candidate * key tiles of b / key tiles of the longest), so that the
// ranges of all sequences are about equally long.
//
// What a kernel knows of the heads fits a few scalars: tables among a kernel's arguments lie in memory that takes microseconds to reach.
#pragma once

#include <math.h>
#include <stdint.h>

namespace rtp {

constexpr int kChunkRows = 256;          // rows of a query tile
constexpr int kMostContext = 1 << 30;
constexpr int kChunkMostKeyTiles = 1 << 22;
constexpr int kChunkCandidates = 64;
// What a unit costs beside its key tiles, in key tiles: its way to the first product and from the last, 12 us where a wide tile of keys takes 1.9
// (plan 1.6, first pages, queries and keys 4.3, reference 0.9, end of the sums and outputs 3, the next workgroup's beginning 2.5; at 3 in place of 6 a
// batch of 12 sequences, 0 to 500 tokens behind 0 to 16001, 172 us and 155); a launch's, that results are merged; and the rows of partial results,
// written and read, that take as long as a key tile per place (two passes over 528 bytes, 32 KiB a tile).
constexpr int kChunkUnitCost = 6, kChunkMergeCost = 4, kChunkRowsPerTile = 31;

struct ChunkShape {
  int32_t B, total_q, max_q;
  int32_t fine;                          // a query tile's rows are halved so often
  int32_t group, n_kv;                   // query heads per KV head (1, 2, 4 or 8), KV heads
  int32_t local, sink, window;
  int32_t cap;                           // most units of tiles that are cut into ranges
  float places;                          // workgroups that run at the same time
  int32_t n_served, widest;              // served query heads; the most of one KV head
  int32_t kv_served, run_shift;          // KV heads with served heads; 2^run_shift units in a row go to one die
  uint32_t per_most;                     // of the KV head with the fewest served heads: the largest tokens per tile
  uint32_t served[4];                    // bit h: query head h is one of them
  int32_t count[8];                      // KV heads with 1 .. 8 of them
  uint32_t per_tile[8];                  // 2^32 / tokens per tile of such a head, as chunk_inverse has it
};

__host__ __device__ __forceinline__ int chunk_min(int a, int b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ int chunk_max(int a, int b) { return a > b ? a : b; }

// Tokens per query tile of a KV head with h served heads, and the number that multiplies in place of a division by them: n tokens, 1 .. 2^24, have
// floor((n - 1) inverse / 2^32) + 1 tiles (the excess of the inverse, less than 1, times n - 1 stays below 2^32 / tokens).
__host__ __device__ __forceinline__ int chunk_tokens(int fine, int h) { return (kChunkRows >> fine) / h; }
__host__ __device__ __forceinline__ uint32_t chunk_inverse(int tokens) { return 0xffffffffu / (uint32_t)tokens + 1u; }
__host__ __device__ __forceinline__ int chunk_query_tiles(int n, uint32_t inverse) {
  return n > 0 ? (int)(((uint64_t)(uint32_t)(n - 1) * inverse) >> 32) + 1 : 0;
}
// The served heads of a KV head, as bits, and how many they are.
__host__ __device__ __forceinline__ uint32_t chunk_members(const ChunkShape& s, int kv) {
  const int at = kv * s.group;
  const uint32_t w01 = (at & 32) ? s.served[1] : s.served[0], w23 = (at & 32) ? s.served[3] : s.served[2];
  return (((at & 64) ? w23 : w01) >> (at & 31)) & ((1u << s.group) - 1u);
}
__host__ __device__ __forceinline__ int chunk_bits(uint32_t m) { return __builtin_popcount(m); }
// The place of the k-th set bit.
__host__ __device__ __forceinline__ int chunk_nth(uint32_t m, int k) {
  int at = 0;
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    at = ((m >> b) & 1u) && k == 0 ? b : at;
    k -= (int)((m >> b) & 1u);
  }
  return at;
}

// Splits of the longest sequence that candidate i (0 .. 63) stands for: 1 .. 32, then 40, 48 .. 288.
__host__ __device__ __forceinline__ int chunk_candidate(int i) { return i < 32 ? i + 1 : 32 + 8 * (i - 31); }

// Query tiles of a sequence with n new tokens, over all KV heads.
__host__ __device__ __forceinline__ int chunk_tiles(const ChunkShape& s, int n) {
  int tiles = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) tiles += s.count[k] * ((int)(((uint64_t)(uint32_t)(n - 1) * s.per_tile[k]) >> 32) + 1);
  return n > 0 ? tiles : 0;
}
// 64-key tiles that one of its query tiles reads (a middling one).
__host__ __device__ __forceinline__ int chunk_key_tiles(const ChunkShape& s, int n, int ctx) {
  int keys = chunk_max(ctx - n / 2, 1);
  if (s.local) {
    const int64_t band = (int64_t)s.sink + s.window + chunk_min(n, 64);
    if (band < keys) keys = (int)band;
  }
  return chunk_max(1, chunk_min((int)(((uint32_t)keys + 63u) >> 6), kChunkMostKeyTiles));
}
// (Every launch of a call has to come to the same splits: whole numbers, multiply-adds where they are
// written and nowhere else, and sums in the same order.  And it is code that
// every workgroup goes through once, from memory: no wide division, no wide sums.)
__host__ __device__ __forceinline__ uint32_t chunk_magic(int longest) { return 0xffffffffu / (uint32_t)longest; }
__host__ __device__ __forceinline__ int chunk_splits(int key_tiles, int longest, int candidate, uint32_t magic) {
  const uint32_t x = (uint32_t)key_tiles * (uint32_t)candidate + (uint32_t)longest - 1u;      // at most 2^22 * 289
  return chunk_max(1, (int)(((uint64_t)x * magic) >> 32));
}
struct ChunkSums {
  float units, cut_units, cut_rows;      // units; those of cut tiles; rows of partial results
  float most;                            // what the units of one sequence take by themselves, at the most
};
__host__ __device__ __forceinline__ float chunk_over(float x, float y) {      // x / y to a few steps
#ifdef __HIP_DEVICE_COMPILE__
  return x * __builtin_amdgcn_rcpf(y);
#else
  return x / y;
#endif
}
__host__ __device__ __forceinline__ void chunk_sum(ChunkSums* sums, float tiles, float rows, float key_tiles, int splits, float per_place) {
#pragma clang fp contract(off)
  const float S = (float)splits, cut = splits > 1 ? S : 0.f;
  sums->most = fmaxf(sums->most, ceilf(tiles * S * per_place - 0.001f) * (ceilf(chunk_over(key_tiles, S)) + (float)kChunkUnitCost));
  sums->units = fmaf(tiles, S, sums->units);
  sums->cut_units = fmaf(tiles, cut, sums->cut_units);
  sums->cut_rows = fmaf(rows, cut, sums->cut_rows);
}
// What a candidate costs.  Units that are alike go in rounds over the places for workgroups; what the longest sequence's are longer than the mean
// comes on top, all of it where every unit has a place at once, half of it otherwise.  Units that differ fill up the places as they come, but for half
// of the longest at the end.  A sequence's own units, which are alike, take whole rounds in any case.  And the partial results.
__host__ __device__ __forceinline__ float chunk_cost(float work, const ChunkSums& sums, int longest, int candidate, float places) {
#pragma clang fp contract(off)
  const float mean = ceilf(chunk_over(work, sums.units)), most = ceilf(chunk_over((float)longest, (float)candidate));
  const float rounds = ceilf(chunk_over(sums.units, places) - 0.001f);
  const float alike = fmaf(most > mean ? most - mean : 0.f, rounds > 1.f ? 0.5f : 1.f, rounds * (mean + (float)kChunkUnitCost));
  const float mixed = fmaf(0.5f, most, chunk_over(fmaf(sums.units, (float)kChunkUnitCost, work), places));
  float cost = fmaxf(rounds > 1.f ? fminf(alike, mixed) : alike, sums.most);
  cost = fmaf(sums.cut_rows, chunk_over(1.f / kChunkRowsPerTile, places), cost);
  return sums.cut_units > 0.f ? cost + (float)kChunkMergeCost : cost;
}
// The range of n key tiles that split k of S has: [first, first of k + 1).
__host__ __device__ __forceinline__ void chunk_range(int n, int k, int S, int* lo, int* hi) {
  const int each = (int)((uint32_t)n / (uint32_t)S), more = n - each * S;
  *lo = k * each + chunk_min(k, more);
  *hi = *lo + each + (k < more ? 1 : 0);
}

struct ChunkUnit {
  int kv, heads;                         // KV head, its served heads
  int split, tile;
  int tiles, before;                     // query tiles of this KV head, and of those before it
  int step;                              // from a tile's range to its next one, in units
};
// Unit r of a sequence with n new tokens and S splits.  Its tile is the (before + tiles - 1 - tile)-th of the sequence.
__host__ __device__ __forceinline__ ChunkUnit chunk_unit(const ChunkShape& s, int n, int S, int r) {
  ChunkUnit u = {0, 1, 0, 0, 1, 0, 1};
  const int groups = chunk_query_tiles(n, s.per_most) >> s.run_shift, block = S << s.run_shift;
  int grouped = 0, group = 0, nth = 0;                                    // tiles of a KV head in groups; the unit's group, its KV head
  bool in_group = false;
  if (groups > 1) {
    grouped = groups << s.run_shift;
    const int units = groups * block * s.kv_served;
    in_group = r < units;
    if (in_group) {
      const int k = (int)((uint32_t)r / (uint32_t)block);
      r -= k * block;
      group = (int)((uint32_t)k / (uint32_t)s.kv_served);
      nth = k - group * s.kv_served;
    } else {
      r -= units;
    }
  }
  for (; u.kv < s.n_kv; ++u.kv) {
    u.heads = chunk_bits(chunk_members(s, u.kv));
    if (u.heads == 0) continue;
    uint32_t inverse = s.per_tile[0];                                     // (scalars: nothing is looked up in memory)
#pragma unroll
    for (int k = 1; k < 8; ++k) inverse = u.heads == k + 1 ? s.per_tile[k] : inverse;
    u.tiles = chunk_query_tiles(n, inverse);
    const int mine = (u.tiles - grouped) * S;
    if (in_group ? nth == 0 : r < mine) break;
    r -= in_group ? 0 : mine;
    --nth;
    u.before += u.tiles;
  }
  if (in_group) {
    u.split = r >> s.run_shift;
    u.tile = u.tiles - 1 - (group << s.run_shift) - (r & ((1 << s.run_shift) - 1));
    u.step = 1 << s.run_shift;
  } else {
    u.step = u.tiles - grouped;
    u.split = (int)((uint32_t)r / (uint32_t)u.step);
    u.tile = u.step - 1 - (r - u.split * u.step);
  }
  return u;
}

}  // namespace rtp
