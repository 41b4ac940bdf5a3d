// How the attention of a batch of new tokens (attn_chunk.hip) is cut into units of work, from the lengths that only the device knows.
// Apart from the kernels so that it also compiles for the host.
//
// A KV head with n served query heads takes floor(256 / n) tokens per query tile; a tile's rows are (token, head) pairs, the heads of a token
// side by side.  A tile's keys are cut into as many ranges as its sequence has splits; a unit is one range of one tile.  A sequence's units are
// numbered (KV head, range, tile from the last to the first): those that read the same keys are neighbours.
//
// One number, the candidate, fixes all splits: sequence b has ceil(candidate * key tiles of b / key tiles of the longest), so that the
// ranges of all sequences are about equally long.
#pragma once

#include <math.h>
#include <stdint.h>

namespace rtp {

constexpr int kChunkRows = 256;          // rows of a query tile
constexpr int kChunkMaxHeads = 128;
constexpr int kChunkMostKeyTiles = 1 << 22;
constexpr int kChunkCandidates = 64;
// What a unit costs beside its key tiles, in key tiles: its way to the first product; its partial results, written and merged.
constexpr int kChunkUnitCost = 3, kChunkPartCost = 2;

struct ChunkShape {
  int32_t B, total_q, max_q;
  int32_t n_slots;                       // KV heads with served query heads
  int32_t local, sink, window;
  int32_t cap;                           // most units of tiles that are cut into ranges
  int32_t n_cu;
  uint16_t tok[9];                       // tokens per tile with n heads per KV head
  uint16_t cnt[9];                       // KV heads with n heads
  uint8_t slot_kv[kChunkMaxHeads], slot_n[kChunkMaxHeads], slot_first[kChunkMaxHeads];   // a slot's KV head, number of heads, first of them
  uint8_t heads[kChunkMaxHeads];         // served query heads, ascending
};

__host__ __device__ __forceinline__ int chunk_min(int a, int b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ int chunk_max(int a, int b) { return a > b ? a : b; }
__host__ __device__ __forceinline__ int chunk_div_up(int a, int b) { return (int)(((uint32_t)a + (uint32_t)b - 1u) / (uint32_t)b); }

// Splits of the longest sequence that candidate i (0 .. 63) stands for: 1 .. 32, then 40, 48 .. 288.
__host__ __device__ __forceinline__ int chunk_candidate(int i) { return i < 32 ? i + 1 : 32 + 8 * (i - 31); }

// Query tiles of a sequence with n new tokens, over all KV heads.
__host__ __device__ __forceinline__ int chunk_tiles(const ChunkShape& s, int n) {
  int t = 0;
  for (int h = 1; h <= 8; ++h)
    if (s.cnt[h]) t += s.cnt[h] * chunk_div_up(n, s.tok[h]);
  return t;
}
// 64-key tiles that one of its query tiles reads (a middling one).
__host__ __device__ __forceinline__ int chunk_key_tiles(const ChunkShape& s, int n, int ctx) {
  int keys = chunk_max(ctx - n / 2, 1);
  if (s.local) {
    const int64_t band = (int64_t)s.sink + s.window + chunk_min(n, 64);
    if (band < keys) keys = (int)band;
  }
  return chunk_max(1, chunk_min(chunk_div_up(keys, 64), kChunkMostKeyTiles));
}
// (whole numbers only: every launch of a call comes to the same splits)
__host__ __device__ __forceinline__ uint32_t chunk_magic(int longest) { return 0xffffffffu / (uint32_t)longest; }
__host__ __device__ __forceinline__ int chunk_splits(int key_tiles, int longest, int candidate, uint32_t magic) {
  const uint32_t x = (uint32_t)key_tiles * (uint32_t)candidate + (uint32_t)longest - 1u;      // at most 2^22 * 289
  return chunk_max(1, (int)(((uint64_t)x * magic) >> 32));
}
// What a candidate costs: rounds of units over the compute units, each as long as the mean one.
__host__ __device__ __forceinline__ float chunk_float(uint64_t x) {      // (in halves: no shift by a count of leading zeros)
  return fmaf((float)(uint32_t)(x >> 32), 4294967296.f, (float)(uint32_t)x);
}
__host__ __device__ __forceinline__ uint32_t chunk_cost(uint64_t work, uint64_t units, uint64_t split_units, int n_cu) {
  if (units > (1u << 26)) return 0x3ffffffu;
  const uint32_t u = units > 0 ? (uint32_t)units : 1u;
  const float length = chunk_float(work) / (float)u;
  const uint32_t rounds = (u + (uint32_t)n_cu - 1u) / (uint32_t)n_cu;
  const uint64_t each = (length < 67108864.f ? (uint32_t)length : 67108864u) + 1u + kChunkUnitCost + (split_units ? kChunkPartCost : 0);
  const uint64_t cost = rounds * each;
  return cost < 0x3ffffffu ? (uint32_t)cost : 0x3ffffffu;
}

struct ChunkUnit {
  int slot, split, tile;
};
// Unit r of a sequence with n new tokens and S splits.
__host__ __device__ __forceinline__ ChunkUnit chunk_unit(const ChunkShape& s, int n, int S, int r) {
  int slot = 0, tiles = 1;
  for (; slot < s.n_slots; ++slot) {
    tiles = chunk_div_up(n, s.tok[s.slot_n[slot]]);
    if (r < tiles * S) break;
    r -= tiles * S;
  }
  const int split = (int)((uint32_t)r / (uint32_t)tiles);
  return ChunkUnit{slot, split, tiles - 1 - (r - split * tiles)};
}
// The other way round: the number of (slot, range 0, tile) and the step from range to range.
__host__ __device__ __forceinline__ int chunk_unit_of(const ChunkShape& s, int n, int S, int slot, int tile, int* step) {
  int r = 0;
  for (int k = 0; k < slot; ++k) r += chunk_div_up(n, s.tok[s.slot_n[k]]) * S;
  *step = chunk_div_up(n, s.tok[s.slot_n[slot]]);
  return r + *step - 1 - tile;
}

}  // namespace rtp
