// The 16-bit K/V cache in pages: where a token's rows lie, and the checks of its descriptor and of a batch of new tokens
// (kv_append.hip fills it, attn_chunk.hip attends over it).
#pragma once

#include "common.h"

namespace rtp {

struct Kv16Cache {
  uint8_t* K;
  uint8_t* V;
  int64_t head_bytes, page_bytes;
  int32_t row_bytes;
  int32_t page_shift, n_pages;
  const int32_t* page_table;
  int64_t pt_stride;
};

int32_t check_kv16_cache(const char* who, const rtp_layer_desc* L, const rtp_kv_cache* c, int64_t max_tokens, Kv16Cache* out);
// q_offset, ctx_len and the bounds; total_q = 0 is allowed.
int32_t check_chunk(const char* who, const rtp_chunk* c);
// n rows of width elements at multiples of two strides: refuses what overlaps without being the same rows at the same places.
bool rows_overlap(const void* x, int64_t x_stride, int64_t x_width, const void* y, int64_t y_stride, int64_t y_width, int64_t n);

constexpr int kMaxSeqs = 65535;

// A sequence's new tokens among the packed rows, whatever the offsets hold: never outside [0, total), never more than most.
struct NewTokens {
  int q0, n;
};
__device__ __forceinline__ NewTokens new_tokens(const int32_t* off, int b, int total, int most) {
  const int q0 = min(max(off[b], 0), total), q1 = min(max(off[b + 1], q0), total);
  return NewTokens{q0, min(q1 - q0, most)};
}

// The last entry i in [0, n) of an ascending list with list[i] <= x (0 where there is none), by a whole wave: 64 entries a step.
__device__ __forceinline__ int wave_last_at_most(const int32_t* list, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 63) >> 6, at = lo + lane * step;
    const bool below = lane * step < len && list[at] <= x;
    const int count = __popcll(__ballot(below));
    if (count == 0) return 0;
    lo += (count - 1) * step;
    len = min(step, n - lo);
  }
  return lo;
}

}  // namespace rtp
