// Whether the probabilities of a row were good enough against a fixed reference (chunk_wide.h), from their sum.  Apart from the kernels so that it also
// compiles for the host.
//
// The reference is the row's largest score in its range's first tile (fp16: or in the first tile that every row sees in full), or, where the row sees
// nothing there, the largest of what it does not see, which says nothing of what it sees.  bf16 has the range of fp32: only sums near its ends need another reference.  fp16 ends at 65504, which the sum shows as
// an infinity, and below 2^-14 a probability is off by up to 2^-25 whatever its size: n of them by n 2^-25 together, which is within 2^-12 of a
// sum of n 2^-13.  A row that sees its reference (`held`) needs no such sum: most of its probabilities are not that much smaller.
#pragma once

#include <stdint.h>

namespace rtp {

// Enough, whatever the row sees.  (Half of what the reference's own probability adds, which is 1 but for roundings of scores above 2^12.)
constexpr float chunk_sure(bool f16) { return f16 ? 0x1p-1f : 0x1p-60f; }
__host__ __device__ __forceinline__ bool chunk_surely_in_reach(bool f16, bool held, float sum) { return (held || !f16) && sum > chunk_sure(f16); }
// The sum of a row that sees `seen` keys of the range.
__host__ __device__ __forceinline__ bool chunk_in_reach(bool f16, bool held, float sum, int seen) {
  return chunk_surely_in_reach(f16, held, sum) || seen <= 0 || (f16 && sum > (float)seen * 0x1p-13f);
}
// How many of the keys [from, end) a row sees: those up to hi that are below the sink or above lo (local), or all of them up to hi.
__host__ __device__ __forceinline__ int chunk_seen_among(int from, int end, bool local, int sink, int lo, int hi) {
  end = end <= hi ? end : hi + 1;
  if (!local) return end > from ? end - from : 0;
  const int sink_end = sink < end ? sink : end;
  int band = lo + 1 > sink ? lo + 1 : sink;
  band = band > from ? band : from;
  return (sink_end > from ? sink_end - from : 0) + (end > band ? end - band : 0);
}

}  // namespace rtp
