// The attention of attn_chunk.hip with the 4-bit cache as the source of K and V.
#include "chunk_narrow.h"

namespace rtp {

template <bool F16, bool LOCAL, bool FULL>
__global__ __launch_bounds__(kCkThreads, 2) void chunk_attn_kv4_kernel(const ChunkArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[kCkLds];
  chunk_unit_attend<F16, LOCAL, true, FULL>(a, smem);
}

void launch_chunk_kv4(const ChunkArgs& a, unsigned grid, bool local, bool full, hipStream_t stream) {
#define RTP_CHUNK(F16, LOCAL, FULL)                         \
  if ((a.f16 != 0) == F16 && local == LOCAL && full == FULL) \
    RTP_LAUNCH((chunk_attn_kv4_kernel<F16, LOCAL, FULL>), dim3(grid), dim3(kCkThreads), 0, stream, a);
  RTP_CHUNK(false, false, false)
  RTP_CHUNK(true, false, false)
  RTP_CHUNK(false, true, false)
  RTP_CHUNK(true, true, false)
  RTP_CHUNK(false, false, true)
  RTP_CHUNK(true, false, true)
  RTP_CHUNK(false, true, true)
  RTP_CHUNK(true, true, true)
#undef RTP_CHUNK
}

}  // namespace rtp
