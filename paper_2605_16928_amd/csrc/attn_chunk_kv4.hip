// The attention of attn_chunk.hip with the 4-bit cache as the source of K and V.
#include "chunk_kernels.h"

namespace rtp {

RTP_CHUNK_KERNELS(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true)

// No tile has more than 16 rows.
template <bool F16, bool LOCAL>
__global__ __launch_bounds__(kCkSmallWaves * 64, 3) void chunk_slim_kv4_kernel(const ChunkArgs a) {
  fetch_arguments<ChunkArgs>();
  __shared__ __attribute__((aligned(16))) unsigned char smem[chunk_slim_lds(kCkSmallWaves)];
  ChunkTile t;
  if (!chunk_tile<LOCAL, true>(a, blockIdx.x, &t)) return;
  if (ChunkSlim<F16, LOCAL, kCkSmallWaves, false>(a, t, smem).run()) ChunkSlim<F16, LOCAL, kCkSmallWaves, true>(a, t, smem).run();
}

void launch_chunk_kv4(const ChunkArgs& a, unsigned grid, int rows, hipStream_t stream) {
  const bool narrow = rows <= kCkNarrowRows;
  if (rows <= kCkSlimRows) {
    const dim3 g(grid), b(kCkSmallWaves * 64);
    if (a.f16 && a.shape.local) RTP_LAUNCH((chunk_slim_kv4_kernel<true, true>), g, b, 0, stream, a);
    else if (a.f16) RTP_LAUNCH((chunk_slim_kv4_kernel<true, false>), g, b, 0, stream, a);
    else if (a.shape.local) RTP_LAUNCH((chunk_slim_kv4_kernel<false, true>), g, b, 0, stream, a);
    else RTP_LAUNCH((chunk_slim_kv4_kernel<false, false>), g, b, 0, stream, a);
    return;
  }
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, false, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, false, true)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true, true)
}

}  // namespace rtp
