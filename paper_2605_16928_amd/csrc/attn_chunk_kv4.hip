// The attention of attn_chunk.hip with the 4-bit cache as the source of K and V.
#include "chunk_kernels.h"

namespace rtp {

RTP_CHUNK_KERNELS(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true)

// No tile has more than 16 rows.
template <bool F16, bool LOCAL, int NW>
__global__ __launch_bounds__(NW * 64, NW == kCkSmallWaves ? 3 : 2) void chunk_slim_kv4_kernel(const ChunkArgs a) {
  fetch_arguments<ChunkArgs>();
  __shared__ __attribute__((aligned(16))) unsigned char smem[chunk_slim_lds(NW)];
  ChunkTile t;
  if (!chunk_tile<LOCAL, true>(a, blockIdx.x, &t)) return;
  if (ChunkSlim<F16, LOCAL, NW, false>(a, t, smem).run()) ChunkSlim<F16, LOCAL, NW, true>(a, t, smem).run();
}

void launch_chunk_kv4(const ChunkArgs& a, unsigned grid, int rows, bool few, hipStream_t stream) {
  const bool narrow = rows <= kCkNarrowRows;
  if (rows <= kCkSlimRows) {
#define RTP_SLIM(F16_, LOCAL_)                                                                                                            \
  if ((a.f16 != 0) == F16_ && (a.shape.local != 0) == LOCAL_) {                                                                           \
    if (few) RTP_LAUNCH((chunk_slim_kv4_kernel<F16_, LOCAL_, kCkWaves>), dim3(grid), dim3(kCkThreads), 0, stream, a);                     \
    else RTP_LAUNCH((chunk_slim_kv4_kernel<F16_, LOCAL_, kCkSmallWaves>), dim3(grid), dim3(kCkSmallWaves * 64), 0, stream, a);            \
  }
    RTP_SLIM(false, false)
    RTP_SLIM(true, false)
    RTP_SLIM(false, true)
    RTP_SLIM(true, true)
#undef RTP_SLIM
    return;
  }
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, false, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, false, true)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true, true)
}

}  // namespace rtp
