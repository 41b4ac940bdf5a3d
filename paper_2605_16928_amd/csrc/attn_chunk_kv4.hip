// The attention of attn_chunk.hip with the 4-bit cache as the source of K and V.
#include "chunk_narrow.h"

namespace rtp {

RTP_CHUNK_KERNELS(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true)

void launch_chunk_kv4(const ChunkArgs& a, unsigned grid, bool narrow, hipStream_t stream) {
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, false, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, false, true)
  RTP_CHUNK_LAUNCH(chunk_attn_kv4_kernel, chunk_again_kv4_kernel, chunk_narrow_kv4_kernel, true, true)
}

}  // namespace rtp
