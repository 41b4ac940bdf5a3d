// The kernels of the attention of a batch of new tokens, for either cache.
#pragma once

#include "chunk_slim.h"

namespace rtp {

// The kernels.  ANY: tiles of any size; what has to be taken again is noted by workgroup, for AGAIN, each size in its own way.  NARROW: where the host knows that no tile has
// more than 32 rows; takes its tiles again itself.  Workgroups of four waves, two to a compute unit, whose beginnings and ends lie beside the other's
// middle; of eight where there are no more units than compute units (`few`): one token of 2 KV heads over 700 keys, whole, 11.7 us with eight and 13.6 with four.
#define RTP_CHUNK_KERNELS(ANY, AGAIN, NARROW, KV4)                                                                      \
  template <bool F16, bool LOCAL, bool FULL>                                                                            \
  __global__ __launch_bounds__(kCkThreads, 2) void ANY(const ChunkArgs a) {                                             \
    fetch_arguments<ChunkArgs>();                                                                                       \
    __shared__ __attribute__((aligned(16))) unsigned char smem[kCkLds];                                                 \
    ChunkTile t;                                                                                                        \
    bool again = false;                                                                                                 \
    if (chunk_tile<LOCAL, KV4>(a, blockIdx.x, &t)) {                                                                    \
      if (t.rows <= kCkNarrowRows) {                                                                                    \
        again = ChunkNarrow<F16, LOCAL, KV4, kCkWaves, false>(a, t, smem).run();                                        \
      } else {                                                                                                          \
        ChunkWide<F16, LOCAL, KV4, FULL> w(a, t, smem);                                                                 \
        if (t.it_lo < t.it_hi) {                                                                                        \
          again = w.fast_pass();                                                                                        \
        } else {                                                                                                        \
          w.m = -__builtin_huge_valf();                                                                                 \
          w.clear();                                                                                                    \
        }                                                                                                               \
        if (!again) w.store();                                                                                          \
      }                                                                                                                 \
    }                                                                                                                   \
    if (threadIdx.x == 0) a.again[blockIdx.x] = again ? 1 : 0;                                                          \
  }                                                                                                                     \
  template <bool F16, bool LOCAL>                                                                                       \
  __global__ __launch_bounds__(kCkThreads, 2) void AGAIN(const ChunkArgs a, int n) {                                    \
    __shared__ __attribute__((aligned(16))) unsigned char smem[kCkLds];                                                 \
    int any = 0;                                                        /* (the usual end, before anything else) */      \
    for (int64_t i = blockIdx.x + (int64_t)threadIdx.x * gridDim.x; i < n; i += (int64_t)kCkThreads * gridDim.x) any |= a.again[i]; \
    if (!__syncthreads_or(any)) return;                                                                                 \
    fetch_arguments<ChunkArgs>();                                                                                       \
    for (int i = blockIdx.x; i < n; i += gridDim.x) {                                                                   \
      ChunkTile t;                                                                                                      \
      if (a.again[i] == 0 || !chunk_tile<LOCAL, KV4>(a, i, &t)) continue;                                               \
      __syncthreads();                                                                                                  \
      if (t.rows <= kCkNarrowRows) {                                                                                    \
        (void)ChunkNarrow<F16, LOCAL, KV4, kCkWaves, true>(a, t, smem).run();                                           \
      } else {                                                                                                          \
        ChunkWide<F16, LOCAL, KV4, true> w(a, t, smem);                                                                 \
        w.exact_pass();                                                                                                 \
        w.store();                                                                                                      \
      }                                                                                                                 \
    }                                                                                                                   \
  }                                                                                                                     \
  template <bool F16, bool LOCAL, int NW>                                                                               \
  __global__ __launch_bounds__(NW * 64, 2) void NARROW(const ChunkArgs a) {                                             \
    fetch_arguments<ChunkArgs>();                                                                                       \
    __shared__ __attribute__((aligned(16))) unsigned char smem[chunk_narrow_lds(NW)];                                   \
    ChunkTile t;                                                                                                        \
    if (!chunk_tile<LOCAL, KV4>(a, blockIdx.x, &t)) return;                                                             \
    if (ChunkNarrow<F16, LOCAL, KV4, NW, false>(a, t, smem).run()) ChunkNarrow<F16, LOCAL, KV4, NW, true>(a, t, smem).run(); \
  }
// Launches those that a call's flags name.
#define RTP_CHUNK_LAUNCH(ANY, AGAIN, NARROW, F16_, LOCAL_)                                                              \
  if ((a.f16 != 0) == F16_ && (a.shape.local != 0) == LOCAL_) {                                                         \
    if (narrow && few) {                                                                                                \
      RTP_LAUNCH((NARROW<F16_, LOCAL_, kCkWaves>), dim3(grid), dim3(kCkThreads), 0, stream, a);                         \
    } else if (narrow) {                                                                                                \
      RTP_LAUNCH((NARROW<F16_, LOCAL_, kCkSmallWaves>), dim3(grid), dim3(kCkSmallWaves * 64), 0, stream, a);            \
    } else {                                                                                                            \
      if (a.lse) RTP_LAUNCH((ANY<F16_, LOCAL_, true>), dim3(grid), dim3(kCkThreads), 0, stream, a);                     \
      else RTP_LAUNCH((ANY<F16_, LOCAL_, false>), dim3(grid), dim3(kCkThreads), 0, stream, a);                          \
      RTP_LAUNCH((AGAIN<F16_, LOCAL_>), dim3(grid < 256 ? grid : 256), dim3(kCkThreads), 0, stream, a, (int)grid);      \
    }                                                                                                                   \
  }

}  // namespace rtp
