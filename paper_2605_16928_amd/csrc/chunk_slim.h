// A query tile of up to 16 rows over the 4-bit cache: single tokens and short drafts.  At 136 bytes per key the vector ALU is as near a limit as HBM
// is, so the products are those of 16 rows (v_mfma_f32_16x16x32): a lane has 8 probabilities per 32 keys where chunk_narrow.h's has 16, and with 40
// registers of state there is room for three workgroups on a compute unit.  8 contexts of 131072, 4 tokens of 32 over 8 heads (1.14 GB) 225 us with the
// merge, 5.0 TB/s; with chunk_narrow.h's products of 32 rows 361.
//
// As there, a wave takes blocks of 32 keys on its own, two ahead in registers, and puts them in operand order by way of its LDS:
//   S^T = K Q^T   A: lane (c, g) has the dims 32 g .. + 31 of token c of 16 -- 16 bytes, one scale; B: the queries alike.
//   O^T = V^T P^T B: lane (c, g) has the probabilities of row c and of the tokens 16 s + 4 g + i, as the scores left them; A: the same tokens, of each
//                 the word with the dims 8 c .. + 7, one to each of the eight accumulators: accumulator n, lane (c, g), i holds dim 32 g + 8 i + n of row c.
#pragma once

#include "chunk_narrow.h"

namespace rtp {

constexpr int kCkSlimRows = 16;
constexpr int kCkSlimWave = kCkSlimRows * kHeadDim * 4;                     // LDS of a wave: 16 rows of 128 outputs; before, 32 records and their scales
constexpr int chunk_slim_lds(int waves) { return waves * (kCkSlimWave + kCkSlimRows * 2 * 4); }
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <bool F16>
__device__ __forceinline__ f32x4 chunk_mfma16(const u32x4 a, const u32x4 b, const f32x4 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool F16, bool LOCAL, int NW, bool CARE>
struct ChunkSlim {
  const ChunkArgs& a;
  const ChunkTile& t;
  unsigned char* const smem;
  const int lane, wave, g, c;
  unsigned char* const mine;
  const float scale;
  const ChunkSight sight;
  ChunkBlocks<LOCAL, true, NW> blocks;
  u32x4 q[4];
  f32x4 O[8];
  float m, l;

  __device__ __forceinline__ ChunkSlim(const ChunkArgs& a_, const ChunkTile& t_, unsigned char* smem_)
      : a(a_), t(t_), smem(smem_), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), g(lane >> 4), c(lane & 15),
        mine(smem_ + wave * kCkSlimWave), scale(a_.scale_log2), sight(chunk_sight(a_.shape, t_, min(lane & 15, t_.rows - 1))), blocks(a_, t_) {
    const int row_c = min(c, t.rows - 1), rt = (row_c * t.over) >> 16;
    const uint16_t* src = a.q + (t.q0 + rt) * a.q_stride + chunk_head(a, t, row_c, rt) * kHeadDim + g * 32;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) q[kk] = *reinterpret_cast<const u32x4*>(src + kk * 8);
    m = -__builtin_huge_valf();
    l = 0.f;
#pragma unroll
    for (int n = 0; n < 8; ++n) O[n] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  __device__ __forceinline__ void step(typename ChunkBlocks<LOCAL, true, NW>::Codes& y, int& k, int behind) {
    const float ninf = -__builtin_huge_valf();
    chunk_put_records(mine, y);
    const int n0 = blocks.n0(k);
    k = blocks.next_seen(behind + 1);
    if (k < blocks.count) {
      blocks.advance(k);
      blocks.fetch(k, y);
    }
    const unsigned char* const sc = mine + kCkScalesAt;
    f32x4 S[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(mine + chunk_record_at(16 * s + c, g));
      const float f = __uint_as_float((uint32_t)sc[(4 * s + (c >> 2)) * kKv4Group + g * 4 + (c & 3)] << 23);
      S[s] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) S[s] = chunk_mfma16<F16>(decode8<F16>(w[kk], f), q[kk], S[s]);
    }
    // ---- what the row does not see; the reference ----
    uint32_t seen = 0xffu;                                                  // bit 4 s + i: key n0 + 16 s + 4 g + i
    if (CARE || !chunk_all_seen<LOCAL>(a.shape, t, t.m_lo, t.m_hi, n0, 32)) {
      seen = 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int n4 = n0 + 16 * s + 4 * g;
        const ChunkSight e = {sight.hi - n4, sight.lo - n4, sight.sink - n4};
        bool there = true;
        if constexpr (CARE) there = n4 < t.kend && chunk_page<true>(a, t, min(n4, t.kend - 1)) >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool ok = there && chunk_sees<LOCAL>(e, i);
          seen |= ok ? 1u << (4 * s + i) : 0u;
          S[s][i] = ok ? S[s][i] : ninf;
        }
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
    if (__ballot((mx - m) * scale > kCkLag<F16> || (m == ninf && mx > ninf)) != 0ull) {
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m, mx), corr = m_new == ninf ? 1.f : fast_exp2((m - m_new) * scale);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int n = 0; n < 8; ++n) O[n] *= corr;
    }
    const float mc = (m == ninf ? 0.f : m * scale) - kCkLift<F16>;
    u32x4 P, R;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const float p0 = fast_exp2(fmaf(S[s][i], scale, -mc)), p1 = fast_exp2(fmaf(S[s][i + 1], scale, -mc));
        const uint32_t w = pack16<F16>(p0, p1);
        l += p0 + p1;
        P[2 * s + (i >> 1)] = w;
        R[2 * s + (i >> 1)] = pack16<F16>(p0 - lo16<F16>(w), p1 - hi16<F16>(w));
      }
    // ---- V: 8 tokens x 8 dims ----
    uint32_t v[2][4], vs[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      vs[s] = *reinterpret_cast<const uint32_t*>(sc + (4 * s + g) * kKv4Group + 16 + (c >> 2) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[s][i] = *reinterpret_cast<const uint32_t*>(mine + chunk_record_at(16 * s + 4 * g + i, 4 + (c >> 2)) + (c & 3) * 4);
    }
    float f[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[s][i] = kv4_scale(vs[s], i);
        if constexpr (CARE) f[s][i] = f[s][i] < kKv4Large<F16> ? f[s][i] : 0.f;
      }
#define RTP_SLIM_PV(B)                                                                                                                \
  {                                                                                                                                   \
    u32x4 even, odd;                                                                                                                  \
    _Pragma("unroll") for (int s = 0; s < 2; ++s) _Pragma("unroll") for (int i = 0; i < 4; i += 2) {                                    \
      if constexpr (F16) {                                                                                                            \
        const f32x2_t x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[s][i], f[s][i], B);                                                \
        const f32x2_t y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[s][i + 1], f[s][i + 1], B);                                        \
        even[2 * s + (i >> 1)] = pack16<true>(x.x, y.x);                                                                                \
        odd[2 * s + (i >> 1)] = pack16<true>(x.y, y.y);                                                                                 \
      } else {                                                                                                                        \
        const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[s][i], f[s][i], B));                \
        const uint32_t y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[s][i + 1], f[s][i + 1], B));        \
        even[2 * s + (i >> 1)] = __builtin_amdgcn_perm(y, x, 0x05040100u);                                                              \
        odd[2 * s + (i >> 1)] = __builtin_amdgcn_perm(y, x, 0x07060302u);                                                               \
      }                                                                                                                               \
    }                                                                                                                                 \
    O[2 * B] = chunk_mfma16<F16>(even, P, O[2 * B]);                                                                                    \
    O[2 * B + 1] = chunk_mfma16<F16>(odd, P, O[2 * B + 1]);                                                                             \
    O[2 * B] = chunk_mfma16<F16>(even, R, O[2 * B]);                                                                                    \
    O[2 * B + 1] = chunk_mfma16<F16>(odd, R, O[2 * B + 1]);                                                                             \
  }
    RTP_SLIM_PV(0)
    RTP_SLIM_PV(1)
    RTP_SLIM_PV(2)
    RTP_SLIM_PV(3)
#undef RTP_SLIM_PV
    if constexpr (CARE) {
      // the blocks of V that may hold infinities, token by token and over the seen ones alone: dims 32 g + 8 e + n, block g
#pragma unroll 1
      for (int k = 0; k < 32; ++k) {                                        // key 16 s + 4 (from's g) + i
        if (!chunk_large<F16>(mine, k)) continue;
        const int i = k & 3, own = 4 * (k >> 4) + i, from = ((k >> 2) & 3) * 16 + c;
        uint32_t w = P[0], x = R[0];
#pragma unroll
        for (int e = 1; e < 4; ++e) {
          w = e == (own >> 1) ? P[e] : w;
          x = e == (own >> 1) ? R[e] : x;
        }
        const float p = __shfl((i & 1) ? hi16<F16>(w) + hi16<F16>(x) : lo16<F16>(w) + lo16<F16>(x), from);
        const float f_own = chunk_value_scale(mine, k, g);
        const bool ok = (((uint32_t)__shfl((int)seen, from) >> own) & 1u) && f_own >= kKv4Large<F16> && f_own < __builtin_huge_valf();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const u32x4 y = decode8<F16>(*reinterpret_cast<const uint32_t*>(mine + chunk_record_at(k, 4 + g) + e * 4), f_own);
#pragma unroll
          for (int n = 0; n < 8; ++n) O[n][e] = ok ? fmaf(p, (n & 1) ? hi16<F16>(y[n >> 1]) : lo16<F16>(y[n >> 1]), O[n][e]) : O[n][e];
        }
      }
      // rows that see a token whose V has a block that is not a number have none there either: dims 32 g + 8 i + n, block g
      uint32_t hit = 0;                                                     // of the lane's own tokens, bit: block
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int blk = 0; blk < 4; ++blk)
            hit |= ((seen >> (4 * s + i)) & 1u) && sc[(4 * s + g) * kKv4Group + 16 + blk * 4 + i] == 255 ? 1u << blk : 0u;
      hit |= (uint32_t)__shfl_xor((int)hit, 16);
      hit |= (uint32_t)__shfl_xor((int)hit, 32);
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) O[n][i] = (hit >> g) & 1u ? __builtin_nanf("") : O[n][i];
    }
  }

  // true: a page was not there or a result is not finite (never with CARE)
  __device__ __forceinline__ bool run() {
    if (blocks.count > 0) {
      typename ChunkBlocks<LOCAL, true, NW>::Codes x[2];
      int at[2];
      at[0] = blocks.next_seen(0);
      at[1] = blocks.next_seen(at[0] + 1);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (at[u] < blocks.count) {
          blocks.advance(at[u]);
          blocks.fetch(at[u], x[u]);
        }
      while (at[0] < blocks.count) {
        step(x[0], at[0], at[1]);
        if (at[1] >= blocks.count) break;
        step(x[1], at[1], at[0]);
      }
    }
    float z = 0.f;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) z = fmaf(O[n][i], 0.f, z);
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if constexpr (CARE) __syncthreads();
    else if (__syncthreads_or(blocks.lost || !(z == 0.f) || !(l < 0x1p120f) ? 1 : 0) != 0) return true;
    // ---- the waves' results, joined: group d of four outputs of row c at d ^ 2 c ----
    float* const sh_m = reinterpret_cast<float*>(smem + NW * kCkSlimWave);
    float* const sh_l = sh_m + NW * kCkSlimRows;
    if (g == 0) {
      sh_m[wave * kCkSlimRows + c] = m;
      sh_l[wave * kCkSlimRows + c] = l;
    }
    if (c < t.rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int d = 8 * g + 2 * i + half;
          *reinterpret_cast<float4*>(mine + c * 512 + ((d ^ (2 * c)) & 31) * 16) =
              make_float4(O[4 * half][i], O[4 * half + 1][i], O[4 * half + 2][i], O[4 * half + 3][i]);
        }
    }
    __syncthreads();
    constexpr int kLanes = NW * 64 / kCkSlimRows, kEach = kHeadDim / 4 / kLanes;
    const int row = threadIdx.x / kLanes, d0 = threadIdx.x % kLanes;
    if (row >= t.rows) return false;
    const float ninf = -__builtin_huge_valf();
    float M = ninf, L = 0.f, o[kEach][4] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sh_m[w * kCkSlimRows + row]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float m_w = sh_m[w * kCkSlimRows + row], cw = m_w == ninf ? 1.f : fast_exp2((m_w - M) * scale);   // (no finite logit: the sum is 0, or none)
      L += sh_l[w * kCkSlimRows + row] * cw;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int d = d0 + kLanes * e;
        const float4 v = *reinterpret_cast<const float4*>(smem + w * kCkSlimWave + row * 512 + ((d ^ (2 * row)) & 31) * 16);
        o[e][0] = fmaf(v.x, cw, o[e][0]);
        o[e][1] = fmaf(v.y, cw, o[e][1]);
        o[e][2] = fmaf(v.z, cw, o[e][2]);
        o[e][3] = fmaf(v.w, cw, o[e][3]);
      }
    }
    chunk_lower<F16>(L, o);
#pragma unroll
    for (int e = 0; e < kEach; ++e) chunk_store4<F16>(a, t, row, 4 * (d0 + kLanes * e), M, L, L, o[e]);
    return false;
  }
};

}  // namespace rtp
