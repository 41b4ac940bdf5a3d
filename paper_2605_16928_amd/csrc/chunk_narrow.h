// A query tile of up to 32 rows -- single tokens, drafts, the ends of chunks: bound by the bytes of K and V.  All rows fit one wave, so the waves of
// the workgroup take blocks of 32 keys in turn, each on its own: no barrier until their results are joined in LDS.
//
// 16-bit rows: a wave owns 16 KiB, K and V of one block.  The next K sets out when the scores have been computed, the next V behind the PV product;
// eight waves at different places keep 64 to 128 KiB of a compute unit's loads in flight, without a second buffer.
// 4-bit rows: a block is 4 KiB and 256 bytes of scales, two blocks ahead in registers, loaded as whole lines and put in operand order by way of the
// wave's LDS:  K: lane (g, r) takes the dims 64 g .. + 63 of token r, and the queries lie alike, so that a word of codes is one product's operand;
// V: lane (g, r) takes the dims 4 r .. + 3 (two bytes) of its 16 tokens, so that accumulator db holds the dims 4 rho + db.
//
// Measured: 32 single tokens over 1500 to 30000 keys, 32 over 8 heads (1.1 GB) 203 us with the merge, 5.4 TB/s, where a copy reaches 4.9;
// as wide tiles, whose buffers the whole workgroup fills and passes on at barriers, 1074.  Bound by HBM; one token over 700 keys takes 7.0 + 2.4: the launches, code that
// comes from memory for the first time, and four dependent loads.
//
// The running reference follows a row's maximum only when it is left behind by more than 2^8.  Probabilities enter the product in two parts, their
// rounding to 16 bits and the rounding of the rest: the matrix cores have the time, and an output is then as exact as its own rounding.  fp16 ends
// at 2^16 and at 2^-24, where nothing is left for a second part: there probabilities are taken times 2^13, against a reference that follows at 2^2, so
// that one is whole down to 2^-27 of its row's largest and gone below 2^-38 (all of 2^20 tokens together then 2^-18 of it).
//
// Where a page was not there or a result is not finite, the tile is taken again with care: keys are masked by their pages too, and what a row does
// not see does not reach it, whatever it holds.
#pragma once

#include "chunk_wide.h"

namespace rtp {

constexpr int kCkNarrowRows = 32;
constexpr int kCkBlockBytes = 2 * 32 * kHeadDim * 2;                        // K and V of 32 keys; 32 rows of 128 outputs
constexpr int chunk_narrow_lds(int waves) { return waves * (kCkBlockBytes + kCkNarrowRows * 2 * 4); }
constexpr int kCkLds = chunk_narrow_lds(kCkWaves) > kCkWideLds ? chunk_narrow_lds(kCkWaves) : kCkWideLds;

// The blocks of 32 keys that a wave takes, and where their rows lie: block k of wave w is block w + NW k of the range.
template <bool LOCAL, bool KV4, int NW>
struct ChunkBlocks {
  const ChunkArgs& a;
  const ChunkTile& t;
  const int lane, wave, g;
  const int count;
  const uint8_t* base0;                          // K or codes, V or scales, of the KV head
  const uint8_t* base1;
  uint32_t at_lo, at_hi, sc_lo, sc_hi;           // places of half blocks (16 keys lie in one page), two per block, of 32 blocks
  int next_page, window;
  bool lost;                                     // a page that some row sees was not there; the first was taken for it

  __device__ __forceinline__ ChunkBlocks(const ChunkArgs& a_, const ChunkTile& t_)
      : a(a_), t(t_), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), g(lane >> 5),
        count((blocks_of(t_) - wave + NW - 1) / NW), window(-2), lost(false) {
    if constexpr (KV4) {
      base0 = a.c4.codes + (int64_t)t.kvh * a.c4.code_head_stride;
      base1 = a.c4.scales + (int64_t)t.kvh * a.c4.scale_head_stride;
    } else {
      base0 = a.c16.K + (int64_t)t.kvh * a.c16.head_bytes;
      base1 = a.c16.V + (int64_t)t.kvh * a.c16.head_bytes;
    }
  }

  // (without a band every block up to the last key is seen by some row)
  static __device__ __forceinline__ int blocks_of(const ChunkTile& t) {
    const int all = 2 * (t.it_hi - t.it_lo);
    return LOCAL ? all : min(all, ((t.kend + 31) >> 5) - 2 * t.it_lo);
  }
  // First key of the wave's block k.
  __device__ __forceinline__ int n0(int k) const {
    const int j = wave + k * NW;
    if (!LOCAL) return t.it_lo * kCkK + j * 32;
    return chunk_tile_n0(t, t.it_lo + (j >> 1)) + (j & 1) * 32;
  }
  __device__ __forceinline__ int next_seen(int k) const {
    if (!LOCAL) return k;
    while (k < count && !chunk_any_seen<LOCAL>(a.shape, t, t.m_lo, t.m_hi, n0(k), 32)) ++k;
    return k;
  }
  // First key of half h of block k, or, where that lies behind the last key, of the 16 that hold it.
  __device__ __forceinline__ int half_n0(int k, int h) const { return min(n0(min(k, count - 1)) + 16 * h, (t.kend - 1) & ~15); }
  __device__ __forceinline__ void look_up(int w) {
    next_page = t.pt[half_n0(w * 32 + (lane >> 1), lane & 1) >> (KV4 ? a.c4.page_shift : a.c16.page_shift)];
  }
  __device__ __forceinline__ void advance(int k) {
    const int w = k >> 5;
    if (w == window) return;
    if (w != window + 1) look_up(w);
    const int n = half_n0(w * 32 + (lane >> 1), lane & 1);
    const bool there = (uint32_t)next_page < (uint32_t)(KV4 ? a.c4.n_pages : a.c16.n_pages);
    const uint32_t page = there ? (uint32_t)next_page : 0u, slot = n & ((1 << (KV4 ? a.c4.page_shift : a.c16.page_shift)) - 1);
    lost = lost || __ballot(!there && (!LOCAL || chunk_any_seen<LOCAL>(a.shape, t, t.m_lo, t.m_hi, n, 16))) != 0ull;
    uint64_t at;
    if constexpr (KV4) {
      at = (uint64_t)page * a.c4.code_page16 * 16u + (uint64_t)slot * kKv4Row;
      const uint64_t sc = (uint64_t)page * a.c4.scale_page16 * 16u + (uint64_t)slot * (kKv4Group / 4);
      sc_lo = (uint32_t)sc;
      sc_hi = (uint32_t)(sc >> 32);
    } else {
      at = (uint64_t)page * (uint64_t)a.c16.page_bytes + (uint64_t)slot * (uint32_t)a.c16.row_bytes;
    }
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
    window = w;
    look_up(w + 1);
  }
  __device__ __forceinline__ int64_t place(uint32_t lo, uint32_t hi, int k, int h) const {
    const int p = (k & 31) * 2 + h;
    return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, p) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)lo, p));
  }
  // Keys of half h behind its first that are there.
  __device__ __forceinline__ int left(int k, int h) const { return t.kend - 1 - half_n0(k, h); }

  // ---- 4-bit records and their scales, as they come from memory ----
  struct Codes {
    u32x4 line[4];                               // token 8 i + lane / 8, 16 bytes of its 128
    uint32_t scales;                             // word lane % 8 of the scales of tokens 4 (lane / 8) .. + 3
  };
  __device__ __forceinline__ void fetch(int k, Codes& x) {
    const bool edge = n0(k) + 32 > t.kend;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int rel = 8 * (i & 1) + (lane >> 3);
      if (edge) rel = min(rel, left(k, i >> 1));
      x.line[i] = *reinterpret_cast<const u32x4*>(base0 + place(at_lo, at_hi, k, i >> 1) + rel * kKv4Row + (lane & 7) * 16);
    }
    const int64_t s0 = place(sc_lo, sc_hi, k, 0), s1 = place(sc_lo, sc_hi, k, 1);
    int group = (lane >> 3) & 3;
    uint32_t keep = 0xffffffffu;
    if (edge) {                                                             // (scales that nobody has written stay out: V times 0 has to be 0)
      const int have = left(k, g);
      group = min(group, have >> 2);
      if (group == have >> 2) keep >>= 24 - 8 * (have & 3);
    }
    x.scales = *reinterpret_cast<const uint32_t*>(base1 + (g ? s1 : s0) + group * kKv4Group + (lane & 7) * 4) & keep;
  }
};

// A record (K in the pieces 0 .. 3 of 16 bytes, V in the rest) and the scales of a wave's 32 tokens in its LDS.
__device__ __forceinline__ int chunk_record_at(int token, int piece) { return token * 128 + (piece ^ ((token >> 1) & 7)) * 16; }
constexpr int kCkScalesAt = 32 * kKv4Row;
template <typename Codes>
__device__ __forceinline__ void chunk_put_records(unsigned char* mine, const Codes& x) {
  const int lane = threadIdx.x & 63;
  chunk_wave_fence();
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(mine + chunk_record_at(8 * i + (lane >> 3), lane & 7)) = x.line[i];
  *reinterpret_cast<uint32_t*>(mine + kCkScalesAt + lane * 4) = x.scales;
  chunk_wave_fence();
}
// The reference is raised when it is left behind by more than 2^kCkLag; probabilities are taken times 2^kCkLift, results by as much less.
template <bool F16>
constexpr float kCkLag = F16 ? 2.f : 8.f;
template <bool F16>
constexpr float kCkLift = F16 ? 13.f : 0.f;
template <bool F16>
constexpr float kCkLower = F16 ? 0x1p-13f : 1.f;

template <bool F16, int N>
__device__ __forceinline__ void chunk_lower(float& L, float (&o)[N][4]) {
  if constexpr (F16) {
    L *= kCkLower<F16>;
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[e][i] *= kCkLower<F16>;
  }
}

// Blocks of this scale and above may hold values that are infinite in 16 bits: 4 or 6 times it (fp16: 2^16, the largest is 65504; bf16: 2^128).
template <bool F16>
constexpr float kKv4Large = F16 ? 0x1p14f : 0x1p126f;
// Scale of a block of token n's V; infinite: the block is not a number.
__device__ __forceinline__ float chunk_value_scale(const unsigned char* mine, int n, int block) {
  return __uint_as_float((uint32_t)mine[kCkScalesAt + (n >> 2) * kKv4Group + 16 + block * 4 + (n & 3)] << 23);
}
// Token n (the same for the whole wave) has such a block that is a number.
template <bool F16>
__device__ __forceinline__ bool chunk_large(const unsigned char* mine, int n) {
  const float f = chunk_value_scale(mine, n, threadIdx.x & 3);
  return __ballot(f >= kKv4Large<F16> && f < __builtin_huge_valf()) != 0ull;
}

template <bool F16, bool LOCAL, bool KV4, int NW, bool CARE>
struct ChunkNarrow {
  const ChunkArgs& a;
  const ChunkTile& t;
  unsigned char* const smem;
  unsigned char* const mine;                     // the wave's own LDS
  const int lane, wave, g, r;
  const float c;
  const ChunkReads rd;
  const ChunkSight sight;
  ChunkBlocks<LOCAL, KV4, NW> blocks;
  u32x4 q[8];
  f32x16 O[4];
  float m, l;

  __device__ __forceinline__ ChunkNarrow(const ChunkArgs& a_, const ChunkTile& t_, unsigned char* smem_)
      : a(a_), t(t_), smem(smem_), mine(smem_ + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kCkBlockBytes), lane(threadIdx.x & 63),
        wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), g(lane >> 5), r(lane & 31), c(a_.scale_log2), rd(chunk_reads()),
        sight(chunk_sight(a_.shape, t_, min(lane & 31, t_.rows - 1))), blocks(a_, t_) {
    const int row_c = min(r, t.rows - 1), rt = (row_c * t.over) >> 16;
    const uint16_t* src = a.q + (t.q0 + rt) * a.q_stride + chunk_head(a, t, row_c, rt) * kHeadDim + g * (KV4 ? 64 : 8);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) q[kk] = *reinterpret_cast<const u32x4*>(src + kk * (KV4 ? 8 : 16));
    m = -__builtin_huge_valf();
    l = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
  }

  // ---- 16-bit rows: eight loads of four rows for K, eight for V ----
  __device__ __forceinline__ void send(int k, bool v) {
    const uint32_t lds = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)mine + (v ? kCkBlockBytes / 2 : 0);
    const int sub = lane >> 4, pos = lane & 15;
    const uint8_t* const base = v ? blocks.base1 : blocks.base0;
    const int64_t half[2] = {blocks.place(blocks.at_lo, blocks.at_hi, k, 0), blocks.place(blocks.at_lo, blocks.at_hi, k, 1)};
    if (blocks.n0(k) + 32 <= t.kend) {
      const uint32_t off = sub * a.c16.row_bytes;
#pragma unroll
      for (int i = 0; i < 8; ++i) {                                         // row 4 (i % 4) + sub of its half
        const int chunk = v ? (((pos >> 1) ^ (2 * sub)) << 1) | (pos & 1) : pos ^ sub ^ (4 * (i & 3));
        chunk_load_lds(lds + i * 1024, base + half[i >> 2] + (i & 3) * 4 * a.c16.row_bytes, off + chunk * 16);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const int rel = 4 * (i & 3) + sub, chunk = v ? (((pos >> 1) ^ (2 * sub)) << 1) | (pos & 1) : pos ^ rel;
        chunk_load_lds(lds + i * 1024, base + (i < 4 ? half[0] : half[1]), (uint32_t)(min(rel, blocks.left(k, i >> 2)) * a.c16.row_bytes + chunk * 16));
      }
    }
  }
  static __device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

  __device__ __forceinline__ void scores4(f32x16& S) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
    for (int w4 = 0; w4 < 2; ++w4) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(mine + chunk_record_at(r, 2 * g + w4));
      const float f = __uint_as_float((uint32_t)mine[kCkScalesAt + (r >> 2) * kKv4Group + (2 * g + w4) * 4 + (r & 3)] << 23);
#pragma unroll
      for (int i = 0; i < 4; ++i) S = mfma32<F16>(decode8<F16>(w[i], f), q[4 * w4 + i], S);
    }
  }
  // V^T of 16 keys (tt), the lane's dims 4 r + db
  __device__ __forceinline__ void values4(int tt, u32x4 (&v)[4]) const {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i4 = 2 * tt + e;
      const uint32_t sc = *reinterpret_cast<const uint32_t*>(mine + kCkScalesAt + (2 * i4 + g) * kKv4Group + 16 + (r >> 3) * 4);
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const int n = 8 * i4 + 4 * g + j;
        const uint32_t x = *reinterpret_cast<const uint16_t*>(mine + chunk_record_at(n, 4 + (r >> 3)) + (r & 7) * 2);
        const uint32_t y = *reinterpret_cast<const uint16_t*>(mine + chunk_record_at(n + 1, 4 + (r >> 3)) + (r & 7) * 2);
        float fx = kv4_scale(sc, j), fy = kv4_scale(sc, j + 1);
        if constexpr (CARE) {                                               // (large_values() and not_numbers() have these blocks)
          fx = fx < kKv4Large<F16> ? fx : 0.f;
          fy = fy < kKv4Large<F16> ? fy : 0.f;
        }
        const int w = 2 * e + (j >> 1);
        if constexpr (F16) {
          const f32x2_t x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, fx, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, fx, 1);
          const f32x2_t y0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(y, fy, 0), y1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(y, fy, 1);
          v[0][w] = pack16<true>(x0.x, y0.x);
          v[1][w] = pack16<true>(x0.y, y0.y);
          v[2][w] = pack16<true>(x1.x, y1.x);
          v[3][w] = pack16<true>(x1.y, y1.y);
        } else {
          const uint32_t x0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, fx, 0));
          const uint32_t x1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, fx, 1));
          const uint32_t y0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y, fy, 0));
          const uint32_t y1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y, fy, 1));
          v[0][w] = __builtin_amdgcn_perm(y0, x0, 0x05040100u);
          v[1][w] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);
          v[2][w] = __builtin_amdgcn_perm(y1, x1, 0x05040100u);
          v[3][w] = __builtin_amdgcn_perm(y1, x1, 0x07060302u);
        }
      }
    }
  }

  // The blocks of V that may hold infinities, token by token and over the seen ones alone.
  __device__ __forceinline__ void large_values(uint32_t seen, const uint32_t (&P)[8], const uint32_t (&R)[8]) {
    const uint32_t seen_other = (uint32_t)__shfl_xor((int)seen, 32);
#pragma unroll 1
    for (int k = 0; k < 32; ++k) {                                          // key 8 (i / 4) + 4 half + i % 4
      const int i = k >> 1, half = k & 1, n = 8 * (i >> 2) + 4 * half + (i & 3);
      if (!chunk_large<F16>(mine, n)) continue;
      const float p_own = chunk_probability<F16>(P, R, i), p_other = __shfl_xor(p_own, 32), p = half == g ? p_own : p_other;
      const bool ok = ((half == g ? seen : seen_other) >> i) & 1u;
#pragma unroll
      for (int e = 0; e < 16; ++e) {                                        // dims 4 rho .. + 3
        const int rho = 8 * (e >> 2) + 4 * g + (e & 3);
        const float f = chunk_value_scale(mine, n, rho >> 3);
        const u32x4 v = decode8<F16>(*reinterpret_cast<const uint16_t*>(mine + chunk_record_at(n, 4 + (rho >> 3)) + (rho & 7) * 2), f);
        const float x[4] = {lo16<F16>(v[0]), hi16<F16>(v[0]), lo16<F16>(v[1]), hi16<F16>(v[1])};
#pragma unroll
        for (int db = 0; db < 4; ++db) O[db][e] = ok && f >= kKv4Large<F16> && f < __builtin_huge_valf() ? fmaf(p, x[db], O[db][e]) : O[db][e];
      }
    }
  }
  // Rows that see a token whose V has a block that is not a number have none there either.
  __device__ __forceinline__ void not_numbers(uint32_t seen) {
    uint32_t hit = 0;                                                       // bit: block of 32 dims
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned char* sc = mine + kCkScalesAt + (2 * (i >> 2) + g) * kKv4Group + 16 + (i & 3);
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) hit |= ((seen >> i) & 1u) && sc[blk * 4] == 255 ? 1u << blk : 0u;
    }
    hit |= (uint32_t)__shfl_xor((int)hit, 32);
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int db = 0; db < 4; ++db) O[db][i] = (hit >> (i >> 2)) & 1u ? __builtin_nanf("") : O[db][i];
  }

  // ---- a block's probabilities, as their rounding P and the rounding of the rest R ----
  // CARE: seen = bit i, the row sees the lane's i-th key, whose page is there.
  __device__ __forceinline__ void softmax(int n, f32x16& S, uint32_t (&P)[8], uint32_t (&R)[8], uint32_t& seen) {
    const float ninf = -__builtin_huge_valf();
    seen = 0xffffu;
    if constexpr (CARE) {
      seen = chunk_seen<LOCAL, KV4>(a, t, sight, n + 4 * g);
#pragma unroll
      for (int i = 0; i < 16; ++i) S[i] = (seen >> i) & 1u ? S[i] : ninf;
    } else if (!chunk_all_seen<LOCAL>(a.shape, t, t.m_lo, t.m_hi, n, 32)) {
      chunk_mask<LOCAL>(sight, n + 4 * g, S);
    }
    float mx = fmaxf(S[0], S[1]);
#pragma unroll
    for (int i = 2; i < 16; ++i) mx = fmaxf(mx, S[i]);
    if (__ballot((mx - m) * c > kCkLag<F16> || (m == ninf && mx > ninf)) != 0ull) {
      const float m_new = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32)));
      const float corr = m_new == ninf ? 1.f : fast_exp2((m - m_new) * c);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] *= corr;
    }
    const float mc = (m == ninf ? 0.f : m * c) - kCkLift<F16>;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float p0 = fast_exp2(fmaf(S[i], c, -mc)), p1 = fast_exp2(fmaf(S[i + 1], c, -mc));
      l += p0 + p1;
      P[i >> 1] = pack16<F16>(p0, p1);
      R[i >> 1] = pack16<F16>(p0 - lo16<F16>(P[i >> 1]), p1 - hi16<F16>(P[i >> 1]));
    }
  }
  __device__ __forceinline__ void pv(const u32x4 (&v)[4], int tt, const uint32_t (&P)[8], const uint32_t (&R)[8]) {
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      O[db] = mfma32<F16>(v[db], (u32x4){P[4 * tt], P[4 * tt + 1], P[4 * tt + 2], P[4 * tt + 3]}, O[db]);
      O[db] = mfma32<F16>(v[db], (u32x4){R[4 * tt], R[4 * tt + 1], R[4 * tt + 2], R[4 * tt + 3]}, O[db]);
    }
  }

  __device__ __forceinline__ void pass16() {
    f32x16 S;
    uint32_t P[8], R[8], seen;
    int k = blocks.next_seen(0);
    if (k < blocks.count) {
      blocks.advance(k);
      send(k, false);
      send(k, true);
    }
    while (k < blocks.count) {
      const int next = blocks.next_seen(k + 1);
      const bool more = next < blocks.count;
      if (more) blocks.advance(next);
      chunk_wait_loads<8>();                                                // K, in front of V's eight
#pragma unroll
      for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) S = mfma32<F16>(chunk_read_k(mine, rd, kk), q[kk], S);
      reads_done();
      if (more) send(next, false);
      softmax(blocks.n0(k), S, P, R, seen);
      if (more) chunk_wait_loads<8>();
      else chunk_wait_loads<0>();
      bool odd = false;
      if constexpr (CARE) {
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) any |= chunk_not_finite<F16>(chunk_read_v(mine + kCkBlockBytes / 2, rd, e >> 2, e & 3));
        odd = __ballot(any != 0u) != 0ull;
        if (odd) chunk_pv_seen<F16>(mine + kCkBlockBytes / 2, seen, P, R, O);
      }
#pragma unroll
      for (int tt = 0; tt < 2 && !odd; ++tt) {
        u32x4 v[4];
#pragma unroll
        for (int db = 0; db < 4; ++db) v[db] = chunk_read_v(mine + kCkBlockBytes / 2, rd, tt, db);
        pv(v, tt, P, R);
      }
      reads_done();
      if (more) send(next, true);
      k = next;
    }
  }
  __device__ __forceinline__ void pass4() {
    typename ChunkBlocks<LOCAL, KV4, NW>::Codes x[2];
    int at[2];
    at[0] = blocks.next_seen(0);
    at[1] = blocks.next_seen(at[0] + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (at[u] < blocks.count) {
        blocks.advance(at[u]);
        blocks.fetch(at[u], x[u]);
      }
    auto step = [&](typename ChunkBlocks<LOCAL, KV4, NW>::Codes& y, int& k, int behind) __attribute__((always_inline)) {      // behind: the block that is on its way behind this one
      f32x16 S;
      uint32_t P[8], R[8], seen;
      chunk_put_records(mine, y);
      const int n = blocks.n0(k);
      k = blocks.next_seen(behind + 1);
      if (k < blocks.count) {
        blocks.advance(k);
        blocks.fetch(k, y);
      }
      scores4(S);
      softmax(n, S, P, R, seen);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        u32x4 v[4];
        values4(tt, v);
        pv(v, tt, P, R);
      }
      if constexpr (CARE) {
        large_values(seen, P, R);
        not_numbers(seen);
      }
    };
    while (at[0] < blocks.count) {
      step(x[0], at[0], at[1]);
      if (at[1] >= blocks.count) break;
      step(x[1], at[1], at[0]);
    }
  }

  // true: a page was not there or a result is not finite (never with CARE)
  __device__ __forceinline__ bool run() {
    if (blocks.count > 0) {
      if constexpr (KV4) pass4();
      else pass16();
    }
    float z = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) z = fmaf(O[db][i], 0.f, z);
    l += __shfl_xor(l, 32);
    if constexpr (CARE) __syncthreads();
    else if (__syncthreads_or(blocks.lost || !(z == 0.f) || !(l < 0x1p120f) ? 1 : 0) != 0) return true;
    // ---- the waves' results, joined: rows of 32 groups of four outputs, group d of row r at d ^ r ----
    float* const sh_m = reinterpret_cast<float*>(smem + NW * kCkBlockBytes);
    float* const sh_l = sh_m + NW * kCkNarrowRows;
    if (g == 0) {
      sh_m[wave * kCkNarrowRows + r] = m;
      sh_l[wave * kCkNarrowRows + r] = l;
    }
    if (r < t.rows) {
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        int d;                                                              // group of four dims
        float4 o;
        if constexpr (KV4) {
          d = (k >> 2) * 8 + g * 4 + (k & 3);
          o = make_float4(O[0][k], O[1][k], O[2][k], O[3][k]);
        } else {
          const int db = k >> 2, i4 = k & 3;
          d = db * 8 + i4 * 2 + g;
          o = make_float4(O[db][i4 * 4], O[db][i4 * 4 + 1], O[db][i4 * 4 + 2], O[db][i4 * 4 + 3]);
        }
        *reinterpret_cast<float4*>(mine + r * 512 + ((d ^ r) & 31) * 16) = o;
      }
    }
    __syncthreads();
    constexpr int kLanes = NW * 64 / kCkNarrowRows, kEach = kHeadDim / 4 / kLanes;       // threads per row, groups of four outputs per thread
    const int row = threadIdx.x / kLanes, d0 = threadIdx.x % kLanes;
    if (row >= t.rows) return false;
    const float ninf = -__builtin_huge_valf();
    float M = ninf, L = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sh_m[w * kCkNarrowRows + row]);
    float o[kEach][4] = {};
    {
      // (a wave without a finite logit: its sum is 0, or not a number)
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float m_w = sh_m[w * kCkNarrowRows + row], cw = m_w == ninf ? 1.f : fast_exp2((m_w - M) * c);
        L += sh_l[w * kCkNarrowRows + row] * cw;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int d = d0 + kLanes * e;
          const float4 v = *reinterpret_cast<const float4*>(smem + w * kCkBlockBytes + row * 512 + ((d ^ row) & 31) * 16);
          o[e][0] = fmaf(v.x, cw, o[e][0]);
          o[e][1] = fmaf(v.y, cw, o[e][1]);
          o[e][2] = fmaf(v.z, cw, o[e][2]);
          o[e][3] = fmaf(v.w, cw, o[e][3]);
        }
      }
    }
    chunk_lower<F16>(L, o);
#pragma unroll
    for (int e = 0; e < kEach; ++e) chunk_store4<F16>(a, t, row, 4 * (d0 + kLanes * e), M, L, L, o[e]);
    return false;
  }
};

}  // namespace rtp
