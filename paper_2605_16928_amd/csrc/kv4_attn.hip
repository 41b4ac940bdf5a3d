// Decode attention over the 4-bit cache: rtp_sparse_attn_decode_kv4 (selected tokens, retrieval heads), rtp_local_attn_kv4 (sink +
// window, the other heads) and rtp_dense_attn_kv4 (every token, every head).
//
//   out_h = sum_n p_n v_n / sum_n p_n,   p_n = 2^(c <q_h, k_n> - m),   c = softmax scale * log2(e)
// over the tokens n of the set, K and V as the values that their codes stand for.
//
// Bound: 136 bytes per token and KV head.  At that size the vector ALU is as near a limit as HBM is, so both products go to the matrix
// cores, 32 tokens (two tiles of 16) per wave and step.  A token's record comes from memory as one whole line, eight lanes of 16 bytes,
// and is turned into the operands in the wave's own LDS (kv4_turn; loaded in operand order every line would be touched twice):
//   S = K q^T    v_mfma_f32_16x16x32_bf16, A = 16 tokens: lane (token c, quarter g) has the dims 32 g .. + 31 of its token -- 16 bytes
//                of codes, one scale -- as bf16, which every code times its scale is exactly.  B = the queries in 8 columns.
//   O += P V     A = P, whose rows are the columns of S: lane (head c, rows g) has the tokens 4 g + i of both tiles in registers and
//                takes them for the k positions 8 g .. + 7, so no probability changes its lane.  B = V: lane (c, g) has the dims
//                8 c .. + 7 (one word of codes) of the tokens 4 g + i, and pairs of converted values are regrouped to pairs of tokens.
// A GQA group has at most 8 heads, so the other 8 columns and rows are free.  They carry what 16 bits lose: P is the sum of its
// bf16 rounding (rows 0 - 7) and the bf16 rounding of the rest (rows 8 - 15; the columns 8 - 15 of S repeat the heads, so the lane
// that needs the rest has p itself), and an fp16 query is split over the columns the same way.  P keeps 16 bits of mantissa thereby,
// and one kernel serves both types.
//
// Work split: a unit (sequence and KV head, or sequence and retrieval head) is cut into items, an item goes to a workgroup of eight or
// four waves, which leaves a partial (max, sum, 128 outputs) per head for the merge launch, or the result where a unit is one item.
//
// Measured: 8 contexts of 131072 tokens, 8 KV heads (1.14 GB) 180 us, 6.3 TB/s; windows of 8192 of 32 sequences (219 MB) 45 us, 4.9; 256
// rows of 200 to 30000 selected tokens (222 MB) 56 + 4 us.  With the products left out the loads alone take 167 and 36 us for the
// first two: some 200 vector instructions per 32 tokens are what is between.  Two rows of 100 selected tokens take 5 us, an empty launch 3.
#include "attn_decode_shared.h"
#include "kv4_cache.h"

namespace rtp {

constexpr int kKv4MaxHeads = 128;

constexpr int kMaxUnits = 1 << 20;   // (sequence, KV head) pairs of a call
constexpr int kMaxLen = 1 << 26;   // longest context or selection: sums of the blocks of 1024 rows, or of 256 sequences, stay inside an int

struct Kv4AttnArgs {
  AttnDecodeArgs d;            // (K, V, strides, seq_start, ring and table fields are not used)
  Kv4Cache c;
  int32_t max_len;             // upper bound of a context / a selection: longer ones are cut there
  int32_t direct;              // a unit is one item and writes its result
  int32_t B;
  int32_t balanced;            // range sources: items are shared out by the lengths on the device, else n_splits to a unit
  int32_t even;                // balanced: items of a unit where the lengths are about equal (0: by target_items like others)
  uint32_t skip[kKv4MaxHeads / 4];   // local source: byte kvh = bits of the group's heads that the call does not serve
};

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2_t v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint16_t out16(float x, bool f16) {       // (NaN stays NaN)
  return f16 ? __builtin_bit_cast(uint16_t, (_Float16)x) : __builtin_bit_cast(uint16_t, (__bf16)x);
}

// 32 tokens of a wave as they come from memory: whole records, 8 lanes of 16 bytes each, so that every load instruction takes full
// cache lines and may be non-temporal (the operand layouts below would touch every line twice, K's half and V's).
// line[q]: token 8 q + lane / 8, piece lane % 8 of its 128 bytes.
struct Kv4Lines {
  u32x4 line[4];
};
// The same 32 tokens as a lane's operands.
struct Kv4Tiles {
  u32x4 k[2];                  // tile s: token c, dims 32 g .. + 31
  uint32_t v[2][4];            // tile s: token 4 g + i, dims 8 c .. + 7
  uint32_t ks[2];              // scale byte of k[s]
  uint32_t vs[2];              // scale bytes of v[s][0 .. 3]
};
// A wave's own LDS: the records on their way from the one form to the other, later its part of the joined outputs.
struct Kv4WaveLds {
  union {
    u32x4 line[32 * 8];        // [token][piece ^ (token / 2 % 8)]: 16 tokens' pieces of one number lie in 16 different bank groups
    float o[8][kHeadDim];
  };
};
__device__ __forceinline__ int kv4_place(int token, int piece) { return token * 8 + (piece ^ ((token >> 1) & 7)); }

// LDS words that only the own wave writes and reads: its accesses stay in program order, no workgroup barrier is needed.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Records -> LDS -> operands (without the scales).
__device__ __forceinline__ void kv4_turn(const Kv4Lines& in, Kv4WaveLds& lds, Kv4Tiles& t) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  wave_lds_fence();
#pragma unroll
  for (int q = 0; q < 4; ++q) lds.line[kv4_place(8 * q + (lane >> 3), lane & 7)] = in.line[q];
  wave_lds_fence();
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    t.k[s] = lds.line[kv4_place(16 * s + c, g)];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      t.v[s][i] = reinterpret_cast<const uint32_t*>(&lds.line[kv4_place(16 * s + 4 * g + i, 4 + (c >> 2))])[c & 3];
  }
}

// A wave's running state: m of head c & 7 (the same in the four lanes of a column and in column c + 8), l per lane, outputs of
// rows 4 g + i at dims 8 c + n.
struct Kv4State {
  float m, l;
  f32x4_t o[8];
};

constexpr float kLateMax = 8.f;   // the reference m follows the maximum only when it is left behind by more than this: p <= 2^8

// valid: bit t = token t of the 32 takes part.  Tokens that do not are masked out of S; their V scales have to be finite.
template <bool F16>
__device__ __forceinline__ void kv4_step(const Kv4Tiles& t, const uint32_t valid, const u32x4 (&qB)[4], const float scale_log2,
                                         Kv4State& st) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  float x[2][4];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const float f = __uint_as_float(t.ks[s] << 23);
    f32x4_t S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      u32x4 a;
      a[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.k[s][kk], f, 0));
      a[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.k[s][kk], f, 1));
      a[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.k[s][kk], f, 2));
      a[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.k[s][kk], f, 3));
      S = mfma16<false>(a, qB[kk], S);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y = S[i];
      if (F16) y += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0x128, 0xf, 0xf, true));   // row_ror:8
      x[s][i] = y;
    }
  }
  const float ninf = -__builtin_huge_valf();
  if (valid != 0xffffffffu) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t mine = valid >> (16 * s + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[s][i] = (mine >> i) & 1u ? x[s][i] : ninf;
    }
  }
  // (max_nn of a NaN and a number is the number, of two NaN +inf: the row is NaN by its sum either way)
  const float mine = scale_log2 * max_nn(max_nn(max_nn(x[0][0], x[0][1]), max_nn(x[0][2], x[0][3])),
                                         max_nn(max_nn(x[1][0], x[1][1]), max_nn(x[1][2], x[1][3])));
  if (__ballot(mine > st.m + kLateMax) != 0ull) {        // (also where m is still -inf)
    const float m_new = fmaxf(st.m, max_over_rows(mine));
    const float corr = m_new == ninf ? 1.f : fast_exp2(st.m - m_new);
    st.l *= corr;
    st.m = m_new;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float ci = __shfl(corr, (lane & 48) | ((4 * g + i) & 7));
#pragma unroll
      for (int n = 0; n < 8; ++n) st.o[n][i] *= ci;
    }
  }
  const float ref = st.m == ninf ? 0.f : st.m;           // (a row without a finite logit so far: NaN stays NaN, -inf gives 0)
  u32x4 pA;
  const bf16x2_t minus_lo = __builtin_bit_cast(bf16x2_t, c < 8 ? 0u : 0x0000bf80u), minus_hi = __builtin_bit_cast(bf16x2_t, c < 8 ? 0u : 0xbf800000u);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] = fast_exp2(fmaf(x[s][i], scale_log2, -ref));
      st.l += p[i];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // rows 0 - 7: p rounded; rows 8 - 15: what that leaves (p - 1 * lo - 0 * hi as one dot product, factors 0 in the rows below)
      const bf16x2_t hi = __builtin_bit_cast(bf16x2_t, pack_bf16(p[2 * h], p[2 * h + 1]));
      pA[2 * s + h] = pack_bf16(__builtin_amdgcn_fdot2_f32_bf16(hi, minus_lo, p[2 * h], false),
                                __builtin_amdgcn_fdot2_f32_bf16(hi, minus_hi, p[2 * h + 1], false));
    }
  }
  float fv[2][4];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) fv[s][i] = kv4_scale(t.vs[s], i);
#define RTP_KV4_PV(B)                                                                                                        \
  {                                                                                                                          \
    u32x4 even, odd;                                                                                                         \
    _Pragma("unroll") for (int s = 0; s < 2; ++s) _Pragma("unroll") for (int h = 0; h < 2; ++h) {                             \
      const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[s][2 * h], fv[s][2 * h], B));          \
      const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[s][2 * h + 1], fv[s][2 * h + 1], B));  \
      even[2 * s + h] = __builtin_amdgcn_perm(b, a, 0x05040100u);                                                             \
      odd[2 * s + h] = __builtin_amdgcn_perm(b, a, 0x07060302u);                                                              \
    }                                                                                                                        \
    st.o[2 * B] = mfma16<false>(pA, even, st.o[2 * B]);                                                                       \
    st.o[2 * B + 1] = mfma16<false>(pA, odd, st.o[2 * B + 1]);                                                                \
  }
  RTP_KV4_PV(0)
  RTP_KV4_PV(1)
  RTP_KV4_PV(2)
  RTP_KV4_PV(3)
#undef RTP_KV4_PV
}

// The queries of heads h0 .. h0 + heads - 1 as the B operand: column c = head c & 7 (zero beyond `heads`); the columns 8 - 15 repeat
// them, or hold what bf16 leaves of an fp16 query.
template <bool F16>
__device__ __forceinline__ void kv4_queries(const AttnDecodeArgs& a, int b, int h0, int heads, u32x4 (&qB)[4]) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    qB[kk] = (u32x4){0u, 0u, 0u, 0u};
    if ((c & 7) < heads) qB[kk] = *reinterpret_cast<const u32x4*>(a.q + ((int64_t)b * a.n_q_heads + h0 + (c & 7)) * kHeadDim + 32 * g + 8 * kk);
    if (F16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo = lo16<true>(qB[kk][i]), hi = hi16<true>(qB[kk][i]);
        const uint32_t top = pack_bf16(lo, hi);
        qB[kk][i] = c < 8 ? top : pack_bf16(lo - bf16_lo(top), hi - bf16_hi(top));
      }
    }
  }
}

// Joins the waves' states of an item through LDS and writes the partials of its heads, or, `direct`, their results.
// skip: heads (of the unit's) that the call does not serve.
template <int WAVES>
__device__ __forceinline__ void kv4_finish(const Kv4AttnArgs& a, Kv4State& st, Kv4WaveLds (&lds)[WAVES], int item, int b, int h0, int heads,
                                           bool direct, uint32_t skip) {
  __shared__ float sh_m[WAVES][8], sh_l[WAVES][8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, g = lane >> 4;
  const float ninf = -__builtin_huge_valf();
  st.l = sum_rows(st.l, st.l, st.l, st.l);
  if (lane < 8) { sh_m[wave][lane] = st.m; sh_l[wave][lane] = st.l; }
  wave_lds_fence();
#pragma unroll
  for (int i = 0; i < 4; ++i) {                // rows r and r + 8 are 32 lanes apart
    float o[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] = st.o[n][i] + __shfl_xor(st.o[n][i], 32);
    if (g < 2 && 4 * g + i < heads) {
      *reinterpret_cast<float4*>(&lds[wave].o[4 * g + i][8 * c]) = make_float4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<float4*>(&lds[wave].o[4 * g + i][8 * c + 4]) = make_float4(o[4], o[5], o[6], o[7]);
    }
  }
  __syncthreads();
  float* part = a.d.part + (int64_t)item * heads * kPartStride;
  for (int e = tid; e < heads * kHeadDim; e += WAVES * 64) {
    const int hh = e >> 7, dim = e & 127;
    if ((skip >> hh) & 1u) continue;
    float M = sh_m[0][hh];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sh_m[w][hh]);
    const float ref = M == ninf ? 0.f : M;
    float L = 0.f, A = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float cw = fast_exp2(sh_m[w][hh] - ref);
      L += sh_l[w][hh] * (sh_m[w][hh] == ninf ? 1.f : cw);       // (a wave without a finite logit: its sum is 0, or NaN)
      A += lds[w].o[hh][dim] * (sh_m[w][hh] == ninf ? 1.f : cw);
    }
    if (direct) {
      const int64_t o = (int64_t)b * a.d.n_q_heads + h0 + hh;
      a.d.out[o * kHeadDim + dim] = out16(L == 0.f ? 0.f : A / L, a.d.f16 != 0);
      if (a.d.lse && dim == 0) a.d.lse[o] = L == 0.f ? ninf : (ref + log2f(L)) * 0.6931471805599453f;
    } else {
      part[hh * kPartStride + 4 + dim] = A;
      if (dim == 0) { part[hh * kPartStride] = M; part[hh * kPartStride + 1] = L; }
    }
  }
}

__device__ __forceinline__ void kv4_clear(Kv4State& st) {
  st.m = -__builtin_huge_valf();
  st.l = 0.f;
#pragma unroll
  for (int n = 0; n < 8; ++n) st.o[n] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
}

// ---- work items ------------------------------------------------------------------------------------------------------------------
// A list of n lengths (in blocks), each worked on `times` times (the KV heads of a sequence) by items of whole rounds.
struct Kv4Share {
  int index, time;        // which length, which of its times
  int j0, j1;             // the item's blocks
  int first, count;       // the partials of (index, time)
};
template <int ROUND>
__device__ __forceinline__ int whole_rounds(int blocks) { return (max(blocks, 1) + ROUND - 1) / ROUND * ROUND; }

// All items of a call take about the same number of blocks, by the lengths that the device holds, so that a ragged batch keeps every
// workgroup busy to the end.  Each wave makes the plan for itself, a lane per length: no LDS, no barrier.  The items of an index are
// consecutive, time by time, and equal (or the last one would often be a small one).  want: an item's number, or (by_unit) the number
// index * times + time; false: there is no such item.
// even: where it is not 0 and the lengths are about equal (the longest at most 5/4 of their mean), an index is cut into that many
// items instead.
template <int ROUND, class BlocksOf>
__device__ __forceinline__ bool kv4_share(BlocksOf blocks_of, int n, int times, int target, int even, int want, bool by_unit, Kv4Share* s) {
  const int lane = threadIdx.x & 63;
  int total = 0, longest = 0;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int blocks = i0 + lane < n ? blocks_of(i0 + lane) : 0;
    total += wave_sum(blocks);
    longest = max(longest, blocks);
  }
  int per = whole_rounds<ROUND>((int)(((int64_t)total * times + target - 1) / target));
  if (even && __ballot((int64_t)longest * n * 4 > (int64_t)total * 5) == 0ull) {
    for (int d = 32; d > 0; d >>= 1) longest = max(longest, __shfl_xor(longest, d));
    per = whole_rounds<ROUND>((longest + even - 1) / even);
  }
  int base = 0;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int blocks = i0 + lane < n ? blocks_of(i0 + lane) : 0;
    const int splits = (blocks + per - 1) / per, incl = wave_incl_scan(splits * times), before = base + incl - splits * times;
    const uint64_t mine = by_unit ? __ballot(i0 + lane == want / times) : __ballot(want >= before && want < base + incl);
    if (mine) {
      const int l = __ffsll((unsigned long long)mine) - 1;
      const int sp = __builtin_amdgcn_readlane(splits, l), at = __builtin_amdgcn_readlane(before, l), len = __builtin_amdgcn_readlane(blocks, l);
      s->index = i0 + l;
      s->time = by_unit ? want % times : (want - at) / sp;
      s->first = at + s->time * sp;
      const int each = whole_rounds<ROUND>((len + sp - 1) / max(sp, 1)), split = by_unit ? 0 : want - s->first;
      s->count = (len + each - 1) / each;
      s->j0 = split * each;
      s->j1 = min(len, s->j0 + each);
      return s->j0 < s->j1;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// ---- every token, or sink + window --------------------------------------------------------------------------------------------
// A unit's tokens as blocks of 16 positions (a block lies in one page): the sink's blocks, then the window's.
struct Kv4Range {
  int n, s0, w0;          // tokens; token t takes part if t < n and (t < s0 or t >= w0)
  int sb, wb0, blocks;    // block j < sb is block j of the sequence, block j >= sb is block wb0 + j - sb
};
__device__ __forceinline__ Kv4Range kv4_range(const Kv4AttnArgs& a, int b, bool local) {
  Kv4Range r;
  r.n = min(max(a.d.ctx_len[b], 0), a.max_len);
  r.s0 = local ? min(a.d.sink, r.n) : r.n;
  r.w0 = local ? max(a.d.sink, r.n - a.d.window) : r.n;
  r.sb = (r.s0 + 15) >> 4;
  r.wb0 = max(r.sb, r.w0 >> 4);
  r.blocks = r.sb + max(0, ((r.n + 15) >> 4) - r.wb0);
  return r;
}
__device__ __forceinline__ uint32_t low16(int n) { return n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1u; }

constexpr int kKv4Waves = 8;           // waves of a workgroup
constexpr int kKv4Round = 2 * kKv4Waves;     // blocks that they take at a time; an item is whole rounds
constexpr int kKv4Items = 256;         // items: one to a compute unit

// The item (or unit) of a range call.  Not balanced: n_splits items to a unit, the trailing ones of a short unit empty.
template <bool LOCAL>
__device__ __forceinline__ bool kv4_range_item(const Kv4AttnArgs& a, int want, bool by_unit, Kv4Share* s, Kv4Range* r) {
  if (a.balanced) {
    const bool there = kv4_share<kKv4Round>([&](int b) { return kv4_range(a, b, LOCAL).blocks; }, a.B, a.d.n_kv_heads, a.d.target_items,
                                            a.even, want, by_unit, s);
    if (there) *r = kv4_range(a, s->index, LOCAL);
    return there;
  }
  const int unit = by_unit ? want : want / a.d.n_splits, split = by_unit ? 0 : want - unit * a.d.n_splits;
  s->index = unit / a.d.n_kv_heads;
  s->time = unit - s->index * a.d.n_kv_heads;
  *r = kv4_range(a, s->index, LOCAL);
  const int per = whole_rounds<kKv4Round>((r->blocks + a.d.n_splits - 1) / a.d.n_splits);
  s->first = unit * a.d.n_splits;
  s->count = (r->blocks + per - 1) / per;
  s->j0 = split * per;
  s->j1 = min(r->blocks, s->j0 + per);
  return s->j0 < s->j1 || (a.direct && split == 0);
}

__device__ __forceinline__ uint32_t kv4_skip(const Kv4AttnArgs& a, int kvh) { return (a.skip[kvh >> 2] >> (8 * (kvh & 3))) & 255u; }

template <bool LOCAL, bool F16>
__global__ __launch_bounds__(kKv4Waves * 64, 2) void kv4_range_kernel(const Kv4AttnArgs a) {
  __shared__ Kv4WaveLds sh_lines[kKv4Waves];
  __shared__ uint32_t sh_scales[kKv4Waves][64];      // two blocks: [group of four tokens][K or V][block][token]
  const int item = blockIdx.x;
  Kv4Share it;
  Kv4Range r;
  if (!kv4_range_item<LOCAL>(a, item, false, &it, &r)) return;
  const int b = it.index, kvh = it.time, j0 = it.j0, j1 = it.j1;
  const int heads = a.d.n_q_heads / a.d.n_kv_heads, h0 = kvh * heads;
  const uint32_t skip = LOCAL ? kv4_skip(a, kvh) : 0;
  if (skip == (1u << heads) - 1u) return;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  u32x4 qB[4];
  kv4_queries<F16>(a.d, b, h0, heads, qB);
  Kv4State st;
  kv4_clear(st);
  const int32_t* pt = a.c.page_table + b * a.c.pt_stride;
  const uint8_t* codes = a.c.codes + kvh * a.c.code_head_stride;
  const uint8_t* scales = a.c.scales + kvh * a.c.scale_head_stride;
  const int bshift = a.c.page_shift - 4, bmask = (1 << bshift) - 1;

  // The blocks j and j + 1 (clamped to the item's last one) and the table's entries for them, which are loaded a step ahead of the
  // bytes.  A context ends inside its table row, so the entry is there; it may name no page of the pool.
  struct Spot {
    int blk[2];
    uint32_t page[2];
  };
  auto look_up = [&](int j) {
    Spot p;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int jj = min(j + s, j1 - 1);
      p.blk[s] = jj + (jj < r.sb ? 0 : r.wb0 - r.sb);
      p.page[s] = (uint32_t)pt[p.blk[s] >> bshift];
    }
    return p;
  };
  // the bytes (sc: lane's word of the two blocks' scales); returns the bits of the tokens that take part
  auto load = [&](int j, const Spot& p, Kv4Lines& in, uint32_t& sc) -> uint32_t {
    uint32_t valid = 0xffffffffu;
    const uint8_t* sp[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int blk = p.blk[s];
      const bool here = p.page[s] < (uint32_t)a.c.n_pages;
      const uint32_t pg = here ? p.page[s] : 0u;
      const uint32_t row = (uint32_t)(blk & bmask);
      const u32x4* cp = reinterpret_cast<const u32x4*>(codes + ((uint64_t)pg * a.c.code_page16 + row * (16 * kKv4Row / 16)) * 16);
      sp[s] = scales + ((uint64_t)pg * a.c.scale_page16 + row * (4 * kKv4Group / 16)) * 16;
      in.line[2 * s] = __builtin_nontemporal_load(cp + lane);
      in.line[2 * s + 1] = __builtin_nontemporal_load(cp + 64 + lane);
      // whole blocks, but for the last one of the sequence, the sink's last and the window's first
      const int jj = j + s;
      if (!here || jj >= j1 || jj == r.blocks - 1 || jj == r.sb || jj == r.sb - 1) {
        const uint32_t v = low16(r.n - 16 * blk) & (low16(r.s0 - 16 * blk) | ~low16(r.w0 - 16 * blk));
        valid &= ~(((here && jj < j1 ? v : 0u) ^ 0xffffu) << (16 * s));
      }
    }
    sc = *(reinterpret_cast<const uint32_t*>(lane < 32 ? sp[0] : sp[1]) + (lane & 31));
    return valid;
  };
  // tokens that do not take part may hold anything: their V scales become 2^-127
  auto clean = [&](uint32_t valid, Kv4Tiles& t) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t mine = valid >> (16 * s + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!((mine >> i) & 1u)) t.vs[s] &= ~(0xffu << (8 * i));
    }
  };
  // 32 tokens, whose bytes have been asked for
  auto attend = [&](const Kv4Lines& in, uint32_t sc, uint32_t valid) {
    if (!valid) return;
    Kv4Tiles t;
    sh_scales[wave][lane] = sc;
    kv4_turn(in, sh_lines[wave], t);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      t.ks[s] = reinterpret_cast<const uint8_t*>(&sh_scales[wave][32 * s + 8 * (c >> 2) + g])[c & 3];
      t.vs[s] = sh_scales[wave][32 * s + 8 * g + 4 + (c >> 2)];
    }
    if (valid != 0xffffffffu) clean(valid, t);
    kv4_step<F16>(t, valid, qB, a.d.scale_log2, st);
  };
  const int step = 2 * kKv4Waves;
  constexpr int kAhead = 2;                     // sets of 32 tokens in flight (3 and 4 measured the same on long contexts, 0.6 and 1.6 us more on short ones)
  int j = j0 + 2 * wave;
  if (j < j1) {
    Kv4Lines in[kAhead];
    uint32_t sc[kAhead], valid[kAhead];
    Spot next = look_up(j);
#pragma unroll
    for (int d = 0; d < kAhead - 1; ++d) {
      valid[d] = load(j + d * step, next, in[d], sc[d]);
      next = look_up(j + (d + 1) * step);
    }
    for (; j < j1; j += kAhead * step) {
#pragma unroll
      for (int d = 0; d < kAhead; ++d) {       // (steps beyond the item's end have no token)
        const int e = (d + kAhead - 1) % kAhead;
        valid[e] = load(j + (d + kAhead - 1) * step, next, in[e], sc[e]);
        next = look_up(j + (d + kAhead) * step);
        attend(in[d], sc[d], valid[d]);
      }
    }
  }
  kv4_finish(a, st, sh_lines, item, b, h0, heads, a.direct || it.count == 1, skip);
}

// Merges the partials i0 .. i1 - 1 of the head slots hh0 .. hh0 + nh - 1 (of `heads` in each) into the output rows of the query heads
// from h on: 32 lanes of four dims each take a slice of a head's partials, THREADS / 32 / nh slices to a head.
template <int THREADS>
__device__ __forceinline__ void kv4_merge(const Kv4AttnArgs& a, int heads, int hh0, int nh, int b, int h, int i0, int i1, uint32_t skip) {
  constexpr int kGroups = THREADS / 32;
  __shared__ float sh_m[kGroups], sh_l[kGroups];
  __shared__ float sh_o[kGroups][kHeadDim];
  const int tid = threadIdx.x, d4 = tid & 31, group = tid >> 5, slices = kGroups / nh;
  const float ninf = -__builtin_huge_valf();
  float M = ninf, L = 0.f;
  float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
  if (group < nh * slices) {
    const int hh = hh0 + group / slices;
    if (!((skip >> hh) & 1u)) {
      for (int i = i0 + group % slices; i < i1; i += slices) {
        const float* p = a.d.part + ((int64_t)i * heads + hh) * kPartStride;
        const float m = p[0], l = p[1];
        const float4 v = *reinterpret_cast<const float4*>(p + 4 + d4 * 4);
        const float Mn = fmaxf(M, m);
        const float c0 = M == ninf ? 1.f : fast_exp2(M - Mn), c1 = m == ninf ? 1.f : fast_exp2(m - Mn);   // (-inf: 0, or NaN, as it is)
        L = L * c0 + l * c1;
        A.x = A.x * c0 + v.x * c1; A.y = A.y * c0 + v.y * c1;
        A.z = A.z * c0 + v.z * c1; A.w = A.w * c0 + v.w * c1;
        M = Mn;
      }
    }
  }
  if (d4 == 0) { sh_m[group] = M; sh_l[group] = L; }
  *reinterpret_cast<float4*>(&sh_o[group][d4 * 4]) = A;
  __syncthreads();
  const int e = tid >> 7, dim = tid & 127;       // (THREADS / 128 heads at least nh)
  if (e >= nh || ((skip >> (hh0 + e)) & 1u)) return;
  float Mt = ninf;
  for (int s = 0; s < slices; ++s) Mt = fmaxf(Mt, sh_m[e * slices + s]);
  const float ref = Mt == ninf ? 0.f : Mt;
  float Lt = 0.f, At = 0.f;
  for (int s = 0; s < slices; ++s) {
    const int w = e * slices + s;
    const float cs = sh_m[w] == ninf ? 1.f : fast_exp2(sh_m[w] - ref);
    Lt += sh_l[w] * cs;
    At += sh_o[w][dim] * cs;
  }
  const int64_t o = (int64_t)b * a.d.n_q_heads + h + e;
  a.d.out[o * kHeadDim + dim] = out16(Lt == 0.f ? 0.f : At / Lt, a.d.f16 != 0);
  if (a.d.lse && dim == 0) a.d.lse[o] = Lt == 0.f ? ninf : (ref + log2f(Lt)) * 0.6931471805599453f;
}

// grid (units, heads), or (units, 1) where a workgroup takes all heads of a unit (WIDE)
template <bool LOCAL, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256) void kv4_range_merge_kernel(const Kv4AttnArgs a) {
  const int heads = a.d.n_q_heads / a.d.n_kv_heads, unit = blockIdx.x, kvh = unit % a.d.n_kv_heads, hh = WIDE ? 0 : (int)blockIdx.y;
  const uint32_t skip = LOCAL ? kv4_skip(a, kvh) : 0;
  Kv4Share it = {};
  Kv4Range r;
  kv4_range_item<LOCAL>(a, unit, true, &it, &r);
  if (it.count == 1) return;                   // (its item wrote the result)
  kv4_merge<WIDE ? 1024 : 256>(a, heads, hh, WIDE ? heads : 1, unit / a.d.n_kv_heads, kvh * heads + hh, it.first, it.first + it.count, skip);
}

// ---- selected tokens ------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int kv4_selected(const Kv4AttnArgs& a, int unit) { return min(max(a.d.sel_count[unit], 0), a.max_len); }

constexpr int kSpWaves = 4;            // waves of a workgroup where rows are cut into items
// An item (or row) of a call over selected tokens, in blocks of 64: a wave's share of a round.
__device__ __forceinline__ bool kv4_sparse_item(const Kv4AttnArgs& a, int want, bool by_unit, Kv4Share* s) {
  return kv4_share<kSpWaves>([&](int unit) { return (kv4_selected(a, unit) + 63) / 64; }, a.d.units, 1, a.d.target_items, 0, want,
                             by_unit, s);
}

// A wave takes 64 tokens at a time.  A lane looks one of them up -- its position a chunk ahead of the page, the page a chunk ahead of
// the bytes -- and fetches its scales; the records are then loaded by eight lanes each, by the offsets that the lanes left in LDS.
// DIRECT: a workgroup of eight waves has a whole row and writes its result; else items of four waves leave partials.
template <bool F16, bool DIRECT>
__global__ __launch_bounds__(DIRECT ? 512 : 256, DIRECT ? 2 : 3) void kv4_sparse_kernel(const Kv4AttnArgs a) {
  constexpr int kWaves = DIRECT ? 8 : kSpWaves, kThreads = kWaves * 64;
  __shared__ Kv4WaveLds sh_lines[kWaves];
  __shared__ int64_t sh_at[kWaves][64];          // a token's record, from the head's first byte
  __shared__ uint32_t sh_ks[kWaves][64];         // its four K scales
  __shared__ __attribute__((aligned(16))) uint8_t sh_vs[kWaves][4][64];       // V scales by block
  const int item = blockIdx.x;
  Kv4Share it = {item, 0, 0, kMaxLen / 64, 0, 0};
  if (!DIRECT && !kv4_sparse_item(a, item, false, &it)) return;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = it.index, b = unit / a.d.n_ret, h = a.d.ret_heads[unit - b * a.d.n_ret], kvh = h / (a.d.n_q_heads / a.d.n_kv_heads);
  const int t0 = it.j0 * 64, t1 = min(kv4_selected(a, unit), it.j1 * 64);
  const int32_t* idx = a.d.sel_idx + (int64_t)unit * a.d.sel_stride;
  const int32_t* pt = a.c.page_table + b * a.c.pt_stride;
  const uint8_t* codes = a.c.codes + kvh * a.c.code_head_stride;
  const uint8_t* scales = a.c.scales + kvh * a.c.scale_head_stride;
  u32x4 qB[4];
  kv4_queries<F16>(a.d, b, h, 1, qB);
  Kv4State st;
  kv4_clear(st);

  // position of this lane's token in the chunk at `base`, and its page (-1: none)
  auto position = [&](int base) { return base + lane < t1 ? idx[base + lane] : -1; };
  auto page_of = [&](int pos) { return kv4_page(a.c, pt, pos); };
  // leaves the records' offsets in LDS and asks for the scales; tokens without a page stand at the head's first record
  auto place = [&](int pos, int page, u32x4& k4, u32x4& v4) {
    const int slot = page < 0 ? 0 : pos & ((1 << a.c.page_shift) - 1);
    const int64_t pg = max(page, 0);
    wave_lds_fence();
    sh_at[wave][lane] = pg * ((int64_t)a.c.code_page16 * 16) + (int64_t)slot * kKv4Row;
    wave_lds_fence();
    const u32x4* sp = reinterpret_cast<const u32x4*>(scales + pg * ((int64_t)a.c.scale_page16 * 16) + (int64_t)(slot >> 2) * kKv4Group);
    k4 = sp[0];
    v4 = sp[1];
  };
  auto load = [&](int half, Kv4Lines& in) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      in.line[q] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + sh_at[wave][32 * half + 8 * q + (lane >> 3)] + (lane & 7) * 16));
  };

  int base = t0 + wave * 64;
  if (base < t1) {
    Kv4Lines in[2];
    u32x4 k4, v4;
    int pos = position(base), next_pos = position(base + kThreads);
    int page = page_of(pos);
    place(pos, page, k4, v4);
    load(0, in[0]);
    load(1, in[1]);
    int next_page = page_of(next_pos), third_pos = position(base + 2 * kThreads);
    for (; base < t1; base += kThreads) {
      // this chunk's scales to where the tiles' lanes read them
      const uint64_t there = __ballot(page >= 0);
      uint32_t ks = 0, vs = 0;
      const int sh = 8 * (pos & 3);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        ks |= ((k4[q] >> sh) & 255u) << (8 * q);
        vs |= ((v4[q] >> sh) & 255u) << (8 * q);
      }
      if (page < 0) vs = 0;                    // (2^-127: what it multiplies stays finite)
      wave_lds_fence();
      sh_ks[wave][lane] = ks;
#pragma unroll
      for (int q = 0; q < 4; ++q) sh_vs[wave][q][lane] = (uint8_t)(vs >> (8 * q));
      pos = next_pos;
      page = next_page;
      place(pos, page, k4, v4);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t valid = (uint32_t)(there >> (32 * half));
        if (valid) {
          Kv4Tiles t;
          kv4_turn(in[half], sh_lines[wave], t);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const int first = 32 * half + 16 * s;
            t.ks[s] = reinterpret_cast<const uint8_t*>(&sh_ks[wave][first + c])[g];
            t.vs[s] = *reinterpret_cast<const uint32_t*>(&sh_vs[wave][c >> 2][first + 4 * g]);
          }
          kv4_step<F16>(t, valid, qB, a.d.scale_log2, st);
        }
        load(half, in[half]);
      }
      next_pos = third_pos;
      next_page = page_of(next_pos);
      third_pos = position(base + 3 * kThreads);
    }
  }
  kv4_finish(a, st, sh_lines, item, b, h, 1, DIRECT, 0);
}

__global__ __launch_bounds__(kAdThreads) void kv4_sparse_merge_kernel(const Kv4AttnArgs a) {
  const int unit = blockIdx.x, b = unit / a.d.n_ret;
  Kv4Share it = {};
  kv4_sparse_item(a, unit, true, &it);
  kv4_merge<kAdThreads>(a, 1, 0, 1, b, a.d.ret_heads[unit - b * a.d.n_ret], it.first, it.first + it.count, 0);
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
struct Kv4RangePlan {
  int32_t units, n_splits, target, even, grid;
  bool balanced, direct;
  size_t ws_bytes;
};
static Kv4RangePlan plan_range(const rtp_layer_desc* L, bool local, int32_t B, int64_t max_ctx) {
  Kv4RangePlan p = {};
  const int G = L->n_q_heads / L->n_kv_heads;
  p.units = B * L->n_kv_heads;
  int64_t blocks = (max_ctx + 15) / 16;
  if (local) {                                 // sink blocks, window blocks, one more where the window starts inside a block
    const int64_t set = ((int64_t)L->sink + 15) / 16 + ((int64_t)L->window + 15) / 16 + 1;
    if (set < blocks) blocks = set;
  }
  const int64_t most = (blocks + kKv4Round - 1) / kKv4Round;             // items of the longest unit
  int64_t n = kKv4Items / p.units;
  if (n > most) n = most;
  if (n < 1) n = 1;
  const bool many = p.units > kKv4Items / 2;
  // share of the compute units that whole rounds of workgroups keep busy, e equal items to a unit
  auto busy = [&](int e) {
    const int items = p.units * e, rounds = (items + kKv4Items - 1) / kKv4Items;
    return (float)items / ((float)rounds * kKv4Items);
  };
  if (blocks <= 48 + p.units) n = 1;
  p.n_splits = (int32_t)n;
  p.grid = p.units * p.n_splits;
  // Lengths can differ: shared out by the lengths, unless a unit in one piece is short.  (Beyond 256 sequences the plan, a pass over the
  // lengths in every wave, costs more than it saves.)  8 KV heads, contexts up to 32768, us, every unit in one piece / shared out:
  //                     all that long   one that long, the others a sixteenth   any length
  //   17 sequences      157 / 116       147 / 26                                 139 /  61
  //   32                177 / 178       143 / 33                                 140 /  91
  //   64                364 / 362       152 / 47                                 249 / 192
  //   128               710 / 720       160 / 69                                 412 / 374
  // Windows of contexts beyond them are full, i.e. equal: where units in one piece fill their rounds (231 - 256 of them, 461 - 512, ..), they
  // stay whole up to 12288 tokens, without the plan and the empty merge launch.  The host knows no lengths, so a ragged batch pays for it,
  // most of all one full window among short ones.  us, in one piece / shared out (full: every window; half: every other one, the rest of any
  // length; any: any length; one: one full, the others a sixteenth):
  //                                          full         half         any         one
  //   8192,  29 sequences of 8 KV heads     54 /  58     45 /  42     41 / 34     42 / 18
  //          32 of 8                        52 /  57     45 /  52     41 / 35     42 / 18
  //          128 of 2                       54 /  60     46 /  59     43 / 39     41 / 19
  //          256 of 1                       54 /  62     47 /  64     44 / 43     41 / 21
  //          58 of 8                        95 / 102     80 /  85     67 / 62     42 / 23
  //   12000, 32 of 8                        77 /  83     64 /  72     60 / 48     59 / 22
  //          64 of 8                       143 / 149    116 / 115     94 / 83     60 / 29
  // Outside the bands one piece loses everywhere (17 sequences of 8, window 8192: 44 / 38 full, 40 / 26 any); longer windows win less and lose
  // more by it (32 of 8, 16384: 90 / 95 and 73 / 53).
  const bool whole = blocks <= 48 + p.units || (local && many && blocks <= 768 && busy(1) >= 0.9f);
  p.balanced = !whole && most > 1 && B > 1 && B <= 256;
  if (p.balanced) {
    p.target = kKv4Items - p.units / 2;                                  // (a unit's number of items is rounded up, by a half on average)
    if (many) {
      p.target = p.units + 128 < 384 ? 384 : p.units + 128;
      float best = 0.f;                                                  // equal lengths: the fewest items that come close to the best
      for (int e = 1; e <= 4; ++e)
        if (busy(e) * 0.9f > best) { best = busy(e); p.even = e; }
    }
    int64_t grid = (int64_t)p.target + p.units;                          // items <= total / ceil(total / target) + units
    if (grid < (int64_t)p.units * p.even) grid = (int64_t)p.units * p.even;
    if (grid > p.units * most) grid = p.units * most;
    p.grid = (int32_t)grid;
  }
  p.direct = n == 1 && !p.balanced;
  p.ws_bytes = p.direct ? 0 : align_up((size_t)p.grid * G * kPartStride * sizeof(float), 256);
  return p;
}

static size_t range_ws(const rtp_layer_desc* L, bool local, int32_t B, int64_t max_ctx) {
  if (!L || B <= 0 || max_ctx <= 0 || max_ctx > kMaxLen || L->n_kv_heads <= 0 || L->n_q_heads < L->n_kv_heads ||
      (int64_t)B * L->n_kv_heads > kMaxUnits)
    return 256;
  // (what any smaller batch or context takes is enough too: fewer units may be cut into more items)
  size_t w = 256;
  for (int b = B < 256 ? B : 256; b > 0; --b) {
    const size_t one = plan_range(L, local, b, max_ctx).ws_bytes;
    if (one > w) w = one;
  }
  return w;
}

static int32_t check_io(const char* who, const void* q, const void* out, const void* ws, size_t ws_bytes, size_t need) {
  if (!q || !out) return fail(RTP_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  if (((uintptr_t)q & 15) || ((uintptr_t)out & 15)) return fail(RTP_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned", who);
  if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
    return fail(RTP_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required, got %zu", who, need, ws_bytes);
  return RTP_OK;
}

static void fill_attn(Kv4AttnArgs& a, const rtp_layer_desc* L, const HeadTable& ht, const void* q, void* out, float* lse, void* ws) {
  a.d = AttnDecodeArgs{};
  for (uint32_t& w : a.skip) w = 0;
  a.B = 0;
  a.balanced = 0;
  a.even = 0;
  a.d.q = (const uint16_t*)q;
  a.d.n_q_heads = L->n_q_heads;
  a.d.n_kv_heads = L->n_kv_heads;
  a.d.n_ret = L->n_ret;
  a.d.sink = L->sink;
  a.d.window = L->window;
  a.d.scale_log2 = softmax_scale_of(L) * 1.4426950408889634f;
  a.d.part = (float*)ws;
  a.d.out = (uint16_t*)out;
  a.d.lse = lse;
  a.d.f16 = L->kv_dtype == RTP_DTYPE_FP16;
  for (int j = 0; j < 64; ++j) a.d.ret_heads[j] = ht.ret_heads[j];
}

template <bool LOCAL>
static int32_t range_attn_kv4(const char* who, const rtp_layer_desc* layer, const void* q, const rtp_kv4_cache* cache,
                              const int32_t* ctx_len, int32_t B, int64_t max_ctx, void* out, float* lse, void* ws,
                              size_t ws_bytes, hipStream_t s) {
  HeadTable ht;
  int32_t rc = fill_head_table(layer, &ht, who);
  if (rc != RTP_OK) return rc;
  if (B <= 0 || max_ctx <= 0 || max_ctx > kMaxLen)
    return fail(RTP_ERR_INVALID_ARG, "%s: B must be positive, max_ctx in [1, 2^26]", who);
  if (!ctx_len) return fail(RTP_ERR_INVALID_ARG, "%s: NULL ctx_len", who);
  Kv4AttnArgs a;
  rc = check_kv4_cache(who, layer, cache, max_ctx, &a.c);
  if (rc != RTP_OK) return rc;
  if ((int64_t)B * layer->n_kv_heads > kMaxUnits)
    return fail(RTP_ERR_UNSUPPORTED, "%s: B * n_kv_heads = %lld exceeds %d", who, (long long)B * layer->n_kv_heads, kMaxUnits);
  const Kv4RangePlan p = plan_range(layer, LOCAL, B, max_ctx);
  const bool none = LOCAL && layer->n_ret == layer->n_q_heads;    // no local head
  rc = check_io(who, q, out, ws, ws_bytes, none ? 0 : p.ws_bytes);
  if (rc != RTP_OK) return rc;
  clear_error();
  if (none) return RTP_OK;
  fill_attn(a, layer, ht, q, out, lse, ws);
  a.d.ctx_len = ctx_len;
  a.d.units = p.units;
  a.d.n_splits = p.n_splits;
  a.d.target_items = p.target;
  a.max_len = (int32_t)max_ctx;
  a.direct = p.direct;
  a.B = B;
  a.balanced = p.balanced;
  a.even = p.even;
  if (LOCAL) {
    const int G = layer->n_q_heads / layer->n_kv_heads;
    for (int j = 0; j < layer->n_ret; ++j) a.skip[ht.ret_heads[j] / G / 4] |= 1u << (8 * (ht.ret_heads[j] / G % 4) + ht.ret_heads[j] % G);
  }
  const dim3 grid((unsigned)p.grid);
  if (a.d.f16) RTP_LAUNCH((kv4_range_kernel<LOCAL, true>), grid, dim3(kKv4Waves * 64), 0, s, a);
  else RTP_LAUNCH((kv4_range_kernel<LOCAL, false>), grid, dim3(kKv4Waves * 64), 0, s, a);
  if (!a.direct) {
    // a workgroup per head, or, with units for every compute unit, one for all heads of a unit (each makes the plan)
    const unsigned units = (unsigned)p.units, heads = (unsigned)(layer->n_q_heads / layer->n_kv_heads);
    if (p.units > kKv4Items / 2) RTP_LAUNCH((kv4_range_merge_kernel<LOCAL, true>), dim3(units), dim3(1024), 0, s, a);
    else RTP_LAUNCH((kv4_range_merge_kernel<LOCAL, false>), dim3(units, heads), dim3(256), 0, s, a);
  }
  return check_launch(who);
}

struct Kv4SparsePlan {
  int32_t target, grid;
  bool direct;
  size_t ws_bytes;
};
static Kv4SparsePlan plan_sparse(int64_t units, int64_t max_sel) {
  Kv4SparsePlan p = {};
  // Rows of up to 1024 tokens, two rounds of eight waves, in one launch (us; 1, 8, 64, 256 rows of 640 tokens 6.6 / 7.0 / 7.2 / 9.0 against
  // 8.5 / 8.9 / 9.2 / 15.4 in two launches, of 1024 tokens 8.3 / 8.7 / 9.0 / 13.6 against 8.5 / 8.8 / 9.2 / 21.8, 1 of 1536 10.6 against 8.5).
  p.direct = max_sel <= 1024;
  const int64_t most = units * ((max_sel + kSpWaves * 64 - 1) / (kSpWaves * 64));
  // All items resident at once, three workgroups on each of 256 compute units; a row's number of items is rounded up, by a half on average.
  // (256 rows of 8000 tokens 62 us, at twice the items 72; 200 to 30000 tokens a row 61 and 63.)
  p.target = (int32_t)(768 - units / 2 < 256 ? 256 : 768 - units / 2);
  int64_t grid = p.target + units;                                       // items <= total / ceil(total / target) + units
  if (grid > most) grid = most;
  p.grid = (int32_t)(p.direct ? units : grid);
  p.ws_bytes = p.direct ? 0 : align_up((size_t)p.grid * kPartStride * sizeof(float), 256);
  return p;
}

}  // namespace rtp

using namespace rtp;

extern "C" size_t rtp_sparse_attn_decode_kv4_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int64_t max_sel) {
  if (!layer || B <= 0 || max_sel <= 0 || max_sel > kMaxLen || layer->n_ret <= 0 || (int64_t)B * layer->n_ret > kAdMaxUnits) return 256;
  const size_t w = plan_sparse((int64_t)B * layer->n_ret, max_sel).ws_bytes;
  return w ? w : 256;
}

extern "C" int32_t rtp_sparse_attn_decode_kv4(const rtp_layer_desc* layer, const void* q, const rtp_kv4_cache* cache,
                                              const int32_t* sel_idx, int64_t sel_stride, const int32_t* sel_count,
                                              int64_t max_sel, int32_t B, void* out, float* lse, void* ws, size_t ws_bytes,
                                              void* stream) {
  const char* who = "rtp_sparse_attn_decode_kv4";
  HeadTable ht;
  int32_t rc = fill_head_table(layer, &ht, who);
  if (rc != RTP_OK) return rc;
  Kv4AttnArgs a;
  rc = check_kv4_cache(who, layer, cache, 0, &a.c);
  if (rc != RTP_OK) return rc;
  if (!sel_idx || !sel_count) return fail(RTP_ERR_INVALID_ARG, "%s: NULL sel_idx/sel_count", who);
  if (B <= 0 || max_sel <= 0 || max_sel > kMaxLen)
    return fail(RTP_ERR_INVALID_ARG, "%s: B must be positive, max_sel in [1, 2^26]", who);
  if (sel_stride < max_sel) return fail(RTP_ERR_INVALID_ARG, "%s: sel_stride must be >= max_sel", who);
  const int64_t units = (int64_t)B * layer->n_ret;
  if (units > kAdMaxUnits) return fail(RTP_ERR_UNSUPPORTED, "%s: B * n_ret = %lld exceeds %d", who, (long long)units, kAdMaxUnits);
  const Kv4SparsePlan p = plan_sparse(units, max_sel);
  rc = check_io(who, q, out, ws, ws_bytes, units ? p.ws_bytes : 0);
  if (rc != RTP_OK) return rc;
  clear_error();
  if (units == 0) return RTP_OK;
  fill_attn(a, layer, ht, q, out, lse, ws);
  a.d.sel_idx = sel_idx;
  a.d.sel_stride = sel_stride;
  a.d.sel_count = sel_count;
  a.d.units = (int32_t)units;
  a.d.target_items = p.target;
  a.max_len = (int32_t)max_sel;
  a.direct = p.direct;
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)p.grid);
  if (p.direct) {
    if (a.d.f16) RTP_LAUNCH((kv4_sparse_kernel<true, true>), grid, dim3(512), 0, s, a);
    else RTP_LAUNCH((kv4_sparse_kernel<false, true>), grid, dim3(512), 0, s, a);
    return check_launch(who);
  }
  if (a.d.f16) RTP_LAUNCH((kv4_sparse_kernel<true, false>), grid, dim3(kSpWaves * 64), 0, s, a);
  else RTP_LAUNCH((kv4_sparse_kernel<false, false>), grid, dim3(kSpWaves * 64), 0, s, a);
  RTP_LAUNCH(kv4_sparse_merge_kernel, dim3((unsigned)units), dim3(kAdThreads), 0, s, a);
  return check_launch(who);
}

extern "C" size_t rtp_local_attn_kv4_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int64_t max_ctx) {
  return range_ws(layer, true, B, max_ctx);
}
extern "C" size_t rtp_dense_attn_kv4_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int64_t max_ctx) {
  return range_ws(layer, false, B, max_ctx);
}
extern "C" int32_t rtp_local_attn_kv4(const rtp_layer_desc* layer, const void* q, const rtp_kv4_cache* cache,
                                      const int32_t* ctx_len, int32_t B, int64_t max_ctx, void* out, float* lse, void* ws,
                                      size_t ws_bytes, void* stream) {
  return range_attn_kv4<true>("rtp_local_attn_kv4", layer, q, cache, ctx_len, B, max_ctx, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_dense_attn_kv4(const rtp_layer_desc* layer, const void* q, const rtp_kv4_cache* cache,
                                      const int32_t* ctx_len, int32_t B, int64_t max_ctx, void* out, float* lse, void* ws,
                                      size_t ws_bytes, void* stream) {
  return range_attn_kv4<false>("rtp_dense_attn_kv4", layer, q, cache, ctx_len, B, max_ctx, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
