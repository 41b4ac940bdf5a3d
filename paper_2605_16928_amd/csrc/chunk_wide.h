// A query tile of up to 256 rows: eight waves of 32 rows, two per SIMD, share every staged tile of 64 keys.
//
// Nothing hides latency by itself at two waves per SIMD, so the loop is pipelined over blocks of 32 keys by hand: while the probabilities of a
// block are computed on the vector ALU, the matrix pipe runs the PV product of the block before and the score product of the one behind.  For that
// nothing may touch the accumulators in between, so there is no running maximum: every row takes its largest score in the range's first tile for a
// reference, and a range after whose pass some row's sum or output says that this did not do (chunk_reach.h; or not finite), or
// which met a page that is not there, is left to a launch that goes through such ranges with a running maximum (exact_pass).
//
// Probabilities enter the product as 16 bits, once: outputs are off by 0.0023 (bf16, relative to their size) where 0.0017 is their own rounding.  The
// second part of tiles of few rows would be half as many products again where the matrix cores are the bound: these alone, without the subtractions and
// roundings, take 4096 tokens behind 126976 from 979 to 1262 us, a mixed batch from 161 to 197.
//
// K/V tiles rotate through three LDS buffers with one barrier per tile, in its middle: it publishes tile x + 1, and behind it every wave is done
// with tile x - 1, whose buffer tile x + 2 fills.  Tiles that every row sees in full run in a loop without a branch; the others -- the first, those
// on the window's edge and on the diagonal -- block by block, with masks.
//
// Measured: 4096 tokens behind 126976, 4 heads (1.08 TFLOP) 950 us with the merge, 1.14 PFLOP/s, where a product of 8192^3 reaches 1.59; a prompt of
// 8192 tokens, 32 over 8 heads, 504 us, 1.09; 4096 behind 28672 over 4 bits 1716, 1.20.  Bound by issue: the matrix cores are busy for 58 % of
// the launch, the LDS reads (every wave reads every tile) for as long, and exponentials, rounding and sums take most of a SIMD's other slots.
//
// 16-bit rows go to LDS by direct loads.  The four rows that a wave brings per instruction lie in one page, whose place is a scalar: 64 of them, for
// 32 tiles, are looked up at a time, a lane each, a window ahead, and taken from there with two lane reads.  4-bit rows come through registers
// a tile ahead, 16 bytes per lane, and are turned into 16 bits on their way to LDS, between the products.
#pragma once

#include "chunk_tile.h"
#include "chunk_reach.h"

namespace rtp {

constexpr int kCkStages = 3;
constexpr int kCkWideLds = kCkTileBytes * kCkStages;

// Sums: l of the probabilities as rounded (what the outputs are divided by), F of them before (what the log-sum is of; FULL only).
template <bool F16, bool LOCAL, bool KV4, bool FULL>
struct ChunkWide {
  const ChunkArgs& a;
  const ChunkTile& t;
  unsigned char* const smem;
  const int lane, wave, g, r, row;
  const bool qok;
  const int w_lo, w_hi;                          // positions of the wave's first and last row; w_hi < 0: the wave has none
  const float c;
  const ChunkReads rd;
  const ChunkSight sight;
  u32x4 q[8];
  f32x16 O[4];
  float m, l, F;
  // staging: places of the rows that this wave brings, relative to the head's pool: piece `lane` of the window, kPieces to a tile
  static constexpr int kPieces = KV4 ? 1 : 2, kWindow = 64 / kPieces, kRowsEach = KV4 ? 8 : 4;
  const uint8_t* base0;                          // K, or codes
  const uint8_t* base1;                          // V, or scales
  uint32_t at_lo, at_hi, sc_lo, sc_hi;           // this window's (scales: 4-bit only)
  int next_page;                                 // the next window's, as the table has it
  uint32_t off0, off1;                           // the lane's place inside its rows
  bool lost;
  u32x4 codes;                                   // 4-bit: the rows on their way
  uint32_t scale;

  __device__ __forceinline__ ChunkWide(const ChunkArgs& a_, const ChunkTile& t_, unsigned char* smem_)
      : a(a_), t(t_), smem(smem_), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), g(lane >> 5), r(lane & 31),
        row(wave * 32 + r), qok(row < t_.rows), w_lo(wave * 32 < t_.rows ? chunk_row_pos(t_, wave * 32) : -1),
        w_hi(wave * 32 < t_.rows ? chunk_row_pos(t_, min(wave * 32 + 31, t_.rows - 1)) : -1), c(a_.scale_log2), rd(chunk_reads()),
        sight(chunk_sight(a_.shape, t_, row)), lost(false), n_tiles(t_.it_hi - t_.it_lo), n_full(0), n_moved(0) {
    if constexpr (KV4) {
      base0 = a.c4.codes + (int64_t)t.kvh * a.c4.code_head_stride;
      base1 = a.c4.scales + (int64_t)t.kvh * a.c4.scale_head_stride;
      off0 = lane * 16;
      off1 = (lane >> 5) * kKv4Group + (lane & 7) * 4 + ((lane >> 3) & 3);
    } else {
      base0 = a.c16.K + (int64_t)t.kvh * a.c16.head_bytes;
      base1 = a.c16.V + (int64_t)t.kvh * a.c16.head_bytes;
      const int sub = lane >> 4, pos = lane & 15;
      off0 = sub * a.c16.row_bytes + (pos ^ ((4 * wave + sub) & 15)) * 16;
      off1 = sub * a.c16.row_bytes + ((((pos >> 1) ^ (2 * sub)) << 1) | (pos & 1)) * 16;
    }
  }

  // The x-th tile of the pass: the range's tiles in order, but that those between its first and the first one that every row sees in full come
  // behind the full ones: so these are neighbours, and the loop over them has one tile in front of it.
  int n_tiles, n_full, n_moved;
  __device__ __forceinline__ int n0_of(int x) const {
    const int y = n_moved > 0 && x >= 1 && x <= n_full + n_moved ? (x <= n_full ? x + n_moved : x - n_full) : x;
    return chunk_tile_n0(t, t.it_lo + y);
  }
  __device__ __forceinline__ void arrange() {
    int lo = t.it_lo, hi = min(t.it_hi, min(t.m_lo + 1, t.kend) / kCkK - t.gap);                // (m_lo >= 0 where there are full tiles)
    if (LOCAL) lo = max(max(lo, t.sink_tiles), (max(t.m_hi - a.shape.window + 1, 0) + kCkK - 1) / kCkK - t.gap);
    lo = max(lo, t.it_lo + 1);
    if (lo < hi) {
      n_moved = lo - t.it_lo - 1;
      n_full = hi - lo;
    }
  }
  __device__ __forceinline__ bool any_seen(int n, int len) const { return chunk_any_seen<LOCAL>(a.shape, t, w_lo, w_hi, n, len); }
  __device__ __forceinline__ bool all_seen(int n, int len) const { return chunk_all_seen<LOCAL>(a.shape, t, w_lo, w_hi, n, len); }
  // ---- staging ----
  // First of the rows of piece p (counted from the pass's first tile) that this wave brings; past the last key and the last tile: those of the last.
  __device__ __forceinline__ int piece_row(int p) const {
    const int n0 = n0_of(min(p / kPieces, n_tiles - 1)) + (p % kPieces) * 32 + kRowsEach * wave;
    return min(n0, (t.kend - 1) & ~(kRowsEach - 1));
  }
  __device__ __forceinline__ void look_up(int window) {
    next_page = t.pt[piece_row(window * 64 + lane) >> (KV4 ? a.c4.page_shift : a.c16.page_shift)];
  }
  // (an entry that names no page is taken for the first page; the range is repeated if some row sees these keys)
  __device__ __forceinline__ void take_window(int window) {
    const int n = piece_row(window * 64 + lane);
    const bool there = (uint32_t)next_page < (uint32_t)(KV4 ? a.c4.n_pages : a.c16.n_pages);
    const uint32_t page = there ? (uint32_t)next_page : 0u;
    const uint32_t slot = n & ((1 << (KV4 ? a.c4.page_shift : a.c16.page_shift)) - 1);
    lost = lost || __ballot(!there && (!LOCAL || chunk_any_seen<LOCAL>(a.shape, t, t.m_lo, t.m_hi, n, kRowsEach))) != 0ull;
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
  }
  __device__ __forceinline__ int64_t place(uint32_t lo, uint32_t hi, int p) const {
    return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, p) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)lo, p));
  }
  // The window of tile x is the current one; called for every x in turn.
  __device__ __forceinline__ void advance(int x) {
    if (x % kWindow == 0) {
      take_window(x / kWindow);
      look_up(x / kWindow + 1);
    }
  }
  __device__ __forceinline__ uint32_t lds_of(int slot) const {
    return (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char*)smem + slot * kCkTileBytes;
  }
  // One of the four loads of tile x: K or V, first or second 32 rows.
  __device__ __forceinline__ void load16(int x, int slot, int jj, bool v, uint32_t off) const {
    const int64_t at = place(at_lo, at_hi, (x % kWindow) * kPieces + jj);
    chunk_load_lds(lds_of(slot) + (v ? kCkTileBytes / 2 : 0) + (jj * kCkWaves + wave) * 1024, (v ? base1 : base0) + at, off);
  }
  // The lane's place where the rows behind the last key have to repeat it (they are masked, but have to be rows that somebody has written).
  __device__ __forceinline__ uint32_t edge_off(int p, bool second) const {
    const int left = t.kend - 1 - piece_row(p);
    if constexpr (KV4) {
      const int n = min(lane >> 3, left), of = lane & 7;
      return second ? (uint32_t)((n >> 2) * kKv4Group + of * 4 + (n & 3)) : (uint32_t)(n * kKv4Row + of * 16);
    } else {
      const int sub = lane >> 4;
      return (second ? off1 : off0) - (uint32_t)((sub - min(sub, left)) * a.c16.row_bytes);
    }
  }
  __device__ __forceinline__ void fetch_codes(int x, bool edge) {
    const int p = x % kWindow;
    const uint32_t o0 = edge ? edge_off(x, false) : off0, o1 = edge ? edge_off(x, true) : off1;
    codes = *reinterpret_cast<const u32x4*>(base0 + place(at_lo, at_hi, p) + o0);
    scale = (base1 + place(sc_lo, sc_hi, p))[o1];
  }
  __device__ __forceinline__ void put_codes(int slot, int i) const {        // a quarter of the lane's values
    const int n = 8 * wave + (lane >> 3), piece = lane & 7, blk = piece & 3;
    const int ck = (4 * blk + i) ^ (n & 15), cv = ((2 * blk + (i >> 1)) ^ (2 * (n & 3))) * 2 + (i & 1);
    *reinterpret_cast<u32x4*>(smem + slot * kCkTileBytes + n * 256 + (piece < 4 ? ck * 16 : kCkTileBytes / 2 + cv * 16)) =
        decode8<F16>(codes[i], __uint_as_float(scale << 23));
  }
  // All of tile x, masked or not.  4-bit: the rows that have come go to LDS, tile x + 1 sets out.
  __device__ __forceinline__ void bring(int x, int slot) {
    if constexpr (KV4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) put_codes(slot, i);
      advance(x + 1);
      fetch_codes(x + 1, true);
    } else {
      advance(x);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        load16(x, slot, jj, false, edge_off(x * kPieces + jj, false));
        load16(x, slot, jj, true, edge_off(x * kPieces + jj, true));
      }
    }
  }
  __device__ __forceinline__ void begin() {                                 // before the first bring()
    look_up(0);
    // (behind the first pages, which the first rows wait for.  Rows behind the tile's last repeat it.)
    const int row_c = min(row, t.rows - 1), rt = (row_c * t.over) >> 16;
    const uint16_t* src = a.q + (t.q0 + rt) * a.q_stride + chunk_head(a, t, row_c, rt) * kHeadDim + g * 8;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) q[kk] = *reinterpret_cast<const u32x4*>(src + kk * 16);
    if constexpr (KV4) {
      advance(0);
      fetch_codes(0, true);
    }
  }
  __device__ __forceinline__ void landed() const {
    if constexpr (!KV4) chunk_wait_loads<0>();
  }

  // ---- products ----
  __device__ __forceinline__ void clear() {
    l = F = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
  }
  __device__ __forceinline__ void scores(const unsigned char* tile, int kb, f32x16& S) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) S = mfma32<F16>(chunk_read_k(tile + kb * 8192, rd, kk), q[kk], S);
  }
  __device__ __forceinline__ void pv(const unsigned char* tile, int kb, const uint32_t (&P)[8]) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int db = 0; db < 4; ++db)
        O[db] = mfma32<F16>(chunk_read_v(tile + kCkTileBytes / 2 + kb * 8192, rd, tt, db), (u32x4){P[4 * tt], P[4 * tt + 1], P[4 * tt + 2], P[4 * tt + 3]}, O[db]);
  }
  // Adds both halves of a packed pair: what the PV product multiplies.  (Assembly, so that it stays between the products where it is written; its
  // result may be read by another kind of instruction after three wait states only.)
  static __device__ __forceinline__ void add_pair(float& s, uint32_t pk) {
    if constexpr (F16) asm volatile("v_dot2c_f32_f16 %0, %1, %2" : "+v"(s) : "v"(pk), "v"(0x3c003c00u));
    else asm volatile("v_dot2c_f32_bf16 %0, %1, %2" : "+v"(s) : "v"(pk), "v"(0x3f803f80u));
  }
  static __device__ __forceinline__ void settled(float& s) { asm volatile("s_nop 3" : "+v"(s)); }

  float mc, l_blk, f_blk;
  __device__ __forceinline__ void pair(int k, const f32x16& S, uint32_t (&P)[8]) {
    const float p0 = fast_exp2(fmaf(S[2 * k], c, -mc)), p1 = fast_exp2(fmaf(S[2 * k + 1], c, -mc));
    P[k] = pack16<F16>(p0, p1);
    add_pair(l_blk, P[k]);
    if constexpr (FULL) {
      asm volatile("v_add_f32 %0, %0, %1" : "+v"(f_blk) : "v"(p0));
      asm volatile("v_add_f32 %0, %0, %1" : "+v"(f_blk) : "v"(p1));
    }
  }
  __device__ __forceinline__ void begin_block() {
    mc = m * c;
    l_blk = f_blk = 0.f;
  }
  __device__ __forceinline__ void end_block() {
    settled(l_blk);
    l += l_blk;
    if constexpr (FULL) F += f_blk;
  }

  // K operands are read kAheadK products ahead, V operands kAheadV, a stream's first ones during the stream before.
  static constexpr int kAheadK = 5, kAheadV = 4;
  u32x4 ka_first[kAheadK], va_first[kAheadV];
  __device__ __forceinline__ void first_k(const unsigned char* tile, int kb) {
#pragma unroll
    for (int kk = 0; kk < kAheadK; ++kk) ka_first[kk] = chunk_read_k(tile + kb * 8192, rd, kk);
  }
  __device__ __forceinline__ void first_v(const unsigned char* tile, int kb) {
#pragma unroll
    for (int k = 0; k < kAheadV; ++k) va_first[k] = chunk_read_v(tile + kCkTileBytes / 2 + kb * 8192, rd, k >> 2, k & 3);
  }
  // PV of the block before (Pin, in `tile`) beside the first half of this block's probabilities
  __device__ __forceinline__ void pv_stream(const unsigned char* tile, int kb, const uint32_t (&Pin)[8], const f32x16& S, uint32_t (&P)[8],
                                            const unsigned char* next_tile, int next_kb) {
    begin_block();
    u32x4 va[8];
#pragma unroll
    for (int k = 0; k < kAheadV; ++k) va[k] = va_first[k];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int tt = k >> 2, db = k & 3;
      if (k + kAheadV < 8) va[k + kAheadV] = chunk_read_v(tile + kCkTileBytes / 2 + kb * 8192, rd, (k + kAheadV) >> 2, (k + kAheadV) & 3);
      if (k == 8 - kAheadV) first_k(next_tile, next_kb);
      O[db] = mfma32<F16>(va[k], (u32x4){Pin[4 * tt], Pin[4 * tt + 1], Pin[4 * tt + 2], Pin[4 * tt + 3]}, O[db]);
      if (k & 1) pair(k / 2, S, P);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // scores of the block behind (Snext) beside the other half
  template <typename Work>
  __device__ __forceinline__ void score_stream(const unsigned char* tile, int kb, f32x16& Snext, const f32x16& S, uint32_t (&P)[8], Work&& work) {
    u32x4 ka[8];
#pragma unroll
    for (int kk = 0; kk < kAheadK; ++kk) ka[kk] = ka_first[kk];
#pragma unroll
    for (int i = 0; i < 16; ++i) Snext[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      if (kk + kAheadK < 8) ka[kk + kAheadK] = chunk_read_k(tile + kb * 8192, rd, kk + kAheadK);
      Snext = mfma32<F16>(ka[kk], q[kk], Snext);
      work(kk);
      if (kk & 1) pair(4 + kk / 2, S, P);
      __builtin_amdgcn_sched_barrier(0);
    }
    end_block();
  }

  static constexpr float kOutstanding = 12.f, kAlike = 10.f;                // (in the logarithm to the base of 2)
  // ---- the pass against fixed references; true: some row needs another ----
  __device__ __forceinline__ bool fast_pass() {
    const float ninf = -__builtin_huge_valf();
    f32x16 S;
    uint32_t P0[8], P1[8];
    clear();
    arrange();
    begin();
    bring(0, 0);
    bring(1, 1);
    landed();
    __syncthreads();
    // the buffers of tile x - 1, which tile x + 2 goes to, of tile x and of tile x + 1
    static_assert(kCkStages == 3, "they go round");
    int slot_before = 2, slot_here = 0, slot_next = 1;
    auto tile_of = [&](int slot) __attribute__((always_inline)) { return smem + slot * kCkTileBytes; };
    auto go_round = [&]() __attribute__((always_inline)) {
      const int freed = slot_before;
      slot_before = slot_here;
      slot_here = slot_next;
      slot_next = freed;
    };
    // (of what the row sees there, if it does see anything)
    float any = ninf;
    m = ninf;
    // fp16: of the first tile that every row sees in full, if there is one, unless one of the two tiles stands out: then 2^12 below its best, or near
    // the other's.  A context's first token often has most of the softmax, at 2^15 or more above the others, and fp16 has 14 binades below the
    // reference in which a probability is whole, 16 above.  (A window: rows see a part of the first tile, or nothing, and a few keys' best may be 2^16 below the
    // row's.  A chunk of 4096 tokens, sink 0, 1210 us and 517, all units having been taken again.)
    float full = ninf;
    if constexpr (F16) {
      if (n_full > 0) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          scores(tile_of(slot_next), kb, S);
#pragma unroll
          for (int i = 0; i < 16; ++i) full = fmaxf(full, S[i]);
        }
        full = fmaxf(full, __shfl_xor(full, 32));
      }
    }
#pragma unroll
    for (int kb = 1; kb >= 0; --kb) {
      scores(smem, kb, S);
      const int nb0 = n0_of(0) + kb * 32;
#pragma unroll
      for (int i = 0; i < 16; ++i) any = fmaxf(any, S[i]);
      if (!all_seen(nb0, 32)) chunk_mask<LOCAL>(sight, nb0 + 4 * g, S);
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, S[i]);
    }
    m = fmaxf(m, __shfl_xor(m, 32));
    any = fmaxf(any, __shfl_xor(any, 32));
    const bool held = m > ninf || full > ninf;
    if (full > ninf) m = m > ninf ? fmaxf(fminf(full, m + kAlike / c), fmaxf(full, m) - kOutstanding / c) : full;
    else if (!held) m = any;
    // At the start of half hf of tile x: S holds the scores of that block if the wave has a row that sees one of its keys; if `pend`, the
    // probabilities of the block before wait in P1 (hf = 0, V in the tile before) or P0; tiles x and x + 1 are in LDS.
    bool pend = false;
    int x = 0;
    auto half = [&](auto hf_tag) __attribute__((always_inline)) {
      constexpr int hf = decltype(hf_tag)::value;
      const int nb0 = n0_of(x) + hf * 32;
      const uint32_t (&Pin)[8] = hf == 0 ? P1 : P0;
      uint32_t (&Pout)[8] = hf == 0 ? P0 : P1;
      if (pend) pv(tile_of(hf == 0 ? slot_before : slot_here), 1 - hf, Pin);
      pend = any_seen(nb0, 32);
      if (pend) {
        if (!all_seen(nb0, 32)) chunk_mask<LOCAL>(sight, nb0 + 4 * g, S);
        begin_block();
#pragma unroll
        for (int k = 0; k < 8; ++k) pair(k, S, Pout);
        end_block();
      }
      if (hf == 0) {
        if (any_seen(nb0 + 32, 32)) scores(tile_of(slot_here), 1, S);
        landed();
        __syncthreads();
      } else {
        bring(x + 2, slot_before);                                         // (behind the last tile: once more into a buffer that nobody reads)
        if (x + 1 < n_tiles && any_seen(n0_of(x + 1), 32)) scores(tile_of(slot_next), 0, S);
      }
    };
    auto edge_tile = [&]() __attribute__((always_inline)) {
      half(std::integral_constant<int, 0>{});
      half(std::integral_constant<int, 1>{});
      ++x;
      go_round();
    };
    // The loop without masks: full tiles, while the rows that it sends for are all there (the last tile may be a part of one).
    constexpr int kSends = KV4 ? 3 : 2;
    const bool part = chunk_tile_n0(t, t.it_hi - 1) + kCkK > t.kend;
    const int x_stop = min(n_full + 1, part ? n_tiles - 1 - kSends : n_tiles);
    edge_tile();
    if (x >= x_stop) {
    } else if (w_hi >= 0) {
      if (!pend) {
#pragma unroll
        for (int k = 0; k < 8; ++k) P1[k] = 0u;
      }
      pend = true;
      f32x16 S1;
      do {
        advance(x + kSends);
        const int x_end = min(x_stop, (x + kSends) / kWindow * kWindow + kWindow - kSends);      // (as far as the window reaches)
        first_v(tile_of(slot_before), 1);
        do {
          pv_stream(tile_of(slot_before), 1, P1, S, P0, tile_of(slot_here), 1);
          score_stream(tile_of(slot_here), 1, S1, S, P0, [](int) __attribute__((always_inline)) {});
          first_v(tile_of(slot_here), 0);
          landed();
          __syncthreads();
          pv_stream(tile_of(slot_here), 0, P0, S1, P1, tile_of(slot_next), 0);
          score_stream(tile_of(slot_next), 0, S, S1, P1, [&](int kk) __attribute__((always_inline)) {
            if constexpr (KV4) {
              if (kk < 4) put_codes(slot_before, kk);
              if (kk == 4) fetch_codes(x + 3, false);
            } else {
              if (kk < 4) load16(x + 2, slot_before, kk >> 1, kk & 1, (kk & 1) ? off1 : off0);
            }
          });
          first_v(tile_of(slot_here), 1);
          ++x;
          go_round();
        } while (x < x_end);
      } while (x < x_stop);
    } else {
      do {
        advance(x + kSends);
        landed();
        __syncthreads();
        if constexpr (KV4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) put_codes(slot_before, i);
          fetch_codes(x + 3, false);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) load16(x + 2, slot_before, k >> 1, k & 1, (k & 1) ? off1 : off0);
        }
        ++x;
        go_round();
      } while (x < x_stop);
    }
    while (x < n_tiles) edge_tile();
    if (pend) pv(tile_of(slot_before), 1, P1);
    landed();
    // Was every reference within reach, and are the outputs finite?  (A row's keys are counted where its sum alone does not say so.)
    const float sum = l + __shfl_xor(l, 32);
    float z = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) z = fmaf(O[db][i], 0.f, z);
    bool bad = lost || !(z == 0.f) || !(sum < 0x1p100f);
    if (qok && sight.hi >= 0 && !chunk_surely_in_reach(F16, held, sum)) {
      const int split = max(t.it_lo, min(t.it_hi, t.sink_tiles));           // the range's tiles in front of the gap, and those behind it
      const int seen = chunk_seen_among(t.it_lo * kCkK, split * kCkK, LOCAL, a.shape.sink, sight.lo, sight.hi) +
                       chunk_seen_among((split + t.gap) * kCkK, (t.it_hi + t.gap) * kCkK, LOCAL, a.shape.sink, sight.lo, sight.hi);
      bad = bad || !chunk_in_reach(F16, held, sum, seen);
    }
    return __syncthreads_or(bad ? 1 : 0) != 0;
  }

  // ---- running maximum, accumulators rescaled in place, keys masked by their pages too (apart from the pass above: its registers are its own).
  // fp16: probabilities are taken times 2^15, the most that it holds, and results by as much less. ----
  static constexpr float kLift = F16 ? 15.f : 0.f, kLower = F16 ? 0x1p-15f : 1.f;
  __device__ __forceinline__ void exact_pass() {
    const float ninf = -__builtin_huge_valf();
    f32x16 S;
    uint32_t P[8];
    const uint32_t none[8] = {};
    clear();
    m = ninf;
    __syncthreads();
    begin();
    if constexpr (!KV4) bring(0, 0);
#pragma unroll 1
    for (int x = 0; x < n_tiles; ++x) {
      const unsigned char* const tile = smem + (x & 1) * kCkTileBytes;
      if constexpr (KV4) bring(x, x & 1);
      landed();
      __syncthreads();
      if constexpr (!KV4) bring(x + 1, (x + 1) & 1);
#pragma unroll 1
      for (int kb = 0; kb < 2; ++kb) {
        const int nb0 = n0_of(x) + kb * 32;
        if (!any_seen(nb0, 32)) continue;                                   // (the same for the whole wave)
        scores(tile, kb, S);
        const uint32_t seen = chunk_seen<LOCAL, KV4>(a, t, sight, nb0 + 4 * g);
        float mx = ninf;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          S[i] = (seen >> i) & 1u ? S[i] : ninf;
          mx = fmaxf(mx, S[i]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx), ref = m_new == ninf ? 0.f : m_new, corr = fast_exp2((m - ref) * c), mc = ref * c - kLift;
        float sum = 0.f, full = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = fast_exp2(fmaf(S[i], c, -mc)), p1 = fast_exp2(fmaf(S[i + 1], c, -mc));
          P[i >> 1] = pack16<F16>(p0, p1);
          full += p0 + p1;
          sum += lo16<F16>(P[i >> 1]) + hi16<F16>(P[i >> 1]);
        }
        l = l * corr + sum;
        F = F * corr + full;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[db][i] *= corr;
        m = m_new;
        const unsigned char* const v_rows = tile + kCkTileBytes / 2 + kb * 8192;
        uint32_t odd = 0;
        if (__ballot(seen != 0xffffu) != 0ull) {
#pragma unroll
          for (int k = 0; k < 8; ++k) odd |= chunk_not_finite<F16>(chunk_read_v(v_rows, rd, k >> 2, k & 3));
        }
        if (__ballot(odd != 0u) == 0ull) pv(tile, kb, P);
        else chunk_pv_seen<F16>(v_rows, seen, P, none, O);
      }
      __syncthreads();
    }
    landed();                                                               // (what the last tile sent for)
    __syncthreads();
    if constexpr (F16) {
      l *= kLower;
      F *= kLower;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] *= kLower;
    }
  }

  // Outputs go by way of the wave's LDS, to be written as whole rows: group u of four outputs of row r at u ^ 2 (r % 16).  (All waves are done with
  // the tiles.)
  __device__ __forceinline__ void store() {
    const float sum = l + __shfl_xor(l, 32), full = F + __shfl_xor(F, 32);
    if (t.splits == 1) {
      unsigned char* const mine = smem + wave * 32 * 256;
      const bool none = sum == 0.f;
      const float inv = none ? 0.f : 1.f / sum;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const u32x2 w = {pack16<F16>(O[db][i4 * 4] * inv, O[db][i4 * 4 + 1] * inv), pack16<F16>(O[db][i4 * 4 + 2] * inv, O[db][i4 * 4 + 3] * inv)};
          *reinterpret_cast<u32x2*>(mine + r * 256 + (((db * 8 + i4 * 2 + g) ^ (2 * (r & 15))) << 3)) = none ? (u32x2){0u, 0u} : w;
        }
      if (a.lse && g == 0 && qok) {
        const int rt = (row * t.over) >> 16;
        a.lse[(t.q0 + rt) * a.n_q_heads + chunk_head(a, t, row, rt)] = none ? -__builtin_huge_valf() : m * a.scale + logf(full);
      }
      chunk_wave_fence();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = 4 * i + (lane >> 4), to = wave * 32 + n, rt = (to * t.over) >> 16, piece = lane & 15;
        const u32x4 w = *reinterpret_cast<const u32x4*>(mine + n * 256 + ((piece ^ (n & 15)) << 4));
        if (to < t.rows) *reinterpret_cast<u32x4*>(a.out + ((t.q0 + rt) * a.n_q_heads + chunk_head(a, t, to, rt)) * kHeadDim + piece * 8) = w;
      }
      return;
    }
    if (!qok) return;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const float o[4] = {O[db][i4 * 4], O[db][i4 * 4 + 1], O[db][i4 * 4 + 2], O[db][i4 * 4 + 3]};
        const int dim = db * 32 + i4 * 8 + g * 4;
        chunk_store4<F16>(a, t, row, dim, m, sum, full, o);
      }
  }
};

}  // namespace rtp
