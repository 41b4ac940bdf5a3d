// rtp_kv_append: the new tokens' K rotated by their positions and V to the pages of a 16-bit cache, their queries rotated to the
// attention; and the checks of that cache's and of a batch's descriptors.
//
//   (x, y) -> scale (x cos a - y sin a, y cos a + x sin a),   a = position * inv_freq[i]
// The product of a 31-bit position and a 24-bit factor is exact in fp64, where its whole turns are taken off; cos and sin of the rest in fp32 are
// off by a few 2^-24 at every position, the rotation rounds once to 16 bits.
//
// Bound: every row of 256 bytes is read and written once.  16 lanes own a row, 8 values (one 16-byte load and store) each; a lane's partner
// values lie in its own word pair (neighbours) or in the lane rotary_dim / 16 further on (halves), which a cross-lane move fetches: no row
// is read twice, and the queries may be rotated in place.  A lane's eight angles are those of its place in the row, the same for every head, so they
// are computed once per token and kept in registers while the wave goes through the token's rows.  Up to 1024 tokens four waves share one.
// Measured: 4096 tokens of 32 + 8 + 8 heads (101 MB read and written) 17.8 us, 5.7 TB/s, where a copy of 4 GiB reaches 4.9; one token for each of 32
// sequences 5.0, of which the launch and the chain offsets -> length -> page -> row are all; a call in a row of calls 7.2, the host's time.
#include "kv16_cache.h"
#include "mfma_tile.h"

namespace rtp {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  Kv16Cache c;
  const int32_t* q_offset;
  const int32_t* ctx_len;
  int32_t B, total_q, max_q;
  const float* inv_freq;       // NULL: no rotation
  int32_t half;                // rotary_dim / 2
  int32_t interleaved;
  float scale;
  const uint16_t* q;           // NULL: K and V alone
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  int32_t n_q, n_kv;           // heads
  int32_t waves;               // per token: 1 or 4
};

template <bool F16>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(const AppendArgs a) {
  fetch_arguments<AppendArgs>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t slot_w = (int64_t)blockIdx.x * (kAppendThreads / 64) + wave;
  const int64_t i64 = slot_w / a.waves;
  if (i64 >= a.total_q) return;
  const int i = (int)i64, part = (int)(slot_w - i64 * a.waves);
  const int b = wave_last_at_most(a.q_offset, a.B, i);
  const NewTokens nt = new_tokens(a.q_offset, b, a.total_q, a.max_q);
  const int pos = a.ctx_len[b] - nt.n + (i - nt.q0);
  if (i < nt.q0 || i >= nt.q0 + nt.n || pos < 0) return;

  // ---- this lane's angles: rotary pairs of the values 8 * piece .. + 7 ----
  const int piece = lane & 15, half_pieces = a.half >> 3;
  const bool rotates = a.inv_freq && piece < 2 * half_pieces;
  const bool second = !a.interleaved && piece >= half_pieces;          // the y of its pairs
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (rotates) {
    auto turn = [&](int f, float& co, float& si) __attribute__((always_inline)) {
      const double x = (double)pos * (double)a.inv_freq[f], per_turn = 0.15915494309189533577;     // 1 / (2 pi)
      const double turns = x * per_turn, rest = (turns - rint(turns)) + fma(x, per_turn, -turns);
      sincospif((float)(2.0 * rest), &si, &co);
      co *= a.scale;
      si *= a.scale;
    };
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        turn(4 * piece + e / 2, cs[e], sn[e]);
        cs[e + 1] = cs[e];
        sn[e + 1] = sn[e];
        sn[e] = -sn[e];                                                // x' = x cos - y sin, y' = y cos + x sin
      }
    } else {
      const int f0 = 8 * (second ? piece - half_pieces : piece);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        turn(f0 + e, cs[e], sn[e]);
        if (!second) sn[e] = -sn[e];
      }
    }
  }
  const int partner = (lane & 48) | (second ? piece - half_pieces : piece + half_pieces);
  auto rotated = [&](const u32x4 x) __attribute__((always_inline)) {
    if (!a.inv_freq) return x;                                          // (the same for the whole launch)
    u32x4 y, out = x;
    if (!a.interleaved) {
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] = (uint32_t)__shfl((int)x[w], partner);
    }
    if (!rotates) return out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float x0 = lo16<F16>(x[w]), x1 = hi16<F16>(x[w]);
      const float y0 = a.interleaved ? x1 : lo16<F16>(y[w]), y1 = a.interleaved ? x0 : hi16<F16>(y[w]);
      out[w] = pack16<F16>(fmaf(x0, cs[2 * w], y0 * sn[2 * w]), fmaf(x1, cs[2 * w + 1], y1 * sn[2 * w + 1]));
    }
    return out;
  };

  // ---- where the token's K and V go ----
  const int32_t* pt = a.c.page_table + (int64_t)b * a.c.pt_stride;
  const int entry = pos >> a.c.page_shift;
  const int page = entry < a.c.pt_stride ? pt[entry] : -1;
  const bool stored = (uint32_t)page < (uint32_t)a.c.n_pages;
  const int64_t at = stored ? (int64_t)page * a.c.page_bytes + (int64_t)(pos & ((1 << a.c.page_shift) - 1)) * a.c.row_bytes + piece * 16 : 0;

  // ---- the token's rows, four at a time: queries, keys, values ----
  const int n_q = a.q ? a.n_q : 0, n_rows = n_q + 2 * a.n_kv;
  constexpr int kAhead = 3;                                            // rows in flight per lane
  for (int r0 = part * 4 + (lane >> 4); r0 - (lane >> 4) < n_rows; r0 += 4 * a.waves * kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int r = r0 + u * 4 * a.waves;
      x[u] = (u32x4){0u, 0u, 0u, 0u};
      if (r < n_rows) {
        const uint16_t* src = r < n_q ? a.q + (int64_t)i * a.q_stride + (int64_t)r * kHeadDim
                              : r < n_q + a.n_kv ? a.k + (int64_t)i * a.k_stride + (int64_t)(r - n_q) * kHeadDim
                                                 : a.v + (int64_t)i * a.v_stride + (int64_t)(r - n_q - a.n_kv) * kHeadDim;
        x[u] = *reinterpret_cast<const u32x4*>(src + piece * 8);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int r = r0 + u * 4 * a.waves;
      const u32x4 y = rotated(x[u]);                                    // (every lane takes part in the moves)
      if (r >= n_rows) continue;
      if (r < n_q) *reinterpret_cast<u32x4*>(a.q_out + (int64_t)i * a.q_out_stride + (int64_t)r * kHeadDim + piece * 8) = y;
      else if (!stored) continue;
      else if (r < n_q + a.n_kv) *reinterpret_cast<u32x4*>(a.c.K + (int64_t)(r - n_q) * a.c.head_bytes + at) = y;
      else *reinterpret_cast<u32x4*>(a.c.V + (int64_t)(r - n_q - a.n_kv) * a.c.head_bytes + at) = x[u];
    }
  }
}

int32_t check_kv16_cache(const char* who, const rtp_layer_desc* L, const rtp_kv_cache* c, int64_t max_tokens, Kv16Cache* out) {
  if (!c) return fail(RTP_ERR_INVALID_ARG, "%s: cache descriptor is NULL", who);
  if (!c->K || !c->V || !c->page_table) return fail(RTP_ERR_INVALID_ARG, "%s: NULL K/V/page_table", who);
  const int32_t ps = c->page_size;
  if (ps < 16 || (ps & (ps - 1)) || ps > (1 << 20))
    return fail(RTP_ERR_INVALID_ARG, "%s: page_size must be a power of two in [16, 2^20]", who);
  if (c->n_pages <= 0 || c->pt_stride <= 0) return fail(RTP_ERR_INVALID_ARG, "%s: n_pages and pt_stride must be positive", who);
  if (((uintptr_t)c->K & 15) || ((uintptr_t)c->V & 15) || (c->row_stride & 7) || (c->page_stride & 7) || (c->head_stride & 7))
    return fail(RTP_ERR_INVALID_ARG, "%s: K and V must be 16-byte aligned, their strides multiples of 8 elements", who);
  if (c->row_stride < kHeadDim || c->row_stride > (1 << 24))
    return fail(RTP_ERR_INVALID_ARG, "%s: row_stride must be in [128, 2^24] elements", who);
  if (c->page_stride < 0 || c->head_stride < 0 || c->page_stride > ((int64_t)1 << 40) || c->head_stride > ((int64_t)1 << 45) ||
      !rows_apart(c->row_stride, ps, c->page_stride, c->n_pages, c->head_stride, L->n_kv_heads))
    return fail(RTP_ERR_INVALID_ARG, "%s: strides let rows, pages or heads overlap", who);
  if (c->pt_stride < (max_tokens + ps - 1) / ps) return fail(RTP_ERR_INVALID_ARG, "%s: pt_stride must cover %lld tokens", who, (long long)max_tokens);
  int sh = 4;
  while ((1 << sh) < ps) ++sh;
  *out = Kv16Cache{(uint8_t*)c->K, (uint8_t*)c->V, c->head_stride * 2, c->page_stride * 2, (int32_t)(c->row_stride * 2), sh, c->n_pages,
                   c->page_table, c->pt_stride};
  return RTP_OK;
}

int32_t check_chunk(const char* who, const rtp_chunk* c) {
  if (!c) return fail(RTP_ERR_INVALID_ARG, "%s: chunk descriptor is NULL", who);
  if (!c->q_offset || !c->ctx_len) return fail(RTP_ERR_INVALID_ARG, "%s: NULL q_offset/ctx_len", who);
  if (c->B <= 0 || c->total_q < 0 || c->max_q <= 0 || c->max_ctx <= 0)
    return fail(RTP_ERR_INVALID_ARG, "%s: B, max_q and max_ctx must be positive, total_q not negative", who);
  if (c->B > kMaxSeqs || c->total_q > (1 << 24) || c->max_ctx > ((int64_t)1 << 30))
    return fail(RTP_ERR_UNSUPPORTED, "%s: more than 65535 sequences, 2^24 new tokens or contexts of 2^30", who);
  return RTP_OK;
}

bool rows_overlap(const void* x, int64_t x_stride, int64_t x_width, const void* y, int64_t y_stride, int64_t y_width, int64_t n) {
  const int64_t x0 = (int64_t)((uintptr_t)x / 2), y0 = (int64_t)((uintptr_t)y / 2);
  const int64_t x1 = x0 + (n - 1) * x_stride + x_width, y1 = y0 + (n - 1) * y_stride + y_width;
  if (x1 <= y0 || y1 <= x0) return false;
  if (x_stride != y_stride || n == 1) return true;
  // the same stride: places inside it
  const int64_t d = ((y0 - x0) % x_stride + x_stride) % x_stride;
  return d < x_width || d + y_width > x_stride;
}

}  // namespace rtp

using namespace rtp;

extern "C" int32_t rtp_kv_append(const rtp_layer_desc* layer, const rtp_kv_cache* cache, const rtp_chunk* chunk, const rtp_rope* rope,
                                 const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                 void* q_out, int64_t q_out_stride, void* stream) {
  const char* who = "rtp_kv_append";
  AppendArgs a = {};
  int32_t rc = check_layer(layer, who);
  if (rc != RTP_OK) return rc;
  rc = check_chunk(who, chunk);
  if (rc != RTP_OK) return rc;
  rc = check_kv16_cache(who, layer, cache, chunk->max_ctx, &a.c);
  if (rc != RTP_OK) return rc;
  if (!k || !v || (q && !q_out)) return fail(RTP_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  const int64_t q_width = (int64_t)layer->n_q_heads * kHeadDim, kv_width = (int64_t)layer->n_kv_heads * kHeadDim, most = (int64_t)1 << 40;
  if (((uintptr_t)k & 15) || ((uintptr_t)v & 15) || (q && (((uintptr_t)q & 15) || ((uintptr_t)q_out & 15))))
    return fail(RTP_ERR_INVALID_ARG, "%s: q, k, v and q_out must be 16-byte aligned", who);
  if ((k_stride & 7) || (v_stride & 7) || k_stride < kv_width || v_stride < kv_width || k_stride > most || v_stride > most ||
      (q && ((q_stride & 7) || (q_out_stride & 7) || q_stride < q_width || q_out_stride < q_width || q_stride > most || q_out_stride > most)))
    return fail(RTP_ERR_INVALID_ARG, "%s: token strides must be multiples of 8 elements that hold a token's rows", who);
  if (rope) {
    if (!rope->inv_freq) return fail(RTP_ERR_INVALID_ARG, "%s: NULL inv_freq", who);
    if (rope->rotary_dim < 16 || rope->rotary_dim > kHeadDim || (rope->rotary_dim & 15))
      return fail(RTP_ERR_UNSUPPORTED, "%s: rotary_dim %d unsupported (a multiple of 16, at most 128)", who, rope->rotary_dim);
    if (!(rope->scale >= 0.f) || rope->scale > 3.4e38f) return fail(RTP_ERR_INVALID_ARG, "%s: scale must be >= 0 (0 selects 1)", who);
    a.inv_freq = rope->inv_freq;
    a.half = rope->rotary_dim / 2;
    a.interleaved = rope->interleaved != 0;
    a.scale = rope->scale != 0.f ? rope->scale : 1.f;
  }
  const int64_t n = chunk->total_q;
  if (q && n > 0 && ((!(q_out == q && q_out_stride == q_stride) && rows_overlap(q, q_stride, q_width, q_out, q_out_stride, q_width, n)) ||
                     rows_overlap(k, k_stride, kv_width, q_out, q_out_stride, q_width, n) ||
                     rows_overlap(v, v_stride, kv_width, q_out, q_out_stride, q_width, n)))
    return fail(RTP_ERR_INVALID_ARG, "%s: q_out overlaps q, k or v without being q itself", who);
  clear_error();
  if (n == 0) return RTP_OK;
  a.q_offset = chunk->q_offset;
  a.ctx_len = chunk->ctx_len;
  a.B = chunk->B;
  a.total_q = chunk->total_q;
  a.max_q = chunk->max_q;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.q_out = (uint16_t*)q_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.n_q = layer->n_q_heads;
  a.n_kv = layer->n_kv_heads;
  a.waves = n <= 1024 ? 4 : 1;
  const dim3 grid((unsigned)((n * a.waves + 3) / 4));
  if (layer->kv_dtype == RTP_DTYPE_FP16) RTP_LAUNCH(kv_append_kernel<true>, grid, dim3(kAppendThreads), 0, (hipStream_t)stream, a);
  else RTP_LAUNCH(kv_append_kernel<false>, grid, dim3(kAppendThreads), 0, (hipStream_t)stream, a);
  return check_launch(who);
}
