// The 4-bit cache's own traffic: rtp_kv4_append stores new tokens, rtp_kv4_read gives stored tokens back at 16 bits (for the prefill
// of a next chunk, whose kernels read 16-bit rows).
//
//   scale  s = max(2, E - 2 + [M >= 0.75]),  amax = max |x| of the block = (1 + M) 2^(E - 127)
//   code   nearest e2m1 value of x 2^(127 - s), ties to the even code
// amax lands in [3.5, 7) steps: where the usual floor(log2 amax) - 2 would leave it in [7, 8), past the largest code 6 by more than
// half a step, the next scale is taken, so a block's maximum is never off by more than half a step either.  The bottom, s = 2, keeps
// every stored value a normal number of bf16; a block of zeros has it too.  A block with an infinity or a NaN gets s = 255.
//
// Both kernels are bound by their bytes: 512 in and 136 out per token and KV head, or the other way round.  16 lanes own a row (8 dims
// each: one 16-byte load, one 4-byte store of codes), a block's maximum is two DPP steps over a quad, and a 16-lane group takes the
// four positions of one scale group: eight loads in flight per lane, and whole scale words where all four positions are written.
// The 16-bit rows that read writes go past the caches: with 32768 tokens of 8 KV heads (170 MB moved) it takes 26 us, 6.5 TB/s, with
// ordinary stores 33; 4096 tokens are appended in 6 us.
#include "kv4_cache.h"

namespace rtp {

constexpr int kStoreThreads = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

struct Kv4StoreArgs {
  Kv4Cache c;
  uint16_t* k;                 // append: source; read: destination
  uint16_t* v;
  int64_t batch_stride, token_stride, head_stride;   // elements
  const int32_t* start;        // first position per sequence
  const int32_t* count;        // tokens per sequence (NULL: T each)
  int32_t B, T, n_kv_heads;
  int32_t quads;               // position groups a sequence can touch
};

template <int CTRL>
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}

// The eight values of a lane as codes, and their block's scale byte (the same in the four lanes of a block).
template <bool F16>
__device__ __forceinline__ uint32_t encode8(const u32x4 x, uint32_t* scale) {
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) amax = max(amax, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
  amax = quad_max<0x4E>(quad_max<0xB1>(amax));
  const bool finite = amax < (F16 ? 0x7c00u : 0x7f80u);
  const uint32_t bits = __float_as_uint(lo16<F16>(amax));
  const int s = max(2, (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) >= 0x600000u ? 1 : 0));
  *scale = finite ? (uint32_t)s : 255u;
  const float f = __uint_as_float((uint32_t)s << 23);
  uint32_t codes = 0;
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];   // (a bit cast of a vector's element takes its first one)
  if constexpr (F16) {
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2_t, x0), f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2_t, x1), f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2_t, x2), f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2_t, x3), f, 3);
  } else {
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x0), f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x1), f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x2), f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x3), f, 3);
  }
  return finite ? codes : 0u;
}

// Eight codes of one block as 16-bit values (bf16: exact; fp16: one rounding where the value is none of fp16's).
template <bool F16>
__device__ __forceinline__ u32x4 decode8(uint32_t codes, float scale) {
  u32x4 r;
  if constexpr (F16) {
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    r[0] = f32_to_f16_rne(a.x) | ((uint32_t)f32_to_f16_rne(a.y) << 16);
    r[1] = f32_to_f16_rne(b.x) | ((uint32_t)f32_to_f16_rne(b.y) << 16);
    r[2] = f32_to_f16_rne(c.x) | ((uint32_t)f32_to_f16_rne(c.y) << 16);
    r[3] = f32_to_f16_rne(d.x) | ((uint32_t)f32_to_f16_rne(d.y) << 16);
  } else {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  }
  return r;
}

// The group of 16 lanes -> (sequence, KV head, positions 4 * quad .. + 3); false: nothing there.
struct StoreSpot {
  int b, kvh, pos0, start, end;
};
__device__ __forceinline__ bool store_spot(const Kv4StoreArgs& a, StoreSpot* s) {
  const int64_t gid = (int64_t)blockIdx.x * (kStoreThreads / 16) + (threadIdx.x >> 4);
  const int64_t row = gid / a.quads;
  if (row >= (int64_t)a.B * a.n_kv_heads) return false;
  s->b = (int)(row / a.n_kv_heads);
  s->kvh = (int)(row - (int64_t)s->b * a.n_kv_heads);
  s->start = a.start[s->b];
  const int n = a.count ? min(a.count[s->b], a.T) : a.T;
  if (s->start < 0 || n <= 0) return false;
  s->end = (int)min((int64_t)s->start + n, (int64_t)0x7fffffff);
  const int64_t pos0 = ((int64_t)(s->start >> 2) + (gid - row * a.quads)) * 4;
  s->pos0 = (int)pos0;
  return pos0 < s->end;
}

template <bool F16>
__global__ __launch_bounds__(kStoreThreads) void kv4_append_kernel(const Kv4StoreArgs a) {
  StoreSpot s;
  if (!store_spot(a, &s)) return;
  const int piece = threadIdx.x & 15;
  const int page = kv4_page(a.c, a.c.page_table + s.b * a.c.pt_stride, s.pos0);   // (four positions of a quad share their page)
  if (page < 0) return;
  const int slot = s.pos0 & ((1 << a.c.page_shift) - 1);
  const int64_t src = s.b * a.batch_stride + s.kvh * a.head_stride + piece * 8;
  u32x4 kx[4], vx[4];
  bool in[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    in[i] = s.pos0 + i >= s.start && s.pos0 + i < s.end;
    kx[i] = vx[i] = (u32x4){0u, 0u, 0u, 0u};
    if (in[i]) {
      const int64_t at = src + (int64_t)(s.pos0 + i - s.start) * a.token_stride;
      kx[i] = *reinterpret_cast<const u32x4*>(a.k + at);
      vx[i] = *reinterpret_cast<const u32x4*>(a.v + at);
    }
  }
  uint8_t* codes = a.c.codes + (int64_t)page * a.c.code_page16 * 16 + s.kvh * a.c.code_head_stride + (int64_t)slot * kKv4Row + piece * 4;
  uint8_t* scales = a.c.scales + (int64_t)page * a.c.scale_page16 * 16 + s.kvh * a.c.scale_head_stride + (int64_t)(slot >> 2) * kKv4Group + (piece & ~3);
  uint32_t ks = 0, vs = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t sk, sv;
    const uint32_t ck = encode8<F16>(kx[i], &sk), cv = encode8<F16>(vx[i], &sv);
    if (in[i]) {
      *reinterpret_cast<uint32_t*>(codes + i * kKv4Row) = ck;
      *reinterpret_cast<uint32_t*>(codes + i * kKv4Row + 64) = cv;
    }
    ks |= sk << (8 * i);
    vs |= sv << (8 * i);
  }
  if (piece & 3) return;                      // one lane of a block writes its scales
  if (in[0] && in[3]) {
    *reinterpret_cast<uint32_t*>(scales) = ks;
    *reinterpret_cast<uint32_t*>(scales + 16) = vs;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!in[i]) continue;
      scales[i] = (uint8_t)(ks >> (8 * i));
      scales[16 + i] = (uint8_t)(vs >> (8 * i));
    }
  }
}

template <bool F16>
__global__ __launch_bounds__(kStoreThreads) void kv4_read_kernel(const Kv4StoreArgs a) {
  StoreSpot s;
  if (!store_spot(a, &s)) return;
  const int piece = threadIdx.x & 15;
  const int page = kv4_page(a.c, a.c.page_table + s.b * a.c.pt_stride, s.pos0);
  const int slot = s.pos0 & ((1 << a.c.page_shift) - 1);
  uint32_t kc[4] = {0u, 0u, 0u, 0u}, vc[4] = {0u, 0u, 0u, 0u}, ks = 0, vs = 0;
  if (page >= 0) {                            // (tokens without a page come back as zeros)
    const uint8_t* codes = a.c.codes + (int64_t)page * a.c.code_page16 * 16 + s.kvh * a.c.code_head_stride + (int64_t)slot * kKv4Row + piece * 4;
    const uint8_t* scales = a.c.scales + (int64_t)page * a.c.scale_page16 * 16 + s.kvh * a.c.scale_head_stride + (int64_t)(slot >> 2) * kKv4Group + (piece & ~3);
    ks = *reinterpret_cast<const uint32_t*>(scales);
    vs = *reinterpret_cast<const uint32_t*>(scales + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kc[i] = *reinterpret_cast<const uint32_t*>(codes + i * kKv4Row);
      vc[i] = *reinterpret_cast<const uint32_t*>(codes + i * kKv4Row + 64);
    }
  }
  const int64_t dst = s.b * a.batch_stride + s.kvh * a.head_stride + piece * 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (s.pos0 + i < s.start || s.pos0 + i >= s.end) continue;
    const int64_t at = dst + (int64_t)(s.pos0 + i - s.start) * a.token_stride;
    __builtin_nontemporal_store(decode8<F16>(kc[i], kv4_scale(ks, i)), reinterpret_cast<u32x4*>(a.k + at));
    __builtin_nontemporal_store(decode8<F16>(vc[i], kv4_scale(vs, i)), reinterpret_cast<u32x4*>(a.v + at));
  }
}

int32_t check_kv4_cache(const char* who, const rtp_layer_desc* L, const rtp_kv4_cache* c, int64_t max_tokens, Kv4Cache* out) {
  if (!c) return fail(RTP_ERR_INVALID_ARG, "%s: cache descriptor is NULL", who);
  if (!c->codes || !c->scales || !c->page_table) return fail(RTP_ERR_INVALID_ARG, "%s: NULL codes/scales/page_table", who);
  const int32_t ps = c->page_size;
  if (ps < 16 || (ps & (ps - 1)) || ps > (1 << 20))
    return fail(RTP_ERR_INVALID_ARG, "%s: page_size must be a power of two in [16, 2^20]", who);
  if (c->n_pages <= 0 || c->pt_stride <= 0) return fail(RTP_ERR_INVALID_ARG, "%s: n_pages and pt_stride must be positive", who);
  if (((uintptr_t)c->codes & 15) || ((uintptr_t)c->scales & 15) || (c->code_page_stride & 15) || (c->code_head_stride & 15) ||
      (c->scale_page_stride & 15) || (c->scale_head_stride & 15))
    return fail(RTP_ERR_INVALID_ARG, "%s: codes, scales and their strides must be 16-byte aligned", who);
  if (!strides_apart(c->code_page_stride, c->n_pages, c->code_head_stride, L->n_kv_heads, (int64_t)ps * kKv4Row) ||
      !strides_apart(c->scale_page_stride, c->n_pages, c->scale_head_stride, L->n_kv_heads, (int64_t)ps / 4 * kKv4Group))
    return fail(RTP_ERR_INVALID_ARG, "%s: strides let pages or heads overlap", who);
  if (c->pt_stride < (max_tokens + ps - 1) / ps) return fail(RTP_ERR_INVALID_ARG, "%s: pt_stride must cover %lld tokens", who, (long long)max_tokens);
  const int64_t page16_most = ((int64_t)1 << 32) - 1;
  if (c->code_page_stride / 16 > page16_most || c->scale_page_stride / 16 > page16_most)
    return fail(RTP_ERR_UNSUPPORTED, "%s: page strides of 2^36 bytes and more", who);
  int sh = 4;
  while ((1 << sh) < ps) ++sh;
  *out = Kv4Cache{(uint8_t*)c->codes, (uint8_t*)c->scales, c->code_head_stride, c->scale_head_stride, (uint32_t)(c->code_page_stride / 16),
                  (uint32_t)(c->scale_page_stride / 16), c->page_table, c->pt_stride, sh, c->n_pages};
  return RTP_OK;
}

// Rows of 128 at the multiples of three strides, nested in any order, do not overlap.
static bool rows_apart(int64_t s0, int64_t n0, int64_t s1, int64_t n1, int64_t s2, int64_t n2) {
  int64_t s[3] = {s0, s1, s2}, n[3] = {n0, n1, n2}, span = kHeadDim;
  for (int round = 0; round < 3; ++round) {    // the smallest stride that is left has to pass what lies inside it
    int i = -1;
    for (int k = 0; k < 3; ++k)
      if (n[k] > 1 && (i < 0 || s[k] < s[i])) i = k;
    if (i < 0) return true;
    if (s[i] < span) return false;
    if (s[i] > (((int64_t)1 << 62) - span) / (n[i] - 1)) return (n[0] > 1) + (n[1] > 1) + (n[2] > 1) == 1;
    span += s[i] * (n[i] - 1);
    n[i] = 1;
  }
  return true;
}

static int32_t store_args(const char* who, const rtp_layer_desc* layer, const rtp_kv4_cache* cache, const void* k, const void* v,
                          int64_t batch_stride, int64_t token_stride, int64_t head_stride, const int32_t* start,
                          const int32_t* count, int32_t B, int32_t T, Kv4StoreArgs* a, unsigned* grid) {
  int32_t rc = check_layer(layer, who);
  if (rc != RTP_OK) return rc;
  rc = check_kv4_cache(who, layer, cache, 0, &a->c);
  if (rc != RTP_OK) return rc;
  if (!k || !v || !start) return fail(RTP_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  if (((uintptr_t)k & 15) || ((uintptr_t)v & 15)) return fail(RTP_ERR_INVALID_ARG, "%s: K and V must be 16-byte aligned", who);
  if (B <= 0 || T <= 0) return fail(RTP_ERR_INVALID_ARG, "%s: B and T must be positive", who);
  if ((batch_stride & 7) || (token_stride & 7) || (head_stride & 7) || batch_stride < 0 || token_stride < 0 || head_stride < 0)
    return fail(RTP_ERR_INVALID_ARG, "%s: strides must be non-negative multiples of 8 elements", who);
  a->k = (uint16_t*)k;
  a->v = (uint16_t*)v;
  a->batch_stride = batch_stride;
  a->token_stride = token_stride;
  a->head_stride = head_stride;
  a->start = start;
  a->count = count;
  a->B = B;
  a->T = T;
  a->n_kv_heads = layer->n_kv_heads;
  a->quads = (int32_t)(((int64_t)T + 6) / 4);          // T consecutive positions touch at most this many groups of four
  const int64_t groups = (int64_t)B * layer->n_kv_heads * a->quads, blocks = (groups + kStoreThreads / 16 - 1) / (kStoreThreads / 16);
  if (blocks > 0x7fffffff / kStoreThreads) return fail(RTP_ERR_UNSUPPORTED, "%s: B * T is too large for one call", who);
  *grid = (unsigned)blocks;
  return RTP_OK;
}

}  // namespace rtp

using namespace rtp;

extern "C" int32_t rtp_kv4_append(const rtp_layer_desc* layer, const rtp_kv4_cache* cache, const void* k, const void* v,
                                  int64_t batch_stride, int64_t token_stride, int64_t head_stride, const int32_t* start,
                                  const int32_t* count, int32_t B, int32_t T, void* stream) {
  const char* who = "rtp_kv4_append";
  Kv4StoreArgs a;
  unsigned grid = 0;
  const int32_t rc = store_args(who, layer, cache, k, v, batch_stride, token_stride, head_stride, start, count, B, T, &a, &grid);
  if (rc != RTP_OK) return rc;
  clear_error();
  if (layer->kv_dtype == RTP_DTYPE_FP16) RTP_LAUNCH(kv4_append_kernel<true>, dim3(grid), dim3(kStoreThreads), 0, (hipStream_t)stream, a);
  else RTP_LAUNCH(kv4_append_kernel<false>, dim3(grid), dim3(kStoreThreads), 0, (hipStream_t)stream, a);
  return check_launch(who);
}

extern "C" int32_t rtp_kv4_read(const rtp_layer_desc* layer, const rtp_kv4_cache* cache, const int32_t* start, const int32_t* count,
                                int32_t B, int32_t T, void* k, void* v, int64_t batch_stride, int64_t token_stride,
                                int64_t head_stride, void* stream) {
  const char* who = "rtp_kv4_read";
  Kv4StoreArgs a;
  unsigned grid = 0;
  const int32_t rc = store_args(who, layer, cache, k, v, batch_stride, token_stride, head_stride, start, count, B, T, &a, &grid);
  if (rc != RTP_OK) return rc;
  if (!rows_apart(batch_stride, B, token_stride, T, head_stride, layer->n_kv_heads))
    return fail(RTP_ERR_INVALID_ARG, "%s: strides let the rows that are written overlap", who);
  clear_error();
  if (layer->kv_dtype == RTP_DTYPE_FP16) RTP_LAUNCH(kv4_read_kernel<true>, dim3(grid), dim3(kStoreThreads), 0, (hipStream_t)stream, a);
  else RTP_LAUNCH(kv4_read_kernel<false>, dim3(grid), dim3(kStoreThreads), 0, (hipStream_t)stream, a);
  return check_launch(who);
}
