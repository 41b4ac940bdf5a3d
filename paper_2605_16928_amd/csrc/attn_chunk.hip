// Causal attention of a batch of new tokens over a cache in pages: rtp_dense_attn_chunk (every token) and rtp_local_attn_chunk (sink +
// window), from 16-bit pages or from the 4-bit cache.
//
//   out_m = sum_n p_n v_n / sum_n p_n,   p_n = 2^(c <q_m, k_n> - r_m),   c = softmax scale * log2(e)
// over the tokens n that position m sees; r_m is a reference that cancels.
//
// Work: a KV head's served query heads share its rows, so a query tile is 256 (token, head) pairs of one KV head -- 64 tokens of a group of
// four, one token's eight heads where there is one -- and eight waves of 32 rows share every staged tile of 64 keys.  Tiles and the ranges of
// their keys are numbered by chunk_plan.h from the lengths on the device: every workgroup finds its own, the host sees bounds only.  Where a
// tile's keys are cut into ranges, the workgroups leave (maximum, sums, unnormalised outputs) per row to a merge launch.
//
// A wave computes the transposed scores S^T = K Q^T of 32 keys (v_mfma_f32_32x32x16): lane (g, r) then holds 16 keys of ONE row, the softmax is
// per lane, and the probabilities, rounded to 16 bits, are in place as the B operand of O^T = V^T P^T.
#include "chunk_kernels.h"

#include <algorithm>

namespace rtp {

// B > 64: the same by one workgroup, once for the launches behind it.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void chunk_plan_kernel(const ChunkArgs a) {
  fetch_arguments<ChunkArgs>();
  constexpr int NW = kPlanThreads / 64;
  __shared__ ChunkSums sh_sums[NW][64];
  __shared__ float sh_work[NW];
  __shared__ int sh_longest[NW], sh_candidate, sh_sum[3][NW];
  const ChunkShape& s = a.shape;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int longest = 1;
  for (int b0 = wave * 64; b0 < s.B; b0 += kPlanThreads) {
    const ChunkLane mine = chunk_lane(a, b0 + lane);
    longest = max(longest, wave_max_ge_m1(mine.n > 0 ? mine.key_tiles : 1));
  }
  if (lane == 0) sh_longest[wave] = longest;
  __syncthreads();
  for (int w = 0; w < NW; ++w) longest = max(longest, sh_longest[w]);
  const uint32_t magic = chunk_magic(longest);
  ChunkSums sums = {};
  float work = 0.f;
  for (int b0 = wave * 64; b0 < s.B; b0 += kPlanThreads) {
    const ChunkLane mine = chunk_lane(a, b0 + lane);
    chunk_add_up(s, mine, min(64, s.B - b0), longest, magic, &sums);
    work += (float)mine.tiles * (float)mine.key_tiles;
  }
  work = wave_sum_f32(work);
  sh_sums[wave][lane] = sums;
  if (lane == 0) sh_work[wave] = work;
  __syncthreads();
  if (wave == 0) {
    sums = ChunkSums{};
    work = 0.f;
    for (int w = 0; w < NW; ++w) {
      sums.units += sh_sums[w][lane].units;
      sums.cut_units += sh_sums[w][lane].cut_units;
      sums.cut_rows += sh_sums[w][lane].cut_rows;
      sums.most = fmaxf(sums.most, sh_sums[w][lane].most);
      work += sh_work[w];
    }
    const int best = s.cap > 0 ? chunk_best(s, longest, work, sums) : 1;
    if (lane == 0) {
      sh_candidate = best;
      a.plan[kPlanCandidate] = best;
      a.plan[kPlanLongest] = longest;
    }
  }
  __syncthreads();
  int32_t* const lists[3] = {a.plan + kPlanHead, a.plan + kPlanHead + s.B + 1, a.plan + kPlanHead + 2 * (s.B + 1)};
  int before[3] = {0, 0, 0};
  for (int b0 = 0; b0 < s.B; b0 += kPlanThreads) {
    const ChunkLane mine = chunk_lane(a, b0 + tid);
    const int S = chunk_splits(mine.key_tiles, longest, sh_candidate, magic), own = mine.tiles * S;
    const int add[3] = {own, S > 1 ? own : 0, mine.tiles};
    int last[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      last[k] = wave_incl_scan(add[k]);
      if (lane == 63) sh_sum[k][wave] = last[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      int first = before[k], all = 0;
      for (int w = 0; w < NW; ++w) {
        if (w < wave) first += sh_sum[k][w];
        all += sh_sum[k][w];
      }
      if (b0 + tid < s.B) lists[k][b0 + tid] = first + last[k] - add[k];
      before[k] += all;
    }
    __syncthreads();
  }
  if (tid < 3) lists[tid][s.B] = before[tid];
}

RTP_CHUNK_KERNELS(chunk_attn_kernel, chunk_again_kernel, chunk_narrow_kernel, false)

// rows: the most that a tile can have; few: no more units than compute units.
static void launch_chunk_16(const ChunkArgs& a, unsigned grid, int rows, bool few, hipStream_t stream) {
  const bool narrow = rows <= kCkNarrowRows;
  RTP_CHUNK_LAUNCH(chunk_attn_kernel, chunk_again_kernel, chunk_narrow_kernel, false, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kernel, chunk_again_kernel, chunk_narrow_kernel, true, false)
  RTP_CHUNK_LAUNCH(chunk_attn_kernel, chunk_again_kernel, chunk_narrow_kernel, false, true)
  RTP_CHUNK_LAUNCH(chunk_attn_kernel, chunk_again_kernel, chunk_narrow_kernel, true, true)
}
// attn_chunk_kv4.hip
void launch_chunk_kv4(const ChunkArgs& a, unsigned grid, int rows, bool few, hipStream_t stream);

// Merges the ranges of the tiles that were cut (blockIdx.x: tile; blockIdx.y takes its rows in turn): SLICES groups of 32 lanes per row take the ranges
// in turn, four at a time, a lane 4 of the 128 dims.
template <int SLICES>
__global__ __launch_bounds__(256) void chunk_merge_kernel(const ChunkMerge* merge, const float* part, int part_rows, float scale, float scale_log2,
                                                          int group, int n_q_heads, int f16, uint16_t* out, float* lse) {
  __shared__ float sh_h[8][3];
  __shared__ __attribute__((aligned(16))) float sh_acc[8][kHeadDim];
  constexpr int kRows = 8 / SLICES;
  const int tid = threadIdx.x, d4 = tid & 31, grp = tid >> 5, slice = grp % SLICES;
  const float ninf = -__builtin_huge_valf();
  const ChunkMerge t = merge[blockIdx.x];
  const int rows = min(t.rows, part_rows);
  const int64_t step = (int64_t)t.step * part_rows * kCkPart;
  for (int row0 = blockIdx.y * kRows; row0 < rows; row0 += gridDim.y * kRows) {
    const int row = row0 + grp / SLICES;
    float M = ninf, L = 0.f, F = 0.f;
    float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* p = part + ((int64_t)t.part * part_rows + row) * kCkPart;
    for (int s0 = slice; row < rows && s0 < t.splits; s0 += 4 * SLICES) {
      float4 h[4], v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = s0 + k * SLICES;
        h[k] = make_float4(ninf, 0.f, 0.f, 0.f);
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s < t.splits) {
          h[k] = *reinterpret_cast<const float4*>(p + s * step);
          v[k] = *reinterpret_cast<const float4*>(p + s * step + 4 + d4 * 4);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float Mn = fmaxf(M, h[k].x);
        if (Mn == ninf) continue;
        const float c0 = fast_exp2((M - Mn) * scale_log2), c1 = fast_exp2((h[k].x - Mn) * scale_log2);
        L = L * c0 + h[k].y * c1;
        F = F * c0 + h[k].z * c1;
        A.x = A.x * c0 + v[k].x * c1; A.y = A.y * c0 + v[k].y * c1;
        A.z = A.z * c0 + v[k].z * c1; A.w = A.w * c0 + v[k].w * c1;
        M = Mn;
      }
    }
    if constexpr (SLICES > 1) {
      if (d4 == 0) { sh_h[grp][0] = M; sh_h[grp][1] = L; sh_h[grp][2] = F; }
      *reinterpret_cast<float4*>(&sh_acc[grp][d4 * 4]) = A;
      __syncthreads();
      float Mt = ninf, Lt = 0.f, Ft = 0.f;
      float4 At = make_float4(0.f, 0.f, 0.f, 0.f);
      if (slice == 0) {
#pragma unroll
        for (int k = 0; k < SLICES; ++k) Mt = fmaxf(Mt, sh_h[grp + k][0]);
        if (Mt != ninf) {
#pragma unroll
          for (int k = 0; k < SLICES; ++k) {
            const float cw = fast_exp2((sh_h[grp + k][0] - Mt) * scale_log2);
            const float4 v = *reinterpret_cast<const float4*>(&sh_acc[grp + k][d4 * 4]);
            Lt += sh_h[grp + k][1] * cw;
            Ft += sh_h[grp + k][2] * cw;
            At.x += v.x * cw; At.y += v.y * cw; At.z += v.z * cw; At.w += v.w * cw;
          }
        }
      }
      __syncthreads();
      M = Mt;
      L = Lt;
      F = Ft;
      A = At;
    }
    if (slice != 0 || row >= rows) continue;
    const int rt = (row * chunk_row_factor(t.heads)) >> 16, k = row - rt * t.heads;
    const int64_t o = (int64_t)(t.q0 + rt) * n_q_heads + t.kvh * group + (t.heads == group ? k : chunk_nth((uint32_t)t.members, k));
    const bool none = L == 0.f;
    const float inv = none ? 0.f : 1.f / L;
    const u32x2 w = f16 ? (u32x2){pack16<true>(A.x * inv, A.y * inv), pack16<true>(A.z * inv, A.w * inv)}
                        : (u32x2){pack16<false>(A.x * inv, A.y * inv), pack16<false>(A.z * inv, A.w * inv)};
    *reinterpret_cast<u32x2*>(out + o * kHeadDim + d4 * 4) = none ? (u32x2){0u, 0u} : w;
    if (lse && d4 == 0) lse[o] = none ? ninf : M * scale + logf(F);
  }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------------
namespace {
int compute_units() {
  static const int n = [] {
    int dev = 0, cu = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cu <= 0) cu = 256;
    (void)hipGetLastError();
    return cu;
  }();
  return n;
}

enum { kServeAll = 0, kServeRet = 1, kServeLocal = 2 };

// The heads that a call serves, and which tokens they see.
void serve(const rtp_layer_desc* L, const HeadTable& ht, int which, ChunkShape* s) {
  s->group = L->n_q_heads / L->n_kv_heads;
  s->n_kv = L->n_kv_heads;
  for (int h = 0; h < L->n_q_heads; ++h)
    if (which == kServeAll || (ht.is_ret[h] != 0) == (which == kServeRet)) {
      s->served[h >> 5] |= 1u << (h & 31);
      ++s->n_served;
    }
  for (int kv = 0; kv < s->n_kv; ++kv)
    if (const int n = chunk_bits(chunk_members(*s, kv))) {
      ++s->count[n - 1];
      ++s->kv_served;
      s->widest = std::max(s->widest, n);
    }
  s->local = which == kServeLocal;
  s->sink = std::min(L->sink, kMostContext);           // (as good as any larger: no position is behind it, and sums of two stay in 32 bits)
  s->window = std::min(L->window, kMostContext);
}

// Contexts up to here are not cut: a workgroup is through with them by the time that the results of ranges would be merged.  One call, whole and cut:
// one token of 32 heads over 8 KV heads, 500 keys 10.9 and 11.2 us, 1000 keys 13.9 and 11.2; 512 tokens, 500 keys 25.9 and 27.6, 2000 keys 62 and 45.
constexpr int kUncutKeys = 512;

// Tiles of 32 rows, whose waves need not wait for each other and which need no second launch for what has to be taken again, are taken in two cases.
// Up to this many rows of a KV head to a sequence: two that read the same keys are neighbours on a die and share its L2.  8 contexts of 8000, 64 over
// 8 heads, 8 new tokens (64 rows) 53 us and 61 as one tile, 12 tokens 90 and 64; 30000 in 4 bits, 8 tokens 143 and 166, 16 tokens 260 and 185.
constexpr int kFineRows = 64;
// And where they all have a place at once, two to a compute unit, and read no more than so many keys together, as wide tiles would leave most of
// the compute units without work.  32 over 8 heads, fine and wide: 60 tokens over as many 9 us and 15; 4 x 60 (256 tiles of 32 rows) over 500 keys 13
// and 25, over 4000 (2^20) 45 and 46, over 8000 73 and 59; 16 x 60 (1024) over 500 32 and 27; 64 over 8 heads, 4 x 60 (480) over 2000 40 and 45, over
// 4000 66 and 58; 4 x 20 (160) over 4000 40 and 39.
constexpr int64_t kFineKeys = 3 << 18;

struct ChunkSizes {
  int64_t tiles;               // query tiles that the bounds allow
  int64_t cap;                 // units of cut tiles
  int32_t part_rows;
  bool narrow;                 // no tile has more than 32 rows
  int32_t fine;
  int64_t run;                 // units in a row on one die
  size_t plan_bytes, again_bytes, merge_bytes, part_bytes;
  size_t total() const { return plan_bytes + again_bytes + merge_bytes + part_bytes; }
};
// Query tiles that the bounds allow, of so many rows: a sequence of n tokens has ceil(n / tok), at most n of them, at most one more than its share.
int64_t chunk_most_tiles(const ChunkShape& s, int32_t B, int64_t total_q, int64_t max_q, int rows) {
  int64_t tiles = 0;
  for (int k = 0; k < 8; ++k) {
    const int64_t tok = rows / (k + 1), per_seq = (max_q + tok - 1) / tok;
    tiles += s.count[k] * std::min(std::min(total_q, total_q / tok + B), per_seq * B);
  }
  return tiles;
}
int64_t chunk_most_keys(const ChunkShape& s, int64_t max_ctx) {       // that a tile reads
  return s.local ? std::min<int64_t>(max_ctx, (int64_t)s.sink + s.window + 64) : max_ctx;
}
bool chunk_fine(const ChunkShape& s, int32_t B, int64_t total_q, int64_t max_q, int64_t max_ctx) {
  max_q = std::max<int64_t>(1, std::min(max_q, total_q));
  if (max_q * std::max(s.widest, 1) <= kFineRows) return true;
  const int64_t tiles = chunk_most_tiles(s, B, total_q, max_q, kCkNarrowRows);
  return tiles <= 2 * (int64_t)compute_units() && tiles * chunk_most_keys(s, max_ctx) <= kFineKeys;
}
// most: there are no more tiles.
ChunkSizes chunk_sizes(const ChunkShape& s, int32_t B, int64_t total_q, int64_t max_q, int64_t max_ctx, bool fine, int64_t most) {
  ChunkSizes z = {};
  max_q = std::max<int64_t>(1, std::min(max_q, total_q));
  const int widest = std::max(s.widest, 1);
  z.narrow = fine;
  z.fine = z.narrow ? 3 : 0;
  const int rows = kChunkRows >> z.fine;
  z.tiles = std::min(chunk_most_tiles(s, B, total_q, max_q, rows), most);
  // ranges of two key tiles and more, at most four per compute unit
  const int64_t keys = chunk_most_keys(s, max_ctx);
  const int64_t ranges = keys <= kUncutKeys ? 1 : std::min<int64_t>((keys + 2 * kCkK - 1) / (2 * kCkK), 289);
  z.cap = ranges > 1 ? std::min<int64_t>(z.tiles * ranges, 4 * (int64_t)compute_units()) : 0;
  z.part_rows = (int32_t)std::min<int64_t>(rows, max_q * widest);
  // so many runs that each die has two of a long sequence at least, one of long and one of short units; tiles of 32 rows are bound by the bytes
  // of their keys, and those of a sequence stay together.  (Whole heads one after the other gave all long tiles to the same dies: a prompt of 8192
  // tokens, 32 over 8 heads, 504 us and 712; 16384 behind 16384 5.5 and 7.0 ms; 16384 of 8 over 2 heads 486 and 779, without the turn 613.)
  int64_t each = 0;
  for (int k = 0; k < 8; ++k) each += s.count[k] * ((max_q + rows / (k + 1) - 1) / (rows / (k + 1)));
  for (z.run = z.fine && max_q * widest > rows ? 2 : 1; z.run < 32 && z.run * 2 * 16 <= each;) z.run *= 2;
  z.again_bytes = z.narrow ? 0 : align_up((size_t)(z.tiles + z.cap + 8 * 32) * sizeof(int32_t), 256);
  z.plan_bytes = B > 64 ? align_up((size_t)(kPlanHead + 3 * ((int64_t)B + 1)) * sizeof(int32_t), 256) : 0;
  z.merge_bytes = z.cap > 0 ? align_up((size_t)z.tiles * sizeof(ChunkMerge), 256) : 0;
  z.part_bytes = align_up((size_t)z.cap * z.part_rows * kCkPart * sizeof(float), 256);
  return z;
}

// What a call needs, and every one with smaller bounds: finer tiles, for either reason, among them.
size_t chunk_bytes(const ChunkShape& s, int32_t B, int64_t total_q, int64_t max_q, int64_t max_ctx) {
  const int64_t any = INT64_MAX;
  size_t bytes = std::max<size_t>(256, chunk_sizes(s, B, total_q, max_q, max_ctx, chunk_fine(s, B, total_q, max_q, max_ctx), any).total());
  bytes = std::max(bytes, chunk_sizes(s, B, total_q, std::min<int64_t>(max_q, kFineRows / std::max(s.widest, 1)), max_ctx, true, any).total());
  return std::max(bytes, chunk_sizes(s, B, total_q, max_q, max_ctx, true, 2 * (int64_t)compute_units()).total());
}

size_t chunk_workspace(const rtp_layer_desc* layer, int which, int32_t B, int32_t total_q, int32_t max_q, int64_t max_ctx) {
  HeadTable ht;
  if (fill_head_table(layer, &ht, "workspace") != RTP_OK || B <= 0 || B > kMaxSeqs || total_q <= 0 || total_q > (1 << 24) || max_q <= 0 ||
      max_ctx <= 0 || max_ctx > ((int64_t)1 << 30))
    return 256;
  ChunkShape s = {};
  serve(layer, ht, which, &s);
  return chunk_bytes(s, B, total_q, max_q, max_ctx);
}

int32_t chunk_call(const char* who, int which, const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv_cache* c16,
                   const rtp_kv4_cache* c4, bool kv4, const rtp_chunk* chunk, void* out, float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  HeadTable ht;
  int32_t rc = fill_head_table(layer, &ht, who);
  if (rc != RTP_OK) return rc;
  rc = check_chunk(who, chunk);
  if (rc != RTP_OK) return rc;
  ChunkArgs a = {};
  rc = kv4 ? check_kv4_cache(who, layer, c4, chunk->max_ctx, &a.c4) : check_kv16_cache(who, layer, c16, chunk->max_ctx, &a.c16);
  if (rc != RTP_OK) return rc;
  if (!q || !out) return fail(RTP_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  if (((uintptr_t)q & 15) || ((uintptr_t)out & 15) || ((uintptr_t)lse & 3))
    return fail(RTP_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned, lse 4-byte aligned", who);
  const int64_t width = (int64_t)layer->n_q_heads * kHeadDim;
  if ((q_stride & 7) || q_stride < width || q_stride > ((int64_t)1 << 40))
    return fail(RTP_ERR_INVALID_ARG, "%s: q_stride must be a multiple of 8 elements that holds a token's rows", who);
  if (chunk->total_q > 0 && rows_overlap(q, q_stride, width, out, width, width, chunk->total_q))
    return fail(RTP_ERR_INVALID_ARG, "%s: out overlaps q", who);
  serve(layer, ht, which, &a.shape);
  if (a.shape.n_served == 0 || chunk->total_q == 0) {
    clear_error();
    return RTP_OK;
  }
  const bool fine = chunk_fine(a.shape, chunk->B, chunk->total_q, chunk->max_q, chunk->max_ctx);
  const ChunkSizes z = chunk_sizes(a.shape, chunk->B, chunk->total_q, chunk->max_q, chunk->max_ctx, fine, INT64_MAX);
  const size_t bytes = chunk_bytes(a.shape, chunk->B, chunk->total_q, chunk->max_q, chunk->max_ctx);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < bytes)
    return fail(RTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, 256-byte aligned, needed", who, bytes);
  const int64_t grid = (z.tiles + z.cap + 8 * z.run - 1) / (8 * z.run) * (8 * z.run);
  if (grid > 0x7fffffff / kCkThreads) return fail(RTP_ERR_UNSUPPORTED, "%s: too many query tiles for one call", who);
  clear_error();
  a.shape.B = chunk->B;
  a.shape.total_q = chunk->total_q;
  a.shape.max_q = chunk->max_q;
  a.shape.fine = z.fine;
  while ((1 << a.shape.run_shift) < z.run) ++a.shape.run_shift;
  for (int h = 1; h <= 8; ++h) a.shape.per_tile[h - 1] = chunk_inverse(chunk_tokens(z.fine, h));
  for (int h = 8; h >= 1; --h)
    if (a.shape.count[h - 1]) a.shape.per_most = a.shape.per_tile[h - 1];
  a.shape.cap = (int32_t)z.cap;
  a.shape.places = (float)(compute_units() * (kv4 && z.part_rows <= kCkSlimRows ? 3 : z.narrow ? 2 : 1));
  a.q = (const uint16_t*)q;
  a.q_stride = q_stride;
  a.q_offset = chunk->q_offset;
  a.ctx_len = chunk->ctx_len;
  a.n_q_heads = layer->n_q_heads;
  a.scale = softmax_scale_of(layer);
  a.scale_log2 = a.scale * 1.4426950408889634f;
  a.out = (uint16_t*)out;
  a.lse = lse;
  a.plan = (int32_t*)ws;
  a.again = (int32_t*)((uint8_t*)ws + z.plan_bytes);
  a.merge = z.cap > 0 ? (ChunkMerge*)((uint8_t*)ws + z.plan_bytes + z.again_bytes) : nullptr;
  a.n_merge = (int32_t)z.tiles;
  a.part = (float*)((uint8_t*)ws + z.plan_bytes + z.again_bytes + z.merge_bytes);
  a.part_rows = z.part_rows;
  a.f16 = layer->kv_dtype == RTP_DTYPE_FP16;
  if (chunk->B > 64) RTP_LAUNCH(chunk_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
  const bool few = z.tiles + z.cap <= compute_units();
  if (kv4) launch_chunk_kv4(a, (unsigned)grid, z.part_rows, few, stream);
  else launch_chunk_16(a, (unsigned)grid, z.part_rows, few, stream);
  if (z.cap > 0) {
    // eight slices of the ranges where there are few rows (and many ranges, then), none where there are many; about 4096 workgroups at the most
    const int slices = (int64_t)chunk->total_q * a.shape.n_served <= 2048 ? 8 : z.part_rows <= 64 ? 2 : 1;
    const int64_t each = (z.part_rows * slices + 7) / 8, rows = std::max<int64_t>(1, std::min<int64_t>(each, 4096 / z.tiles));
    const dim3 grid((unsigned)z.tiles, (unsigned)rows), block(256);
#define RTP_CHUNK_MERGE(SLICES)                                                                                                      \
  RTP_LAUNCH(chunk_merge_kernel<SLICES>, grid, block, 0, stream, a.merge, a.part, a.part_rows, a.scale, a.scale_log2, a.shape.group, \
             a.n_q_heads, a.f16, a.out, a.lse)
    if (slices == 8) RTP_CHUNK_MERGE(8);
    else if (slices == 2) RTP_CHUNK_MERGE(2);
    else RTP_CHUNK_MERGE(1);
#undef RTP_CHUNK_MERGE
  }
  return check_launch(who);
}
}  // namespace

}  // namespace rtp

using namespace rtp;

extern "C" size_t rtp_dense_attn_chunk_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int32_t total_q, int32_t max_q, int64_t max_ctx,
                                                       int32_t heads) {
  return chunk_workspace(layer, heads == RTP_HEADS_RETRIEVAL ? kServeRet : kServeAll, B, total_q, max_q, max_ctx);
}
extern "C" size_t rtp_local_attn_chunk_workspace_bytes(const rtp_layer_desc* layer, int32_t B, int32_t total_q, int32_t max_q, int64_t max_ctx) {
  return chunk_workspace(layer, kServeLocal, B, total_q, max_q, max_ctx);
}

static int32_t dense_which(const char* who, int32_t heads, int* which) {
  if (heads != RTP_HEADS_ALL && heads != RTP_HEADS_RETRIEVAL)
    return fail(RTP_ERR_INVALID_ARG, "%s: heads must be RTP_HEADS_ALL or RTP_HEADS_RETRIEVAL", who);
  *which = heads == RTP_HEADS_ALL ? kServeAll : kServeRet;
  return RTP_OK;
}

extern "C" int32_t rtp_dense_attn_chunk(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv_cache* cache,
                                        const rtp_chunk* chunk, int32_t heads, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  int which = 0;
  const int32_t rc = dense_which("rtp_dense_attn_chunk", heads, &which);
  return rc != RTP_OK ? rc : chunk_call("rtp_dense_attn_chunk", which, layer, q, q_stride, cache, nullptr, false, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_dense_attn_chunk_kv4(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv4_cache* cache,
                                            const rtp_chunk* chunk, int32_t heads, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  int which = 0;
  const int32_t rc = dense_which("rtp_dense_attn_chunk_kv4", heads, &which);
  return rc != RTP_OK ? rc : chunk_call("rtp_dense_attn_chunk_kv4", which, layer, q, q_stride, nullptr, cache, true, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_local_attn_chunk(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv_cache* cache,
                                        const rtp_chunk* chunk, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return chunk_call("rtp_local_attn_chunk", kServeLocal, layer, q, q_stride, cache, nullptr, false, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int32_t rtp_local_attn_chunk_kv4(const rtp_layer_desc* layer, const void* q, int64_t q_stride, const rtp_kv4_cache* cache,
                                            const rtp_chunk* chunk, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return chunk_call("rtp_local_attn_chunk_kv4", kServeLocal, layer, q, q_stride, nullptr, cache, true, chunk, out, lse, ws, ws_bytes, (hipStream_t)stream);
}
