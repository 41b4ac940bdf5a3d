// Pages of a cache: handing them out, sharing them between sequences, releasing and compacting them, and copying their bytes.  The
// bookkeeping is two device arrays of the caller's -- the page table and a reference count per pool page; a page is free when its count
// is 0 -- so a step needs no host round trip to grow a batch, and it is deterministic: fresh pages are the lowest free ones, in the order
// of the requests.  The bytes are moved by a call of their own (rtp_kv_pages_copy), which takes the page pairs that the bookkeeping
// left on the device and any list of pools: one table serves every layer.
//
// Bound: the counts (4 bytes a page) and the table entries concerned, i.e. the launch's latency, and the bytes of the copied pages.
// Ranks of free or used pages come from bit masks of 64 pages, a workgroup's word per thread: 65536 pages are one workgroup (one launch,
// 256 KB of counts), larger pools leave masks and counts per workgroup in the workspace for a second launch.
// Measured (us; an empty launch is 3): release of 64 rows 3.9, fork of 64 4.0, growth of 64 sequences with 64 copies 8.0 -- a chain: lengths,
// table, counts, two prefix sums, entries --, moves of 4096 pages 5.0, the table rewritten 4.1, 983 pages of 256 KB copied 93, 5.5 TB/s.
#include "common.h"

namespace rtp {

constexpr int kPgThreads = 1024;
constexpr int kPgChunk = kPgThreads * 64;       // pages per workgroup
constexpr int kPgMaxSeqs = 4096;                // requests of one extend call (their prefix sums are in LDS)
constexpr int kPgMaxPages = 1 << 26;
constexpr int kPgPools = 32;                    // pools per copy launch
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct PageMap {
  int32_t* table;
  int64_t pt_stride;
  int32_t* refs;
  int32_t n_seqs, page_shift, n_pages, n_chunks;
};

// Workspace of a pool of several chunks: masks [n_pages / 64], masks' prefixes inside their chunk, counts per chunk, request prefixes.
struct PageWork {
  uint64_t* mask;
  int32_t* before;       // set bits of the chunk in front of a mask
  int32_t* count;        // set bits of a chunk
  int32_t* need;         // [n + 1] exclusive prefix of the requests' pages
};

struct ExtendArgs {
  PageMap m;
  PageWork w;
  const int32_t* seq;
  const int32_t* old_len;
  const int32_t* new_len;
  int32_t n;
  int32_t* copy_src;
  int32_t* copy_dst;
  int32_t* status;
};

__device__ __forceinline__ bool in_pool(const PageMap& m, int page) { return (uint32_t)page < (uint32_t)m.n_pages; }

// Exclusive prefix sum over a workgroup of kPgThreads threads (T: int, or uint64_t where sums may pass 31 bits); *total gets the sum.
// sh: one word per wave.
template <typename T>
__device__ __forceinline__ T pg_scan(T v, uint64_t* sh, T* total) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const T incl = wave_incl_scan(v);
  __syncthreads();
  if (lane == 63) sh[wave] = (uint64_t)incl;
  __syncthreads();
  T off = 0, tot = 0;
  for (int i = 0; i < kPgThreads / 64; ++i) {
    if (i < wave) off += (T)sh[i];
    tot += (T)sh[i];
  }
  *total = tot;
  return off + incl - v;
}

// A chunk's masks in LDS (bit i of word w = page 64 w + i of the chunk is free, or in use where FREE is false) and, for every word, the
// set bits in front of it; *total: all of them.
struct ChunkMasks {
  uint64_t mask[kPgThreads];
  int32_t before[kPgThreads];
};
constexpr int kPgWaves = kPgThreads / 64, kPgAhead = 16;
// Counts of the pages of rounds r0 .. r0 + kPgAhead - 1 (round r of a wave: word r * kPgWaves + wave, a page per lane); what is behind the
// pool counts as neither free nor in use.
template <bool FREE>
__device__ __forceinline__ void pg_counts(const PageMap& m, int chunk, int r0, int (&v)[kPgAhead]) {
  const int64_t first = (int64_t)chunk * kPgChunk + (r0 * kPgWaves + (threadIdx.x >> 6)) * 64 + (threadIdx.x & 63);
#pragma unroll
  for (int r = 0; r < kPgAhead; ++r) {
    const int64_t p = first + r * kPgWaves * 64;
    v[r] = p < m.n_pages ? m.refs[p] : (FREE ? 1 : 0);
  }
}
template <bool FREE>
__device__ __forceinline__ void pg_masks(const PageMap& m, int chunk, int (&v)[kPgAhead], ChunkMasks& c, uint64_t* sh, int* total) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  c.mask[threadIdx.x] = 0;
  __syncthreads();
  for (int r0 = 0;;) {
#pragma unroll
    for (int r = 0; r < kPgAhead; ++r) {
      const uint64_t bits = __ballot(FREE ? v[r] <= 0 : v[r] > 0);
      if (lane == 0) c.mask[(r0 + r) * kPgWaves + wave] = bits;
    }
    r0 += kPgAhead;
    if (r0 >= 64 || (int64_t)chunk * kPgChunk + r0 * kPgWaves * 64 >= m.n_pages) break;
    pg_counts<FREE>(m, chunk, r0, v);
  }
  __syncthreads();
  c.before[threadIdx.x] = pg_scan<int>(__popcll(c.mask[threadIdx.x]), sh, total);
  __syncthreads();
}

// Pages that request i takes: one to copy its shared last page to, then what the new length adds.  lacks: entries that the table row has
// no room for.  first: 2 * the first entry of the table that takes one, + 1 if that is the shared page's.
struct Request {
  int pages, lacks;
  int64_t first;
};
__device__ __forceinline__ Request pg_request(const ExtendArgs& a, int i) {
  Request r = {0, 0, 0};
  const int seq = a.seq[i];
  if (seq < 0 || seq >= a.m.n_seqs) return r;
  const int sh = a.m.page_shift;
  const int64_t size = (int64_t)1 << sh, from = max(a.old_len[i], 0), to = a.new_len[i];
  if (to <= from) return r;
  const int64_t k0 = (from + size - 1) >> sh, k1 = (to + size - 1) >> sh;
  r.lacks = (int)max((int64_t)0, k1 - max(k0, a.m.pt_stride));
  r.pages = (int)max((int64_t)0, min(k1, a.m.pt_stride) - k0);
  r.first = 2 * (seq * a.m.pt_stride + k0);
  if ((from & (size - 1)) && k0 <= a.m.pt_stride) {
    const int page = a.m.table[seq * a.m.pt_stride + k0 - 1];
    if (in_pool(a.m, page) && a.m.refs[page] > 1) {
      r.pages += 1;
      r.first -= 1;
    }
  }
  return r;
}

// Prefix sums of the requests' pages into need[0 .. n] (cut at 2^30, more than any pool has: with a total beyond the pool nobody reads
// them), and into first[0 .. n - 1] (if there is one) the requests' own; returns the entries that do not fit their rows, cut likewise.
// r: request threadIdx.x (nothing, if there is none).
__device__ __forceinline__ int pg_needs(const ExtendArgs& a, Request r, int32_t* need, int64_t* first, uint64_t* sh) {
  constexpr uint64_t kMost = 1ull << 30;
  uint64_t base = 0, lacking = 0;
  for (int i = threadIdx.x;; ) {
    uint64_t total, lacks;
    const uint64_t off = pg_scan<uint64_t>((uint64_t)r.pages, sh, &total);
    if (__syncthreads_or(r.lacks != 0)) {
      pg_scan<uint64_t>((uint64_t)r.lacks, sh, &lacks);
      lacking += lacks;
    }
    if (i < a.n) {
      need[i] = (int32_t)min(base + off, kMost);
      if (first) first[i] = r.first;
    }
    base += total;
    i += kPgThreads;
    if (i - (int)threadIdx.x >= a.n) break;
    r = i < a.n ? pg_request(a, i) : Request{0, 0, 0};
  }
  if (threadIdx.x == 0) need[a.n] = (int32_t)min(base, kMost);
  return (int)min(lacking, kMost);
}

// Chunks of a large pool: masks and prefixes to the workspace, and, by the first workgroup, the requests' prefix sums.
template <bool FREE, bool REQUESTS>
__global__ __launch_bounds__(kPgThreads) void kv_pages_scan_kernel(const ExtendArgs a) {
  __shared__ ChunkMasks c;
  __shared__ uint64_t sh[kPgWaves];
  int v[kPgAhead], total;
  pg_counts<FREE>(a.m, blockIdx.x, 0, v);
  pg_masks<FREE>(a.m, blockIdx.x, v, c, sh, &total);
  const int64_t word = (int64_t)blockIdx.x * kPgThreads + threadIdx.x;
  a.w.mask[word] = c.mask[threadIdx.x];
  a.w.before[word] = c.before[threadIdx.x];
  if (threadIdx.x == 0) a.w.count[blockIdx.x] = total;
  if (REQUESTS && blockIdx.x == 0) {
    const int lacking = pg_needs(a, (int)threadIdx.x < a.n ? pg_request(a, threadIdx.x) : Request{0, 0, 0}, a.w.need, nullptr, sh);
    if (threadIdx.x == 0) a.w.need[a.n + 1] = lacking;
  }
}

// Set bits in the chunks in front of this one, and in all.
__device__ __forceinline__ int pg_chunks_before(const PageWork& w, int n_chunks, int chunk, uint64_t* sh, int* total) {
  int mine = 0, all = 0;
  for (int i = threadIdx.x; i < n_chunks; i += kPgThreads) {
    const int c = w.count[i];
    all += c;
    if (i < chunk) mine += c;
  }
  int before;
  pg_scan<int>(mine, sh, &before);
  pg_scan<int>(all, sh, total);
  return before;
}

// The chunk's masks and prefixes, from the workspace; *first: set bits in the chunks in front, *total: in all.
__device__ __forceinline__ void pg_load_chunk(const ExtendArgs& a, ChunkMasks& c, uint64_t* sh, int* first, int* total) {
  const int64_t word = (int64_t)blockIdx.x * kPgThreads + threadIdx.x;
  c.mask[threadIdx.x] = a.w.mask[word];
  c.before[threadIdx.x] = a.w.before[word];
  *first = pg_chunks_before(a.w, a.m.n_chunks, blockIdx.x, sh, total);
  __syncthreads();
}

// Entries that request i grows by, beside one for its shared last page; *k0: the first of them.
__device__ __forceinline__ int pg_grown(const ExtendArgs& a, int i, int64_t* k0) {
  const int64_t size1 = ((int64_t)1 << a.m.page_shift) - 1;
  *k0 = (max(a.old_len[i], 0) + size1) >> a.m.page_shift;
  return (int)(min((a.new_len[i] + size1) >> a.m.page_shift, a.m.pt_stride) - *k0);
}

// Gives the requests their pages, a lane per page of the pool.  ONE: the pool is one chunk, nothing has been prepared.
template <bool ONE>
__global__ __launch_bounds__(kPgThreads) void kv_pages_extend_kernel(const ExtendArgs a) {
  __shared__ ChunkMasks c;
  __shared__ uint64_t sh[kPgWaves];
  __shared__ int32_t sh_need[kPgMaxSeqs + 1];
  __shared__ int64_t sh_first[kPgMaxSeqs];     // (Request::first)
  int first = 0, total, lacking;
  if (ONE) {
    int v[kPgAhead];
    pg_counts<true>(a.m, 0, 0, v);              // (asked for before the request, a chain of loads of its own)
    const Request r = (int)threadIdx.x < a.n ? pg_request(a, threadIdx.x) : Request{0, 0, 0};
    pg_masks<true>(a.m, 0, v, c, sh, &total);
    lacking = pg_needs(a, r, sh_need, sh_first, sh);
  } else {
    pg_load_chunk(a, c, sh, &first, &total);
    for (int i = threadIdx.x; i <= a.n; i += kPgThreads) {
      sh_need[i] = a.w.need[i];
      if (i == a.n) break;
      int64_t k0 = 0;                           // (what a request takes beyond its growth is its shared page)
      const int pages = a.w.need[i + 1] - sh_need[i];
      const int copies = pages ? pages - pg_grown(a, i, &k0) : 0;
      sh_first[i] = pages ? 2 * (a.seq[i] * a.m.pt_stride + k0) - copies : 0;
    }
    lacking = a.w.need[a.n + 1];
  }
  __syncthreads();
  const int need = sh_need[a.n];
  const int short_of = (int)min((int64_t)lacking + max(0, need - total), (int64_t)1 << 29);   // (exact up to the cut: both sums are up to 2^30)
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) {
      a.status[0] = short_of;
      a.status[1] = total - (short_of ? 0 : need);
    }
    for (int i = threadIdx.x; i < a.n; i += kPgThreads) {      // pairs of requests that copy nothing; the others are written with their page
      if (short_of || sh_need[i + 1] == sh_need[i] || !(sh_first[i] & 1)) a.copy_src[i] = a.copy_dst[i] = -1;
    }
  }
  if (short_of) return;
  const int lane = threadIdx.x & 63;
  for (int w = threadIdx.x >> 6; w < kPgThreads; w += kPgWaves) {
    const uint64_t mask = c.mask[w];
    const int before = first + c.before[w];
    if (before >= need) break;
    const int r = before + lanes_below(mask);
    if (!mask_bit(mask, lane) || r >= need) continue;
    const int page = blockIdx.x * kPgChunk + w * 64 + lane;
    int lo = 0, hi = a.n - 1;                   // the request that rank r belongs to: the last one whose prefix is <= r
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sh_need[mid] <= r) lo = mid; else hi = mid - 1;
    }
    const int64_t f = sh_first[lo];
    const int j = r - sh_need[lo];
    int32_t* entry = a.m.table + (f >> 1) + j;
    if ((f & 1) && j == 0) {
      const int src = *entry;
      a.copy_src[lo] = src;
      a.copy_dst[lo] = page;
      if (in_pool(a.m, src)) atomicSub(&a.m.refs[src], 1);     // (a sequence listed twice may have changed the entry)
    }
    *entry = page;
    a.m.refs[page] = 1;
  }
}

__global__ __launch_bounds__(256) void kv_pages_init_kernel(const PageMap m) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, entries = (int64_t)m.n_seqs * m.pt_stride;
  for (int64_t e = i; e < entries; e += (int64_t)gridDim.x * 256) m.table[e] = -1;
  for (int64_t p = i; p < m.n_pages; p += (int64_t)gridDim.x * 256) m.refs[p] = 0;
}

// grid (entries / 256, requests)
__global__ __launch_bounds__(256) void kv_pages_truncate_kernel(const PageMap m, const int32_t* seq, const int32_t* keep_len) {
  const int i = blockIdx.y, b = seq[i];
  if (b < 0 || b >= m.n_seqs) return;
  const int64_t keep = keep_len ? max(keep_len[i], 0) : 0;
  const int64_t k = ((keep + ((int64_t)1 << m.page_shift) - 1) >> m.page_shift) + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= m.pt_stride) return;
  int32_t* entry = m.table + b * m.pt_stride + k;
  if (*entry == -1) return;
  const int page = atomicExch(entry, -1);        // (a sequence that is listed twice releases its pages once)
  if (in_pool(m, page) && atomicSub(&m.refs[page], 1) <= 0) atomicAdd(&m.refs[page], 1);
}

__global__ __launch_bounds__(256) void kv_pages_fork_kernel(const PageMap m, const int32_t* src, const int32_t* dst, const int32_t* len) {
  const int i = blockIdx.y, from = src[i], to = dst[i];
  if (from < 0 || from >= m.n_seqs || to < 0 || to >= m.n_seqs || from == to) return;
  const int64_t pages = min(((int64_t)max(len[i], 0) + ((int64_t)1 << m.page_shift) - 1) >> m.page_shift, m.pt_stride);
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= pages) return;
  const int page = m.table[from * m.pt_stride + k];
  m.table[to * m.pt_stride + k] = in_pool(m, page) ? page : -1;
  if (in_pool(m, page)) atomicAdd(&m.refs[page], 1);
}

// Lists the moves: with U pages in use, the r-th free page below U takes the r-th page in use from the top.
template <bool ONE>
__global__ __launch_bounds__(kPgThreads) void kv_pages_moves_kernel(const ExtendArgs a) {
  __shared__ ChunkMasks c;
  __shared__ uint64_t sh[kPgWaves];
  int first = 0, total;
  if (ONE) {
    int v[kPgAhead];
    pg_counts<false>(a.m, 0, 0, v);
    pg_masks<false>(a.m, 0, v, c, sh, &total);
    a.w.mask[threadIdx.x] = c.mask[threadIdx.x];
    a.w.before[threadIdx.x] = c.before[threadIdx.x];
  } else {
    pg_load_chunk(a, c, sh, &first, &total);
  }
  const int lane = threadIdx.x & 63, chunk0 = blockIdx.x * kPgChunk;
  const int words = (min(a.m.n_pages - chunk0, kPgChunk) + 63) / 64;
  for (int w = threadIdx.x >> 6; w < words; w += kPgWaves) {
    const uint64_t mask = c.mask[w];
    const int page = chunk0 + w * 64 + lane, used = first + c.before[w] + lanes_below(mask);
    const bool here = mask_bit(mask, lane);
    if (!here && page < total) a.copy_dst[page - used] = page;
    if (here && page >= total) a.copy_src[total - 1 - used] = page;
    if (page == max(total - 1, 0)) {            // moves: the pages in use from U on, which page U - 1 can tell
      a.status[0] = total;
      a.status[1] = total - used - (here ? 1 : 0);
    }
  }
}

// Follows the moves in the table and the counts.
__global__ __launch_bounds__(256) void kv_pages_remap_kernel(const ExtendArgs a) {
  __shared__ int sh_chunk[1024 + 1];                   // pages in use in front of a chunk
  const int used = a.status[0], moves = a.status[1];
  if (moves == 0) return;
  if (a.m.n_chunks > 1) {
    // (at most kPgMaxPages / kPgChunk = 1024 chunks: four per thread, summed by waves)
    __shared__ int sh_w[4];
    int c[4], sum = 0;
    for (int i = 0; i < 4; ++i) {
      const int k = threadIdx.x * 4 + i;
      c[i] = k < a.m.n_chunks ? a.w.count[k] : 0;
      sum += c[i];
    }
    const int incl = wave_incl_scan(sum);
    if ((threadIdx.x & 63) == 63) sh_w[threadIdx.x >> 6] = incl;
    __syncthreads();
    int off = incl - sum;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) off += sh_w[w];
    for (int i = 0; i < 4; ++i) {
      sh_chunk[threadIdx.x * 4 + i] = off;
      off += c[i];
    }
    __syncthreads();
  }
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256, entries = (int64_t)a.m.n_seqs * a.m.pt_stride;
  for (int64_t e = t; e < entries; e += step) {
    const int page = a.m.table[e];
    if (page < used || page >= a.m.n_pages) continue;
    const uint64_t mask = a.w.mask[page >> 6];
    if (!mask_bit(mask, page & 63)) continue;
    const int rank = (a.m.n_chunks > 1 ? sh_chunk[page / kPgChunk] : 0) + a.w.before[page >> 6] + mask_below(mask, page & 63);
    a.m.table[e] = a.copy_dst[used - 1 - rank];
  }
  for (int64_t r = t; r < moves; r += step) {
    const int from = a.copy_src[r], to = a.copy_dst[r];
    a.m.refs[to] = a.m.refs[from];
    a.m.refs[from] = 0;
  }
}

// ---- bytes ------------------------------------------------------------------------------------------------------------------------
struct CopyPool {
  uint8_t* base;
  int64_t page_stride, head_stride;
  int32_t page16;                 // 16-byte words of a page of one head
  int32_t pieces;                 // pieces of kPieceWords words of it
};
struct CopyArgs {
  CopyPool pool[kPgPools];
  int32_t first[kPgPools + 1];    // pieces of a page pair in front of a pool
  int32_t n_pools, n_pages, n;
  const int32_t* src;
  const int32_t* dst;
  const int32_t* count;
};
constexpr int kPieceWords = 256;  // a wave's piece: four 16-byte words per lane, 4 KB
// What passes this many pieces (64 MB) streams: it is read past the caches, by two workgroups per compute unit only (983 pages of
// 256 KB: 92 us, 5.6 TB/s; 97 with eight, 105 with ordinary loads and stores).  Less is copied by all that fit (64 such pages: 6 us, 8 by
// two workgroups).  Stores pass the caches either way (64 pages 6.5 us without, 983 pages 105).
constexpr int64_t kStreamPieces = 16384;
constexpr unsigned kStreamGroups = 512;

template <bool STREAM>
__device__ __forceinline__ void copy_pieces(const CopyArgs& a, int64_t items, int per_pair, int64_t waves) {
  const int lane = threadIdx.x & 63;
  for (int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < items; item += waves) {
    const int pair = (int)(item / per_pair), rest = (int)(item - (int64_t)pair * per_pair);
    const int src = a.src[pair], dst = a.dst[pair];
    if ((uint32_t)src >= (uint32_t)a.n_pages || (uint32_t)dst >= (uint32_t)a.n_pages || src == dst) continue;
    int k = 0;
    while (rest >= a.first[k + 1]) ++k;
    const CopyPool& p = a.pool[k];
    const int head = (rest - a.first[k]) / p.pieces, piece = rest - a.first[k] - head * p.pieces;
    const int64_t at = head * p.head_stride;
    const u32x4* s = reinterpret_cast<const u32x4*>(p.base + at + src * p.page_stride);
    u32x4* d = reinterpret_cast<u32x4*>(p.base + at + dst * p.page_stride);
    u32x4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int w = piece * kPieceWords + i * 64 + lane;
      if (w < p.page16) v[i] = STREAM ? __builtin_nontemporal_load(s + w) : s[w];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int w = piece * kPieceWords + i * 64 + lane;
      if (w < p.page16) __builtin_nontemporal_store(v[i], d + w);
    }
  }
}

__global__ __launch_bounds__(256) void kv_pages_copy_kernel(const CopyArgs a) {
  const int n = a.count ? min(max(*a.count, 0), a.n) : a.n;
  const int per_pair = a.first[a.n_pools];
  const int64_t items = (int64_t)n * per_pair;
  if (items > kStreamPieces) {
    const unsigned groups = min(gridDim.x, kStreamGroups);
    if (blockIdx.x < groups) copy_pieces<true>(a, items, per_pair, (int64_t)groups * 4);
  } else {
    copy_pieces<false>(a, items, per_pair, (int64_t)gridDim.x * 4);
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------------------
static int32_t check_map(const char* who, const rtp_page_map* map, PageMap* m) {
  if (!map) return fail(RTP_ERR_INVALID_ARG, "%s: page map is NULL", who);
  if (!map->page_table || !map->page_refs) return fail(RTP_ERR_INVALID_ARG, "%s: NULL page_table/page_refs", who);
  const int32_t ps = map->page_size;
  if (ps < 16 || (ps & (ps - 1)) || ps > (1 << 20))
    return fail(RTP_ERR_INVALID_ARG, "%s: page_size must be a power of two in [16, 2^20]", who);
  if (map->n_seqs <= 0 || map->pt_stride <= 0 || map->n_pages <= 0)
    return fail(RTP_ERR_INVALID_ARG, "%s: n_seqs, pt_stride and n_pages must be positive", who);
  if (map->n_pages > kPgMaxPages || map->pt_stride > kPgMaxPages)
    return fail(RTP_ERR_UNSUPPORTED, "%s: more than 2^26 pages", who);
  int sh = 4;
  while ((1 << sh) < ps) ++sh;
  *m = PageMap{map->page_table, map->pt_stride, map->page_refs, map->n_seqs, sh, map->n_pages, (map->n_pages + kPgChunk - 1) / kPgChunk};
  return RTP_OK;
}

static size_t work_layout(int64_t n_pages, int64_t n, void* ws, PageWork* w) {
  const size_t chunks = (size_t)((n_pages + kPgChunk - 1) / kPgChunk), words = chunks * kPgThreads;
  const size_t mask = 0, before = words * 8, count = before + words * 4, need = align_up(count + chunks * 4, 256);
  if (w) *w = PageWork{(uint64_t*)((char*)ws + mask), (int32_t*)((char*)ws + before), (int32_t*)((char*)ws + count), (int32_t*)((char*)ws + need)};
  return align_up(need + (size_t)(n + 2) * 4, 256);
}

static int32_t check_work(const char* who, const PageMap& m, int64_t n, void* ws, size_t ws_bytes, PageWork* w) {
  const size_t need = work_layout(m.n_pages, n, ws, w);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(RTP_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required, got %zu", who, need, ws_bytes);
  return RTP_OK;
}

static unsigned grid_of(int64_t items, int64_t most) {
  const int64_t g = (items + 255) / 256;
  return (unsigned)(g < 1 ? 1 : g > most ? most : g);
}

}  // namespace rtp

using namespace rtp;

extern "C" size_t rtp_kv_pages_workspace_bytes(const rtp_page_map* map, int32_t n) {
  if (!map || map->n_pages <= 0 || n < 0) return 256;
  return work_layout(map->n_pages, n < kPgMaxSeqs ? n : kPgMaxSeqs, nullptr, nullptr);
}

extern "C" int32_t rtp_kv_pages_init(const rtp_page_map* map, void* stream) {
  const char* who = "rtp_kv_pages_init";
  PageMap m;
  const int32_t rc = check_map(who, map, &m);
  if (rc != RTP_OK) return rc;
  clear_error();
  const int64_t entries = (int64_t)m.n_seqs * m.pt_stride;
  RTP_LAUNCH(kv_pages_init_kernel, dim3(grid_of(entries > m.n_pages ? entries : m.n_pages, 2048)), dim3(256), 0, (hipStream_t)stream, m);
  return check_launch(who);
}

static int32_t check_requests(const char* who, int32_t n) {
  if (n <= 0 || n > 65535) return fail(RTP_ERR_INVALID_ARG, "%s: n must be in [1, 65535]", who);
  return RTP_OK;
}

extern "C" int32_t rtp_kv_pages_truncate(const rtp_page_map* map, const int32_t* seq, const int32_t* keep_len, int32_t n,
                                         void* stream) {
  const char* who = "rtp_kv_pages_truncate";
  PageMap m;
  int32_t rc = check_map(who, map, &m);
  if (rc == RTP_OK) rc = check_requests(who, n);
  if (rc != RTP_OK) return rc;
  if (!seq) return fail(RTP_ERR_INVALID_ARG, "%s: NULL seq", who);
  clear_error();
  RTP_LAUNCH(kv_pages_truncate_kernel, dim3((unsigned)((m.pt_stride + 255) / 256), (unsigned)n), dim3(256), 0, (hipStream_t)stream, m, seq,
             keep_len);
  return check_launch(who);
}

extern "C" int32_t rtp_kv_pages_fork(const rtp_page_map* map, const int32_t* src_seq, const int32_t* dst_seq, const int32_t* len,
                                     int32_t n, void* stream) {
  const char* who = "rtp_kv_pages_fork";
  PageMap m;
  int32_t rc = check_map(who, map, &m);
  if (rc == RTP_OK) rc = check_requests(who, n);
  if (rc != RTP_OK) return rc;
  if (!src_seq || !dst_seq || !len) return fail(RTP_ERR_INVALID_ARG, "%s: NULL src_seq/dst_seq/len", who);
  clear_error();
  RTP_LAUNCH(kv_pages_fork_kernel, dim3((unsigned)((m.pt_stride + 255) / 256), (unsigned)n), dim3(256), 0, (hipStream_t)stream, m, src_seq,
             dst_seq, len);
  return check_launch(who);
}

extern "C" int32_t rtp_kv_pages_extend(const rtp_page_map* map, const int32_t* seq, const int32_t* old_len, const int32_t* new_len,
                                       int32_t n, int32_t* copy_src, int32_t* copy_dst, int32_t* status, void* ws, size_t ws_bytes,
                                       void* stream) {
  const char* who = "rtp_kv_pages_extend";
  ExtendArgs a = {};
  int32_t rc = check_map(who, map, &a.m);
  if (rc != RTP_OK) return rc;
  if (n <= 0) return fail(RTP_ERR_INVALID_ARG, "%s: n must be positive", who);
  if (n > kPgMaxSeqs) return fail(RTP_ERR_UNSUPPORTED, "%s: more than %d sequences in one call", who, kPgMaxSeqs);
  if (!seq || !old_len || !new_len || !copy_src || !copy_dst || !status) return fail(RTP_ERR_INVALID_ARG, "%s: NULL pointer", who);
  rc = check_work(who, a.m, n, ws, ws_bytes, &a.w);
  if (rc != RTP_OK) return rc;
  clear_error();
  a.seq = seq;
  a.old_len = old_len;
  a.new_len = new_len;
  a.n = n;
  a.copy_src = copy_src;
  a.copy_dst = copy_dst;
  a.status = status;
  hipStream_t s = (hipStream_t)stream;
  const dim3 block(kPgThreads), grid((unsigned)a.m.n_chunks);
  if (a.m.n_chunks == 1) {
    RTP_LAUNCH(kv_pages_extend_kernel<true>, grid, block, 0, s, a);
  } else {
    RTP_LAUNCH((kv_pages_scan_kernel<true, true>), grid, block, 0, s, a);
    RTP_LAUNCH(kv_pages_extend_kernel<false>, grid, block, 0, s, a);
  }
  return check_launch(who);
}

extern "C" int32_t rtp_kv_pages_compact(const rtp_page_map* map, int32_t* move_src, int32_t* move_dst, int32_t* status, void* ws,
                                        size_t ws_bytes, void* stream) {
  const char* who = "rtp_kv_pages_compact";
  ExtendArgs a = {};
  int32_t rc = check_map(who, map, &a.m);
  if (rc != RTP_OK) return rc;
  if (!move_src || !move_dst || !status) return fail(RTP_ERR_INVALID_ARG, "%s: NULL pointer", who);
  rc = check_work(who, a.m, 0, ws, ws_bytes, &a.w);
  if (rc != RTP_OK) return rc;
  clear_error();
  a.copy_src = move_src;
  a.copy_dst = move_dst;
  a.status = status;
  hipStream_t s = (hipStream_t)stream;
  const dim3 block(kPgThreads), grid((unsigned)a.m.n_chunks);
  if (a.m.n_chunks == 1) {
    RTP_LAUNCH(kv_pages_moves_kernel<true>, grid, block, 0, s, a);
  } else {
    RTP_LAUNCH((kv_pages_scan_kernel<false, false>), grid, block, 0, s, a);
    RTP_LAUNCH(kv_pages_moves_kernel<false>, grid, block, 0, s, a);
  }
  const int64_t entries = (int64_t)a.m.n_seqs * a.m.pt_stride;
  RTP_LAUNCH(kv_pages_remap_kernel, dim3(grid_of(entries > a.m.n_pages ? entries : a.m.n_pages, 1024)), dim3(256), 0, s, a);
  return check_launch(who);
}

extern "C" int32_t rtp_kv_pages_copy(const rtp_page_pool* pools, int32_t n_pools, int32_t n_pages, const int32_t* src,
                                     const int32_t* dst, int32_t n, const int32_t* count, void* stream) {
  const char* who = "rtp_kv_pages_copy";
  if (!pools || !src || !dst) return fail(RTP_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (n_pools <= 0 || n_pages <= 0 || n <= 0) return fail(RTP_ERR_INVALID_ARG, "%s: n_pools, n_pages and n must be positive", who);
  for (int i = 0; i < n_pools; ++i) {
    const rtp_page_pool& p = pools[i];
    if (!p.base || ((uintptr_t)p.base & 15) || (p.page_stride & 15) || (p.head_stride & 15) || (p.page_bytes & 15))
      return fail(RTP_ERR_INVALID_ARG, "%s: pool %d: base, strides and page_bytes must be 16-byte aligned", who, i);
    if (p.page_bytes <= 0 || p.page_bytes > ((int64_t)1 << 32) || p.n_heads <= 0 || p.n_heads > 65535)
      return fail(RTP_ERR_INVALID_ARG, "%s: pool %d: page_bytes must be in (0, 2^32], n_heads in [1, 65535]", who, i);
    if (!strides_apart(p.page_stride, n_pages, p.head_stride, p.n_heads, p.page_bytes))
      return fail(RTP_ERR_INVALID_ARG, "%s: pool %d: strides let pages or heads overlap", who, i);
    if ((p.page_bytes / 16 + kPieceWords - 1) / kPieceWords * p.n_heads > (1 << 24))
      return fail(RTP_ERR_UNSUPPORTED, "%s: pool %d: a page of all heads is larger than 2^36 bytes", who, i);
  }
  clear_error();
  for (int at = 0; at < n_pools; at += kPgPools) {
    CopyArgs a = {};
    a.n_pools = n_pools - at < kPgPools ? n_pools - at : kPgPools;
    for (int k = 0; k < a.n_pools; ++k) {
      const rtp_page_pool& p = pools[at + k];
      const int32_t words = (int32_t)(p.page_bytes / 16), pieces = (words + kPieceWords - 1) / kPieceWords;
      a.pool[k] = CopyPool{(uint8_t*)p.base, p.page_stride, p.head_stride, words, pieces};
      a.first[k + 1] = a.first[k] + pieces * p.n_heads;
    }
    a.n_pages = n_pages;
    a.n = n;
    a.src = src;
    a.dst = dst;
    a.count = count;
    const int64_t items = (int64_t)n * a.first[a.n_pools];
    const unsigned grid = (unsigned)((items + 3) / 4 < 2048 ? (items + 3) / 4 : 2048);
    RTP_LAUNCH(kv_pages_copy_kernel, dim3(grid), dim3(256), 0, (hipStream_t)stream, a);
  }
  return check_launch(who);
}
