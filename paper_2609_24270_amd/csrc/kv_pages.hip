// The pages of a paged key/value cache, managed on the device: rows of a table
// take, share, copy and give up pages of a pool without the host knowing which.
//
// State: table [R][H][pph] (page of each (row, head, 32-token page), -1 where there is
// none), lens [R] (tokens of each row), refs [pool_pages] (table entries that name a
// page; 0: the page is free).  Pages are taken lowest first, in an order fixed by the
// arguments, so that the result never depends on timing; refs is changed with integer
// atomics, whose order does not matter.
//
// A call is a few short launches, since each step needs the whole of the one before:
//   1. segments of 4096 pages are counted (free or live); beside them one workgroup lays
//      out what the call needs (a prefix over its requests);
//   2. each segment adds up the counts before it and writes its pages' numbers to their
//      places in a list;
//   3. the tables, the counts and the pages themselves are changed.
// (Free and keep need no pages, and are one launch.)
// Up to 16384 pages and 1024 requests one workgroup does 1 and 2, and all of an extend:
// short calls are bound by their launches.  Large ones are bound by the copies (each page
// read and written once).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "kv_fp4.h"

namespace asym {
namespace {

constexpr int kSeg = 4096;     // pages counted by a workgroup
constexpr int kThreads = 256;
constexpr int kPer = kSeg / kThreads;  // pages of a thread
constexpr int kSmallThreads = 1024;    // of the one workgroup of a small call
constexpr int kMoveWords = 4;          // 16-byte words that a thread moves at a time

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Words of the workspace, in order: the header; counts [segments]; list [pool_pages]; then
// holes [pool_pages] and where [pool_pages] (compact), or first [n] (place of a request's
// first page in the list), flag [n] and claim [R] (the first request that names a row), and
// new_len [n] and rows [n][H][pph] (fork).
enum { kNeed = 0, kTotal = 1, kHoles = 2, kHeader = 16 };

struct PagesParams {
  int* table;
  int* lens;
  int* refs;
  const int *a, *b;  // extend: rows, new lengths; fork: sources, targets; free: rows
  int* status;       // [2], nullable
  uint8_t *k_pool, *v_pool;
  int64_t page_bytes;
  int R, H, pph, pool, n, segs;
  int *head, *counts, *first, *flag, *claim, *list, *rows, *new_len, *holes, *where;
};

__device__ __forceinline__ int pages_of(int len, int pph) {
  return min((int)(((int64_t)max(len, 0) + kKvPageTokens - 1) / kKvPageTokens), pph);
}

// Sum over the workgroup's threads before this one, and over all of them.
template <int THREADS>
__device__ __forceinline__ int block_scan(int x, int* red, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = wave_scan_add(x);
  __syncthreads();  // (red may still be read from the call before)
  if (lane == 63) red[wave] = upto;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += red[w];
    all += red[w];
  }
  return before + upto - x;
}

enum { kExtend, kFork, kCompact };

// Pages that request i needs (-1: it is left out, `first`: no earlier request names its row).
template <int OP>
__device__ __forceinline__ int request_needs(const PagesParams& p, int i, bool first) {
  if constexpr (OP == kExtend) {
    const int r = p.a[i], to = p.b[i];
    // (a row outside the table, a length that is no longer or does not fit: left as it is)
    if (!first || r < 0 || r >= p.R || to <= p.lens[r] || (int64_t)to > (int64_t)p.pph * kKvPageTokens) return -1;
    return (pages_of(to, p.pph) - pages_of(p.lens[r], p.pph)) * p.H;
  } else {
    const int s = p.a[i], d = p.b[i];
    if (!first || s < 0 || s >= p.R || d < 0 || d >= p.R || s == d) return -1;
    return min(max(p.lens[s], 0), p.pph * kKvPageTokens) % kKvPageTokens ? p.H : 0;
  }
}

// A thread's kPer pages: bit i says whether page first + i is live (compact) or free.
template <int OP>
__device__ __forceinline__ uint32_t page_bits(const PagesParams& p, int64_t first) {
  uint32_t bits = 0;
  int r[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) r[i] = first + i < p.pool ? p.refs[first + i] : OP == kCompact ? 0 : 1;
#pragma unroll
  for (int i = 0; i < kPer; ++i) bits |= (uint32_t)((r[i] > 0) == (OP == kCompact)) << i;
  return bits;
}

// 2. list[r]: the r-th free page (as many as are needed), or the r-th live one; compact:
// holes[r], the r-th free page below the number of live ones, and where[page] = page.
// `rank`: of the thread's first page.
template <int OP>
__device__ __forceinline__ void place_pages(const PagesParams& p, int64_t first, uint32_t bits, int rank, int need,
                                            int total) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t page = first + i;
    const bool x = (bits >> i) & 1;
    if (page >= p.pool) break;
    if constexpr (OP == kCompact) {
      if (x) p.list[rank] = (int)page;
      p.where[page] = (int)page;
      if (!x && page < total) p.holes[page - rank] = (int)page;
      if (page == total - 1) p.head[kHoles] = total - rank - (x ? 1 : 0);  // free pages below `total`
    } else {
      if (x && rank < need) p.list[rank] = (int)page;
    }
    rank += x;
  }
}

// 1. counts[s]: free pages (extend, fork) or live ones (compact) of segment s; the last
// workgroup: what the requests need.
template <int OP>
__global__ void __launch_bounds__(kThreads) pages_count(PagesParams p) {
  __shared__ int red[kThreads / 64];
  const int seg = blockIdx.x;
  if (seg < p.segs) {
    int all;
    block_scan<kThreads>(__popc(page_bits<OP>(p, (int64_t)seg * kSeg + (int)threadIdx.x * kPer)), red, all);
    if (threadIdx.x == 0) p.counts[seg] = all;
    return;
  }
  if constexpr (OP != kCompact) {
    const int* row_of = OP == kExtend ? p.a : p.b;  // the row that a request changes
    for (int r = threadIdx.x; r < p.R; r += kThreads) p.claim[r] = 0x7FFFFFFF;
    __syncthreads();
    for (int i = threadIdx.x; i < p.n; i += kThreads)
      if (row_of[i] >= 0 && row_of[i] < p.R) atomicMin(&p.claim[row_of[i]], i);
    __syncthreads();
    int base = 0;
    for (int i0 = 0; i0 < p.n; i0 += kThreads) {
      const int i = i0 + threadIdx.x;
      int need = -1;
      if (i < p.n) {
        const int r = row_of[i];
        const bool first = r >= 0 && r < p.R &&
                           __hip_atomic_load(&p.claim[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
        need = request_needs<OP>(p, i, first);
      }
      int all;
      const int before = block_scan<kThreads>(max(need, 0), red, all);
      if (i < p.n) {
        p.first[i] = base + before;
        p.flag[i] = need >= 0;
      }
      base += all;
    }
    if (threadIdx.x == 0) p.head[kNeed] = base;
  }
}

// 2.
template <int OP>
__global__ void __launch_bounds__(kThreads) pages_list(PagesParams p) {
  __shared__ int red[kThreads / 64];
  const int seg = blockIdx.x;
  const int64_t first = (int64_t)seg * kSeg + (int)threadIdx.x * kPer;
  const uint32_t bits = page_bits<OP>(p, first);
  int mine = 0, tot = 0;
  for (int s = threadIdx.x; s < p.segs; s += kThreads) {
    const int c = p.counts[s];
    tot += c;
    if (s < seg) mine += c;
  }
  int base, total, all;
  block_scan<kThreads>(mine, red, base);
  block_scan<kThreads>(tot, red, total);
  if (seg == 0 && threadIdx.x == 0) {
    p.head[kTotal] = total;
    if (OP == kCompact && total == 0) p.head[kHoles] = 0;
  }
  const int need = OP == kCompact ? 0 : p.head[kNeed];
  if (OP != kCompact && base >= need) return;  // (the whole workgroup)
  const int rank = base + block_scan<kThreads>(__popc(bits), red, all);
  place_pages<OP>(p, first, bits, rank, need, total);
}

__device__ __forceinline__ void write_status(const PagesParams& p, int need, int total) {
  if (!p.status) return;
  p.status[0] = need <= total ? need : 0;
  p.status[1] = need <= total ? 0 : need - total;
}

// 1 and 2 of a small call, and 3 of an extend.
template <int OP>
__global__ void __launch_bounds__(kSmallThreads) pages_small(PagesParams p) {
  __shared__ int red[kSmallThreads / 64];
  __shared__ int row_of[kSmallThreads], start[kSmallThreads];
  const int i = threadIdx.x;
  const uint32_t bits = page_bits<OP>(p, (int64_t)i * kPer);
  int need = 0, total;
  if constexpr (OP != kCompact) {
    const int row = i < p.n ? (OP == kExtend ? p.a : p.b)[i] : -1;
    row_of[i] = row;
    __syncthreads();
    bool first = i < p.n;
    for (int j = 0; j < i && j < p.n; ++j) first &= row_of[j] != row;
    const int x = i < p.n ? request_needs<OP>(p, i, first) : -1;
    start[i] = block_scan<kSmallThreads>(max(x, 0), red, need);
    if (i < p.n) {
      p.first[i] = start[i];
      p.flag[i] = x >= 0;
    }
    if (x < 0) row_of[i] = -1;  // (each thread's own; read after the next barrier)
  }
  const int rank = block_scan<kSmallThreads>(__popc(bits), red, total);
  place_pages<OP>(p, (int64_t)i * kPer, bits, rank, need, total);
  if (i == 0) {
    p.head[kNeed] = need;
    p.head[kTotal] = total;
    if (OP == kCompact && total == 0) p.head[kHoles] = 0;
  }
  if constexpr (OP == kExtend) {
    if (i == 0) write_status(p, need, total);
    if (need > total) return;
    __syncthreads();  // (the list is there)
    for (int x = i; x < need; x += kSmallThreads) {
      int lo = 0, hi = p.n;  // the last request whose pages begin at or before x (those that take none are passed over)
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (start[mid] <= x)
          lo = mid;
        else
          hi = mid;
      }
      const int r = row_of[lo], had = pages_of(p.lens[r], p.pph), add = pages_of(p.b[lo], p.pph) - had;
      const int at = x - start[lo], h = at / add, page = p.list[x];
      p.table[((int64_t)r * p.H + h) * p.pph + had + (at - h * add)] = page;
      p.refs[page] = 1;
    }
    __syncthreads();  // (every thread has read the old lengths)
    if (i < p.n && row_of[i] >= 0) p.lens[row_of[i]] = p.b[i];
  }
}

// The 16-byte word w of a pair of pages (keys, then values)
__device__ __forceinline__ u32x4* pair_word(const PagesParams& p, int64_t page, uint32_t w) {
  const uint32_t words = (uint32_t)(p.page_bytes / 16);
  uint8_t* pool = w < words ? p.k_pool : p.v_pool;
  return reinterpret_cast<u32x4*>(pool + page * p.page_bytes) + (w < words ? w : w - words);
}

// Page `to` of both pools := page `from`, four loads a thread on their way at a time
__device__ __forceinline__ void copy_pages(const PagesParams& p, int64_t to, int64_t from) {
  const uint32_t all = (uint32_t)(p.page_bytes / 16) * (p.v_pool ? 2 : 1);
  for (uint32_t w0 = threadIdx.x; w0 < all; w0 += 4 * kThreads) {
    u32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (w0 + u * kThreads < all) x[u] = *pair_word(p, from, w0 + u * kThreads);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (w0 + u * kThreads < all) *pair_word(p, to, w0 + u * kThreads) = x[u];
  }
}

// 3. extend: a workgroup a request
__global__ void __launch_bounds__(kThreads) pages_extend(PagesParams p) {
  const int need = p.head[kNeed], total = p.head[kTotal];
  const int i = blockIdx.x;
  const bool enough = need <= total;
  if (i == 0 && threadIdx.x == 0) write_status(p, need, total);
  if (!enough || i >= p.n || !p.flag[i]) return;
  const int r = p.a[i], to = p.b[i];
  const int had = pages_of(p.lens[r], p.pph), add = pages_of(to, p.pph) - had;
  for (int x = threadIdx.x; x < add * p.H; x += kThreads) {
    const int h = x / add, c = x - h * add;
    const int page = p.list[p.first[i] + x];
    p.table[((int64_t)r * p.H + h) * p.pph + had + c] = page;
    p.refs[page] = 1;
  }
  __syncthreads();  // (every thread has read the old length)
  if (threadIdx.x == 0) p.lens[r] = to;
}

// 3. fork: a workgroup a (request, head) lays out the new row beside the table, takes
// its references, and copies the part page
__global__ void __launch_bounds__(kThreads) pages_fork(PagesParams p) {
  const int need = p.head[kNeed], total = p.head[kTotal];
  const bool enough = need <= total;
  const int i = blockIdx.x / p.H, h = blockIdx.x - i * p.H;
  if (blockIdx.x == 0 && threadIdx.x == 0) write_status(p, need, total);
  if (!enough || i >= p.n || !p.flag[i]) return;
  const int s = p.a[i];
  const int len = min(max(p.lens[s], 0), p.pph * kKvPageTokens), whole = len / kKvPageTokens;
  const int* from = p.table + ((int64_t)s * p.H + h) * p.pph;
  int* to = p.rows + ((int64_t)i * p.H + h) * p.pph;
  for (int c = threadIdx.x; c < p.pph; c += kThreads) {
    const int page = c < whole ? from[c] : -1;
    to[c] = page;
    if (page >= 0 && page < p.pool) atomicAdd(&p.refs[page], 1);
  }
  if (h == 0 && threadIdx.x == 0) p.new_len[i] = len;
  if (len % kKvPageTokens == 0) return;
  const int page = p.list[p.first[i] + h], old = from[whole];
  __syncthreads();  // (the row's entry was -1 until here)
  if (threadIdx.x == 0) {
    to[whole] = page;
    p.refs[page] = 1;
  }
  if (old < 0 || old >= p.pool) return;
  copy_pages(p, page, old);
}

__device__ void release_row(const PagesParams& p, int r) {
  const int used = pages_of(p.lens[r], p.pph);
  for (int x = threadIdx.x; x < used * p.H; x += kThreads) {
    const int h = x / used, c = x - h * used;
    const int page = p.table[((int64_t)r * p.H + h) * p.pph + c];
    if (page >= 0 && page < p.pool) atomicSub(&p.refs[page], 1);
  }
  __syncthreads();
}

// 4. fork: the targets' old rows are given up, the new ones take their place
__global__ void __launch_bounds__(kThreads) pages_fork_rows(PagesParams p) {
  if (p.head[kNeed] > p.head[kTotal] || !p.flag[blockIdx.x]) return;
  const int r = p.b[blockIdx.x];
  release_row(p, r);
  const int64_t row = (int64_t)p.H * p.pph;
  for (int64_t x = threadIdx.x; x < row; x += kThreads) p.table[r * row + x] = p.rows[blockIdx.x * row + x];
  if (threadIdx.x == 0) p.lens[r] = p.new_len[blockIdx.x];
}

__global__ void __launch_bounds__(kThreads) pages_free(PagesParams p) {
  const int i = blockIdx.x, r = p.a[i];
  if (r < 0 || r >= p.R) return;
  bool seen = false;
  for (int j = threadIdx.x; j < i; j += kThreads) seen |= p.a[j] == r;
  if (__syncthreads_or(seen)) return;
  release_row(p, r);
  const int64_t row = (int64_t)p.H * p.pph;
  for (int64_t x = threadIdx.x; x < row; x += kThreads) p.table[r * row + x] = -1;
  if (threadIdx.x == 0) p.lens[r] = 0;
}

// 3. compact: the live pages at or above the number of live ones go, in order, into the
// holes below it (sources and targets never meet)
__global__ void __launch_bounds__(kThreads) pages_move(PagesParams p) {
  const int total = p.head[kTotal], holes = p.head[kHoles];
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.status) {
    p.status[0] = holes;
    p.status[1] = total;
  }
  for (int j = blockIdx.x * kThreads + threadIdx.x; j < holes; j += gridDim.x * kThreads) {
    const int from = p.list[total - holes + j], to = p.holes[j];
    p.where[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  // The pages' words as one list, kMoveWords * kThreads a workgroup at a time, so that small
  // pages fill it as well as large ones.  256 rows, 42734 pairs of 8 KiB pages moved, 1.40 GB:
  // 271 us with a workgroup a pair in 4096 workgroups, 257 to 280 with eight words a thread,
  // 238 (5.9 TB/s; a plain copy of 2 GiB 5.0) with four, non-temporal, a workgroup to almost
  // every pair.
  const uint32_t all = (uint32_t)(p.page_bytes / 16) * (p.v_pool ? 2 : 1);
  const int64_t words = (int64_t)holes * all;
  for (int64_t c = (int64_t)blockIdx.x * (kMoveWords * kThreads); c < words; c += (int64_t)gridDim.x * (kMoveWords * kThreads)) {
    const int j0 = (int)(c / all);
    const uint32_t w0 = (uint32_t)(c - (int64_t)j0 * all) + threadIdx.x;
    u32x4 x[kMoveWords];
    u32x4* to[kMoveWords];
#pragma unroll
    for (int u = 0; u < kMoveWords; ++u) {
      const uint32_t w = w0 + u * kThreads, d = w / all;
      to[u] = nullptr;
      if (c + (u * kThreads + (int)threadIdx.x) < words) {
        const int j = j0 + (int)d;
        x[u] = __builtin_nontemporal_load(pair_word(p, p.list[total - holes + j], w - d * all));
        to[u] = pair_word(p, p.holes[j], w - d * all);
      }
    }
#pragma unroll
    for (int u = 0; u < kMoveWords; ++u)
      if (to[u]) __builtin_nontemporal_store(x[u], to[u]);
  }
}

// 4. compact: the tables' entries follow
__global__ void __launch_bounds__(kThreads) pages_rename(PagesParams p) {
  if (p.head[kHoles] == 0) return;
  const int64_t n = (int64_t)p.R * p.H * p.pph;
  for (int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x; x < n; x += (int64_t)gridDim.x * kThreads) {
    const int page = p.table[x];
    if (page >= 0 && page < p.pool) {
      const int to = p.where[page];
      if (to != page) p.table[x] = to;
    }
  }
}

// keep: a workgroup a request.  Of the row's last n tokens (the drafted ones) those that path names move down to
// their head, in order; the rest and the pages behind them are given up.  A thread has a 16-byte word of a
// token of one head and pool, and moves it token by token, kKeepTokens loads on their way at a time: path rises, so
// that the j-th token comes from place path[j] >= j, and what is written, places up to j, is no later token's
// source (places above j).
// Bound by a chain of reads that depend on each other where rows are few (8 of 8 nodes behind 900 tokens: 6.8 us), by
// how the words lie where they are many (256 of 32 behind up to 4000, 7 MB in pieces of 256 bytes over 2 GB: 16 us).
constexpr int kKeepTokens = 8;
__global__ void __launch_bounds__(kSmallThreads) pages_keep(PagesParams p, int T, const int* cu, const int* path, const int* count) {
  const int i = blockIdx.x, r = p.a[i];
  if (r < 0 || r >= p.R) return;
  bool bad = false;
  for (int j = threadIdx.x; j < i; j += blockDim.x) bad |= p.a[j] == r;  // (an earlier request of the call has the row,
  if (__syncthreads_or(bad)) return;                                     // and changes what is read from here on)
  int at, n;
  packed_rows(cu, i, T, at, n);
  const int len = min(p.lens[r], p.pph * kKvPageTokens), keep = count[i], base = len - n;
  if (base < 0 || keep < 0 || keep > n) return;
  for (int j = threadIdx.x; j < keep; j += blockDim.x) {
    const int x = path[at + j];
    bad |= x < 0 || x >= n || (j > 0 && path[at + j - 1] >= x);
  }
  // (a page that another row has as well is not written to)
  for (int64_t x = threadIdx.x; x < (int64_t)keep * p.H; x += blockDim.x) {
    const int64_t head = x / keep;
    const int j = (int)(x - head * keep);
    if (path[at + j] == j) continue;
    const int page = p.table[((int64_t)r * p.H + head) * p.pph + (base + j) / kKvPageTokens];
    bad |= page >= 0 && page < p.pool && p.refs[page] > 1;
  }
  // (nor does the row come to end inside one, where its next tokens would be written)
  const int now = base + keep;
  if (now < len && now % kKvPageTokens)
    for (int head = threadIdx.x; head < p.H; head += blockDim.x) {
      const int page = p.table[((int64_t)r * p.H + head) * p.pph + now / kKvPageTokens];
      bad |= page >= 0 && page < p.pool && p.refs[page] > 1;
    }
  if (__syncthreads_or(bad)) return;
  const uint32_t words = (uint32_t)(p.page_bytes / (16 * kKvPageTokens));  // of a token
  const int64_t columns = (int64_t)p.H * words * (p.v_pool ? 2 : 1);
  for (int64_t c = threadIdx.x; c < columns; c += blockDim.x) {
    const int64_t head = c / words;
    const uint32_t w = (uint32_t)(c - head * words);
    uint8_t* pool = head < p.H ? p.k_pool : p.v_pool;
    const int* entries = p.table + ((int64_t)r * p.H + (head < p.H ? head : head - p.H)) * p.pph;
    auto word = [&](int pos) -> u32x4* {
      const int page = entries[pos / kKvPageTokens];
      if (page < 0 || page >= p.pool) return nullptr;
      return reinterpret_cast<u32x4*>(pool + page * p.page_bytes) + (uint32_t)(pos % kKvPageTokens) * words + w;
    };
    for (int j0 = 0; j0 < keep; j0 += kKeepTokens) {
      u32x4 x[kKeepTokens];
      u32x4* to[kKeepTokens];
#pragma unroll
      for (int u = 0; u < kKeepTokens; ++u) {
        to[u] = nullptr;
        if (j0 + u >= keep) continue;
        const int from = path[at + j0 + u];
        if (from == j0 + u) continue;
        const u32x4* src = word(base + from);
        if (src) {
          x[u] = *src;
          to[u] = word(base + j0 + u);
        }
      }
#pragma unroll
      for (int u = 0; u < kKeepTokens; ++u)
        if (to[u]) *to[u] = x[u];
    }
  }
  __syncthreads();  // (the entries have been read)
  const int left = pages_of(now, p.pph), gone = pages_of(len, p.pph) - left;
  for (int64_t x = threadIdx.x; x < (int64_t)gone * p.H; x += blockDim.x) {
    int* e = p.table + ((int64_t)r * p.H + x / gone) * p.pph + left + x % gone;
    if (*e >= 0 && *e < p.pool) atomicSub(&p.refs[*e], 1);
    *e = -1;
  }
  if (threadIdx.x == 0) p.lens[r] = now;
}

// The checks that every call shares; lays the workspace out (words, counted in `words`).
int pages_setup(const char* what, int op, int R, int H, int pph, int32_t* table, int32_t* lens, int32_t* refs,
                size_t pool_pages, int n, void* workspace, size_t workspace_bytes, PagesParams* p) {
  const std::string w(what);
  if (R < 1 || H < 1 || pph < 1 || n < 0) return fail(ASYM_EINVAL, w + ": R, H and pages_per_head must be >= 1, n >= 0");
  if (pph > (1 << 25)) return fail(ASYM_EUNSUPPORTED, w + ": more than 2^30 tokens a row");
  // (entries, and with them the pages that a call may need, are counted in 32 bits)
  if ((int64_t)H * pph > 0x7FFFFFFF || (int64_t)H * pph * R > 0x7FFFFFFF)
    return fail(ASYM_EUNSUPPORTED, w + ": the table has 2^31 entries or more");
  if (pool_pages < 1 || pool_pages > 0x7FFFFFFFu) return fail(ASYM_EINVAL, w + ": pool_pages must be in [1, 2^31)");
  if ((int64_t)n * H >= (1 << 24))  // (threads of a launch are counted in 32 bits)
    return fail(ASYM_EUNSUPPORTED, w + ": too many requests");
  if (!table || !lens || !refs) return fail(ASYM_EINVAL, w + ": null pointer");
  if (((uintptr_t)table | (uintptr_t)lens | (uintptr_t)refs) & 3u)
    return fail(ASYM_EINVAL, w + ": tables, lengths and counts must be 4-byte aligned");
  *p = PagesParams{};
  p->table = table; p->lens = lens; p->refs = refs;
  p->R = R; p->H = H; p->pph = pph; p->pool = (int)pool_pages; p->n = n;
  p->segs = (int)((pool_pages + kSeg - 1) / kSeg);
  if (op < 0) return ASYM_OK;  // (free: no workspace)
  size_t bytes = 0;
  const int rc = asym_kv_pages_workspace(op, R, H, pph, pool_pages, n, &bytes);
  if (rc != ASYM_OK) return rc;
  if (!workspace || workspace_bytes < bytes || ((uintptr_t)workspace & 15u))
    return fail(ASYM_EINVAL, w + ": the workspace must be 16-byte aligned and hold asym_kv_pages_workspace's bytes");
  int* at = static_cast<int*>(workspace);
  auto take = [&](size_t words) {
    int* x = at;
    at += words;
    return x;
  };
  p->head = take(kHeader);
  p->counts = take(p->segs);
  p->list = take(pool_pages);
  if (op == ASYM_KV_COMPACT) {
    p->holes = take(pool_pages);
    p->where = take(pool_pages);
  } else {
    p->first = take(n);
    p->flag = take(n);
    p->claim = take(R);
    if (op == ASYM_KV_FORK) {
      p->new_len = take(n);
      p->rows = take((size_t)n * H * pph);
    }
  }
  return ASYM_OK;
}

bool small_call(const PagesParams& p) { return p.pool <= kSmallThreads * kPer && p.n <= kSmallThreads; }

int pools_check(const char* what, const void* k_pool, const void* v_pool, size_t page_bytes) {
  const std::string w(what);
  if (!k_pool) return fail(ASYM_EINVAL, w + ": null pointer");
  if (((uintptr_t)k_pool | (uintptr_t)v_pool) & 15u) return fail(ASYM_EINVAL, w + ": pools must be 16-byte aligned");
  if (page_bytes < 16 || page_bytes % 16 || page_bytes > (1u << 30))
    return fail(ASYM_EINVAL, w + ": page_bytes must be a multiple of 16, at most 2^30");
  if (k_pool == v_pool) return fail(ASYM_EINVAL, w + ": one pool given twice (leave v_pool null)");
  return ASYM_OK;
}

}  // namespace
}  // namespace asym

using namespace asym;

extern "C" int asym_kv_pages_workspace(int op, int R, int H, int pages_per_head, size_t pool_pages, int n, size_t* bytes) {
  if (!bytes) return fail(ASYM_EINVAL, "kv pages workspace: null output");
  if (op != ASYM_KV_EXTEND && op != ASYM_KV_FORK && op != ASYM_KV_COMPACT)
    return fail(ASYM_EINVAL, "kv pages workspace: unknown operation");
  if (R < 1 || H < 1 || pages_per_head < 1 || n < 0 || pool_pages < 1 || pool_pages > 0x7FFFFFFFu)
    return fail(ASYM_EINVAL, "kv pages workspace: bad sizes");
  size_t words = kHeader + (pool_pages + kSeg - 1) / kSeg + pool_pages;
  if (op == ASYM_KV_COMPACT)
    words += 2 * pool_pages;
  else
    words += 2 * (size_t)n + R;
  if (op == ASYM_KV_FORK) words += (size_t)n + (size_t)n * H * pages_per_head;
  *bytes = words * sizeof(int);
  return ASYM_OK;
}

extern "C" int asym_kv_extend(int R, int H, int pages_per_head, int32_t* table, int32_t* lens, int32_t* refs,
                              size_t pool_pages, int n, const int32_t* rows, const int32_t* new_lens, int32_t* status,
                              void* workspace, size_t workspace_bytes, void* stream) {
  PagesParams p;
  const int rc = pages_setup("kv extend", ASYM_KV_EXTEND, R, H, pages_per_head, table, lens, refs, pool_pages, n, workspace,
                             workspace_bytes, &p);
  if (rc != ASYM_OK) return rc;
  if (n > 0 && (!rows || !new_lens)) return fail(ASYM_EINVAL, "kv extend: null pointer");
  if (((uintptr_t)rows | (uintptr_t)new_lens | (uintptr_t)status) & 3u)
    return fail(ASYM_EINVAL, "kv extend: rows, lengths and status must be 4-byte aligned");
  p.a = rows; p.b = new_lens; p.status = status;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (small_call(p)) {
    hipLaunchKernelGGL((pages_small<kExtend>), dim3(1), dim3(kSmallThreads), 0, s, p);
    ASYM_HIP(hipGetLastError());
    return ASYM_OK;
  }
  hipLaunchKernelGGL((pages_count<kExtend>), dim3(p.segs + 1), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL((pages_list<kExtend>), dim3(p.segs), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL(pages_extend, dim3(std::max(n, 1)), dim3(kThreads), 0, s, p);  // (status with no request too)
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}

extern "C" int asym_kv_fork(int R, int H, int pages_per_head, int32_t* table, int32_t* lens, int32_t* refs, void* k_pool,
                            void* v_pool, size_t page_bytes, size_t pool_pages, int n, const int32_t* src,
                            const int32_t* dst, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  PagesParams p;
  int rc = pages_setup("kv fork", ASYM_KV_FORK, R, H, pages_per_head, table, lens, refs, pool_pages, n, workspace,
                       workspace_bytes, &p);
  if (rc == ASYM_OK) rc = pools_check("kv fork", k_pool, v_pool, page_bytes);
  if (rc != ASYM_OK) return rc;
  if (n > 0 && (!src || !dst)) return fail(ASYM_EINVAL, "kv fork: null pointer");
  if (((uintptr_t)src | (uintptr_t)dst | (uintptr_t)status) & 3u)
    return fail(ASYM_EINVAL, "kv fork: sources, targets and status must be 4-byte aligned");
  p.a = src; p.b = dst; p.status = status;
  p.k_pool = static_cast<uint8_t*>(k_pool);
  p.v_pool = static_cast<uint8_t*>(v_pool);
  p.page_bytes = (int64_t)page_bytes;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (small_call(p)) {
    hipLaunchKernelGGL((pages_small<kFork>), dim3(1), dim3(kSmallThreads), 0, s, p);
  } else {
    hipLaunchKernelGGL((pages_count<kFork>), dim3(p.segs + 1), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL((pages_list<kFork>), dim3(p.segs), dim3(kThreads), 0, s, p);
  }
  hipLaunchKernelGGL(pages_fork, dim3(std::max(n * H, 1)), dim3(kThreads), 0, s, p);  // (status with no request too)
  if (n > 0) hipLaunchKernelGGL(pages_fork_rows, dim3(n), dim3(kThreads), 0, s, p);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}

extern "C" int asym_kv_free(int R, int H, int pages_per_head, int32_t* table, int32_t* lens, int32_t* refs,
                            size_t pool_pages, int n, const int32_t* rows, void* stream) {
  PagesParams p;
  const int rc = pages_setup("kv free", -1, R, H, pages_per_head, table, lens, refs, pool_pages, n, nullptr, 0, &p);
  if (rc != ASYM_OK) return rc;
  if (n == 0) return ASYM_OK;
  if (!rows || ((uintptr_t)rows & 3u)) return fail(ASYM_EINVAL, "kv free: rows must be given, 4-byte aligned");
  p.a = rows;
  hipLaunchKernelGGL(pages_free, dim3(n), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}

extern "C" int asym_kv_keep(int R, int H, int pages_per_head, int32_t* table, int32_t* lens, int32_t* refs, void* k_pool,
                            void* v_pool, size_t page_bytes, size_t pool_pages, int n, const int32_t* rows, int T,
                            const int32_t* cu, const int32_t* path, const int32_t* count, void* stream) {
  PagesParams p;
  int rc = pages_setup("kv keep", -1, R, H, pages_per_head, table, lens, refs, pool_pages, n, nullptr, 0, &p);
  if (rc == ASYM_OK) rc = pools_check("kv keep", k_pool, v_pool, page_bytes);
  if (rc != ASYM_OK) return rc;
  if (page_bytes % (16 * kKvPageTokens))
    return fail(ASYM_EUNSUPPORTED, "kv keep: pages must hold 32 tokens one after the other, of a multiple of 16 bytes each");
  if (T < 0) return fail(ASYM_EINVAL, "kv keep: T must be >= 0");
  if (n == 0) return ASYM_OK;
  if (!rows || !cu || !count || (T && !path)) return fail(ASYM_EINVAL, "kv keep: null pointer");
  if (((uintptr_t)rows | (uintptr_t)cu | (uintptr_t)path | (uintptr_t)count) & 3u)
    return fail(ASYM_EINVAL, "kv keep: rows, offsets, paths and counts must be 4-byte aligned");
  p.a = rows;
  p.k_pool = static_cast<uint8_t*>(k_pool);
  p.v_pool = static_cast<uint8_t*>(v_pool);
  p.page_bytes = (int64_t)page_bytes;
  // a thread a 16-byte word of a token, as far as a workgroup goes
  const int64_t columns = (int64_t)H * (int64_t)(page_bytes / (16 * kKvPageTokens)) * (v_pool ? 2 : 1);
  const unsigned threads = (unsigned)std::min<int64_t>((columns + 63) / 64 * 64, kSmallThreads);
  if ((int64_t)n * threads > 0xFFFFFFFFll)  // (threads of a launch are counted in 32 bits)
    return fail(ASYM_EUNSUPPORTED, "kv keep: too many requests for pages of this size");
  hipLaunchKernelGGL(pages_keep, dim3(n), dim3(threads), 0, static_cast<hipStream_t>(stream), p, T, cu, path, count);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}

extern "C" int asym_kv_compact(int R, int H, int pages_per_head, int32_t* table, int32_t* refs, void* k_pool, void* v_pool,
                               size_t page_bytes, size_t pool_pages, int32_t* status, void* workspace,
                               size_t workspace_bytes, void* stream) {
  PagesParams p;
  int32_t none = 0;
  int rc = pages_setup("kv compact", ASYM_KV_COMPACT, R, H, pages_per_head, table, &none, refs, pool_pages, 0, workspace,
                       workspace_bytes, &p);
  if (rc == ASYM_OK) rc = pools_check("kv compact", k_pool, v_pool, page_bytes);
  if (rc != ASYM_OK) return rc;
  if ((uintptr_t)status & 3u) return fail(ASYM_EINVAL, "kv compact: status must be 4-byte aligned");
  p.lens = nullptr;
  p.status = status;
  p.k_pool = static_cast<uint8_t*>(k_pool);
  p.v_pool = static_cast<uint8_t*>(v_pool);
  p.page_bytes = (int64_t)page_bytes;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t entries = (int64_t)R * H * pages_per_head;
  if (small_call(p)) {
    hipLaunchKernelGGL((pages_small<kCompact>), dim3(1), dim3(kSmallThreads), 0, s, p);
  } else {
    hipLaunchKernelGGL((pages_count<kCompact>), dim3(p.segs), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL((pages_list<kCompact>), dim3(p.segs), dim3(kThreads), 0, s, p);
  }
  const size_t chunks = pool_pages * (page_bytes / 16 * (v_pool ? 2 : 1)) / (kMoveWords * kThreads) + 1;
  hipLaunchKernelGGL(pages_move, dim3((unsigned)std::min<size_t>(chunks, 65536)), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL(pages_rename, dim3((unsigned)std::min<int64_t>((entries + kThreads - 1) / kThreads, 4096)),
                     dim3(kThreads), 0, s, p);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
