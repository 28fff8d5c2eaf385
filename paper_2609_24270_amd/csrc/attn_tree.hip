// Attention of a tree of drafted tokens over a 16-bit paged cache: a request's n nodes, which
// are the last n of its len tokens in the cache, against all that each of them sees:
//
//   O[i, h] = softmax_t(scale * <q[i, h], K[g, t]>) . V[g, t],  g = h / G, G = H_q / H_kv,
//
// over every token t before the nodes (t < base = len - n) and the nodes t = base + j whose
// bit j is set in node i's mask (without masks: j <= i, a chain; n = 1 is plain decoding with
// a length per request).
//
// A row is a (node, query head of the group) pair, node-major.  A workgroup of four or eight waves (tree_plan says when, and NQ)
// serves up to 16 NQ rows a wave (NQ 1 or 2) of one request and key/value head, and takes its tokens 64 at a time, two pages.  K and V
// come by LDS loads, each wave's part of the block, STAGES - 1 blocks ahead; per block a wave computes
//   S^T = K . Q^T   v_mfma_f32_16x16x32_bf16, Q in registers, K by ds_read_b128;
//   softmax         a row's 64 scores lie in four lanes; its running max is raised only when
//                   some row's grows by more than 2^8;
//   O^T += V^T . P^T  in the scores' registers, V^T by ds_read_b64_tr_b16.  The products take bf16, so a weight is the
//                   sum of two: itself rounded, and what that left of it, rounded (2^-16 of the weight are lost).
// Scores, max, sum and output are fp32, and rounded to bf16 once, at the end.  One barrier a block.
//
// The pages of the batch, request by request and head by head, are one list, cut into equal
// shares, one a workgroup, whatever the lengths (which only the device knows).  A segment is what a
// share has of one request and head.  Whole ones are written; of cut ones the unscaled output, max and sum go to
// the caller's workspace in fp32 and a second launch joins them in order.  Where the longest request is short
// for the number of segments, a share is a segment and one launch does it (tree_plan).
//
// Bound by HBM where the rows are few: 64 requests of one token behind up to 8000 (32 / 8 heads, 1.39 GB) take 224 us, 6.2
// TB/s.  32 trees of 24 nodes in the mean behind up to 8000 tokens (0.72 GB) take 177 us, 12 of them the joining: 4.1
// TB/s; matrix instructions take 38 % of the cycles and vector ones 42 %, one after the other within a wave.  8 trees of 64
// nodes in the mean behind up to 32768 tokens: 420 us (503 TFLOP/s of the definition's; the second part of the weights is half as
// many again), 793 thousand cycles at 1.9 GHz of 2.4 (the power cap), 40 % in matrix instructions and 44 % in vector ones.
// A unit with few rows costs its pages nearly as much as a full one: 8 trees of 64 nodes exactly 405 us, of 65 657, of 96
// 700 (200, 314 and 317 million busy cycles), and half of the trees above have such a second unit.
//
// The weights' second part costs 1 to 4 % where one block of rows is enough and up to a third where the matrix cores are busy
// (32 trees of 24 160 -> 177 us, 8 of 64 320 -> 420); with weights of one bf16 value the error against 64 bits was 2.2e-3, and is
// 1.65e-3, the output's rounding.
//
// Each wave with its own pages, K fragments straight from memory and no barrier, took twice as long on trees (348 us
// for the 32 above): every wave of a unit loaded every page.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "kv_fp4.h"
#include "read_policy.h"

namespace asym {
namespace {

constexpr int kRowBytes = kKvD * 2;
constexpr int kPageBytes = kKvPageTokens * kRowBytes;
constexpr int kJoinWaves = 4;  // of the joining launch's workgroups
constexpr int kLonger = 8;     // pages

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

struct TreeParams {
  const uint16_t* q;
  int64_t q_tok, q_head;         // strides, values
  const uint8_t *k_pool, *v_pool;
  const int *k_pages, *v_pages;  // [B][Hkv][pph]
  const int *cu, *lens;
  const uint64_t* mask;          // [T][words], nullable
  int words;
  uint16_t* o;                   // [T][Hq][128]
  float* lse;                    // [T][Hq], nullable
  float* part_o;                 // [shares][2][rows][128]
  float* part_ml;                // [shares][2][rows][2]: max (of the raw scores), sum
  int2* cut;                     // null: nothing is cut, a workgroup has a segment.  Else per (unit, key/value head), a unit being the rows of a request that one workgroup
                                 // serves: of one that was cut, 2 (its first share) + (1: that share's last piece),
                                 // its last share; -1 of one that was not
  int B, Hq, Hkv, G, T, S, pph, pool_pages;
  int rows;                      // of a workgroup: 16 NQ a wave
  int shares, least;             // a share has `least` pages;
  bool fit;                      // or the batch's pages over the shares, if they are more, or a few more than that
  float c, scale;                // |scale| * log2(e), |scale|
  uint32_t q_flip;
};

// f over this lane and those 16, 32 and 48 on: the four that share a row
template <class F>
__device__ __forceinline__ float over_quarters(float x, F f) {
  uint32_t u = __float_as_uint(x);
  auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = f(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
  u = __float_as_uint(x);
  sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return f(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// Request b: its first row of q, nodes, tokens, the units that its rows make and its pages
struct Request {
  int first, n, len, units, pages;
};
__device__ __forceinline__ int units_of(const TreeParams& p, int n) { return (n * p.G + p.rows - 1) / p.rows; }  // (rows of the call: fewer than 2^26)
__device__ __forceinline__ Request request(const TreeParams& p, int b) {
  Request r;
  packed_rows(p.cu, b, p.T, r.first, r.n);
  r.len = min(max(p.lens[b], 0), p.S);
  r.units = units_of(p, r.n);
  r.pages = (r.len + kKvPageTokens - 1) / kKvPageTokens;
  if (!p.cut) r.pages = max(r.pages, 1);  // (no other launch writes the rows that see nothing)
  return r;
}
// The unit's place in `cut` (a request's units follow the rows before it, one more a request)
__device__ __forceinline__ int unit_id(const TreeParams& p, int b, int first, int unit) {
  return first * p.G / p.rows + b + unit;  // (rows of the call: fewer than 2^26)
}

// Where the requests' pages lie in the list, 64 requests at a time: lane l has request base + l.  A segment of the list is a
// unit's pages for one head, rounded up to a multiple of `pad`.
struct Batch {
  int base, pad;
  int upto;  // the list's places (of one head) up to and with the request
  bool falls;  // some offset lies below the one before: requests would have rows in common
  Request r;
  __device__ __forceinline__ int padded(int pages) const { return (pages + pad - 1) / pad * pad; }
  __device__ __forceinline__ void load(const TreeParams& p, int from, int before, int lane) {
    base = from;
    r = Request{};
    falls = false;
    if (from + lane < p.B) {
      r = request(p, from + lane);
      falls = p.cu[from + lane + 1] < p.cu[from + lane];
    }
    place(before);
  }
  __device__ __forceinline__ void place(int before) { upto = before + wave_scan_add(r.units * padded(r.pages)); }
  __device__ __forceinline__ int end() const { return __builtin_amdgcn_readlane(upto, 63); }
};

// 16-byte chunk c of V's row t lies at chunk c ^ swz(t), so that the rows that one transposing read takes
// together (8 rows, two chunks of each) lie on different ones of the 64 banks.
__device__ __forceinline__ int swz(int row) { return (row & 7) << 1; }

// A lane's place of V^T operand g: channels of group g of 16, tokens 4 q + n / 4
__device__ __forceinline__ uint32_t v_place(int g, int lane) {
  const int n = lane & 15, q = lane >> 4;
  const int row = 4 * q + (n >> 2), chunk = 2 * g + ((n & 3) >> 1);
  return (uint32_t)(row * kRowBytes + ((chunk ^ swz(row)) << 4) + ((n & 1) << 3));
}
__device__ __forceinline__ bf16x8 v_frag(const lds_byte* vt, uint32_t at) {
  union {
    s16x4 s[2];
    bf16x8 b;
  } u;
#pragma unroll
  for (int part = 0; part < 2; ++part)
    u.s[part] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + at + 16 * part * kRowBytes));
  return u.b;
}
// Which of tokens 32 page .. + 31 node i sees, a bit each (node 0 is token `base`, which may be negative)
__device__ __forceinline__ uint32_t seen_bits(const TreeParams& p, const uint64_t* words, int i, int n, int base, int page) {
  const int j0 = page * kKvPageTokens - base;  // the node at the page's first token
  if (j0 <= -kKvPageTokens) return 0xFFFFFFFFu;
  auto up_to = [&](int k) {  // the bits below k
    return k <= 0 ? 0u : k >= 32 ? 0xFFFFFFFFu : (1u << k) - 1u;
  };
  const uint32_t exist = up_to(n - j0), prefix = up_to(-j0);
  if (!words) return prefix | (up_to(i + 1 - j0) & exist);
  auto word = [&](int w) { return w < p.words ? words[w] : 0ull; };
  uint64_t bits;
  if (j0 < 0) {
    bits = word(0) << -j0;
  } else {
    const int off = j0 & 63;
    bits = word(j0 >> 6) >> off;
    if (off > 32) bits |= word((j0 >> 6) + 1) << (64 - off);
  }
  return prefix | ((uint32_t)bits & exist);
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kTokens = 2 * kKvPageTokens;         // of a block
constexpr int kTileBytes = kTokens * kRowBytes;    // of its keys, or its values
constexpr int NT = kTokens / 16, NK = kTokens / 32;  // 16-token and 32-token steps

// (for keys: 16 rows, one chunk of each, are read together)
__device__ __forceinline__ int swz_k(int row) { return row & 15; }

// 1 KiB from lane addresses voff to LDS bytes dst .. dst + 1023, in lane order (the load takes dst from M0, whose write
// needs a wait state before it, which the compiler does not add here)
template <int POLICY>
__device__ __forceinline__ void lds_load_1k(uint32_t dst, i32x4 rs, uint32_t voff) {
  if constexpr (POLICY)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(dst), "v"(voff), "s"(rs)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(voff), "s"(rs)
                 : "memory", "m0");
}
__device__ __forceinline__ i32x4 page_words(const uint8_t* pool, int page, int pool_pages) {
  const bool in = page >= 0 && page < pool_pages;
  const uint64_t a = (uint64_t)pool + (uint64_t)(uint32_t)(in ? page : 0) * kPageBytes;
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
  r[2] = __builtin_amdgcn_readfirstlane(in ? kPageBytes : 0);  // (a page that is none reads zeros)
  r[3] = 0x00020000;
  return r;
}

// f, N times
template <int N, class F>
__device__ __forceinline__ void steps(F f) {
  if constexpr (N > 0) {
    f();
    steps<N - 1>(f);
  }
}

// The kernel's arguments, read again (scalar loads): what a phase needs of them does not stay in registers through the others
__device__ __forceinline__ TreeParams arguments() {
  auto at = (const __attribute__((address_space(4))) TreeParams*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const TreeParams*)at;
}

template <int NW, int STAGES, int NQ, int POLICY>
__global__ void __launch_bounds__(64 * NW, 2) attn_tree_kernel(TreeParams args) {
  constexpr int WR = 16 * NQ;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGES * kTileBytes];  // K tiles, then V tiles
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, q4 = lane >> 4;
  const int w = blockIdx.x;

  // A segment: request b, unit, head hk, its pages pg .. pg + count - 1
  struct Segment {
    int b, first, nodes, len, pages, unit, hk, pg, count;
    int end;  // in the list
  } x;
  const TreeParams p0 = arguments();
  Batch bt;
  int share = p0.least, f1 = 0;  // f1: the share's end in the list
  if (p0.cut) {
    bt.pad = 1;
    bt.load(p0, 0, 0, lane);
    int total = bt.end();
    bool falls = bt.falls;
    int more = 0;
#pragma unroll 4
    for (int b = 64 + lane; b < p0.B; b += 64) {
      const Request r = request(p0, b);
      more += r.units * r.pages;
      falls |= p0.cu[b + 1] < p0.cu[b];
    }
    if (__any(falls)) return;  // (the joining launch too)
    if (p0.B > 64) total += wave_sum(more);
    total *= p0.Hkv;
    if (p0.fit) share = max(share, (total + p0.shares - 1) / p0.shares);
    // A share that goes on in a second segment costs as much as a few pages more would; where shares of up to kLonger more
    // pages suffice with every segment beginning a share of its own, they do: a tree of 8 nodes behind 777 tokens 14.1 ->
    // 9.7 us, 4 requests of a token with 8 / 1 heads behind up to 30000 25.9 -> 22.4 (in a graph).
    if (p0.fit && p0.B <= 64)
      for (int longer = (share + 1) & ~1; longer <= share + kLonger; longer += 2)
        if (wave_sum(bt.r.units * ((bt.r.pages + longer - 1) / longer)) * p0.Hkv <= p0.shares) {
          share = bt.pad = longer;
          bt.place(0);
          total = bt.end() * p0.Hkv;
          break;
        }
    if ((int64_t)w * share >= total) return;
    f1 = min((w + 1) * share, total);
  } else {
    // Whole segments, unit by unit and head by head: the workgroup's unit among those of requests lo .. hi - 1, a 64th of them
    // a lane, then of that lane's, until it is one.  1024 requests of 4 nodes behind up to 200 tokens 219 us (by the list 73 more).
    x.unit = w / p0.Hkv;
    x.hk = w - x.unit * p0.Hkv;
    int lo = 0, hi = p0.B, per;
    do {
      per = (hi - lo + 63) / 64;
      int mine = 0;
      bool falls = false;
#pragma unroll 4
      for (int k = 0; k < per; ++k) {
        const int b = lo + lane * per + k;
        if (b < hi) {
          int first, n;
          packed_rows(p0.cu, b, p0.T, first, n);
          mine += units_of(p0, n);
          falls |= p0.cu[b + 1] < p0.cu[b];
        }
      }
      if (__any(falls)) return;
      const int upto = wave_scan_add(mine);
      const unsigned long long above = __ballot(upto > x.unit);
      if (!above) return;
      const int at = __builtin_ctzll(above);
      x.unit -= __builtin_amdgcn_readlane(upto - mine, at);
      lo += at * per;
      hi = min(lo + per, hi);
    } while (per > 1);
    const Request r = request(p0, lo);  // (the same for all lanes)
    x.b = lo;
    x.first = __builtin_amdgcn_readfirstlane(r.first);
    x.nodes = __builtin_amdgcn_readfirstlane(r.n);
    x.len = __builtin_amdgcn_readfirstlane(r.len);
    x.pages = x.count = __builtin_amdgcn_readfirstlane(r.pages);
    x.pg = x.end = 0;
  }

  const uint32_t lds0 = (uint32_t)(size_t)lds;
  uint32_t ka[4], va[8];  // a lane's places in the tiles: key n of 16, chunks 4 c + q; V^T operand g
#pragma unroll
  for (int c = 0; c < 4; ++c) ka[c] = (uint32_t)(n * kRowBytes + (((4 * c + q4) ^ swz_k(n)) << 4));
#pragma unroll
  for (int g = 0; g < 8; ++g) va[g] = v_place(g, lane);
  // 1 KiB is 4 rows of a tile, 16 KiB of keys and 16 of values a block: the wave's pieces lie in one of its two pages
  constexpr int PIECES = kTileBytes / 1024 / NW;
  const int half = wave * PIECES / 8;
  uint32_t ko[PIECES], vo[PIECES];  // from the page's start
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int r = 4 * (wave * PIECES + i) + (lane >> 4);
    ko[i] = (uint32_t)((r & 31) * kRowBytes + (((lane & 15) ^ swz_k(r)) << 4));
    vo[i] = (uint32_t)((r & 31) * kRowBytes + (((lane & 15) ^ swz(r)) << 4));
  }
  auto k_tile = [&](int j) { return (lds_byte*)lds + (j % STAGES) * kTileBytes; };
  auto v_tile = [&](int j) { return (lds_byte*)lds + (STAGES + j % STAGES) * kTileBytes; };

  auto find = [&](const TreeParams& p, int f) {
    while (bt.end() * p.Hkv <= f) bt.load(p, bt.base + 64, bt.end(), lane);
    const int at = __builtin_ctzll(__ballot(bt.upto * p.Hkv > f));
    Segment x;
    x.b = bt.base + at;
    x.first = __builtin_amdgcn_readlane(bt.r.first, at);
    x.nodes = __builtin_amdgcn_readlane(bt.r.n, at);
    x.len = __builtin_amdgcn_readlane(bt.r.len, at);
    x.pages = __builtin_amdgcn_readlane(bt.r.pages, at);
    const int units = __builtin_amdgcn_readlane(bt.r.units, at), places = bt.padded(x.pages);
    const int in = f - (__builtin_amdgcn_readlane(bt.upto, at) - units * places) * p.Hkv;
    x.unit = in / (p.Hkv * places);
    x.hk = (in - x.unit * p.Hkv * places) / places;
    x.pg = in % places;
    x.count = min(x.pages - x.pg, f1 - f);
    x.end = f - x.pg + places;
    return x;
  };
  // The numbers of the wave's pages of blocks j .. j + 63 of a segment, one a lane
  auto numbers = [&](const TreeParams& p, const Segment& x, int j, int& k, int& v) {
    const size_t entry = ((size_t)x.b * p.Hkv + x.hk) * p.pph + x.pg + half;
    k = v = -1;
    if (2 * (j + lane) + half < x.count) {
      k = p.k_pages[entry + 2 * (size_t)(j + lane)];
      v = p.v_pages[entry + 2 * (size_t)(j + lane)];
    }
  };
  int kpg, vpg, kpg2, vpg2;  // of blocks chunk .. chunk + 63, and of the next 64
  // (waited for here and not, by the compiler, at every use in the loops below, the tiles' loads with them)
  auto settle = [&] { asm volatile("" : "+v"(kpg), "+v"(vpg), "+v"(kpg2), "+v"(vpg2)); };
  int chunk;
  auto load = [&](const TreeParams& p, int j) {  // block j, chunk <= j < chunk + 128
    const int e = j & 63;
    const bool next = j >= chunk + 64;
    const int kn = __builtin_amdgcn_readlane(kpg, e), kn2 = __builtin_amdgcn_readlane(kpg2, e);
    const int vn = __builtin_amdgcn_readlane(vpg, e), vn2 = __builtin_amdgcn_readlane(vpg2, e);
    const i32x4 rk = page_words(p.k_pool, next ? kn2 : kn, p.pool_pages);
    const i32x4 rv = page_words(p.v_pool, next ? vn2 : vn, p.pool_pages);
    const uint32_t dst = lds0 + (uint32_t)(j % STAGES) * kTileBytes + (uint32_t)(wave * PIECES) * 1024;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) lds_load_1k<POLICY>(dst + i * 1024, rk, ko[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) lds_load_1k<POLICY>(dst + STAGES * kTileBytes + i * 1024, rv, vo[i]);
  };
  // A segment's first blocks, and the wave's rows of q, on their way (the tiles are free, its first pages' numbers are there)
  u32x4 qf[NQ][4];
  auto begin = [&](const TreeParams& p, const Segment& x) {
    settle();
    chunk = 0;
    const int nblk = (x.count + 1) / 2;
#pragma unroll
    for (int j = 0; j < STAGES - 1; ++j)
      if (j < nblk) load(p, j);
    const int row0 = x.unit * p.rows, rows = min(x.nodes * p.G - row0, p.rows);
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
      const int row = row0 + min(wave * WR + 16 * k + n, rows - 1);
      const int tok = row / p.G, g = row - tok * p.G;
      const uint16_t* qr = p.q + (int64_t)(x.first + tok) * p.q_tok + ((int64_t)x.hk * p.G + g) * p.q_head + 8 * q4;
#pragma unroll
      for (int c = 0; c < 4; ++c) qf[k][c] = *reinterpret_cast<const u32x4*>(qr + 32 * c);
    }
  };

  if (p0.cut) x = find(p0, w * share);
  numbers(p0, x, 0, kpg, vpg);
  numbers(p0, x, 64, kpg2, vpg2);
  begin(p0, x);
  for (bool start = true;; start = false) {
    const TreeParams p = arguments();
    const int count = x.count, nblk = (count + 1) / 2;
    const int row0 = x.unit * p.rows, rows = min(x.nodes * p.G - row0, p.rows);  // of the unit
    const bool work = wave * WR < rows;
    const int base = x.len - x.nodes;
    // blocks of two pages of the segment that every row sees whole
    const int nfull = max(0, min((base < 0 ? 0 : base / kKvPageTokens) - x.pg, count) / 2);
    auto turn_chunk = [&](int j) {  // before block j: the next 64 blocks' pages
      if (j < chunk + 64) return;
      chunk += 64;
      kpg = kpg2;
      vpg = vpg2;
      const TreeParams turn = arguments();
      numbers(turn, x, chunk + 64, kpg2, vpg2);
      settle();
    };
    // this wave's loads of block j, behind which those of STAGES - 2 are on their way, and with them everyone's
    auto arrived = [&](int j) {
      if (j + STAGES - 2 < nblk)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * 2 * PIECES) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (j + STAGES - 1 < nblk) load(p, j + STAGES - 1);
    };
#pragma unroll
    for (int k = 0; k < NQ; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[k][c][e] ^= p.q_flip;
        asm volatile("" : "+v"(qf[k][c]));  // (waited for here, as the numbers)
      }
    // the next segment's first numbers, for its loads to begin when this one's are done
    int kn[2], vn[2];
    if (x.end < f1) {
      const Segment next = find(p, x.end);
      numbers(p, next, 0, kn[0], vn[0]);
      numbers(p, next, 64, kn[1], vn[1]);
    }
    const float c = p.c;
    f32x4 o[NQ][8], s[NQ][NT];
    bf16x8 pf[NQ][NK], pr[NQ][NK];  // the weights rounded to bf16, and what that left of them
    float m[NQ], l[NQ];
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
      m[k] = -INFINITY;
      l[k] = 0.f;
#pragma unroll
      for (int g = 0; g < 8; ++g) o[k][g] = f32x4{};
    }
    auto scores = [&](int j) {
      const lds_byte* kt = k_tile(j);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const bf16x8 x = *(const __attribute__((address_space(3))) bf16x8*)(kt + ka[c] + t * 16 * kRowBytes);
#pragma unroll
          for (int k = 0; k < NQ; ++k)
            s[k][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, qf[k][c]), c ? s[k][t] : f32x4{}, 0, 0, 0);
        }
    };
    auto raise = [&] {
      bool up = false;
      float top[NQ];
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        float x = fmaxf(fmaxf(s[k][0][0], s[k][0][1]), s[k][0][2]);
#pragma unroll
        for (int i = 3; i + 1 < 4 * NT; i += 2) x = fmaxf(fmaxf(x, s[k][i >> 2][i & 3]), s[k][(i + 1) >> 2][(i + 1) & 3]);
        x = fmaxf(x, s[k][NT - 1][3]);
        top[k] = over_quarters(x, [](float x, float y) { return fmaxf(x, y); });
        up |= (top[k] - m[k]) * c > 8.f;  // (a first finite max: inf; NaN never)
      }
      if (__any(up)) {
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
          const float m_new = fmaxf(m[k], top[k]);
          const float alpha = __builtin_amdgcn_exp2f((m[k] - (m_new == -INFINITY ? 0.f : m_new)) * c);
          l[k] *= alpha;
#pragma unroll
          for (int g = 0; g < 8; ++g) o[k][g] *= alpha;
          m[k] = m_new;
        }
      }
    };
    // What a pair's rounding left is e - (y0, y1) . (1, 0) and e - (y0, y1) . (0, 1), one instruction each (exact: the difference
    // has 16 bits at most).  The factors are kept in registers: for a constant (-1, 0) the compiler writes the inline constant
    // -1.0, which gave other differences.
    uint32_t minus[2] = {0xBF80u, 0xBF800000u};
    asm volatile("" : "+s"(minus[0]), "+s"(minus[1]));
    auto weights = [&](int ks) {
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        const float ms = m[k] == -INFINITY ? 0.f : m[k];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          // (the difference first: scores of the type's lowest values times c would be infinite; one instruction for both
          // took 4 % fewer cycles)
          const float e0 = __builtin_amdgcn_exp2f((s[k][2 * ks + (j >> 2)][j & 3] - ms) * c);
          const float e1 = __builtin_amdgcn_exp2f((s[k][2 * ks + (j >> 2)][(j & 3) + 1] - ms) * c);
          l[k] += e0;
          l[k] += e1;
          const bf16x2 y = {(__bf16)e0, (__bf16)e1};
          pf[k][ks][j] = y[0];
          pf[k][ks][j + 1] = y[1];
          pr[k][ks][j] = (__bf16)__builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, minus[0]), e0, false);
          pr[k][ks][j + 1] = (__bf16)__builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, minus[1]), e1, false);
        }
      }
    };
    // (The order of a block's instructions: operands are read from LDS a few ahead of the products that take them.  Each of these
    // takes the named number of instructions of a kind: 8 products, 0x100 reads; each: products of an operand.)
    auto pace = [](auto reads, auto ahead, auto total, auto each) {
      __builtin_amdgcn_sched_group_barrier(0x100, decltype(reads)::value * decltype(ahead)::value, 0);
      steps<decltype(total)::value - decltype(ahead)::value>([] {
        __builtin_amdgcn_sched_group_barrier(8, decltype(each)::value, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, decltype(reads)::value, 0);
      });
      __builtin_amdgcn_sched_group_barrier(8, decltype(each)::value * decltype(ahead)::value, 0);
    };
    auto v_op = [&](const lds_byte* vt, int g, int ks) { return v_frag(vt, va[g] + (uint32_t)(32 * ks * kRowBytes)); };
    auto add_pv = [&](int j) {
      const lds_byte* vt = v_tile(j);
#pragma unroll
      for (int ks = 0; ks < NK; ++ks)
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const bf16x8 x = v_op(vt, g, ks);
#pragma unroll
          for (int k = 0; k < NQ; ++k) o[k][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pr[k][ks], o[k][g], 0, 0, 0);
#pragma unroll
          for (int k = 0; k < NQ; ++k) o[k][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pf[k][ks], o[k][g], 0, 0, 0);
        }
    };

    for (int j0 = 0; j0 < nfull; j0 += 64) {
      turn_chunk(j0);
      const int j1 = min(j0 + 64, nfull);
      for (int j = j0; j < j1; ++j) {
        arrived(j);
        if (work) {
          // (the waves in step with each other otherwise: one that is at it goes on before the others)
          __builtin_amdgcn_s_setprio(1);
          scores(j);
          pace(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{}, std::integral_constant<int, 4 * NT>{}, std::integral_constant<int, NQ>{});
          raise();
          weights(0);
          weights(1);
          add_pv(j);
          pace(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{}, std::integral_constant<int, 8 * NK>{}, std::integral_constant<int, 2 * NQ>{});
          __builtin_amdgcn_s_setprio(0);
        }
      }
    }
    // An infinity among the values times a weight's second part, which may be 0 or negative, is NaN or has the wrong sign, and
    // NaN in the sum.  Where a sum is NaN and its weights are not, what the values of its channel hold decides.
    if (work && nfull > 0) {
      f32x4 all[NQ];
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        all[k] = o[k][0];
#pragma unroll
        for (int g = 1; g < 8; ++g) all[k] += o[k][g];
      }
      bool odd = false;
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        const float y = (all[k][0] + all[k][1]) + (all[k][2] + all[k][3]), lt = over_quarters(l[k], [](float a, float b) { return a + b; });
        odd |= y != y && lt == lt;
      }
      if (__any(odd)) {
        const TreeParams at = arguments();
        const int* entries = at.v_pages + ((size_t)x.b * at.Hkv + x.hk) * at.pph + x.pg;
        uint32_t none = 0, up = 0, down = 0;  // NaN, infinity, minus infinity: bit 4 g + r, channel 16 g + 4 q4 + r
        for (int t = n; t < kTokens * nfull; t += 16) {
          const int page = entries[t / kKvPageTokens];
          if (page < 0 || page >= at.pool_pages) continue;
          const uint8_t* row = at.v_pool + (int64_t)page * kPageBytes + t % kKvPageTokens * kRowBytes + 8 * q4;
#pragma unroll 1
          for (int g = 0; g < 8; ++g) {
            const s16x4 y = *reinterpret_cast<const s16x4*>(row + 32 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const uint32_t u = (uint16_t)y[r], bit = 1u << (4 * g + r);
              if ((u & 0x7FFFu) > 0x7F80u) none |= bit;
              if (u == 0x7F80u) up |= bit;
              if (u == 0xFF80u) down |= bit;
            }
          }
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
          none |= (uint32_t)__shfl_xor((int)none, d);
          up |= (uint32_t)__shfl_xor((int)up, d);
          down |= (uint32_t)__shfl_xor((int)down, d);
        }
        const uint32_t one = (up ^ down) & ~none;  // (infinities of one sign)
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t bit = 1u << (4 * g + r);
            const float y = up & bit ? INFINITY : -INFINITY;
#pragma unroll
            for (int k = 0; k < NQ; ++k)
              if (o[k][g][r] != o[k][g][r] && (one & bit)) o[k][g][r] = y;
          }
        }
      }
    }
    const TreeParams edge = arguments();
    // Blocks that hold nodes, end behind the tokens or with the segment: what a row does not see has weight 0, which an
    // infinity or NaN among the values would make NaN.  Where the block has any, they are taken out of V, and each row's
    // seen ones added to its output by a product of its own: weights 1, and for a value 1 (infinity), 128 (minus infinity) or
    // 16384 (NaN), whole numbers whose sums over 64 tokens tell how many there are of each.  They take the keys' place.
    for (int j = nfull; j < nblk; ++j) {
      // (what depends on the lane is computed here again: kept through the loop above, it would take registers there)
      int tid = (int)threadIdx.x;
      asm volatile("" : "+v"(tid));
      const int n = tid & 15, q4 = (tid >> 4) & 3;
      uint32_t seen[NQ][2];
      if (work)
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
          const int i = (row0 + min(wave * WR + 16 * k + n, rows - 1)) / edge.G;
          const uint64_t* words = edge.mask ? edge.mask + (int64_t)(x.first + i) * edge.words : nullptr;
#pragma unroll
          for (int h = 0; h < 2; ++h) seen[k][h] = 2 * j + h < count ? seen_bits(edge, words, i, x.nodes, base, x.pg + 2 * j + h) : 0u;
        }
      turn_chunk(j);
      arrived(j);
      auto each_word = [&](auto f) {  // the thread's words of the V tile
#pragma unroll
        for (int i = 0; i < kTileBytes / 16 / (64 * NW); ++i) {
          const uint32_t at = (uint32_t)(i * 64 * NW + tid) * 16;
          f(at, *(lds_u32x4*)(v_tile(j) + at));
        }
      };
      uint32_t bad = 0;
      each_word([&](uint32_t, u32x4 y) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (y[e] & 0x7F807F80u) + 0x00800080u;  // an exponent of all ones carries
      });
      const bool guard = __syncthreads_or((bad & 0x80008000u) != 0);
      if (work) {
        scores(j);
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (!((seen[k][t >> 1] >> (16 * (t & 1) + 4 * q4 + r)) & 1)) s[k][t][r] = -INFINITY;
        raise();
        weights(0);
        weights(1);
      }
      if (guard) {
        __syncthreads();  // (the K tile has been read)
        each_word([&](uint32_t at, u32x4 y) {
          u32x4 fin, code;
#pragma unroll
          for (int e = 0; e < 4; ++e) {  // two values a word
            const uint32_t mask = ((((y[e] & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xFFFFu;
            auto kind = [](uint32_t u) { return (u & 0x7Fu) ? 0x4680u : (u & 0x8000u) ? 0x4300u : 0x3F80u; };
            fin[e] = y[e] & ~mask;
            code[e] = (kind(y[e] & 0xFFFFu) | (kind(y[e] >> 16) << 16)) & mask;
          }
          *(lds_u32x4*)(v_tile(j) + at) = fin;
          *(lds_u32x4*)(k_tile(j) + at) = code;
        });
        __syncthreads();
        if (work) {
#pragma unroll
          for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int g = 0; g < 8; ++g) {
              __builtin_amdgcn_sched_barrier(0);  // (one product's registers at a time)
              f32x4 y = {};
#pragma unroll
              for (int ks = 0; ks < NK; ++ks) {
                u32x4 vis;
                const uint32_t bits = seen[k][ks] >> (4 * q4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int i = 16 * (e >> 1) + 2 * (e & 1);
                  vis[e] = (((bits >> i) & 1) ? 0x3F80u : 0u) | (((bits >> (i + 1)) & 1) ? 0x3F800000u : 0u);
                }
                y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_op(k_tile(j), g, ks), __builtin_bit_cast(bf16x8, vis), y, 0, 0, 0);
              }
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int c = (int)y[r];
                o[k][g][r] += ((c & 127) ? INFINITY : 0.f) + (((c >> 7) & 127) ? -INFINITY : 0.f) + (c >= 16384 ? NAN : 0.f);
              }
            }
        }
      }
      if (work) add_pv(j);
    }

    const TreeParams last = arguments();
    // the next segment's loads, before this one's results
    Segment next = x;
    if (x.end < f1) {
      next = find(last, x.end);
      kpg = kn[0], vpg = vn[0], kpg2 = kn[1], vpg2 = vn[1];
      __syncthreads();  // (the tiles have been read)
      begin(last, next);
    }
    const bool whole = count == x.pages;
    const size_t piece = ((size_t)w * 2 + (start ? 0 : 1)) * last.rows;
    if (work) {
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        const float lt = over_quarters(l[k], [](float a, float b) { return a + b; });
        const int in_unit = wave * WR + 16 * k + n;
        const bool on = in_unit < rows;
        if (!whole) {  // the unscaled output, max and sum to the joining launch
          if (on) {
            float* po = last.part_o + (piece + in_unit) * kKvD + 4 * q4;
#pragma unroll
            for (int g = 0; g < 8; ++g) *reinterpret_cast<f32x4*>(po + 16 * g) = o[k][g];
            if (q4 == 0) *reinterpret_cast<float2*>(last.part_ml + (piece + in_unit) * 2) = float2{m[k], lt};
          }
          continue;
        }
        // a lane has 4 of every 16 channels of a row; two groups of them, exchanged between the quarters, make 16 bytes
        const float inv = lt > 0.f ? 1.f / lt : (lt == 0.f ? 0.f : lt);  // (NaN stays)
        const int row = row0 + min(in_unit, rows - 1), tok = row / last.G;
        const int64_t out = (int64_t)(x.first + tok) * last.Hq + x.hk * last.G + (row - tok * last.G);
#pragma unroll
        for (int g = 0; g < 8; g += 2) {
          uint32_t u[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x4& y = o[k][g + (e >> 1)];
            const bf16x2 z = {(__bf16)(y[2 * (e & 1)] * inv), (__bf16)(y[2 * (e & 1) + 1] * inv)};
            u[e] = __builtin_bit_cast(uint32_t, z);
          }
          const auto y = __builtin_amdgcn_permlane16_swap(u[0], u[2], false, false);
          const auto z = __builtin_amdgcn_permlane16_swap(u[1], u[3], false, false);
          // quarter 0: channels 0 .. 7 of group g, 1: 0 .. 7 of group g + 1, 2: 8 .. 15 of g, 3: of g + 1
          if (on) *reinterpret_cast<u32x4*>(last.o + out * kKvD + 16 * (g + (q4 & 1)) + 8 * (q4 >> 1)) = u32x4{y[0], z[0], y[1], z[1]};
        }
        if (last.lse && on && q4 == 0) last.lse[out] = lt == 0.f ? -INFINITY : m[k] * last.scale + __logf(lt);
      }
    }
    if (x.pg == 0 && threadIdx.x == 0 && last.cut)
      last.cut[unit_id(last, x.b, x.first, x.unit) * last.Hkv + x.hk] =
          whole ? int2{-1, 0} : int2{2 * w + (start ? 0 : 1), (x.end - 1) / share};
    if (x.end >= f1) return;
    x = next;
  }
}

// The joining launch: a wave has kJoinHeads query heads of a token, or, where rows are few and have many pieces (SPLIT), a
// workgroup's waves share one.  Rows of a request without tokens are written, those that were cut are joined in the order
// of the shares (SPLIT: each wave's every kJoinWaves-th piece, then the waves), the first kJoinPieces of each loaded at once.
// us for 32 trees of 24 nodes behind up to 8000 tokens and for 8 of 64 behind up to 32768 (the launch alone), at 2 heads a wave and 2, 3, 4, 5,
// 6 and 8 pieces: 18.3 14.4 11.9 12.2 12.5 13.0, 14.0 13.8 11.2 8.7 9.0 11.6; 4 heads and 4 pieces 12.1 14.7; one head and 6 14.4 10.6.
constexpr int kJoinHeads = 2, kJoinPieces = 5;
template <bool SPLIT>
__global__ void __launch_bounds__(64 * kJoinWaves) attn_tree_join(TreeParams p) {
  constexpr int HEADS = SPLIT ? 1 : kJoinHeads, STEP = SPLIT ? kJoinWaves : 1;
  __shared__ float red[SPLIT ? kJoinWaves : 1][kKvD], red_ml[SPLIT ? kJoinWaves : 1][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (p.Hq + HEADS - 1) / HEADS, id = SPLIT ? (int)blockIdx.x : (int)blockIdx.x * kJoinWaves + wave;
  if (id >= p.T * groups) return;
  const int tok = id / groups, h0 = (id - tok * groups) * HEADS, sub = SPLIT ? wave : 0;
  int b = 0;  // requests that end at or before the token
  bool falls = false;
  for (int j = 0; j < p.B; j += 64) {
    const int at = min(j + lane, p.B - 1), end = p.cu[at + 1];
    falls |= end < p.cu[at];
    const bool before = j + lane < p.B && min(max(end, 0), p.T) <= tok;
    b += __popcll(__ballot(before));
  }
  if (b >= p.B || __any(falls)) return;
  const Request r = request(p, b);
  if (tok < r.first || tok >= r.first + r.n) return;
  const int64_t out0 = (int64_t)tok * p.Hq + h0;
  if (r.pages == 0) {
    for (int k = 0; k < HEADS && h0 + k < p.Hq && sub == 0; ++k) {
      *reinterpret_cast<uint32_t*>(p.o + (out0 + k) * kKvD + 2 * lane) = 0;
      if (p.lse && lane == 0) p.lse[out0 + k] = -INFINITY;
    }
    return;
  }
  // lane k < HEADS: head h0 + k
  const int h = min(h0 + min(lane, HEADS - 1), p.Hq - 1), hk = h / p.G;
  const int row = (tok - r.first) * p.G + (h - hk * p.G);
  const int unit = row / p.rows, in_unit = row - unit * p.rows;
  const int2 cut = p.cut[unit_id(p, b, r.first, unit) * p.Hkv + hk];
  struct Head {
    int w0, w1, slot, in_unit;
  };
  auto head = [&](int k) {  // (w1 < w0: nothing to join)
    const int x = __builtin_amdgcn_readlane(cut.x, k), y = __builtin_amdgcn_readlane(cut.y, k);
    const bool any = h0 + k < p.Hq && x >= 0;
    return Head{any ? x >> 1 : 0, any ? y : -1, x & 1, __builtin_amdgcn_readlane(in_unit, k)};
  };
  auto piece = [&](const Head& d, int w) { return ((size_t)w * 2 + (w == d.w0 ? d.slot : 0)) * p.rows + d.in_unit; };
  float2 x[HEADS][kJoinPieces], q[HEADS][kJoinPieces];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const Head d = head(k);
#pragma unroll
    for (int u = 0; u < kJoinPieces; ++u) {
      const int w = d.w0 + sub + u * STEP;
      if (w > d.w1) continue;
      const size_t e = piece(d, w);
      x[k][u] = *reinterpret_cast<const float2*>(p.part_o + e * kKvD + 2 * lane);
      q[k][u] = *reinterpret_cast<const float2*>(p.part_ml + e * 2);
    }
  }
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const Head d = head(k);
    if (d.w1 < 0) continue;  // (written by its workgroup)
    const int from = d.w0 + sub;
    float M = -INFINITY;
#pragma unroll
    for (int u = 0; u < kJoinPieces; ++u)
      if (from + u * STEP <= d.w1) M = fmaxf(M, q[k][u].x);
    if (from + kJoinPieces * STEP <= d.w1) {
      for (int w = from + (kJoinPieces + lane) * STEP; w <= d.w1; w += 64 * STEP) M = fmaxf(M, p.part_ml[piece(d, w) * 2]);
#pragma unroll
      for (int s = 32; s >= 1; s >>= 1) M = fmaxf(M, __shfl_xor(M, s));
    }
    float ref = M == -INFINITY ? 0.f : M;
    float a0 = 0.f, a1 = 0.f, L = 0.f;
    auto add = [&](float2 y, float2 z) {
      const float s = __builtin_amdgcn_exp2f((z.x - ref) * p.c);
      L = fmaf(z.y, s, L);
      a0 = fmaf(y.x, s, a0);
      a1 = fmaf(y.y, s, a1);
    };
#pragma unroll
    for (int u = 0; u < kJoinPieces; ++u)
      if (from + u * STEP <= d.w1) add(x[k][u], q[k][u]);
    for (int w = from + kJoinPieces * STEP; w <= d.w1; w += 8 * STEP) {
      float2 y[8], z[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const size_t e = piece(d, min(w + u * STEP, d.w1));
        y[u] = *reinterpret_cast<const float2*>(p.part_o + e * kKvD + 2 * lane);
        z[u] = *reinterpret_cast<const float2*>(p.part_ml + e * 2);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (w + u * STEP <= d.w1) add(y[u], z[u]);
    }
    if constexpr (SPLIT) {
      *reinterpret_cast<float2*>(&red[wave][2 * lane]) = float2{a0, a1};
      if (lane == 0) *reinterpret_cast<float2*>(red_ml[wave]) = float2{M, L};
      __syncthreads();  // (the whole workgroup has this row)
      if (wave) return;
      M = fmaxf(fmaxf(red_ml[0][0], red_ml[1][0]), fmaxf(red_ml[2][0], red_ml[3][0]));
      ref = M == -INFINITY ? 0.f : M;
      a0 = a1 = L = 0.f;
#pragma unroll
      for (int j = 0; j < kJoinWaves; ++j) add(*reinterpret_cast<const float2*>(&red[j][2 * lane]), *reinterpret_cast<const float2*>(red_ml[j]));
    }
    const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);  // (NaN stays)
    const bf16x2 y = {(__bf16)(a0 * inv), (__bf16)(a1 * inv)};
    *reinterpret_cast<uint32_t*>(p.o + (out0 + k) * kKvD + 2 * lane) = __builtin_bit_cast(uint32_t, y);
    if (p.lse && lane == 0) p.lse[out0 + k] = L == 0.f ? -INFINITY : M * p.scale + __logf(L);
  }
}

struct TreePlan {
  int waves = 4, blocks = 2, rows = 128, shares = 0, least = 1;
  bool fit = true, whole = false;
  int64_t units = 0;
  size_t bytes = 0;
};

// The forms, the number of shares and the non-temporal loads are chosen for the whole chip: a stream with fewer CUs gets
// the same forms (and the same results), whose measurements below do not hold there.
int tree_plan(int B, int Hq, int Hkv, int T, int S, int split_tokens, TreePlan* plan) {
  if (B < 0 || T < 0 || Hq < 1 || Hkv < 1 || S < 1)
    return fail(ASYM_EINVAL, "tree attention: B and T must be >= 0, H_q, H_kv and S_max >= 1");
  if (Hq % Hkv) return fail(ASYM_EINVAL, "tree attention: H_kv must divide H_q");
  if (split_tokens < 0 || split_tokens % kKvPageTokens || split_tokens > (1 << 20))
    return fail(ASYM_EINVAL, "tree attention: split_tokens must be 0 (automatic) or a multiple of 32 up to 2^20");
  TreePlan P;
  if (B == 0 || T == 0) {
    *plan = P;
    return ASYM_OK;
  }
  // (threads are counted in 32 bits: the joining launch has a wave for kJoinHeads heads of a token, kJoinWaves a workgroup)
  const int64_t joins = ((int64_t)T * ((Hq + kJoinHeads - 1) / kJoinHeads) + kJoinWaves - 1) / kJoinWaves;
  if ((int64_t)T * Hq >= (1 << 26) || joins * 64 * kJoinWaves > 0xFFFFFFFFll)
    return fail(ASYM_EUNSUPPORTED, "tree attention: too many rows");
  const int64_t all = (int64_t)T * (Hq / Hkv), mean = (all + B - 1) / B;
  const int64_t pages = ((int64_t)S + kKvPageTokens - 1) / kKvPageTokens, most = (all / 64 + B) * Hkv;
  if (most > (1 << 30) || most * pages > (1 << 30)) return fail(ASYM_EUNSUPPORTED, "tree attention: more than 2^30 pages");
  const int64_t segments = (all / 128 + B) * Hkv;  // of four waves and two blocks of rows each
  // One block of 16 rows a wave spreads few rows over more waves, and a wave's chain of products, softmax and products again, which
  // is what a block of tokens costs where the matrix cores have little to do, is half as long; the pages of more than 64 rows
  // are read again.  us, two blocks first, 32 / 8 heads, n nodes in the mean, lengths from a quarter of S on, in a graph, S 250,
  // 777, 2048, 8000: 1 request of 8 nodes 13.3 9.3, 11.2 9.8, 12.7 10.8; 64 of 1 15.8 12.8, 30.7 25.7, 70 60, 208 202; 64 of 10
  // 19.3 15.7, 38.3 28.5, 86 63, 247 235; 64 of 16 21.5 21.7, 39.3 36.6, 87 82; 32 of 16 15.4 13.7, 28.2 22.9, 54 47, 136 165; 8 of
  // 32 13.7 10.1, 31.5 20.2, 38.6 27.6, 59 49; 8 of 64 15.9 11.5, 29.6 20.6, 39.6 33.1, 81 98; 32 of 32 20.3 18.6, 38.3 28.8, 82
  // 63, 192 269; 1 of 512 34.0 19.7 (S 512), 39.2 24.6, 48.6 39.3, 84 106.
  // Near the line either may be a fifth faster.  It gives up 32 of 32 at S 1500 and 2048 (63 46), 8 of 32 at 8000, 16 of 16 at
  // 4000 (49 39), 32 of 16 at 2048 (also with 8 / 8, 40 / 8 and 64 / 8 heads: 45 39, 58 47, 80 58), 1 of 512 at 6000 (69 83) and 4 of
  // 256 with 16 / 2 heads at 6000 (63 74); twice the pages would give up 16 of 32 at 3000 (50 58) and 32 of 20 at 2500 (63 72).
  const bool narrow = mean <= 40 || (segments <= 512 && segments * pages <= 16384);
  // Whole segments need no pieces, no second launch and no workspace, and take as long as the longest request: about 5 us
  // and 0.5 a page where it is alone.  Cut ones take two launches and what the pieces of T x H_q rows cost to write and
  // join.  us, cut first, as above: one block of rows: 1 request of 8 nodes, S 300 10.8 10.3, 380 10.7 11.2, 512 10.8
  // 13.1; 16 of 8, 500 15.9 13.9, 1000 21.3 23.4; 8 of 16, 1000 21.5 21.6, 1500 21.3 29.7; 8 of 64, 1000 26.1 23.0, 1500 28.6
  // 31.9; 24 of 8, 1500 24.1 29.6; 16 of 32, 2000 36.4 45.8; 32 of 10, 2000 38.5 39.2, 3000 56 61; 64 of 1, 2000 62 58, 4000
  // 110 110, 8000 204 215; 64 of 10, 4000 131 114, 5000 158 141; 256 of 1, 8000 778 809.  Two: 64 of 16, 2000 92 83; 32 of 24, 1500
  // 51 54, 2000 60 68, 4000 94 127, 8000 166 254; 16 of 64, 2000 61 79; 64 of 32, 2000 131 119, 4000 211 214; 64 of 64, 500 111
  // 59, 2000 239 177; 32 of 64, 4000 195 179.
  // The line is a fit to these heads.  It gives up 16 of 8 at 1000 and 32 of 24 at 1500 (it takes whole ones), 64 of 10 at 5000
  // and 32 of 64 at 4000 (it cuts them).
  const int64_t weight = (int64_t)T * Hq / 1200;
  const int64_t longest = !narrow           ? segments / 11 + weight
                          : segments >= 512 ? 128 + weight
                          : segments >= 256 ? 64
                                            : std::max<int64_t>(12, std::min<int64_t>(segments * 2 / 5, 32));
  P.whole = split_tokens == 0 && pages <= longest;
  // Eight waves read the pages of up to 256 rows once, four of 128; but of four there are two workgroups a CU, which hide each
  // other's starts, ends and waits, and rows past 128 cost a wave what it has of them.  us, four first, as above: 16 requests, n
  // 40, S 4000 70 92; 8, n 48, S 32768 212 258; n 64: 4 of 8000 52 59, 8 of 8000 82 87, 16 of 8000 170 179, 32 of 4000 185 199, 8 of
  // 32768 285 295, and 422 412 where calls follow each other until the power cap holds; n 512: 2 of 4000 74 70, 4 of 8000 205 223.
  // It gives up 5 to 8 % at 16 of 8000 and 32 of 4000 in short runs.  Whole segments of four waves, cut ones of eight: n 64, 64 of
  // 2000 175 239, 64 of 4000 329 380, 128 of 1000 206 348, 128 of 4000 688 764.
  P.waves = !narrow && !P.whole && mean > 192 && (all / 256 + B) * Hkv * pages >= 180 * 256 ? 8 : 4;
  P.blocks = narrow ? 1 : 2;
  P.rows = 16 * P.blocks * P.waves;
  P.units = all / P.rows + B;
  const int64_t heads = P.units * Hkv;  // segments, where none is cut
  P.fit = split_tokens == 0;
  // (us in a graph with shares of 2, 4, 6 and 8 pages at least: 1 request of 8 nodes, S 500 9.7 10.7 11.8 13.4, 777 10.0 9.7 10.6
  // 11.5, 2048 11.9 10.8 11.0 12.7; 16 of 8 with 8 / 1 heads, 777 12.9 12.5 13.4 14.2, 2048 18.3 14.0 14.1 15.5)
  P.least = P.fit ? 4 : split_tokens / kKvPageTokens;
  int64_t shares = P.whole ? heads : heads * pages / P.least + heads;  // (a segment may end in a part of one)
  if (P.fit && !P.whole) shares = std::min<int64_t>(shares, P.waves == 8 ? 256 : 512);
  if (shares >= (1 << 22)) return fail(ASYM_EUNSUPPORTED, "tree attention: too many shares");
  P.shares = (int)shares;
  P.bytes = P.whole ? 0 : (size_t)shares * 2 * P.rows * (kKvD + 2) * sizeof(float) + (size_t)heads * sizeof(int2);
  *plan = P;
  return ASYM_OK;
}

}  // namespace
}  // namespace asym

extern "C" int asym_attn_tree_paged_workspace(int B, int H_q, int H_kv, int T, int S_max, int split_tokens, size_t* bytes) {
  if (!bytes) return asym::fail(ASYM_EINVAL, "tree attention workspace: null output");
  asym::TreePlan P;
  const int rc = asym::tree_plan(B, H_q, H_kv, T, S_max, split_tokens, &P);
  if (rc == ASYM_OK) *bytes = P.bytes;
  return rc;
}

extern "C" int asym_attn_tree_paged_bf16(int B, int H_q, int H_kv, int T, int S_max, int D, const void* q, int64_t q_token,
                                         int64_t q_head, const void* k_pool, const void* v_pool, size_t pool_pages,
                                         const int32_t* k_pages, const int32_t* v_pages, int pages_per_head, const int32_t* cu,
                                         const int32_t* lens, const uint64_t* mask, int mask_words, void* o, float* lse,
                                         float scale, int split_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace asym;
  TreePlan P;
  int rc = tree_plan(B, H_q, H_kv, T, S_max, split_tokens, &P);
  if (rc != ASYM_OK) return rc;
  if (D != kKvD) return fail(ASYM_EUNSUPPORTED, "tree attention: the head dimension must be 128");
  if (pages_per_head < 1 || (int64_t)pages_per_head * kKvPageTokens < S_max)
    return fail(ASYM_EINVAL, "tree attention: the page tables end before S_max");
  if (pool_pages < 1 || pool_pages > 0x7FFFFFFFu) return fail(ASYM_EINVAL, "tree attention: pool_pages must be in [1, 2^31)");
  if (!std::isfinite(scale)) return fail(ASYM_EINVAL, "tree attention: scale must be finite");
  if (mask && mask_words < 1) return fail(ASYM_EINVAL, "tree attention: a mask must have a word or more a node");
  if (B == 0 || T == 0) return ASYM_OK;
  if (!q || !k_pool || !v_pool || !k_pages || !v_pages || !cu || !lens || !o)
    return fail(ASYM_EINVAL, "tree attention: null pointer");
  if (((uintptr_t)q | (uintptr_t)k_pool | (uintptr_t)v_pool | (uintptr_t)o) & 15u)
    return fail(ASYM_EINVAL, "tree attention: q, the pools and O must be 16-byte aligned");
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)cu | (uintptr_t)lens | (uintptr_t)lse) & 3u || ((uintptr_t)mask & 7u))
    return fail(ASYM_EINVAL, "tree attention: tables, offsets, lengths and lse must be 4-byte aligned, masks 8-byte aligned");
  for (int64_t s : {q_token, q_head})
    if (s < 0 || s % 8) return fail(ASYM_EINVAL, "tree attention: strides must be multiples of 8 values and not negative");
  if (P.bytes && (!workspace || workspace_bytes < P.bytes || ((uintptr_t)workspace & 15u)))
    return fail(ASYM_EINVAL, "tree attention: the workspace must be 16-byte aligned and hold asym_attn_tree_paged_workspace's bytes");
  TreeParams p = {};
  p.q = static_cast<const uint16_t*>(q);
  p.q_tok = q_token; p.q_head = q_head;
  p.k_pool = static_cast<const uint8_t*>(k_pool);
  p.v_pool = static_cast<const uint8_t*>(v_pool);
  p.k_pages = k_pages; p.v_pages = v_pages; p.cu = cu; p.lens = lens;
  p.mask = mask; p.words = mask_words;
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  const size_t pieces = (size_t)P.shares * 2 * P.rows;
  p.part_o = static_cast<float*>(workspace);
  p.part_ml = p.part_o + pieces * kKvD;
  p.cut = P.whole ? nullptr : reinterpret_cast<int2*>(p.part_ml + pieces * 2);
  p.B = B; p.Hq = H_q; p.Hkv = H_kv; p.G = H_q / H_kv; p.T = T; p.S = S_max; p.pph = pages_per_head;
  p.pool_pages = (int)pool_pages;
  p.rows = P.rows; p.shares = P.shares; p.least = P.least; p.fit = P.fit;
  p.scale = std::fabs(scale);
  p.c = std::fmax(p.scale * 1.4426950408889634f, 1.17549435e-38f);  // (0 weighs all tokens alike, a masked one not at all)
  p.q_flip = scale < 0 ? 0x80008000u : 0u;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // (at most: the requests may be shorter than S_max)
  const int64_t bytes = 2ll * B * H_kv * ((S_max + (int64_t)kKvPageTokens - 1) / kKvPageTokens) * kPageBytes;
  const bool once = attn_streams_kv(paged_kv_bytes(bytes, (int64_t)pool_pages * kPageBytes, k_pool == v_pool));
  auto kernel = P.waves == 8    ? (once ? attn_tree_kernel<8, 4, 2, 2> : attn_tree_kernel<8, 4, 2, 0>)
                : P.blocks == 2 ? (once ? attn_tree_kernel<4, 2, 2, 2> : attn_tree_kernel<4, 2, 2, 0>)
                                : (once ? attn_tree_kernel<4, 2, 1, 2> : attn_tree_kernel<4, 2, 1, 0>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)P.shares), dim3(64 * P.waves), 0, s, p);
  ASYM_HIP(hipGetLastError());
  if (P.whole) return ASYM_OK;
  // (a row has about as many pieces as there are shares to a unit and head; threads are counted in 32 bits.  4 nodes of 8 / 1
  // heads behind 30000 tokens, 85 pieces a row: 22 us, and 64 more with a wave for two heads)
  if (P.shares >= 4 * P.units * H_kv && T <= (1 << 22) / H_q) {
    hipLaunchKernelGGL(attn_tree_join<true>, dim3((unsigned)(T * H_q)), dim3(64 * kJoinWaves), 0, s, p);
  } else {
    const int64_t waves = (int64_t)T * ((H_q + kJoinHeads - 1) / kJoinHeads);
    hipLaunchKernelGGL(attn_tree_join<false>, dim3((unsigned)((waves + kJoinWaves - 1) / kJoinWaves)), dim3(64 * kJoinWaves), 0, s, p);
  }
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
