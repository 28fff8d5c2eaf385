// Decode attention over a paged cache in microscaled 4-bit floating point (format
// and page layout: kv_fp4.h), one query token per request, a length per request:
//
//   O[b, h] = softmax_t(scale * <q[b, h], K[b, g, t]>) . V[b, g, :],  t < lens[b], g = h / G
//
// The pages of the batch, request by request and head by head, are one list, cut into equal
// shares, one a wave, whatever the requests' lengths (which only the device knows): a grid
// of (request, head, split) tasks left waves idle behind the short ones (64 requests of up to
// 32768 tokens, 1.41 GB: 319 us, in shares 226, 6.2 TB/s: HBM's rate for reads).  A wave walks
// its share; for each (request, key/value head) that it meets it serves the G <= 16 query
// heads that read that head, 32 tokens (a page) at a time:
//   scores   two v_mfma_scale_f32_16x16x128_f8f6f4 a 16 tokens: the page's codes and scales
//            are the operand as they lie, with no conversion at all.  The other operand
//            takes 8 bits at most, so q, whose bf16 has 8 significant bits, goes in as
//            two e4m3 values of 4 bits each, hi + lo, with a scale of the row's own (hi
//            reaches [128, 256), lo carries 2^-5 of hi's scale): exact for values within
//            2^-7 of the row's largest, and within 2^-22 of it otherwise;
//   softmax  in fp32, a lane has 8 tokens of one head; the running max is raised only
//            when some head's grows by more than 2^8;
//   P.V      the value scales vary along the product's tokens, so they go into the
//            probabilities: 4 operands (one per block of 32 channels) of
//            bf16(p * X), rounded as p alone would be, since X is a power of two; the
//            codes become bf16 by v_cvt_scalef32_pk_bf16_fp4 (exact), two an instruction.
// No LDS, no barrier.  A (request, head) that lies in one share is written by its wave;
// of one that is cut, each share leaves its unnormalised output, max and sum in fp32 (at
// most two such pieces a wave: its first and its last), which a second launch joins in the
// order of the shares.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "kv_fp4.h"
#include "read_policy.h"

namespace asym {
namespace {

constexpr int kWaves = 4;
constexpr int kMaxG = 16;
constexpr int kShares = 2048;     // waves: 8 a CU of 256 (12 fit, and join more pieces: 64 requests of up to 1000
                                  // tokens 20.1 us, with 8 a CU 18.1)
constexpr int kMostPieces = 128;  // that the longest request is cut into
constexpr int kJoinWaves = 16;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp4DecodeParams {
  const uint16_t* q;             // [B][Hq][128]
  const uint8_t *k_pool, *v_pool;
  const int *k_pages, *v_pages;  // [B][Hkv][pph]
  const int* lens;
  uint16_t* o;                   // [B][Hq][128]
  float* lse;                    // [B][Hq], nullable
  float* part_o;                 // [shares][2][G][128]
  float* part_ml;                // [shares][2][G][2]: max (of the raw scores), sum
  int B, Hq, Hkv, G, S, pph, pool_pages;
  int2* cut;                     // [B][Hkv]: of a (request, head) that was cut, 2 (its first share) + (1: that share's
                                 // last piece), its last share; -1 of one that was not
  int shares, share_pages, least;  // share_pages 0: the batch's pages over the shares, at least `least`
  float c, scale;                // |scale| * log2(e), |scale|
  uint32_t q_flip;
};

__device__ __forceinline__ float max_quarters(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// The 32 values of q that the lane (head n, quarter p) holds as the 8-bit operand:
// channels 16 p + 0 .. 15 and 64 + 16 p + 0 .. 15, as hi and lo, and their scale bytes
__device__ __forceinline__ void load_q(const uint16_t* row, bool on, int quarter, uint32_t flip, i32x8& hi, i32x8& lo,
                                       int& s_hi, int& s_lo) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x4 x = {};
    if (on) x = *reinterpret_cast<const u32x4*>(row + 16 * quarter + 64 * (i >> 1) + 8 * (i & 1));
#pragma unroll
    for (int e = 0; e < 4; ++e) w[4 * i + e] = on ? x[e] ^ flip : 0u;
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  const int e = min(max((int)(top >> 7), 13), 254);  // the row's exponent field
  s_hi = e - 7;
  s_lo = e - 12;
  const float up = __uint_as_float((uint32_t)(261 - e) << 23);  // 2^(134 - e): 1 / the scale of hi
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float x[4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      x[2 * t] = __uint_as_float(w[2 * i + t] << 16) * up;
      x[2 * t + 1] = __uint_as_float(w[2 * i + t] & 0xFFFF0000u) * up;
    }
    int a = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], a, true);
    hi[i] = a;
    const float r0 = (x[0] - __builtin_amdgcn_cvt_f32_fp8(a, 0)) * 32.f, r1 = (x[1] - __builtin_amdgcn_cvt_f32_fp8(a, 1)) * 32.f;
    const float r2 = (x[2] - __builtin_amdgcn_cvt_f32_fp8(a, 2)) * 32.f, r3 = (x[3] - __builtin_amdgcn_cvt_f32_fp8(a, 3)) * 32.f;
    int d = __builtin_amdgcn_cvt_pk_fp8_f32(r0, r1, 0, false);
    lo[i] = __builtin_amdgcn_cvt_pk_fp8_f32(r2, r3, d, true);
  }
}

struct PageRegs {
  u32x4 k[2], v[2], vs[2];
  uint32_t ks;
};

template <int POLICY>
__device__ __forceinline__ void load_page(const Fp4DecodeParams& p, int kp, int vp, int lane, PageRegs& r) {
  const __amdgpu_buffer_rsrc_t rk = page_rsrc(p.k_pool, kp, p.pool_pages), rv = page_rsrc(p.v_pool, vp, p.pool_pages);
  const uint32_t ko = (uint32_t)((lane & 15) * 64 + (lane >> 4) * 16);
#pragma unroll
  for (int t = 0; t < 2; ++t) r.k[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, ko + 1024 * t, 0, POLICY));
  r.ks = __builtin_amdgcn_raw_buffer_load_b16(rk, kFp4ScaleOff + (uint32_t)lane * 2, 0, POLICY);
#pragma unroll
  for (int t = 0; t < 2; ++t)
    r.v[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, (uint32_t)lane * 16 + 1024 * t, 0, POLICY));
#pragma unroll
  for (int t = 0; t < 2; ++t)
    r.vs[t] = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, kFp4ScaleOff + (uint32_t)(lane >> 4) * 32 + 16 * t, 0, POLICY));
}

// One wave's running result for the G heads of its group: column lane % 16 is a head;
// o[g] holds channels 16 g + 4 (lane / 16) + 0 .. 3.
struct Running {
  f32x4 o[8];
  float m, l;
};

// 32 tokens, of which `left` exist (32 or more: all)
__device__ __forceinline__ void add_page(const Fp4DecodeParams& p, const PageRegs& cur, int left, int quarter,
                                         const i32x8& q_hi, const i32x8& q_lo, int s_hi, int s_lo, Running& a) {
  f32x4 s[2];  // scores: rows 4 quarter + r of tokens 16 t .., column n
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const i32x8 k = {(int)cur.k[t][0], (int)cur.k[t][1], (int)cur.k[t][2], (int)cur.k[t][3], 0, 0, 0, 0};
    const int ks = (int)(cur.ks >> (8 * t));
    s[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q_lo, f32x4{}, 4, 0, 0, ks, 0, s_lo);
    s[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q_hi, s[t], 4, 0, 0, ks, 0, s_hi);
  }
  uint32_t vs[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) vs[j] = cur.vs[j >> 2][j & 3];
  if (left < kKvPageTokens) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool on = 4 * quarter + (j & 3) + 16 * (j >> 2) < left;
      if (!on) s[j >> 2][j & 3] = -INFINITY;
      if (!on) vs[j] = 0;  // (as 0: whatever scale lies there cannot reach the sum)
    }
  }
  float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                    fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
  top = max_quarters(top);
  if (__any((top - a.m) * p.c > 8.f)) {
    const float m_new = fmaxf(a.m, top);
    const float alpha = __builtin_amdgcn_exp2f((a.m - (m_new == -INFINITY ? 0.f : m_new)) * p.c);
    a.l *= alpha;
#pragma unroll
    for (int g = 0; g < 8; ++g) a.o[g] *= alpha;
    a.m = m_new;
  }
  const float ms = a.m == -INFINITY ? 0.f : a.m * p.c;
  float e[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    e[j] = __builtin_amdgcn_exp2f(fmaf(s[j >> 2][j & 3], p.c, -ms));
    a.l += e[j];
  }
#pragma unroll
  for (int blk = 0; blk < 4; ++blk) {
    bf16x8 pf;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t x = blk == 0 ? vs[j] << 23 : blk == 1 ? vs[j] << 15 : blk == 2 ? vs[j] << 7 : vs[j] >> 1;
      pf[j] = (__bf16)(e[j] * __uint_as_float(x & 0x7F800000u));
    }
#pragma unroll
    for (int g2 = 0; g2 < 2; ++g2) {
      const int g = 2 * blk + g2;
      const uint32_t w = cur.v[g >> 2][g & 3];
      union {
        bf16x2 p[4];
        bf16x8 v;
      } f;
      f.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0);
      f.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1);
      f.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2);
      f.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3);
      a.o[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, pf, a.o[g], 0, 0, 0);
    }
  }
}

// Where the requests' pages lie in the list, 256 requests at a time: lane l has requests
// base + l, + 64, + 128 and + 192.  (Named members: the compiler would put an array that is
// indexed at run time into LDS.)
struct Requests {
  int base;
  int len0, len1, len2, len3;
  int upto0, upto1, upto2, upto3;  // pages (of one head) of the batch up to and with the request

  static __device__ __forceinline__ int pages_of(int len) { return (int)((uint32_t)(len + kKvPageTokens - 1) / kKvPageTokens); }
  static __device__ __forceinline__ int pick(int i, int a, int b, int c, int d) { return i < 2 ? (i ? b : a) : (i == 2 ? c : d); }
  __device__ __forceinline__ void load(const Fp4DecodeParams& p, int from, int before, int lane) {
    base = from;
    const int b = from + lane;
    len0 = b < p.B ? p.lens[b] : 0;
    len1 = b + 64 < p.B ? p.lens[b + 64] : 0;
    len2 = b + 128 < p.B ? p.lens[b + 128] : 0;
    len3 = b + 192 < p.B ? p.lens[b + 192] : 0;
    auto held = [&](int x) { return min(max(x, 0), p.S); };
    len0 = held(len0);
    upto0 = before + wave_scan_add(pages_of(len0));
    upto1 = upto2 = upto3 = before = __builtin_amdgcn_readlane(upto0, 63);
    len1 = held(len1), len2 = held(len2), len3 = held(len3);
    if (from + 64 < p.B) {
      upto1 = before + wave_scan_add(pages_of(len1));
      before = __builtin_amdgcn_readlane(upto1, 63);
      upto2 = before + wave_scan_add(pages_of(len2));
      before = __builtin_amdgcn_readlane(upto2, 63);
      upto3 = before + wave_scan_add(pages_of(len3));
    }
  }
  __device__ __forceinline__ int end() const { return __builtin_amdgcn_readlane(upto3, 63); }
  __device__ __forceinline__ int len_of(int at) const {  // of request base + at
    return __builtin_amdgcn_readlane(pick(at >> 6, len0, len1, len2, len3), at & 63);
  }
  // The request (at) whose pages hold the list's page f; returns the place of its first page
  __device__ __forceinline__ int find(const Fp4DecodeParams& p, int f, int lane, int& at) {
    while (end() * p.Hkv <= f) load(p, base + 256, end(), lane);
    auto last = [&](int upto) { return __builtin_amdgcn_readlane(upto, 63) * p.Hkv <= f; };
    const int i = last(upto0) + last(upto1) + last(upto2);
    const int x = pick(i, upto0, upto1, upto2, upto3), l = __builtin_ctzll(__ballot(x * p.Hkv > f));
    at = 64 * i + l;
    return (__builtin_amdgcn_readlane(x, l) - pages_of(len_of(at))) * p.Hkv;
  }
};
// The batch's pages (of one head)
__device__ __forceinline__ int batch_pages(const Fp4DecodeParams& p, int lane, const Requests& r0) {
  int sum = r0.end();
  if (p.B > 256) {
    int more = 0;
    for (int b = 256 + lane; b < p.B; b += 64) more += Requests::pages_of(min(max(p.lens[b], 0), p.S));
    sum += wave_sum(more);
  }
  return sum;
}

// ROWS: a wave has one (request, key/value head), whole.
template <int POLICY, bool ROWS>
__global__ void __launch_bounds__(64 * kWaves) fp4_decode_share(Fp4DecodeParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = blockIdx.x * kWaves + wave;
  const int n = lane & 15, quarter = lane >> 4;
  Requests rq;
  int f, f1, at, len, pages, hk, pg, share = 0;  // pages f .. f1 - 1 of the list
  if constexpr (ROWS) {
    if (w >= p.B * p.Hkv) return;
    at = w / p.Hkv;
    hk = w - at * p.Hkv;
    rq.base = 0;
    len = __builtin_amdgcn_readfirstlane(min(max(p.lens[at], 0), p.S));
    f = pg = 0;
    f1 = pages = Requests::pages_of(len);  // (none: the result below is that of no token)
  } else {
    rq.load(p, 0, 0, lane);
    const int total = batch_pages(p, lane, rq) * p.Hkv;
    share = p.share_pages ? p.share_pages : max((total + p.shares - 1) / p.shares, p.least);
    if ((int64_t)w * share >= total) return;
    f = w * share;
    f1 = min(f + share, total);
    const int in = f - rq.find(p, f, lane, at);  // the page, over its request's heads
    len = rq.len_of(at);
    pages = Requests::pages_of(len);
    hk = in / pages;
    pg = in - hk * pages;
  }

  for (bool first = true;; first = false) {
    const int b = rq.base + at, bh = b * p.Hkv + hk;
    const int count = min(pages - pg, f1 - f);
    // a lane holds the number of one page of 64, and of one of the next 64
    const size_t row = (size_t)bh * p.pph + pg;
    auto numbers = [&](int i, int& k, int& v) {
      k = v = -1;
      if (i + lane < count) {
        k = p.k_pages[row + i + lane];
        v = p.v_pages[row + i + lane];
      }
    };
    int kpg, vpg, kpg2, vpg2;
    numbers(0, kpg, vpg);
    PageRegs cur, nxt;
    load_page<POLICY>(p, __builtin_amdgcn_readlane(kpg, 0), __builtin_amdgcn_readlane(vpg, 0), lane, cur);
    i32x8 q_hi, q_lo;
    int s_hi, s_lo;
    const int head = hk * p.G + n;  // this lane's query head
    load_q(p.q + ((size_t)b * p.Hq + (n < p.G ? head : 0)) * kKvD, n < p.G, quarter, p.q_flip, q_hi, q_lo, s_hi, s_lo);
    Running a;
#pragma unroll
    for (int g = 0; g < 8; ++g) a.o[g] = f32x4{};
    a.m = -INFINITY;
    a.l = 0.f;
    for (int i = 0; i < count; ++i) {
      const int e = i & 63;
      if (e == 0) numbers(i + 64, kpg2, vpg2);
      if (e == 63) {
        kpg = kpg2;
        vpg = vpg2;
      }
      // (behind the last page: none, which loads nothing)
      const int ne = (e + 1) & 63, kn = __builtin_amdgcn_readlane(kpg, ne), vn = __builtin_amdgcn_readlane(vpg, ne);
      load_page<POLICY>(p, i + 1 < count ? kn : -1, i + 1 < count ? vn : -1, lane, nxt);
      add_page(p, cur, len - (pg + i) * kKvPageTokens, quarter, q_hi, q_lo, s_hi, s_lo, a);
      cur = nxt;
    }
    a.l += __shfl_xor(a.l, 16);
    a.l += __shfl_xor(a.l, 32);
    if (n < p.G) {
      if (count == pages) {  // all of it
        const size_t out = (size_t)b * p.Hq + head;
        const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
        uint16_t* dst = p.o + out * kKvD + 4 * quarter;
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const bf16x2 x = {(__bf16)(a.o[g][0] * inv), (__bf16)(a.o[g][1] * inv)};
          const bf16x2 y = {(__bf16)(a.o[g][2] * inv), (__bf16)(a.o[g][3] * inv)};
          *reinterpret_cast<uint2*>(dst + 16 * g) = uint2{__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y)};
        }
        if (p.lse && quarter == 0) p.lse[out] = a.l == 0.f ? -INFINITY : a.m * p.scale + __logf(a.l);
      } else {
        const size_t piece = ((size_t)w * 2 + (first ? 0 : 1)) * p.G + n;
        float* dst = p.part_o + piece * kKvD + 4 * quarter;
#pragma unroll
        for (int g = 0; g < 8; ++g) *reinterpret_cast<f32x4*>(dst + 16 * g) = a.o[g];
        if (quarter == 0) *reinterpret_cast<float2*>(p.part_ml + piece * 2) = float2{a.m, a.l};
      }
    }
    // (for the join: which waves have a piece of it, and whether the first of them is its wave's second)
    if (!ROWS && pg == 0 && lane == 0)
      p.cut[bh] = count == pages ? int2{-1, 0} : int2{2 * w + (first ? 0 : 1), (f + pages - 1) / share};
    f += count;
    if (ROWS || f >= f1) return;
    pg = 0;
    if (++hk == p.Hkv) {  // the next request that has tokens (there is one)
      hk = 0;
      do {
        if (++at == 256) {
          rq.load(p, rq.base + 256, rq.end(), lane);
          at = 0;
        }
        len = rq.len_of(at);
      } while (len == 0);
      pages = Requests::pages_of(len);
    }
  }
}

// A few waves (`per`, a power of two) a (request, query head): one without tokens is written,
// one that was cut is joined.  Wave j takes pieces j, j + per, ..., eight loads at a time (the
// first eight go out before the row's max is known); the waves' sums are added in order.
__global__ void __launch_bounds__(64 * kJoinWaves) fp4_decode_join(Fp4DecodeParams p, int per) {
  __shared__ float red[kJoinWaves][kKvD], red_l[kJoinWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = wave & (per - 1);
  const int row = (int)(blockIdx.x * (blockDim.x >> 6) + wave) / per;
  float a0 = 0.f, a1 = 0.f, L = 0.f, M = -INFINITY;
  bool join = false;
  if (row < p.B * p.Hq) {
    const int b = row / p.Hq, h = row - b * p.Hq, hk = h / p.G, g = h - hk * p.G;
    const int2 cut = p.cut[b * p.Hkv + hk];  // (of a request without tokens: not written, and not used)
    if (min(p.lens[b], p.S) <= 0) {
      if (sub == 0) {
        *reinterpret_cast<uint32_t*>(p.o + (size_t)row * kKvD + 2 * lane) = 0;
        if (p.lse && lane == 0) p.lse[row] = -INFINITY;
      }
    } else if (cut.x >= 0) {
      join = true;
      const int w0 = cut.x >> 1, w1 = cut.y;
      auto piece = [&](int w) { return ((size_t)w * 2 + (w == w0 ? cut.x & 1 : 0)) * p.G + g; };
      float2 x[8], q[8];
      auto load = [&](int w) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const size_t e = piece(min(w + u * per, w1));
          x[u] = *reinterpret_cast<const float2*>(p.part_o + e * kKvD + 2 * lane);
          q[u] = *reinterpret_cast<const float2*>(p.part_ml + e * 2);
        }
      };
      load(w0 + sub);
      for (int w = w0 + lane; w <= w1; w += 64) M = fmaxf(M, p.part_ml[piece(w) * 2]);
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
      for (int w = w0 + sub; w <= w1; w += 8 * per) {
        if (w != w0 + sub) load(w);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if (w + u * per > w1) break;
          // (M minus infinity: nothing but NaN, which goes on)
          const float s = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((q[u].x - M) * p.c);
          L = fmaf(q[u].y, s, L);
          a0 = fmaf(x[u].x, s, a0);
          a1 = fmaf(x[u].y, s, a1);
        }
      }
    }
  }
  if (per > 1) {
    red[wave][2 * lane] = a0;
    red[wave][2 * lane + 1] = a1;
    if (lane == 0) red_l[wave] = L;
    __syncthreads();
    if (sub) return;
    for (int j = 1; j < per; ++j) {
      a0 += red[wave + j][2 * lane];
      a1 += red[wave + j][2 * lane + 1];
      L += red_l[wave + j];
    }
  }
  if (!join || sub) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const bf16x2 r = {(__bf16)(a0 * inv), (__bf16)(a1 * inv)};
  *reinterpret_cast<uint32_t*>(p.o + (size_t)row * kKvD + 2 * lane) = __builtin_bit_cast(uint32_t, r);
  if (p.lse && lane == 0) p.lse[row] = L == 0.f ? -INFINITY : M * p.scale + __logf(L);
}

struct Fp4Plan {
  int shares = 0, share_pages = 0, least = 1, per = 1;
  bool rows = false;
};

int fp4_plan(int B, int Hq, int Hkv, int S, int D, int split_tokens, asym_attn_plan_info* out, Fp4Plan* plan) {
  if (B < 0 || Hq < 1 || Hkv < 1 || S < 1) return fail(ASYM_EINVAL, "fp4 attention: B must be >= 0, H_q, H_kv and S_max >= 1");
  if (Hq % Hkv) return fail(ASYM_EINVAL, "fp4 attention: H_kv must divide H_q");
  if (Hq / Hkv > kMaxG) return fail(ASYM_EUNSUPPORTED, "fp4 attention: at most 16 query heads per key/value head");
  if (D != kKvD) return fail(ASYM_EUNSUPPORTED, "fp4 attention: the head dimension must be 128");
  if (split_tokens < 0 || split_tokens % kKvPageTokens || split_tokens > (1 << 20))
    return fail(ASYM_EINVAL, "fp4 attention: split_tokens must be 0 (automatic) or a multiple of 32 up to 2^20");
  const int64_t pages = ((int64_t)S + kKvPageTokens - 1) / kKvPageTokens, heads = (int64_t)B * Hkv, most = heads * pages;
  if (most > (1 << 30)) return fail(ASYM_EUNSUPPORTED, "fp4 attention: more than 2^30 pages");
  Fp4Plan P;
  // Enough heads for every wave, and short: a wave a head, whole.  Shares balance unequal
  // lengths, but cost a search, pieces and their join.  8 key/value heads, lengths from a
  // quarter of S_max on, us, shares first: 256 requests of up to 300 tokens 26.2 15.4, 600
  // 37.6 27.1, 1200 58.9 51.5, 2400 85.4 95.5; 512 of 1200 93.8 98.6; 1024 of 600 112 95.
  P.rows = !split_tokens && heads >= kShares && S <= 1024;
  P.least = split_tokens ? split_tokens / kKvPageTokens : (int)std::max<int64_t>(1, (pages + kMostPieces - 1) / kMostPieces);
  P.share_pages = split_tokens / kKvPageTokens;
  int64_t shares = P.rows ? heads : (most + P.least - 1) / P.least;
  if (!P.rows && !split_tokens) shares = std::min<int64_t>(shares, kShares);
  if (shares > (1 << 26) - kWaves || (int64_t)B * Hq * kJoinWaves >= (1 << 26))  // (threads of a launch are counted in 32 bits)
    return fail(ASYM_EUNSUPPORTED, "fp4 attention: too many tasks");
  P.shares = (int)shares;
  const int64_t share = P.rows ? pages : std::max<int64_t>(P.least, shares ? (most + shares - 1) / shares : 0);
  const int64_t pieces = P.rows ? 1 : std::min(shares, (pages + P.least - 2) / P.least + 1);
  // the join's waves of a query head, by the pieces that it has if all requests are of S_max:
  // about eight each
  const int64_t usual = std::min(pieces, heads ? (shares + heads - 1) / heads : 0);
  while (P.per < kJoinWaves && P.per * 8 < usual) P.per *= 2;
  *out = asym_attn_plan_info{};
  out->split_tokens = (int)std::min<int64_t>(share * kKvPageTokens, 1 << 30);
  out->n_splits = (int)pieces;
  out->tasks = P.shares;
  out->grid = (P.shares + kWaves - 1) / kWaves;
  out->tasks_per_workgroup = kWaves;
  out->workspace_bytes = P.rows ? 0 : (size_t)shares * 2 * (Hq / Hkv) * (kKvD + 2) * sizeof(float) + heads * sizeof(int2);
  *plan = P;
  return ASYM_OK;
}

}  // namespace
}  // namespace asym

extern "C" int asym_attn_decode_paged_fp4_plan(int B, int H_q, int H_kv, int S_max, int D, int split_tokens,
                                               asym_attn_plan_info* out) {
  if (!out) return asym::fail(ASYM_EINVAL, "fp4 attention plan: null output");
  asym::Fp4Plan plan;
  return asym::fp4_plan(B, H_q, H_kv, S_max, D, split_tokens, out, &plan);
}

extern "C" int asym_attn_decode_paged_fp4(int B, int H_q, int H_kv, int S_max, int D, const void* q, const void* k_pool,
                                          const void* v_pool, size_t pool_pages, const int32_t* k_pages,
                                          const int32_t* v_pages, int pages_per_head, const int32_t* lens, void* o,
                                          float* lse, float scale, int split_tokens, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  using namespace asym;
  asym_attn_plan_info plan;
  Fp4Plan P;
  int rc = fp4_plan(B, H_q, H_kv, S_max, D, split_tokens, &plan, &P);
  if (rc != ASYM_OK) return rc;
  if (pages_per_head < 1 || (int64_t)pages_per_head * kKvPageTokens < S_max)
    return fail(ASYM_EINVAL, "fp4 attention: the page tables end before S_max");
  if (pool_pages < 1 || pool_pages > 0x7FFFFFFFu) return fail(ASYM_EINVAL, "fp4 attention: pool_pages must be in [1, 2^31)");
  if (!std::isfinite(scale)) return fail(ASYM_EINVAL, "fp4 attention: scale must be finite");
  if (B == 0) return ASYM_OK;
  if (!q || !k_pool || !v_pool || !k_pages || !v_pages || !lens || !o) return fail(ASYM_EINVAL, "fp4 attention: null pointer");
  if (((uintptr_t)q | (uintptr_t)k_pool | (uintptr_t)v_pool | (uintptr_t)o) & 15u)
    return fail(ASYM_EINVAL, "fp4 attention: q, the pools and O must be 16-byte aligned");
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)lens | (uintptr_t)lse) & 3u)
    return fail(ASYM_EINVAL, "fp4 attention: tables, lengths and lse must be 4-byte aligned");
  if (plan.workspace_bytes && (!workspace || workspace_bytes < plan.workspace_bytes || ((uintptr_t)workspace & 15u)))
    return fail(ASYM_EINVAL, "fp4 attention: the workspace must be 16-byte aligned and hold the plan's workspace_bytes");
  Fp4DecodeParams p = {};
  p.q = static_cast<const uint16_t*>(q);
  p.k_pool = static_cast<const uint8_t*>(k_pool);
  p.v_pool = static_cast<const uint8_t*>(v_pool);
  p.k_pages = k_pages; p.v_pages = v_pages; p.lens = lens;
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.part_o = static_cast<float*>(workspace);
  if (!P.rows) {
    const size_t pieces = (size_t)P.shares * 2 * (H_q / H_kv);
    p.part_ml = p.part_o + pieces * kKvD;
    p.cut = reinterpret_cast<int2*>(p.part_ml + pieces * 2);
  }
  p.B = B; p.Hq = H_q; p.Hkv = H_kv; p.G = H_q / H_kv; p.S = S_max; p.pph = pages_per_head;
  p.pool_pages = (int)pool_pages;
  p.shares = P.shares;
  p.share_pages = P.share_pages;
  p.least = P.least;
  p.scale = std::fabs(scale);
  p.c = std::fmax(p.scale * 1.4426950408889634f, 1.17549435e-38f);  // (0 weighs all keys alike, a masked one not at all)
  p.q_flip = scale < 0 ? 0x80008000u : 0u;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // (at most: the requests may be shorter than S_max)
  // (Small CU sets stream too: what costs the 16-bit cache there does not cost this one.  us, ordinary loads first, 64
  // requests of up to 16384 tokens, 674 MiB: 256 CUs 137 121, 240 162 148, 192 146 133, 128 183 169, 64 302 302; 16 of 8000
  // with 32 key/value heads, 294 MiB: 65 57, 75 68, 70 65, 87 83, 145 144.)
  const int64_t bytes = 2ll * B * H_kv * ((S_max + (int64_t)kKvPageTokens - 1) / kKvPageTokens) * kFp4PageBytes;
  const bool once = attn_streams_kv(paged_kv_bytes(bytes, (int64_t)pool_pages * kFp4PageBytes, k_pool == v_pool));
  auto kernel = P.rows ? (once ? fp4_decode_share<2, true> : fp4_decode_share<0, true>)
                       : (once ? fp4_decode_share<2, false> : fp4_decode_share<0, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)plan.grid), dim3(64 * kWaves), 0, s, p);
  ASYM_HIP(hipGetLastError());
  if (!P.rows) {
    const int waves = std::max(P.per, 4);
    const int64_t all = (int64_t)B * H_q * P.per;
    hipLaunchKernelGGL(fp4_decode_join, dim3((unsigned)((all + waves - 1) / waves)), dim3(64 * waves), 0, s, p, P.per);
    ASYM_HIP(hipGetLastError());
  }
  return ASYM_OK;
}
