// Writing tokens into, and reading them back from, a paged cache in microscaled
// 4-bit floating point (format and page layout: kv_fp4.h).
//
// A wave has one page of one head: the tokens of the call that fall into it.  A page
// is written by one wave only, so that tokens that share a byte (values: two tokens
// a byte) need no atomics; what a page holds of other tokens stays.
//
// Bound by HBM: 324 bytes move for a token of a head (256 of bf16, 68 of the page).  8
// heads: 16381 tokens are written in 17.6 us and read in 16.2 (4.8 and 5.2 TB/s; a plain
// copy of 2 GiB 5.0), 65536 in 66 and 88, one token of each of 64 requests in 4.7 and 3.8.
// Writing asks for a half page's tokens at once: with a load a step a single token took
// 7.3, with a whole page's 4.3, but 16381 tokens 20.5 (registers, so waves).  Reading with
// stores of 8 and 16 bytes a row took 22.3 and 122; non-temporal ones 19 and 74, but what
// attends to the tokens next then takes as much longer.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "kv_fp4.h"

namespace asym {
namespace {

constexpr int kWaves = 4;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct KvParams {
  const uint16_t *k, *v;       // write: tokens [T][H][128], strides below
  uint16_t *ko, *vo;           // read: [T][H][128]
  int64_t k_tok, k_head, v_tok, v_head;
  uint8_t *k_pool, *v_pool;
  const int *k_pages, *v_pages;  // [B][H][pph]
  const int *cu, *start;
  int B, H, T, pph, pool_pages, ranks;
};

// The rank-th page that the call touches, over the sequences in order: its sequence,
// its place in the sequence's tables, the sequence's first row and position, and its
// tokens [lo, hi) of the page.  One wave.
__device__ bool find_page(const KvParams& p, int rank, int& seq, int& page, int& row, int& lo, int& hi) {
  const int lane = threadIdx.x & 63;
  for (int c = 0; 64 * c < p.B; ++c) {
    const int b = 64 * c + lane;
    int s = 0, n = 0, at = 0, pages = 0;
    if (b < p.B) {
      packed_rows(p.cu, b, p.T, s, n);
      at = p.start[b];
      // positions before 0 or behind the tables have no page
      const int64_t cap = (int64_t)p.pph * kKvPageTokens;
      if (at < 0 || n < 1 || at >= cap) n = 0;
      n = (int)min((int64_t)n, cap - at);
      if (n > 0) pages = (at + n - 1) / kKvPageTokens - at / kKvPageTokens + 1;
    }
    const int upto = wave_scan_add(pages);
    const unsigned long long in = __ballot(rank < upto);
    if (in) {
      const int l = __builtin_ctzll(in);
      seq = 64 * c + l;
      const int first = __builtin_amdgcn_readlane(upto - pages, l);
      at = __builtin_amdgcn_readlane(at, l);
      n = __builtin_amdgcn_readlane(n, l);
      s = __builtin_amdgcn_readlane(s, l);
      page = at / kKvPageTokens + (rank - first);
      lo = max(at - page * kKvPageTokens, 0);
      hi = min(at + n - page * kKvPageTokens, kKvPageTokens);
      row = s + page * kKvPageTokens - at;  // of the page's token 0
      return true;
    }
    rank -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// largest magnitude's bits over a group of 4 lanes; an infinity or a NaN stays the largest
__device__ __forceinline__ uint32_t max4(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));  // quad_perm 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));  // quad_perm 2 3 0 1
}

__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {  // of a block's largest magnitude (bf16 bits)
  const uint32_t e = top >> 7;
  return e == 255u ? 255u : max(e, 4u) - 2u;
}

// two bf16 -> two codes in byte `sel` of a word (the hardware rounds to nearest even
// and saturates, as the format says)
template <int SEL>
__device__ __forceinline__ uint32_t codes2(uint32_t old, uint32_t pair, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, pair), scale, SEL);
}
__device__ __forceinline__ uint32_t codes8(u32x4 x, uint32_t s) {
  if (s == 255u) return 0u;
  const float f = __uint_as_float(s << 23);
  uint32_t w = codes2<0>(0u, x[0], f);
  w = codes2<1>(w, x[1], f);
  w = codes2<2>(w, x[2], f);
  return codes2<3>(w, x[3], f);
}

__global__ void __launch_bounds__(64 * kWaves) kv_write_kernel(KvParams p) {
  __shared__ uint32_t tile[kWaves][kKvPageTokens][17];  // codes of 32 tokens (16 words each, one of padding)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x * kWaves + wave;
  const int head = item % p.H;
  int seq, page, row, lo, hi;
  const bool any = item / p.H < p.ranks && find_page(p, item / p.H, seq, page, row, lo, hi);
  if (!any) return;  // (no barriers below: LDS is the wave's own)
  const size_t entry = ((size_t)seq * p.H + head) * p.pph + page;
  const int kp = __builtin_amdgcn_readfirstlane(p.k_pages[entry]), vp = __builtin_amdgcn_readfirstlane(p.v_pages[entry]);
  const int c16 = lane & 15, t4 = lane >> 4;  // 8 channels, one of four tokens
  const bool k_on = kp >= 0 && kp < p.pool_pages, v_on = vp >= 0 && vp < p.pool_pages;
  uint8_t* kd = p.k_pool + (size_t)(k_on ? kp : 0) * kFp4PageBytes;
  uint8_t* vd = p.v_pool + (size_t)(v_on ? vp : 0) * kFp4PageBytes;
  // lane (m, q) of the value page: 8 words, of channels 16 g + m, tokens 4 q + 0 .. 3 and
  // 16 + 4 q + 0 .. 3; nibbles of tokens that are not written stay
  uint32_t keep = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = 4 * t4 + (j & 3) + 16 * (j >> 2);
    if (t < lo || t >= hi) keep |= 0xFu << (4 * j);
  }
  const bool some = v_on && keep != 0xFFFFFFFFu;
  u32x4 old[2] = {};
  if (some && keep) {
#pragma unroll
    for (int i = 0; i < 2; ++i) old[i] = *reinterpret_cast<const u32x4*>(vd + 1024 * i + 16 * lane);
  }
  auto block_scale = [](u32x4 x) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(x[e] & 0x7FFFu, (x[e] >> 16) & 0x7FFFu));
    return scale_byte(max4(top));
  };
  // 16 tokens at a time, their loads all at once
#pragma unroll 1
  for (int t0 = 0; t0 < kKvPageTokens; t0 += 16) {
    if (t0 + 16 <= lo || t0 >= hi) continue;
    u32x4 xk[4], xv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + 4 * i + t4;
      xk[i] = xv[i] = u32x4{};
      if (t >= lo && t < hi) {
        xk[i] = *reinterpret_cast<const u32x4*>(p.k + (int64_t)(row + t) * p.k_tok + (int64_t)head * p.k_head + 8 * c16);
        xv[i] = *reinterpret_cast<const u32x4*>(p.v + (int64_t)(row + t) * p.v_tok + (int64_t)head * p.v_head + 8 * c16);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + 4 * i + t4, u = 4 * i + t4;  // u = t % 16
      const bool on = t >= lo && t < hi;
      uint32_t s = block_scale(xk[i]);
      if (on && k_on) {
        *reinterpret_cast<uint32_t*>(kd + 64 * t + 4 * c16) = codes8(xk[i], s);
        if ((c16 & 3) == 0) kd[kFp4ScaleOff + 2 * (u + 16 * (c16 >> 2)) + (t0 >> 4)] = (uint8_t)s;
      }
      s = block_scale(xv[i]);
      tile[wave][t][c16] = codes8(xv[i], s);
      if (on && v_on && (c16 & 3) == 0)
        vd[kFp4ScaleOff + 32 * (u >> 2) + 4 * ((u & 3) + (t0 >> 2)) + (c16 >> 2)] = (uint8_t)s;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  if (some) {
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = 4 * t4 + (j & 3) + 16 * (j >> 2), c = 16 * g + c16;
        w |= ((tile[wave][t][c >> 3] >> (4 * (c & 7))) & 0xFu) << (4 * j);
      }
      old[g >> 2][g & 3] = (w & ~keep) | (old[g >> 2][g & 3] & keep);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4*>(vd + 1024 * i + 16 * lane) = old[i];
  }
}

// 8 codes of one scale -> 8 bf16
__device__ __forceinline__ u32x4 values8(uint32_t w, uint32_t s) {
  const float f = __uint_as_float(s == 255u ? 0x7FC00000u : s << 23);
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3));
  return x;
}

__global__ void __launch_bounds__(64 * kWaves) kv_read_kernel(KvParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x * kWaves + wave;
  const int head = item % p.H;
  int seq, page, row, lo, hi;
  if (item / p.H >= p.ranks || !find_page(p, item / p.H, seq, page, row, lo, hi)) return;
  const size_t entry = ((size_t)seq * p.H + head) * p.pph + page;
  const int kp = __builtin_amdgcn_readfirstlane(p.k_pages[entry]), vp = __builtin_amdgcn_readfirstlane(p.v_pages[entry]);
  const __amdgpu_buffer_rsrc_t rk = page_rsrc(p.k_pool, kp, p.pool_pages), rv = page_rsrc(p.v_pool, vp, p.pool_pages);
  const int n = lane & 15, q = lane >> 4;
  // keys: lane (token n of either half, block q) has 32 channels
  u32x4 kc[2], vc[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    kc[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, 1024 * t + 64 * n + 16 * q, 0, 0));
    vc[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, 1024 * t + 16 * lane, 0, 0));
  }
  uint32_t kscale[4];  // of block i, token n of either half, one a byte
#pragma unroll
  for (int i = 0; i < 4; ++i) kscale[i] = __builtin_amdgcn_raw_buffer_load_b16(rk, kFp4ScaleOff + 2 * (n + 16 * i), 0, 0);
  uint32_t vscale[2];  // of token n of either half: 4 blocks, one a byte
#pragma unroll
  for (int t = 0; t < 2; ++t)
    vscale[t] = __builtin_amdgcn_raw_buffer_load_b32(rv, kFp4ScaleOff + 32 * (n >> 2) + 4 * ((n & 3) + 4 * t), 0, 0);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    // codes of 8 channels exchanged between a token's four lanes (a 4 x 4 transpose):
    // word i of lane q then belongs to channels 32 i + 8 q, and a store fills 64 bytes of a row
    const auto x = __builtin_amdgcn_permlane16_swap(kc[t][0], kc[t][1], false, false);
    const auto y = __builtin_amdgcn_permlane16_swap(kc[t][2], kc[t][3], false, false);
    const auto even = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
    const auto odd = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
    const u32x4 c = {even[0], odd[0], even[1], odd[1]};
    const int tok = 16 * t + n;
    if (tok < lo || tok >= hi) continue;
    u32x4* dst = reinterpret_cast<u32x4*>(p.ko + ((int64_t)(row + tok) * p.H + head) * kKvD + 8 * q);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[4 * i] = values8(c[i], (kscale[i] >> (8 * t)) & 0xFFu);
  }
  // values: the page has them channel by channel; a matrix product with the tokens' scales
  // on a diagonal turns them (exact: every sum has one term).  Column n is token 16 t + n,
  // which lies in slot (n % 4) + 4 t of quarter n / 4.
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int tok = 16 * t + n;
    const bool on = tok >= lo && tok < hi;
    u32x4* dst = reinterpret_cast<u32x4*>(p.vo + ((int64_t)(row + tok) * p.H + head) * kKvD + 16 * (q & 1) + 8 * (q >> 1));
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
      const uint32_t sb = (vscale[t] >> (8 * blk)) & 0xFFu;
      // (a power of two, or NaN, as bf16)
      const uint32_t h = q == (n >> 2) ? (sb == 255u ? 0x7FC0u : sb << 7) : 0u;
      u32x4 d = {};
#pragma unroll
      for (int w = 0; w < 2; ++w)
        d[2 * t + w] = (n & 3) >> 1 == w ? ((n & 1) ? h << 16 : h) : 0u;
      uint32_t o[4];  // 4 channels of group 2 blk, 4 of group 2 blk + 1
#pragma unroll
      for (int g2 = 0; g2 < 2; ++g2) {
        const int g = 2 * blk + g2;
        const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, values8(vc[g >> 2][g & 3], 127u)), __builtin_bit_cast(bf16x8, d), f32x4{}, 0, 0, 0);
        const bf16x2 y0 = {(__bf16)x[0], (__bf16)x[1]}, y1 = {(__bf16)x[2], (__bf16)x[3]};
        o[2 * g2] = __builtin_bit_cast(uint32_t, y0);
        o[2 * g2 + 1] = __builtin_bit_cast(uint32_t, y1);
      }
      // quarter 0: channels 0 .. 7 of the first group, 1: of the second, 2 and 3: 8 .. 15
      const auto x = __builtin_amdgcn_permlane16_swap(o[0], o[2], false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(o[1], o[3], false, false);
      if (on) dst[4 * blk] = u32x4{x[0], y[0], x[1], y[1]};
    }
  }
}

int kv_check(const char* what, int B, int H, int T, int pph, size_t pool_pages, const void* k_pool, const void* v_pool,
             const void* k_pages, const void* v_pages, const void* cu, const void* start) {
  const std::string w(what);
  if (B < 0 || T < 0 || H < 1 || pph < 1) return fail(ASYM_EINVAL, w + ": B and T must be >= 0, H and pages_per_head >= 1");
  if (pool_pages < 1 || pool_pages > 0x7FFFFFFFu) return fail(ASYM_EINVAL, w + ": pool_pages must be in [1, 2^31)");
  if (pph > (1 << 25)) return fail(ASYM_EUNSUPPORTED, w + ": more than 2^30 tokens a request");
  if (B == 0 || T == 0) return ASYM_OK;
  if (!k_pool || !v_pool || !k_pages || !v_pages || !cu || !start) return fail(ASYM_EINVAL, w + ": null pointer");
  if (((uintptr_t)k_pool | (uintptr_t)v_pool) & 15u) return fail(ASYM_EINVAL, w + ": pools must be 16-byte aligned");
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)cu | (uintptr_t)start) & 3u)
    return fail(ASYM_EINVAL, w + ": tables, offsets and positions must be 4-byte aligned");
  return ASYM_OK;
}

// n tokens from any position touch at most n / 32 + 2 pages: ranks, and the grid of a
// wave per (rank, head)
int kv_grid(const char* what, KvParams& p, unsigned* grid) {
  const int64_t ranks = (int64_t)p.T / kKvPageTokens + 2ll * p.B;
  const int64_t items = ranks * p.H;
  if (items > (1 << 26) - kWaves) return  // (threads of a launch are counted in 32 bits)
    fail(ASYM_EUNSUPPORTED, std::string(what) + ": too many pages");
  p.ranks = (int)ranks;
  *grid = (unsigned)((items + kWaves - 1) / kWaves);
  return ASYM_OK;
}

}  // namespace
}  // namespace asym

extern "C" int asym_kv_write_fp4(int B, int H_kv, int T, const void* k, int64_t k_token, int64_t k_head, const void* v,
                                 int64_t v_token, int64_t v_head, void* k_pool, void* v_pool, size_t pool_pages,
                                 const int32_t* k_pages, const int32_t* v_pages, int pages_per_head, const int32_t* cu,
                                 const int32_t* start, void* stream) {
  using namespace asym;
  int rc = kv_check("kv write", B, H_kv, T, pages_per_head, pool_pages, k_pool, v_pool, k_pages, v_pages, cu, start);
  if (rc != ASYM_OK) return rc;
  if (B == 0 || T == 0) return ASYM_OK;
  if (!k || !v) return fail(ASYM_EINVAL, "kv write: null pointer");
  if (((uintptr_t)k | (uintptr_t)v) & 15u) return fail(ASYM_EINVAL, "kv write: K and V must be 16-byte aligned");
  for (int64_t s : {k_token, k_head, v_token, v_head})
    if (s < 0 || s % 8) return fail(ASYM_EINVAL, "kv write: strides must be multiples of 8 values and not negative");
  KvParams p = {};
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.k_tok = k_token; p.k_head = k_head; p.v_tok = v_token; p.v_head = v_head;
  p.k_pool = static_cast<uint8_t*>(k_pool);
  p.v_pool = static_cast<uint8_t*>(v_pool);
  p.k_pages = k_pages; p.v_pages = v_pages; p.cu = cu; p.start = start;
  p.B = B; p.H = H_kv; p.T = T; p.pph = pages_per_head; p.pool_pages = (int)pool_pages;
  unsigned grid;
  rc = kv_grid("kv write", p, &grid);
  if (rc != ASYM_OK) return rc;
  hipLaunchKernelGGL(kv_write_kernel, dim3(grid), dim3(64 * kWaves), 0, static_cast<hipStream_t>(stream), p);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}

extern "C" int asym_kv_read_fp4(int B, int H_kv, int T, const void* k_pool, const void* v_pool, size_t pool_pages,
                                const int32_t* k_pages, const int32_t* v_pages, int pages_per_head, const int32_t* cu,
                                const int32_t* start, void* k, void* v, void* stream) {
  using namespace asym;
  int rc = kv_check("kv read", B, H_kv, T, pages_per_head, pool_pages, k_pool, v_pool, k_pages, v_pages, cu, start);
  if (rc != ASYM_OK) return rc;
  if (B == 0 || T == 0) return ASYM_OK;
  if (!k || !v) return fail(ASYM_EINVAL, "kv read: null pointer");
  if (((uintptr_t)k | (uintptr_t)v) & 15u) return fail(ASYM_EINVAL, "kv read: K and V must be 16-byte aligned");
  KvParams p = {};
  p.ko = static_cast<uint16_t*>(k);
  p.vo = static_cast<uint16_t*>(v);
  p.k_pool = static_cast<uint8_t*>(const_cast<void*>(k_pool));
  p.v_pool = static_cast<uint8_t*>(const_cast<void*>(v_pool));
  p.k_pages = k_pages; p.v_pages = v_pages; p.cu = cu; p.start = start;
  p.B = B; p.H = H_kv; p.T = T; p.pph = pages_per_head; p.pool_pages = (int)pool_pages;
  unsigned grid;
  rc = kv_grid("kv read", p, &grid);
  if (rc != ASYM_OK) return rc;
  hipLaunchKernelGGL(kv_read_kernel, dim3(grid), dim3(64 * kWaves), 0, static_cast<hipStream_t>(stream), p);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
