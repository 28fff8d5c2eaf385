// Decode attention over a paged cache in microscaled 4-bit floating point (format
// and page layout: kv_fp4.h), one query token per request, a length per request:
//
//   O[b, h] = softmax_t(scale * <q[b, h], K[b, g, t]>) . V[b, g, :],  t < lens[b], g = h / G
//
// The sequence is cut into splits; a wave has one (request, key/value head, split) and
// serves the G <= 16 query heads that read that head, 32 tokens (a page) at a time:
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
// No LDS, no barrier.  Each split leaves its unnormalised output, max and sum in fp32
// for the second launch; with one split the wave writes the result itself.
#include <hip/hip_runtime.h>

#include <cmath>

#include "internal.h"
#include "kv_fp4.h"

namespace asym {
namespace {

constexpr int kWaves = 4;
constexpr int kMaxG = 16;
constexpr int kMaxSplitPages = 64;  // a lane holds the number of one page of the split

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
  float* part_o;                 // [B][Hq][n_splits][128]
  float* part_ml;                // [B][Hq][n_splits][2]: max (of the raw scores), sum
  int B, Hq, Hkv, G, S, pph, pool_pages;
  int split_pages, n_splits, tasks;
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

__device__ __forceinline__ void load_page(const Fp4DecodeParams& p, int kp, int vp, int lane, PageRegs& r) {
  const __amdgpu_buffer_rsrc_t rk = page_rsrc(p.k_pool, kp, p.pool_pages), rv = page_rsrc(p.v_pool, vp, p.pool_pages);
  const uint32_t ko = (uint32_t)((lane & 15) * 64 + (lane >> 4) * 16);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    r.k[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, ko + 1024 * t, 0, 0));
    r.v[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, (uint32_t)lane * 16 + 1024 * t, 0, 0));
    r.vs[t] = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, kFp4ScaleOff + (uint32_t)(lane >> 4) * 32 + 16 * t, 0, 0));
  }
  r.ks = __builtin_amdgcn_raw_buffer_load_b16(rk, kFp4ScaleOff + (uint32_t)lane * 2, 0, 0);
}

__global__ void __launch_bounds__(64 * kWaves) fp4_decode_split(Fp4DecodeParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int task = blockIdx.x * kWaves + wave;
  if (task >= p.tasks) return;
  const int split = task % p.n_splits, bh = task / p.n_splits;
  const int b = bh / p.Hkv, hk = bh - b * p.Hkv;
  const int len = __builtin_amdgcn_readfirstlane(min(max(p.lens[b], 0), p.S));
  const int pg0 = split * p.split_pages;
  const int n_pg = min((len + kKvPageTokens - 1) / kKvPageTokens - pg0, p.split_pages);
  if (n_pg <= 0 && (p.n_splits > 1 || split > 0)) return;  // (the merge knows the lengths)
  const int n = lane & 15, quarter = lane >> 4;

  int kpg = -1, vpg = -1;
  if (lane < n_pg) {
    const size_t e = (size_t)bh * p.pph + pg0 + lane;
    kpg = p.k_pages[e];
    vpg = p.v_pages[e];
  }
  i32x8 q_hi, q_lo;
  int s_hi, s_lo;
  const int head = hk * p.G + n;  // this lane's query head
  load_q(p.q + ((size_t)b * p.Hq + (n < p.G ? head : 0)) * kKvD, n < p.G, quarter, p.q_flip, q_hi, q_lo, s_hi, s_lo);

  f32x4 o[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) o[g] = f32x4{};
  float m = -INFINITY, l = 0.f;
  PageRegs cur, nxt;
  if (n_pg > 0)
    load_page(p, __builtin_amdgcn_readlane(kpg, 0), __builtin_amdgcn_readlane(vpg, 0), lane, cur);
  for (int i = 0; i < n_pg; ++i) {
    const int ni = min(i + 1, n_pg - 1);  // (the last page again: no branch around the loads)
    load_page(p, __builtin_amdgcn_readlane(kpg, ni), __builtin_amdgcn_readlane(vpg, ni), lane, nxt);
    const int left = len - (pg0 + i) * kKvPageTokens;
    // scores: rows 4 quarter + r of tokens 16 t .., column n
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const i32x8 a = {(int)cur.k[t][0], (int)cur.k[t][1], (int)cur.k[t][2], (int)cur.k[t][3], 0, 0, 0, 0};
      const int ks = (int)(cur.ks >> (8 * t));
      s[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q_lo, f32x4{}, 4, 0, 0, ks, 0, s_lo);
      s[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q_hi, s[t], 4, 0, 0, ks, 0, s_hi);
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
    if (__any((top - m) * p.c > 8.f)) {
      const float m_new = fmaxf(m, top);
      const float alpha = __builtin_amdgcn_exp2f((m - (m_new == -INFINITY ? 0.f : m_new)) * p.c);
      l *= alpha;
#pragma unroll
      for (int g = 0; g < 8; ++g) o[g] *= alpha;
      m = m_new;
    }
    const float ms = m == -INFINITY ? 0.f : m * p.c;
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      e[j] = __builtin_amdgcn_exp2f(fmaf(s[j >> 2][j & 3], p.c, -ms));
      l += e[j];
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
        o[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, pf, o[g], 0, 0, 0);
      }
    }
    cur = nxt;
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (n >= p.G) return;
  const size_t row = (size_t)b * p.Hq + head;
  if (p.n_splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* dst = p.o + row * kKvD + 4 * quarter;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      const bf16x2 a = {(__bf16)(o[g][0] * inv), (__bf16)(o[g][1] * inv)}, c = {(__bf16)(o[g][2] * inv), (__bf16)(o[g][3] * inv)};
      *reinterpret_cast<uint2*>(dst + 16 * g) = uint2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
    }
    if (p.lse && quarter == 0) p.lse[row] = l == 0.f ? -INFINITY : m * p.scale + __logf(l);
    return;
  }
  float* dst = p.part_o + (row * p.n_splits + split) * kKvD + 4 * quarter;
#pragma unroll
  for (int g = 0; g < 8; ++g) *reinterpret_cast<f32x4*>(dst + 16 * g) = o[g];
  if (quarter == 0) {
    float* ml = p.part_ml + (row * p.n_splits + split) * 2;
    ml[0] = m;
    ml[1] = l;
  }
}

// Merge: a workgroup has one (request, head) row; wave w takes splits w, w + 4, ... of
// those that the request's length reaches, in an order fixed by the length.
__global__ void __launch_bounds__(64 * kWaves) fp4_decode_merge(Fp4DecodeParams p) {
  __shared__ float red[kWaves][kKvD], red_l[kWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t row = blockIdx.x;
  const int b = (int)(row / p.Hq);
  const int len = min(max(p.lens[b], 0), p.S);
  const int per = p.split_pages * kKvPageTokens, ns = (len + per - 1) / per;
  const float* ml = p.part_ml + row * p.n_splits * 2;
  const float* po = p.part_o + row * p.n_splits * kKvD + 2 * lane;
  float M = -INFINITY;
  for (int s = lane; s < ns; s += 64) M = fmaxf(M, ml[2 * s]);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
  float a0 = 0.f, a1 = 0.f, L = 0.f;
  for (int s = wave; s < ns; s += kWaves) {
    const float w = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ml[2 * s] - M) * p.c);  // (no finite score: NaN comes through)
    const float2 x = *reinterpret_cast<const float2*>(po + (size_t)s * kKvD);
    L = fmaf(ml[2 * s + 1], w, L);
    a0 = fmaf(x.x, w, a0);
    a1 = fmaf(x.y, w, a1);
  }
  red[wave][2 * lane] = a0;
  red[wave][2 * lane + 1] = a1;
  if (lane == 0) red_l[wave] = L;
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < kWaves; ++w) {
    a0 += red[w][2 * lane];
    a1 += red[w][2 * lane + 1];
    L += red_l[w];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const bf16x2 r = {(__bf16)(a0 * inv), (__bf16)(a1 * inv)};
  *reinterpret_cast<uint32_t*>(p.o + row * kKvD + 2 * lane) = __builtin_bit_cast(uint32_t, r);
  if (p.lse && lane == 0) p.lse[row] = L == 0.f ? -INFINITY : M * p.scale + __logf(L);
}

// The split: the longest power-of-two number of pages, up to 32, that still gives 2048
// waves at the longest length.
int fp4_plan(int B, int Hq, int Hkv, int S, int D, int split_tokens, asym_attn_plan_info* out) {
  if (B < 0 || Hq < 1 || Hkv < 1 || S < 1) return fail(ASYM_EINVAL, "fp4 attention: B must be >= 0, H_q, H_kv and S_max >= 1");
  if (Hq % Hkv) return fail(ASYM_EINVAL, "fp4 attention: H_kv must divide H_q");
  if (Hq / Hkv > kMaxG) return fail(ASYM_EUNSUPPORTED, "fp4 attention: at most 16 query heads per key/value head");
  if (D != kKvD) return fail(ASYM_EUNSUPPORTED, "fp4 attention: the head dimension must be 128");
  if (S > (1 << 30)) return fail(ASYM_EUNSUPPORTED, "fp4 attention: S_max above 2^30");
  if (split_tokens < 0 || split_tokens % kKvPageTokens || split_tokens > kMaxSplitPages * kKvPageTokens)
    return fail(ASYM_EINVAL, "fp4 attention: split_tokens must be 0 (automatic) or a multiple of 32 up to 2048");
  const int64_t heads = (int64_t)B * Hkv;
  int L = split_tokens;
  if (!L) {
    L = 1024;
    while (L > kKvPageTokens && heads * ((S + L - 1) / L) < 2048) L /= 2;
  }
  const int64_t n = ((int64_t)S + L - 1) / L, tasks = heads * n;
  if (tasks > (1 << 26) - kWaves || (int64_t)B * Hq >= (1 << 24))  // (threads of a launch are counted in 32 bits)
    return fail(ASYM_EUNSUPPORTED, "fp4 attention: too many tasks");
  *out = asym_attn_plan_info{};
  out->split_tokens = L;
  out->n_splits = (int)n;
  out->tasks = (int)tasks;
  out->grid = (int)((tasks + kWaves - 1) / kWaves);
  out->tasks_per_workgroup = kWaves;
  out->workspace_bytes = n > 1 ? (size_t)B * Hq * n * (kKvD + 2) * sizeof(float) : 0;
  return ASYM_OK;
}

}  // namespace
}  // namespace asym

extern "C" int asym_attn_decode_paged_fp4_plan(int B, int H_q, int H_kv, int S_max, int D, int split_tokens,
                                               asym_attn_plan_info* out) {
  if (!out) return asym::fail(ASYM_EINVAL, "fp4 attention plan: null output");
  return asym::fp4_plan(B, H_q, H_kv, S_max, D, split_tokens, out);
}

extern "C" int asym_attn_decode_paged_fp4(int B, int H_q, int H_kv, int S_max, int D, const void* q, const void* k_pool,
                                          const void* v_pool, size_t pool_pages, const int32_t* k_pages,
                                          const int32_t* v_pages, int pages_per_head, const int32_t* lens, void* o,
                                          float* lse, float scale, int split_tokens, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  using namespace asym;
  asym_attn_plan_info plan;
  int rc = fp4_plan(B, H_q, H_kv, S_max, D, split_tokens, &plan);
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
  p.part_ml = p.part_o ? p.part_o + (size_t)B * H_q * plan.n_splits * kKvD : nullptr;
  p.B = B; p.Hq = H_q; p.Hkv = H_kv; p.G = H_q / H_kv; p.S = S_max; p.pph = pages_per_head;
  p.pool_pages = (int)pool_pages;
  p.split_pages = plan.split_tokens / kKvPageTokens;
  p.n_splits = plan.n_splits;
  p.tasks = plan.tasks;
  p.scale = std::fabs(scale);
  p.c = std::fmax(p.scale * 1.4426950408889634f, 1.17549435e-38f);  // (0 weighs all keys alike, a masked one not at all)
  p.q_flip = scale < 0 ? 0x80008000u : 0u;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(fp4_decode_split, dim3((unsigned)plan.grid), dim3(64 * kWaves), 0, s, p);
  ASYM_HIP(hipGetLastError());
  if (plan.n_splits > 1) {
    hipLaunchKernelGGL(fp4_decode_merge, dim3((unsigned)((size_t)B * H_q)), dim3(64 * kWaves), 0, s, p);
    ASYM_HIP(hipGetLastError());
  }
  return ASYM_OK;
}
