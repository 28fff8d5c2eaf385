// Rotary positions, alone and on the way into a 16-bit paged cache.
//
// The first `rotary` channels of a row are pairs (a, b): channels j and j + rotary / 2 (half
// layout) or 2 j and 2 j + 1 (interleaved).  With t = position * freq[j],
//
//   a' = A (a cos t - b sin t),  b' = A (b cos t + a sin t),
//
// A an amplitude that long-context scalings ask for; the gradient is the same with -t.  The
// other channels are copied.  The angle is taken in 64 bits, as turns, and its whole turns
// dropped there: a position of 10^6 has 2^20 radians at the first pair, of which 32 bits
// would keep 2^-4.  cos, sin and the two products are 32 bits, rounded to bf16 once.
//
// A thread has one unit of a row: two runs of E channels that hold E whole pairs (half: E
// of either half; interleaved: 2 E neighbours), or 2 E that are copied.  E is 8 (16-byte
// loads) where rotary and the row are multiples of 16, 4 where they are of 8, else 1.  A
// workgroup has the units of one token (or of a few, where a token has few), so that the
// cosines of a token are computed once for it, a pair a thread, in LDS, while the rows' loads
// are on their way.
//
// Bound by HBM: the gradient of 16384 tokens of 32 heads takes 48 us, 5.6 TB/s (a plain copy 4.8 to 5.4); with runs of 4 (104
// of the channels turned) 49 to 50, of 1 (6 turned) 119 to 126, bound by the number of its loads.  64 tokens of 128 heads
// of 64 channels 3.4, as short launches do.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "kv_fp4.h"

namespace asym {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxD = 1024;
constexpr int kPageRow = kKvD * 2;                       // bytes of a token in a page
constexpr int64_t kPageBytes = kKvPageTokens * kPageRow;  // of a page

struct Turn {
  const double* freq;  // [rotary / 2]
  int rotary;
  float amp;           // amplitude
  float dir;           // 1, or -1 for the gradient
};

template <int E>
struct alignas(2 * E) Run {
  uint16_t x[E];
};

__device__ __forceinline__ float up(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t down(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// (A cos, A sin) of one pair, the sine's sign that of the direction
__device__ __forceinline__ float2 cos_sin(const Turn& r, int pair, double pos) {
  const double each = r.freq[pair] * 0.15915494309189535;  // turns a position
  const double t = __builtin_fma(pos, each, -__builtin_rint(pos * each));
  float s, c;
  sincospif(2.f * (float)t, &s, &c);
  return float2{c * r.amp, s * r.amp * r.dir};
}

// Where the two runs of unit c of a row begin
template <int E, bool INTER>
__device__ __forceinline__ void runs_of(int c, int rotary, int& a, int& b) {
  const int turned = rotary / (2 * E);
  if (INTER || c >= turned) {
    a = 2 * E * c;
    b = a + E;
  } else {
    a = E * c;
    b = a + rotary / 2;
  }
}
// cs: of the unit's E pairs.  (Which product is rounded is written out: left to the compiler, it differed between the kernels and
// between a unit's pairs, and a key appended with 4096 tokens or more from the same one appended alone, 8 of a million.)
template <int E, bool INTER>
__device__ __forceinline__ void turn_unit(Run<E>& a, Run<E>& b, const float2* cs) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    // (interleaved: pair e is values 2 e and 2 e + 1 of the two runs in order)
    const int i = INTER ? 2 * e : e, j = INTER ? 2 * e + 1 : E + e;
    uint16_t& x = i < E ? a.x[i] : b.x[i - E];
    uint16_t& y = j < E ? a.x[j] : b.x[j - E];
    const float u = up(x), v = up(y);
    x = down(fmaf(u, cs[e].x, -(v * cs[e].y)));
    y = down(fmaf(v, cs[e].x, u * cs[e].y));
  }
}

struct RopeParams {
  const uint16_t* x;
  uint16_t* y;
  int64_t x_tok, x_head, y_tok, y_head;
  const int* pos;
  Turn turn;
  int T, H, units;  // units of a row
  int tokens;       // of a workgroup
  int parts;        // workgroups of a token
};

template <int E, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeParams p) {
  __shared__ float2 cs[kThreads * 8];  // [tokens][rotary / 2]
  const int t0 = (int)(blockIdx.x / p.parts) * p.tokens, part = (int)(blockIdx.x % p.parts);
  const int each = p.H * p.units;  // units of a token
  const int id = part * kThreads + (int)threadIdx.x;
  const int k = id / each, in = id - k * each;  // (parts > 1: one token)
  const int t = t0 + k, h = in / p.units, c = in - h * p.units;
  const bool on = k < p.tokens && t < p.T;
  int a = 0, b = 0;
  Run<E> u, v;
  if (on) {
    runs_of<E, INTER>(c, p.turn.rotary, a, b);
    const uint16_t* row = p.x + (int64_t)t * p.x_tok + (int64_t)h * p.x_head;
    u = *reinterpret_cast<const Run<E>*>(row + a);
    v = *reinterpret_cast<const Run<E>*>(row + b);
  }
  const int pairs = p.turn.rotary / 2;
  for (int i = threadIdx.x; i < p.tokens * pairs; i += kThreads) {
    const int q = i / pairs;
    if (t0 + q < p.T) cs[i] = cos_sin(p.turn, i - q * pairs, p.pos[t0 + q]);
  }
  __syncthreads();
  if (!on) return;
  if (E * c < pairs) turn_unit<E, INTER>(u, v, cs + k * pairs + E * c);
  uint16_t* row = p.y + (int64_t)t * p.y_tok + (int64_t)h * p.y_head;
  *reinterpret_cast<Run<E>*>(row + a) = u;
  *reinterpret_cast<Run<E>*>(row + b) = v;
}

struct AppendParams {
  const uint16_t *q, *k, *v;
  uint16_t* qo;
  int64_t q_tok, q_head, qo_tok, qo_head, k_tok, k_head, v_tok, v_head;
  uint8_t *k_pool, *v_pool;
  const int *k_pages, *v_pages;  // [B][Hkv][pph]
  const int *cu, *start, *pos;
  Turn turn;
  int B, Hq, Hkv, T, pph, pool_pages;
  int tokens, parts;
};

// A workgroup has kAppend units at most, and SLOTS tokens of that many one after the other: a thread's loads of all of them
// are on their way at once.
// us at 1, 2 and 4, 32 / 8 heads: 16381 tokens 82.2 78.3 (5.1 TB/s; a plain copy 5.0 to 5.4) 83.6, 2000 tokens 12.9 13.1
// 13.6; with a token a workgroup of 256 threads, twice where it has more units, 91.8 and 14.0.
constexpr int kAppend = 512;
constexpr int kSlots = 2;  // where there are enough tokens for every CU
constexpr int kMostTokens = 4 * kSlots;  // of a workgroup

template <int E, bool INTER, int SLOTS>
__global__ void __launch_bounds__(kAppend) kv_append_kernel(AppendParams p) {
  constexpr int units = kKvD / (2 * E);
  __shared__ float2 cs[kMostTokens * (kKvD / 2)];
  __shared__ int seq_of[kMostTokens];      // a token's request (-1: it has none)
  __shared__ int64_t at_of[kMostTokens];  // its place in the cache
  const int t0 = (int)(blockIdx.x / p.parts) * p.tokens * SLOTS, part = (int)(blockIdx.x % p.parts);
  const int heads = p.Hq + 2 * p.Hkv, each = heads * units;
  const int id = part * (int)blockDim.x + (int)threadIdx.x;
  const int k = id / each, in = id - k * each;  // (parts > 1: one token)
  const int hh = in / units, c = in - hh * units;
  const int kind = hh < p.Hq ? 0 : hh < p.Hq + p.Hkv ? 1 : 2;  // query, key, value
  const int h = kind == 0 ? hh : kind == 1 ? hh - p.Hq : hh - p.Hq - p.Hkv;
  int a, b;
  runs_of<E, INTER>(c, p.turn.rotary, a, b);
  const uint16_t* from = kind == 0   ? p.q + (int64_t)h * p.q_head
                         : kind == 1 ? p.k + (int64_t)h * p.k_head
                                     : p.v + (int64_t)h * p.v_head;
  const int64_t tok = kind == 0 ? p.q_tok : kind == 1 ? p.k_tok : p.v_tok;
  Run<E> u[SLOTS], v[SLOTS];
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    const int t = t0 + s * p.tokens + k;
    if (k < p.tokens && t < p.T) {
      u[s] = *reinterpret_cast<const Run<E>*>(from + t * tok + a);
      v[s] = *reinterpret_cast<const Run<E>*>(from + t * tok + b);
    }
  }
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int all = p.tokens * SLOTS;
  for (int j = wave; j < all; j += (int)blockDim.x / 64) {  // (a wave looks a token up)
    const int i = t0 + j;
    int seq = 0;  // requests that end at or before the token
    for (int r = 0; r < p.B; r += 64) {
      const bool before = r + lane < p.B && min(max(p.cu[min(r + lane, p.B - 1) + 1], 0), p.T) <= i;
      seq += __popcll(__ballot(before));
    }
    if (lane == 0) {
      int64_t at = -1;
      if (i < p.T && seq < p.B) {
        int s, n;
        packed_rows(p.cu, seq, p.T, s, n);
        const int first = p.start[seq];
        if (i >= s && i < s + n && first >= 0) at = (int64_t)first + (i - s);
      }
      seq_of[j] = at < 0 ? -1 : seq;
      at_of[j] = at;
    }
  }
  __syncthreads();
  const int pairs = p.turn.rotary / 2;
  for (int i = threadIdx.x; i < all * pairs; i += (int)blockDim.x) {
    const int q = i / pairs;
    if (seq_of[q] >= 0) cs[i] = cos_sin(p.turn, i - q * pairs, p.pos ? (double)p.pos[t0 + q] : (double)at_of[q]);
  }
  uint16_t* to[SLOTS];
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    to[s] = nullptr;
    const int j = s * p.tokens + k;
    if (k >= p.tokens || t0 + j >= p.T || seq_of[j] < 0) continue;
    const int64_t at = at_of[j];
    if (kind == 0) {
      to[s] = p.qo + (int64_t)(t0 + j) * p.qo_tok + (int64_t)h * p.qo_head;
    } else if (at < p.pph * (int64_t)kKvPageTokens) {
      const int64_t entry = ((int64_t)seq_of[j] * p.Hkv + h) * p.pph + at / kKvPageTokens;
      const int page = (kind == 1 ? p.k_pages : p.v_pages)[entry];
      if (page >= 0 && page < p.pool_pages)
        to[s] = reinterpret_cast<uint16_t*>((kind == 1 ? p.k_pool : p.v_pool) + page * kPageBytes + at % kKvPageTokens * kPageRow);
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    if (!to[s]) continue;
    if (kind < 2 && E * c < pairs) turn_unit<E, INTER>(u[s], v[s], cs + (s * p.tokens + k) * pairs + E * c);
    *reinterpret_cast<Run<E>*>(to[s] + a) = u[s];
    *reinterpret_cast<Run<E>*>(to[s] + b) = v[s];
  }
}

// Channels of a run: whole runs of pairs, and of what is copied
int run_of(int D, int rotary) { return D % 16 == 0 && rotary % 16 == 0 ? 8 : rotary % 8 == 0 ? 4 : 1; }

int turn_check(const char* what, int rotary, int D, const double* freq, int layout, float amplitude) {
  const std::string w(what);
  if (rotary < 0 || rotary > D || rotary % 2) return fail(ASYM_EINVAL, w + ": rotary must be even, from 0 to the head dimension");
  if (layout != ASYM_ROPE_HALF && layout != ASYM_ROPE_INTERLEAVED) return fail(ASYM_EINVAL, w + ": unknown layout");
  if (!std::isfinite(amplitude)) return fail(ASYM_EINVAL, w + ": the amplitude must be finite");
  if (rotary && (!freq || ((uintptr_t)freq & 7u))) return fail(ASYM_EINVAL, w + ": frequencies must be given, 8-byte aligned");
  return ASYM_OK;
}

bool bad_strides(std::initializer_list<int64_t> strides) {
  for (int64_t s : strides)
    if (s < 0 || s % 8) return true;
  return false;
}

// Output rows that lie on each other
bool rows_overlap(int T, int64_t token, int H, int64_t head, int D) {
  return (T > 1 && token < D) || (H > 1 && head < D) || (T > 1 && H > 1 && token == head);
}

template <class F>
void with_run(int e, bool inter, F f) {
  auto go = [&](auto E) { inter ? f(E, std::true_type{}) : f(E, std::false_type{}); };
  if (e == 8)
    go(std::integral_constant<int, 8>{});
  else if (e == 4)
    go(std::integral_constant<int, 4>{});
  else
    go(std::integral_constant<int, 1>{});
}

}  // namespace
}  // namespace asym

extern "C" int asym_rope_bf16(int T, int H, int D, int rotary, const void* x, int64_t x_token, int64_t x_head, void* y,
                              int64_t y_token, int64_t y_head, const int32_t* positions, const double* freq, int layout,
                              float amplitude, int backward, void* stream) {
  using namespace asym;
  if (T < 0 || H < 1) return fail(ASYM_EINVAL, "rope: T must be >= 0, H >= 1");
  if (H > (1 << 20)) return fail(ASYM_EUNSUPPORTED, "rope: too many heads");
  if (D < 8 || D % 8 || D > kMaxD) return fail(ASYM_EUNSUPPORTED, "rope: rows must have a multiple of 8 channels, at most 1024");
  int rc = turn_check("rope", rotary, D, freq, layout, amplitude);
  if (rc != ASYM_OK) return rc;
  if (T == 0) return ASYM_OK;
  if (!x || !y || !positions) return fail(ASYM_EINVAL, "rope: null pointer");
  if (((uintptr_t)x | (uintptr_t)y) & 15u) return fail(ASYM_EINVAL, "rope: x and y must be 16-byte aligned");
  if ((uintptr_t)positions & 3u) return fail(ASYM_EINVAL, "rope: positions must be 4-byte aligned");
  if (bad_strides({x_token, x_head, y_token, y_head}))
    return fail(ASYM_EINVAL, "rope: strides must be multiples of 8 values and not negative");
  if (rows_overlap(T, y_token, H, y_head, D)) return fail(ASYM_EINVAL, "rope: rows of y lie on each other");
  RopeParams p = {};
  p.x = static_cast<const uint16_t*>(x);
  p.y = static_cast<uint16_t*>(y);
  p.x_tok = x_token; p.x_head = x_head; p.y_tok = y_token; p.y_head = y_head;
  p.pos = positions;
  p.turn = Turn{freq, rotary, amplitude, backward ? -1.f : 1.f};
  p.T = T; p.H = H;
  const int e = run_of(D, rotary);
  p.units = D / (2 * e);
  const int64_t each = (int64_t)H * p.units;  // units of a token
  p.tokens = (int)std::max<int64_t>(1, std::min<int64_t>(32, kThreads / each));
  p.parts = (int)((each + kThreads - 1) / kThreads);
  const int64_t grid = ((int64_t)T + p.tokens - 1) / p.tokens * p.parts;
  if (grid >= (1 << 24)) return fail(ASYM_EUNSUPPORTED, "rope: too many rows");  // (threads are counted in 32 bits)
  with_run(e, layout == ASYM_ROPE_INTERLEAVED, [&](auto E, auto I) {
    hipLaunchKernelGGL((rope_kernel<decltype(E)::value, decltype(I)::value>), dim3((unsigned)grid), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), p);
  });
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}

extern "C" int asym_kv_append_bf16(int B, int H_q, int H_kv, int T, const void* q, int64_t q_token, int64_t q_head, void* q_out,
                                   int64_t qo_token, int64_t qo_head, const void* k, int64_t k_token, int64_t k_head,
                                   const void* v, int64_t v_token, int64_t v_head, void* k_pool, void* v_pool,
                                   size_t pool_pages, const int32_t* k_pages, const int32_t* v_pages, int pages_per_head,
                                   const int32_t* cu, const int32_t* start, const int32_t* positions, int rotary,
                                   const double* freq, int layout, float amplitude, void* stream) {
  using namespace asym;
  if (B < 0 || T < 0 || H_q < 0 || H_kv < 1 || pages_per_head < 1)
    return fail(ASYM_EINVAL, "kv append: B, T and H_q must be >= 0, H_kv and pages_per_head >= 1");
  if (pool_pages < 1 || pool_pages > 0x7FFFFFFFu) return fail(ASYM_EINVAL, "kv append: pool_pages must be in [1, 2^31)");
  if (pages_per_head > (1 << 25)) return fail(ASYM_EUNSUPPORTED, "kv append: more than 2^30 tokens a request");
  int rc = turn_check("kv append", rotary, kKvD, freq, layout, amplitude);
  if (rc != ASYM_OK) return rc;
  if (B == 0 || T == 0) return ASYM_OK;
  if (!k || !v || !k_pool || !v_pool || !k_pages || !v_pages || !cu || !start || (H_q && (!q || !q_out)))
    return fail(ASYM_EINVAL, "kv append: null pointer");
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_pool | (uintptr_t)v_pool) & 15u || (H_q && ((uintptr_t)q | (uintptr_t)q_out) & 15u))
    return fail(ASYM_EINVAL, "kv append: q, K, V and the pools must be 16-byte aligned");
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)cu | (uintptr_t)start | (uintptr_t)positions) & 3u)
    return fail(ASYM_EINVAL, "kv append: tables, offsets and positions must be 4-byte aligned");
  if (bad_strides({k_token, k_head, v_token, v_head}) || (H_q && bad_strides({q_token, q_head, qo_token, qo_head})))
    return fail(ASYM_EINVAL, "kv append: strides must be multiples of 8 values and not negative");
  if (H_q && rows_overlap(T, qo_token, H_q, qo_head, kKvD)) return fail(ASYM_EINVAL, "kv append: rows of q_out lie on each other");
  AppendParams p = {};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.qo = static_cast<uint16_t*>(q_out);
  p.q_tok = q_token; p.q_head = q_head; p.qo_tok = qo_token; p.qo_head = qo_head;
  p.k_tok = k_token; p.k_head = k_head; p.v_tok = v_token; p.v_head = v_head;
  p.k_pool = static_cast<uint8_t*>(k_pool);
  p.v_pool = static_cast<uint8_t*>(v_pool);
  p.k_pages = k_pages; p.v_pages = v_pages; p.cu = cu; p.start = start; p.pos = positions;
  p.turn = Turn{freq, rotary, amplitude, 1.f};
  p.B = B; p.Hq = H_q; p.Hkv = H_kv; p.T = T; p.pph = pages_per_head; p.pool_pages = (int)pool_pages;
  const int e = run_of(kKvD, rotary);
  const int64_t heads = (int64_t)H_q + 2ll * H_kv;
  if (heads > (1 << 20)) return fail(ASYM_EUNSUPPORTED, "kv append: too many heads");
  const int64_t each = heads * (kKvD / (2 * e));  // units of a token
  p.parts = (int)((each + kAppend - 1) / kAppend);
  const int64_t share = (each + p.parts - 1) / p.parts;
  p.tokens = (int)std::max<int64_t>(1, std::min<int64_t>(kMostTokens / kSlots, 256 / share));
  const unsigned threads = (unsigned)((share * p.tokens + 63) / 64 * 64);
  const bool many = (int64_t)T * p.parts >= 4096;
  const int64_t slots = many ? kSlots : 1;
  const int64_t grid = ((int64_t)T + p.tokens * slots - 1) / (p.tokens * slots) * p.parts;
  if (grid >= (1 << 23)) return fail(ASYM_EUNSUPPORTED, "kv append: too many rows");  // (threads are counted in 32 bits)
  with_run(e, layout == ASYM_ROPE_INTERLEAVED, [&](auto E, auto I) {
    auto kernel = many ? kv_append_kernel<decltype(E)::value, decltype(I)::value, kSlots>
                       : kv_append_kernel<decltype(E)::value, decltype(I)::value, 1>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), 0, static_cast<hipStream_t>(stream), p);
  });
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
