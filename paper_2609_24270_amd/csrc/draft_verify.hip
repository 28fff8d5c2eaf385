// Drafted tokens against the target's probabilities, from given random numbers.
//
// A request's nodes are a tree (chains: each node's parent is the one before): node 0 is the
// root, and target[i] and draft[i] are what the two models say about the token behind node i.
// Nodes are taken in order; a node whose parent is the current one, with token t, is accepted if
//
//   u q(t) m < R(t),  R = max(p - c q, 0),  p = target[current], q = draft[current],
//
// c = 0 and m = 1 at first.  Accepted, it becomes the current one.  Rejected, c grows by m and m
// becomes the sum of R: what is left of p without what the rejected sibling stood for (that q
// is subtracted after each rejection from R / m makes R = max(p - c q, 0) with one c, so that any
// number of siblings is one pass over the row each).  When no node is left, the last token is
// the lowest t with R(0) + .. + R(t) > w sum R (p itself where nothing is left of R).  The token of a
// node so accepted or drawn has the target's distribution, whatever the draft's, if each token
// was drawn from its parent's draft[] row.
// Without draft probabilities a token counts as certain: R is p without the rejected siblings'
// tokens, m = 1 - their p.
//
// All of it is in 64 bits.  Before a node's first rejection (c = 0, m = 1) both sides of the comparison are exact; behind it
// c, m, the product and the difference are rounded, and sums of a row are V roundings: the choices are those of the
// definition but for borders nearer than about 10^-15 of the probabilities that a difference is of, V 2^-53 of a sum.  What is
// not a positive finite number counts as 0.
//
// A row is cut into slices; a launch (`round`; none for small vocabularies) sums one each a workgroup, after it has
// walked the request's nodes as far as the sums so far allow, which all of the request's
// workgroups do alike (the nodes' p and q, one a lane, are on their way at once).  The last launch has a
// workgroup a request: it walks to the end (summing slices alone if need be) and draws.
//
// Bound by the chain of sums, and each by HBM: only rows that a sum is needed of are read, one a rejection and one for
// the draw at most.  64 trees of 31 tokens, V 128000, fp32: 54 us in six launches, which read 63, 49, 23, 2, 0 and 2 MB;
// bf16 48 to 49 (half the bytes: the launches' starts are most of it), without draft probabilities 18 (one sum a request).  16
// chains of 4, V 32000: 4.7 and 6.2 us in two, fp32 as bf16.
// The slices' lengths are chosen for the whole chip, whatever the stream's CUs.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "kv_fp4.h"

namespace asym {
namespace {

constexpr int kThreads = 256;   // of a workgroup that sums a slice
constexpr int kLast = 1024;     // of one that ends a request
constexpr int kMinSlice = 2048, kMaxSlice = 8192;
constexpr int kOneLaunch = 16384;  // of vocabularies up to this size one launch does everything

// Where a request's walk stands
struct State {
  double c, m;
  int cur, next;   // the current node, the first that has not been looked at
  int kept;        // nodes on the path
  int what;        // kWalk, kMass or kDraw
};
// kMass: a sibling was rejected, m is the sum of R to come; kDraw: no node is left, the sums of R are to draw from
// (both: of row `cur` with c); kWalk: at the start
enum { kWalk, kMass, kDraw };

struct VerifyParams {
  const void *target, *draft;  // [T][V], rows target_row and draft_row values apart
  int64_t target_row, draft_row;
  const int *tokens, *parents, *cu;
  const float *accept, *final;
  int *path, *count, *token;
  State* state;   // [2][B]: of the round before, of this one
  double* sums;   // [2][B][slices]
  int B, T, V, slice, slices;
  int round;
};

// value i of a row, as a probability
__device__ __forceinline__ float clean(float x) { return x > 0.f && x < INFINITY ? x : 0.f; }
template <class T>
__device__ __forceinline__ float value(const void* base, int64_t i) {
  if constexpr (sizeof(T) == 4)
    return clean(static_cast<const float*>(base)[i]);
  else
    return clean(__uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[i] << 16));
}
// four neighbours (rows may begin at any value)
template <class T>
__device__ __forceinline__ float4 values4(const void* base, int64_t i) {
  if constexpr (sizeof(T) == 4) {
    typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
    const f32x4u x = *reinterpret_cast<const f32x4u*>(static_cast<const float*>(base) + i);
    return float4{clean(x[0]), clean(x[1]), clean(x[2]), clean(x[3])};
  } else {
    typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
    const u16x4u x = *reinterpret_cast<const u16x4u*>(static_cast<const uint16_t*>(base) + i);
    float4 r;
    r.x = clean(__uint_as_float((uint32_t)x[0] << 16));
    r.y = clean(__uint_as_float((uint32_t)x[1] << 16));
    r.z = clean(__uint_as_float((uint32_t)x[2] << 16));
    r.w = clean(__uint_as_float((uint32_t)x[3] << 16));
    return r;
  }
}

__device__ __forceinline__ double of_lane(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Walks from `s` until a sum is needed or no node is left.  One wave, all of its lanes; `write`: the path is written.
template <class T, bool DRAFT>
__device__ void walk(const VerifyParams& p, int first, int n, State& s, bool write) {
  const int lane = threadIdx.x & 63;
  for (int base = s.next & ~63; base < n; base += 64) {
    // a lane holds node base + lane
    const int i = base + lane;
    int tok = -1, par = -1;
    float u = 0.f, pt = 0.f, qt = 0.f;
    if (i < n) {
      tok = p.tokens[first + i];
      par = p.parents ? p.parents[first + i] : i - 1;
      u = p.accept[first + i];
    }
    const bool ok = i < n && i > 0 && par >= 0 && par < i && tok >= 0 && tok < p.V;
    if (ok) {
      pt = value<T>(p.target, (int64_t)(first + par) * p.target_row + tok);
      if (DRAFT) qt = value<T>(p.draft, (int64_t)(first + par) * p.draft_row + tok);
    }
    while (true) {
      const unsigned long long may = __ballot(ok && par == s.cur && i >= s.next);
      if (!may) break;
      const int l = __builtin_ctzll(may), node = base + l;
      const double P = (double)__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(pt), l));
      const double Q = (double)__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(qt), l));
      const double U = (double)__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(u), l));
      const int t = __builtin_amdgcn_readlane(tok, l);
      bool took, again = false;  // again: the token of a rejected sibling
      if (DRAFT) {
        took = U * Q * s.m < fmax(P - s.c * Q, 0.);
      } else {
        again = __ballot(ok && par == s.cur && tok == t && lane < l) != 0;
        for (int b = 0; b < base && !again; b += 64) {
          const int j = b + lane;
          const bool same = j > 0 && p.tokens[first + j] == t && (p.parents ? p.parents[first + j] : j - 1) == s.cur && s.cur < j;
          again = __ballot(same) != 0;
        }
        took = !again && U * s.m < P;
      }
      s.next = node + 1;
      if (took) {
        if (write && lane == 0) p.path[first + s.kept] = node;
        s.cur = node;
        ++s.kept;
        s.c = 0.;
        s.m = 1.;
      } else if (DRAFT) {
        s.c += s.m;
        s.what = kMass;
        return;
      } else if (!again) {
        s.m -= P;
      }
    }
    s.next = max(s.next, min(base + 64, n));
  }
  s.what = kDraw;
}

// x of the lane that CTRL names (data-parallel primitives), 0 where the row mask leaves a lane out
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// The sums up to and with each lane (every lane on)
__device__ __forceinline__ double wave_prefix(double x) {
  x += moved<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8
  x += moved<0x112, 0xF>(x);
  x += moved<0x114, 0xF>(x);
  x += moved<0x118, 0xF>(x);
  x += moved<0x142, 0xA>(x);  // row_bcast 15 into rows 1 and 3
  x += moved<0x143, 0xC>(x);  // row_bcast 31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ double wave_total(double x) { return of_lane(wave_prefix(x), 63); }

// The sum of x over the workgroup, in an order that depends on the number of its threads alone; all threads get it.
template <int THREADS>
__device__ double block_sum(double x, double* red) {
  x = wave_total(x);
  __syncthreads();  // (red may still be read from the call before)
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double all = 0.;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) all += red[w];
  return all;
}

// What is left of row `row`: with draft probabilities max(p - c q, 0), without them p but for the tokens marked in `dead`
// (bits of the slice that begins at `from`)
struct Left {
  const void *target, *draft;
  int64_t p_at, q_at;  // the row's first values
  double c;
};
template <class T, bool DRAFT>
__device__ __forceinline__ Left left_of(const VerifyParams& p, int first, int row, double c) {
  return Left{p.target, p.draft, (int64_t)(first + row) * p.target_row, (int64_t)(first + row) * p.draft_row, c};
}
// the four from value i on (i + k >= to: 0)
template <class T, bool DRAFT>
__device__ __forceinline__ void left4(const Left& r, int i, int to, const uint32_t* dead, int from, double* x) {
  float4 a = {}, b = {};
  if (i + 4 <= to) {
    a = values4<T>(r.target, r.p_at + i);
    if (DRAFT && r.c != 0.) b = values4<T>(r.draft, r.q_at + i);
  } else {
    float* pa = &a.x;
    float* pb = &b.x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < to) {
        pa[e] = value<T>(r.target, r.p_at + i + e);
        if (DRAFT && r.c != 0.) pb[e] = value<T>(r.draft, r.q_at + i + e);
      }
  }
  const float pv[4] = {a.x, a.y, a.z, a.w}, qv[4] = {b.x, b.y, b.z, b.w};
  const uint32_t gone = !DRAFT && dead && i < to ? dead[(i - from) >> 5] >> ((i - from) & 31) : 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = DRAFT ? fmax((double)pv[e] - r.c * (double)qv[e], 0.) : (double)pv[e];
    if (!DRAFT && ((gone >> e) & 1)) x[e] = 0.;
  }
}

// Marks the tokens of the current node's children (all of them rejected) that lie in [from, to).  The whole workgroup
// comes here, each THREADS of it with a slice and marks of their own.
template <int THREADS>
__device__ void mark_dead(const VerifyParams& p, int first, int n, int cur, int from, int to, uint32_t* dead) {
  const int id = (int)threadIdx.x % THREADS;
  __syncthreads();
  for (int i = id; i < kMaxSlice / 32; i += THREADS) dead[i] = 0;
  __syncthreads();
  for (int i = cur + 1 + id; i < n; i += THREADS) {
    const int t = p.tokens[first + i];
    if ((p.parents ? p.parents[first + i] : i - 1) == cur && t >= from && t < to) atomicOr(&dead[(t - from) >> 5], 1u << ((t - from) & 31));
  }
  __syncthreads();
}

// A thread's part of what is left in one slice (thread `id` of 256: every 256th group of four); a slice's sum is that of its four
// waves' sums, in order.
template <class T, bool DRAFT>
__device__ double slice_part(const VerifyParams& p, const Left& r, int slice, int id, const uint32_t* dead) {
  const int from = slice * p.slice, to = min(from + p.slice, p.V);
  double sum = 0.;
#pragma unroll 4
  for (int i = from + id * 4; i < to; i += 4 * kThreads) {
    double x[4];
    left4<T, DRAFT>(r, i, to, dead, from, x);
    sum += (x[0] + x[1]) + (x[2] + x[3]);
  }
  return sum;
}

// The state at the start of round `round` (of the launch before, or of the request's beginning) walked on: one wave's work, told to
// all threads through LDS.
template <class T, bool DRAFT, int THREADS>
__device__ State advance(const VerifyParams& p, int b, int first, int n, bool write, State* lds, double* red) {
  State s = {0., 1., 0, 1, 1, kWalk};
  if (p.round > 0) {
    const int prev = (p.round - 1) & 1;
    s = p.state[(size_t)prev * p.B + b];
    if (s.what == kMass) {  // (what == kDraw: nothing is left to walk)
      double x = 0.;
      for (int k = threadIdx.x; k < p.slices; k += THREADS) x += p.sums[((size_t)prev * p.B + b) * p.slices + k];
      s.m = block_sum<THREADS>(x, red);
    }
  }
  if (s.what == kDraw) return s;
  s.what = kWalk;
  if (threadIdx.x < 64) {
    walk<T, DRAFT>(p, first, n, s, write);
    if (threadIdx.x == 0) *lds = s;
  }
  __syncthreads();
  s = *lds;
  __syncthreads();
  return s;
}

template <class T, bool DRAFT>
__global__ void __launch_bounds__(kThreads) verify_round(VerifyParams p) {
  __shared__ double red[kThreads / 64];
  __shared__ State told;
  __shared__ uint32_t dead[kMaxSlice / 32];
  const int b = blockIdx.x / p.slices, slice = blockIdx.x - b * p.slices;
  int first, n;
  packed_rows(p.cu, b, p.T, first, n);
  if (n == 0) return;
  State s = {};
  const size_t now = (size_t)(p.round & 1) * p.B + b, before = (size_t)((p.round - 1) & 1) * p.B + b;
  if (p.round > 0 && p.state[before].what == kDraw) {  // (the sums are there: they go on to the next round)
    if (threadIdx.x == 0) {
      if (slice == 0) p.state[now] = p.state[before];
      p.sums[now * p.slices + slice] = p.sums[before * p.slices + slice];
    }
    return;
  }
  const State was = p.round > 0 ? p.state[before] : State{};
  s = advance<T, DRAFT, kThreads>(p, b, first, n, slice == 0, &told, red);
  if (slice == 0 && threadIdx.x == 0) p.state[now] = s;
  if (p.round > 0 && s.what == kDraw && s.cur == was.cur && s.c == was.c) {  // (no node was left: the sums of the round before)
    if (threadIdx.x == 0) p.sums[now * p.slices + slice] = p.sums[before * p.slices + slice];
    return;
  }
  const int from = slice * p.slice, to = min(from + p.slice, p.V);
  if (!DRAFT) mark_dead<kThreads>(p, first, n, s.cur, from, to, dead);
  const double sum = block_sum<kThreads>(slice_part<T, DRAFT>(p, left_of<T, DRAFT>(p, first, s.cur, s.c), slice, threadIdx.x, dead), red);
  if (threadIdx.x == 0) p.sums[now * p.slices + slice] = sum;
}

// A workgroup a request: the walk's end, the draw, the outputs.
template <class T, bool DRAFT>
__global__ void __launch_bounds__(kLast) verify_last(VerifyParams p) {
  constexpr int kBatch = 64;  // slices that are summed between two barriers
  __shared__ double red[kLast / 64], part[kBatch][4];
  __shared__ State told;
  __shared__ uint32_t dead[kLast / kThreads][kMaxSlice / 32];
  __shared__ double own[kOneLaunch / kMinSlice];
  __shared__ int marks[kLast / 64], found;
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  int first, n;
  packed_rows(p.cu, b, p.T, first, n);
  const int prev = (p.round - 1) & 1;
  double* sums = p.round > 0 ? p.sums + ((size_t)prev * p.B + b) * p.slices : own;  // (this workgroup's own from here on)
  const State was = p.round > 0 ? p.state[(size_t)prev * p.B + b] : State{};
  const float draw = p.final[b];
  if (n == 0) {
    if (threadIdx.x == 0) {
      p.count[b] = 0;
      p.token[b] = -1;
    }
    return;
  }
  State s = advance<T, DRAFT, kLast>(p, b, first, n, true, &told, red);
  bool there = p.round > 0 && s.what == kDraw && s.cur == was.cur && s.c == was.c;  // the sums are those of (cur, c)
  // Every slice's sum, in the order that the slices' own launches have: 256 threads a slice.
  auto all_sums = [&](const Left& r, bool all) {  // all: rejected tokens too
    const int group = (int)threadIdx.x / kThreads;
    for (int k0 = 0; k0 < p.slices; k0 += kBatch) {
      const int end = min(p.slices - k0, kBatch);
      for (int k1 = 0; k1 < end; k1 += kLast / kThreads) {
        const int k = k1 + group;
        if (!DRAFT && !all) {
          const int from = (k0 + k) * p.slice;
          mark_dead<kThreads>(p, first, n, s.cur, from, k < end ? min(from + p.slice, p.V) : from, dead[group]);
        }
        if (k >= end) continue;
        const double x = wave_total(slice_part<T, DRAFT>(p, r, k0 + k, threadIdx.x % kThreads, all ? nullptr : dead[group]));
        if (lane == 0) part[k][threadIdx.x % kThreads / 64] = x;
      }
      __syncthreads();
      if ((int)threadIdx.x < end) {
        const double* x = part[threadIdx.x];
        sums[k0 + threadIdx.x] = ((0. + x[0]) + x[1]) + x[2] + x[3];
      }
      __threadfence_block();
      __syncthreads();
    }
  };
  while (!there) {  // (without draft probabilities once at most: the walk ends before the first sum)
    all_sums(left_of<T, DRAFT>(p, first, s.cur, s.c), false);
    if (s.what == kDraw) break;
    double x = 0.;
    for (int k = threadIdx.x; k < p.slices; k += kLast) x += sums[k];
    s.m = block_sum<kLast>(x, red);
    const int cur = s.cur;
    const double c = s.c;
    if (threadIdx.x < 64) {
      walk<T, DRAFT>(p, first, n, s, true);
      if (threadIdx.x == 0) told = s;
    }
    __syncthreads();
    s = told;
    __syncthreads();
    there = s.what == kDraw && s.cur == cur && s.c == c;
  }
  // The draw: the slice, by the sums in order (every wave alike), then the token in it
  Left r = left_of<T, DRAFT>(p, first, s.cur, s.c);
  uint32_t* bits = dead[0];
  auto mass = [&] {
    double all = 0.;
    for (int k = 0; k < p.slices; k += 64) all += wave_total(k + lane < p.slices ? sums[k + lane] : 0.);
    return all;
  };
  double M = mass();
  if (!(M > 0.)) {  // nothing is left: from p as it is
    r.c = 0.;
    bits = nullptr;
    all_sums(r, true);
    M = mass();
  }
  int token = -1;
  if (M > 0.) {
    const double aim = (double)draw * M;
    // the first slice whose end lies above the aim (or the last that holds anything)
    double below = 0., upto = 0.;
    int at = -1;
    bool over = false;
    for (int k = 0; k < p.slices && !over; k += 64) {
      const double x = k + lane < p.slices ? sums[k + lane] : 0.;
      const double here = upto + wave_prefix(x);
      const unsigned long long some = __ballot(x > 0.), above = __ballot(x > 0. && here > aim);
      over = above != 0;
      if (some) {
        const int l = over ? __builtin_ctzll(above) : 63 - __builtin_clzll(some);
        at = k + l;
        below = l ? of_lane(here, l - 1) : upto;
      }
      upto = of_lane(here, 63);
    }
    const int from = at * p.slice, to = min(from + p.slice, p.V);
    if (!DRAFT && bits) mark_dead<kLast>(p, first, n, s.cur, from, to, bits);
    double so = below;
    int last = -1;  // the last value that is not 0
    for (int i0 = from; i0 < to && token < 0; i0 += 4 * kLast) {
      const int i = i0 + (int)threadIdx.x * 4;
      double x[4];
      left4<T, DRAFT>(r, i, to, bits, from, x);
      // the sums before this thread's four: of the wave's earlier lanes, of the earlier waves
      const double mine = (x[0] + x[1]) + (x[2] + x[3]);
      const double incl = wave_prefix(mine);
      __syncthreads();  // (red may still be read from the round before)
      if (lane == 63) red[threadIdx.x >> 6] = incl;
      __syncthreads();
      double at0 = so;
      for (int w = 0; w < kLast / 64; ++w) {
        if (w < (int)(threadIdx.x >> 6)) at0 += red[w];
        so += red[w];
      }
      at0 += incl - mine;
      int mark = -1;  // the first of the four that lies above the aim
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        at0 += x[e];
        if (x[e] > 0.) {
          last = i + e;
          if (at0 > aim && mark < 0) mark = i + e;
        }
      }
      // (of a wave its first such lane has it, of the workgroup the first wave)
      const unsigned long long above = __ballot(mark >= 0);
      if (lane == 0) marks[threadIdx.x >> 6] = above ? __builtin_amdgcn_readlane(mark, __builtin_ctzll(above)) : -1;
      __syncthreads();
      for (int w = kLast / 64 - 1; w >= 0; --w)
        if (marks[w] >= 0) token = marks[w];
    }
    if (token < 0) {  // (the aim within a rounding of the slice's end)
      if (threadIdx.x == 0) found = -1;
      __syncthreads();
      if (last >= 0) atomicMax(&found, last);
      __syncthreads();
      token = found;
    }
  }
  if (threadIdx.x == 0) {
    p.path[first] = 0;
    p.count[b] = s.kept;
    p.token[b] = token;
  }
  for (int i = s.kept + (int)threadIdx.x; i < n; i += kLast) p.path[first + i] = -1;
}

struct VerifyPlan {
  int slice = 0, slices = 0, rounds = 1;
  size_t bytes = 0;
};
int verify_plan(int B, int T, int V, VerifyPlan* plan) {
  if (B < 0 || T < 0 || V < 1) return fail(ASYM_EINVAL, "draft verify: B and T must be >= 0, V >= 1");
  if (V > (1 << 30)) return fail(ASYM_EUNSUPPORTED, "draft verify: more than 2^30 tokens in the vocabulary");
  VerifyPlan P;
  // slices of 2048, 4096 or 8192 values: enough for four workgroups a CU, or the smallest
  P.slice = kMaxSlice;
  while (P.slice > kMinSlice && (int64_t)B * ((V + P.slice - 1) / P.slice) < 1024) P.slice /= 2;
  P.slices = (int)(((int64_t)V + P.slice - 1) / P.slice);
  if ((int64_t)B * P.slices >= (1 << 22)) return fail(ASYM_EUNSUPPORTED, "draft verify: too many requests, or too large a vocabulary");
  P.bytes = V <= kOneLaunch ? 0 : (size_t)2 * B * (sizeof(State) + P.slices * sizeof(double));
  *plan = P;
  return ASYM_OK;
}

template <class T, bool DRAFT>
void launch_verify(VerifyParams p, int rounds, hipStream_t s) {
  for (p.round = 0; p.round < rounds; ++p.round)
    hipLaunchKernelGGL((verify_round<T, DRAFT>), dim3((unsigned)(p.B * p.slices)), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL((verify_last<T, DRAFT>), dim3((unsigned)p.B), dim3(kLast), 0, s, p);
}

}  // namespace
}  // namespace asym

extern "C" int asym_draft_verify_workspace(int B, int T, int V, size_t* bytes) {
  if (!bytes) return asym::fail(ASYM_EINVAL, "draft verify workspace: null output");
  asym::VerifyPlan P;
  const int rc = asym::verify_plan(B, T, V, &P);
  if (rc == ASYM_OK) *bytes = P.bytes;
  return rc;
}

extern "C" int asym_draft_verify(int B, int T, int V, int bf16, const void* target, int64_t target_row, const void* draft,
                                 int64_t draft_row, const int32_t* tokens, const int32_t* parents, const int32_t* cu,
                                 const float* accept, const float* final, int32_t* path, int32_t* count, int32_t* token,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  using namespace asym;
  VerifyPlan P;
  const int rc = verify_plan(B, T, V, &P);
  if (rc != ASYM_OK) return rc;
  if (target_row < V || (draft && draft_row < V)) return fail(ASYM_EINVAL, "draft verify: rows must be V values apart or more");
  if (B == 0) return ASYM_OK;
  if (!cu || !final || !count || !token || (T && (!target || !tokens || !accept || !path)))
    return fail(ASYM_EINVAL, "draft verify: null pointer");
  const uintptr_t odd = bf16 ? 1u : 3u;
  if (((uintptr_t)target | (uintptr_t)draft) & odd) return fail(ASYM_EINVAL, "draft verify: probabilities must be aligned to their type");
  if (((uintptr_t)tokens | (uintptr_t)parents | (uintptr_t)cu | (uintptr_t)accept | (uintptr_t)final | (uintptr_t)path |
       (uintptr_t)count | (uintptr_t)token) & 3u)
    return fail(ASYM_EINVAL, "draft verify: nodes, random numbers and outputs must be 4-byte aligned");
  if (P.bytes && (!workspace || workspace_bytes < P.bytes || ((uintptr_t)workspace & 15u)))
    return fail(ASYM_EINVAL, "draft verify: the workspace must be 16-byte aligned and hold asym_draft_verify_workspace's bytes");
  VerifyParams p = {};
  p.target = target; p.draft = draft;
  p.target_row = target_row; p.draft_row = draft_row;
  p.tokens = tokens; p.parents = parents; p.cu = cu;
  p.accept = accept; p.final = final;
  p.path = path; p.count = count; p.token = token;
  p.state = static_cast<State*>(workspace);
  p.sums = P.bytes ? reinterpret_cast<double*>(p.state + 2 * (size_t)B) : nullptr;
  p.B = B; p.T = T; p.V = V; p.slice = P.slice; p.slices = P.slices;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // Up to kOneLaunch tokens the last launch sums a row as fast as another begins, does all of it and needs no workspace.  us
  // with none, 1 and 2 launches before it, V 5000: chains of 16 nodes, 1 request 10.5 13.6 15.9, 64 10.5 13.7 16.1; trees 10.9 14.0
  // 16.5, 15.0 17.7 19.8; V 16000: chains 10.7 13.6 16.1, 12.1 13.6 16.1, trees 11.0 13.7 16.4, 22.1 23.5 24.2 (in graphs 9.8 9.6
  // 11.8, 12.1 13.4 15.5, 10.6 10.8 11.9, 22.0 23.7 24.4); V 64000: chains 17.3 13.7 16.3, 19.6 16.0 18.4.
  // A chain rejects once at most, and without draft probabilities no sum is needed before the last.  A tree with them
  // needs a sum a rejection, the last launch takes what is over one by one, and waits for the request that needs the
  // most.  us with 1, 2, 3 and 4 launches before it, trees of 16 nodes, V 32000: 1 request 15.7 18.0 20.7 24.3, 4 24.8 22.8 22.3
  // 24.3, 16 30.6 28.8 26.4 26.0, 64 34.0 32.9 31.4 30.7; V 48000: 15.9 17.9 20.6 24.5, 21.0 18.4 21.1 24.2, 33.7 30.2 25.4
  // 26.1, 39.2 35.9 31.5 31.3; V 128000 (1 to 6): 1 24 19 23 27 29 32, 4 48 30 22 26 28 30, 16 70 54 37 30 32 34, 64 of 32
  // nodes 92 84 72 64 57 60.
  int rounds = V > kOneLaunch;
  if (draft && parents && V > kOneLaunch) {
    rounds = V > 65536 ? 2 : 1;
    for (int64_t requests = 4; requests <= B && rounds < 6; requests *= 4) ++rounds;
  }
  if (bf16)
    draft ? launch_verify<uint16_t, true>(p, rounds, s) : launch_verify<uint16_t, false>(p, rounds, s);
  else
    draft ? launch_verify<float, true>(p, rounds, s) : launch_verify<float, false>(p, rounds, s);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
