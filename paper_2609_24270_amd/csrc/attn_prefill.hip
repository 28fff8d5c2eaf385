// Prompt attention over packed sequences, grouped key/value heads:
//
//   O[i, h] = softmax_j(scale * <q[i, h], K[j, g]>) . V[j, g],  g = h / G, G = H_q / H_kv,
//
// over the keys j that row i of a sequence sees: all of the sequence's, or (causal)
// j <= i + L_k - L_q, so that the last query sees the last key.
//
// A workgroup computes 32 * NW rows of one sequence and one key/value head; a row is
// a (token, query head of the group) pair, token-major, so a tile of few tokens
// serves all heads that read the same keys and the diagonal is 32 * NW / G tokens
// wide.  Each wave has 32 rows.  Blocks of 64 keys and values stream through LDS
// (buffer_load ... lds, two buffers); per block
//   S^T = K . Q^T   (v_mfma_f32_32x32x16_bf16, K from LDS, Q in registers):
//                   a lane holds 32 of the 64 scores of ONE row;
//   softmax         over the lane's own registers and one exchange with lane ^ 32;
//                   the running max is raised only when a row's grows by more than
//                   2^8 (the sums stay in range, the output is rescaled rarely);
//   O^T += V^T . P^T: the score registers, rounded to bf16 (the type of the products'
//                   operands; 2^-9 relative, the output's own rounding), are the
//                   operand as they lie, because the order of tokens inside a product
//                   is free: V^T is read in that order with ds_read_b64_tr_b16, which
//                   transposes 16-bit values on the way from LDS.
// Scores, max, sum and output are fp32.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "internal.h"
#include "kv_fp4.h"

namespace asym {
namespace {

constexpr int PD = 128;   // head dimension
constexpr int PN = 64;    // keys per block
constexpr int kXcds = 8;  // workgroup i is dealt to XCD i mod 8 (only speed depends on it)
constexpr int kRowBytes = PD * 2;
constexpr int kTileBytes = PN * kRowBytes;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct PrefillParams {
  const uint16_t *q, *k, *v;
  uint16_t* o;          // [Tq][Hq][128]
  float* lse;           // [Tq][Hq], nullable
  const int *cu_q, *cu_k;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;  // strides, values
  int B, Hq, Hkv, G, Tq, Tk;
  int tiles;            // at least the number of tiles of all sequences
  int causal, aware;
  float c;              // |scale| * log2(e), positive
  float scale;          // |scale|
  uint32_t q_flip;      // sign bits to flip in q (a negative scale)
};

// The k-th tile of the batch, longest first: the sequence and the tile in it.  A
// tile's level is the number of row tiles' worth of keys it sees; tiles are
// numbered by falling level, sequences in order within a level.  One wave.
__device__ bool find_tile(const PrefillParams& p, int BM, int k, int& seq, int& tile) {
  const int lane = threadIdx.x & 63;
  // of sequence 64 c + lane: tiles n at levels base .. base + n - 1
  auto shape = [&](int c, int& n, int& base) {
    const int b = 64 * c + lane;
    n = base = 0;
    if (b < p.B) {
      int qs, qn, ks, kn;
      packed_rows(p.cu_q, b, p.Tq, qs, qn);
      packed_rows(p.cu_k, b, p.Tk, ks, kn);
      n = (int)(((int64_t)qn * p.G + BM - 1) / BM);
      base = (int)((int64_t)max(kn - qn, 0) * p.G / BM);
    }
  };
  const int nc = (p.B + 63) >> 6;
  int n0, base0;
  shape(0, n0, base0);
  auto count = [&](int level) {  // tiles at this level or above
    int x = min(max(base0 + n0 - level, 0), n0);
    for (int c = 1; c < nc; ++c) {
      int n, base;
      shape(c, n, base);
      x += min(max(base + n - level, 0), n);
    }
    return wave_sum(x);
  };
  if (count(0) <= k) return false;
  int lo = 0, hi = 1;  // count(lo) > k >= count(hi)
  while (count(hi) > k) {
    lo = hi;
    hi *= 2;
  }
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (count(mid) > k)
      lo = mid;
    else
      hi = mid;
  }
  int r = k - count(hi);  // the r-th sequence that has a tile at level lo
  for (int c = 0; c < nc; ++c) {
    int n = n0, base = base0;
    if (c) shape(c, n, base);
    unsigned long long has = __ballot(base <= lo && lo < base + n);
    const int cnt = __popcll(has);
    if (r < cnt) {
      for (; r > 0; --r) has &= has - 1;
      const int l = __builtin_ctzll(has);
      seq = 64 * c + l;
      tile = lo - __builtin_amdgcn_readlane(base, l);
      return true;
    }
    r -= cnt;
  }
  return false;
}

__device__ __forceinline__ i32x4 tile_rsrc(const uint16_t* base, int64_t tok, int rows) {
  // `rows` rows of a block; a row past them reads zeros
  const uint64_t a = (uint64_t)base;
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
  r[2] = __builtin_amdgcn_readfirstlane(rows > 0 ? (int)((uint32_t)(rows - 1) * (uint32_t)tok * 2u + kRowBytes) : 0);
  r[3] = 0x00020000;
  return r;
}

// 1 KiB from lane addresses voff to LDS bytes dst .. dst + 1023, in lane order
__device__ __forceinline__ void lds_load_1k(uint32_t dst, i32x4 rs, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(voff), "s"(rs)
               : "memory");
}

__device__ __forceinline__ float max16(const f32x16& s) {
  float m = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
  for (int i = 3; i < 15; i += 2) m = fmaxf(fmaxf(m, s[i]), s[i + 1]);
  return fmaxf(m, s[15]);
}

// max over this lane and lane ^ 32
__device__ __forceinline__ float max_halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// 16-byte chunk c of a tile's row r lies at chunk c ^ swz(r): the rows that one read
// takes together then lie on different banks (K: 8 rows, one chunk of each; V: 4 rows,
// two chunks of each).
__device__ __forceinline__ int swz_k(int row) { return row & 7; }
__device__ __forceinline__ int swz_v(int row) { return (row & 3) << 1; }

typedef __attribute__((address_space(3))) unsigned char lds_byte;

// A lane's places in the K and V tiles (bytes from a tile's start).
struct Places {
  uint32_t k[4];  // row n, chunks 2 c + h of c = 0 .. 3 (c + 4: 128 bytes on; rows 32 + n: 32 rows on)
  uint32_t v[2];  // channels of blocks cb = 0, 1 (cb + 2: 128 bytes on), tokens 4 h + (lane % 16) / 4
};
__device__ __forceinline__ Places places(int lane) {
  Places p;
  const int n = lane & 31, h = lane >> 5, i = lane & 15, half = (lane >> 4) & 1;
#pragma unroll
  for (int c = 0; c < 4; ++c) p.k[c] = (uint32_t)(n * kRowBytes + (((2 * c + h) ^ swz_k(n)) << 4));
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const int row = 4 * h + (i >> 2), chunk = 4 * cb + 2 * half + ((i & 3) >> 1);
    p.v[cb] = (uint32_t)(row * kRowBytes + ((chunk ^ swz_v(row)) << 4) + ((i & 1) << 3));
  }
  return p;
}

// K operand: 32 keys (half t of the block) x 16 channels (step c)
__device__ __forceinline__ bf16x8 k_frag(const lds_byte* kt, const Places& pl, int t, int c) {
  return *(const __attribute__((address_space(3))) bf16x8*)(kt + pl.k[c & 3] + (c >> 2) * 128 + t * 32 * kRowBytes);
}

// V^T operand: 32 channels (block cb) x 16 tokens (step ks of the block)
__device__ __forceinline__ bf16x8 v_frag(const lds_byte* vt, const Places& pl, int cb, int ks) {
  union {
    s16x4 s[2];
    bf16x8 b;
  } u;
#pragma unroll
  for (int part = 0; part < 2; ++part)
    u.s[part] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(vt + pl.v[cb & 1] + (cb >> 1) * 128 + (16 * ks + 8 * part) * kRowBytes));
  return u.b;
}

template <int NW>
__global__ void __launch_bounds__(64 * NW, 2) attn_prefill_kernel(PrefillParams p) {
  constexpr int BM = 32 * NW;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTileBytes];  // two K tiles, two V tiles
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;

  // which head and tile
  int hk, rank;
  const int blk = blockIdx.x;
  if (!p.aware) {
    hk = blk / p.tiles;
    rank = blk - hk * p.tiles;
  } else if (p.Hkv % kXcds == 0) {
    const int per = p.Hkv / kXcds, r = blk / kXcds;
    hk = (blk % kXcds) * per + r % per;
    rank = r / per;
  } else if (kXcds % p.Hkv == 0) {
    const int x = blk % kXcds;
    hk = x % p.Hkv;
    rank = (blk / kXcds) * (kXcds / p.Hkv) + x / p.Hkv;
  } else {
    hk = blk % p.Hkv;
    rank = blk / p.Hkv;
  }
  int seq, tile;
  if (!find_tile(p, BM, rank, seq, tile)) return;
  int qs, Lq, ks, Lk;
  packed_rows(p.cu_q, seq, p.Tq, qs, Lq);
  packed_rows(p.cu_k, seq, p.Tk, ks, Lk);
  const int off = Lk - Lq;

  // this lane's row (rows past the last repeat it, and are not stored)
  const int64_t rows = (int64_t)Lq * p.G;
  const int64_t row0 = (int64_t)tile * BM + wave * 32;
  const int64_t row = min(row0 + n, rows - 1);
  const int tok = (int)(row / p.G), g = (int)(row - (int64_t)tok * p.G);
  const int64_t orow = (int64_t)(qs + tok) * p.Hq + (int64_t)hk * p.G + g;
  // keys that the row sees; the most over the wave, the least and most over the workgroup
  auto limit = [&](int64_t r) { return p.causal ? max(off + (int)(min(r, rows - 1) / p.G) + 1, 0) : Lk; };
  const int lim = p.causal ? max(off + tok + 1, 0) : Lk;
  const int lim_hi = __builtin_amdgcn_readfirstlane(limit(row0 + 31));
  const int nblk = (__builtin_amdgcn_readfirstlane(limit((int64_t)tile * BM + BM - 1)) + PN - 1) / PN;
  const int nfull = __builtin_amdgcn_readfirstlane(limit((int64_t)tile * BM)) / PN;  // blocks that every row sees whole

  bf16x8 qf[8];
  {
    const uint16_t* qr = p.q + (int64_t)(qs + tok) * p.q_tok + ((int64_t)hk * p.G + g) * p.q_head + 8 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      u32x4 w = *reinterpret_cast<const u32x4*>(qr + 16 * s);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] ^= p.q_flip;
      qf[s] = __builtin_bit_cast(bf16x8, w);
    }
  }
  const uint16_t* kb = p.k + (int64_t)ks * p.k_tok + (int64_t)hk * p.k_head;
  const uint16_t* vb = p.v + (int64_t)ks * p.v_tok + (int64_t)hk * p.v_head;
  const uint32_t lds0 = (uint32_t)(size_t)lds;
  const Places pl = places(lane);
  // 1 KiB is 4 rows of a tile: lane -> row lane / 16, 16-byte place lane % 16
  constexpr int PIECES = kTileBytes / 1024 / NW;
  auto load_k = [&](int j) {
    const i32x4 rs = tile_rsrc(kb + (int64_t)j * PN * p.k_tok, p.k_tok, min(Lk - j * PN, PN));
    const uint32_t dst = lds0 + (uint32_t)(j & 1) * kTileBytes;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = wave * PIECES + i, r = 4 * piece + (lane >> 4);
      lds_load_1k(dst + piece * 1024, rs, (uint32_t)r * (uint32_t)p.k_tok * 2u + (((lane & 15) ^ swz_k(r)) << 4));
    }
  };
  auto load_v = [&](int j) {
    const i32x4 rs = tile_rsrc(vb + (int64_t)j * PN * p.v_tok, p.v_tok, min(Lk - j * PN, PN));
    const uint32_t dst = lds0 + (uint32_t)(2 + (j & 1)) * kTileBytes;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = wave * PIECES + i, r = 4 * piece + (lane >> 4);
      lds_load_1k(dst + piece * 1024, rs, (uint32_t)r * (uint32_t)p.v_tok * 2u + (((lane & 15) ^ swz_v(r)) << 4));
    }
  };
  auto k_tile = [&](int j) { return (lds_byte*)lds + (j & 1) * kTileBytes; };
  auto v_tile = [&](int j) { return (lds_byte*)lds + (2 + (j & 1)) * kTileBytes; };

  f32x16 o[4];
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) o[cb] = f32x16{};
  float m = -INFINITY, l = 0.f;
  f32x16 s[2];
  bf16x8 pf[4];

  auto scores = [&](int j) {
    const lds_byte* kt = k_tile(j);
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(kt, pl, t, c), qf[c], s[t], 0, 0, 0);
  };
  auto softmax = [&] {
    const float top = max_halves(fmaxf(max16(s[0]), max16(s[1])));
    if (__any((top - m) * p.c > 8.f)) {  // (a first finite max: inf; NaN never)
      const float m_new = fmaxf(m, top);
      const float alpha = __builtin_amdgcn_exp2f((m - (m_new == -INFINITY ? 0.f : m_new)) * p.c);
      l *= alpha;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cb][r] *= alpha;
      m = m_new;
    }
    const float ms = m == -INFINITY ? 0.f : m * p.c;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[t][r], p.c, -ms));
        l += e;
        pf[2 * t + (r >> 3)][r & 7] = (__bf16)e;
      }
  };
  auto add_pv = [&](int j) {
    const lds_byte* vt = v_tile(j);
#pragma unroll
    for (int kst = 0; kst < 4; ++kst)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(vt, pl, cb, kst), pf[kst], o[cb], 0, 0, 0);
  };
  auto arrived = [&] {  // this wave's loads, and with them everyone's
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  // Blocks that every row sees whole.
  if (nfull > 0) {
    load_k(0);
    load_v(0);
  }
  for (int j = 0; j < nfull; ++j) {
    arrived();
    if (j + 1 < nfull) {
      load_k(j + 1);
      load_v(j + 1);
    }
    scores(j);
    softmax();
    add_pv(j);
  }
  // The rest.  A masked key's probability is 0, but 0 times an infinity or a NaN among
  // its values is NaN, in a row that does not see it.  Where a block holds such values
  // they are taken out of the V tile and kept, as small whole numbers, in the K tile's
  // place (1: inf, 128: -inf, 16384: NaN), and a product of their own with the rows' masks
  // says what they do to the rows that see them (sums over 64 keys, exact in fp32).
  if (nfull < nblk) {
    __syncthreads();
    load_k(nfull);
    load_v(nfull);
  }
  for (int j = nfull; j < nblk; ++j) {
    arrived();
    if (j + 1 < nblk) {
      load_k(j + 1);
      load_v(j + 1);
    }
    const bool mine = j * PN < lim_hi;  // (else the wave's rows see none of it)
    auto each_word = [&](auto f) {      // the thread's words of the V tile
#pragma unroll
      for (int i = 0; i < kTileBytes / 16 / (64 * NW); ++i) {
        const uint32_t at = (uint32_t)(i * 64 * NW + (int)threadIdx.x) * 16;
        f(at, *(__attribute__((address_space(3))) u32x4*)(v_tile(j) + at));
      }
    };
    uint32_t bad = 0;
    if (p.causal)
      each_word([&](uint32_t, u32x4 w) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7F807F80u) + 0x00800080u;  // an exponent of all ones carries
      });
    const bool guard = p.causal && __syncthreads_or((bad & 0x80008000u) != 0);
    if (mine) {
      scores(j);
      const int left = lim - j * PN - 4 * h;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * t + (r & 3) + 8 * (r >> 2) >= left) s[t][r] = -INFINITY;
      softmax();
    }
    if (guard) {
      __syncthreads();  // (the K tile has been read)
      each_word([&](uint32_t at, u32x4 w) {
        u32x4 fin, code;
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // two values a word
          const uint32_t mask = ((((w[e] & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xFFFFu;
          auto kind = [](uint32_t u) { return (u & 0x7Fu) ? 0x4680u : (u & 0x8000u) ? 0x4300u : 0x3F80u; };
          fin[e] = w[e] & ~mask;
          code[e] = (kind(w[e] & 0xFFFFu) | (kind(w[e] >> 16) << 16)) & mask;
        }
        *(__attribute__((address_space(3))) u32x4*)(v_tile(j) + at) = fin;
        *(__attribute__((address_space(3))) u32x4*)(k_tile(j) + at) = code;
      });
      __syncthreads();
      if (mine) {
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          f32x16 seen = {};
#pragma unroll
          for (int kst = 0; kst < 4; ++kst) {
            u32x4 vis;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = 8 * (kst & 1) + 2 * e, key = j * PN + 32 * (kst >> 1) + (r & 3) + 8 * (r >> 2) + 4 * h;
              vis[e] = (key < lim ? 0x3F80u : 0u) | (key + 1 < lim ? 0x3F800000u : 0u);
            }
            seen = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(k_tile(j), pl, cb, kst), __builtin_bit_cast(bf16x8, vis),
                                                           seen, 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int k = (int)seen[r];
            o[cb][r] += ((k & 127) ? INFINITY : 0.f) + (((k >> 7) & 127) ? -INFINITY : 0.f) + (k >= 16384 ? NAN : 0.f);
          }
        }
      }
    }
    if (mine) add_pv(j);
  }

  // a lane has 64 of the row's 128 channels: 4 of every 8, the other half's in lane ^ 32
  l = sum_halves(l);
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);  // (NaN stays)
  const bool store = row0 + n < rows;
  uint16_t* dst = p.o + orow * PD;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w[4];  // channels 16 i + 4 h + 0 .. 3 and 16 i + 8 + 4 h + 0 .. 3
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x2 b = {(__bf16)(o[cb][8 * i + 2 * e] * inv), (__bf16)(o[cb][8 * i + 2 * e + 1] * inv)};
        w[e] = __builtin_bit_cast(uint32_t, b);
      }
      const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
      if (store)
        *reinterpret_cast<u32x4*>(dst + 32 * cb + 16 * i + 8 * h) = u32x4{x[0], y[0], x[1], y[1]};
    }
  if (p.lse && store && h == 0) p.lse[orow] = l == 0.f ? -INFINITY : m * p.scale + __logf(l);
}

}  // namespace
}  // namespace asym

extern "C" int asym_attn_prefill_bf16(int B, int H_q, int H_kv, int D, int T_q, int T_k, const void* q, int64_t q_token,
                                      int64_t q_head, const void* k, int64_t k_token, int64_t k_head, const void* v,
                                      int64_t v_token, int64_t v_head, void* o, float* lse, const int32_t* cu_q,
                                      const int32_t* cu_k, float scale, int causal, int mapping, void* stream) {
  using namespace asym;
  if (B < 0 || T_q < 0 || T_k < 0 || H_q < 1 || H_kv < 1)
    return fail(ASYM_EINVAL, "prefill: B, T_q and T_k must be >= 0, H_q and H_kv >= 1");
  if (H_q % H_kv) return fail(ASYM_EINVAL, "prefill: H_kv must divide H_q");
  if (D != PD) return fail(ASYM_EUNSUPPORTED, "prefill: the head dimension must be 128");
  if (mapping != ASYM_MAP_AWARE && mapping != ASYM_MAP_OBLIVIOUS_GROUPED && mapping != ASYM_MAP_OBLIVIOUS_ROWMAJOR)
    return fail(ASYM_EINVAL, "prefill: unknown mapping");
  if (!std::isfinite(scale)) return fail(ASYM_EINVAL, "prefill: scale must be finite");
  if (B == 0 || T_q == 0) return ASYM_OK;
  if (!q || !o || !cu_q || !cu_k || (T_k && (!k || !v))) return fail(ASYM_EINVAL, "prefill: null pointer");
  auto off16 = [](const void* x) { return ((uintptr_t)x & 15u) != 0; };
  if (off16(q) || off16(k) || off16(v) || off16(o) || ((uintptr_t)lse & 3u) || ((uintptr_t)cu_q & 3u) ||
      ((uintptr_t)cu_k & 3u))
    return fail(ASYM_EINVAL, "prefill: q, K, V and O must be 16-byte aligned, lse and the offsets 4-byte aligned");
  for (int64_t s : {q_token, q_head, k_token, k_head, v_token, v_head})
    if (s < 0 || s % 8) return fail(ASYM_EINVAL, "prefill: strides must be multiples of 8 values and not negative");
  // (64 rows of a block are addressed with 32-bit offsets; a row past a sequence's last must lie past its end)
  for (int64_t s : {k_token, v_token})
    if (s < PD || s > (1 << 23)) return fail(ASYM_EUNSUPPORTED, "prefill: K and V token strides must be in [128, 2^23] values");
  PrefillParams p;
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.cu_q = cu_q;
  p.cu_k = cu_k;
  p.q_tok = q_token; p.q_head = q_head;
  p.k_tok = k_token; p.k_head = k_head;
  p.v_tok = v_token; p.v_head = v_head;
  p.B = B; p.Hq = H_q; p.Hkv = H_kv; p.G = H_q / H_kv; p.Tq = T_q; p.Tk = T_k;
  p.causal = causal != 0;
  p.aware = mapping == ASYM_MAP_AWARE;
  p.scale = std::fabs(scale);
  // a scale of 0 weighs all keys alike: the least factor that still sends a masked
  // score (minus infinity) to minus infinity
  p.c = std::fmax(p.scale * 1.4426950408889634f, 1.17549435e-38f);
  p.q_flip = scale < 0 ? 0x80008000u : 0u;
  // Tiles of 256 rows read the keys half as often and are faster once there is one for
  // every CU (us, 128 rows first: 16384 tokens, 32 / 8 heads 2031 1953, 4096 tokens 149 137,
  // two of 4096 with 16 / 16 heads 149 138, eight chunks of 1000 tokens behind
  // prefixes 329 329); with fewer, CUs would idle (1024 tokens, 32 / 8 heads 25 32).
  auto count = [&](int rows) { return (int64_t)T_q * p.G / rows + B; };  // sequences end in a part tile each
  const bool wide = count(256) * H_kv >= 256;
  const int64_t tiles = count(wide ? 256 : 128);
  int64_t grid = tiles * H_kv;
  if (p.aware && kXcds % H_kv == 0) {
    const int share = kXcds / H_kv;
    grid = (tiles + share - 1) / share * kXcds;
  }
  if (grid >= (1 << 23))  // (threads of a launch are counted in 32 bits)
    return fail(ASYM_EUNSUPPORTED, "prefill: too many rows");
  p.tiles = (int)tiles;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (wide)
    hipLaunchKernelGGL((attn_prefill_kernel<8>), dim3((unsigned)grid), dim3(512), 0, s, p);
  else
    hipLaunchKernelGGL((attn_prefill_kernel<4>), dim3((unsigned)grid), dim3(256), 0, s, p);
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
