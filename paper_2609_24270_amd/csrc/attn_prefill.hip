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
// wide.  Each wave has two blocks of 16 rows.  Blocks of 64 keys and values stream
// through LDS (buffer_load ... lds, two buffers); per block
//   S^T = K . Q^T   (v_mfma_f32_16x16x32_bf16, K from LDS, Q in registers): a row's 64
//                   scores lie in four lanes, 16 apart;
//   softmax         over the lane's own registers and two exchanges between those four;
//                   the running max is raised only when a row's grows by more than
//                   2^8 (the sums stay in range, the output is rescaled rarely);
//   O^T += V^T . P^T: the score registers, rounded to bf16 (the type of the products'
//                   operands; 2^-8 relative, as the output's own rounding), are the
//                   operand as they lie, because the order of tokens inside a product
//                   is free: V^T is read in that order with ds_read_b64_tr_b16, which
//                   transposes 16-bit values on the way from LDS.
// Scores, max, sum and output are fp32.
//
// What bounds it: the clock that the power cap leaves, and the matrix cores at it.  16384
// causal tokens, 32 query and 8 key heads, take 1870 to 1920 us, 1145 to 1180 TFLOP/s.  The
// clock is 2.1 of 2.4 GHz; the matrix cores work in 51 % of the cycles, the vector units
// (softmax) in 45 %, LDS reads in 25 % and without conflicts.  Fewer cycles give little
// time: with the next block's scores computed beside this block's softmax, and a maximum
// only where a block's sum asks for one, the launch took 15 % fewer of them, at 1.9 GHz, and
// 1 to 3 % less time (and more with as many key as query heads), for registers that
// spill.  Matrix products of 32 rows took 1990 us; 48 rows a wave 2620 (spills); two
// groups of waves in turn on products and softmax 1950 to 2280.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "kv_fp4.h"
#include "prefill_form.h"

namespace asym {
namespace {

constexpr int PD = 128;   // head dimension
constexpr int PN = 64;    // keys per block
constexpr int NT = PN / 16, NK = PN / 32;  // 16-key and 32-key steps of a block
constexpr int NQ = 2;     // 16-row blocks of a wave
constexpr int kXcds = 8;  // workgroup i is dealt to XCD i mod 8 (only speed depends on it)
constexpr int kRowBytes = PD * 2;
constexpr int kTileBytes = PN * kRowBytes;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct PrefillParams {
  const uint16_t *q, *k, *v;
  uint16_t* o;          // [Tq][Hq][128]
  float* lse;           // [Tq][Hq], nullable
  const int *cu_q, *cu_k;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;  // strides, values
  int B, Hq, Hkv, G, Tq, Tk;
  int tiles;            // at least the number of tiles (cut: of pieces) of all sequences
  float* part;          // cut: [H_kv * tiles][kCutRows] of O [128], then of max and sum [2]
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

// Few rows over many keys: the tiles (kCutRows rows) are cut along their keys.  With W the
// blocks of all tiles and heads, pieces of P blocks take the time of P blocks, and W / P of
// them have to be written and joined: P = max(W / kPieces, sqrt(kJoinCost * W), kLeastBlocks).
// A sequence that has at least two pieces' blocks is cut into n = ceil(its key blocks / P),
// which divide each tile's own blocks evenly.  Pieces are numbered by sequence, tile and place.
constexpr int kCutRows = 128;
constexpr int kPieces = 512, kLeastBlocks = 4, kMostPieces = 128;
constexpr float kJoinCost = 0.03f;  // blocks' time that a piece costs to join
__host__ __device__ inline int least_blocks(float work) {
  // (1.001: not less, whatever was rounded)
  const float x = fmaxf(work * (1.001f / kPieces), sqrtf(kJoinCost * work));
  return x < 1e9f ? (int)fmaxf(x, kLeastBlocks - 1) + 1 : 1000000000;
}
__host__ __device__ inline int pieces_of(int blocks, int least) {
  if (blocks < 2 * least) return 1;
  const int n = (blocks + least - 1) / least;
  return n < kMostPieces ? n : kMostPieces;
}
struct Cut {
  int nc, least;
  int t0, nb0;  // of sequence `lane`
};
__device__ void cut_shape(const PrefillParams& p, int c, int& t, int& nb) {
  const int b = 64 * c + (int)(threadIdx.x & 63);
  t = nb = 0;
  if (b < p.B) {
    int qs, qn, ks, kn;
    packed_rows(p.cu_q, b, p.Tq, qs, qn);
    packed_rows(p.cu_k, b, p.Tk, ks, kn);
    t = (int)(((int64_t)qn * p.G + kCutRows - 1) / kCutRows);
    nb = (kn + PN - 1) / PN;
  }
}
__device__ Cut cut_of(const PrefillParams& p) {
  Cut cut;
  cut.nc = (p.B + 63) >> 6;
  cut_shape(p, 0, cut.t0, cut.nb0);
  float work = 0.f;  // (a wave's sum of 16 + 16 bits: tiles are few, so that neither overflows)
  for (int c = 0; c < cut.nc; ++c) {
    int t = cut.t0, nb = cut.nb0;
    if (c) cut_shape(p, c, t, nb);
    work += 65536.f * (float)wave_sum(t * (nb >> 16)) + (float)wave_sum(t * (nb & 0xFFFF));
  }
  cut.least = least_blocks(work * (float)p.Hkv);
  return cut;
}
// The k-th piece (tiles: the k-th tile): its sequence, tile, place among the tile's n
// pieces, and the number of the tile's first piece.  One wave.
template <bool TILES>
__device__ bool find_piece(const PrefillParams& p, int k, int& seq, int& tile, int& place, int& n, int& first) {
  const Cut cut = cut_of(p);
  int before = 0;  // pieces of earlier sequences
  for (int c = 0; c < cut.nc; ++c) {
    int t = cut.t0, nb = cut.nb0;
    if (c) cut_shape(p, c, t, nb);
    const int each = pieces_of(nb, cut.least), mine = TILES ? t : t * each;
    const int upto = wave_scan_add(mine);
    int all = 0;
    if (TILES) all = wave_scan_add(t * each);
    const unsigned long long in = __ballot(k < upto);
    if (in) {
      const int l = __builtin_ctzll(in);
      seq = 64 * c + l;
      n = __builtin_amdgcn_readlane(each, l);
      k -= __builtin_amdgcn_readlane(upto - mine, l);
      tile = TILES ? k : k / n;
      place = TILES ? 0 : k - tile * n;
      first = before + (TILES ? __builtin_amdgcn_readlane(all - t * each, l) + tile * n
                              : __builtin_amdgcn_readlane(upto - mine, l) + tile * n);
      return true;
    }
    k -= __builtin_amdgcn_readlane(upto, 63);
    before += __builtin_amdgcn_readlane(TILES ? all : upto, 63);
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

// 1 KiB from lane addresses voff to LDS bytes dst .. dst + 1023, in lane order (the load takes
// dst from M0, whose write needs a wait state before it, which the compiler does not add here)
__device__ __forceinline__ void lds_load_1k(uint32_t dst, i32x4 rs, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(voff), "s"(rs)
               : "memory", "m0");
}

// 16-byte chunk c of a tile's row r lies at chunk c ^ swz(r): the rows that one read
// takes together (K: 16 rows, one chunk of each; V: 8 rows, two chunks of each) then
// lie on different ones of the 64 banks.  Rows are 256 bytes, all banks once.
__device__ __forceinline__ int swz_k(int row) { return row & 15; }
__device__ __forceinline__ int swz_v(int row) { return (row & 7) << 1; }

typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

// A lane's places in the K and V tiles (bytes from a tile's start).
struct Places {
  uint32_t k[4];  // key n of 16, chunks 4 c + q of channel steps c
  uint32_t v[8];  // channels of groups g of 16, tokens 4 q + n / 4
};
__device__ __forceinline__ Places places(int lane) {
  Places p;
  const int n = lane & 15, q = lane >> 4;
#pragma unroll
  for (int c = 0; c < 4; ++c) p.k[c] = (uint32_t)(n * kRowBytes + (((4 * c + q) ^ swz_k(n)) << 4));
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    const int row = 4 * q + (n >> 2), chunk = 2 * g + ((n & 3) >> 1);
    p.v[g] = (uint32_t)(row * kRowBytes + ((chunk ^ swz_v(row)) << 4) + ((n & 1) << 3));
  }
  return p;
}
// K operand: 16 keys (t-th of the block) x 32 channels (step c)
__device__ __forceinline__ bf16x8 k_frag(const lds_byte* kt, const Places& pl, int t, int c) {
  return *(const __attribute__((address_space(3))) bf16x8*)(kt + pl.k[c] + t * 16 * kRowBytes);
}
// V^T operand: 16 channels (group g) x 32 tokens (step ks of the block)
__device__ __forceinline__ bf16x8 v_frag(const lds_byte* vt, const Places& pl, int g, int ks) {
  union {
    s16x4 s[2];
    bf16x8 b;
  } u;
#pragma unroll
  for (int part = 0; part < 2; ++part)
    u.s[part] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(vt + pl.v[g] + (32 * ks + 16 * part) * kRowBytes));
  return u.b;
}

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

template <int NW, bool CUT>
__global__ void __launch_bounds__(64 * NW, 2) attn_prefill_kernel(PrefillParams p) {
  constexpr int WR = 16 * NQ, BM = WR * NW;
  static_assert(!CUT || BM == kCutRows);
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTileBytes];  // two K tiles, two V tiles
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, q4 = lane >> 4;

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
  int place = 0, pieces = 1, first = 0;
  if constexpr (CUT) {
    if (rank >= p.tiles || !find_piece<false>(p, rank, seq, tile, place, pieces, first)) return;
  } else {
    if (!find_tile(p, BM, rank, seq, tile)) return;
  }
  int qs, Lq, ks, Lk;
  packed_rows(p.cu_q, seq, p.Tq, qs, Lq);
  packed_rows(p.cu_k, seq, p.Tk, ks, Lk);
  const int off = Lk - Lq;
  const int64_t rows = (int64_t)Lq * p.G;
  const int64_t row0 = (int64_t)tile * BM + wave * WR;
  // keys that a row sees; the most over the wave, the least and most over the workgroup
  auto limit = [&](int64_t r) { return p.causal ? max(off + (int)(min(r, rows - 1) / p.G) + 1, 0) : Lk; };
  const int lim_hi = __builtin_amdgcn_readfirstlane(limit(row0 + WR - 1));
  int nblk = (__builtin_amdgcn_readfirstlane(limit((int64_t)tile * BM + BM - 1)) + PN - 1) / PN;
  int nfull = __builtin_amdgcn_readfirstlane(limit((int64_t)tile * BM)) / PN;  // blocks that every row sees whole
  int j0 = 0;
  if (CUT) {
    j0 = (int)((int64_t)nblk * place / pieces);
    nblk = (int)((int64_t)nblk * (place + 1) / pieces);
    nfull = min(max(nfull, j0), nblk);
  }

  // this lane's rows, one of each block of 16 (rows past the last repeat it, and are not stored)
  bf16x8 qf[NQ][4];
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const int64_t row = min(row0 + 16 * b + n, rows - 1);
    const int tok = (int)(row / p.G), g = (int)(row - (int64_t)tok * p.G);
    const uint16_t* qr = p.q + (int64_t)(qs + tok) * p.q_tok + ((int64_t)hk * p.G + g) * p.q_head + 8 * q4;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      u32x4 w = *reinterpret_cast<const u32x4*>(qr + 32 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] ^= p.q_flip;
      qf[b][c] = __builtin_bit_cast(bf16x8, w);
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

  f32x4 o[NQ][8], s[NQ][NT];
  bf16x8 pf[NQ][NK];
  float m[NQ], l[NQ];
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    m[b] = -INFINITY;
    l[b] = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g) o[b][g] = f32x4{};
  }
  auto scores = [&](int j) {
    const lds_byte* kt = k_tile(j);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bf16x8 f = k_frag(kt, pl, t, c);
#pragma unroll
        for (int b = 0; b < NQ; ++b)
          s[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[b][c], c ? s[b][t] : f32x4{}, 0, 0, 0);
      }
  };
  auto softmax = [&] {
    bool up = false;
    float top[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      float x = fmaxf(fmaxf(s[b][0][0], s[b][0][1]), s[b][0][2]);
#pragma unroll
      for (int i = 3; i + 1 < 4 * NT; i += 2) x = fmaxf(fmaxf(x, s[b][i >> 2][i & 3]), s[b][(i + 1) >> 2][(i + 1) & 3]);
      x = fmaxf(x, s[b][NT - 1][3]);
      top[b] = over_quarters(x, [](float a, float c) { return fmaxf(a, c); });
      up |= (top[b] - m[b]) * p.c > 8.f;  // (a first finite max: inf; NaN never)
    }
    if (__any(up)) {
#pragma unroll
      for (int b = 0; b < NQ; ++b) {
        const float m_new = fmaxf(m[b], top[b]);
        const float alpha = __builtin_amdgcn_exp2f((m[b] - (m_new == -INFINITY ? 0.f : m_new)) * p.c);
        l[b] *= alpha;
#pragma unroll
        for (int g = 0; g < 8; ++g) o[b][g] *= alpha;
        m[b] = m_new;
      }
    }
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const float ms = m[b] == -INFINITY ? 0.f : m[b] * p.c;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[b][t][r], p.c, -ms));
          l[b] += e;
          pf[b][t >> 1][4 * (t & 1) + r] = (__bf16)e;
        }
    }
  };
  auto add_pv = [&](int j) {
    const lds_byte* vt = v_tile(j);
#pragma unroll
    for (int kst = 0; kst < NK; ++kst)
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const bf16x8 f = v_frag(vt, pl, g, kst);
#pragma unroll
        for (int b = 0; b < NQ; ++b) o[b][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[b][kst], o[b][g], 0, 0, 0);
      }
  };
  auto arrived = [&] {  // this wave's loads, and with them everyone's
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  // Blocks that every row sees whole.
  if (nfull > j0) {
    load_k(j0);
    load_v(j0);
  }
  for (int j = j0; j < nfull; ++j) {
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
        f(at, *(lds_u32x4*)(v_tile(j) + at));
      }
    };
    uint32_t bad = 0;
    if (p.causal)
      each_word([&](uint32_t, u32x4 w) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7F807F80u) + 0x00800080u;  // an exponent of all ones carries
      });
    const bool guard = p.causal && __syncthreads_or((bad & 0x80008000u) != 0);
    int lim[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) lim[b] = limit(row0 + 16 * b + n);
    if (mine) {
      scores(j);
#pragma unroll
      for (int b = 0; b < NQ; ++b) {
        const int left = lim[b] - j * PN - 4 * q4;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * t + r >= left) s[b][t][r] = -INFINITY;
      }
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
        *(lds_u32x4*)(v_tile(j) + at) = fin;
        *(lds_u32x4*)(k_tile(j) + at) = code;
      });
      __syncthreads();
      if (mine) {
#pragma unroll
        for (int b = 0; b < NQ; ++b)
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            __builtin_amdgcn_sched_barrier(0);  // (one product's registers at a time)
            f32x4 seen = {};
#pragma unroll
            for (int kst = 0; kst < NK; ++kst) {
              u32x4 vis;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = j * PN + 32 * kst + 4 * q4 + 16 * (e >> 1) + 2 * (e & 1);
                vis[e] = (key < lim[b] ? 0x3F80u : 0u) | (key + 1 < lim[b] ? 0x3F800000u : 0u);
              }
              seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(k_tile(j), pl, g, kst), __builtin_bit_cast(bf16x8, vis),
                                                             seen, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int k = (int)seen[r];
              o[b][g][r] += ((k & 127) ? INFINITY : 0.f) + (((k >> 7) & 127) ? -INFINITY : 0.f) + (k >= 16384 ? NAN : 0.f);
            }
          }
      }
    }
    if (mine) add_pv(j);
  }

  if (CUT && pieces > 1) {  // the piece's unscaled output, max and sum (-1: it is empty) to the joining launch
    const size_t slot = ((size_t)hk * p.tiles + first + place) * kCutRows;
    float* po = p.part + slot * PD;
    float* pm = p.part + (size_t)p.Hkv * p.tiles * kCutRows * PD + slot * 2;
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const int r = wave * WR + 16 * b + n;
      const float lt = over_quarters(l[b], [](float a, float c) { return a + c; });
      if ((int64_t)tile * BM + r >= rows) continue;
      if (q4 == 0) *reinterpret_cast<float2*>(pm + 2 * r) = float2{m[b], j0 < nblk ? lt : -1.f};
      if (j0 < nblk) {
#pragma unroll
        for (int g = 0; g < 8; ++g) *reinterpret_cast<f32x4*>(po + (size_t)r * PD + 16 * g + 4 * q4) = o[b][g];
      }
    }
    return;
  }
  // a lane has 4 of every 16 channels of a row; two groups of them, exchanged between the
  // quarters, make 16 bytes
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const float lt = over_quarters(l[b], [](float a, float c) { return a + c; });
    const float inv = lt > 0.f ? 1.f / lt : (lt == 0.f ? 0.f : lt);  // (NaN stays)
    const int64_t r = row0 + 16 * b + n, row = min(r, rows - 1);
    const int tok = (int)(row / p.G);
    const int64_t orow = (int64_t)(qs + tok) * p.Hq + (int64_t)hk * p.G + (row - (int64_t)tok * p.G);
    uint16_t* dst = p.o + orow * PD;
#pragma unroll
    for (int g = 0; g < 8; g += 2) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4& x = o[b][g + (e >> 1)];
        const bf16x2 y = {(__bf16)(x[2 * (e & 1)] * inv), (__bf16)(x[2 * (e & 1) + 1] * inv)};
        w[e] = __builtin_bit_cast(uint32_t, y);
      }
      const auto x = __builtin_amdgcn_permlane16_swap(w[0], w[2], false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(w[1], w[3], false, false);
      // quarter 0: channels 0 .. 7 of group g, 1: 0 .. 7 of group g + 1, 2: 8 .. 15 of g, 3: of g + 1
      if (r < rows)
        *reinterpret_cast<u32x4*>(dst + 16 * (g + (q4 & 1)) + 8 * (q4 >> 1)) = u32x4{x[0], y[0], x[1], y[1]};
    }
    if (p.lse && r < rows && q4 == 0) p.lse[orow] = lt == 0.f ? -INFINITY : m[b] * p.scale + __logf(lt);
  }
}

// Joins the pieces of the tiles that were cut, in order: a wave has four rows of a tile,
// a lane eight channels of one.
constexpr int kJoinRows = 16, kJoinWaves = 4;
__global__ void __launch_bounds__(64 * kJoinWaves) attn_prefill_join_kernel(PrefillParams p) {
  constexpr int kParts = kCutRows / kJoinRows;
  const int hk = (blockIdx.x / kParts) % p.Hkv, rank = blockIdx.x / kParts / p.Hkv;
  int seq, tile, place, pieces, first;
  if (!find_piece<true>(p, rank, seq, tile, place, pieces, first)) return;
  if (pieces == 1 || first + pieces > p.tiles) return;
  int qs, Lq;
  packed_rows(p.cu_q, seq, p.Tq, qs, Lq);
  const int64_t rows = (int64_t)Lq * p.G;
  const int c = threadIdx.x & 15, r = (int)(blockIdx.x % kParts) * kJoinRows + (int)(threadIdx.x >> 4);
  const int64_t row = (int64_t)tile * kCutRows + r;
  if (row >= rows) return;  // (a row's 16 lanes leave together)
  const size_t slot = ((size_t)hk * p.tiles + first) * kCutRows + r;
  const float* po = p.part + slot * PD + 8 * c;
  const float* pm = p.part + (size_t)p.Hkv * p.tiles * kCutRows * PD + slot * 2;
  float top = -INFINITY;
  for (int s = c; s < pieces; s += 16) {
    const float2 x = *reinterpret_cast<const float2*>(pm + (size_t)s * kCutRows * 2);
    if (!(x.y < 0.f)) top = fmaxf(top, x.x);
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  const float at = top == -INFINITY ? 0.f : top;
  float lt = 0.f;
  f32x4 acc[2] = {};
#pragma unroll 4
  for (int s = 0; s < pieces; ++s) {
    const float2 x = *reinterpret_cast<const float2*>(pm + (size_t)s * kCutRows * 2);
    const f32x4* y = reinterpret_cast<const f32x4*>(po + (size_t)s * kCutRows * PD);
    const f32x4 y0 = y[0], y1 = y[1];
    const bool on = !(x.y < 0.f);  // (an empty piece has no output)
    const float w = __builtin_amdgcn_exp2f((x.x - at) * p.c);
    lt += on ? x.y * w : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[0][e] += on ? y0[e] * w : 0.f;
      acc[1][e] += on ? y1[e] * w : 0.f;
    }
  }
  const float inv = lt > 0.f ? 1.f / lt : (lt == 0.f ? 0.f : lt);  // (NaN stays)
  const int tok = (int)(row / p.G);
  const int64_t orow = (int64_t)(qs + tok) * p.Hq + (int64_t)hk * p.G + (row - (int64_t)tok * p.G);
  u32x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x4& a = acc[e >> 1];
    const bf16x2 y = {(__bf16)(a[2 * (e & 1)] * inv), (__bf16)(a[2 * (e & 1) + 1] * inv)};
    out[e] = __builtin_bit_cast(uint32_t, y);
  }
  *reinterpret_cast<u32x4*>(p.o + orow * PD + 8 * c) = out;
  if (p.lse && c == 0) p.lse[orow] = lt == 0.f ? -INFINITY : top * p.scale + __logf(lt);
}

// Which form a call takes, from its sizes alone.
struct Form {
  bool wide, cut;
  int64_t tiles;  // of a head, at least (cut: pieces)
  int64_t whole;  // cut: tiles of a head, at least
};
Form form_of(int B, int Hq, int Hkv, int Tq, int Tk) {
  const int G = Hq / Hkv;
  auto count = [&](int rows) { return (int64_t)Tq * G / rows + B; };  // sequences end in a part tile each
  Form f = {};
  f.wide = prefill_wide(B, G, Hkv, Tq);
  f.tiles = f.whole = count(f.wide ? 256 : kCutRows);
  if (!f.wide && f.tiles * Hkv < 512) {
    // Cut (us, whole tiles first; 32 / 8 heads): 8 tokens behind 1000 keys 24 14, 4 behind
    // 4000 76 16, 256 behind 16125 298 92, 4 behind 32000 and 39 times 4 behind 300 569 49.
    // It costs a launch (12 of 100 behind 700, which it would leave whole: 33 37).  The pieces'
    // places grow with the tiles, of which each sequence has one at least, so from 512 tiles
    // over all heads on nothing is cut (56 sequences of 4 tokens, one of them behind 32000 and
    // the others behind 300: 46 us; 57: 567).
    const int blocks = Tk / PN / B;  // of the mean sequence; a long batch may hold a long one
    f.cut = Tk >= 8192 || pieces_of(blocks, least_blocks((float)(f.tiles * Hkv) * (float)blocks)) > 1;
    if (f.cut) f.tiles += (kPieces + Hkv - 1) / Hkv;
  }
  return f;
}
size_t part_bytes(const Form& f, int Hkv) {
  return f.cut ? (size_t)Hkv * (size_t)f.tiles * kCutRows * (PD + 2) * sizeof(float) : 0;
}

}  // namespace
}  // namespace asym

extern "C" int asym_attn_prefill_workspace(int B, int H_q, int H_kv, int T_q, int T_k, size_t* bytes) {
  using namespace asym;
  if (B < 0 || T_q < 0 || T_k < 0 || H_q < 1 || H_kv < 1)
    return fail(ASYM_EINVAL, "prefill: B, T_q and T_k must be >= 0, H_q and H_kv >= 1");
  if (H_q % H_kv) return fail(ASYM_EINVAL, "prefill: H_kv must divide H_q");
  if (!bytes) return fail(ASYM_EINVAL, "prefill: null pointer");
  *bytes = B == 0 || T_q == 0 ? 0 : part_bytes(form_of(B, H_q, H_kv, T_q, T_k), H_kv);
  return ASYM_OK;
}

extern "C" int asym_attn_prefill_bf16(int B, int H_q, int H_kv, int D, int T_q, int T_k, const void* q, int64_t q_token,
                                      int64_t q_head, const void* k, int64_t k_token, int64_t k_head, const void* v,
                                      int64_t v_token, int64_t v_head, void* o, float* lse, const int32_t* cu_q,
                                      const int32_t* cu_k, float scale, int causal, int mapping, void* workspace,
                                      size_t workspace_bytes, void* stream) {
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
  PrefillParams p = {};
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
  const Form form = form_of(B, H_q, H_kv, T_q, T_k);
  if (form.cut && (!workspace || ((uintptr_t)workspace & 15u) || workspace_bytes < part_bytes(form, H_kv)))
    return fail(ASYM_EINVAL, "prefill: workspace null, misaligned or too small");
  const int64_t tiles = form.tiles;
  int64_t grid = tiles * H_kv;
  if (p.aware && kXcds % H_kv == 0) {
    const int share = kXcds / H_kv;
    grid = (tiles + share - 1) / share * kXcds;
  }
  if (!prefill_fits(grid, form.wide)) return fail(ASYM_EUNSUPPORTED, "prefill: too many rows");
  p.tiles = (int)tiles;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (form.cut) {
    p.part = static_cast<float*>(workspace);
    hipLaunchKernelGGL((attn_prefill_kernel<4, true>), dim3((unsigned)grid), dim3(256), 0, s, p);
    ASYM_HIP(hipGetLastError());
    const int64_t rows = form.whole * H_kv * (kCutRows / kJoinRows);
    hipLaunchKernelGGL(attn_prefill_join_kernel, dim3((unsigned)rows), dim3(64 * kJoinWaves), 0, s, p);
  } else if (form.wide) {
    hipLaunchKernelGGL((attn_prefill_kernel<8, false>), dim3((unsigned)grid), dim3(512), 0, s, p);
  } else {
    hipLaunchKernelGGL((attn_prefill_kernel<4, false>), dim3((unsigned)grid), dim3(256), 0, s, p);
  }
  ASYM_HIP(hipGetLastError());
  return ASYM_OK;
}
