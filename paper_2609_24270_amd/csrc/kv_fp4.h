// A paged key/value cache in microscaled 4-bit floating point: the page, and the
// wave helpers that its kernels share.
//
// Format.  A block is 32 consecutive channels of one token.  Its scale is a power
// of two, X = 2^(s - 127), s = max(e, 4) - 2 with e the exponent field of the
// block's largest magnitude (so that magnitude / X lies in [4, 8)); a value is
// held as the 4-bit float (1 sign, 2 exponent, 1 mantissa bits: 0, 0.5, 1, 1.5,
// 2, 3, 4, 6) nearest to value / X, ties to the even code, saturated at 6.  s >= 2
// keeps every value a normal bf16, so what is read back is exact.  A block that
// holds an infinity or a NaN is held as s = 255 (NaN) and codes 0.  17 bytes for
// 32 values, 4.25 bits each.
//
// Page: 2176 bytes, 32 tokens of one head: 2048 bytes of codes, 128 of scales, in
// the order in which the matrix instructions of the decode take them, so that a
// wave's loads are whole lines and nothing is transposed on the way (token t,
// channel c, block b = c / 32):
//   keys    token-major: code in nibble c % 2 of byte 64 t + c / 2 (lane (t % 16, b) of
//           v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 bytes of token t, channels
//           32 b ..); scale in byte 2048 + 2 (t % 16 + 16 b) + t / 16.
//   values  channel-major: with q = t % 16 / 4 and j = t % 4 + 4 (t / 16), lane
//           (c % 16, q) of v_mfma_f32_16x16x32_bf16 takes 8 tokens j of channel
//           c: code in nibble j % 2 of byte 1024 (c / 64) + 16 (c % 16 + 16 q) +
//           4 (c / 16 % 4) + j / 2; scale in byte 2048 + 32 q + 4 j + b.  (The
//           scores' result registers hold tokens in this order.)
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace asym {
namespace {

constexpr int kFp4PageBytes = 2176;
constexpr int kFp4ScaleOff = 2048;
constexpr int kKvPageTokens = 32;
constexpr int kKvD = 128;

// The bytes of one page; a page outside the pool reads as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_rsrc(const uint8_t* pool, int page, int pool_pages) {
  const bool in = page >= 0 && page < pool_pages;
  const uint64_t a = (uint64_t)pool + (uint64_t)(uint32_t)(in ? page : 0) * kFp4PageBytes;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(a), (short)0, in ? kFp4PageBytes : 0, 0x00020000);
}

// Sum over the lanes up to and including this one (64 lanes; every lane on).
__device__ __forceinline__ int wave_scan_add(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, true);  // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, true);  // row_bcast 31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan_add(x), 63); }

// Rows of a packed batch: sequence b's are [cu[b], cu[b + 1]), held within [0, total]
// whatever the array says.
__device__ __forceinline__ void packed_rows(const int* __restrict__ cu, int b, int total, int& start, int& n) {
  start = min(max(cu[b], 0), total);
  n = min(max(cu[b + 1], start), total) - start;
}

}  // namespace
}  // namespace asym
