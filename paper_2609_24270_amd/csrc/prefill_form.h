// Which row tiles prompt attention takes.  Host rules, plain functions of sizes.
#pragma once
#include <cstdint>

namespace asym {

// Tiles of 256 rows (a row: a token and one of its G query heads of a group) read the keys
// half as often as tiles of 128, and are faster once the rows fill two for every CU (us, 128
// rows first: 16384 tokens, 32 / 8 heads 1958 1908, 4096 tokens 142 132, two of 4096 with 16
// / 16 heads 147 136); with fewer the last ones are waited for (2048 tokens, 32 / 8 heads 51
// 61, 3000 behind 8000 436 479, 1024 26 34).  Sequences that one tile of 128 rows holds fill
// half of a wide one at most, and a wave without rows works as long as one with them: 256
// rows only if the mean sequence has more than 128.  us, 128 rows first, n sequences of r
// rows, alone and behind 1000 keys each (the lengths of a call are on the device; one such
// mean with lengths from 1 to twice it gives the same order):
//   32 / 8 heads   n 1025, r 32   291  565   1295 2124    32 / 32 heads   n 513, r 16    400  790   1987 3000
//                  n 257, r 128    56   91    297  421                    n 65, r 128     63  103    283  394
//                  n 171, r 192    60   62    351  266                    n 52, r 160     79   99    408  337
//                  n 129, r 256    56   58    290  223                    n 33, r 256     82   95    297  243
//                  n 103, r 320    59   76    313  311                    n 26, r 320     79  110    340  348
inline bool prefill_wide(int B, int G, int H_kv, int T_q) {
  const int64_t rows = (int64_t)T_q * G;
  return rows / 256 * H_kv >= 512 && rows > 128ll * B;
}

// Threads of a launch are counted in 32 bits; a workgroup has two for a row.
inline bool prefill_fits(int64_t workgroups, bool wide) { return workgroups * (wide ? 512 : 256) < (1ll << 32); }

}  // namespace asym
