// Which kernels a product of 8-bit integers runs: rules for few rows and few tiles, then those of the block-scaled product.
// Plain C++, shared by the device code, the host code and a CPU build.
#pragma once

#include "fd_scaled_rules.h"

namespace fd {

FD_RULE bool int_one_round(int M, int N, int bm, int bn, int cus) { return static_cast<long long>((M + bm - 1) / bm) * ((N + bn - 1) / bn) <= cus; }

// Few rows rather than 32 x 32 tiles of split K-blocks, where both could be: short sums, and few results of sums that the few-row
// kernel's workgroups of 16 columns (N up to 4096) walk.  us, few-row kernel and tiles: 32 x 1536 x 1088 3.3 and 4.1, x 1536 4.4 and 4.2, x 6144
// 10.5 and 7.5; 64 rows of them 3.9 and 4.1, 5.8 and 4.3, 16.2 and 7.7; 1 x 1536 x 4096 4.9 and 5.3, 16 rows 6.3 and 5.8;
// 1 x 4608 x 2048 4.9 and 4.9, x 4096 7.2 and 6.5, x 6144 9.2 and 7.2.
FD_RULE bool int_few(int M, int N, int K, int cus) {
  if (M <= 16) return K <= 18 * 128 || (M <= 8 && !scaled_few_wide(N, cus)) || !int_one_round(M, N, 32, 32, cus);
  return K <= 10 * 128 && scaled_few(M, N, K, false, false, cus);
}

// Tiles whose K-blocks the waves split, where each has a CU: the smallest that do.  us, and in the tiles of the block-scaled rules: 128 x 1536 x
// 6144 (192 of 32 x 32) 8.1 and 17.7, 256 rows (192 of 32 x 64) 10.3 and 17.7, 512 rows (192 of 64 x 64) 13.3 and 18.0; 256 x 1536 x 1088
// 5.0 and 6.3.  A second round costs as much as the first: 256 x 1536 x 6144 in 32 x 32 (384) 13.9, 700 rows in 64 x 64 (264) 23.2
// and 17.9.  64 x 64 with short sums: 1664 x 512 x 1536 (208) 8.5 and 7.7, 512 x 1536 x 1536 6.6 and 7.4.
enum { kSplitNone, kSplit32, kSplit32x64, kSplit64 };
FD_RULE int int_split(int M, int N, int K, int cus) {
  return int_one_round(M, N, 32, 32, cus) ? kSplit32 : int_one_round(M, N, 32, 64, cus) ? kSplit32x64
         : K > 14 * 128 && int_one_round(M, N, 64, 64, cus) ? kSplit64 : kSplitNone;
}

}  // namespace fd
