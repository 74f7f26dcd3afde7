// Which kernels a product of 8-bit integers runs.
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

// 256 x 256 tiles, one workgroup a CU, rather than 128 x 128, two: the shorter of what their rounds take, in hundredths of a K-block of
// 128 x 128 tiles on full CUs (0.82 us).  A round of small tiles on half the CUs' places (one each) takes 0.52 a K-block and 2.7 at its
// ends, of large ones 1.2 on up to half the CUs, 1.9 and more on all of them (power), and 9, 12 with fp32 results.  us, small and
// large: 5000 x 1600 x 6400 (1.02 rounds and 0.55) 74 and 66, 2048 x 6400 x 6400 (1.56, 0.78) 99 and 80, 2600 rows (2.05, 1.07) 125 and
// 149, 9828 rows (7.52, 3.81) 423 and 351; 6000 x 4608 x 1536 to fp32 (3.30, 1.69) 52 and 58, 4000 x 3200 x 3200 (1.56, 0.81) 52 and 46.
FD_RULE bool int_large(int M, int N, int K, bool wide, int cus) {
  const long long blocks = (K + 127) / 128, ends = wide ? 1200 : 900;
  const long long small = static_cast<long long>((M + 127) / 128) * ((N + 127) / 128), large = static_cast<long long>((M + 255) / 256) * ((N + 255) / 256);
  const long long full = large / cus, rest = large % cus, over = 2 * rest > cus ? 2 * rest - cus : 0;
  return full * (190 * blocks + ends) + (rest ? 120 * blocks + 80 * blocks * over / cus + ends : 0) < (small + cus - 1) / cus * (52 * blocks + 270);
}

// Whether a call whose row count only the device knows launches both kernels, of which one ends at once (4 to 5 us): where large tiles
// win at capacity by more than that, or may at a part of it as in the block-scaled product.
FD_RULE bool int_both(int n_max, int N, int K, bool wide, int cus) {
  return scaled_both(n_max, N, K, false, cus) || (2.0 * n_max * N * K >= 8e10 && int_large(n_max, N, K, wide, cus));
}

// The kernel of a call of `rows` rows on a device of `num_cus` CUs: few rows, tiles of split K-blocks, tiles of 64 x 128, 128 x 128
// alone on their CUs or two, 256 x 256, or (both) whichever of the last two the row count on the device calls for.
enum IntKernel { kIntFew, kIntSplit32, kIntSplit32x64, kIntSplit64, kInt64, kIntAlone, kInt128, kInt256, kIntBoth };
FD_RULE IntKernel int_kernel(int rows, int N, int K, bool wide, bool counted_on_device, int num_cus) {
  if (int_few(rows, N, K, num_cus)) return kIntFew;
  switch (int_split(rows, N, K, num_cus)) {
    case kSplit32: return kIntSplit32;
    case kSplit32x64: return kIntSplit32x64;
    case kSplit64: return kIntSplit64;
    default: break;
  }
  const int cus = num_cus / 8 * 8;   // the tile order counts on whole rounds of the 8 XCDs
  if (scaled_small(rows, N, cus)) return kInt64;
  if (counted_on_device && int_both(rows, N, K, wide, cus)) return kIntBoth;
  if (!counted_on_device && int_large(rows, N, K, wide, cus)) return kInt256;
  return int_one_round(rows, N, 128, 128, cus) ? kIntAlone : kInt128;
}

}  // namespace fd
