// Which kernels a block-scaled product runs.  Plain C++, shared by the device code (M is only known
// there), the host code and a CPU build.
#pragma once

#include "fd_rules.h"

namespace fd {

// Row capacities up to which the few-row kernel runs (a larger capacity with few rows at work runs the tiles): 16
// with results in 8 bits, whose blocks want 128 columns of a workgroup, 64 otherwise.  64 x 1536 x 6144: 26 us in
// tiles, whose 12 workgroups walk 48 K-blocks each.
FD_RULE int scaled_few_rows(bool codes) { return codes ? 16 : 64; }
// The tiles' loads run two K-blocks ahead; fewer blocks than three run the few-row kernel at any size.
constexpr int kTileBlocks = 3;

// 256 x 256 tiles, one workgroup per CU, instead of 128 x 128, two: half the LDS and L2 traffic per flop, but nothing
// to run while results leave.  Worth it where its rounds are full.  To bf16, 128 and 256 tiles: 9828 x 1536 x 6144 (234
// large tiles on 256 CUs) 98 and 80 us, 5000 rows of it (120 tiles) 48 and 61; 9828 x 4608 x 1536 75 and 73.  Results
// in 8 bits cost more per tile (their block maxima), so short sums stay with the small tiles: 9828 x 6144 x 1536 with
// GELU 110 and 115, 14280 x 4096 x 1024 68 and 73.
FD_RULE bool scaled_large(int M, int N, int K, bool codes, int cus) {
  const long long tiles = static_cast<long long>((M + 255) / 256) * ((N + 255) / 256);
  const long long rounds = (tiles + cus - 1) / cus;
  return 10 * tiles >= 9 * rounds * cus && (!codes || K >= 24 * 128);
}
// Whether a call whose row count only the device knows launches both kernels.  The one that ends at once takes 4 to
// 5 us, so only where a product at capacity takes some twenty times that; else the small tiles run alone.
FD_RULE bool scaled_both(int n_max, int N, int K, bool codes, int cus) {
  const long long tiles = static_cast<long long>((n_max + 255) / 256) * ((N + 255) / 256);
  return 10 * tiles >= 9LL * cus && (!codes || K >= 24 * 128) && 2.0 * n_max * N * K >= 1.45e11;
}

}  // namespace fd
