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

// 256 x 256 tiles, one workgroup per CU, instead of 128 x 128, two: a sixth of the LDS and L2 traffic less per
// flop, but nothing to run while results leave.  Worth it where its rounds are full.  K = 6144, 1536 columns: 9828
// rows (234 tiles on 256 CUs) 84 us against 97, 5000 rows (120 tiles) 61 against 48.  Results in 8 bits cost more
// per tile (their block maxima), so short sums stay with the small tiles: 14280 x 4096 x 1024 (896 tiles) 73
// against 68.
FD_RULE bool scaled_large(int M, int N, int K, bool codes, int cus) {
  const long long tiles = static_cast<long long>((M + 255) / 256) * ((N + 255) / 256);
  const long long rounds = (tiles + cus - 1) / cus;
  return 10 * tiles >= 9 * rounds * cus && (!codes || K >= 24 * 128);
}
// Whether a call whose row count only the device knows launches both kernels.  The one that ends at once takes 4 to
// 5 us, so only where a product at capacity takes ten times that (about 2 PFLOP/s); else the small tiles run alone.
FD_RULE bool scaled_both(int n_max, int N, int K, bool codes, int cus) {
  const long long tiles = static_cast<long long>((n_max + 255) / 256) * ((N + 255) / 256);
  return 10 * tiles >= 9LL * cus && (!codes || K >= 24 * 128) && 2.0 * n_max * N * K >= 1e11;
}

}  // namespace fd
