// Which kernels a block-scaled product runs.  Plain C++, shared by the device code (M is only known
// there), the host code and a CPU build.
#pragma once

#include "fd_rules.h"

namespace fd {

// bf16 and fp32 results of few rows come from the few-row kernel, whose workgroups take 16, 32 or 64 rows and 16 columns,
// or 32 where those of 16 would not each have a CU: every workgroup reads all of the rows.  16 columns and 32, us: 16 x
// 1536 x 6144 8.9 and 11.4, 16 x 4608 x 6144 14.9 and 11.4, 64 x 4608 x 1536 10.2 and 7.4.
FD_RULE bool scaled_few_wide(int N, int cus) { return (N + 15) / 16 > cus; }
FD_RULE int scaled_few_frags(int M) { return M <= 16 ? 1 : M <= 32 ? 2 : 4; }   // of 16 rows
// Up to 16 rows it is the faster one at every size: 1 x 65536 x 4096 to bf16 51 us, in tiles 74.  Beyond, where each of
// its workgroups has a CU; bf16 results of more than 32 rows, whose sums cost the tiles less, up to 26 K-blocks.  Few-row
// kernel and tiles, us: to bf16 32 x 12288 x 4096 (384 workgroups) 22.5 and 15.6, 32 x 8192 x 4096 (256) 12.5 and 15.4,
// 128 x 1536 x 1536 (192) 6.3 and 7.0, 128 x 1536 x 2560 9.6 and 10.1, x 4096 15.6 and 13.3; to fp32 128 x 1536 x 6144
// 19.4 and 29.3, 128 x 4608 x 6144 (288) 40.8 and 29.8.  Codes, whose blocks want 128 columns of a workgroup, would leave
// it too few of them: 1 x 6144 x 1536 with GELU 11.9, in tiles 10.3.
FD_RULE bool scaled_few(int M, int N, int K, bool codes, bool exact, int cus) {
  const int f = scaled_few_frags(M), columns = scaled_few_wide(N, cus) ? 32 : 16;
  const long long groups = static_cast<long long>((M + 16 * f - 1) / (16 * f)) * ((N + columns - 1) / columns);
  return !codes && (f == 1 || (groups <= cus && (exact || f == 2 || K <= 26 * 128)));
}

// 64 x 128 tiles with three stages of loads instead of 128 x 128 with two, where each has a CU: nothing runs beside a
// workgroup that is alone while it waits, and what bounds it is the K-blocks that it walks.  To bf16, us: 512 x 1536 x
// 6144 (96 tiles of 64 rows) 19.1 and 27.1, 1312 x 1024 x 4096 (168) 14.4 and 20.0; 512 x 4608 x 1536 (288) 11.0 and
// 10.2, 1664 x 1536 x 6144 (312) 33.6 and 28.7.  In 32 x 128 a wave 21.5 and 16.3; to fp32 42.6 for 30.0.
FD_RULE bool scaled_small(int M, int N, int cus) { return static_cast<long long>((M + 63) / 64) * ((N + 127) / 128) <= cus; }

// 256 x 256 tiles, one workgroup per CU, instead of 128 x 128, two: half the LDS and L2 traffic per flop, but nothing
// to run while results leave.  Worth it where its rounds are full.  To bf16, 128 and 256 tiles: 9828 x 1536 x 6144 (234
// large tiles on 256 CUs) 96 and 76 us, 5000 rows of it (120 tiles) 48 and 56; 9828 x 4608 x 1536 72 and 68.  Results
// in 8 bits cost more per tile (their block maxima), so short sums stay with the small tiles: 9828 x 6144 x 1536 with
// GELU 107 and 110.
FD_RULE bool scaled_large(int M, int N, int K, bool codes, int cus) {
  const long long tiles = static_cast<long long>((M + 255) / 256) * ((N + 255) / 256);
  const long long rounds = (tiles + cus - 1) / cus;
  return 10 * tiles >= 9 * rounds * cus && (!codes || K > 22 * 128);
}
// Whether a call whose row count only the device knows launches both kernels.  The one that ends at once takes 4 to
// 5 us, so only where a product at capacity takes some twenty times that; else the small tiles run alone.
FD_RULE bool scaled_both(int n_max, int N, int K, bool codes, int cus) {
  const long long tiles = static_cast<long long>((n_max + 255) / 256) * ((N + 255) / 256);
  return 10 * tiles >= 9LL * cus && (!codes || K > 22 * 128) && 2.0 * n_max * N * K >= 1.45e11;
}

}  // namespace fd
