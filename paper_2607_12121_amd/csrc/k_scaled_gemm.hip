// The product of 8-bit rows and weights with block scales:
//   Y[M][N] = act(sum over K-blocks kb of 2^(sa[row][kb] + sw[col / 128][kb] - 254) (A . W^T)_kb + bias)
// on v_mfma_scale_f32_16x16x128_f8f6f4 and 32x32x64: a block is one or two steps of the instruction, the scale bytes
// are its operands and the sum is kept in fp32 accumulators.
#include <type_traits>

#include "fd_scaled.h"
#include "fd_scaled_rules.h"
#include "fd_tile_loads.h"

namespace {

using fd::bf16x2_t;
using fd::kScaleBlock;

enum { kToBf16, kToF32, kToCodes };

// Two ways to the sum of one K-block of 128:
// - 8-bit: v_mfma_scale_f32_*_f8f6f4.  It adds 8 products at a time on a grid 2^-13 below the
//   largest of them (measured: 1 + 2^-14 gives 1 within such a group, and is exact across groups and
//   with the accumulator; v_mfma_f32_32x32x16_fp8_fp8 is no different), which leaves random operands'
//   sums off by 2e-5 of their size.  Outputs of 8 (bf16) or 4 (e4m3) bits of mantissa round by 100 times
//   that at least; one that near a tie, or a block maximum that near a scale's limit, may go the other way.
//   Codes through the exact way below: 1021 x 4288 x 1088 20.7 us for 14.4, 9828 x 6144 x 1536 183 for 107.
// - exact: the codes times their scales as bf16 (exact from 2^-126 on) through v_mfma_f32_*_bf16, half the
//   rate, whose sums are fp32's.  fp32 outputs take this one.
struct Mma8 {
  typedef i32x8_t frag;
  static FD_DEVICE frag make(i32x8_t x, uint32_t) { return x; }
  static FD_DEVICE f32x4_t mma(const frag& w, const frag& a, f32x4_t c, uint32_t sw, uint32_t sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, static_cast<int>(sw), 0, static_cast<int>(sa));
  }
  static FD_DEVICE f32x16_t mma(const frag& a, const frag& w, f32x16_t c, uint32_t sa, uint32_t sw) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, w, c, 0, 0, 0, static_cast<int>(sa), 0, static_cast<int>(sw));
  }
};
struct MmaExact {
  struct frag { bf16x8_t p[4]; };   // piece p: the lane's values 8 p .. 8 p + 7 (the same ones of both operands)
  static FD_DEVICE frag make(i32x8_t x, uint32_t s) {
    const float scale = __uint_as_float((s & 255u) << 23);
    frag f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, false);
      const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, true);
      f.p[i >> 1][4 * (i & 1) + 0] = lo[0]; f.p[i >> 1][4 * (i & 1) + 1] = lo[1];
      f.p[i >> 1][4 * (i & 1) + 2] = hi[0]; f.p[i >> 1][4 * (i & 1) + 3] = hi[1];
    }
    return f;
  }
  static FD_DEVICE f32x4_t mma(const frag& w, const frag& a, f32x4_t c, uint32_t, uint32_t) {
#pragma unroll
    for (int p = 0; p < 4; ++p) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[p], a.p[p], c, 0, 0, 0);
    return c;
  }
  static FD_DEVICE f32x16_t mma(const frag& a, const frag& w, f32x16_t c, uint32_t, uint32_t) {
#pragma unroll
    for (int p = 0; p < 4; ++p) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[p], w.p[p], c, 0, 0, 0);
    return c;
  }
};

// The few-row kernel's blocks are 16 x 16 with the weight fragment as the first operand, so that an accumulator
// holds the transposed block: lane l a row (l & 15) and four columns.  The 16 weight rows of fragment j of a
// wave's 16 NF columns are 4 NF (x >> 2) + 4 j + (x & 3), x < 16: together the NF fragments give a lane 4 NF
// consecutive columns, 4 NF (l >> 4) on.
//
// One row's 4 NF columns from col on (col a multiple of 4 NF; N is a multiple of 16, so each 16 lie
// inside or outside).
template <int KIND, int NF>
FD_DEVICE void store_row(const fdh::ScaledArgs& g, bool row_ok, int row, int col, const f32x4_t (&acc)[NF], const float4 (&bias)[NF]) {
  float v[4 * NF];
#pragma unroll
  for (int j = 0; j < NF; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) v[4 * j + r] = acc[j][r] + (r == 0 ? bias[j].x : r == 1 ? bias[j].y : r == 2 ? bias[j].z : bias[j].w);
  if (g.gelu) {
#pragma unroll
    for (int e = 0; e < 4 * NF; ++e) v[e] = fd::gelu(v[e]);
  }
  const size_t at = static_cast<size_t>(row) * g.N + col;
  if constexpr (KIND == kToBf16 && NF == 1) {
    if (row_ok && col < g.N) *reinterpret_cast<uint2*>(g.y_bf16 + at) = make_uint2(fd::pack_bf2(v[0], v[1]), fd::pack_bf2(v[2], v[3]));
  } else if constexpr (KIND == kToBf16) {
#pragma unroll
    for (int i = 0; i < NF / 2; ++i) {
      const float* x = v + 8 * i;
      if (row_ok && col + (8 * i & 16) < g.N)
        *reinterpret_cast<uint4*>(g.y_bf16 + at + 8 * i) = make_uint4(fd::pack_bf2(x[0], x[1]), fd::pack_bf2(x[2], x[3]), fd::pack_bf2(x[4], x[5]), fd::pack_bf2(x[6], x[7]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const float* x = v + 4 * i;
      if (row_ok && col + (4 * i & 16) < g.N) *reinterpret_cast<float4*>(g.y_f32 + at + 4 * i) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
}

// ---------------------------------------------------------------- few rows

// Few rows: the weights are read once (by every 64 rows), so what counts is how many of their bytes are on the way.  A workgroup
// takes the rows' FM fragments and 16 NF columns, its waves the K-blocks in turn, operands straight from memory into
// registers, up to DEEP blocks at a time; the waves' sums meet in LDS.  DEEP is about what 128 registers hold, so that a
// CU takes two workgroups: with six blocks and one workgroup, 16 x 4608 x 4096 12.6 us, with three 11.6.  Past its last
// block a wave loads nothing (loads of nothing, cleared afterwards: 17.1 us).
constexpr int kFewWaves = 8;

template <int KIND, class Mma, int FM, int NF, int DEEP>
__global__ __launch_bounds__(kFewWaves * 64) void scaled_few_kernel(fdh::ScaledArgs g) {
  __shared__ f32x4_t part[kFewWaves][FM][NF][64];
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lg = lane >> 4;
  const int K = g.K, nk = (K + kScaleBlock - 1) / kScaleBlock, ld = fd::scale_stride(K);
  const int n0 = blockIdx.x * 16 * NF, m0 = blockIdx.y * 16 * FM;
  if (m0 >= M) return;
  const uint8_t* sw = g.w_scale + static_cast<size_t>(n0 / kScaleBlock) * ld;
  const uint8_t* w[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j)
    w[j] = g.w + static_cast<size_t>(min(n0 + 4 * NF * (l16 >> 2) + 4 * j + (l16 & 3), g.N - 1)) * K;
  float4 bias[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j) bias[j] = g.bias ? *reinterpret_cast<const float4*>(g.bias + min(n0 + 4 * NF * lg + 4 * j, g.N - 4)) : make_float4(0, 0, 0, 0);
  f32x4_t acc[FM][NF] = {};
  for (int kb = wave; kb < nk; kb += kFewWaves * DEEP) {
    Piece wf[DEEP][NF], af[DEEP][FM];
    uint32_t s_w[DEEP], s_a[DEEP][FM];
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      const int b = kb + d * kFewWaves, k = b * kScaleBlock + 32 * lg;
      if (b >= nk) break;
#pragma unroll
      for (int j = 0; j < NF; ++j) wf[d][j] = load32(w[j], k, K);
      s_w[d] = sw[b];
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const size_t row = min(m0 + 16 * i + l16, M - 1);
        af[d][i] = load32(g.a + row * K, k, K);
        s_a[d][i] = g.a_scale[row * ld + b];
      }
    }
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      const int b = kb + d * kFewWaves, k = b * kScaleBlock + 32 * lg;
      if (b >= nk) break;
      typename Mma::frag wd[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) wd[j] = Mma::make(inside(wf[d][j], k, K), s_w[d]);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const typename Mma::frag ad = Mma::make(inside(af[d][i], k, K), s_a[d][i]);
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = Mma::mma(wd[j], ad, acc[i][j], s_w[d], s_a[d][i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) part[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  if (wave < FM) {   // a wave per 16 rows adds the waves' sums in order
    f32x4_t sum[NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      sum[j] = part[0][wave][j][lane];
#pragma unroll
      for (int p = 1; p < kFewWaves; ++p) sum[j] += part[p][wave][j][lane];
    }
    const int row = m0 + 16 * wave + l16;
    store_row<KIND, NF>(g, row < M, row, n0 + 4 * NF * lg, sum, bias);
  }
}

// ---------------------------------------------------------------- tiles

// A workgroup of WM x WN waves with a tile of 32 FI WM rows x 32 NJ WN columns, K-steps of one block; a
// wave owns FI x NJ blocks of 32 x 32.  Tiles stream from memory into a ring of LDS stages
// (buffer_load ... lds); in LDS a tile row is eight 16-byte chunks, chunk c of row r at c ^ swz(r), so
// that the 16 lanes that read a fragment together meet 16 different 16-byte bank groups.
template <int FI_, int NJ_, int WM_, int WN_, int STAGES_>
struct Tile {
  static constexpr int FI = FI_, NJ = NJ_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int BM = 32 * FI * WM, BN = 32 * NJ * WN;
  static constexpr int LOADS_A = BM / 8 / WAVES, LOADS_W = BN / 8 / WAVES;        // 8 rows of 128 bytes per wave-load
  static constexpr int SCALE_WAVES = (BM + 63) / 64;                              // waves that load row scales; the others column scales
  static constexpr int ISSUED = LOADS_A + LOADS_W + 1;                            // and one of scales or bias
  static constexpr int SIDE = (BM + BN) * 8;                                      // chunk where a stage's scales begin
  static constexpr int CHUNKS = SIDE + SCALE_WAVES * 16 + 16;                     // row scales, then 256 bytes of column scales
  static constexpr int BIAS = STAGES * CHUNKS;                                    // four slots of the columns' bias
  static constexpr int TOTAL = BIAS + 4 * BN / 4;
  static_assert(BN % kScaleBlock == 0 && (NJ == 4 || NJ == 2), "whole blocks of columns");
  static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && WAVES % 2 == 0 && SCALE_WAVES < WAVES && BN <= 64 * WAVES, "whole wave-loads");
  static FD_DEVICE int swz(int r) { return (r >> 1) & 7; }
  // Column of LDS row p: fragment j of a wave's columns holds every NJ-th, from j on, so that a lane of the product
  // has NJ consecutive columns in its NJ fragments.
  static FD_DEVICE int column(int p) { return (p & ~(32 * NJ - 1)) + NJ * (p & 31) + ((p >> 5) & (NJ - 1)); }
};

// 32 rows x 32 NJ columns to memory: acc[j][r] is row 8 (r >> 2) + 4 half + (r & 3) and column NJ l32 + j, so that
// 32 lanes store one row's columns side by side (with rows spread over the lanes, 16 bytes of 64 rows a store,
// the L2 took 19 us for the 32 MB of a round of tiles).  Every store issues whatever the row, rows and columns
// outside go nowhere: the waits count the stores.  rows: how many rows from the first on lie inside; off: byte
// offset of the first row's columns of this lane; pitch: bytes of a row.
template <int KIND, int NJ>
struct Rows32 {
  static_assert(KIND != kToCodes || NJ == 4, "32 lanes hold a block's columns");
  static constexpr int STORES = KIND == kToCodes ? 17 : 16;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

  // The largest of each of 16 rows over the 32 lanes of a half, row r's in the lanes with l32 % 16 == r: at each
  // level a lane hands its partner (mirrored within 16, 8, 4, 2) the half of the rows that the partner keeps.
  template <int CTRL>
  static FD_DEVICE uint32_t level(uint32_t low, uint32_t high, bool up) {
    const uint32_t give = up ? low : high, keep = up ? high : low;
    return max(keep, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(give), CTRL, 0xf, 0xf, true)));
  }
  static FD_DEVICE uint32_t row_tops(uint32_t (&t)[16], int l32) {
#pragma unroll
    for (int r = 0; r < 8; ++r) t[r] = level<0x140>(t[r], t[r + 8], l32 & 8);   // row_mirror
#pragma unroll
    for (int r = 0; r < 4; ++r) t[r] = level<0x141>(t[r], t[r + 4], l32 & 4);   // row_half_mirror
#pragma unroll
    for (int r = 0; r < 2; ++r) t[r] = level<0x1b>(t[r], t[r + 2], l32 & 2);    // quad_perm 3 2 1 0
    const uint32_t top = level<0xb1>(t[0], t[1], l32 & 1);                      // quad_perm 1 0 3 2
    return max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16, fd::kWave)));
  }
  template <int R>
  static FD_DEVICE void put_codes(const f32x16_t (&v)[4], float inv, __amdgpu_buffer_rsrc_t y, bool col_ok, int half, int rows,
                                  uint32_t off, uint32_t pitch) {
    const float x = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(inv), 0x150 + R, 0xf, 0xf, true));   // row_newbcast
    const uint32_t w = fd::pack_codes(v[0][R] * x, v[1][R] * x, v[2][R] * x, v[3][R] * x);
    constexpr int row = 8 * (R >> 2) + (R & 3);
    __builtin_amdgcn_raw_buffer_store_b32(w, y, col_ok && row + 4 * half < rows ? off : kNowhere, row * pitch, 0);
    if constexpr (R < 15) put_codes<R + 1>(v, inv, y, col_ok, half, rows, off, pitch);
  }
  static FD_DEVICE void store(f32x16_t (&v)[NJ], const float (&bias)[NJ], bool gelu, __amdgpu_buffer_rsrc_t y, bool col_ok, int l32, int half,
                              int rows, uint32_t off, uint32_t pitch, __amdgpu_buffer_rsrc_t scale, uint32_t scale_off, uint32_t scale_pitch) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) v[j] += bias[j];
    if (gelu) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) v[j][r] = fd::gelu(v[j][r]);
    }
    if constexpr (KIND == kToCodes) {
      uint32_t t[16];
#pragma unroll
      for (int r = 0; r < 16; ++r)
        t[r] = col_ok ? max(max(fd::mag_bits(v[0][r]), fd::mag_bits(v[1][r])), max(fd::mag_bits(v[2][r]), fd::mag_bits(v[3][r]))) : 0u;
      const uint32_t s = fd::scale_byte(row_tops(t, l32));
      const int row = 8 * ((l32 >> 2) & 3) + 4 * half + (l32 & 3);
      __builtin_amdgcn_raw_buffer_store_b8(static_cast<uint8_t>(s), scale, l32 < 16 && row < rows ? scale_off + row * scale_pitch : kNowhere, 0, 0);
      put_codes<0>(v, fd::scale_inverse(s), y, col_ok, half, rows, off, pitch);
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + (r & 3);
        const uint32_t to = col_ok && row + 4 * half < rows ? off : kNowhere;
        if constexpr (KIND == kToBf16 && NJ == 2)
          __builtin_amdgcn_raw_buffer_store_b32(fd::pack_bf2(v[0][r], v[1][r]), y, to, row * pitch, kStream);
        else if constexpr (NJ == 2)
          __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v[0][r]), __float_as_uint(v[1][r])}, y, to, row * pitch, kStream);
        else if constexpr (KIND == kToBf16)
          __builtin_amdgcn_raw_buffer_store_b64(u32x2{fd::pack_bf2(v[0][r], v[1][r]), fd::pack_bf2(v[2][r], v[3][r])}, y, to, row * pitch, kStream);
        else
          store_f4(v[0][r], v[1][r], v[2][r], v[3][r], y, to, row * pitch);
      }
    }
  }
};

// The K-steps of all of a workgroup's tiles are one sequence: the loads run STAGES steps ahead of the
// products, into the next tile too, and a tile's results leave while the next one's first stages land.
//
// A step's eight sub-steps s = (half of K, column fragment) each read one weight fragment two sub-steps
// ahead.  After sub-step 1 the wave has read its rows, after sub-step 5 its columns; a barrier there frees
// that part of the stage for the load STAGES steps on, which goes out a few instructions at a time behind
// products.  The second barrier also publishes the next stage, whose first fragments are read behind
// sub-steps 6 and 7, so that no sub-step waits for LDS or for the barrier with nothing to compute.  (Waves of two
// fragments a half have four sub-steps and the one barrier after sub-step 1, which frees all of the stage.  One barrier
// in the middle of a step, with its operands in registers: the loads have 5 sub-steps to land instead of 7 and 10,
// 1664 x 1536 x 6144 in 128 x 128 tiles 36.4 us against 28.2.)  A step is one basic block: across branches the
// compiler gathers the products at the end.
//
// The 256 x 256 tiles leave the results' offsets no registers: the compiler keeps 10 (bf16), 12 (fp32) and 14 (codes) of
// them in scratch, and waits for each reload between the stores, which holds the stores before it and the next tile's
// loads up.  The counted waits only get stricter by it.
template <class T, int KIND, class Mma>
FD_DEVICE void scaled_tiles(const fdh::ScaledArgs& g, int M, uint4* ring) {
  constexpr int FI = T::FI, NJ = T::NJ, STAGES = T::STAGES, kSubs = 2 * NJ;
  constexpr int kSize = KIND == kToCodes ? 1 : KIND == kToBf16 ? 2 : 4;
  constexpr int kStores = FI * Rows32<KIND, NJ>::STORES;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WN, wn = wave % T::WN;
  const int K = g.K, blocks = (K + kScaleBlock - 1) / kScaleBlock, nk = max(blocks, STAGES), ld = fd::scale_stride(K);
  const int tiles_m = (M + T::BM - 1) / T::BM, tiles_n = (g.N + T::BN - 1) / T::BN, tiles = tiles_m * tiles_n;
  const int per_xcd = (tiles + 7) / 8;
  const uint32_t ring_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)ring));

  // Tile of turn u of this workgroup: consecutive tiles on one XCD (a workgroup runs on XCD
  // blockIdx.x % 8), in groups of 8 row tiles x every column tile, row tile fastest, so that the tiles
  // an XCD runs at once share operand rows in its L2.
  auto tile_at = [&](int u, int& m0, int& n0) -> bool {
    const int tile = (u % 8) * per_xcd + u / 8;
    if (u >= per_xcd * 8 || tile >= tiles) return false;
    const int grp = tile / (8 * tiles_n), in = tile - grp * 8 * tiles_n, gm = min(8, tiles_m - 8 * grp);
    m0 = (8 * grp + in % gm) * T::BM;
    n0 = in / gm * T::BN;
    return true;
  };

  // ---- the loads: of K-block lk of the tile at (lm0, ln0)
  int u = blockIdx.x, lk = 0, lm0, ln0;
  if (!tile_at(u, lm0, ln0)) return;
  i32x4_t ra, rw, rside;
  int turn = 3;
  uint32_t off_a[T::LOADS_A], off_w[T::LOADS_W], off_side;
  auto row_of = [&](int q) { return (wave + T::WAVES * q) * 8 + (lane >> 3); };
  const int chunk = (lane & 7) ^ T::swz(row_of(0));   // of every load's row: 8 WAVES q leaves the swizzle
  auto aim = [&] {   // the tile's bases, and this lane's row and chunk of each load (rows past the end re-read the last)
    ra = buffer_of(g.a + static_cast<size_t>(lm0) * K);
    rw = buffer_of(g.w + static_cast<size_t>(ln0) * K);
#pragma unroll
    for (int q = 0; q < T::LOADS_A; ++q) off_a[q] = static_cast<uint32_t>(min(row_of(q), M - lm0 - 1)) * static_cast<uint32_t>(K) + 16 * chunk;
#pragma unroll
    for (int q = 0; q < T::LOADS_W; ++q) off_w[q] = static_cast<uint32_t>(min(T::column(row_of(q)), g.N - ln0 - 1)) * static_cast<uint32_t>(K) + 16 * chunk;
    if (wave < T::SCALE_WAVES) {
      rside = buffer_of(g.a_scale + static_cast<size_t>(lm0) * ld);
      off_side = static_cast<uint32_t>(min(64 * wave + lane, M - lm0 - 1)) * static_cast<uint32_t>(ld);
    } else {
      rside = buffer_of(g.w_scale + static_cast<size_t>(ln0 / kScaleBlock) * ld);
      off_side = static_cast<uint32_t>(min(lane % (T::BN / kScaleBlock), (g.N - ln0 - 1) / kScaleBlock) * ld);
    }
    // the columns' bias (zeros without one), ahead of the tile's first stage.  The tile before this one has
    // yet to read its own, and with STAGES blocks no barrier has passed since the one before that did: four slots.
    turn = (turn + 1) & 3;
    const int c = 64 * (wave % (T::BN / 64));
    dma4(ring_at + static_cast<uint32_t>(T::BIAS * 16 + turn * T::BN * 4 + c * 4), static_cast<uint32_t>(ln0 + c + lane) * 4,
         buffer_of(g.bias, g.bias ? 4u * g.N : 0u), 0);
  };
  // The chunks past K of a last, shorter K-block read zeros, and all of those that fill a short sum up to STAGES
  // blocks: called before such a block's loads.  The next tile's aim sets the offsets anew.
  auto last_block = [&] {
    const bool inside = lk * kScaleBlock + 16 * chunk < K;
#pragma unroll
    for (int q = 0; q < T::LOADS_A; ++q) off_a[q] = inside ? off_a[q] : kNowhere;
#pragma unroll
    for (int q = 0; q < T::LOADS_W; ++q) off_w[q] = inside ? off_w[q] : kNowhere;
  };
  // Loads `from` to `to` of the rows (q < LOADS_A) and of the columns (the rest) into a slot, and the scales.
  constexpr int kSlot = T::CHUNKS * 16;
  const uint32_t wave_at = ring_at + wave * 1024;
  auto issue = [&](uint32_t slot_at, auto from, auto to) {
    constexpr int FROM = decltype(from)::value, TO = decltype(to)::value;
    auto go = [&](auto self, auto i) {
      constexpr int q = decltype(i)::value;
      if constexpr (q < TO) {
        // tile rows are 128 bytes, the columns' follow the rows', and WAVES loads of 1024 bytes lie between q and q + 1
        if constexpr (q < T::LOADS_A) dma16<T::WAVES * q * 1024>(wave_at + slot_at, off_a[q], ra, static_cast<uint32_t>(lk * kScaleBlock));
        else dma16<T::WAVES * q * 1024>(wave_at + slot_at, off_w[q - T::LOADS_A], rw, static_cast<uint32_t>(lk * kScaleBlock));
        self(self, std::integral_constant<int, q + 1>{});
      }
    };
    go(go, std::integral_constant<int, FROM>{});
  };
  auto issue_scales = [&](uint32_t slot_at) {
    dma4(ring_at + slot_at + static_cast<uint32_t>(T::SIDE * 16 + min(wave, T::SCALE_WAVES) * 256), off_side, rside, static_cast<uint32_t>(lk & ~3));
  };

  // ---- the products
  const int arow = 32 * FI * wm + l32;
  const int wrow = 32 * NJ * wn + l32;
  // byte offsets in a stage of this lane's two chunks of a half K-block, of its first row and its first column (32 rows on: 4096 bytes)
  uint32_t at_a[2][2], at_w[2][2];
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      at_a[kh][c] = arow * 128 + ((4 * kh + 2 * half + c) ^ T::swz(arow)) * 16;
      at_w[kh][c] = (T::BM + wrow) * 128 + ((4 * kh + 2 * half + c) ^ T::swz(wrow)) * 16;
    }
  const char* lds = reinterpret_cast<const char*>(ring);
  auto read = [&](const char* lo_at, const char* hi_at) {
    const uint4 lo = *reinterpret_cast<const uint4*>(lo_at), hi = *reinterpret_cast<const uint4*>(hi_at);
    return i32x8_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                   static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
  };
  i32x8_t a[2][FI], w[4];
  uint32_t sa[FI], sw, sa_next[FI], sw_next;   // a step's scale bytes, and the next one's words as they come from LDS
  auto read_a = [&](uint32_t slot_at, int kh) {
#pragma unroll
    for (int i = 0; i < FI; ++i) a[kh][i] = read(lds + (slot_at + at_a[kh][0]) + 4096 * i, lds + (slot_at + at_a[kh][1]) + 4096 * i);
  };
  auto read_w = [&](uint32_t slot_at, int s) {
    const int kh = s / NJ, j = s % NJ;
    w[s & 3] = read(lds + (slot_at + at_w[kh][0]) + 4096 * j, lds + (slot_at + at_w[kh][1]) + 4096 * j);
  };
  auto read_scales = [&](uint32_t slot_at) {
    const uint32_t* side = reinterpret_cast<const uint32_t*>(lds + slot_at + T::SIDE * 16);
#pragma unroll
    for (int i = 0; i < FI; ++i) sa_next[i] = side[arow + 32 * i];
    sw_next = side[64 * T::SCALE_WAVES + 32 * NJ * wn / kScaleBlock];
  };

  aim();
#pragma unroll
  for (int p = 0; p < STAGES; ++p) {
    if (lk >= blocks - 1) last_block();
    issue(p * kSlot, std::integral_constant<int, 0>{}, std::integral_constant<int, T::LOADS_A + T::LOADS_W>{});
    issue_scales(p * kSlot);
    ++lk;
  }
  wait_barrier<(STAGES - 1) * T::ISSUED, 0>(0);
  read_a(0, 0);
  read_w(0, 0);
  read_w(0, 1);
  read_scales(0);

  uint32_t slot = 0;   // byte offset of the step's stage
  int stored = 0;   // in a tile's first step: the previous tile's stores were issued after the last stage's loads
  for (;;) {
    const int m0 = lm0, n0 = ln0;
    f32x16_t acc[FI][NJ] = {};
    bool more = false;
    int kb = 0;
    // the steps that load this tile, then the last STAGES, which load the next one (or this one's end again)
    for (int part = 0; part < 2; ++part) {
      if (part == 1) {
        more = tile_at(u + gridDim.x, lm0, ln0);
        lk = more ? 0 : nk - STAGES;
        if (more) aim();
      }
      for (const int end = part == 0 ? nk - STAGES : nk; kb < end; ++kb, ++lk) {
        if (lk >= blocks - 1) last_block();
        const uint32_t next = slot == (STAGES - 1) * kSlot ? 0 : slot + kSlot;
        const int shift = 8 * (min(kb, blocks - 1) & 3);   // blocks of zeros take the last one's scales
#pragma unroll
        for (int i = 0; i < FI; ++i) sa[i] = sa_next[i] >> shift;
        sw = sw_next >> shift;
#pragma unroll
        for (int s = 0; s < kSubs; ++s) {
          // waves of two fragments have read all of the stage by the barrier after sub-step 1
          if (NJ == 4 && s == 2) wait_reads_barrier();
          if (s == kSubs - 2) wait_barrier<(STAGES - 2) * T::ISSUED + (NJ == 4 ? T::LOADS_A : 0), kStores>(stored);
          if (s == 0) read_a(slot, 1);
          if (s < kSubs - 2) read_w(slot, s + 2);
          if (s == kSubs - 2) {
            read_a(next, 0);
            read_w(next, 0);
            read_scales(next);
          }
          if (s == kSubs - 1) read_w(next, 1);
          const typename Mma::frag wf = Mma::make(w[s & 3], sw);
#pragma unroll
          for (int i = 0; i < FI; ++i) acc[i][s % NJ] = Mma::mma(Mma::make(a[s / NJ][i], sa[i]), wf, acc[i][s % NJ], sa[i], sw);
          __builtin_amdgcn_sched_barrier(0);
          if (s == 2) issue(slot, std::integral_constant<int, 0>{}, std::integral_constant<int, T::LOADS_A / 2>{});
          if (s == (NJ == 4 ? 4 : 2)) issue(slot, std::integral_constant<int, T::LOADS_A / 2>{}, std::integral_constant<int, T::LOADS_A>{});
          if (s == kSubs - 2) issue(slot, std::integral_constant<int, T::LOADS_A>{}, std::integral_constant<int, T::LOADS_A + T::LOADS_W / 2>{});
          if (s == kSubs - 1) {
            issue(slot, std::integral_constant<int, T::LOADS_A + T::LOADS_W / 2>{}, std::integral_constant<int, T::LOADS_A + T::LOADS_W>{});
            issue_scales(slot);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        slot = next;
        stored = 0;
      }
    }

    stored = 1;
    const int col = 32 * NJ * wn + NJ * l32;   // this lane's first column of the tile
    const bool col_ok = n0 + col < g.N;
    const float* columns = reinterpret_cast<const float*>(ring + T::BIAS + (turn - (more ? 1 : 0) & 3) * (T::BN / 4)) + col;
    float bias[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) bias[j] = columns[j];
    void* base;
    if constexpr (KIND == kToCodes) base = g.y_q;
    else if constexpr (KIND == kToBf16) base = g.y_bf16;
    else base = g.y_f32;
    const int row0 = 32 * FI * wm, lds_y = fd::scale_stride(g.N);
    const auto y = __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t*>(base) + (static_cast<size_t>(m0 + row0) * g.N + n0) * kSize, 0, 0x7fffffff, 0x00020000);
    const auto ys = __builtin_amdgcn_make_buffer_rsrc(g.y_scale + static_cast<size_t>(m0 + row0) * lds_y + (n0 + 32 * NJ * wn) / kScaleBlock, 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const bool block_ok = n0 + 32 * NJ * wn < g.N;   // else no column of this wave
      Rows32<KIND, NJ>::store(acc[i], bias, g.gelu, y, col_ok, l32, half, block_ok ? M - m0 - row0 - 32 * i : 0,
                          static_cast<uint32_t>((32 * i + 4 * half) * g.N + col) * kSize, static_cast<uint32_t>(g.N) * kSize, ys,
                          static_cast<uint32_t>(32 * i * lds_y), static_cast<uint32_t>(lds_y));
      __builtin_amdgcn_sched_barrier(0);   // 32 rows at a time: fewer registers
    }
    if (!more) break;
    u += gridDim.x;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the repeats of the last stage
}

// A K-step of 128 x 128 loads 32 KB into LDS at 64 bytes a clock of its CU (measured 63), 512 clocks, as long as its matrix
// instructions take; it reads 80 KB from LDS at 256 (measured 225 with 16 waves), 320.  Of 256 x 256: 64 KB, 1024 beside
// 2048, and 192 KB, 768.  No pipe is full.  9828 x 6144 x 1536 to codes with GELU in 128 x 128 tiles 104 us (1780 TFLOP/s):
// matrix instructions 42% of the clocks, vector ones (GELU, maxima, codes) 40%, loads 42%, LDS reads 28% without
// conflicts.  9828 x 1536 x 6144 to bf16 in 256 x 256 72 us (2560 TFLOP/s; a large fp8 product of the library 2720), 32760 x
// 1536 x 6144 to fp32 457 us (1350, at half the rate): matrix 70%, vector (the codes to bf16) 39%, loads 17%, reads 14%.
using Tile64 = Tile<1, 2, 2, 2, 3>;        // 64 x 128, two workgroups per CU, in 32 x 64 a wave: all four SIMDs of a CU that has one
using Tile64Codes = Tile<1, 4, 2, 1, 3>;   // 64 x 128 where a wave has to hold a block's 128 columns
using Tile128 = Tile<1, 4, 4, 1, 2>;       // 128 x 128, two
using TileLarge = Tile<2, 4, 4, 2, 2>;     // 256 x 256, one

// Where both kernels are launched (cus > 0), the one that the row count does not call for ends at once.
template <int KIND, class Mma, class T, int PER_CU>
__global__ __launch_bounds__(T::THREADS, (PER_CU * T::WAVES + 3) / 4) void scaled_tile_kernel(fdh::ScaledArgs g, int cus) {
  __shared__ uint4 ring[T::TOTAL];
  static_assert(T::TOTAL * 16 * PER_CU <= 160 * 1024, "the LDS of a CU");
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  if (M <= 0 || (cus > 0 && fd::scaled_large(M, g.N, g.K, KIND == kToCodes, cus) != (T::BM == TileLarge::BM))) return;
  scaled_tiles<T, KIND, Mma>(g, M, ring);
}

}  // namespace

namespace fdh {

hipError_t launch_scaled_linear(const ScaledArgs& g, hipStream_t s) {
  auto run = [&](auto kind, auto mma) {
    constexpr int KIND = decltype(kind)::value;
    using Mma = decltype(mma);
    constexpr bool codes = KIND == kToCodes;
    if constexpr (!codes) {
      if (fd::scaled_few(g.n_rows, g.N, g.K, codes, KIND == kToF32, num_cus())) {
        auto few = [&](auto fm, auto nf, auto deep) {
          constexpr int FM = decltype(fm)::value, NF = decltype(nf)::value;
          scaled_few_kernel<KIND, Mma, FM, NF, decltype(deep)::value><<<dim3((g.N + 16 * NF - 1) / (16 * NF), (g.n_rows + 16 * FM - 1) / (16 * FM)), kFewWaves * 64, 0, s>>>(g);
        };
        const std::integral_constant<int, 1> one{};
        const std::integral_constant<int, 2> two{};
        const std::integral_constant<int, 3> three{};
        const std::integral_constant<int, 4> four{};
        const int frags = fd::scaled_few_frags(g.n_rows);
        if (fd::scaled_few_wide(g.N, num_cus())) {
          if (frags == 1) few(one, two, two);
          else if (frags == 2) few(two, two, two);
          else few(four, two, one);
        } else {
          if (frags == 1) few(one, one, three);
          else if (frags == 2) few(two, one, two);
          else few(four, one, one);
        }
        return;
      }
    }
    const int cus = num_cus() / 8 * 8;   // the tile order counts on whole rounds of the 8 XCDs
    const bool both = g.m && fd::scaled_both(g.n_rows, g.N, g.K, codes, cus), large = !g.m && fd::scaled_large(g.n_rows, g.N, g.K, codes, cus);
    auto tiles = [&](auto tile, auto per_cu, int check) {
      using T = decltype(tile);
      constexpr int PER_CU = decltype(per_cu)::value;
      const long long all = static_cast<long long>((g.n_rows + T::BM - 1) / T::BM) * ((g.N + T::BN - 1) / T::BN), most = PER_CU * cus;
      scaled_tile_kernel<KIND, Mma, T, PER_CU><<<static_cast<int>(all < most ? (all + 7) / 8 * 8 : most), T::THREADS, 0, s>>>(g, check);
    };
    using std::integral_constant;
    using Small = std::conditional_t<codes, Tile64Codes, Tile64>;
    if (fd::scaled_small(g.n_rows, g.N, cus)) return tiles(Small{}, integral_constant<int, 2>{}, 0);
    if (both || !large) tiles(Tile128{}, integral_constant<int, 2>{}, both ? cus : 0);
    if (both || large) tiles(TileLarge{}, integral_constant<int, 1>{}, both ? cus : 0);
  };
  if (g.y_q) run(std::integral_constant<int, kToCodes>{}, Mma8{});
  else if (g.y_bf16) run(std::integral_constant<int, kToBf16>{}, Mma8{});
  else run(std::integral_constant<int, kToF32>{}, MmaExact{});
  return hipGetLastError();
}

}  // namespace fdh
