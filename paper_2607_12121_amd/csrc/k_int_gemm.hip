// The product of 8-bit integers with a scale per row and per column:
//   Y[M][N] = act(float(sum_k A[i][k] W[j][k]) * w_scale[j] * a_scale[i] + bias[j])
// on v_mfma_i32_16x16x64_i8 and 32x32x32: the sums are whole numbers of at most 2^30 (K <= 2^16) and exact.  A sum meets the
// scales one after the other: 0 or at least 1, it stays a normal number times scales from 2^-107 to 2^98.  The scales' product
// need not be one: below 2^-126 it loses bits, past 2^128 it makes NaN of a sum of zero.
#include <type_traits>

#include "fd_int.h"
#include "fd_int_rules.h"
#include "fd_tile_loads.h"

namespace {

typedef int i32x16_t __attribute__((ext_vector_type(16)));
constexpr int kBlock = 128;   // bytes of K in a step

FD_DEVICE i32x4_t half_of(const i32x8_t& x, int c) { return c ? i32x4_t{x[4], x[5], x[6], x[7]} : i32x4_t{x[0], x[1], x[2], x[3]}; }
// The lanes' 32 bytes of both operands are the same ones of K, which is all that a sum asks of their order.
FD_DEVICE i32x4_t mma(const i32x8_t& w, const i32x8_t& a, i32x4_t c) {
  c = __builtin_amdgcn_mfma_i32_16x16x64_i8(half_of(w, 0), half_of(a, 0), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(half_of(w, 1), half_of(a, 1), c, 0, 0, 0);
}
FD_DEVICE i32x16_t mma(const i32x8_t& a, const i32x8_t& w, i32x16_t c) {
  c = __builtin_amdgcn_mfma_i32_32x32x32_i8(half_of(a, 0), half_of(w, 0), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(half_of(a, 1), half_of(w, 1), c, 0, 0, 0);
}

// ---------------------------------------------------------------- few rows

// As the few-row kernel of the block-scaled product: what counts is how many of the weights' bytes are on the way.  A
// workgroup takes the rows' FM fragments and 16 NF columns, its waves the K-blocks in turn, operands straight from memory
// into registers, DEEP blocks at a time; the waves' sums meet in LDS.  The first operand is the weights, so that a lane
// holds a row (l & 15) and, of its NF fragments, 4 NF consecutive columns.  1 x 4608 x 1536 4.4 us alone (7.1 MB: launch and two
// round trips to memory), 64 x 4608 x 1088 4.7, 1 x 65536 x 4096 52 (5.2 TB/s).
constexpr int kFewWaves = 8;

template <bool WIDE, int FM, int NF, int DEEP>
__global__ __launch_bounds__(kFewWaves * 64) void int_few_kernel(fdh::IntLinearArgs g) {
  __shared__ i32x4_t part[kFewWaves][FM][NF][64];
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lg = lane >> 4;
  const int K = g.K, nk = (K + kBlock - 1) / kBlock;
  const int n0 = blockIdx.x * 16 * NF, m0 = blockIdx.y * 16 * FM;
  if (m0 >= M) return;
  const uint8_t* w[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j)
    w[j] = reinterpret_cast<const uint8_t*>(g.w) + static_cast<size_t>(min(n0 + 4 * NF * (l16 >> 2) + 4 * j + (l16 & 3), g.N - 1)) * K;
  i32x4_t acc[FM][NF] = {};
  for (int kb = wave; kb < nk; kb += kFewWaves * DEEP) {
    Piece wf[DEEP][NF], af[DEEP][FM];
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      const int b = kb + d * kFewWaves, k = b * kBlock + 32 * lg;
      if (b >= nk) break;
#pragma unroll
      for (int j = 0; j < NF; ++j) wf[d][j] = load32(w[j], k, K);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const size_t row = min(m0 + 16 * i + l16, M - 1);
        af[d][i] = load32(reinterpret_cast<const uint8_t*>(g.a) + row * K, k, K);
      }
    }
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      const int b = kb + d * kFewWaves, k = b * kBlock + 32 * lg;
      if (b >= nk) break;
      i32x8_t wd[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) wd[j] = inside(wf[d][j], k, K);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const i32x8_t ad = inside(af[d][i], k, K);
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = mma(wd[j], ad, acc[i][j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) part[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  if (wave >= FM) return;
  // a wave per 16 rows adds the waves' sums
  const int row = m0 + 16 * wave + l16, col = n0 + 4 * NF * lg;
  const float sa = g.a_scale[min(row, M - 1)];
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    i32x4_t sum = part[0][wave][j][lane];
#pragma unroll
    for (int p = 1; p < kFewWaves; ++p) sum += part[p][wave][j][lane];
    const int c = min(col + 4 * j, g.N - 4);
    const float4 sw = *reinterpret_cast<const float4*>(g.w_scale + c), bias = g.bias ? *reinterpret_cast<const float4*>(g.bias + c) : make_float4(0, 0, 0, 0);
    float v[4] = {static_cast<float>(sum[0]) * sw.x * sa + bias.x, static_cast<float>(sum[1]) * sw.y * sa + bias.y,
                  static_cast<float>(sum[2]) * sw.z * sa + bias.z, static_cast<float>(sum[3]) * sw.w * sa + bias.w};
    if (g.gelu) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fd::gelu(v[e]);
    }
    if (row >= M || col + 4 * j >= g.N) continue;
    const size_t at = static_cast<size_t>(row) * g.N + col + 4 * j;
    if constexpr (WIDE) *reinterpret_cast<float4*>(g.y_f32 + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(g.y_bf16 + at) = make_uint2(fd::pack_bf2(v[0], v[1]), fd::pack_bf2(v[2], v[3]));
  }
}

// ---------------------------------------------------------------- tiles of their own K-blocks

// Few tiles: every wave of a workgroup has K-blocks of its own, every fourth, and the whole tile's sums of them (32 FI x 32 NJ);
// the waves' sums, whole numbers, meet in LDS.  Operands come to the wave's own LDS, STAGES blocks ahead, by loads of whole
// 128-byte rows, and each byte is read from there once: no barrier in the loop.  What bounds it is the loads to LDS (64 bytes a
// clock and CU; 64 x 1536 x 6144 7.7 us, of which 4 are the start and the end).  The few-row kernel's loads take 16 bytes of 16 rows
// side by side, which the L1 serves at a quarter of its rate (there 16.2 us); the tiles below, most CUs without one, 17.4.
// Larger tiles, one stage: 512 x 1536 x 6144 in 64 x 128 20.8, in 128 x 128 31.6, where 64 x 64 take 13.3.
template <int FI_, int NJ_, int STAGES_>
struct IntSplit {
  static constexpr int FI = FI_, NJ = NJ_, STAGES = STAGES_, WAVES = 4, THREADS = 64 * WAVES;
  static constexpr int BM = 32 * FI, BN = 32 * NJ, LOADS_A = BM / 8, LOADS_W = BN / 8, ISSUED = LOADS_A + LOADS_W;   // 8 rows a wave-load
  static constexpr int SLOT = (BM + BN) * kBlock;                   // bytes
  static constexpr int SIDE = WAVES * STAGES * SLOT;                // column scales, bias and row scales, 64 each
  static constexpr int TOTAL = (SIDE + 3 * 256) / 16;
  static_assert(BM <= 64 && BN <= 64 && (STAGES - 1) * ISSUED < 64, "one load of scales, the counter's range");
  static_assert(WAVES * FI * NJ * 4096 <= SIDE, "the waves' sums");
  static FD_DEVICE int column(int p) { return NJ * (p & 31) + (p >> 5); }   // of LDS row p, so that a lane has NJ consecutive columns
};

template <bool WIDE, class T>
__global__ __launch_bounds__(T::THREADS) void int_split_kernel(fdh::IntLinearArgs g) {
  constexpr int FI = T::FI, NJ = T::NJ, STAGES = T::STAGES, WAVES = T::WAVES;
  __shared__ uint4 ring[T::TOTAL];
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows, K = g.K, blocks = (K + kBlock - 1) / kBlock;
  const int m0 = blockIdx.y * T::BM, n0 = blockIdx.x * T::BN;
  if (m0 >= M) return;
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5, l8 = lane >> 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ring_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)ring)), wave_at = ring_at + wave * STAGES * T::SLOT;
  const char* lds = reinterpret_cast<const char*>(ring);
  const i32x4_t ra = buffer_of(g.a + static_cast<size_t>(m0) * K), rw = buffer_of(g.w + static_cast<size_t>(n0) * K);
  if (wave == 0) {   // ahead of this wave's first stage; of zeros where there is no bias
    dma4(ring_at + T::SIDE, static_cast<uint32_t>(n0 + lane) * 4, buffer_of(g.w_scale, 4u * g.N), 0);
    dma4(ring_at + T::SIDE + 256, static_cast<uint32_t>(n0 + lane) * 4, buffer_of(g.bias, g.bias ? 4u * g.N : 0u), 0);
    dma4(ring_at + T::SIDE + 512, static_cast<uint32_t>(lane) * 4, buffer_of(g.a_scale + m0, 4u * min(T::BM, M - m0)), 0);
  }
  // chunk c of LDS row r lies at c ^ swz(r) = c ^ ((r >> 1) & 7); this lane's chunk of the rows 8 q + l8, even q and odd
  const int chunk = (lane & 7) ^ (l8 >> 1);
  uint32_t off[T::ISSUED];
#pragma unroll
  for (int q = 0; q < T::LOADS_A; ++q) off[q] = static_cast<uint32_t>(min(8 * q + l8, M - m0 - 1)) * static_cast<uint32_t>(K) + 16 * (chunk ^ (4 * (q & 1)));
#pragma unroll
  for (int q = 0; q < T::LOADS_W; ++q)
    off[T::LOADS_A + q] = static_cast<uint32_t>(min(T::column(8 * q + l8), g.N - n0 - 1)) * static_cast<uint32_t>(K) + 16 * (chunk ^ (4 * (q & 1)));
  auto issue = [&](uint32_t slot_at, int b) {   // K-block b; chunks past K read zeros
    const bool in[2] = {b * kBlock + 16 * chunk < K, b * kBlock + 16 * (chunk ^ 4) < K};
    auto go = [&](auto self, auto i) {
      constexpr int q = decltype(i)::value;
      if constexpr (q < T::ISSUED) {
        const uint32_t from = in[(q < T::LOADS_A ? q : q - T::LOADS_A) & 1] ? off[q] : kNowhere;
        dma16<q * 1024>(wave_at + slot_at, from, q < T::LOADS_A ? ra : rw, static_cast<uint32_t>(b) * kBlock);
        self(self, std::integral_constant<int, q + 1>{});
      }
    };
    go(go, std::integral_constant<int, 0>{});
  };
#pragma unroll
  for (int p = 0; p < STAGES; ++p) issue(p * T::SLOT, wave + p * WAVES);

  uint32_t at[2][2];   // byte offsets in a slot of this lane's chunks of a half K-block; rows 32 on: 4096 bytes
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int c = 0; c < 2; ++c) at[kh][c] = wave * STAGES * T::SLOT + l32 * kBlock + ((4 * kh + 2 * half + c) ^ ((l32 >> 1) & 7)) * 16;
  auto read = [&](const char* lo_at, const char* hi_at) {
    const uint4 lo = *reinterpret_cast<const uint4*>(lo_at), hi = *reinterpret_cast<const uint4*>(hi_at);
    return i32x8_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                   static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
  };
  i32x16_t acc[FI][NJ] = {};
  uint32_t slot = 0;
  for (int b = wave; b < blocks; b += WAVES) {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"((STAGES - 1) * T::ISSUED) : "memory");
    i32x8_t f[2][FI + NJ];
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int i = 0; i < FI + NJ; ++i) f[kh][i] = read(lds + (slot + at[kh][0]) + 4096 * i, lds + (slot + at[kh][1]) + 4096 * i);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // the slot is read
    issue(slot, b + STAGES * WAVES);
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = mma(f[kh][i], f[kh][FI + j], acc[i][j]);
    slot = slot == (STAGES - 1) * T::SLOT ? 0 : slot + T::SLOT;
  }
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // loads past the end write zeros
  __syncthreads();
  i32x4_t* part = reinterpret_cast<i32x4_t*>(ring);   // [wave][rows 8 r4 + 4 half + 0 .. 3 of fragment i][j][lane], as acc holds them
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        part[((wave * FI * 4 + 4 * i + r4) * NJ + j) * 64 + lane] = i32x4_t{acc[i][j][4 * r4], acc[i][j][4 * r4 + 1], acc[i][j][4 * r4 + 2], acc[i][j][4 * r4 + 3]};
  __syncthreads();
  const float* side = reinterpret_cast<const float*>(lds + T::SIDE);
  const int col = n0 + NJ * l32;
  float sw[NJ], bias[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    sw[j] = side[NJ * l32 + j];
    bias[j] = side[64 + NJ * l32 + j];
  }
#pragma unroll
  for (int i = 0; i < FI; ++i) {   // wave r4 adds up and stores the rows of r4
    const int at4 = 4 * i + wave, row0 = 8 * at4 + 4 * half;
    i32x4_t sum[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      sum[j] = part[(at4 * NJ + j) * 64 + lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum[j] += part[((w * FI * 4 + at4) * NJ + j) * 64 + lane];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float sa = side[128 + row0 + e];
      float v[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        v[j] = static_cast<float>(sum[j][e]) * sw[j] * sa + bias[j];
        if (g.gelu) v[j] = fd::gelu(v[j]);
      }
      if (m0 + row0 + e >= M || col >= g.N) continue;
      const size_t to = static_cast<size_t>(m0 + row0 + e) * g.N + col;
      if constexpr (WIDE && NJ == 2) *reinterpret_cast<float2*>(g.y_f32 + to) = make_float2(v[0], v[1]);
      else if constexpr (WIDE) g.y_f32[to] = v[0];
      else if constexpr (NJ == 2) *reinterpret_cast<uint32_t*>(g.y_bf16 + to) = fd::pack_bf2(v[0], v[1]);
      else g.y_bf16[to] = static_cast<uint16_t>(fd::pack_bf2(v[0], v[0]));
    }
  }
}

// ---------------------------------------------------------------- tiles

// A workgroup of WM x WN waves with a tile of 32 FI WM rows x 32 NJ WN columns, K-steps of one block; a wave owns FI x NJ
// blocks of 32 x 32.  In LDS a tile row is eight 16-byte chunks, chunk c of row r at c ^ swz(r), so that the 16 lanes
// that read a fragment together meet 16 different 16-byte bank groups.  A tile's scales and bias come with its first stage.
template <int FI_, int NJ_, int WM_, int WN_, int STAGES_>
struct IntTile {
  static constexpr int FI = FI_, NJ = NJ_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int BM = 32 * FI * WM, BN = 32 * NJ * WN;
  static constexpr int LOADS_A = BM / 8 / WAVES, LOADS_W = BN / 8 / WAVES;        // 8 rows of 128 bytes per wave-load
  static constexpr int ISSUED = LOADS_A + LOADS_W;
  static constexpr int CHUNKS = (BM + BN) * 8;                                    // of a stage
  static constexpr int SIDE = STAGES * CHUNKS;                                    // four slots of column scales, bias and row scales
  static constexpr int SIDE_FLOATS = 2 * BN + BM;
  static constexpr int TOTAL = SIDE + 4 * SIDE_FLOATS / 4;
  static_assert(NJ == 4 || NJ == 2, "a step's parts");
  static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && BN % 64 == 0 && BM % 64 == 0 && BN <= 64 * WAVES && BM <= 64 * WAVES, "whole wave-loads");
  static FD_DEVICE int swz(int r) { return (r >> 1) & 7; }
  // Column of LDS row p: fragment j of a wave's columns holds every NJ-th, from j on, so that a lane has NJ consecutive
  // columns in its NJ fragments.
  static FD_DEVICE int column(int p) { return (p & ~(32 * NJ - 1)) + NJ * (p & 31) + ((p >> 5) & (NJ - 1)); }
};

// The K-steps of all of a workgroup's tiles are one sequence: the loads run STAGES steps ahead of the products, into the
// next tile too, and a tile's results leave while the next one's first stages land.  A step's 2 NJ sub-steps (half of K,
// column fragment) read their weight fragment two sub-steps ahead; after the barrier behind sub-step 1 the stage's rows
// may be loaded over, after the one before the last two its columns, and the next stage is there (waves of two
// fragments: the one barrier frees all of it).  A step is one basic block, its loads go out behind products.
//
// TOP/s: 32760 x 1536 x 6144 2230 to 2310 (the library's product alone 2230), 9828 x 1536 x 6144 2190, x 4608 x 1536 1750, x 6144 x
// 1536 with GELU to bf16 1750 (matrix pipes 43% busy, vector instructions 34%, little of it at once: the results have no product
// beside them, one workgroup a CU; in 128 x 128 tiles 120 us for 123).  Where a 128 x 128 workgroup is alone on its CU it has eight
// waves: more reads of LDS (96 KB a K-block for 80, beside 32 written), which bound it at 0.43 us a K-block, but two waves a SIMD:
// 1664 x 1536 x 6144 28.1 -> 25.3 us, 700 x 3200 x 3200 16.8 -> 15.9; four waves of 64 x 64 and three or four stages 27.5 and 27.9.
// 1021 x 4288 x 1088 14: 16 of 256 CUs have two tiles.
template <class T, bool WIDE>
FD_DEVICE void int_tiles(const fdh::IntLinearArgs& g, int M, uint4* ring) {
  constexpr int FI = T::FI, NJ = T::NJ, STAGES = T::STAGES, kSubs = 2 * NJ, kSize = WIDE ? 4 : 2;
  constexpr int kStores = FI * 16;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WN, wn = wave % T::WN;
  const int K = g.K, blocks = (K + kBlock - 1) / kBlock, nk = max(blocks, STAGES);
  const int tiles_m = (M + T::BM - 1) / T::BM, tiles_n = (g.N + T::BN - 1) / T::BN, tiles = tiles_m * tiles_n;
  const int per_xcd = (tiles + 7) / 8;
  const uint32_t ring_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)ring));

  // Tile of turn u of this workgroup: consecutive tiles on one XCD, in groups of 8 row tiles x every column tile, row tile
  // fastest, so that the tiles an XCD runs at once share operand rows in its L2.
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
  i32x4_t ra, rw;
  int turn = 3;
  uint32_t off_a[T::LOADS_A], off_w[T::LOADS_W];
  auto row_of = [&](int q) { return (wave + T::WAVES * q) * 8 + (lane >> 3); };
  const int chunk = (lane & 7) ^ T::swz(row_of(0));   // of every load's row: 8 WAVES q leaves the swizzle
  auto side_at = [&](int slot) { return static_cast<uint32_t>(T::SIDE * 16 + slot * T::SIDE_FLOATS * 4); };
  auto aim = [&] {   // the tile's bases, and this lane's row and chunk of each load (rows past the end re-read the last)
    ra = buffer_of(g.a + static_cast<size_t>(lm0) * K);
    rw = buffer_of(g.w + static_cast<size_t>(ln0) * K);
#pragma unroll
    for (int q = 0; q < T::LOADS_A; ++q) off_a[q] = static_cast<uint32_t>(min(row_of(q), M - lm0 - 1)) * static_cast<uint32_t>(K) + 16 * chunk;
#pragma unroll
    for (int q = 0; q < T::LOADS_W; ++q) off_w[q] = static_cast<uint32_t>(min(T::column(row_of(q)), g.N - ln0 - 1)) * static_cast<uint32_t>(K) + 16 * chunk;
    // the columns' scales and bias (zeros without one) and the rows' scales, ahead of the tile's first stage.  The tile before this
    // one has yet to read its own, and with STAGES blocks no barrier has passed since the one before that did: four slots.
    turn = (turn + 1) & 3;
    const int c = 64 * (wave % (T::BN / 64)), r = 64 * (wave % (T::BM / 64));
    const uint32_t to = ring_at + side_at(turn);
    dma4(to + static_cast<uint32_t>(c * 4), static_cast<uint32_t>(ln0 + c + lane) * 4, buffer_of(g.w_scale, 4u * g.N), 0);
    dma4(to + static_cast<uint32_t>((T::BN + c) * 4), static_cast<uint32_t>(ln0 + c + lane) * 4, buffer_of(g.bias, g.bias ? 4u * g.N : 0u), 0);
    dma4(to + static_cast<uint32_t>((2 * T::BN + r) * 4), static_cast<uint32_t>(r + lane) * 4, buffer_of(g.a_scale + lm0, 4u * min(T::BM, M - lm0)), 0);
  };
  // The chunks past K of a last, shorter K-block read zeros, and all of those that fill a short sum up to STAGES
  // blocks: called before such a block's loads.  The next tile's aim sets the offsets anew.
  auto last_block = [&] {
    const bool in = lk * kBlock + 16 * chunk < K;
#pragma unroll
    for (int q = 0; q < T::LOADS_A; ++q) off_a[q] = in ? off_a[q] : kNowhere;
#pragma unroll
    for (int q = 0; q < T::LOADS_W; ++q) off_w[q] = in ? off_w[q] : kNowhere;
  };
  // Loads `from` to `to` of the rows (q < LOADS_A) and of the columns (the rest) into a slot.
  constexpr int kSlot = T::CHUNKS * 16;
  const uint32_t wave_at = ring_at + wave * 1024;
  auto issue = [&](uint32_t slot_at, auto from, auto to) {
    constexpr int FROM = decltype(from)::value, TO = decltype(to)::value;
    auto go = [&](auto self, auto i) {
      constexpr int q = decltype(i)::value;
      if constexpr (q < TO) {
        // tile rows are 128 bytes, the columns' follow the rows', and WAVES loads of 1024 bytes lie between q and q + 1
        if constexpr (q < T::LOADS_A) dma16<T::WAVES * q * 1024>(wave_at + slot_at, off_a[q], ra, static_cast<uint32_t>(lk * kBlock));
        else dma16<T::WAVES * q * 1024>(wave_at + slot_at, off_w[q - T::LOADS_A], rw, static_cast<uint32_t>(lk * kBlock));
        self(self, std::integral_constant<int, q + 1>{});
      }
    };
    go(go, std::integral_constant<int, FROM>{});
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
  auto read_a = [&](uint32_t slot_at, int kh) {
#pragma unroll
    for (int i = 0; i < FI; ++i) a[kh][i] = read(lds + (slot_at + at_a[kh][0]) + 4096 * i, lds + (slot_at + at_a[kh][1]) + 4096 * i);
  };
  auto read_w = [&](uint32_t slot_at, int s) {
    const int kh = s / NJ, j = s % NJ;
    w[s & 3] = read(lds + (slot_at + at_w[kh][0]) + 4096 * j, lds + (slot_at + at_w[kh][1]) + 4096 * j);
  };

  aim();
#pragma unroll
  for (int p = 0; p < STAGES; ++p) {
    if (lk >= blocks - 1) last_block();
    issue(p * kSlot, std::integral_constant<int, 0>{}, std::integral_constant<int, T::LOADS_A + T::LOADS_W>{});
    ++lk;
  }
  wait_barrier<(STAGES - 1) * T::ISSUED, 0>(0);
  read_a(0, 0);
  read_w(0, 0);
  read_w(0, 1);

  uint32_t slot = 0;   // byte offset of the step's stage
  int stored = 0;   // in a tile's first step: the previous tile's stores were issued after the last stage's loads
  for (;;) {
    const int m0 = lm0, n0 = ln0;
    i32x16_t acc[FI][NJ] = {};
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
#pragma unroll
        for (int s = 0; s < kSubs; ++s) {
          if (NJ == 4 && s == 2) wait_reads_barrier();
          if (s == kSubs - 2) wait_barrier<(STAGES - 2) * T::ISSUED + (NJ == 4 ? T::LOADS_A : 0), kStores>(stored);
          if (s == 0) read_a(slot, 1);
          if (s < kSubs - 2) read_w(slot, s + 2);
          if (s == kSubs - 2) {
            read_a(next, 0);
            read_w(next, 0);
          }
          if (s == kSubs - 1) read_w(next, 1);
#pragma unroll
          for (int i = 0; i < FI; ++i) acc[i][s % NJ] = mma(a[s / NJ][i], w[s & 3], acc[i][s % NJ]);
          __builtin_amdgcn_sched_barrier(0);
          if (s == 2) issue(slot, std::integral_constant<int, 0>{}, std::integral_constant<int, T::LOADS_A / 2>{});
          if (s == (NJ == 4 ? 4 : 2)) issue(slot, std::integral_constant<int, T::LOADS_A / 2>{}, std::integral_constant<int, T::LOADS_A>{});
          if (s == kSubs - 2) issue(slot, std::integral_constant<int, T::LOADS_A>{}, std::integral_constant<int, T::LOADS_A + T::LOADS_W / 2>{});
          if (s == kSubs - 1) issue(slot, std::integral_constant<int, T::LOADS_A + T::LOADS_W / 2>{}, std::integral_constant<int, T::LOADS_A + T::LOADS_W>{});
          __builtin_amdgcn_sched_barrier(0);
        }
        slot = next;
        stored = 0;
      }
    }

    stored = 1;
    const int col = 32 * NJ * wn + NJ * l32;   // this lane's first column of the tile
    const bool col_ok = n0 + col < g.N;
    const float* side = reinterpret_cast<const float*>(lds + side_at(turn - (more ? 1 : 0) & 3));
    float sw[NJ], bias[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      sw[j] = side[col + j];
      bias[j] = side[T::BN + col + j];
    }
    const int row0 = 32 * FI * wm;
    uint8_t* base = WIDE ? reinterpret_cast<uint8_t*>(g.y_f32) : reinterpret_cast<uint8_t*>(g.y_bf16);
    const auto y = __builtin_amdgcn_make_buffer_rsrc(base + (static_cast<size_t>(m0 + row0) * g.N + n0) * kSize, 0, 0x7fffffff, 0x00020000);
    const bool block_ok = n0 + 32 * NJ * wn < g.N;   // else no column of this wave
    const uint32_t pitch = static_cast<uint32_t>(g.N) * kSize;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      // acc[i][j][r] is row 8 (r >> 2) + 4 half + (r & 3) of 32: 32 lanes store a row's columns side by side.  Every store
      // issues, rows and columns outside go nowhere: the waits count the stores.
      const int rows = block_ok ? M - m0 - row0 - 32 * i - 4 * half : 0;
      const uint32_t off = (static_cast<uint32_t>(32 * i + 4 * half) * g.N + col) * kSize;
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const float4 sa4 = *reinterpret_cast<const float4*>(side + 2 * T::BN + row0 + 32 * i + 8 * r4 + 4 * half);
        const float sa[4] = {sa4.x, sa4.y, sa4.z, sa4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 8 * r4 + e;
          float v[NJ];
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            v[j] = static_cast<float>(acc[i][j][4 * r4 + e]) * sw[j] * sa[e] + bias[j];
            if (g.gelu) v[j] = fd::gelu(v[j]);
          }
          const uint32_t to = col_ok && row < rows ? off : kNowhere;
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          if constexpr (!WIDE && NJ == 2)
            __builtin_amdgcn_raw_buffer_store_b32(fd::pack_bf2(v[0], v[1]), y, to, row * pitch, kStream);
          else if constexpr (NJ == 2)
            __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v[0]), __float_as_uint(v[1])}, y, to, row * pitch, kStream);
          else if constexpr (!WIDE)
            __builtin_amdgcn_raw_buffer_store_b64(u32x2{fd::pack_bf2(v[0], v[1]), fd::pack_bf2(v[2], v[3])}, y, to, row * pitch, kStream);
          else
            store_f4(v[0], v[1], v[2], v[3], y, to, row * pitch);
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // 32 rows at a time: fewer registers
    }
    if (!more) break;
    u += gridDim.x;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the repeats of the last stage
}

using Tile64 = IntTile<1, 2, 2, 2, 3>;      // 64 x 128, two workgroups per CU
using Tile128 = IntTile<1, 4, 4, 1, 2>;     // 128 x 128, two
using TileAlone = IntTile<1, 2, 4, 2, 4>;   // 128 x 128, one, of eight waves
using TileLarge = IntTile<2, 4, 4, 2, 2>;   // 256 x 256, one

// Where both kernels are launched (cus > 0), the one that the row count does not call for ends at once.
template <bool WIDE, class T, int PER_CU>
__global__ __launch_bounds__(T::THREADS, (PER_CU * T::WAVES + 3) / 4) void int_tile_kernel(fdh::IntLinearArgs g, int cus) {
  __shared__ uint4 ring[T::TOTAL];
  static_assert(T::TOTAL * 16 * PER_CU <= 160 * 1024, "the LDS of a CU");
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  if (M <= 0 || (cus > 0 && fd::int_large(M, g.N, g.K, WIDE, cus) != (T::BM == TileLarge::BM))) return;
  int_tiles<T, WIDE>(g, M, ring);
}

}  // namespace

namespace fdh {

hipError_t launch_int_linear(const IntLinearArgs& g, hipStream_t s) {
  auto run = [&](auto wide) {
    constexpr bool WIDE = decltype(wide)::value;
    using std::integral_constant;
    const integral_constant<int, 1> one{};
    const integral_constant<int, 2> two{};
    const integral_constant<int, 3> three{};
    const integral_constant<int, 4> four{};
    auto few = [&](auto fm, auto nf, auto deep) {
      constexpr int FM = decltype(fm)::value, NF = decltype(nf)::value;
      int_few_kernel<WIDE, FM, NF, decltype(deep)::value><<<dim3((g.N + 16 * NF - 1) / (16 * NF), (g.n_rows + 16 * FM - 1) / (16 * FM)), kFewWaves * 64, 0, s>>>(g);
    };
    auto split = [&](auto tile) {
      using T = decltype(tile);
      int_split_kernel<WIDE, T><<<dim3((g.N + T::BN - 1) / T::BN, (g.n_rows + T::BM - 1) / T::BM), T::THREADS, 0, s>>>(g);
    };
    const int cus = num_cus() / 8 * 8;
    auto tiles = [&](auto tile, auto per_cu, int check) {
      using T = decltype(tile);
      constexpr int PER_CU = decltype(per_cu)::value;
      const long long all = static_cast<long long>((g.n_rows + T::BM - 1) / T::BM) * ((g.N + T::BN - 1) / T::BN), most = PER_CU * cus;
      int_tile_kernel<WIDE, T, PER_CU><<<static_cast<int>(all < most ? (all + 7) / 8 * 8 : most), T::THREADS, 0, s>>>(g, check);
    };
    const int frags = fd::scaled_few_frags(g.n_rows);
    switch (fd::int_kernel(g.n_rows, g.N, g.K, WIDE, g.m != nullptr, num_cus())) {
      case fd::kIntFew:
        if (fd::scaled_few_wide(g.N, num_cus())) {
          if (frags == 1) few(one, two, two);
          else if (frags == 2) few(two, two, two);
          else few(four, two, one);
        } else {
          if (frags == 1) few(one, one, three);
          else if (frags == 2) few(two, one, two);
          else few(four, one, one);
        }
        break;
      case fd::kIntSplit32: split(IntSplit<1, 1, 4>{}); break;
      case fd::kIntSplit32x64: split(IntSplit<1, 2, 3>{}); break;
      case fd::kIntSplit64: split(IntSplit<2, 2, 2>{}); break;
      case fd::kInt64: tiles(Tile64{}, two, 0); break;
      case fd::kIntAlone: tiles(TileAlone{}, one, 0); break;
      case fd::kInt128: tiles(Tile128{}, two, 0); break;
      case fd::kInt256: tiles(TileLarge{}, one, 0); break;
      case fd::kIntBoth:
        tiles(Tile128{}, two, cus);
        tiles(TileLarge{}, one, cus);
        break;
    }
  };
  if (g.y_f32) run(std::true_type{});
  else run(std::false_type{});
  return hipGetLastError();
}

}  // namespace fdh
