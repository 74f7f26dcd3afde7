// The product of 8-bit rows and weights with block scales:
//   Y[M][N] = act(sum over K-blocks kb of 2^(sa[row][kb] + sw[col / 128][kb] - 254) (A . W^T)_kb + bias)
// on v_mfma_scale_f32_16x16x128_f8f6f4, whose K is one block: the scale bytes are operands of the
// instruction and the sum is kept in fp32 accumulators.
//
// The weight fragment is the first operand, so an accumulator holds the transposed block: lane l a
// row of Y (l & 15) and four columns per fragment.  The 16 weight rows of fragment j of a wave's 128
// columns are 32 (x >> 2) + 4 j + (x & 3), x < 16: the eight fragments then give lane l the 32
// consecutive columns 32 (l >> 4) .. + 31, which leave in 16-byte stores, and four lanes hold the
// 128 columns that share an output scale.
#include <stdlib.h>

#include <type_traits>

#include "fd_scaled.h"

namespace {

using fd::bf16x2_t;
using fd::kScaleBlock;
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

enum { kToBf16, kToF32, kToCodes };

// Two ways to the sum of one K-block of 128:
// - 8-bit: v_mfma_scale_f32_16x16x128_f8f6f4.  It adds 8 products at a time on a grid 2^-13 below the
//   largest of them (measured: 1 + 2^-14 gives 1 within such a group, and is exact across groups and
//   with the accumulator), which leaves random operands' sums off by 1.5e-5 of their size.
//   Outputs of 8 (bf16) or 4 (e4m3) bits of mantissa round by 100 times that at least.
// - exact: the codes times their scales as bf16 (exact) through v_mfma_f32_16x16x32_bf16, half the
//   rate, whose sums are fp32's.  fp32 outputs take this one.
struct Mma8 {
  typedef i32x8_t frag;
  static FD_DEVICE frag make(i32x8_t x, uint32_t) { return x; }
  static FD_DEVICE f32x4_t mma(const frag& w, const frag& a, f32x4_t c, uint32_t sw, uint32_t sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, static_cast<int>(sw), 0, static_cast<int>(sa));
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
};

// One row's 4 NF columns from col on (col a multiple of 4 NF; N is a multiple of 16, so each 16 lie
// inside or outside).  Every lane of the wave runs it; codes need the whole block (NF = 8).
template <int KIND, int NF>
FD_DEVICE void store_row(const fdh::ScaledArgs& g, bool row_ok, int row, int col, const f32x4_t (&acc)[NF]) {
  static_assert(KIND != kToCodes || NF == 8, "four lanes hold a block's columns");
  float v[4 * NF];
#pragma unroll
  for (int j = 0; j < NF; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) v[4 * j + r] = acc[j][r];
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int c = col + 4 * j;
    if (g.bias && c < g.N) {
      const float4 b = *reinterpret_cast<const float4*>(g.bias + c);
      v[4 * j] += b.x; v[4 * j + 1] += b.y; v[4 * j + 2] += b.z; v[4 * j + 3] += b.w;
    }
  }
  if (g.gelu) {
#pragma unroll
    for (int e = 0; e < 4 * NF; ++e) v[e] = fd::gelu_tanh_fast(v[e]);
  }
  const size_t at = static_cast<size_t>(row) * g.N + col;
  if constexpr (KIND == kToCodes) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 32; ++e) top = (col + (e & 16) < g.N) ? max(top, fd::mag_bits(v[e])) : top;
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16, fd::kWave)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32, fd::kWave)));
    const uint32_t s = fd::scale_byte(top);
    const float inv = fd::scale_inverse(s);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* x = v + 16 * h + 4 * i;
        w[i] = fd::pack_codes(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
      }
      if (row_ok && col + 16 * h < g.N) *reinterpret_cast<uint4*>(g.y_q + at + 16 * h) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (row_ok && col < g.N && (col & (kScaleBlock - 1)) == 0)
      g.y_scale[static_cast<size_t>(row) * fd::scale_stride(g.N) + col / kScaleBlock] = static_cast<uint8_t>(s);
  } else if constexpr (KIND == kToBf16 && NF == 1) {
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

// 32 bytes at p + k of a row of K bytes, zeros past its end (K is a multiple of 16).
FD_DEVICE i32x8_t load32(const uint8_t* p, int k, int K) {
  const uint4 z = make_uint4(0, 0, 0, 0);
  const uint4 lo = k < K ? *reinterpret_cast<const uint4*>(p + k) : z, hi = k + 16 < K ? *reinterpret_cast<const uint4*>(p + k + 16) : z;
  return i32x8_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                 static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
}

// ---------------------------------------------------------------- few rows

// Up to FM * 16 rows: the weights are read once and are all there is to read.  A workgroup takes the
// rows' FM fragments and 16 NF columns, its waves the K-blocks in turn, operands straight from memory
// into registers; the waves' sums meet in LDS.
constexpr int kFewWaves = 8;

template <int KIND, class Mma, int FM, int NF>
__global__ __launch_bounds__(kFewWaves * 64) void scaled_few_kernel(fdh::ScaledArgs g) {
  __shared__ f32x4_t part[kFewWaves][FM * NF][64];
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, lg = lane >> 4;
  const int nk = (g.K + kScaleBlock - 1) / kScaleBlock, ld = fd::scale_stride(g.K);
  const int n0 = blockIdx.x * 16 * NF;
  const uint8_t* sw = g.w_scale + static_cast<size_t>(n0 / kScaleBlock) * ld;
  const uint8_t* w[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j)
    w[j] = g.w + static_cast<size_t>(min(n0 + 4 * NF * (l16 >> 2) + 4 * j + (l16 & 3), g.N - 1)) * g.K;
  for (int m0 = blockIdx.y * 16 * FM; m0 < M; m0 += gridDim.y * 16 * FM) {
    f32x4_t acc[FM][NF] = {};
    for (int kb = wave; kb < nk; kb += kFewWaves) {
      const int k = kb * kScaleBlock + 32 * lg;
      typename Mma::frag wf[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) wf[j] = Mma::make(load32(w[j], k, g.K), sw[kb]);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const size_t r = min(m0 + 16 * i + l16, M - 1);
        const uint32_t sa = g.a_scale[r * ld + kb];
        const typename Mma::frag af = Mma::make(load32(g.a + r * g.K, k, g.K), sa);
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = Mma::mma(wf[j], af, acc[i][j], sw[kb], sa);
      }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) part[wave][i * NF + j][lane] = acc[i][j];
    __syncthreads();
    for (int i = wave; i < FM; i += kFewWaves) {   // a wave per 16 rows adds the waves' sums in order
      f32x4_t sum[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        sum[j] = part[0][i * NF + j][lane];
#pragma unroll
        for (int p = 1; p < kFewWaves; ++p) sum[j] += part[p][i * NF + j][lane];
      }
      const int row = m0 + 16 * i + l16;
      store_row<KIND, NF>(g, row < M, row, n0 + 4 * NF * lg, sum);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- tiles

// A workgroup of four waves, one per SIMD, with a tile of 16 FM WM rows x 128 WN columns: a wave owns
// FM x 8 fragments (its accumulators fill up to 256 accumulation registers).
template <int FM_, int WM_, int WN_, int STAGES_>
struct Tile {
  static constexpr int FM = FM_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int BM = 16 * FM * WM, BN = 128 * WN, WAVES = 4;
  static constexpr int LOADS_A = BM / 8 / WAVES, LOADS = (BM + BN) / 8 / WAVES;   // 8 rows of 128 bytes per wave-load
  static constexpr int ISSUED = LOADS + 2;                                        // and two of scales
  static constexpr int SIDE = (BM + BN) * 8;                                      // chunk where the scales begin
  static constexpr int CHUNKS = SIDE + 2 * WAVES * 16;                            // 16-byte chunks per stage
  static_assert(WM * WN == WAVES && BM % 32 == 0, "four waves, whole wave-loads");
};

typedef __attribute__((address_space(3))) void* lds_ptr_t;

FD_DEVICE i32x4_t buffer_of(const void* base) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return i32x4_t{static_cast<int>(static_cast<uint32_t>(p)), static_cast<int>(static_cast<uint32_t>(p >> 32) & 0xffffu), 0x7fffffff, 0x00020000};
}
// 16 (4) bytes per lane from buffer offset voff + soff into LDS at lds + 16 (4) * lane; offsets past
// 2 GiB read zeros.  In assembly so that the compiler does not wait for it before unrelated LDS reads.
FD_DEVICE void dma16(uint32_t lds, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff));
}
FD_DEVICE void dma4(uint32_t lds, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff));
}
template <int N>
FD_DEVICE void wait_vm_barrier() {
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(N) : "memory");
}

template <class T, int KIND, class Mma>
FD_DEVICE void scaled_tiles(const fdh::ScaledArgs& g, int M, uint4* ring) {
  constexpr int FM = T::FM, STAGES = T::STAGES;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WN, wn = wave % T::WN;
  const int K = g.K, nk = (K + kScaleBlock - 1) / kScaleBlock, ld = fd::scale_stride(K);
  const int tiles_m = (M + T::BM - 1) / T::BM, tiles_n = (g.N + T::BN - 1) / T::BN, tiles = tiles_m * tiles_n;
  const int per_xcd = (tiles + 7) / 8;
  const uint32_t ring_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)ring));

  for (int u = blockIdx.x; u < per_xcd * 8; u += gridDim.x) {
    // consecutive tiles on one XCD (a workgroup runs on XCD blockIdx.x % 8), in groups of 8 row tiles x
    // every column tile, so that the tiles an XCD runs at once share operand rows in its L2
    const int tile = (u % 8) * per_xcd + u / 8;
    if (tile >= tiles) break;
    const int grp = tile / (8 * tiles_n), in = tile - grp * 8 * tiles_n, gm = min(8, tiles_m - 8 * grp);
    const int m0 = (8 * grp + in % gm) * T::BM, n0 = in / gm * T::BN;

    const i32x4_t ra = buffer_of(g.a + static_cast<size_t>(m0) * K), rw = buffer_of(g.w + static_cast<size_t>(n0) * K);
    const i32x4_t rsa = buffer_of(g.a_scale + static_cast<size_t>(m0) * ld);
    const i32x4_t rsw = buffer_of(g.w_scale + static_cast<size_t>(n0 / kScaleBlock) * ld);
    // this lane's row and chunk of each wave-load; rows past M (N) re-read the last one
    auto chunk_of = [&](int q) {
      const bool a = q < T::LOADS_A;
      const int r = (wave + 4 * (a ? q : q - T::LOADS_A)) * 8 + (lane >> 3);
      return (lane & 7) ^ (a ? (r >> 1) & 7 : ((r >> 1) & 1) | ((r >> 5) & 3) << 1);
    };
    uint32_t off[T::LOADS];
#pragma unroll
    for (int q = 0; q < T::LOADS; ++q) {
      const bool a = q < T::LOADS_A;
      const int r = (wave + 4 * (a ? q : q - T::LOADS_A)) * 8 + (lane >> 3);
      off[q] = static_cast<uint32_t>(min(r, (a ? M - m0 : g.N - n0) - 1)) * static_cast<uint32_t>(K) + 16 * chunk_of(q);
    }
    const uint32_t off_sa = static_cast<uint32_t>(min((64 * wave + lane) % T::BM, M - m0 - 1) * ld);
    const uint32_t off_sw = static_cast<uint32_t>(min(lane % T::WN, (g.N - n0 - 1) / kScaleBlock) * ld);
    auto issue = [&](int kb, int slot) {
      const uint32_t at = ring_at + static_cast<uint32_t>(slot * T::CHUNKS * 16), k = static_cast<uint32_t>(kb * kScaleBlock);
      auto load = [&](int q, uint32_t v) {
        const uint32_t blk = q < T::LOADS_A ? wave + 4 * q : T::BM / 8 + wave + 4 * (q - T::LOADS_A);
        dma16(at + blk * 1024, v, q < T::LOADS_A ? ra : rw, k);
      };
      if (kb * kScaleBlock + kScaleBlock <= K) {
#pragma unroll
        for (int q = 0; q < T::LOADS; ++q) load(q, off[q]);
      } else {   // the last, shorter K-block: chunks past K read zeros
        const int left = (K - kb * kScaleBlock) / 16;
#pragma unroll
        for (int q = 0; q < T::LOADS; ++q) load(q, chunk_of(q) < left ? off[q] : 0x80000000u);
      }
      const uint32_t kb4 = static_cast<uint32_t>(kb & ~3);
      dma4(at + T::SIDE * 16 + wave * 256, off_sa, rsa, kb4);
      dma4(at + T::SIDE * 16 + 1024 + wave * 256, off_sw, rsw, kb4);
    };
    auto frag_at = [&](const uint4* sm, int row, int swz) {
      const uint4 lo = sm[row * 8 + ((2 * lg) ^ swz)], hi = sm[row * 8 + ((2 * lg + 1) ^ swz)];
      return i32x8_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                     static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
    };

    f32x4_t acc[FM][8] = {};
#pragma unroll
    for (int p = 0; p < STAGES - 1; ++p) issue(min(p, nk - 1), p);
    for (int kb = 0; kb < nk; ++kb) {
      wait_vm_barrier<(STAGES - 2) * T::ISSUED>();
      issue(min(kb + STAGES - 1, nk - 1), (kb + STAGES - 1) % STAGES);
      const uint4* sm = ring + (kb % STAGES) * T::CHUNKS;
      const uint32_t* side = reinterpret_cast<const uint32_t*>(sm + T::SIDE);
      const int sh = 8 * (kb & 3);
      const uint32_t sw = side[256 + 64 * wave + wn] >> sh;
      typename Mma::frag wf[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = 128 * wn + 32 * (l16 >> 2) + 4 * j + (l16 & 3);
        wf[j] = Mma::make(frag_at(sm + T::BM * 8, r, ((r >> 1) & 1) | ((r >> 5) & 3) << 1), sw);
      }
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int r = 16 * FM * wm + 16 * i + l16;
        const uint32_t sa = side[r] >> sh;
        const typename Mma::frag af = Mma::make(frag_at(sm, r, (r >> 1) & 7), sa);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = Mma::mma(wf[j], af, acc[i][j], sw, sa);
      }
    }
    // the last stages' repeats may still be landing: drained before the ring is used again
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = m0 + 16 * FM * wm + 16 * i + l16;
      store_row<KIND, 8>(g, row < M, row, n0 + 128 * wn + 32 * lg, acc[i]);
    }
  }
}

using TileLarge = Tile<8, 2, 2, 2>;   // 256 x 256
using TileMid = Tile<4, 2, 2, 3>;     // 128 x 256
using TileSmall = Tile<2, 4, 1, 4>;   // 128 x 128
constexpr int kRing = TileMid::STAGES * TileMid::CHUNKS;
static_assert(kRing >= TileLarge::STAGES * TileLarge::CHUNKS && kRing >= TileSmall::STAGES * TileSmall::CHUNKS && kRing * 16 <= 160 * 1024, "one ring for all");

template <int KIND, class Mma>
__global__ __launch_bounds__(256, 1) void scaled_tile_kernel(fdh::ScaledArgs g, int shape) {
  __shared__ uint4 ring[kRing];
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  if (M <= 0) return;
  switch (shape) {
    case 0: scaled_tiles<TileLarge, KIND, Mma>(g, M, ring); break;
    case 1: scaled_tiles<TileMid, KIND, Mma>(g, M, ring); break;
    default: scaled_tiles<TileSmall, KIND, Mma>(g, M, ring); break;
  }
}

}  // namespace

namespace fdh {

hipError_t launch_scaled_linear(const ScaledArgs& g, hipStream_t s) {
  auto run = [&](auto kind, auto mma) {
    constexpr int KIND = decltype(kind)::value;
    using Mma = decltype(mma);
    if (g.n_rows <= 64) {
      constexpr int NF = KIND == kToCodes ? 8 : 1;
      const int gx = (g.N + 16 * NF - 1) / (16 * NF);
      if (g.n_rows <= 16) scaled_few_kernel<KIND, Mma, 1, NF><<<dim3(gx, 1), kFewWaves * 64, 0, s>>>(g);
      else scaled_few_kernel<KIND, Mma, 2, NF><<<dim3(gx, (g.n_rows + 31) / 32), kFewWaves * 64, 0, s>>>(g);
      return;
    }
    const char* e = getenv("FD_SHAPE");
    const int shape = e ? atoi(e) : 0;
    scaled_tile_kernel<KIND, Mma><<<num_cus() / 8 * 8, 256, 0, s>>>(g, shape);
  };
  if (g.y_q) run(std::integral_constant<int, kToCodes>{}, Mma8{});
  else if (g.y_bf16) run(std::integral_constant<int, kToBf16>{}, Mma8{});
  else run(std::integral_constant<int, kToF32>{}, MmaExact{});
  return hipGetLastError();
}

}  // namespace fdh
