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
#include <type_traits>

#include "fd_scaled.h"

namespace {

using fd::kScaleBlock;
typedef int i32x8_t __attribute__((ext_vector_type(8)));

enum { kToBf16, kToF32, kToCodes };

FD_DEVICE f32x4_t mma(i32x8_t w, i32x8_t a, f32x4_t c, uint32_t sw, uint32_t sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, static_cast<int>(sw), 0, static_cast<int>(sa));
}

// One row's 32 columns col .. col + 31 (col a multiple of 32; N is a multiple of 16, so each half
// lies inside or outside).  Every lane of the wave runs it.
template <int KIND>
FD_DEVICE void store_row(const fdh::ScaledArgs& g, bool row_ok, int row, int col, const f32x4_t (&acc)[8]) {
  float v[32];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) v[4 * j + r] = acc[j][r];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = col + 4 * j;
    if (g.bias && c < g.N) {
      const float4 b = *reinterpret_cast<const float4*>(g.bias + c);
      v[4 * j] += b.x; v[4 * j + 1] += b.y; v[4 * j + 2] += b.z; v[4 * j + 3] += b.w;
    }
  }
  if (g.gelu) {
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = fd::gelu_tanh_fast(v[e]);
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
  } else if constexpr (KIND == kToBf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* x = v + 8 * i;
      if (row_ok && col + (8 * i & 16) < g.N)
        *reinterpret_cast<uint4*>(g.y_bf16 + at + 8 * i) = make_uint4(fd::pack_bf2(x[0], x[1]), fd::pack_bf2(x[2], x[3]), fd::pack_bf2(x[4], x[5]), fd::pack_bf2(x[6], x[7]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
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

// 16 rows x 128 columns per wave, operands straight from memory.
template <int KIND>
__global__ __launch_bounds__(256) void scaled_plain_kernel(fdh::ScaledArgs g) {
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows;
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int tiles_m = (M + 15) / 16, tiles_n = (g.N + kScaleBlock - 1) / kScaleBlock;
  const long long tiles = static_cast<long long>(tiles_m) * tiles_n;
  const int nk = (g.K + kScaleBlock - 1) / kScaleBlock, ld = fd::scale_stride(g.K);
  for (long long t = blockIdx.x * 4LL + (threadIdx.x >> 6); t < tiles; t += gridDim.x * 4LL) {
    const int tn = static_cast<int>(t / tiles_m), m0 = static_cast<int>(t - static_cast<long long>(tn) * tiles_m) * 16, n0 = tn * kScaleBlock;
    const int row = m0 + l16, ra = min(row, M - 1);
    const uint8_t* a = g.a + static_cast<size_t>(ra) * g.K;
    const uint8_t* sa = g.a_scale + static_cast<size_t>(ra) * ld;
    const uint8_t* sw = g.w_scale + static_cast<size_t>(tn) * ld;
    f32x4_t acc[8] = {};
    for (int kb = 0; kb < nk; ++kb) {
      const int k = kb * kScaleBlock + 32 * lg;
      const i32x8_t af = load32(a, k, g.K);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int n = min(n0 + 32 * (l16 >> 2) + 4 * j + (l16 & 3), g.N - 1);
        acc[j] = mma(load32(g.w + static_cast<size_t>(n) * g.K, k, g.K), af, acc[j], sw[kb], sa[kb]);
      }
    }
    store_row<KIND>(g, row < M, row, n0 + 32 * lg, acc);
  }
}

}  // namespace

namespace fdh {

hipError_t launch_scaled_linear(const ScaledArgs& g, hipStream_t s) {
  const long long tiles = static_cast<long long>((g.n_rows + 15) / 16) * ((g.N + kScaleBlock - 1) / kScaleBlock);
  const long long want = (tiles + 3) / 4, cap = 8LL * num_cus();
  const int grid = static_cast<int>(want < cap ? want : cap);
  if (g.y_q) scaled_plain_kernel<kToCodes><<<grid, 256, 0, s>>>(g);
  else if (g.y_bf16) scaled_plain_kernel<kToBf16><<<grid, 256, 0, s>>>(g);
  else scaled_plain_kernel<kToF32><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace fdh
