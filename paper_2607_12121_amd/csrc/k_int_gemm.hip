// The product of 8-bit integers with a scale per row and per column:
//   Y[M][N] = act(float(sum_k A[i][k] W[j][k]) * (a_scale[i] * w_scale[j]) + bias[j])
// on v_mfma_i32_32x32x32_i8: the sums are whole numbers below 2^31 (K <= 2^16) and exact.
#include <type_traits>

#include "fd_int.h"

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

constexpr int BM = 128, BN = 128, BK = 128, kPitch = BK + 16;   // bytes of a tile row in LDS

template <bool WIDE>   // fp32 results, else bf16
__global__ __launch_bounds__(256) void int_tile_kernel(fdh::IntLinearArgs g) {
  __shared__ __align__(16) uint8_t ta[BM * kPitch], tw[BN * kPitch];
  const int M = g.m ? min(*g.m, g.n_rows) : g.n_rows, K = g.K, N = g.N;
  const int m0 = blockIdx.y * BM, n0 = blockIdx.x * BN;
  if (m0 >= M) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
  i32x16_t acc[4] = {};
  for (int k0 = 0; k0 < K; k0 += BK) {
    for (int i = threadIdx.x; i < BM * BK / 16; i += 256) {
      const int r = i / (BK / 16), c = i % (BK / 16) * 16, k = k0 + c;
      const uint4 none = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(ta + r * kPitch + c) = m0 + r < M && k < K ? *reinterpret_cast<const uint4*>(g.a + static_cast<size_t>(m0 + r) * K + k) : none;
      *reinterpret_cast<uint4*>(tw + r * kPitch + c) = n0 + r < N && k < K ? *reinterpret_cast<const uint4*>(g.w + static_cast<size_t>(n0 + r) * K + k) : none;
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < BK / 32; ++ks) {
      const i32x4_t a = *reinterpret_cast<const i32x4_t*>(ta + (32 * wave + l32) * kPitch + 32 * ks + 16 * half);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const i32x4_t w = *reinterpret_cast<const i32x4_t*>(tw + (32 * j + l32) * kPitch + 32 * ks + 16 * half);
        acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, w, acc[j], 0, 0, 0);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int col = n0 + 32 * j + l32;
    if (col >= N) continue;
    const float sw = g.w_scale[col], bias = g.bias ? g.bias[col] : 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = m0 + 32 * wave + 8 * (r >> 2) + 4 * half + (r & 3);
      if (row >= M) continue;
      float v = static_cast<float>(acc[j][r]) * (g.a_scale[row] * sw) + bias;
      if (g.gelu) v = fd::gelu(v);
      const size_t at = static_cast<size_t>(row) * N + col;
      if constexpr (WIDE) g.y_f32[at] = v;
      else g.y_bf16[at] = fd::f2bf(v);
    }
  }
}

}  // namespace

namespace fdh {

hipError_t launch_int_linear(const IntLinearArgs& g, hipStream_t s) {
  const dim3 grid((g.N + BN - 1) / BN, (g.n_rows + BM - 1) / BM);
  if (g.y_f32) int_tile_kernel<true><<<grid, 256, 0, s>>>(g);
  else int_tile_kernel<false><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace fdh
