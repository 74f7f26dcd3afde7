// Rows to 8-bit codes with block scales: bf16 rows and weights as they are, and the residual
// stream through its RMS norm.
#include "fd_scaled.h"

namespace {

using fd::kScaleBlock;

// bf16 rows [M][cols], one scale per 1 x 128: 16 lanes per block, 8 values (16 bytes) per lane.
// Bound by HBM: 3 bytes a value.
__global__ __launch_bounds__(256) void quant_rows_kernel(const uint16_t* __restrict__ x, int n_rows, int cols,
                                                         const int32_t* __restrict__ m_dev, uint8_t* __restrict__ q,
                                                         uint8_t* __restrict__ scale) {
  const int M = m_dev ? min(*m_dev, n_rows) : n_rows;
  const int nk = (cols + kScaleBlock - 1) / kScaleBlock, ld = fd::scale_stride(cols);
  const long long blocks = static_cast<long long>(M) * nk;
  const int sub = threadIdx.x & 15;
  for (long long t = (blockIdx.x * 256LL + threadIdx.x) >> 4; t < blocks; t += gridDim.x * 16LL) {
    const long long row = t / nk;
    const int kb = static_cast<int>(t - row * nk), c = kb * kScaleBlock + 8 * sub;
    const size_t at = static_cast<size_t>(row) * cols + c;
    float v[8];
    fd::unpack_bf8(c < cols ? *reinterpret_cast<const uint4*>(x + at) : make_uint4(0, 0, 0, 0), v);
    uint2 codes;
    const uint32_t s = fd::quant_lane8(v, codes);
    if (c < cols) *reinterpret_cast<uint2*>(q + at) = codes;
    if (sub == 0) scale[static_cast<size_t>(row) * ld + kb] = static_cast<uint8_t>(s);
  }
}

// bf16 weights [rows][cols], one scale per 128 x 128: a workgroup per block, its 128 x 128 values
// in registers (8 pieces of 8 per thread) between the maximum and the codes.
__global__ __launch_bounds__(256) void quant_weights_kernel(const uint16_t* __restrict__ x, int rows, int cols,
                                                            uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  __shared__ uint32_t tops[4];
  const int nk = (cols + kScaleBlock - 1) / kScaleBlock, ld = fd::scale_stride(cols);
  const int rb = blockIdx.x / nk, kb = blockIdx.x - rb * nk;
  const int c = kb * kScaleBlock + 8 * (threadIdx.x & 15), r0 = rb * kScaleBlock + (threadIdx.x >> 4);
  uint4 x8[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    x8[i] = (r < rows && c < cols) ? *reinterpret_cast<const uint4*>(x + static_cast<size_t>(r) * cols + c) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    fd::unpack_bf8(x8[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, fd::mag_bits(v[e]));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, fd::kWave)));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  const uint32_t s = fd::scale_byte(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  const float inv = fd::scale_inverse(s);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    float v[8];
    fd::unpack_bf8(x8[i], v);
    uint2 codes;
    codes.x = fd::pack_codes(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    codes.y = fd::pack_codes(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    if (r < rows && c < cols) *reinterpret_cast<uint2*>(q + static_cast<size_t>(r) * cols + c) = codes;
  }
  if (threadIdx.x == 0) scale[static_cast<size_t>(rb) * ld + kb] = static_cast<uint8_t>(s);
}

// h += gate_b * y, then a = h / sqrt(mean(h^2) + eps) * weight * (1 + scale_b) + shift_b to codes.
// WAVES waves per row hold it in registers between the sum of squares and the codes: lane t of the
// row's 64 * WAVES takes the 8 columns at 8 * (t + 64 * WAVES * j), j < VEC, so that 16 lanes hold
// one block.  Sums in fp32.  Bound by HBM: 4 bytes of h read and 4 written, 2 of y, 1 of codes per
// value.
template <int VEC, int WAVES>
__global__ __launch_bounds__(256) void rms_quant_kernel(fdh::RmsArgs g) {
  constexpr int ROWS = 4 / WAVES, LANES = 64 * WAVES;
  __shared__ float part[4];
  const int wave = threadIdx.x >> 6, t = threadIdx.x % LANES;
  const int row = blockIdx.x * ROWS + (WAVES == 1 ? wave : 0);
  if (row >= min(*g.m, g.n_rows)) return;   // the whole row's waves together
  const int D = g.D;
  const int b = g.n_req == 1 ? 0 : fd::row_request(g.cu_q, g.n_req, row);
  float* h = g.h + static_cast<size_t>(row) * D;
  const size_t mod = static_cast<size_t>(b) * g.mod_stride;
  float v[VEC][8];
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    const int c = 8 * (t + LANES * j);
    if (c < D) {
      const float4 lo = *reinterpret_cast<const float4*>(h + c), hi = *reinterpret_cast<const float4*>(h + c + 4);
      v[j][0] = lo.x; v[j][1] = lo.y; v[j][2] = lo.z; v[j][3] = lo.w;
      v[j][4] = hi.x; v[j][5] = hi.y; v[j][6] = hi.z; v[j][7] = hi.w;
      if (g.y) {
        float y[8];
        fd::unpack_bf8(*reinterpret_cast<const uint4*>(g.y + static_cast<size_t>(row) * D + c), y);
        if (g.gate) {
          const float4 g0 = *reinterpret_cast<const float4*>(g.gate + mod + c), g1 = *reinterpret_cast<const float4*>(g.gate + mod + c + 4);
          y[0] *= g0.x; y[1] *= g0.y; y[2] *= g0.z; y[3] *= g0.w;
          y[4] *= g1.x; y[5] *= g1.y; y[6] *= g1.z; y[7] *= g1.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] += y[e];
        *reinterpret_cast<float4*>(h + c) = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
        *reinterpret_cast<float4*>(h + c + 4) = make_float4(v[j][4], v[j][5], v[j][6], v[j][7]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[j][e] * v[j][e];
  }
  if (!g.q) return;   // the residual alone
  sum = fd::wave_sum(sum);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[wave] = sum;
    __syncthreads();
    sum = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const float r = 1.0f / sqrtf(sum / static_cast<float>(D) + g.eps);
  const int ld = fd::scale_stride(D);
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    const int c = 8 * (t + LANES * j);
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = v[j][e] * r;
    if (c < D) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int cp = c + 4 * p;
        float* a4 = a + 4 * p;
        if (g.weight) {
          const float4 w = *reinterpret_cast<const float4*>(g.weight + cp);
          a4[0] *= w.x; a4[1] *= w.y; a4[2] *= w.z; a4[3] *= w.w;
        }
        if (g.scale) {
          const float4 s = *reinterpret_cast<const float4*>(g.scale + mod + cp);
          a4[0] *= 1.f + s.x; a4[1] *= 1.f + s.y; a4[2] *= 1.f + s.z; a4[3] *= 1.f + s.w;
        }
        if (g.shift) {
          const float4 s = *reinterpret_cast<const float4*>(g.shift + mod + cp);
          a4[0] += s.x; a4[1] += s.y; a4[2] += s.z; a4[3] += s.w;
        }
      }
    } else {   // past the row's end, also where r is infinite or NaN
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = 0.f;
    }
    uint2 codes;
    const uint32_t s = fd::quant_lane8(a, codes);
    if (c < D) {
      *reinterpret_cast<uint2*>(g.q + static_cast<size_t>(row) * D + c) = codes;
      if ((t & 15) == 0) g.q_scale[static_cast<size_t>(row) * ld + c / kScaleBlock] = static_cast<uint8_t>(s);
    }
  }
}

}  // namespace

namespace fdh {

hipError_t launch_quant_blocks(const uint16_t* x, int n_rows, int cols, int block_rows, const int32_t* m, uint8_t* q,
                               uint8_t* scale, hipStream_t s) {
  const int nk = (cols + kScaleBlock - 1) / kScaleBlock;
  if (block_rows == 1) {
    const long long blocks = static_cast<long long>(n_rows) * nk, cap = 32LL * num_cus();
    const long long grid = (blocks + 15) / 16;
    quant_rows_kernel<<<static_cast<int>(grid < cap ? grid : cap), 256, 0, s>>>(x, n_rows, cols, m, q, scale);
  } else {
    quant_weights_kernel<<<(n_rows + kScaleBlock - 1) / kScaleBlock * nk, 256, 0, s>>>(x, n_rows, cols, q, scale);
  }
  return hipGetLastError();
}

hipError_t launch_rms_quant(const RmsArgs& g, hipStream_t s) {
  // one wave per row up to 2048 columns (32 floats of the row per lane), four above
  if (g.D <= 2048) {
    const int grid = (g.n_rows + 3) / 4;
    switch ((g.D + 511) / 512) {
      case 1: rms_quant_kernel<1, 1><<<grid, 256, 0, s>>>(g); break;
      case 2: rms_quant_kernel<2, 1><<<grid, 256, 0, s>>>(g); break;
      case 3: rms_quant_kernel<3, 1><<<grid, 256, 0, s>>>(g); break;
      default: rms_quant_kernel<4, 1><<<grid, 256, 0, s>>>(g);
    }
  } else {
    switch ((g.D + 2047) / 2048) {
      case 2: rms_quant_kernel<2, 4><<<g.n_rows, 256, 0, s>>>(g); break;
      case 3: rms_quant_kernel<3, 4><<<g.n_rows, 256, 0, s>>>(g); break;
      case 4: rms_quant_kernel<4, 4><<<g.n_rows, 256, 0, s>>>(g); break;
      default: rms_quant_kernel<6, 4><<<g.n_rows, 256, 0, s>>>(g);
    }
  }
  return hipGetLastError();
}

}  // namespace fdh
