// Rows to 8-bit codes with block scales: bf16 rows and weights as they are, and the residual
// stream through its RMS norm.
#include <type_traits>

#include "fd_scaled.h"

namespace {

using fd::kScaleBlock;

// bf16 rows [M][cols], one scale per 1 x 128: 16 lanes per block, 8 values (16 bytes) per lane.
// Bound by HBM: 3 bytes a value; 9828 x 1536 9.5 us (4.8 TB/s).
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
// in registers (8 pieces of 8 per thread) between the maximum and the codes: one read.  4352 x 1088 4.8 us, of
// which 2.8 are its bytes and the rest the launch and one round trip to HBM (306 workgroups, all resident at once).
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
// value.  The gate, the weight and the modulation are 16 bytes per value again, from the L2, where each row
// reads its own: so a row's waves take a run of rows and keep them in registers while the request stays.
// 8937 x 1536 rows of 8 requests 32.8 us (4.6 TB/s; with a row per wave and no runs 41.7, with runs of a wave
// each 36), 32760 rows 117 (4.7 TB/s), the branch's addition alone 22 and 104.
template <int WAVES>
constexpr int rms_threads() { return WAVES == 1 ? 256 : 64 * WAVES; }   // four rows of a wave each, or one row

template <int VEC, int WAVES>
__global__ __launch_bounds__(rms_threads<WAVES>()) void rms_quant_kernel(fdh::RmsArgs g) {
  constexpr int TEAMS = WAVES == 1 ? 4 : 1, LANES = 64 * WAVES;
  __shared__ float part[2][WAVES];
  const int wave = threadIdx.x >> 6, t = threadIdx.x % LANES;
  const int D = g.D, M = min(*g.m, g.n_rows), ld = fd::scale_stride(D);
  const int team = blockIdx.x * TEAMS + (WAVES == 1 ? wave : 0), teams = gridDim.x * TEAMS;
  const int run = (M + teams - 1) / teams, first = team * run, end = min(first + run, M);
  if (first >= end) return;   // the whole team together
  float gain[VEC][8], bias[VEC][8], gate[VEC][8];
  auto load8 = [&](const float* p, float (&v)[8]) {
    const float4 lo = *reinterpret_cast<const float4*>(p), hi = *reinterpret_cast<const float4*>(p + 4);
    v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
    v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
  };
  auto request = [&](int b) {   // its factors of a value: weight * (1 + scale), shift and gate
    const size_t mod = static_cast<size_t>(b) * g.mod_stride;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        gain[j][e] = gate[j][e] = 1.f;
        bias[j][e] = 0.f;
      }
      if (c >= D) continue;
      if (g.y && g.gate) load8(g.gate + mod + c, gate[j]);
      if (!g.q) continue;
      if (g.scale) {
        load8(g.scale + mod + c, gain[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) gain[j][e] += 1.f;
      }
      if (g.weight) {
        float w[8];
        load8(g.weight + c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) gain[j][e] *= w[e];
      }
      if (g.shift) load8(g.shift + mod + c, bias[j]);
    }
  };
  float v[VEC][8];
  uint4 y[VEC];
  auto fetch = [&](int row) {   // a row's values, zeros past its end
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
      y[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
      if (c >= D) continue;
      load8(g.h + static_cast<size_t>(row) * D + c, v[j]);
      if (g.y) y[j] = *reinterpret_cast<const uint4*>(g.y + static_cast<size_t>(row) * D + c);
    }
  };
  int b = g.n_req == 1 ? 0 : fd::row_request(g.cu_q, g.n_req, first);
  int b_end = g.n_req == 1 ? M : g.cu_q[b + 1];   // rows of the request
  fetch(first);
  request(b);
  for (int row = first; row < end; ++row) {
    if (row >= b_end) {
      b = fd::row_request(g.cu_q, g.n_req, row);
      b_end = g.cu_q[b + 1];
      request(b);
    }
    float a[VEC][8];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
      float y8[8];
      fd::unpack_bf8(y[j], y8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        a[j][e] = g.y ? v[j][e] + gate[j][e] * y8[e] : v[j][e];
        sum += a[j][e] * a[j][e];
      }
      if (g.y && c < D) {
        float* h = g.h + static_cast<size_t>(row) * D + c;
        *reinterpret_cast<float4*>(h) = make_float4(a[j][0], a[j][1], a[j][2], a[j][3]);
        *reinterpret_cast<float4*>(h + 4) = make_float4(a[j][4], a[j][5], a[j][6], a[j][7]);
      }
    }
    if (row + 1 < end) fetch(row + 1);   // on its way while this row is summed and rounded
    if (!g.q) continue;                  // the residual alone
    sum = fd::wave_sum(sum);
    if constexpr (WAVES > 1) {
      float* p = part[row & 1];   // two sets: a wave may be a row ahead of one that has yet to read
      if ((threadIdx.x & 63) == 0) p[wave] = sum;
      __syncthreads();
      if constexpr (WAVES == 2) sum = p[0] + p[1];
      else sum = (p[0] + p[1]) + (p[2] + p[3]);
    }
    const float r = 1.0f / sqrtf(sum / static_cast<float>(D) + g.eps);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[j][e] = c < D ? a[j][e] * r * gain[j][e] + bias[j][e] : 0.f;   // zeros past the end, whatever r is
      uint2 codes;
      const uint32_t s = fd::quant_lane8(a[j], codes);
      if (c < D) {
        *reinterpret_cast<uint2*>(g.q + static_cast<size_t>(row) * D + c) = codes;
        if ((t & 15) == 0) g.q_scale[static_cast<size_t>(row) * ld + c / kScaleBlock] = static_cast<uint8_t>(s);
      }
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
  // 512 columns a wave, so that a lane holds eight of every operand and 16 to 20 waves fit a CU; from 2048
  // columns on four waves hold more each.  As many workgroups as are resident at 1024 to 2048 columns: runs of
  // about the same length, whose factors are read once.
  const int cap = 4 * num_cus();
  auto run = [&](auto vec, auto waves) {
    constexpr int VEC = decltype(vec)::value, WAVES = decltype(waves)::value;
    const int most = WAVES == 2 ? 2 * cap : cap, rows = WAVES == 1 ? (g.n_rows + 3) / 4 : g.n_rows;
    rms_quant_kernel<VEC, WAVES><<<rows < most ? rows : most, rms_threads<WAVES>(), 0, s>>>(g);
  };
  using std::integral_constant;
  const integral_constant<int, 4> four;
  if (g.D <= 512) run(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (g.D <= 1024) run(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else switch ((g.D + 2047) / 2048) {
    case 1: run(integral_constant<int, 1>{}, four); break;
    case 2: run(integral_constant<int, 2>{}, four); break;
    case 3: run(integral_constant<int, 3>{}, four); break;
    case 4: run(integral_constant<int, 4>{}, four); break;
    default: run(integral_constant<int, 6>{}, four);
  }
  return hipGetLastError();
}

}  // namespace fdh
