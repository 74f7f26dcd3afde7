// Rows of 8-bit integers: bf16 rows as they are, and the residual stream through the norms behind and before a
// block's branches (which also come as bf16 rows and as codes).
#include <type_traits>

#include "fd_int.h"

namespace {

// A row belongs to a team of LANES lanes: 16, 32 or a wave, several of which make a workgroup, or whole waves, which are one.
template <int LANES>
constexpr int team_threads() { return LANES <= 64 ? 256 : LANES; }
template <int LANES>
FD_DEVICE int first_team() {   // number of this lane's team
  constexpr int TEAMS = team_threads<LANES>() / LANES;
  if constexpr (TEAMS == 1) return blockIdx.x;
  else if constexpr (LANES == 64) return blockIdx.x * TEAMS + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  else return blockIdx.x * TEAMS + threadIdx.x / LANES;
}
// f over the values of a team's lanes, or of a wave's where it is more.
template <int LANES, class T, class F>
FD_DEVICE T over_lanes(T v, F f) {
#pragma unroll
  for (int o = LANES < 64 ? LANES / 2 : 32; o > 0; o >>= 1) v = f(v, __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(int, v), o, fd::kWave)));
  return v;
}

// bf16 rows [M][cols] to integers.  A team holds a row in registers between its maximum and its integers: lane t takes the 8
// columns at 8 * (t + LANES * j), j < VEC.  Bound by HBM: 3 bytes a value; 9828 x 6144 34.8 us (5.2 TB/s), 943488 x 64 51, where one wave
// a row took 161.
template <int VEC, int LANES>
__global__ __launch_bounds__(team_threads<LANES>()) void int_rows_kernel(const uint16_t* __restrict__ x, int n_rows, int cols,
                                                                       const int32_t* __restrict__ m_dev, uint8_t* __restrict__ q,
                                                                       float* __restrict__ scale) {
  constexpr int TEAMS = team_threads<LANES>() / LANES, WAVES = (LANES + 63) / 64;
  __shared__ uint32_t part[2][WAVES];
  const int M = m_dev ? min(*m_dev, n_rows) : n_rows;
  const int wave = threadIdx.x >> 6, t = threadIdx.x % LANES;
  int odd = 0;
  for (int row = first_team<LANES>(); row < M; row += gridDim.x * TEAMS, odd ^= 1) {
    const size_t at = static_cast<size_t>(row) * cols;
    uint4 x8[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
      x8[j] = c < cols ? *reinterpret_cast<const uint4*>(x + at + c) : make_uint4(0, 0, 0, 0);
    }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float v[8];
      fd::unpack_bf8(x8[j], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, fd::mag_bits(v[e]));
    }
    top = over_lanes<LANES>(top, [](uint32_t a, uint32_t b) { return max(a, b); });
    if constexpr (WAVES > 1) {   // two sets: a wave may be a row ahead of one that has yet to read
      if ((threadIdx.x & 63) == 0) part[odd][wave] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = max(top, part[odd][w]);
    }
    const fd::IntScale s = fd::int_scale(top);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
      float v[8];
      fd::unpack_bf8(x8[j], v);
      if (c < cols) *reinterpret_cast<uint2*>(q + at + c) = fd::pack_ints(v, s.up);
    }
    if (t == 0) scale[row] = s.scale;
  }
}

enum { kNone, kBf16, kCodes, kInts };

// For row i of request b, with sums in fp32:
//   r = y / sqrt(mean(y^2) + eps) * post_weight;  h = residual * h + gate_b * r              (only with y)
//   a = h / sqrt(mean(h^2) + eps) * weight * (1 + scale_b) + shift_b                         (only with a result)
// A team of LANES lanes (16, 32 or whole waves) takes a run of rows, lane t the 8 columns at 8 * (t + LANES * j), j < VEC, and
// keeps a request's factors of a value (gate * post_weight, weight * (1 + scale), shift) in registers while the request stays;
// the next row is on its way while one is summed.  Bound by HBM: 4 bytes of h read and 4 written, 2 of y, 1 or 2 of the result
// per value; 8937 x 1536 with y to codes 27 us alone, 32 among other calls (4.7 TB/s), to integers 29, h alone 23.
template <int VEC, int LANES, int OUT>
__global__ __launch_bounds__(team_threads<LANES>()) void norm_residual_kernel(fdh::ResidualArgs g) {
  constexpr int TEAMS = team_threads<LANES>() / LANES, WAVES = (LANES + 63) / 64;
  __shared__ float part[2][3][WAVES];
  const int wave = threadIdx.x >> 6, t = threadIdx.x % LANES;
  const int D = g.D, M = min(*g.m, g.n_rows), ld = fd::scale_stride(D);
  const int team = first_team<LANES>(), teams = gridDim.x * TEAMS;
  const int run = (M + teams - 1) / teams, first = min(static_cast<long long>(team) * run, static_cast<long long>(M)), end = min(first + run, M);
  if (first >= end) return;   // the whole team together
  float gain[VEC][8], bias[VEC][8], gate[VEC][8];
  auto load8 = [&](const float* p, float (&v)[8]) {
    const float4 lo = *reinterpret_cast<const float4*>(p), hi = *reinterpret_cast<const float4*>(p + 4);
    v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
    v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
  };
  auto request = [&](int b) {
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
      float w[8];
      if (g.y) {
        if (g.gate) load8(g.gate + mod + c, gate[j]);
        if (g.post_weight) {
          load8(g.post_weight + c, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) gate[j][e] *= w[e];
        }
      }
      if constexpr (OUT != kNone) {
        if (g.scale) {
          load8(g.scale + mod + c, gain[j]);
#pragma unroll
          for (int e = 0; e < 8; ++e) gain[j][e] += 1.f;
        }
        if (g.weight) {
          load8(g.weight + c, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) gain[j][e] *= w[e];
        }
        if (g.shift) load8(g.shift + mod + c, bias[j]);
      }
    }
  };
  struct Row { float v[VEC][8]; uint4 y[VEC]; };
  auto fetch = [&](int row, Row& x) {   // a row's values, zeros past its end
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = 8 * (t + LANES * j);
      x.y[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[j][e] = 0.f;
      if (c >= D) continue;
      load8(g.h + static_cast<size_t>(row) * D + c, x.v[j]);
      if (g.y) x.y[j] = *reinterpret_cast<const uint4*>(g.y + static_cast<size_t>(row) * D + c);
    }
  };
  // The sum over the row's lanes, the same in all of them: over the lanes of a wave, then over the waves' sums in order.  Set `at`
  // of this row's parity is not written again before every wave has passed the barrier of the row after.
  auto row_sum = [&](float s, int row, int at) {
    s = over_lanes<LANES>(s, [](float a, float b) { return a + b; });
    if constexpr (WAVES > 1) {
      float* p = part[row & 1][at];
      if ((threadIdx.x & 63) == 0) p[wave] = s;
      __syncthreads();
      if constexpr (WAVES == 2) s = p[0] + p[1];
      else if constexpr (WAVES == 3) s = (p[0] + p[1]) + p[2];
      else if constexpr (WAVES == 4) s = (p[0] + p[1]) + (p[2] + p[3]);
      else s = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    }
    return s;
  };
  int b = g.n_req == 1 ? 0 : fd::row_request(g.cu_q, g.n_req, first);
  int b_end = g.n_req == 1 ? M : g.cu_q[b + 1];   // rows of the request
  Row cur, next;
  fetch(first, cur);
  request(b);
  for (int row = first; row < end; ++row) {
    if (row >= b_end && g.n_req > 1) {
      b = fd::row_request(g.cu_q, g.n_req, row);
      b_end = g.cu_q[b + 1];
      request(b);
    }
    if (row + 1 < end) fetch(row + 1, next);   // on its way while this row is summed and rounded
    float a[VEC][8];
    if (g.y) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float y8[8];
        fd::unpack_bf8(cur.y[j], y8);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += y8[e] * y8[e];
      }
      const float r = 1.0f / sqrtf(row_sum(sum, row, 0) / static_cast<float>(D) + g.eps);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int c = 8 * (t + LANES * j);
        float y8[8];
        fd::unpack_bf8(cur.y[j], y8);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[j][e] = g.residual * cur.v[j][e] + gate[j][e] * (y8[e] * r);
        if (c < D) {
          float* h = g.h + static_cast<size_t>(row) * D + c;
          *reinterpret_cast<float4*>(h) = make_float4(a[j][0], a[j][1], a[j][2], a[j][3]);
          *reinterpret_cast<float4*>(h + 4) = make_float4(a[j][4], a[j][5], a[j][6], a[j][7]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) a[j][e] = cur.v[j][e];
    }
    if constexpr (OUT != kNone) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < VEC; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += 8 * (t + LANES * j) < D ? a[j][e] * a[j][e] : 0.f;   // past the end y r may be NaN
      const float r = 1.0f / sqrtf(row_sum(sum, row, 1) / static_cast<float>(D) + g.eps);
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < VEC; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          a[j][e] = 8 * (t + LANES * j) < D ? a[j][e] * r * gain[j][e] + bias[j][e] : 0.f;   // zeros past the end, whatever r is
          if constexpr (OUT == kInts) top = max(top, fd::mag_bits(a[j][e]));
        }
      fd::IntScale s = {};
      if constexpr (OUT == kInts) {
        top = over_lanes<LANES>(top, [](uint32_t a, uint32_t b) { return max(a, b); });
        if constexpr (WAVES > 1) {
          float* p = part[row & 1][2];
          if ((threadIdx.x & 63) == 0) p[wave] = __uint_as_float(top);
          __syncthreads();
#pragma unroll
          for (int w = 0; w < WAVES; ++w) top = max(top, __float_as_uint(p[w]));
        }
        s = fd::int_scale(top);
        if (t == 0) g.row_scale[row] = s.scale;
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int c = 8 * (t + LANES * j);
        const size_t at = static_cast<size_t>(row) * D + c;
        if constexpr (OUT == kCodes) {
          uint2 codes;
          const uint32_t sb = fd::quant_lane8(a[j], codes);
          if (c < D) {
            *reinterpret_cast<uint2*>(g.a8 + at) = codes;
            if ((t & 15) == 0) g.code_scale[static_cast<size_t>(row) * ld + c / fd::kScaleBlock] = static_cast<uint8_t>(sb);
          }
        } else if constexpr (OUT == kInts) {
          if (c < D) *reinterpret_cast<uint2*>(g.a8 + at) = fd::pack_ints(a[j], s.up);
        } else if (c < D) {
          *reinterpret_cast<uint4*>(g.a_bf16 + at) = make_uint4(fd::pack_bf2(a[j][0], a[j][1]), fd::pack_bf2(a[j][2], a[j][3]),
                                                                fd::pack_bf2(a[j][4], a[j][5]), fd::pack_bf2(a[j][6], a[j][7]));
        }
      }
    }
    cur = next;
  }
}

}  // namespace

namespace fdh {

hipError_t launch_int_rows(const uint16_t* x, int n_rows, int cols, const int32_t* m, uint8_t* q, float* scale, hipStream_t s) {
  using std::integral_constant;
  auto run = [&](auto vec, auto lanes) {
    constexpr int VEC = decltype(vec)::value, LANES = decltype(lanes)::value, TEAMS = team_threads<LANES>() / LANES;
    const int groups = (n_rows + TEAMS - 1) / TEAMS, most = 16 * num_cus();
    int_rows_kernel<VEC, LANES><<<groups < most ? groups : most, team_threads<LANES>(), 0, s>>>(x, n_rows, cols, m, q, scale);
  };
  // Teams by width.  Some 60 million values, us, these and the fastest of 16 to 1024 lanes with 8 to 64 columns each: up to 128
  // columns these (64 columns 51, 128 34.6; on 32 lanes 49), 208 columns 37.3 and 35.7 (16 lanes of 16), 512 36.1 and 33.8 (16 of 64), 768 35.2 and
  // 33.9 (16 of 64), 1024 34.6 and 33.9 (32 of 64; three waves of 8 would be 36), 1088 46.0 and 33.8 (32 of 64), 1536 37.7 and 34.0 (32 of
  // 64), 2048 36 and 33.8 (64 of 64), 4096 34.7 and 34.3 (64 of 64), 6144 34.6 and 34.1 (512 of 32), 8192 34.3 and 33.2 (256 of 64), 12288 47.7 and
  // 33.5 (512 of 32), 16384 44.4 and 34.2 (1024 of 16), 32768 41.5 and 37.1 (512 of 64).  1021 rows take the same 6.3 to 6.6 with any, up to 8192 columns.
  const integral_constant<int, 1> one{};
  const integral_constant<int, 2> two{};
  const integral_constant<int, 4> four{};
  const integral_constant<int, 192> three_waves{};
  const integral_constant<int, 256> four_waves{};
  const integral_constant<int, 1024> widest{};
  if (cols <= 128) run(one, integral_constant<int, 16>{});
  else if (cols <= 256) run(one, integral_constant<int, 32>{});
  else if (cols <= 512) run(one, integral_constant<int, 64>{});
  else if (cols <= 1024) run(two, integral_constant<int, 64>{});
  else if (cols <= 1536) run(one, three_waves);
  else if (cols <= 2048) run(one, four_waves);
  else if (cols <= 4096) run(two, four_waves);
  else if (cols <= 8192) run(four, four_waves);
  else if (cols <= 32768) run(four, widest);
  else run(integral_constant<int, 8>{}, widest);
  return hipGetLastError();
}

hipError_t launch_norm_residual(const ResidualArgs& g, hipStream_t s) {
  using std::integral_constant;
  auto out = [&](auto kind) {
    auto run = [&](auto vec, auto lanes) {
      constexpr int VEC = decltype(vec)::value, LANES = decltype(lanes)::value, TEAMS = team_threads<LANES>() / LANES, WAVES = team_threads<LANES>() / 64, OUT = decltype(kind)::value;
      const int most = (WAVES == 3 ? 6 : 16 / WAVES) * num_cus(), groups = (g.n_rows + TEAMS - 1) / TEAMS;
      norm_residual_kernel<VEC, LANES, OUT><<<groups < most ? groups : most, team_threads<LANES>(), 0, s>>>(g);
    };
    // eight columns a lane, up to eight waves; as many workgroups as are resident, whose runs are read with the
    // next row on its way.  13.7 million values with y to bf16, us, these and the next best of 16 to 512 lanes with 8 to 24 columns
    // each: 128 columns 34.5 and 42.0, 256 34.4 and 37.1, 512 35.5 and 41.8, 1024 33.9 and 35.9 (192 lanes; 64 of 16 columns 40.0), 1536 34.2 and
    // 36.1, 2048 34.5 and 38.1, 4096 34.2 and 39.3, 8192 43.3 and 44.0; another is ahead at 640 (40.5 and 40.1, 32 lanes of 24),
    // 2560 (39.3 and 39.1, 128 of 24) and 6144 (44.9 and 40.4, 256 of 24); to integers in the same order
    const integral_constant<int, 1> one{};
    const integral_constant<int, 512> widest{};
    if (g.D <= 128) run(one, integral_constant<int, 16>{});
    else if (g.D <= 256) run(one, integral_constant<int, 32>{});
    else if (g.D <= 512) run(one, integral_constant<int, 64>{});
    else if (g.D <= 1024) run(one, integral_constant<int, 128>{});
    else if (g.D <= 1536) run(one, integral_constant<int, 192>{});
    else if (g.D <= 2048) run(one, integral_constant<int, 256>{});
    else if (g.D <= 4096) run(one, widest);
    else if (g.D <= 8192) run(integral_constant<int, 2>{}, widest);
    else run(integral_constant<int, 3>{}, widest);
  };
  if (g.a_bf16) out(integral_constant<int, kBf16>{});
  else if (g.code_scale) out(integral_constant<int, kCodes>{});
  else if (g.row_scale) out(integral_constant<int, kInts>{});
  else out(integral_constant<int, kNone>{});
  return hipGetLastError();
}

}  // namespace fdh
