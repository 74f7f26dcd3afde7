// Rotary positions on several axes, on the active rows of a fused q | k | v product: pair j of axis
// a (of the axis' own section of the head) is turned by
//   angle = pos_a * step_a * theta_a^(-2j / dim_a),
// q goes to its rows, k and v to the cache rows of their tokens.  Bound by HBM: every value is read
// and written once, 4 bytes.
//
// One wave per row.  The angle is the same for every head, so lane p < dh / 2 forms the cosine and
// sine of pair p once per row, from the angle in turns: pos * (step theta^.. / 2 pi) in fp64, whose
// nearest integer is taken off before the rest, at most half a turn, is rounded to fp32 (an error of 2^-26 of a
// turn, and of |pos| 2^-52 from the product and its factor where theta >= 1 and the step is at most 1; in fp32 a
// position of 10^5 would be off by 2^-8 of a turn).  Pairs that turn more than half a turn per position come with
// their whole turns taken off in 64 bits of mantissa: |pos| 2^-58 of their turns per position.  Each
// lane then takes 8 consecutive values of a head at a time; 64 lanes are a whole number of heads, so
// a lane meets the same place in every head and keeps its cosines and sines in registers.  9828 rows of 36 heads of
// 128: 40 us (4.5 TB/s); 1664 rows of 40 heads of 64: 8, a chain of index, position, values and results.
#include "fd_scaled.h"

namespace {

enum { kInterleaved, kHalvesWide, kHalves };

// KIND kInterleaved: pairs (2j, 2j + 1); the lane holds both.  kHalves: pairs (j, j + dim / 2) of
// the axis' section; the partner is read again from the row (it is in the L1), 16 bytes at a time
// where every dim is a multiple of 16 (kHalvesWide), else value by value.
//
// CODES: k and v go to an 8-bit cache, straight from the fp32 results: the dh / 8 lanes of a head agree on its scale.
template <int KIND, bool CODES>
__global__ __launch_bounds__(256) void rope_kernel(fdh::RopeArgs g, int row0) {
  __shared__ float2 turn[4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int row = row0 + blockIdx.x * 4 + wave;
  if (row >= min(*g.m, g.n_rows)) return;   // no barrier follows: each wave reads its own table
  const int tok = g.idx ? g.idx[row] : row;
  const int dh = g.dh;
  if (lane < g.pairs) {
    int axis = 0, first = 0;
    while (lane >= first + g.dim[axis] / 2) first += g.dim[axis++] / 2;
    const double turns = static_cast<double>(g.coord[static_cast<size_t>(tok) * g.n_axes + axis]) * g.turns[lane];
    float2 cs;
    if constexpr (CODES) {   // rounded once: a code near a tie goes the way of the exact angle's as often as fp32 lets it
      double c, n;
      sincospi(2.0 * (turns - rint(turns)), &n, &c);
      cs = make_float2(static_cast<float>(c), static_cast<float>(n));
    } else {
      const float rest = static_cast<float>(turns - rint(turns));
      sincospif(2.f * rest, &cs.y, &cs.x);
    }
    turn[wave][lane] = cs;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // this lane's place in every head, its pairs, and where its partners are
  const int e0 = (8 * lane) % dh;
  float c[8], n[8];
  int partner[8];
  bool turned[8];   // else past the axes: as it is, also where it is infinite
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int at = e0 + e;
    int pair, other;
    float sign;
    if constexpr (KIND == kInterleaved) {
      pair = at >> 1;
      other = at ^ 1;
      sign = (at & 1) ? 1.f : -1.f;
    } else {
      int axis = 0, first = 0;
      while (axis < g.n_axes && at >= first + g.dim[axis]) first += g.dim[axis++];
      const int half = axis < g.n_axes ? g.dim[axis] / 2 : 0;
      const bool upper = at - first >= half;
      pair = axis < g.n_axes ? first / 2 + (at - first) - (upper ? half : 0) : g.pairs;
      other = axis < g.n_axes ? (upper ? at - half : at + half) : at;
      sign = upper ? 1.f : -1.f;
    }
    turned[e] = pair < g.pairs;
    const float2 cs = turn[wave][turned[e] ? pair : 0];
    c[e] = cs.x;
    n[e] = sign * cs.y;
    partner[e] = other - at;
  }
  const int qk8 = (g.hq + g.hk) * dh / 8, q8 = g.hq * dh / 8, k8 = g.hk * dh / 8;
  const uint16_t* src = g.qkv + static_cast<size_t>(row) * (g.hq + 2 * g.hk) * dh;
  uint16_t* q = g.q + static_cast<size_t>(row) * g.hq * dh;
  uint16_t* k = g.k + static_cast<size_t>(tok) * g.hk * dh;
  uint16_t* v = g.v + static_cast<size_t>(tok) * g.hk * dh;
  // values 8 i .. 8 i + 7 of the token's row of a cache
  auto put_codes = [&](const float (&o)[8], int i, uint8_t* cache, uint8_t* scale) {
    const int lanes = dh / 8;   // the lanes of a head run this together: 64 and the heads' first values are multiples of it
    uint2 codes;
    const uint32_t s = fd::quant_lanes8(o, lanes, codes);
    *reinterpret_cast<uint2*>(cache + static_cast<size_t>(tok) * g.hk * dh + 8 * i) = codes;
    if (i % lanes == 0) scale[static_cast<size_t>(i / lanes) * g.n_tokens + tok] = static_cast<uint8_t>(s);
  };
  for (int i = lane; i < qk8; i += 64) {
    float x[8], y[8], o[8];
    fd::unpack_bf8(*reinterpret_cast<const uint4*>(src + 8 * i), x);
    if constexpr (KIND == kInterleaved) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
    } else if constexpr (KIND == kHalvesWide) {
      fd::unpack_bf8(*reinterpret_cast<const uint4*>(src + 8 * i + partner[0]), y);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fd::bf2f(src[8 * i + e + partner[e]]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = turned[e] ? x[e] * c[e] + y[e] * n[e] : x[e];
    if (CODES && i >= q8) {
      put_codes(o, i - q8, g.k8, g.k_scale);
      continue;
    }
    const uint4 out = make_uint4(fd::pack_bf2(o[0], o[1]), fd::pack_bf2(o[2], o[3]), fd::pack_bf2(o[4], o[5]), fd::pack_bf2(o[6], o[7]));
    *reinterpret_cast<uint4*>(i < q8 ? q + 8 * i : k + 8 * (i - q8)) = out;
  }
  for (int i = lane; i < k8; i += 64) {
    const uint4 x = *reinterpret_cast<const uint4*>(src + 8 * (qk8 + i));
    if constexpr (CODES) {
      float o[8];
      fd::unpack_bf8(x, o);
      put_codes(o, i, g.v8, g.v_scale);
    } else {
      *reinterpret_cast<uint4*>(v + 8 * i) = x;
    }
  }
}

}  // namespace

namespace fdh {

namespace {
template <bool CODES>
hipError_t launch_to(const RopeArgs& g, bool halves, hipStream_t s) {
  bool wide = true;
  for (int a = 0; a < g.n_axes; ++a) wide = wide && g.dim[a] % 16 == 0;
  // a launch has fewer than 2^32 threads, 64 of them a row
  constexpr int kRows = 1 << 25;
  for (int row0 = 0; row0 < g.n_rows; row0 += kRows) {
    const int rows = g.n_rows - row0 < kRows ? g.n_rows - row0 : kRows, grid = (rows + 3) / 4;
    if (!halves) rope_kernel<kInterleaved, CODES><<<grid, 256, 0, s>>>(g, row0);
    else if (wide) rope_kernel<kHalvesWide, CODES><<<grid, 256, 0, s>>>(g, row0);
    else rope_kernel<kHalves, CODES><<<grid, 256, 0, s>>>(g, row0);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}
}  // namespace

hipError_t launch_rope(const RopeArgs& g, bool halves, hipStream_t s) {
  return g.k8 ? launch_to<true>(g, halves, s) : launch_to<false>(g, halves, s);
}

}  // namespace fdh
