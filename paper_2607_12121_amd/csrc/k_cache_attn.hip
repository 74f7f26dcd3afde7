// Attention of the active rows over every token of their request, keys and values from an 8-bit cache: e4m3 codes
// with a power-of-two scale per token and key head.  Codes times scales are bf16 values without a rounding, so both
// contractions run on v_mfma_f32_32x32x16_bf16 as for a bf16 cache; fp32 online softmax, base 2.
//
// The query heads that share a key head are rows of one problem: row r of a request under key head kh is query
// r / group, head kh * group + r % group.  An item is (key head, 256 of these rows), eight waves of 32 rows.
#include "fd_attn_sched.h"
#include "fd_scaled.h"

namespace {

constexpr int KB = fd::kKeyTile;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
using fd::bf16x2_t;
using fd::SchedTables;
typedef __attribute__((address_space(3))) void* lds_ptr_t;

template <int DH>
struct Cfg {
  static constexpr int WAVES = DH >= 64 ? 8 : 4, THREADS = 64 * WAVES, QB = 32 * WAVES;
  static constexpr int KCH = DH / 8;                 // 16-byte chunks of a row of bf16 values in LDS
  static constexpr int TILE = KB * KCH;              // chunks of a tile
  static constexpr int KS = DH / 16, DT = (DH + 31) / 32;
  static constexpr int PIECE = KB * DH / THREADS;    // codes of a tile that a thread brings: 4, 8 or 16 of a row
  // chunk c of key row r lies at c ^ fk(r) of K's tile and c ^ fv(r) of V's, so that the lanes that read together
  // meet different bank groups
  static FD_DEVICE int fk(int r) { return KCH >= 16 ? (r & 15) : KCH == 8 ? ((r >> 1) & 7) : ((r >> 3) & (KCH - 1)); }
  static FD_DEVICE int fv(int r) { return KCH >= 16 ? 4 * (r & 3) : KCH == 8 ? 4 * ((r >> 1) & 1) : 0; }
};

FD_DEVICE float half_max(float v) {   // over lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
FD_DEVICE float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Prefix tables over the requests: tiles of QB rows and their tile-steps (tiles x key tiles), of one key head.
// Requests without tokens have no tile-steps; returns whether one of them has rows.
template <int THREADS>
FD_DEVICE bool build_tables(SchedTables& t, const fdh::CacheAttnArgs& g, int group, int QB) {
  __shared__ int empty;
  const int tid = threadIdx.x;
  if (tid == 0) empty = 0;
  __syncthreads();
  for (int b = tid; b < g.n_req; b += THREADS) {
    const int rows = (g.cu_q[b + 1] - g.cu_q[b]) * group, keys = g.tok_off[b + 1] - g.tok_off[b];
    if (rows > 0 && keys <= 0) empty = 1;
    t.tpre[b] = rows > 0 && keys > 0 ? (rows + QB - 1) / QB : 0;
    t.wpre[b] = rows > 0 && keys > 0 ? static_cast<long long>(t.tpre[b]) * ((keys + KB - 1) / KB) : 0;
  }
  __syncthreads();
  if (tid == 0) {
    int tiles = 0;
    long long steps = 0;
    for (int b = 0; b < g.n_req; ++b) {
      const int nt = t.tpre[b];
      const long long nw = t.wpre[b];
      t.tpre[b] = tiles;
      t.wpre[b] = steps;
      tiles += nt;
      steps += nw;
    }
    t.tpre[g.n_req] = tiles;
    t.wpre[g.n_req] = steps;
  }
  __syncthreads();
  return empty != 0;
}

template <int DH>
__global__ __launch_bounds__(Cfg<DH>::THREADS) void cache_attn_kernel(fdh::CacheAttnArgs g) {
  using C = Cfg<DH>;
  constexpr int KS = C::KS, DT = C::DT, KCH = C::KCH;
  __shared__ uint4 kt[C::TILE], vt[C::TILE];
  __shared__ SchedTables tabs;
  const int group = g.heads / g.kv_heads, ldq = g.heads * DH, ldk = g.kv_heads * DH;
  const bool empty = build_tables<C::THREADS>(tabs, g, group, C::QB);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lg = lane >> 5;
  if (empty)   // a request without tokens: its rows are zeros
    for (int b = blockIdx.x; b < g.n_req; b += gridDim.x) {
      if (g.tok_off[b + 1] > g.tok_off[b]) continue;
      for (long long i = static_cast<long long>(g.cu_q[b]) * ldq / 8 + tid; i < static_cast<long long>(g.cu_q[b + 1]) * ldq / 8; i += C::THREADS)
        reinterpret_cast<uint4*>(g.o)[i] = make_uint4(0, 0, 0, 0);
    }
  using Sched = fd::AttnSched<C::QB, DH, true, false>;
  const Sched sch(&tabs, g.cu_q, g.tok_off, g.n_req, g.kv_heads, static_cast<int>(gridDim.x), 0);
  if (sch.work == 0) return;
  const float scale_log2 = g.scale * 1.4426950408889634f;
  const uint32_t k_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)&kt[0]));
  const uint32_t v_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)&vt[0]));
  // V^T operand, ds_read_b64_tr_b16: in a group of 16 lanes lane j addresses four d of key K0 + j / 4 and gets its own
  // d for the keys K0 .. K0 + 3
  const int grp = lane >> 4, jj = lane & 15, tr_key = 4 * lg + (jj >> 2), tr_d = 16 * (grp & 1) + 4 * (jj & 3);
  const bool tr_live = DH >= 32 || (grp & 1) == 0;

  const int w = sch.share(static_cast<int>(blockIdx.x));
  long long p = sch.bound(w);
  const long long p_end = sch.bound(w + 1);
  while (p < p_end) {
    long long i_start;
    int nkv, head, b, first, tau;
    sch.locate(p, i_start, nkv, head, b, first, tau);
    const int q0 = g.cu_q[b], rows = (g.cu_q[b + 1] - q0) * group, k_beg = g.tok_off[b], k_end = g.tok_off[b + 1];
    const int r = (tau - first) * C::QB + 32 * wave + l32;   // this lane's row
    const bool live = r < rows;
    const size_t at = static_cast<size_t>(q0 + r / group) * ldq + static_cast<size_t>(head * group + r % group) * DH;
    bf16x8_t qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4_t t = {0, 0, 0, 0};
      if (live) t = *reinterpret_cast<const u32x4_t*>(g.q + at + ks * 16 + lg * 8);
      qf[ks] = __builtin_bit_cast(bf16x8_t, t);
    }
    f32x16_t o[DT] = {};
    float m_run = -INFINITY, l_run = 0.f;
    for (int kt0 = 0; kt0 < nkv; ++kt0) {
      const int key0 = k_beg + kt0 * KB;
      {   // the tile's codes as bf16 values to LDS; rows past the end repeat the last
        constexpr int PER_ROW = DH / C::PIECE;
        const int row = tid / PER_ROW, c0 = tid % PER_ROW * C::PIECE;
        const size_t tok = min(key0 + row, k_end - 1);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const uint8_t* src = (kv ? g.v : g.k) + tok * ldk + static_cast<size_t>(head) * DH + c0;
          const float sc = __uint_as_float(static_cast<uint32_t>((kv ? g.v_scale : g.k_scale)[static_cast<size_t>(head) * g.n_tokens + tok]) << 23);
          uint32_t codes[C::PIECE / 4], vals[C::PIECE / 2];
          __builtin_memcpy(codes, src, C::PIECE);
#pragma unroll
          for (int i = 0; i < C::PIECE / 4; ++i) {
            vals[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], sc, false));
            vals[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], sc, true));
          }
          char* dst = reinterpret_cast<char*>(kv ? vt : kt);
#pragma unroll
          for (int i = 0; i < C::PIECE; i += 4) {
            const int c = (c0 + i) / 8;
            *reinterpret_cast<uint2*>(dst + (row * KCH + (c ^ (kv ? C::fv(row) : C::fk(row)))) * 16 + (c0 + i) % 8 * 2) = make_uint2(vals[i / 2], vals[i / 2 + 1]);
          }
        }
      }
      __syncthreads();
      f32x16_t s[2] = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
          const int key = 32 * kh + l32;
          const bf16x8_t a = __builtin_bit_cast(bf16x8_t, kt[key * KCH + ((2 * ks + lg) ^ C::fk(key))]);
          s[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[ks], s[kh], 0, 0, 0);
        }
      const int lim = k_end - key0 - 4 * lg;
      float top = -INFINITY;
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if (32 * kh + 8 * (e >> 2) + (e & 3) >= lim) s[kh][e] = -INFINITY;
          top = __builtin_elementwise_maximum(top, s[kh][e]);
        }
      top = half_max(top) * scale_log2;
      const float m_new = top > m_run ? top : m_run, alpha = m_run == m_new ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      const float sub = m_new == -INFINITY ? 0.f : m_new;
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
      bf16x8_t pk[4];
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[st >> 1][8 * (st & 1) + e], scale_log2, -sub));
          pk[st][e] = static_cast<__bf16>(x);
          l_run += static_cast<float>(pk[st][e]);   // of the rounded values that the product takes
        }
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          short4_t lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
          if (tr_live) {
            const int c = (32 * d + tr_d) >> 3;
            const uint32_t a_lo = v_base + static_cast<uint32_t>(((16 * st + tr_key) * KCH + (c ^ C::fv(tr_key))) * 16 + (tr_d & 7) * 2);
            lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(uintptr_t)a_lo);
            hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(uintptr_t)(a_lo + 8 * KCH * 16));
          }
          const short lo_hi[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, lo_hi), pk[st], o[d], 0, 0, 0);
        }
      __syncthreads();
    }
    const float inv = 1.0f / half_sum(l_run);
    if (live)
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int d0 = 32 * d + 8 * r4 + 4 * lg;
          if (d0 < DH)
            *reinterpret_cast<uint2*>(g.o + at + d0) = make_uint2(fd::pack_bf2(o[d][4 * r4] * inv, o[d][4 * r4 + 1] * inv),
                                                                  fd::pack_bf2(o[d][4 * r4 + 2] * inv, o[d][4 * r4 + 3] * inv));
        }
    p += nkv;
  }
  (void)k_base;
}

}  // namespace

namespace fdh {

size_t cache_attention_scratch_bytes(int, int, int, int) { return 256; }

hipError_t launch_cache_attention(const CacheAttnArgs& g, hipStream_t s) {
  const int grid = (num_cus() + fd::kXcds - 1) / fd::kXcds * fd::kXcds;
  switch (g.dh) {
    case 16: cache_attn_kernel<16><<<grid, Cfg<16>::THREADS, 0, s>>>(g); break;
    case 64: cache_attn_kernel<64><<<grid, Cfg<64>::THREADS, 0, s>>>(g); break;
    default: cache_attn_kernel<128><<<grid, Cfg<128>::THREADS, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace fdh
