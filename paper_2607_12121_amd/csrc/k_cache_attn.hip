// Attention of the active rows over every token of their request, keys and values from an 8-bit cache: e4m3 codes
// with a power-of-two scale per token and key head.  Codes times scales are bf16 values without a rounding (but for scales of
// 2^-126 and 2^-125, whose least codes are below bf16's least value, 2^-133), so both contractions run on
// v_mfma_f32_32x32x16_bf16 as for a bf16 cache; fp32 online softmax, base 2.
//
// The query heads that share a key head are rows of one problem: row r of a request under key head kh is query
// r / group, head kh * group + r % group.  A wave computes S^T = K Q^T (64 keys x 32 rows), so that a lane owns one
// row: its maximum needs one exchange between the half-waves per tile, its sum none until the end, and S^T feeds
// O^T = V^T P^T as the second operand.
//
// Two ways through the work, chosen by the row counts on the device (fd_cache_sched.h):
//
// - Tiles: an item is (key head, 256 rows), a wave per 32 rows (head dim 16: 128 rows, four waves).  The key tile's
//   codes go to LDS as bf16 values, converted once for all waves (8 conversions a wave and tile; fragments converted
//   by the wave that uses them would take 128).  Software pipeline: the iteration of key tile t runs the matrix
//   instructions of S(t + 1) and of O += V P(t) between the element pairs of tile t's softmax, with the codes of K's
//   tile t + 2 and V's t + 1 on their way to registers.
// - Few rows: an item is (key head, 32 rows), every wave has key tiles of its own, 64 keys at a time, K straight
//   from memory into fragments, V through a tile of the wave's own in LDS that transposes it; the waves' results
//   meet in LDS.  What bounds it is the cache's bytes: 128 KB are on their way to a CU.
//
// Schedule: the key steps of all items, head-major, are one range cut into equal shares, one per workgroup.  Pieces of
// a cut item go to scratch as O / sum with their maximum and sum, and a second kernel joins them in key order (the same
// bits for the same sizes); no workgroup waits for another.
//
// Measured, both kernels: 9828 rows of 12 heads of 128 over 32760 keys 1.72 to 1.80 ms (1.1 PFLOP/s; matrix pipes 53% busy at 1.9
// GHz: power), 8937 rows of 8 requests, 24 heads of 64 on 8 key heads, 249 us (0.77 PFLOP/s; matrix pipes 35%, vector
// instructions 58%: two exponentials a pair of scores and their packing take as long as the products), 4000 rows of 64 heads of 16 over
// 8000 keys 475 us (0.28 PFLOP/s; vector instructions 72%, matrix pipes 17%), one row of 12 heads over
// 32760 keys 34 us (101 MB: 16 us of reads at 6.5 TB/s behind 5 us of schedule and first loads, 4 us of joining the waves, 5 us of
// joining the pieces).
#include <type_traits>

#include "fd_cache_sched.h"
#include "fd_scaled.h"

namespace {

constexpr int KB = fd::kKeyTile;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef short short4_t __attribute__((ext_vector_type(4)));
using fd::bf16x2_t;
using fd::f32x2_t;
using fd::SchedTables;
typedef __attribute__((address_space(3))) void* lds_ptr_t;

template <int DH>
struct Cfg {
  static constexpr int WAVES = DH >= 64 ? 8 : 4, THREADS = 64 * WAVES;
  static constexpr int QB = fd::cache_tile_rows(DH);   // rows of an item, in tiles and of few rows
  static constexpr int QF = fd::kFewRows;
  static constexpr int KCH = DH / 8;                   // 16-byte chunks of a key row of bf16 values in LDS
  static constexpr int TILE = KB * KCH;                // chunks of a tile
  static constexpr int KS = DH / 16, DT = (DH + 31) / 32;
  static constexpr int PIECE = KB * DH / THREADS;      // codes of a tile that a thread brings: 4, 8 or 16 of a row
  static constexpr int FEW_KEYS = fd::cache_few_keys(DH);   // keys of a step of few rows
  static_assert(FEW_KEYS == KB * WAVES, "a tile a wave");
  static constexpr int VHALVES = DH >= 128 ? 2 : 1;    // parts in which V's values of 64 keys pass a wave's LDS
  static constexpr int FEW_WAVE_BYTES = KB * DH + TILE * 16 / VHALVES;   // K's codes and V's values
  static constexpr int AHEAD = DH >= 128 ? 2 : 3;      // operand reads ahead of their matrix instructions (registers)
  static constexpr int E = DT * 16 + 2;                // floats of a thread in a tile's piece
  static constexpr int FEW_SLOT = 32 * (DH + 2);       // floats of a piece of few rows
  static constexpr int JOIN_PARTS = DT * 2;            // workgroups that join an item: two quads of a thread each
  static_assert(QB == 32 * WAVES, "a wave per 32 rows");
  // chunk c of key row r lies at c ^ fk(r) of K's tile and c ^ fv(r) of V's, so that the lanes that read together
  // meet different bank groups.  fk(r + 32) = fk(r), fv(r + 8) = fv(r).
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
FD_DEVICE float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
// This wave's LDS writes are done; then the barrier.
FD_DEVICE void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
FD_DEVICE float scale_of(uint32_t s) { return __uint_as_float(s << 23); }
// Four codes times a scale as two pairs of bf16 (exact).
FD_DEVICE uint2 values4(uint32_t codes, float scale) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)));
}
FD_DEVICE bf16x8_t lds_chunk(uint32_t addr) {
  return __builtin_bit_cast(bf16x8_t, *(__attribute__((address_space(3))) const u32x4_t*)(uintptr_t)addr);
}
// Eight keys of one d of V's tile: ds_read_b64_tr_b16 twice, the second 8 keys on.
FD_DEVICE u32x4_t lds_transposed(uint32_t addr, uint32_t eight_keys) {
  const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(uintptr_t)addr);
  const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(uintptr_t)(addr + eight_keys));
  const short v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(u32x4_t, v);
}

// Requests with rows and keys: their items of QB rows and key steps.
struct Lengths {
  const fdh::CacheAttnArgs* g;
  int group;
  FD_DEVICE int rows(int b) const { return (g->cu_q[b + 1] - g->cu_q[b]) * group; }
  FD_DEVICE int keys(int b) const { return g->tok_off[b + 1] - g->tok_off[b]; }
  FD_DEVICE int items(int b, int qb) const {
    const int r = rows(b);
    return r > 0 && keys(b) > 0 ? (r + qb - 1) / qb : 0;
  }
};

// The schedule's tables, and the requests' first rows and tokens: from LDS they are there 1 us before they would be from memory.
struct Tables : SchedTables {
  int q0[fd::kMaxSchedRequests + 1], k0[fd::kMaxSchedRequests + 1];
};
// What the schedule is built from, by every workgroup alike: the way, and the prefix tables of its items and key steps over the
// requests.  Up to a wave's lanes of requests, each wave reads them at once and counts in scalar registers (1024 rows of
// one request 32.7 -> 31.3 us); more: each thread takes a run of requests, the runs' sums are scanned over the waves and the workgroup.
struct Way { bool few, empty; int extra; };   // empty: a request has rows but no keys; extra: key steps that an item's start counts for
template <int DH>
FD_DEVICE Way build_tables(Tables& t, const fdh::CacheAttnArgs& g, int group) {
  using C = Cfg<DH>;
  constexpr int NW = C::WAVES;
  __shared__ int s_items[2][NW], s_empty[NW];
  __shared__ long long s_steps[NW];
  const Lengths len{&g, group};
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (g.n_req <= 64) {
    const bool mine = lane < g.n_req;
    const int at = mine ? lane : 0, q0 = g.cu_q[at], q1 = g.cu_q[at + 1], k0 = g.tok_off[at], k1 = g.tok_off[at + 1];
    const int rows = mine ? (q1 - q0) * group : 0, keys = mine ? k1 - k0 : 0;
    const bool has = rows > 0 && keys > 0;
    const int few = has ? (rows + C::QF - 1) / C::QF : 0, tiles = has ? (rows + C::QB - 1) / C::QB : 0;
    int all_few = 0, all_tiles = 0;
    for (int b = 0; b < g.n_req; ++b) {
      all_few += __builtin_amdgcn_readlane(few, b);
      all_tiles += __builtin_amdgcn_readlane(tiles, b);
    }
    const bool is_few = fd::cache_few_rows(DH, all_few, all_tiles);
    const Way way{is_few, __any(rows > 0 && keys <= 0) != 0, is_few ? 0 : fd::cache_item_steps(static_cast<long long>(all_tiles) * g.kv_heads, static_cast<int>(gridDim.x))};
    const int kb = is_few ? C::FEW_KEYS : KB, items = is_few ? few : tiles, steps = has ? (keys + kb - 1) / kb + way.extra : 0;
    int pi = 0, mine_i = 0;
    long long ps = 0, mine_s = 0;
    for (int b = 0; b < g.n_req; ++b) {
      if (b == lane) {
        mine_i = pi;
        mine_s = ps;
      }
      const int n = __builtin_amdgcn_readlane(items, b);
      pi += n;
      ps += static_cast<long long>(n) * __builtin_amdgcn_readlane(steps, b);
    }
    if (wave == 0 && mine) {
      t.tpre[lane] = mine_i;
      t.wpre[lane] = mine_s;
      t.q0[lane] = q0;
      t.k0[lane] = k0;
      if (lane == g.n_req - 1) {
        t.tpre[g.n_req] = pi;
        t.wpre[g.n_req] = ps;
        t.q0[g.n_req] = q1;
        t.k0[g.n_req] = k1;
      }
    }
    __syncthreads();
    return way;
  }
  const int per = (g.n_req + C::THREADS - 1) / C::THREADS, b0 = min(tid * per, g.n_req), b1 = min(b0 + per, g.n_req);
  int few = 0, tiles = 0, empty = 0;
  for (int b = b0; b < b1; ++b) {
    few += len.items(b, C::QF);
    tiles += len.items(b, C::QB);
    empty |= len.rows(b) > 0 && len.keys(b) <= 0;
  }
  few = fd::wave_sum(few);
  tiles = fd::wave_sum(tiles);
  empty = __any(empty);
  if (lane == 0) {
    s_items[0][wave] = few;
    s_items[1][wave] = tiles;
    s_empty[wave] = empty;
  }
  __syncthreads();
  few = tiles = empty = 0;
  for (int w = 0; w < NW; ++w) {
    few += s_items[0][w];
    tiles += s_items[1][w];
    empty |= s_empty[w];
  }
  const bool is_few = fd::cache_few_rows(DH, few, tiles);
  const Way way{is_few, empty != 0, is_few ? 0 : fd::cache_item_steps(static_cast<long long>(tiles) * g.kv_heads, static_cast<int>(gridDim.x))};
  const int qb = way.few ? C::QF : C::QB, kb = way.few ? C::FEW_KEYS : KB, more = way.extra;
  int it = 0;
  long long st = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = len.items(b, qb);
    it += n;
    st += static_cast<long long>(n) * ((len.keys(b) + kb - 1) / kb + more);
  }
  int it_in = it;
  long long st_in = st;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(it_in, o, 64);
    const long long y = __shfl_up(st_in, o, 64);
    if (lane >= o) {
      it_in += x;
      st_in += y;
    }
  }
  __syncthreads();
  if (lane == 63) {
    s_items[0][wave] = it_in;
    s_steps[wave] = st_in;
  }
  __syncthreads();
  int pi = it_in - it;
  long long ps = st_in - st;
  for (int w = 0; w < wave; ++w) {
    pi += s_items[0][w];
    ps += s_steps[w];
  }
  for (int b = b0; b < b1; ++b) {
    t.tpre[b] = pi;
    t.wpre[b] = ps;
    t.q0[b] = g.cu_q[b];
    t.k0[b] = g.tok_off[b];
    const int n = len.items(b, qb);
    pi += n;
    ps += static_cast<long long>(n) * ((len.keys(b) + kb - 1) / kb + more);
  }
  if (b0 < b1 && b1 == g.n_req) {
    t.tpre[g.n_req] = pi;
    t.wpre[g.n_req] = ps;
    t.q0[g.n_req] = g.cu_q[g.n_req];
    t.k0[g.n_req] = g.tok_off[g.n_req];
  }
  __syncthreads();
  return way;
}

template <int DH>
using Sched = fd::CacheSched<DH>;
template <int DH, bool FEW_ONLY>   // FEW_ONLY: known to be so
FD_DEVICE Sched<DH> schedule(const SchedTables* t, const fdh::CacheAttnArgs& g, const Way& way) {
  return Sched<DH>(t, g.cu_q, g.tok_off, g.n_req, g.kv_heads, static_cast<int>(gridDim.x), (g.max_req_tokens + KB - 1) / KB,
                   FEW_ONLY || fd::uniform(static_cast<int>(way.few)) != 0, g.may_cut, FEW_ONLY ? 0 : fd::uniform(way.extra));
}

// The cut item whose first piece a workgroup has, for the join; no pieces: none.  Every workgroup writes its own.
struct CutItem { int pieces, share, head, request, tile_few; };
FD_DEVICE CutItem* g_cut_items(const fdh::CacheAttnArgs& g) { return static_cast<CutItem*>(g.cut_items); }

// A request: its first query and rows under a key head, its first key and the one behind its last.
struct Request { int q0, rows, k_beg, k_end; };
// One lane's row of an item: where its query (and result) begins, and whether there is one.
struct RowAt { size_t at; bool live; };
template <int DH>
FD_DEVICE RowAt row_at(const fdh::CacheAttnArgs& g, int group, const Request& of, int head, int r) {
  const int query = group == 1 ? r : r / group;
  return {(static_cast<size_t>(of.q0 + query) * g.heads + static_cast<size_t>(head) * group + (r - query * group)) * DH, r < of.rows};
}

// This lane's part of O^T blocks as a bf16 row: register 4 r4 + e of block dt is d = 32 dt + 8 r4 + 4 lg + e.
template <int DH>
FD_DEVICE void store_o(uint16_t* row, int lg, const f32x16_t (&o)[Cfg<DH>::DT], float inv) {
#pragma unroll
  for (int d = 0; d < Cfg<DH>::DT; ++d)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d0 = 32 * d + 8 * r4 + 4 * lg;
      if (d0 >= DH) continue;
      *reinterpret_cast<uint2*>(row + d0) = make_uint2(fd::pack_bf2(o[d][4 * r4] * inv, o[d][4 * r4 + 1] * inv),
                                                       fd::pack_bf2(o[d][4 * r4 + 2] * inv, o[d][4 * r4 + 3] * inv));
    }
}

// The largest of a lane's 32 scores of a tile in eight steps of two, four independent chains; then of the row's.
struct TileMax {
  float mx[4];
  FD_DEVICE void first(const f32x16_t (&s)[2]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) mx[c] = __builtin_elementwise_maximum(s[c >> 1][8 * (c & 1)], s[c >> 1][8 * (c & 1) + 1]);
  }
  FD_DEVICE void next(const f32x16_t (&s)[2], int i) {   // i = 0 .. 11
    const int c = i & 3, r = 8 * (c & 1) + 2 + 2 * (i >> 2);
    mx[c] = max3(mx[c], s[c >> 1][r], s[c >> 1][r + 1]);
  }
  FD_DEVICE float row(float scale_log2) const {
    return half_max(__builtin_elementwise_maximum(__builtin_elementwise_maximum(mx[0], mx[1]), __builtin_elementwise_maximum(mx[2], mx[3]))) * scale_log2;
  }
};
// LIMIT: the scores of the lane's keys from `lim` on are not the request's.
template <bool LIMIT>
FD_DEVICE float tile_max(f32x16_t (&s)[2], int lim, float scale_log2) {
  if constexpr (LIMIT) {
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (32 * kh + 8 * (r >> 2) + (r & 3) >= lim) s[kh][r] = -INFINITY;
  }
  TileMax m;
  m.first(s);
#pragma unroll
  for (int i = 0; i < 12; ++i) m.next(s, i);
  return m.row(scale_log2);
}

// The running maximum of a row takes a tile's, and O and the sum are rescaled where it grew by more than 8 (P stays below 2^8;
// the softmax does not depend on what is subtracted).  Returns what to subtract.
template <int DH>
FD_DEVICE float take_max(float top, float& m_run, float& l_run, f32x16_t (&o)[Cfg<DH>::DT]) {
  const bool grow = top > m_run + 8.0f;
  const float m_new = grow ? top : m_run;
  if (__any(grow)) {
    const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.0f;
    l_run *= alpha;
#pragma unroll
    for (int d = 0; d < Cfg<DH>::DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
  }
  m_run = m_new;
  return m_new == -INFINITY ? 0.0f : m_new;   // no finite score yet: exp2(-inf) is zero, not NaN
}

// P = exp2(s scale - sub) in bf16, the second operand of O^T, and its sum: of the rounded values that the product takes.
FD_DEVICE void take_p(const f32x16_t (&s)[2], float scale_log2, float sub, bf16x8_t (&pk)[4], float& l_run) {
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int st = 0; st < 4; ++st)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const f32x2_t f = {__builtin_amdgcn_exp2f(fmaf(s[st >> 1][8 * (st & 1) + e], scale_log2, -sub)),
                         __builtin_amdgcn_exp2f(fmaf(s[st >> 1][8 * (st & 1) + e + 1], scale_log2, -sub))};
      const bf16x2_t pb = __builtin_convertvector(f, bf16x2_t);
      sum[(e >> 1) & 1] = __builtin_amdgcn_fdot2_f32_bf16(pb, bf16x2_t{(__bf16)1.0f, (__bf16)1.0f}, sum[(e >> 1) & 1], false);
      pk[st][e] = pb[0];
      pk[st][e + 1] = pb[1];
    }
  l_run += sum[0] + sum[1];
}

template <int DH>
struct Lane {   // addressing that does not depend on the work
  uint32_t k_off[Cfg<DH>::KS], v_off[Cfg<DH>::DT];   // byte offsets in a tile of this lane's fragments
  bool tr_live;                                      // d is below the head dim, else the operand's rows are zeros
  FD_DEVICE explicit Lane(int lane) {
    using C = Cfg<DH>;
    const int l32 = lane & 31, lg = lane >> 5, grp = lane >> 4, jj = lane & 15;
    // ds_read_b64_tr_b16: in a group of 16 lanes lane j addresses four d of key K0 + j / 4, and gets its own d of the
    // keys K0 .. K0 + 3
    const int tr_key = 4 * lg + (jj >> 2), tr_d = 16 * (grp & 1) + 4 * (jj & 3);
    tr_live = DH >= 32 || (grp & 1) == 0;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) k_off[ks] = static_cast<uint32_t>((l32 * C::KCH + ((2 * ks + lg) ^ C::fk(l32))) * 16);
#pragma unroll
    for (int d = 0; d < C::DT; ++d) {
      const int at = 32 * d + tr_d;
      v_off[d] = static_cast<uint32_t>((tr_key * C::KCH + ((at >> 3) ^ C::fv(tr_key))) * 16 + (at & 7) * 2);
    }
  }
  // V^T of 16-key step st, block d, of the tile at `tile`
  FD_DEVICE u32x4_t v_frag(uint32_t tile, int st, int d) const {
    u32x4_t v = {0, 0, 0, 0};
    if (tr_live) v = lds_transposed(tile + v_off[d] + static_cast<uint32_t>(16 * st * Cfg<DH>::KCH * 16), 8 * Cfg<DH>::KCH * 16);
    return v;
  }
};

// ---------------------------------------------------------------- tiles

// Key tiles [kt0, kt1) of query tile `tile` of a request under key head `head`, to the outputs or, of a cut item, to
// scratch slot `slot_no`.
template <int DH>
FD_DEVICE void tile_piece(const fdh::CacheAttnArgs& g, int group, float scale_log2, uint32_t lds, int head, int tile, const Request& of, int kt0,
                          int kt1, int slot_no) {
  using C = Cfg<DH>;
  constexpr int DT = C::DT, KS = C::KS, KCH = C::KCH;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lg = lane >> 5;
  const Lane<DH> ln(lane);
  const int k_beg = of.k_beg, k_end = of.k_end, nkt = kt1 - kt0, ldk = g.kv_heads * DH;
  const RowAt me = row_at<DH>(g, group, of, head, tile * C::QB + 32 * wave + l32);
  bf16x8_t qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    u32x4_t t = {0, 0, 0, 0};
    if (me.live) t = *reinterpret_cast<const u32x4_t*>(g.q + me.at + ks * 16 + lg * 8);
    qf[ks] = __builtin_bit_cast(bf16x8_t, t);
  }

  // a thread's codes of a tile: PIECE of row `row` from column c0 on; rows past the end repeat the last one
  constexpr int PER_ROW = DH / C::PIECE;
  const int row = tid / PER_ROW, c0 = tid % PER_ROW * C::PIECE;
  struct Codes { uint32_t c[C::PIECE / 4]; uint32_t scale; };
  const uint32_t off = static_cast<uint32_t>(row) * static_cast<uint32_t>(ldk) + static_cast<uint32_t>(c0);
  // Successive tiles of a cache: the next tile's place and its last row of the request, in scalar registers.  (Formed anew from the
  // tile's number, the addresses took 300 to 400 clocks of an iteration's 2700 at head dim 64.)
  struct Stream { const uint8_t* codes; const uint8_t* scale; int last, left; };
  auto stream = [&](const uint8_t* cache, const uint8_t* scale) {
    const int key0 = k_beg + kt0 * KB;
    return Stream{cache + static_cast<size_t>(key0) * ldk + static_cast<size_t>(head) * DH, scale + static_cast<size_t>(head) * g.n_tokens + key0,
                  k_end - 1 - key0, nkt};
  };
  // without a branch: the iteration stays one block, in which the compiler may order
  auto fetch_codes = [&](const Stream& from, Codes& x) {
    __builtin_memcpy(x.c, __builtin_assume_aligned(from.codes + (row <= from.last ? off : static_cast<uint32_t>(from.last) * static_cast<uint32_t>(ldk) + static_cast<uint32_t>(c0)), C::PIECE), C::PIECE);
  };
  auto fetch_scale = [&](Stream& from, Codes& x) {   // and on to the next tile; past the piece's last one that one again
    x.scale = from.scale[min(row, from.last)];
    const bool more = --from.left > 0;
    from.codes += more ? KB * ldk : 0;
    from.scale += more ? KB : 0;
    from.last -= more ? KB : 0;
  };
  auto fetch = [&](Stream& from) {
    Codes x;
    fetch_codes(from, x);
    fetch_scale(from, x);
    return x;
  };
  Stream from_k = stream(g.k, g.k_scale), from_v = stream(g.v, g.v_scale);
  const uint32_t put_k = static_cast<uint32_t>((row * KCH + ((c0 / 8) ^ C::fk(row))) * 16 + c0 % 8 * 2);
  const uint32_t put_v = static_cast<uint32_t>((row * KCH + ((c0 / 8) ^ C::fv(row))) * 16 + c0 % 8 * 2);
  auto put = [&](const Codes& x, uint32_t at) {   // as bf16 values to LDS
    const float s = scale_of(x.scale);
    if constexpr (C::PIECE == 4) {
      const uint2 v = values4(x.c[0], s);
      *(__attribute__((address_space(3))) uint64_t*)(uintptr_t)at = __builtin_bit_cast(uint64_t, v);
    } else {
#pragma unroll
      for (int i = 0; i < C::PIECE / 8; ++i) {
        const uint2 lo = values4(x.c[2 * i], s), hi = values4(x.c[2 * i + 1], s);
        // the piece's second chunk is the first one's neighbour: c0 / 8 is even
        *(__attribute__((address_space(3))) u32x4_t*)(uintptr_t)(at ^ (16u * i)) = u32x4_t{lo.x, lo.y, hi.x, hi.y};
      }
    }
  };
  // rings of two tiles each: K, then V
  auto k_tile = [&](int t) { return lds + static_cast<uint32_t>((t & 1) * C::TILE * 16); };
  auto v_tile = [&](int t) { return lds + static_cast<uint32_t>((2 + (t & 1)) * C::TILE * 16); };

  f32x16_t o[DT] = {};
  float m_run = -INFINITY, l_run = 0.f;
  bf16x8_t pk[4];
  float top = 0.f;   // the maximum of the next iteration's scores
  auto s_step = [&](uint32_t tile_at, f32x16_t (&s)[2], int ks) {
    const f32x16_t zero = {};
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) {
      const bf16x8_t a = lds_chunk(tile_at + ln.k_off[ks] + static_cast<uint32_t>(kh * 32 * KCH * 16));
      s[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[ks], ks == 0 ? zero : s[kh], 0, 0, 0);
    }
  };

  // Iteration t: S(t + 1), the softmax of tile t and O += V P(t).  At its barrier K(t + 1) and V(t) are in LDS and every
  // wave is done with K(t) and V(t - 1), whose places K(t + 2) and V(t + 1) take.
  auto body = [&](int t, f32x16_t (&cur)[2], f32x16_t (&nxt)[2]) {
    lds_barrier();
    const uint32_t kt_at = k_tile(t + 1), vt_at = v_tile(t);
    // jobs: one operand read feeding one matrix instruction; first S(t + 1), then O by quarters of P as they come; reads run
    // AH jobs ahead
    constexpr int NS = KS * 2, NJ = NS + DT * 4, AH = C::AHEAD < NJ ? C::AHEAD : NJ, PAIRS = 16, PER = (NJ + PAIRS - 1) / PAIRS;
    constexpr int S_DONE = (NS + PER - 1) / PER;   // the pair from which on S(t + 1) is complete
    const f32x16_t zero = {};
    auto read = [&](int j) -> u32x4_t {
      if (j < NS) return __builtin_bit_cast(u32x4_t, lds_chunk(kt_at + ln.k_off[j / 2] + static_cast<uint32_t>(j % 2 * 32 * KCH * 16)));
      return ln.v_frag(vt_at, (j - NS) / DT, (j - NS) % DT);
    };
    auto run = [&](int j, u32x4_t op) {
      const bf16x8_t a = __builtin_bit_cast(bf16x8_t, op);
      if (j < NS) nxt[j % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[j / 2], j < 2 ? zero : nxt[j % 2], 0, 0, 0);
      else o[(j - NS) % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pk[(j - NS) / DT], o[(j - NS) % DT], 0, 0, 0);
    };
    auto earliest = [&](int j) { return j < NS ? 0 : 4 * ((j - NS) / DT + 1); };   // pair behind which job j may run
    u32x4_t ops[AH];
#pragma unroll
    for (int j = 0; j < AH; ++j) ops[j] = read(j);
    const float sub = take_max<DH>(top, m_run, l_run, o);
    Codes ck, cv;   // K's tile t + 2 and V's t + 1
    TileMax nm;
    // P in three stages that overlap across pairs: exponentials of pair pp, scaled scores of pp + 1, packing and sum of pp - 1
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    int cursor = 0, compared = 0;
    auto next_job = [&] {
      run(cursor, ops[cursor % AH]);
      if (cursor + AH < NJ) ops[cursor % AH] = read(cursor + AH);
      ++cursor;
    };
    auto arg = [&](int pp, float (&x)[2]) {
      const int st = pp / 4, e = 2 * (pp % 4);
      x[0] = fmaf(cur[st / 2][(st % 2) * 8 + e], scale_log2, -sub);
      x[1] = fmaf(cur[st / 2][(st % 2) * 8 + e + 1], scale_log2, -sub);
    };
    auto pack = [&](int pp, float p0, float p1) {
      const int st = pp / 4, e = 2 * (pp % 4);
      const f32x2_t f = {p0, p1};
      const bf16x2_t pb = __builtin_convertvector(f, bf16x2_t);
      sum[pp % 4] = __builtin_amdgcn_fdot2_f32_bf16(pb, bf16x2_t{(__bf16)1.0f, (__bf16)1.0f}, sum[pp % 4], false);
      pk[st][e] = pb[0];
      pk[st][e + 1] = pb[1];
    };
    float x[2], p0 = 0.f, p1 = 0.f;
    arg(0, x);
#pragma unroll
    for (int pp = 0; pp < PAIRS; ++pp) {
      const float e0 = __builtin_amdgcn_exp2f(x[0]), e1 = __builtin_amdgcn_exp2f(x[1]);
      if (pp + 1 < PAIRS) arg(pp + 1, x);
      if (pp > 0) pack(pp - 1, p0, p1);
      p0 = e0;
      p1 = e1;
#pragma unroll
      for (int k = 0; k < PER; ++k)
        if (cursor < NJ && earliest(cursor) <= pp) next_job();
      // the loads apart from each other: all waves' at once wait for the address unit
      if (pp == 0) fetch_codes(from_k, ck);
      if (pp == 2) fetch_codes(from_v, cv);
      if (pp == 4) fetch_scale(from_k, ck);
      if (pp == 6) fetch_scale(from_v, cv);
      // the maximum of S(t + 1), two steps a pair
      if (pp == S_DONE + 1) nm.first(nxt);
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (pp > S_DONE + 1 && compared < 12) nm.next(nxt, compared++);
      __builtin_amdgcn_sched_barrier(0);
    }
    pack(PAIRS - 1, p0, p1);
#pragma unroll
    for (int k = 0; k < NJ; ++k)
      if (cursor < NJ) next_job();
#pragma unroll
    for (int k = 0; k < 12; ++k)
      if (compared < 12) nm.next(nxt, compared++);
    top = nm.row(scale_log2);
    put(ck, k_tile(t + 2) + put_k);
    put(cv, v_tile(t + 1) + put_v);
    l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    asm volatile("" : "+v"(l_run));   // here, and not beside the next iteration's work with P kept until then
  };
  auto tail = [&](int t, f32x16_t (&cur)[2]) {
    lds_barrier();
    const int lim = k_end - (k_beg + (kt0 + t) * KB) - 4 * lg;   // this lane's keys below it are the request's
    const float sub = take_max<DH>(tile_max<true>(cur, lim, scale_log2), m_run, l_run, o);
    take_p(cur, scale_log2, sub, pk, l_run);
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ln.v_frag(v_tile(t), st, d)), pk[st], o[d], 0, 0, 0);
  };
  {
    const Codes k0 = fetch(from_k), k1 = fetch(from_k), v0 = fetch(from_v);
    put(k0, k_tile(0) + put_k);
    put(k1, k_tile(1) + put_k);
    put(v0, v_tile(0) + put_v);
  }
  lds_barrier();
  f32x16_t sa[2], sb[2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) s_step(k_tile(0), sa, ks);
  if (nkt > 1) top = tile_max<false>(sa, 0, scale_log2);   // of the tile whose turn is next: all but the last one's are the request's
  int t = 0;
  for (; t + 2 <= nkt - 1; t += 2) {
    body(t, sa, sb);
    body(t + 1, sb, sa);
  }
  if (t < nkt - 1) {
    body(t, sa, sb);
    tail(t + 1, sb);
  } else {
    tail(t, sa);
  }
  lds_barrier();   // the rings are filled again by the next piece
  l_run = half_sum(l_run);
  // a piece whose keys all scored below fp32's range has the weight zero beside the others; alone such a row is NaN
  const float inv = slot_no >= 0 && l_run == 0.f ? 0.f : 1.0f / l_run;
  if (slot_no < 0) {
    if (me.live) store_o<DH>(g.o + me.at, lg, o, inv);
    return;
  }
  // a piece: O / sum in quads, then (maximum, sum), lane-major
  float* slot = g.partial + static_cast<size_t>(slot_no) * (C::E * C::THREADS);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      reinterpret_cast<float4*>(slot)[(4 * d + r4) * C::THREADS + tid] =
          make_float4(o[d][4 * r4] * inv, o[d][4 * r4 + 1] * inv, o[d][4 * r4 + 2] * inv, o[d][4 * r4 + 3] * inv);
  reinterpret_cast<f32x2_t*>(slot + DT * 16 * C::THREADS)[tid] = f32x2_t{m_run, l_run};
}

// ---------------------------------------------------------------- few rows

// Key steps [s0, s1) of 32 rows; the piece's slot holds O / sum [32][DH] and (maximum, sum) [32].
template <int DH>
FD_DEVICE void few_piece(const fdh::CacheAttnArgs& g, int group, float scale_log2, uint4* ring, uint32_t lds, int head, int tile,
                         const Request& of, int s0, int s1, int slot_no) {
  using C = Cfg<DH>;
  constexpr int DT = C::DT, KS = C::KS, KCH = C::KCH;
  // Formed anew for each piece: kept from one to the next, the lane's addresses were spilled, and what read them back waited for
  // every load under way.
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = fd::uniform(tid >> 6), l32 = lane & 31, lg = lane >> 5;
  const Lane<DH> ln(lane);
  const int k_beg = of.k_beg, k_end = of.k_end, ldk = g.kv_heads * DH;
  // A tile's codes come 16 a lane, whole rows side by side.  K's go to LDS as they are and come back as fragments: the
  // contraction's order is free, so that a lane's two steps 2 j and 2 j + 1 take its chunk 2 j + lg of the key's row (head dim 16,
  // of one step: 8 codes of the chunk).  V's go there as values, head dim 128 half the keys at a time.
  constexpr int PER_ROW = DH / 16, ROWS = 64 / PER_ROW, N = KB / ROWS;   // ROWS rows a load, N loads
  constexpr int VH = C::VHALVES;
  // The lane's rows of a load are ROWS apart, which leaves the swizzles: addresses are a base and a constant.
  const int lrow = lane / PER_ROW, lc = lane % PER_ROW;
  auto kswz = [](int r) { return PER_ROW == 8 ? (r & 7) : PER_ROW == 4 ? ((r >> 1) & 3) : 0; };
  const uint32_t k_at = lds + static_cast<uint32_t>(wave * C::FEW_WAVE_BYTES), v_at = k_at + KB * DH;   // this wave's own: no barriers
  const uint32_t put_k = k_at + static_cast<uint32_t>(lrow * DH + (lc ^ kswz(lrow)) * 16);
  const uint32_t put_v0 = v_at + static_cast<uint32_t>((lrow * KCH + ((2 * lc) ^ C::fv(lrow))) * 16), put_v1 = put_v0 ^ 16u;
  uint32_t get_k[(KS + 1) / 2];   // of key l32; key l32 + 32 has the same swizzle
#pragma unroll
  for (int j = 0; j < (KS + 1) / 2; ++j)
    get_k[j] = k_at + static_cast<uint32_t>(l32 * DH + (DH == 16 ? 8 * lg : ((2 * j + lg) ^ kswz(l32)) * 16));
  const uint8_t* ksc = g.k_scale + static_cast<size_t>(head) * g.n_tokens;
  const uint8_t* vsc = g.v_scale + static_cast<size_t>(head) * g.n_tokens;
  const uint32_t off = static_cast<uint32_t>(lrow) * static_cast<uint32_t>(ldk) + static_cast<uint32_t>(16 * lc);
  auto fetch = [&](const uint8_t* cache, const uint8_t* scale, int key0, u32x4_t (&x)[N], uint32_t& sc) {   // keys past the end repeat the last one
    const int last = k_end - 1 - key0;
    const uint8_t* p = cache + static_cast<size_t>(key0) * ldk + static_cast<size_t>(head) * DH;
    if (last >= KB - 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = *reinterpret_cast<const u32x4_t*>(p + static_cast<size_t>(ROWS * i) * ldk + off);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        x[i] = *reinterpret_cast<const u32x4_t*>(p + static_cast<uint32_t>(min(ROWS * i + lrow, last)) * static_cast<uint32_t>(ldk) + 16 * lc);
    }
    sc = (scale + key0)[min(lane, last)];
  };
  f32x16_t o[DT] = {};
  float m_run = -INFINITY, l_run = 0.f;
  bf16x8_t qf[KS];
  u32x4_t xk[N], xv[N];
  uint32_t sk, sv;
  auto own_lds = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
  auto put_v = [&](int half) {
#pragma unroll
    for (int i = half * (N / VH); i < (half + 1) * (N / VH); ++i) {
      const float sc = scale_of(__shfl(static_cast<int>(sv), ROWS * i + lrow, fd::kWave));
      const uint2 a = values4(xv[i][0], sc), b2 = values4(xv[i][1], sc), c = values4(xv[i][2], sc), d = values4(xv[i][3], sc);
      const uint32_t on = static_cast<uint32_t>((i - half * (N / VH)) * ROWS * KCH * 16);
      *(__attribute__((address_space(3))) u32x4_t*)(uintptr_t)(put_v0 + on) = u32x4_t{a.x, a.y, b2.x, b2.y};
      *(__attribute__((address_space(3))) u32x4_t*)(uintptr_t)(put_v1 + on) = u32x4_t{c.x, c.y, d.x, d.y};
    }
  };
  auto step = [&](int key0, int next) {   // the tile in xk and xv, whose places the one from `next` on takes
#pragma unroll
    for (int i = 0; i < N; ++i) *(__attribute__((address_space(3))) u32x4_t*)(uintptr_t)(put_k + static_cast<uint32_t>(ROWS * i * DH)) = xk[i];
    float ksl[2];
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) ksl[kh] = scale_of(__shfl(static_cast<int>(sk), 32 * kh + l32, fd::kWave));
    own_lds();
    f32x16_t s[2] = {};
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) {
      constexpr int kHalf = 32 * DH;
      __builtin_amdgcn_sched_barrier(0);   // as many fragments at once as there are registers for
      if constexpr (DH == 16) {
        const u32x2_t c = *(__attribute__((address_space(3))) const u32x2_t*)(uintptr_t)(get_k[0] + static_cast<uint32_t>(kh * kHalf));
        const uint2 lo = values4(c[0], ksl[kh]), hi = values4(c[1], ksl[kh]);
        s[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, u32x4_t{lo.x, lo.y, hi.x, hi.y}), qf[0], s[kh], 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < KS / 2; ++j) {
          const u32x4_t c = *(__attribute__((address_space(3))) const u32x4_t*)(uintptr_t)(get_k[j] + static_cast<uint32_t>(kh * kHalf));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint2 lo = values4(c[2 * i], ksl[kh]), hi = values4(c[2 * i + 1], ksl[kh]);
            s[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, u32x4_t{lo.x, lo.y, hi.x, hi.y}), qf[2 * j + i], s[kh], 0, 0, 0);
          }
        }
      }
    }
    put_v(0);
    __builtin_amdgcn_sched_barrier(0);
    fetch(g.k, ksc, next, xk, sk);   // not before: the fragments need the registers
    const float sub = take_max<DH>(tile_max<true>(s, k_end - key0 - 4 * lg, scale_log2), m_run, l_run, o);
    bf16x8_t pk[4];
    take_p(s, scale_log2, sub, pk, l_run);
#pragma unroll
    for (int half = 0; half < VH; ++half) {
      if (half) put_v(half);
      if (half == VH - 1) {
        __builtin_amdgcn_sched_barrier(0);
        fetch(g.v, vsc, next, xv, sv);
      }
      own_lds();
#pragma unroll
      for (int st = 0; st < 4 / VH; ++st) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < DT; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ln.v_frag(v_at, st, d)), pk[half * (4 / VH) + st], o[d], 0, 0, 0);
      }
      own_lds();
    }
  };
  const int key_end = min(k_end, k_beg + s1 * C::FEW_KEYS);
  int key0 = k_beg + s0 * C::FEW_KEYS + wave * KB;
  if (key0 < key_end) {
    fetch(g.k, ksc, key0, xk, sk);
    // rows past the last repeat it; without branches, as what stands here costs its fetch from memory (a call of a few MB has the L2
    // full of something else)
    const uint16_t* q = g.q + row_at<DH>(g, group, of, head, min(tile * C::QF + l32, of.rows - 1)).at;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(q + (DH == 16 ? 8 * lg : 16 * (2 * (ks >> 1) + lg) + 8 * (ks & 1))));
    fetch(g.v, vsc, key0, xv, sv);
    for (; key0 < key_end; key0 += C::FEW_KEYS) step(key0, min(key0 + C::FEW_KEYS, k_end - 1));   // the last one fetches in vain
  }
  l_run = half_sum(l_run);
  // the waves' results: O [wave][32][DH + 4] unnormalised, (maximum, sum) [wave][32]
  __syncthreads();
  constexpr int LD = DH + 4;
  float* part = reinterpret_cast<float*>(ring);
  f32x2_t* ml = reinterpret_cast<f32x2_t*>(part + C::WAVES * 32 * LD);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d0 = 32 * d + 8 * r4 + 4 * lg;
      if (d0 < DH)
        *reinterpret_cast<float4*>(part + (wave * 32 + l32) * LD + d0) = make_float4(o[d][4 * r4], o[d][4 * r4 + 1], o[d][4 * r4 + 2], o[d][4 * r4 + 3]);
    }
  if (lg == 0) ml[wave * 32 + l32] = f32x2_t{m_run, l_run};
  __syncthreads();
  const int rows = min(C::QF, of.rows - tile * C::QF);
  float* slot = g.partial + static_cast<size_t>(max(slot_no, 0)) * C::FEW_SLOT;
  for (int i = tid; i < rows * (DH / 4); i += C::THREADS) {
    const int r = i / (DH / 4), d0 = i % (DH / 4) * 4;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < C::WAVES; ++w) m = __builtin_elementwise_maximum(m, ml[w * 32 + r][0]);
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll
    for (int w = 0; w < C::WAVES; ++w) {
      const f32x2_t p = ml[w * 32 + r];
      const float4 v = *reinterpret_cast<const float4*>(part + (w * 32 + r) * LD + d0);
      // a wave without keys, or without a finite score, has the sum 0 (or NaN)
      const float a = p[0] == -INFINITY ? (p[1] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(p[0] - m);
      l += a * p[1];
      sum.x += a * v.x; sum.y += a * v.y; sum.z += a * v.z; sum.w += a * v.w;
    }
    const float inv = slot_no >= 0 && l == 0.f ? 0.f : 1.0f / l;
    sum = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    if (slot_no < 0) {
      const RowAt to = row_at<DH>(g, group, of, head, tile * C::QF + r);
      *reinterpret_cast<uint2*>(g.o + to.at + d0) = make_uint2(fd::pack_bf2(sum.x, sum.y), fd::pack_bf2(sum.z, sum.w));
    } else {
      *reinterpret_cast<float4*>(slot + r * DH + d0) = sum;
      if (d0 == 0) reinterpret_cast<f32x2_t*>(slot + 32 * DH)[r] = f32x2_t{m, l};
    }
  }
  __syncthreads();   // the next piece fills the tiles again
}

// FEW_ONLY: no call of this many rows runs in tiles, and the kernel does without their code and registers.
template <int DH, bool FEW_ONLY>
__global__ __launch_bounds__(Cfg<DH>::THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void cache_attn_kernel(fdh::CacheAttnArgs g) {
  using C = Cfg<DH>;
  // tiles: two of K and two of V; few rows: the waves' own, then their results
  constexpr int kTileBytes = FEW_ONLY ? 0 : 4 * C::TILE * 16, kFewBytes = C::WAVES * C::FEW_WAVE_BYTES, kJoinBytes = C::WAVES * 32 * ((DH + 4) * 4 + 8);
  constexpr int kMore = kFewBytes > kJoinBytes ? kFewBytes : kJoinBytes, kBytes = kMore > kTileBytes ? kMore : kTileBytes;
  __shared__ __align__(256) uint4 ring[(kBytes + 15) / 16];   // chunk addresses are formed by exclusive or
  __shared__ Tables tabs;
  const int group = fd::uniform(g.heads / g.kv_heads);
  const Way way = build_tables<DH>(tabs, g, group);
  const int tid = threadIdx.x;
  if (way.empty)   // a request without tokens: its rows are zeros
    for (int b = blockIdx.x; b < g.n_req; b += gridDim.x) {
      if (g.tok_off[b + 1] > g.tok_off[b]) continue;
      const long long per = static_cast<long long>(g.heads) * DH / 8, end = per * g.cu_q[b + 1];
      for (long long i = per * g.cu_q[b] + tid; i < end; i += C::THREADS) reinterpret_cast<uint4*>(g.o)[i] = make_uint4(0, 0, 0, 0);
    }
  const bool few = FEW_ONLY || fd::uniform(static_cast<int>(way.few)) != 0;
  const Sched<DH> sch = schedule<DH, FEW_ONLY>(&tabs, g, way);
  if (tid == 0 && g.may_cut) g_cut_items(g)[blockIdx.x] = CutItem{};
  if (sch.work == 0) return;
  const float scale_log2 = g.scale * 1.4426950408889634f;
  const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)&ring[0]));
  // waves w and w + WAVES / 2 share a SIMD: the second issues first when both are ready, so that the pair drifts apart
  if (__builtin_amdgcn_readfirstlane(tid >> 6) >= C::WAVES / 2) __builtin_amdgcn_s_setprio(1);
  const int w = sch.share(static_cast<int>(blockIdx.x));
  long long p = sch.bound(w);
  const long long p_end = sch.bound(w + 1);
  while (p < p_end) {
    long long i_start;
    int n, head, b, first, tau;
    sch.locate(p, i_start, n, head, b, first, tau);
    const int s0 = static_cast<int>(p - i_start), s1 = static_cast<int>(min(p_end, i_start + n) - i_start);
    const int slot = sch.cut ? sch.slot_of(w, s0, s1, n) : -1;
    const int t0 = sch.tile(s0), t1 = sch.tile(s1), q0 = fd::uniform(tabs.q0[b]);
    const Request of{q0, (fd::uniform(tabs.q0[b + 1]) - q0) * group, fd::uniform(tabs.k0[b]), fd::uniform(tabs.k0[b + 1])};
    if (FEW_ONLY || few) few_piece<DH>(g, group, scale_log2, ring, lds, head, tau - first, of, t0, t1, slot);
    else if constexpr (!FEW_ONLY) tile_piece<DH>(g, group, scale_log2, lds, head, tau - first, of, t0, t1, slot);
    if (tid == 0 && slot >= 0 && s0 == 0)   // its first piece
      g_cut_items(g)[blockIdx.x] = CutItem{sch.last_share(i_start + n) - w + 1, w, head, b, 2 * (tau - first) + few};
    p = i_start + s1;
  }
}

// The pieces of the cut items, joined in key order: workgroups (x, 0 ..) take the item whose first piece workgroup x of
// the attention had, a part of its values each (one workgroup an item: 256 rows of 12 heads, 21 pieces each, 45 us).  Each piece's
// O is divided by its own sum: its weight is 2^(maximum - the largest) * sum.  Eight pieces' loads are in flight together; what
// came before is rescaled to the new maximum.
template <int VALUES>
struct Joined {
  float top = -INFINITY, l = 0.f;
  float4 o[VALUES] = {};
  template <int AT_ONCE, class Ml, class Value>
  FD_DEVICE void add(int pieces, Ml ml_of, Value value_of) {
    for (int j0 = 0; j0 < pieces; j0 += AT_ONCE) {
      f32x2_t ml[AT_ONCE];
      float4 v[AT_ONCE][VALUES];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int p = min(j0 + j, pieces - 1);
        ml[j] = ml_of(p);
#pragma unroll
        for (int i = 0; i < VALUES; ++i) v[j][i] = value_of(p, i);
      }
      float next = top;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) next = __builtin_elementwise_maximum(next, ml[j][0]);
      const float back = top == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(top - next);
      l *= back;
#pragma unroll
      for (int i = 0; i < VALUES; ++i) o[i] = make_float4(o[i].x * back, o[i].y * back, o[i].z * back, o[i].w * back);
      top = next;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        if (j0 + j >= pieces) continue;
        // a piece without a finite score has the sum 0 and zeros (or NaN)
        const float a = ml[j][0] == -INFINITY ? ml[j][1] : __builtin_amdgcn_exp2f(ml[j][0] - top) * ml[j][1];
        l += a;
#pragma unroll
        for (int i = 0; i < VALUES; ++i)
          o[i] = make_float4(o[i].x + a * v[j][i].x, o[i].y + a * v[j][i].y, o[i].z + a * v[j][i].z, o[i].w + a * v[j][i].w);
      }
    }
  }
  FD_DEVICE uint2 row(int i) const {
    const float inv = 1.0f / l;
    return make_uint2(fd::pack_bf2(o[i].x * inv, o[i].y * inv), fd::pack_bf2(o[i].z * inv, o[i].w * inv));
  }
};
template <int DH>
__global__ __launch_bounds__(Cfg<DH>::THREADS) void cache_join_kernel(fdh::CacheAttnArgs g) {
  using C = Cfg<DH>;
  const CutItem it = g_cut_items(g)[blockIdx.x];
  if (it.pieces == 0) return;
  const int group = g.heads / g.kv_heads, few = it.tile_few & 1, tile = it.tile_few >> 1, head = it.head, b = it.request, x = it.share, first = g.cu_q[b];
  const Request of{first, (g.cu_q[b + 1] - first) * group, 0, 0};
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lg = lane >> 5;
  auto slot = [&](int j, int floats) { return g.partial + static_cast<size_t>(Sched<DH>::slot_at(x, j)) * floats; };
  if (few) {
    const int rows = min(C::QF, of.rows - tile * C::QF);
    for (int i = blockIdx.y * C::THREADS + tid; i < rows * (DH / 4); i += gridDim.y * C::THREADS) {
      const int r = i / (DH / 4), d0 = i % (DH / 4) * 4;
      Joined<1> sum;
      sum.template add<24>(it.pieces, [&](int j) { return reinterpret_cast<const f32x2_t*>(slot(j, C::FEW_SLOT) + 32 * DH)[r]; },
                           [&](int j, int) { return *reinterpret_cast<const float4*>(slot(j, C::FEW_SLOT) + r * DH + d0); });
      *reinterpret_cast<uint2*>(g.o + row_at<DH>(g, group, of, head, tile * C::QF + r).at + d0) = sum.row(0);
    }
    return;
  }
  const RowAt me = row_at<DH>(g, group, of, head, tile * C::QB + 32 * wave + l32);
  if (!me.live) return;
  const int q0 = blockIdx.y * 2;   // this workgroup's quads q0 and q0 + 1: d = 8 q + 4 lg ..
  Joined<2> sum;
  auto ml_of = [&](int j) { return reinterpret_cast<const f32x2_t*>(slot(j, C::E * C::THREADS) + C::DT * 16 * C::THREADS)[tid]; };
  auto value_of = [&](int j, int i) { return reinterpret_cast<const float4*>(slot(j, C::E * C::THREADS))[(q0 + i) * C::THREADS + tid]; };
  // two pieces are what most items of a packed batch have: 255 of them 14.2 -> 11.9 us
  if (it.pieces <= 2) sum.template add<2>(it.pieces, ml_of, value_of);
  else sum.template add<8>(it.pieces, ml_of, value_of);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int d0 = 8 * (q0 + i) + 4 * lg;
    if (d0 < DH) *reinterpret_cast<uint2*>(g.o + me.at + d0) = sum.row(i);
  }
}

}  // namespace

namespace fdh {

namespace {
// Workgroups: eight waves a CU, two a SIMD.
int cache_grid(int dh) { return (num_cus() + fd::kXcds - 1) / fd::kXcds * fd::kXcds * (256 / fd::cache_tile_rows(dh)); }
// The items' records come first in the workspace, then the pieces.
size_t cut_items_bytes(int dh) { return (cache_grid(dh) * sizeof(CutItem) + 255) / 256 * 256; }
}  // namespace

size_t cache_attention_scratch_bytes(int n_rows, int heads, int kv_heads, int dh) {
  // two slots per share: 32 rows where no call of these rows runs in tiles
  const bool few = fd::cache_always_few(dh, static_cast<long long>(n_rows) * (heads / kv_heads));
  const size_t floats = few ? 32 * (dh + 2) : static_cast<size_t>(2 * fd::cache_tile_rows(dh)) * ((dh + 31) / 32 * 16 + 2);
  return cut_items_bytes(dh) + 2 * static_cast<size_t>(cache_grid(dh)) * floats * sizeof(float);
}

hipError_t launch_cache_attention(const CacheAttnArgs& args, hipStream_t s) {
  CacheAttnArgs g = args;
  g.cut_items = args.partial;
  g.partial = args.partial + cut_items_bytes(g.dh) / sizeof(float);
  g.may_cut = g.max_req_tokens > fd::cache_few_keys(g.dh);
  auto run = [&](auto tag) {
    constexpr int DH = decltype(tag)::value;
    if (fd::cache_always_few(DH, static_cast<long long>(g.n_rows) * (g.heads / g.kv_heads))) cache_attn_kernel<DH, true><<<cache_grid(DH), Cfg<DH>::THREADS, 0, s>>>(g);
    else cache_attn_kernel<DH, false><<<cache_grid(DH), Cfg<DH>::THREADS, 0, s>>>(g);
    if (g.may_cut) cache_join_kernel<DH><<<dim3(cache_grid(DH), Cfg<DH>::JOIN_PARTS), Cfg<DH>::THREADS, 0, s>>>(g);
  };
  switch (g.dh) {
    case 16: run(std::integral_constant<int, 16>{}); break;
    case 64: run(std::integral_constant<int, 64>{}); break;
    default: run(std::integral_constant<int, 128>{});
  }
  return hipGetLastError();
}

}  // namespace fdh
