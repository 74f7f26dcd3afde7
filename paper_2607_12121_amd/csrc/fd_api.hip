// C ABI entry points: argument validation, workspace carving and launch order of
// the region-sparse DiT step.  Nothing here allocates device memory.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <mutex>
#include <vector>

#include "fd_common.h"
#include "fd_rules.h"
#include "fd_scaled.h"

namespace {

thread_local char g_err[512] = "";

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }

int score_rows_per_chunk(int C) {
  const int r = 2048 / C;
  return r < 1 ? 1 : r;
}

// Token rows per workgroup of the score: a whole region (one pass) or a chunk of one.
int score_rows(const fd_plan* p, int C) {
  return fd::score_one_pass(p->n_regions, static_cast<long long>(p->max_region_tokens) * C, fdh::num_cus())
             ? p->max_region_tokens
             : score_rows_per_chunk(C);
}

struct BlockWs {
  float* mod;
  uint16_t* a;
  uint16_t* q;
  uint16_t* o;
  uint16_t* g;
  float* partial;      // split-K partial tiles
  float* lse;          // [N][H] base-2 log-sum-exp of each active query's scaled scores
  size_t bytes;
};

BlockWs carve_block_ws(const fd_plan* p, const fd_dims* d, void* base) {
  const size_t n = static_cast<size_t>(p->n_tokens);
  size_t off = 0;
  BlockWs w;
  const uintptr_t b0 = reinterpret_cast<uintptr_t>(base);
  auto take = [&](size_t bytes) {
    const uintptr_t ptr = b0 + off;
    off += align_up(bytes);
    return reinterpret_cast<void*>(ptr);
  };
  w.mod = static_cast<float*>(take(static_cast<size_t>(p->n_requests) * 6 * d->D * sizeof(float)));
  w.a = static_cast<uint16_t*>(take(n * d->D * 2));
  w.q = static_cast<uint16_t*>(take(n * d->D * 2));
  w.o = static_cast<uint16_t*>(take(n * d->D * 2));
  w.g = static_cast<uint16_t*>(take(n * d->F * 2));
  const size_t gemm_part = fdh::gemm_scratch_bytes();
  const size_t attn_part = fdh::attn_scratch_bytes(d->dh);
  w.partial = static_cast<float*>(take(gemm_part > attn_part ? gemm_part : attn_part));
  w.lse = static_cast<float*>(take(n * d->H * sizeof(float)));
  w.bytes = off;
  return w;
}

// The 8-bit block's workspace: the block's own (fd_region_importance finds its queries and normalisers where
// fd_block_forward leaves them), then the rows in 8 bits and the fused projection.  The MLP's hidden codes and
// scales take the place of its bf16 rows, a branch's output that of the norm's.
struct ScaledWs {
  BlockWs block;
  uint8_t *a, *sa, *g, *sg;
  uint16_t* qkv;
  size_t bytes;
};

ScaledWs carve_scaled_ws(const fd_plan* p, const fd_dims* d, void* base) {
  const size_t n = static_cast<size_t>(p->n_tokens);
  ScaledWs w;
  w.block = carve_block_ws(p, d, base);
  size_t off = w.block.bytes;
  const uintptr_t b0 = reinterpret_cast<uintptr_t>(base);
  auto take = [&](size_t bytes) {
    const uintptr_t ptr = b0 + off;
    off += align_up(bytes);
    return reinterpret_cast<void*>(ptr);
  };
  w.a = static_cast<uint8_t*>(take(n * d->D));
  w.sa = static_cast<uint8_t*>(take(n * fd::scale_stride(d->D)));
  w.qkv = static_cast<uint16_t*>(take(n * 3 * d->D * 2));
  w.sg = static_cast<uint8_t*>(take(n * fd::scale_stride(d->F)));
  w.g = reinterpret_cast<uint8_t*>(w.block.g);
  w.bytes = off;
  return w;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

fd_status check_plan(const fd_plan* p) {
  if (!p) return fdh::set_error("plan is null"), FD_E_ARG;
  if (p->n_tokens < 1 || p->n_regions < 1 || p->n_requests < 1 || p->max_region_tokens < 1 ||
      p->max_request_tokens < 1)
    return fdh::set_error("plan sizes must be positive"), FD_E_ARG;
  if (!p->region_ptr || !p->region_tokens || !p->region_req || !p->token_region || !p->req_tok_off ||
      !p->req_reg_off)
    return fdh::set_error("plan has a null device array"), FD_E_ARG;
  return FD_OK;
}

fd_status check_dims(const fd_dims* d) {
  if (!d) return fdh::set_error("dims is null"), FD_E_ARG;
  if (d->C < 1 || d->D < 1 || d->H < 1 || d->dh < 1 || d->F < 1)
    return fdh::set_error("dims must be positive"), FD_E_ARG;
  if (d->D != d->H * d->dh) return fdh::set_error("D (%d) != H * dh (%d * %d)", d->D, d->H, d->dh), FD_E_SHAPE;
  if (d->dh != 16 && d->dh != 64 && d->dh != 128)
    return fdh::set_error("head dim %d not in {16, 64, 128}", d->dh), FD_E_UNSUPPORTED;
  if (d->D % 64 || d->F % 64) return fdh::set_error("D and F must be multiples of 64"), FD_E_UNSUPPORTED;
  if (d->D > 12288) return fdh::set_error("D > 12288 unsupported"), FD_E_UNSUPPORTED;
  if (d->C % 16 || d->C > 256) return fdh::set_error("C must be a multiple of 16, <= 256"), FD_E_UNSUPPORTED;
  return FD_OK;
}

fd_status check_C(int C) {
  if (C < 16 || C % 16 || C > 256) return fdh::set_error("C must be a multiple of 16 in [16, 256]"), FD_E_UNSUPPORTED;
  return FD_OK;
}

#define FD_REQUIRE(cond, ...)                  \
  do {                                         \
    if (!(cond)) {                             \
      fdh::set_error(__VA_ARGS__);             \
      return FD_E_ARG;                         \
    }                                          \
  } while (0)

#define FD_TRY(expr)                  \
  do {                                \
    fd_status st_ = (expr);           \
    if (st_ != FD_OK) return st_;     \
  } while (0)

// Column counts of 8-bit rows: 16-byte aligned rows, and column numbers that run past the last by at most a block.
fd_status check_cols(int cols) {
  if (cols > (1 << 30)) return fdh::set_error("%d columns, more than 2^30", cols), FD_E_UNSUPPORTED;
  if (cols % 16) return fdh::set_error("%d columns, not a multiple of 16", cols), FD_E_UNSUPPORTED;
  return FD_OK;
}

// Row counts: a kernel's 32-bit row numbers run past the last by at most a launch's rows.
fd_status check_rows(int rows) {
  if (rows > (1 << 30)) return fdh::set_error("%d rows, more than 2^30", rows), FD_E_UNSUPPORTED;
  return FD_OK;
}

// Checks a rotary descriptor and fills the kernel's sections and the turns of its pairs.
fd_status rope_turns(const fd_rope* r, int dh, fdh::RopeArgs* g) {
  FD_REQUIRE(r, "rope is null");
  if (dh != 16 && dh != 64 && dh != 128)
    return fdh::set_error("head dim %d not in {16, 64, 128}", dh), FD_E_UNSUPPORTED;
  FD_REQUIRE(r->n_axes >= 1 && r->n_axes <= fdh::kMaxRopeAxes, "%d axes, not 1 to 4", r->n_axes);
  FD_REQUIRE(r->pairing == FD_ROPE_INTERLEAVED || r->pairing == FD_ROPE_HALVES, "unknown pairing %d", r->pairing);
  g->n_axes = r->n_axes;
  g->pairs = 0;
  for (int a = 0; a < r->n_axes; ++a) {
    const int d = r->dim[a];
    FD_REQUIRE(d >= 2 && d % 2 == 0 && d <= dh - 2 * g->pairs, "axis %d: %d values of a head of %d", a, d, dh);
    FD_REQUIRE(r->theta[a] > 0 && isfinite(r->theta[a]) && isfinite(r->step[a]), "axis %d: theta or step", a);
    g->dim[a] = d;
    for (int j = 0; j < d / 2; ++j) {
      double turns = r->step[a] * pow(r->theta[a], -2.0 * j / d) / 6.283185307179586;
      FD_REQUIRE(fabs(turns) <= 1 << 20, "axis %d: %g turns per position", a, turns);
      if (fabs(turns) > 0.5) {   // positions are whole numbers: whole turns of each go, and the rest keeps its bits
        const long double t = r->step[a] * powl(r->theta[a], -2.0L * j / d) / 6.283185307179586476925L;
        turns = static_cast<double>(t - rintl(t));
      }
      g->turns[g->pairs++] = turns;
    }
  }
  return FD_OK;
}

// What the attention of a block takes.
fd_status check_attention(const fd_plan* plan, const fd_dims* dims) {
  if (plan->n_requests > fdh::kMaxAttnRequests)
    return fdh::set_error("the block supports at most %d requests per call (%d given)", fdh::kMaxAttnRequests,
                          plan->n_requests),
           FD_E_UNSUPPORTED;
  // it addresses a request's key and value rows with 32-bit offsets
  if (static_cast<long long>(plan->max_request_tokens) * dims->D * 2 >= (1LL << 32))
    return fdh::set_error("the block supports at most 4 GiB of keys per request (%d tokens x %d given)",
                          plan->max_request_tokens, dims->D),
           FD_E_UNSUPPORTED;
  return FD_OK;
}

#define FD_LAUNCH(kernel_id, stream, call)               \
  do {                                                   \
    fdh::timer_begin(kernel_id, stream);                 \
    hipError_t e_ = (call);                              \
    fdh::timer_end(kernel_id, stream);                   \
    if (e_ != hipSuccess) return fdh::hip_fail(e_, #call); \
  } while (0)

// ---------------------------------------------------------------- kernel timer
struct Timer {
  std::mutex mu;
  int kernel = 0;
  int capacity = 0;
  int count = 0;
  std::vector<hipEvent_t> ev;
} g_timer;

}  // namespace

namespace fdh {

void set_error(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
}

fd_status hip_fail(hipError_t e, const char* what) {
  set_error("%s: %s", what, hipGetErrorString(e));
  return FD_E_HIP;
}

int num_cus() {
  static int cache[64];
  static std::once_flag once[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = 0;
  std::call_once(once[dev], [&] {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) n = 256;
    cache[dev] = n;
  });
  return cache[dev];
}

void timer_begin(int kernel, hipStream_t s) {
  std::lock_guard<std::mutex> lk(g_timer.mu);
  if (g_timer.kernel != kernel || g_timer.count >= g_timer.capacity) return;
  (void)hipEventRecord(g_timer.ev[2 * g_timer.count], s);
}

void timer_end(int kernel, hipStream_t s) {
  std::lock_guard<std::mutex> lk(g_timer.mu);
  if (g_timer.kernel != kernel || g_timer.count >= g_timer.capacity) return;
  (void)hipEventRecord(g_timer.ev[2 * g_timer.count + 1], s);
  ++g_timer.count;
}

}  // namespace fdh

extern "C" {

const char* fd_last_error(void) { return g_err; }
const char* fd_version(void) { return "flashdiff-mi355x 0.1 (gfx950)"; }

fd_status fd_plan_build(int32_t n_tokens, int32_t n_regions, int32_t n_requests, const int32_t* token_region,
                        const int32_t* req_tok_off, int32_t* region_ptr, int32_t* region_tokens, int32_t* region_req,
                        int32_t* req_reg_off, int32_t* max_region_tokens, int32_t* max_request_tokens) {
  FD_REQUIRE(n_tokens >= 1 && n_regions >= 1 && n_requests >= 1, "sizes must be positive");
  FD_REQUIRE(n_regions <= n_tokens, "more regions (%d) than tokens (%d)", n_regions, n_tokens);
  FD_REQUIRE(token_region && req_tok_off && region_ptr && region_tokens && region_req && req_reg_off &&
                 max_region_tokens && max_request_tokens,
             "null pointer");
  FD_REQUIRE(req_tok_off[0] == 0 && req_tok_off[n_requests] == n_tokens, "req_tok_off must span [0, N]");
  int max_req = 0;
  for (int b = 0; b < n_requests; ++b) {
    const int nb = req_tok_off[b + 1] - req_tok_off[b];
    FD_REQUIRE(nb >= 1, "request %d has no tokens", b);
    if (nb > max_req) max_req = nb;
  }
  std::vector<int32_t> cnt(n_regions, 0);
  for (int u = 0; u < n_tokens; ++u) {
    const int r = token_region[u];
    FD_REQUIRE(r >= 0 && r < n_regions, "token %d has region %d outside [0, %d)", u, r, n_regions);
    ++cnt[r];
  }
  region_ptr[0] = 0;
  int max_reg = 0;
  for (int r = 0; r < n_regions; ++r) {
    FD_REQUIRE(cnt[r] >= 1, "region %d is empty", r);
    region_ptr[r + 1] = region_ptr[r] + cnt[r];
    if (cnt[r] > max_reg) max_reg = cnt[r];
    region_req[r] = -1;
  }
  std::vector<int32_t> fill(region_ptr, region_ptr + n_regions);
  int b = 0;
  for (int u = 0; u < n_tokens; ++u) {
    while (u >= req_tok_off[b + 1]) ++b;
    const int r = token_region[u];
    if (region_req[r] < 0) region_req[r] = b;
    FD_REQUIRE(region_req[r] == b, "region %d spans requests %d and %d", r, region_req[r], b);
    region_tokens[fill[r]++] = u;
  }
  for (int r = 1; r < n_regions; ++r)
    FD_REQUIRE(region_req[r] >= region_req[r - 1], "region ids are not request-major at region %d", r);
  int r = 0;
  for (int bb = 0; bb < n_requests; ++bb) {
    req_reg_off[bb] = r;
    while (r < n_regions && region_req[r] == bb) ++r;
  }
  req_reg_off[n_requests] = r;
  *max_region_tokens = max_reg;
  *max_request_tokens = max_req;
  return FD_OK;
}

size_t fd_region_score_ws_size(const fd_plan* plan, int32_t C) {
  if (!plan || C < 1) return 0;
  const int rows = score_rows_per_chunk(C);
  const int nchunk = (plan->max_region_tokens + rows - 1) / rows;
  return align_up(static_cast<size_t>(plan->n_regions) * nchunk * sizeof(double));
}

fd_status fd_region_score(const fd_plan* plan, int32_t C, const float* x_cur, const float* x_prev, double* score,
                          void* ws, size_t ws_bytes, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_C(C));
  FD_REQUIRE(x_cur && x_prev && score && ws, "null pointer");
  FD_REQUIRE(aligned(x_cur, 16) && aligned(x_prev, 16) && aligned(ws, 8), "misaligned buffer");
  if (ws_bytes < fd_region_score_ws_size(plan, C)) return fdh::set_error("score workspace too small"), FD_E_SHAPE;
  const int rows = score_rows(plan, C);
  const int nchunk = (plan->max_region_tokens + rows - 1) / rows;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_SCORE, s,
            fdh::launch_region_score(plan, C, x_cur, x_prev, score, static_cast<double*>(ws), nchunk, rows, s));
  return FD_OK;
}

// ---------------------------------------------------------------- region score without allocation
// The partial sums of fd_region_score_noalloc live in this file-scope device array
// (one copy per GPU, held until the process ends).  In host code its name is not a
// device address: every host use goes through the address hipGetSymbolAddress
// returns for the current device, taken once per device.
}  // extern "C"

namespace {

constexpr size_t kScoreScratchBytes = size_t(1) << 20;   // 131072 (region, chunk) partial sums
__device__ __align__(256) unsigned char scratch[kScoreScratchBytes];

constexpr int kMaxDevices = 64;
struct ScratchAddr {
  std::once_flag once;
  void* ptr = nullptr;
  hipError_t err = hipSuccess;
};
ScratchAddr g_scratch[kMaxDevices];

// Device address of `scratch` on the current device (looked up on the first call per device).
fd_status scratch_address(void** out) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fdh::hip_fail(e, "hipGetDevice");
  if (dev < 0 || dev >= kMaxDevices) return fdh::set_error("device %d beyond the scratch table", dev), FD_E_UNSUPPORTED;
  ScratchAddr& a = g_scratch[dev];
  std::call_once(a.once, [&] { a.err = hipGetSymbolAddress(&a.ptr, HIP_SYMBOL(scratch)); });
  if (a.err != hipSuccess || !a.ptr) return fdh::hip_fail(a.err, "hipGetSymbolAddress(scratch)");
  *out = a.ptr;
  return FD_OK;
}

}  // namespace

extern "C" {

fd_status fd_region_score_noalloc(const fd_plan* plan, int32_t C, const float* x_cur, const float* x_prev,
                                  double* score, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_C(C));
  FD_REQUIRE(x_cur && x_prev && score, "null pointer");
  FD_REQUIRE(aligned(x_cur, 16) && aligned(x_prev, 16), "misaligned buffer");
  const size_t need = fd_region_score_ws_size(plan, C);
  if (need > kScoreScratchBytes)
    return fdh::set_error("score partials need %zu bytes, beyond the %zu-byte built-in scratch (use fd_region_score)",
                          need, kScoreScratchBytes),
           FD_E_UNSUPPORTED;
  void* ws = nullptr;
  FD_TRY(scratch_address(&ws));
  const int rows = score_rows(plan, C);
  const int nchunk = (plan->max_region_tokens + rows - 1) / rows;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_SCORE, s,
            fdh::launch_region_score(plan, C, x_cur, x_prev, score, static_cast<double*>(ws), nchunk, rows, s));
  return FD_OK;
}

fd_status fd_select(const fd_plan* plan, const double* score, const double* eps, fd_gate gate, double* s_tilde,
                    int32_t* skip_run, const uint8_t* prev_active, uint8_t* active, int32_t* idx, int32_t* cu_q,
                    int32_t* m, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_REQUIRE(score && eps && s_tilde && skip_run && prev_active && active && idx && cu_q && m, "null pointer");
  if (plan->n_regions > 4096 || plan->n_requests > 1024)
    return fdh::set_error("select supports R <= 4096 and B <= 1024"), FD_E_UNSUPPORTED;
  FD_REQUIRE(gate.eta >= 0.0 && gate.max_skip >= 0, "eta and max_skip must be >= 0");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_SELECT, s,
            fdh::launch_select(plan, score, eps, gate, s_tilde, skip_run, prev_active, active, idx, cu_q, m, s));
  return FD_OK;
}

fd_status fd_gather(const fd_plan* plan, int32_t C, const float* x_cur, const int32_t* idx, const int32_t* m,
                    uint16_t* xa, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_C(C));
  FD_REQUIRE(x_cur && idx && m && xa, "null pointer");
  FD_REQUIRE(aligned(x_cur, 16) && aligned(xa, 8), "misaligned buffer");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_GATHER, s, fdh::launch_gather(plan, C, x_cur, idx, m, xa, s));
  return FD_OK;
}

fd_status fd_embed(const fd_plan* plan, const fd_dims* dims, const uint16_t* xa, const uint16_t* w_e, const float* b_e,
                   const float* pos, const int32_t* idx, const int32_t* m, float* h, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_dims(dims));
  FD_REQUIRE(xa && w_e && b_e && pos && idx && m && h, "null pointer");
  FD_REQUIRE(aligned(xa, 16) && aligned(w_e, 16), "misaligned buffer");
  fdh::GemmArgs g{};
  g.act = xa; g.wt = w_e; g.bias = b_e; g.n_max = plan->n_tokens; g.m = m; g.N = dims->D; g.K = dims->C;
  g.idx = idx; g.out_f32 = h; g.pos = pos;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_EMBED, s, fdh::launch_gemm(fdh::GEMM_EMBED, g, s));
  return FD_OK;
}

fd_status fd_adaln(const fd_dims* dims, int32_t n_blocks, int32_t n_out, int32_t n_requests, const uint16_t* w_ada,
                   const float* b_ada, const float* cond, float* mod, fd_stream_t stream) {
  FD_TRY(check_dims(dims));
  FD_REQUIRE(w_ada && b_ada && cond && mod, "null pointer");
  FD_REQUIRE(n_blocks >= 1 && n_out >= 1 && n_requests >= 1, "n_blocks, n_out and n_requests must be positive");
  FD_REQUIRE(static_cast<long long>(n_blocks) * n_out <= (1LL << 28), "too many modulation rows");
  FD_REQUIRE(aligned(w_ada, 16) && aligned(cond, 16), "misaligned buffer");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_ADALN, s,
            fdh::launch_adaln(w_ada, b_ada, cond, n_requests, dims->D, n_out, n_blocks, mod, s));
  return FD_OK;
}

size_t fd_block_ws_size(const fd_plan* plan, const fd_dims* dims) {
  if (!plan || !dims) return 0;
  return carve_block_ws(plan, dims, nullptr).bytes;
}

fd_status fd_block_forward(const fd_plan* plan, const fd_dims* dims, const fd_block_weights* w, const float* cond,
                           float* h, const int32_t* idx, const int32_t* cu_q, const int32_t* m, uint16_t* k_cache,
                           uint16_t* v_cache, void* ws, size_t ws_bytes, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_dims(dims));
  FD_REQUIRE(w && h && idx && cu_q && m && k_cache && v_cache && ws, "null pointer");
  FD_REQUIRE(w->w_qkv && w->b_qkv && w->w_o && w->b_o && w->w_1 && w->b_1 && w->w_2 && w->b_2 &&
                 (w->mod || (w->w_ada && w->b_ada && cond)),
             "null weight pointer");
  FD_REQUIRE(aligned(w->w_qkv, 16) && aligned(w->w_o, 16) && aligned(w->w_1, 16) && aligned(w->w_2, 16) &&
                 (w->mod ? aligned(w->mod, 16) : aligned(w->w_ada, 16)) && aligned(h, 16) && aligned(k_cache, 16) &&
                 aligned(v_cache, 16) && aligned(ws, kAlign),
             "misaligned buffer");
  FD_TRY(check_attention(plan, dims));
  // the tile loads address the weights of one product with 31-bit offsets
  const long long widest = dims->F > 3LL * dims->D ? dims->F : 3LL * dims->D;
  if (2 * widest * dims->D > fdh::kMaxGemmBytes)
    return fdh::set_error("the block supports weights below 2 GiB per product (%lld x %d given)", widest, dims->D),
           FD_E_UNSUPPORTED;
  const BlockWs bw = carve_block_ws(plan, dims, ws);
  if (ws_bytes < bw.bytes) return fdh::set_error("block workspace too small (%zu < %zu)", ws_bytes, bw.bytes), FD_E_SHAPE;
  const int D = dims->D, F = dims->F, B = plan->n_requests, N = plan->n_tokens;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);

  // modulation: precomputed by fd_adaln, else computed here
  const float* mod = w->mod ? w->mod : bw.mod;
  if (!w->mod)
    FD_LAUNCH(FD_K_ADALN, s,
              fdh::launch_adaln(w->w_ada, w->b_ada, cond, B, D, 6 * D, 1, bw.mod, s));
  FD_LAUNCH(FD_K_LN, s, fdh::launch_ln_modulate(h, cu_q, B, m, N, D, mod, 6 * D, 0, D, bw.a, idx, plan->token_region,
                                                        plan->region_req, s));
  fdh::GemmArgs g{};
  g.n_max = N; g.m = m; g.idx = idx; g.cu_q = cu_q; g.n_req = B; g.D = D;
  g.partial = bw.partial; g.max_units = fdh::gemm_max_tiles();
  g.act = bw.a; g.wt = w->w_qkv; g.bias = w->b_qkv; g.N = 3 * D; g.K = D;
  g.out_bf16 = bw.q; g.k_cache = k_cache; g.v_cache = v_cache;
  FD_LAUNCH(FD_K_GEMM_QKV, s, fdh::launch_gemm(fdh::GEMM_QKV, g, s));
  FD_LAUNCH(FD_K_ATTN, s,
            fdh::launch_attention(bw.q, k_cache, v_cache, bw.o, D, dims->H, dims->dh, cu_q, plan->req_tok_off, B, N,
                                  plan->max_request_tokens, bw.partial, bw.lse, s));
  g = fdh::GemmArgs{};
  g.n_max = N; g.m = m; g.idx = idx; g.cu_q = cu_q; g.n_req = B; g.D = D;
  g.partial = bw.partial; g.max_units = fdh::gemm_max_tiles();
  g.act = bw.o; g.wt = w->w_o; g.bias = w->b_o; g.N = D; g.K = D;
  g.out_f32 = h; g.gate = mod + 2 * D; g.gate_stride = 6 * D;
  FD_LAUNCH(FD_K_GEMM_O, s, fdh::launch_gemm(fdh::GEMM_RESID, g, s));
  FD_LAUNCH(FD_K_LN, s, fdh::launch_ln_modulate(h, cu_q, B, m, N, D, mod, 6 * D, 3 * D, 4 * D, bw.a, idx,
                                                        plan->token_region, plan->region_req, s));
  g = fdh::GemmArgs{};
  g.n_max = N; g.m = m; g.idx = idx; g.cu_q = cu_q; g.n_req = B; g.D = D;
  g.partial = bw.partial; g.max_units = fdh::gemm_max_tiles();
  g.act = bw.a; g.wt = w->w_1; g.bias = w->b_1; g.N = F; g.K = D; g.out_bf16 = bw.g;
  FD_LAUNCH(FD_K_GEMM_MLP1, s, fdh::launch_gemm(fdh::GEMM_GELU, g, s));
  g = fdh::GemmArgs{};
  g.n_max = N; g.m = m; g.idx = idx; g.cu_q = cu_q; g.n_req = B; g.D = D;
  g.partial = bw.partial; g.max_units = fdh::gemm_max_tiles();
  g.act = bw.g; g.wt = w->w_2; g.bias = w->b_2; g.N = D; g.K = F;
  g.out_f32 = h; g.gate = mod + 5 * D; g.gate_stride = 6 * D;
  FD_LAUNCH(FD_K_GEMM_MLP2, s, fdh::launch_gemm(fdh::GEMM_RESID, g, s));
  return FD_OK;
}

size_t fd_importance_ws_size(const fd_plan* plan, const fd_dims* dims) {
  if (!plan || !dims) return 0;
  return align_up(static_cast<size_t>(plan->n_tokens) * sizeof(int32_t)) +
         align_up(static_cast<size_t>(plan->n_regions) * dims->H * sizeof(float));
}

fd_status fd_region_importance(const fd_plan* plan, const fd_dims* dims, const void* block_ws, size_t block_ws_bytes,
                               const uint16_t* k_cache, const int32_t* idx, const int32_t* m, const uint8_t* active,
                               double* r_bar, double* delta, double* importance, void* ws, size_t ws_bytes,
                               fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_dims(dims));
  FD_REQUIRE(block_ws && k_cache && idx && m && active && r_bar && delta && ws, "null pointer");
  FD_REQUIRE(aligned(block_ws, kAlign) && aligned(ws, kAlign) && aligned(k_cache, 16), "misaligned buffer");
  const BlockWs bw = carve_block_ws(plan, dims, const_cast<void*>(block_ws));
  if (block_ws_bytes < bw.bytes)
    return fdh::set_error("block workspace too small (%zu < %zu)", block_ws_bytes, bw.bytes), FD_E_SHAPE;
  const size_t need = fd_importance_ws_size(plan, dims);
  if (ws_bytes < need) return fdh::set_error("importance workspace too small (%zu < %zu)", ws_bytes, need), FD_E_SHAPE;
  if (fdh::importance_lds_bytes(dims->dh, plan->max_region_tokens) > 156 * 1024)
    return fdh::set_error("regions of %d tokens exceed the importance kernel's LDS staging", plan->max_region_tokens),
           FD_E_UNSUPPORTED;
  const uintptr_t b0 = reinterpret_cast<uintptr_t>(ws);
  int32_t* pos = reinterpret_cast<int32_t*>(b0);
  float* part = reinterpret_cast<float*>(b0 + align_up(static_cast<size_t>(plan->n_tokens) * sizeof(int32_t)));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_IMPORTANCE, s,
            fdh::launch_importance(plan, dims->D, dims->H, dims->dh, idx, m, active, bw.q, k_cache, bw.lse, pos, part,
                                   r_bar, delta, importance, s));
  return FD_OK;
}

size_t fd_partition_ws_size(int32_t n_tokens, int32_t n_requests) {
  if (n_tokens < 0 || n_requests < 1) return 0;
  return fdh::partition_ws_bytes(n_tokens, n_requests);
}

fd_status fd_partition(int32_t n_requests, const int32_t* req_tok_off, const int32_t* req_reg_off,
                       const uint16_t* saliency, int32_t* token_region, void* ws, size_t ws_bytes,
                       fd_stream_t stream) {
  FD_REQUIRE(req_tok_off && req_reg_off && saliency && token_region && ws, "null pointer");
  FD_REQUIRE(n_requests >= 1, "n_requests = %d", n_requests);
  if (n_requests > fd::kMaxPartRequests)
    return fdh::set_error("%d requests exceed the partitioner's %d per call", n_requests, fd::kMaxPartRequests),
           FD_E_UNSUPPORTED;
  FD_REQUIRE(req_tok_off[0] == 0 && req_reg_off[0] == 0, "offsets must start at 0");
  for (int b = 0; b < n_requests; ++b) {
    const int n = req_tok_off[b + 1] - req_tok_off[b], r = req_reg_off[b + 1] - req_reg_off[b];
    FD_REQUIRE(r >= 1 && n >= r, "request %d: %d tokens cannot fill %d regions", b, n, r);
    if (n > fd::kMaxPartTokens || r > fd::kMaxPartRegions)
      return fdh::set_error("request %d: %d tokens / %d regions exceed the partitioner's %d / %d", b, n, r,
                            fd::kMaxPartTokens, fd::kMaxPartRegions),
             FD_E_UNSUPPORTED;
  }
  FD_REQUIRE(aligned(ws, kAlign), "misaligned buffer");
  const size_t need = fdh::partition_ws_bytes(req_tok_off[n_requests], n_requests);
  if (ws_bytes < need) return fdh::set_error("partition workspace too small (%zu < %zu)", ws_bytes, need), FD_E_SHAPE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_PARTITION, s,
            fdh::launch_partition(n_requests, req_tok_off, req_reg_off, saliency, token_region, ws, s));
  return FD_OK;
}

fd_status fd_final(const fd_plan* plan, const fd_dims* dims, const fd_final_weights* w, const float* cond,
                   const float* h, const int32_t* cu_q, const int32_t* m, float* v, void* ws, size_t ws_bytes,
                   fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_dims(dims));
  FD_REQUIRE(w && w->w_ada && w->b_ada && w->w_out && w->b_out && cond && h && cu_q && m && v && ws, "null pointer");
  FD_REQUIRE(aligned(w->w_ada, 16) && aligned(w->w_out, 16) && aligned(h, 16) && aligned(ws, kAlign),
             "misaligned buffer");
  const BlockWs bw = carve_block_ws(plan, dims, ws);
  if (ws_bytes < bw.bytes) return fdh::set_error("final workspace too small"), FD_E_SHAPE;
  const int D = dims->D, B = plan->n_requests, N = plan->n_tokens;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_ADALN, s,
            fdh::launch_adaln(w->w_ada, w->b_ada, cond, B, D, 2 * D, 1, bw.mod, s));
  FD_LAUNCH(FD_K_LN, s, fdh::launch_ln_modulate(h, cu_q, B, m, N, D, bw.mod, 2 * D, 0, D, bw.a, nullptr, nullptr, nullptr, s));
  fdh::GemmArgs g{};
  g.n_max = N; g.m = m; g.cu_q = cu_q; g.n_req = B;
  g.partial = bw.partial; g.max_units = fdh::gemm_max_tiles();
  g.act = bw.a; g.wt = w->w_out; g.bias = w->b_out; g.N = dims->C; g.K = D; g.out_f32 = v;
  FD_LAUNCH(FD_K_FINAL, s, fdh::launch_gemm(fdh::GEMM_OUT, g, s));
  return FD_OK;
}

fd_status fd_scatter_update(const fd_plan* plan, int32_t C, float* x, const float* v, const int32_t* idx,
                            const int32_t* m, const float* dt, float* vcache, const uint8_t* active, int32_t skip_mode,
                            fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_C(C));
  FD_REQUIRE(x && v && idx && m && dt && vcache && active, "null pointer");
  FD_REQUIRE(skip_mode == FD_SKIP_FREEZE || skip_mode == FD_SKIP_REUSE_DRIFT, "unknown skip mode %d", skip_mode);
  FD_REQUIRE(aligned(x, 16) && aligned(v, 16) && aligned(vcache, 16), "misaligned buffer");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_SCATTER, s, fdh::launch_scatter_update(plan, C, x, v, idx, m, dt, vcache, active, skip_mode, s));
  return FD_OK;
}

int32_t fd_scale_stride(int32_t cols) { return cols < 1 ? 0 : fd::scale_stride(cols); }

fd_status fd_quant_blocks(int32_t n_rows, int32_t cols, int32_t block_rows, const uint16_t* x, const int32_t* m,
                          uint8_t* q, uint8_t* scale, fd_stream_t stream) {
  FD_REQUIRE(n_rows >= 1 && cols >= 1, "sizes must be positive");
  FD_REQUIRE(block_rows == 1 || block_rows == fd::kScaleBlock, "block_rows = %d, not 1 or 128", block_rows);
  FD_TRY(check_rows(n_rows));
  FD_TRY(check_cols(cols));
  FD_REQUIRE(x && q && scale, "null pointer");
  FD_REQUIRE(!m || block_rows == 1, "a row count with 128-row blocks");
  FD_REQUIRE(aligned(x, 16) && aligned(q, 16), "misaligned buffer");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_QUANT, s, fdh::launch_quant_blocks(x, n_rows, cols, block_rows, m, q, scale, s));
  return FD_OK;
}

fd_status fd_rms_quant(int32_t n_rows, int32_t D, int32_t n_requests, float* h, const uint16_t* y, const float* gate,
                       const float* weight, const float* shift, const float* scale, int32_t mod_stride, float eps,
                       const int32_t* cu_q, const int32_t* m, uint8_t* q, uint8_t* q_scale, fd_stream_t stream) {
  FD_REQUIRE(n_rows >= 1 && D >= 1 && n_requests >= 1, "sizes must be positive");
  FD_TRY(check_rows(n_rows));
  FD_TRY(check_cols(D));
  if (D > 12288) return fdh::set_error("D > 12288 unsupported"), FD_E_UNSUPPORTED;
  FD_REQUIRE(h && m && (cu_q || n_requests == 1), "null pointer");
  FD_REQUIRE(!q == !q_scale && (q || y), "neither codes with scales nor a branch to add");
  FD_REQUIRE(eps >= 0.f, "eps must be >= 0");
  FD_REQUIRE(mod_stride >= 0 && mod_stride % 4 == 0, "mod_stride = %d, not a multiple of 4", mod_stride);
  FD_REQUIRE(aligned(h, 16) && aligned(y, 16) && aligned(gate, 16) && aligned(weight, 16) && aligned(shift, 16) &&
                 aligned(scale, 16) && aligned(q, 16),
             "misaligned buffer");
  fdh::RmsArgs g{};
  g.n_rows = n_rows; g.D = D; g.n_req = n_requests; g.mod_stride = mod_stride; g.cu_q = cu_q; g.m = m; g.eps = eps;
  g.h = h; g.y = y; g.gate = gate; g.weight = weight; g.shift = shift; g.scale = scale; g.q = q; g.q_scale = q_scale;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_RMS, s, fdh::launch_rms_quant(g, s));
  return FD_OK;
}

fd_status fd_rope_axes(int32_t n_rows, int32_t n_tokens, const fd_rope* rope, int32_t heads, int32_t kv_heads, int32_t dh,
                       const int32_t* coord, const uint16_t* qkv, const int32_t* idx, const int32_t* m, uint16_t* q,
                       uint16_t* k_cache, uint16_t* v_cache, fd_stream_t stream) {
  FD_REQUIRE(n_rows >= 1 && n_rows <= n_tokens, "%d rows of %d tokens", n_rows, n_tokens);
  FD_TRY(check_rows(n_rows));
  FD_REQUIRE(heads >= 1 && kv_heads >= 1, "heads must be positive");
  FD_REQUIRE(coord && qkv && m && q && k_cache && v_cache, "null pointer");
  FD_REQUIRE(aligned(qkv, 16) && aligned(q, 16) && aligned(k_cache, 16) && aligned(v_cache, 16), "misaligned buffer");
  fdh::RopeArgs g{};
  FD_TRY(rope_turns(rope, dh, &g));
  if (heads > 4096 || kv_heads > 4096) return fdh::set_error("more than 4096 heads"), FD_E_UNSUPPORTED;
  g.n_rows = n_rows; g.hq = heads; g.hk = kv_heads; g.dh = dh; g.m = m; g.idx = idx; g.coord = coord;
  g.qkv = qkv; g.q = q; g.k = k_cache; g.v = v_cache;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_ROPE, s, fdh::launch_rope(g, rope->pairing == FD_ROPE_HALVES, s));
  return FD_OK;
}

fd_status fd_scaled_linear(int32_t n_rows, int32_t n_out, int32_t n_in, const uint8_t* a, const uint8_t* a_scale,
                           const uint8_t* w, const uint8_t* w_scale, const float* bias, int32_t gelu, const int32_t* m,
                           uint16_t* y_bf, float* y_fp, uint8_t* y_q, uint8_t* y_scale, fd_stream_t stream) {
  FD_REQUIRE(n_rows >= 1 && n_out >= 1 && n_in >= 1, "sizes must be positive");
  FD_TRY(check_rows(n_rows));
  FD_TRY(check_cols(n_in));
  FD_TRY(check_cols(n_out));
  FD_REQUIRE(a && a_scale && w && w_scale, "null pointer");
  FD_REQUIRE((y_bf != nullptr) + (y_fp != nullptr) + (y_q != nullptr) == 1 && !y_q == !y_scale, "not one output");
  FD_REQUIRE(gelu == 0 || gelu == 1, "gelu = %d", gelu);
  FD_REQUIRE(aligned(a, 16) && aligned(w, 16) && aligned(a_scale, 4) && aligned(w_scale, 4) && aligned(bias, 16) &&
                 aligned(y_bf, 16) && aligned(y_fp, 16) && aligned(y_q, 16),
             "misaligned buffer");
  if (n_out > (1 << 20) || n_in > (1 << 20) || static_cast<long long>(n_out) * n_in > fdh::kMaxGemmBytes)
    return fdh::set_error("more than 2^20 columns, or weights of 2 GiB or more (%d x %d given)", n_out, n_in), FD_E_UNSUPPORTED;
  fdh::ScaledArgs g{};
  g.n_rows = n_rows; g.N = n_out; g.K = n_in; g.m = m; g.a = a; g.a_scale = a_scale; g.w = w; g.w_scale = w_scale;
  g.bias = bias; g.gelu = gelu; g.y_bf16 = y_bf; g.y_f32 = y_fp; g.y_q = y_q; g.y_scale = y_scale;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FD_LAUNCH(FD_K_LINEAR, s, fdh::launch_scaled_linear(g, s));
  return FD_OK;
}

size_t fd_scaled_block_ws_size(const fd_plan* plan, const fd_dims* dims) {
  if (!plan || !dims) return 0;
  return carve_scaled_ws(plan, dims, nullptr).bytes;
}

fd_status fd_scaled_block_forward(const fd_plan* plan, const fd_dims* dims, const fd_scaled_weights* w, const fd_rope* rope,
                                  const int32_t* coord, float* h, const int32_t* idx, const int32_t* cu_q, const int32_t* m,
                                  uint16_t* k_cache, uint16_t* v_cache, void* ws, size_t ws_bytes, fd_stream_t stream) {
  FD_TRY(check_plan(plan));
  FD_TRY(check_dims(dims));
  FD_REQUIRE(w && h && idx && cu_q && m && k_cache && v_cache && ws, "null pointer");
  FD_REQUIRE(w->w_qkv && w->s_qkv && w->b_qkv && w->w_o && w->s_o && w->b_o && w->w_1 && w->s_1 && w->b_1 && w->w_2 && w->s_2 &&
                 w->b_2 && w->mod,
             "null weight pointer");
  FD_REQUIRE(!rope || coord, "rotary positions without coordinates");
  FD_REQUIRE(aligned(h, 16) && aligned(k_cache, 16) && aligned(v_cache, 16) && aligned(ws, kAlign) && aligned(w->mod, 16),
             "misaligned buffer");
  FD_TRY(check_attention(plan, dims));
  FD_TRY(check_rows(plan->n_tokens));
  const int D = dims->D, F = dims->F, B = plan->n_requests, N = plan->n_tokens;
  const long long widest = F > 3LL * D ? F : 3LL * D;
  if (widest > (1 << 20) || widest * D > fdh::kMaxGemmBytes)
    return fdh::set_error("the block supports weights below 2 GiB per product (%lld x %d given)", widest, D), FD_E_UNSUPPORTED;
  fdh::RopeArgs r{};
  if (rope) FD_TRY(rope_turns(rope, dims->dh, &r));
  const ScaledWs s8 = carve_scaled_ws(plan, dims, ws);
  const BlockWs& bw = s8.block;
  if (ws_bytes < s8.bytes) return fdh::set_error("block workspace too small (%zu < %zu)", ws_bytes, s8.bytes), FD_E_SHAPE;
  // every argument of the steps below is checked: nothing has been enqueued when one is refused
  for (const void* p : {static_cast<const void*>(w->w_qkv), static_cast<const void*>(w->w_o), static_cast<const void*>(w->w_1),
                        static_cast<const void*>(w->w_2), static_cast<const void*>(w->b_qkv), static_cast<const void*>(w->b_o),
                        static_cast<const void*>(w->b_1), static_cast<const void*>(w->b_2), static_cast<const void*>(w->norm_1),
                        static_cast<const void*>(w->norm_2)})
    FD_REQUIRE(aligned(p, 16), "misaligned buffer");
  for (const uint8_t* p : {w->s_qkv, w->s_o, w->s_1, w->s_2}) FD_REQUIRE(aligned(p, 4), "misaligned buffer");

  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const float* mod = w->mod;
  uint16_t* y = bw.a;   // a branch's output
  fdh::RmsArgs n{};
  n.n_rows = N; n.D = D; n.n_req = B; n.mod_stride = 6 * D; n.cu_q = cu_q; n.m = m; n.eps = 1e-6f; n.h = h;
  n.weight = w->norm_1; n.shift = mod; n.scale = mod + D; n.q = s8.a; n.q_scale = s8.sa;
  FD_LAUNCH(FD_K_RMS, s, fdh::launch_rms_quant(n, s));
  fdh::ScaledArgs g{};
  g.n_rows = N; g.m = m;
  g.N = 3 * D; g.K = D; g.a = s8.a; g.a_scale = s8.sa; g.w = w->w_qkv; g.w_scale = w->s_qkv; g.bias = w->b_qkv; g.y_bf16 = s8.qkv;
  FD_LAUNCH(FD_K_LINEAR, s, fdh::launch_scaled_linear(g, s));
  r.n_rows = N; r.hq = dims->H; r.hk = dims->H; r.dh = dims->dh; r.m = m; r.idx = idx; r.coord = coord;
  r.qkv = s8.qkv; r.q = bw.q; r.k = k_cache; r.v = v_cache;
  FD_LAUNCH(FD_K_ROPE, s, fdh::launch_rope(r, rope && rope->pairing == FD_ROPE_HALVES, s));
  FD_LAUNCH(FD_K_ATTN, s,
            fdh::launch_attention(bw.q, k_cache, v_cache, bw.o, D, dims->H, dims->dh, cu_q, plan->req_tok_off, B, N,
                                  plan->max_request_tokens, bw.partial, bw.lse, s));
  FD_LAUNCH(FD_K_QUANT, s, fdh::launch_quant_blocks(bw.o, N, D, 1, m, s8.a, s8.sa, s));
  g.N = D; g.w = w->w_o; g.w_scale = w->s_o; g.bias = w->b_o; g.y_bf16 = y;
  FD_LAUNCH(FD_K_LINEAR, s, fdh::launch_scaled_linear(g, s));
  n.y = y; n.gate = mod + 2 * D; n.weight = w->norm_2; n.shift = mod + 3 * D; n.scale = mod + 4 * D;
  FD_LAUNCH(FD_K_RMS, s, fdh::launch_rms_quant(n, s));
  g.N = F; g.w = w->w_1; g.w_scale = w->s_1; g.bias = w->b_1; g.gelu = 1; g.y_bf16 = nullptr; g.y_q = s8.g; g.y_scale = s8.sg;
  FD_LAUNCH(FD_K_LINEAR, s, fdh::launch_scaled_linear(g, s));
  g.N = D; g.K = F; g.a = s8.g; g.a_scale = s8.sg; g.w = w->w_2; g.w_scale = w->s_2; g.bias = w->b_2; g.gelu = 0;
  g.y_bf16 = y; g.y_q = nullptr; g.y_scale = nullptr;
  FD_LAUNCH(FD_K_LINEAR, s, fdh::launch_scaled_linear(g, s));
  n.gate = mod + 5 * D; n.q = nullptr; n.q_scale = nullptr;
  FD_LAUNCH(FD_K_RMS, s, fdh::launch_rms_quant(n, s));
  return FD_OK;
}

fd_status fd_timer_arm(int32_t kernel, int32_t capacity) {
  FD_REQUIRE(kernel >= FD_K_SCORE && kernel <= FD_K_LINEAR && capacity >= 1 && capacity <= (1 << 20),
             "bad timer arguments");
  std::lock_guard<std::mutex> lk(g_timer.mu);
  for (hipEvent_t e : g_timer.ev) (void)hipEventDestroy(e);
  g_timer.ev.assign(2 * static_cast<size_t>(capacity), nullptr);
  // timing-only events: no system-scope fence (cache write-back and invalidate) at
  // each record, which would stall the stream between the kernels around it
  for (auto& e : g_timer.ev) {
    hipError_t r = hipEventCreateWithFlags(&e, hipEventDisableSystemFence);
    if (r != hipSuccess) {
      g_timer.kernel = 0;
      g_timer.capacity = 0;
      return fdh::hip_fail(r, "hipEventCreateWithFlags");
    }
  }
  g_timer.kernel = kernel;
  g_timer.capacity = capacity;
  g_timer.count = 0;
  return FD_OK;
}

int32_t fd_timer_read(float* ms, int32_t capacity) {
  std::lock_guard<std::mutex> lk(g_timer.mu);
  const int n = g_timer.count < capacity ? g_timer.count : capacity;
  for (int i = 0; i < n; ++i) {
    if (hipEventSynchronize(g_timer.ev[2 * i + 1]) != hipSuccess ||
        hipEventElapsedTime(&ms[i], g_timer.ev[2 * i], g_timer.ev[2 * i + 1]) != hipSuccess)
      ms[i] = -1.f;
  }
  return n;
}

void fd_timer_disarm(void) {
  std::lock_guard<std::mutex> lk(g_timer.mu);
  for (hipEvent_t e : g_timer.ev) (void)hipEventDestroy(e);
  g_timer.ev.clear();
  g_timer.kernel = 0;
  g_timer.capacity = 0;
  g_timer.count = 0;
}

}  // extern "C"
