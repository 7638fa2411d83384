// C ABI of the resident-expert MoE layer: argument validation on the host,
// then the kernel launchers.  Declarations and contracts: moe_resident.h.
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <string>
#include <vector>

#include "gemm.h"
#include "kernels.h"
#include "mx.h"
#include "moe_resident.h"
#include "timing.h"

namespace {

thread_local std::string g_err;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

int ok() {
  g_err.clear();
  return MOE_OK;
}

int hip_status(hipError_t e, const char* where) {
  if (e != hipSuccess) return fail(MOE_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
  return ok();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#define REQUIRE(cond, ...) \
  do {                     \
    if (!(cond)) return fail(MOE_ERR_ARG, __VA_ARGS__); \
  } while (0)
#define SUPPORT(cond, ...) \
  do {                     \
    if (!(cond)) return fail(MOE_ERR_UNSUPPORTED, __VA_ARGS__); \
  } while (0)

int check_dtype(int dtype) {
  SUPPORT(dtype == MOE_F32 || dtype == MOE_BF16, "unsupported dtype %d", dtype);
  return MOE_OK;
}

// A launch of `threads` per token, in blocks of up to 32 tokens: a grid of 2^32 threads or more is
// not refused but taken modulo 2^32.
int check_grid(int T, int threads) {
  const long long most = (1LL << 32) / threads - 32;
  SUPPORT(T < most, "T = %d: fewer than %lld tokens", T, most);
  return MOE_OK;
}

// row vectors of 16 bytes: d % 8 == 0 and 16-byte aligned base pointers
int check_rows16(int d, const char* name, const void* p) {
  SUPPORT(d % 8 == 0, "d = %d must be a multiple of 8", d);
  SUPPORT(p == nullptr || aligned16(p), "%s must be 16-byte aligned", name);
  return MOE_OK;
}

// ---------------------------------------------------------------- timing pool
std::mutex g_tmu;
std::atomic<bool> g_ton{false};
std::vector<hipEvent_t> g_pool;
struct TimingRec {
  const char* name;
  int ev;
};
std::vector<TimingRec> g_recs;
int g_next = 0;
thread_local int t_open = -1;

void release_pool() {
  for (hipEvent_t e : g_pool) (void)hipEventDestroy(e);
  g_pool.clear();
  g_recs.clear();
  g_next = 0;
}

}  // namespace

namespace moe {
bool timing_on() { return g_ton.load(std::memory_order_relaxed); }

void timing_begin(const char* name, hipStream_t s) {
  std::lock_guard<std::mutex> lock(g_tmu);
  t_open = -1;
  if (g_next + 2 > (int)g_pool.size()) return;
  const int ev = g_next;
  g_next += 2;
  if (hipEventRecord(g_pool[ev], s) != hipSuccess) return;
  g_recs.push_back({name, ev});
  t_open = ev;
}

void timing_end(hipStream_t s) {
  if (t_open < 0) return;
  std::lock_guard<std::mutex> lock(g_tmu);
  (void)hipEventRecord(g_pool[t_open + 1], s);
  t_open = -1;
}
}  // namespace moe

extern "C" {

int moe_timing_enable(int capacity) {
  REQUIRE(capacity >= 0, "capacity = %d must be >= 0", capacity);
  std::lock_guard<std::mutex> lock(g_tmu);
  g_ton.store(false);
  release_pool();
  if (capacity == 0) return ok();
  g_pool.resize(2 * (size_t)capacity);
  for (auto& e : g_pool) {
    if (hipEventCreate(&e) != hipSuccess) {
      e = nullptr;
      release_pool();
      return fail(MOE_ERR_HIP, "hipEventCreate failed");
    }
  }
  g_recs.reserve(capacity);
  g_ton.store(true);
  return ok();
}

int moe_timing_collect(moe_kernel_time* out, int max_out, int* n_out) {
  REQUIRE(out && n_out && max_out >= 0, "out and n_out must not be NULL");
  std::lock_guard<std::mutex> lock(g_tmu);
  int n = 0;
  for (const TimingRec& r : g_recs) {
    hipError_t e = hipEventSynchronize(g_pool[r.ev + 1]);
    float ms = 0.f;
    if (e == hipSuccess) e = hipEventElapsedTime(&ms, g_pool[r.ev], g_pool[r.ev + 1]);
    if (e != hipSuccess) {
      g_recs.clear();
      g_next = 0;
      return fail(MOE_ERR_HIP, "timing: %s", hipGetErrorString(e));
    }
    int i = 0;
    while (i < n && std::strcmp(out[i].name, r.name) != 0) ++i;
    if (i == n) {
      if (n == max_out) continue;
      out[n++] = moe_kernel_time{r.name, 0, 0.f, 1e30f, 0.f};
    }
    out[i].launches += 1;
    out[i].total_ms += ms;
    out[i].min_ms = std::min(out[i].min_ms, ms);
    out[i].max_ms = std::max(out[i].max_ms, ms);
  }
  g_recs.clear();
  g_next = 0;
  *n_out = n;
  return ok();
}

const char* moe_last_error(void) { return g_err.c_str(); }

int moe_abi_version(void) { return 3; }

int moe_route_mask(const void* x, const void* w_router, const float* router_bias, int dtype,
                   int T, int d, int E, int k, float inv_tau, int gate,
                   const uint8_t* resident, float* logits, int32_t* topk_idx, float* topk_w,
                   int32_t* topk_local, hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0, "T = %d must be >= 0", T);
  REQUIRE(d >= 1, "d = %d must be >= 1", d);
  REQUIRE(E >= 1 && E <= 256, "E = %d must be in [1, 256]", E);
  REQUIRE(k >= 1 && k <= E, "k = %d must be in [1, E = %d]", k, E);
  REQUIRE(gate >= MOE_GATE_SOFTMAX_TOPK && gate <= MOE_GATE_SIGMOID, "unknown gate %d", gate);
  REQUIRE(std::isfinite(inv_tau) && inv_tau > 0.f, "inv_tau must be finite and > 0");
  REQUIRE(w_router && resident, "w_router and resident must not be NULL");
  REQUIRE(T == 0 || (x && topk_idx && topk_w && topk_local), "x and the top-k outputs must not be NULL");
  if ((r = check_grid(T, 16)) != MOE_OK) return r;
  if (dtype == MOE_BF16) {
    if ((r = check_rows16(d, "x", x)) != MOE_OK) return r;
    if ((r = check_rows16(d, "w_router", w_router)) != MOE_OK) return r;
  }
  return hip_status(moe::launch_route_fwd(x, w_router, router_bias, dtype == MOE_BF16, T, d, E, k,
                                          inv_tau, gate, resident, logits, topk_idx, topk_w,
                                          topk_local, stream),
                    "moe_route_mask");
}

size_t moe_route_bwd_workspace_size(int T, int d, int E) {
  if (T < 0 || d < 1 || E < 1) return 0;
  return moe::route_bwd_ws_bytes(T, d, E);
}

int moe_route_bwd(const void* x, const void* w_router, int dtype, int T, int d, int E, int k,
                  float inv_tau, int gate, const int32_t* topk_idx, const float* topk_w,
                  const float* logits, const float* d_topk_w, float* dz, float* dw_router,
                  float* d_bias, void* dx, int accumulate_dx, void* ws, size_t ws_bytes,
                  hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1, "bad sizes T = %d, d = %d", T, d);
  REQUIRE(E >= 1 && E <= 256, "E = %d must be in [1, 256]", E);
  REQUIRE(k >= 1 && k <= E, "k = %d must be in [1, E = %d]", k, E);
  REQUIRE(gate >= MOE_GATE_SOFTMAX_TOPK && gate <= MOE_GATE_SIGMOID, "unknown gate %d", gate);
  REQUIRE(std::isfinite(inv_tau) && inv_tau > 0.f, "inv_tau must be finite and > 0");
  REQUIRE(w_router && dw_router, "w_router and dw_router must not be NULL");
  REQUIRE(T == 0 || (x && topk_idx && topk_w && d_topk_w && dz && dx),
          "x, topk_idx, topk_w, d_topk_w, dz and dx must not be NULL");
  REQUIRE(gate != MOE_GATE_SOFTMAX || T == 0 || logits, "logits are required for MOE_GATE_SOFTMAX");
  if ((r = check_grid(T, 64)) != MOE_OK) return r;
  const size_t need = moe::route_bwd_ws_bytes(T, d, E);
  REQUIRE(ws && ws_bytes >= need, "workspace of %zu bytes needed (got %zu)", need, ws_bytes);
  if ((r = check_rows16(d, "x", x)) != MOE_OK) return r;
  if ((r = check_rows16(d, "dx", dx)) != MOE_OK) return r;
  if ((r = check_rows16(d, "w_router", w_router)) != MOE_OK) return r;
  SUPPORT(aligned16(ws), "the workspace must be 16-byte aligned");
  return hip_status(moe::launch_route_bwd(x, w_router, dtype == MOE_BF16, T, d, E, k, inv_tau, gate,
                                          topk_idx, topk_w, logits, d_topk_w, dz, dw_router,
                                          d_bias, dx, accumulate_dx, ws, stream),
                    "moe_route_bwd");
}

size_t moe_dispatch_workspace_size(int T, int k, int E_r) {
  if (T < 0 || k < 1 || E_r < 0) return 0;
  return moe::dispatch_ws_bytes(T, k, E_r);
}

int moe_dispatch(const void* x, int dtype, int T, int d, int k, int E_r,
                 const int32_t* topk_local, int32_t* counts, int32_t* offsets, int32_t* perm,
                 int32_t* inv_perm, void* xp, void* ws, size_t ws_bytes, hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1 && k >= 1, "bad sizes T = %d, d = %d, k = %d", T, d, k);
  REQUIRE(E_r >= 0 && E_r <= 256, "E_r = %d must be in [0, 256]", E_r);
  REQUIRE(offsets && (E_r == 0 || counts), "counts and offsets must not be NULL");
  REQUIRE(T == 0 || (x && topk_local && inv_perm && (E_r == 0 || (perm && xp))),
          "x, topk_local, perm, inv_perm and xp must not be NULL");
  if ((r = check_grid(T, k > 8 ? 64 : 8)) != MOE_OK) return r;
  const size_t need = moe::dispatch_ws_bytes(T, k, E_r);
  REQUIRE(ws && ws_bytes >= need, "workspace of %zu bytes needed (got %zu)", need, ws_bytes);
  if ((r = check_rows16(d, "x", x)) != MOE_OK) return r;
  if ((r = check_rows16(d, "xp", xp)) != MOE_OK) return r;
  return hip_status(moe::launch_dispatch(x, dtype == MOE_BF16, T, d, k, E_r, topk_local, counts,
                                         offsets, perm, inv_perm, xp, ws, stream),
                    "moe_dispatch");
}

int moe_dispatch_noalloc(const void* x, int dtype, int T, int d, int k, int E_r,
                         const int32_t* topk_local, int32_t* counts, int32_t* offsets,
                         int32_t* perm, int32_t* inv_perm, void* xp, hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1 && k >= 1, "bad sizes T = %d, d = %d, k = %d", T, d, k);
  REQUIRE(E_r >= 0 && E_r <= 256, "E_r = %d must be in [0, 256]", E_r);
  REQUIRE(offsets && (E_r == 0 || counts), "counts and offsets must not be NULL");
  REQUIRE(T == 0 || (x && topk_local && inv_perm && (E_r == 0 || (perm && xp))),
          "x, topk_local, perm, inv_perm and xp must not be NULL");
  if ((r = check_grid(T, k > 8 ? 64 : 8)) != MOE_OK) return r;
  const size_t need = moe::dispatch_ws_bytes(T, k, E_r);
  SUPPORT(need <= MOE_DISPATCH_NOALLOC_MAX_WS,
          "moe_dispatch_noalloc: T = %d, E_r = %d need a %zu-byte workspace, above the "
          "library's %zu-byte array (use moe_dispatch with a workspace)",
          T, E_r, need, (size_t)MOE_DISPATCH_NOALLOC_MAX_WS);
  if ((r = check_rows16(d, "x", x)) != MOE_OK) return r;
  if ((r = check_rows16(d, "xp", xp)) != MOE_OK) return r;
  return hip_status(moe::launch_dispatch_noalloc(x, dtype == MOE_BF16, T, d, k, E_r, topk_local,
                                                 counts, offsets, perm, inv_perm, xp, stream),
                    "moe_dispatch_noalloc");
}

int moe_dispatch_bwd(const void* dxp, int dtype, int T, int d, int k, int cap,
                     const int32_t* inv_perm, void* dx, int accumulate, hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1 && k >= 1 && cap >= 0, "bad sizes T = %d, d = %d, k = %d, cap = %d",
          T, d, k, cap);
  REQUIRE(T == 0 || (inv_perm && dx && dxp), "dxp, inv_perm and dx must not be NULL");
  if ((r = check_grid(T, 64)) != MOE_OK) return r;
  if ((r = check_rows16(d, "dxp", dxp)) != MOE_OK) return r;
  if ((r = check_rows16(d, "dx", dx)) != MOE_OK) return r;
  return hip_status(moe::launch_dispatch_bwd(dxp, dtype == MOE_BF16, T, d, k, cap, inv_perm, dx,
                                             accumulate, stream),
                    "moe_dispatch_bwd");
}

static int check_ffn(int dtype, int cap, int d, int H, int n_groups, const int32_t* offsets) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(cap >= 0 && d >= 1 && H >= 1, "bad sizes cap = %d, d = %d, H = %d", cap, d, H);
  REQUIRE(n_groups >= 0, "n_groups = %d must be >= 0", n_groups);
  SUPPORT(n_groups <= 256, "n_groups = %d: at most 256 groups per set", n_groups);
  REQUIRE(offsets, "offsets must not be NULL");
  SUPPORT(H % 64 == 0, "H = %d must be a multiple of 64", H);
  if (dtype == MOE_BF16) SUPPORT(d % 64 == 0, "d = %d must be a multiple of 64 for bf16", d);
  else SUPPORT(d % 8 == 0, "d = %d must be a multiple of 8", d);
  return MOE_OK;
}

namespace {

int check_set(const moe_ffn_set& f, int dtype, int d, bool fwd) {
  int r;
  if ((r = check_ffn(dtype, f.cap, d, f.H, f.n_groups, f.offsets)) != MOE_OK) return r;
  REQUIRE(f.n_groups == 0 || (f.w_gate_up && f.w_down), "expert weights must not be NULL");
  if (fwd) {
    REQUIRE(f.cap == 0 || (f.xp && f.gu && f.h && f.yp), "xp, gu, h and yp must not be NULL");
  } else {
    REQUIRE(f.n_groups == 0 || (f.dw_gate_up && f.dw_down),
            "the expert weight gradients must not be NULL");
    REQUIRE(f.cap == 0 || (f.dyp && f.xp && f.gu && f.h && f.dgu && f.dxp),
            "dyp, xp, gu, h, dgu and dxp must not be NULL");
  }
  if (dtype == MOE_BF16) {
    // the bf16 GEMMs address each operand with 32-bit byte offsets
    const long rows_bytes = 2L * f.cap * std::max<long>(d, 2L * f.H);
    const long w_bytes = 2L * f.n_groups * 2L * f.H * d;
    // and each expert's fp32 weight gradient (stored with 32-bit offsets)
    const long dw_bytes = 4L * 2L * f.H * d;
    SUPPORT(std::max(std::max(rows_bytes, w_bytes), dw_bytes) < 0xFFFFFFF0L,
            "bf16 expert operands must each stay below 4 GiB (cap = %d, H = %d, groups = %d)",
            f.cap, f.H, f.n_groups);
  }
  for (const void* p : {f.xp, f.w_gate_up, f.w_down, (const void*)f.gu, (const void*)f.h,
                        (const void*)f.yp, f.dyp, (const void*)f.dgu, (const void*)f.dxp,
                        (const void*)f.dw_gate_up, (const void*)f.dw_down})
    SUPPORT(p == nullptr || aligned16(p), "operands must be 16-byte aligned");
  return MOE_OK;
}

int check_sets(const moe_ffn_set* sets, int n_sets, int dtype, int d, bool fwd) {
  REQUIRE(sets != nullptr && n_sets >= 1 && n_sets <= 2, "n_sets = %d must be 1 or 2", n_sets);
  for (int i = 0; i < n_sets; ++i) {
    REQUIRE(sets[i].activation == MOE_ACT_SWIGLU || sets[i].activation == MOE_ACT_SILU,
            "sets[%d].activation = %d is not an expert form", i, sets[i].activation);
    REQUIRE(sets[i].activation == sets[0].activation, "all sets must have the same activation");
  }
  for (int i = 0; i < n_sets; ++i) {
    const int r = check_set(sets[i], dtype, d, fwd);
    if (r != MOE_OK) return r;
  }
  return MOE_OK;
}

}  // namespace

size_t moe_grouped_ffn_fwd_workspace_size(const moe_ffn_set* sets, int n_sets, int dtype, int d) {
  if (!sets || n_sets < 1 || n_sets > 2 || d < 1) return 0;
  return moe::ffn_fwd_ws_bytes(sets, n_sets, dtype == MOE_BF16, d);
}

int moe_grouped_ffn_fwd_sets(const moe_ffn_set* sets, int n_sets, int dtype, int d, void* ws,
                             size_t ws_bytes, hipStream_t stream) {
  int r;
  if ((r = check_sets(sets, n_sets, dtype, d, true)) != MOE_OK) return r;
  if (ws) {
    const size_t need = moe::ffn_fwd_ws_bytes(sets, n_sets, dtype == MOE_BF16, d);
    REQUIRE(ws_bytes >= need, "workspace of %zu bytes needed (got %zu)", need, ws_bytes);
    SUPPORT((reinterpret_cast<uintptr_t>(ws) & 255u) == 0, "the workspace must be 256-byte aligned");
    if (need == 0) ws = nullptr;
  }
  return hip_status(moe::launch_ffn_fwd_sets(sets, n_sets, dtype == MOE_BF16, d, ws, stream),
                    "moe_grouped_ffn_fwd_sets");
}

size_t moe_grouped_ffn_bwd_workspace_size(const moe_ffn_set* sets, int n_sets, int dtype, int d) {
  if (!sets || n_sets < 1 || n_sets > 2 || d < 1) return 0;
  return moe::ffn_bwd_ws_bytes(sets, n_sets, dtype == MOE_BF16, d);
}

int moe_grouped_ffn_bwd_sets(const moe_ffn_set* sets, int n_sets, int dtype, int d,
                             int accumulate_dw, void* ws, size_t ws_bytes, hipStream_t stream) {
  int r;
  if ((r = check_sets(sets, n_sets, dtype, d, false)) != MOE_OK) return r;
  if (ws) {
    const size_t need = moe::ffn_bwd_ws_bytes(sets, n_sets, dtype == MOE_BF16, d);
    REQUIRE(ws_bytes >= need, "workspace of %zu bytes needed (got %zu)", need, ws_bytes);
    SUPPORT((reinterpret_cast<uintptr_t>(ws) & 255u) == 0, "the workspace must be 256-byte aligned");
  }
  return hip_status(
      moe::launch_ffn_bwd_sets(sets, n_sets, dtype == MOE_BF16, d, accumulate_dw, ws, stream),
      "moe_grouped_ffn_bwd_sets");
}

int moe_grouped_ffn_fwd(const void* xp, const void* w_gate_up, const void* w_down, int dtype,
                        int cap, int d, int H, int n_groups, const int32_t* offsets, void* gu,
                        void* h, void* yp, hipStream_t stream) {
  moe_ffn_set f{};
  f.xp = xp; f.w_gate_up = w_gate_up; f.w_down = w_down; f.offsets = offsets;
  f.cap = cap; f.H = H; f.n_groups = n_groups;
  f.gu = gu; f.h = h; f.yp = yp;
  return moe_grouped_ffn_fwd_sets(&f, 1, dtype, d, nullptr, 0, stream);
}

int moe_grouped_ffn_bwd(const void* dyp, const void* xp, const void* gu, const void* h,
                        const void* w_gate_up, const void* w_down, int dtype, int cap, int d,
                        int H, int n_groups, const int32_t* offsets, void* dgu, void* dxp,
                        float* dw_gate_up, float* dw_down, int accumulate_dw,
                        hipStream_t stream) {
  moe_ffn_set f{};
  f.xp = xp; f.w_gate_up = w_gate_up; f.w_down = w_down; f.offsets = offsets;
  f.cap = cap; f.H = H; f.n_groups = n_groups;
  f.gu = const_cast<void*>(gu); f.h = const_cast<void*>(h);
  f.dyp = dyp; f.dgu = dgu; f.dxp = dxp; f.dw_gate_up = dw_gate_up; f.dw_down = dw_down;
  return moe_grouped_ffn_bwd_sets(&f, 1, dtype, d, accumulate_dw, nullptr, 0, stream);
}

int moe_combine_fwd(const void* yp, int dtype, int T, int d, int k, int cap, const float* topk_w,
                    const int32_t* inv_perm, const void* y_add, void* y, hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1 && k >= 1 && cap >= 0, "bad sizes T = %d, d = %d, k = %d, cap = %d",
          T, d, k, cap);
  REQUIRE(T == 0 || (topk_w && inv_perm && y), "topk_w, inv_perm and y must not be NULL");
  if ((r = check_grid(T, 64)) != MOE_OK) return r;
  if ((r = check_rows16(d, "yp", yp)) != MOE_OK) return r;
  if ((r = check_rows16(d, "y_add", y_add)) != MOE_OK) return r;
  if ((r = check_rows16(d, "y", y)) != MOE_OK) return r;
  return hip_status(moe::launch_combine_fwd(yp, dtype == MOE_BF16, T, d, k, cap, topk_w, inv_perm,
                                            y_add, y, stream),
                    "moe_combine_fwd");
}

int moe_combine_bwd(const void* dy, const void* yp, int dtype, int T, int d, int k, int cap,
                    const float* topk_w, const int32_t* inv_perm, void* dyp, float* d_topk_w,
                    hipStream_t stream) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1 && k >= 1 && cap >= 0, "bad sizes T = %d, d = %d, k = %d, cap = %d",
          T, d, k, cap);
  REQUIRE(T == 0 || (dy && topk_w && inv_perm && d_topk_w), "dy, topk_w, inv_perm and d_topk_w must not be NULL");
  if ((r = check_rows16(d, "dy", dy)) != MOE_OK) return r;
  if ((r = check_grid(T, 64)) != MOE_OK) return r;
  if ((r = check_rows16(d, "yp", yp)) != MOE_OK) return r;
  if ((r = check_rows16(d, "dyp", dyp)) != MOE_OK) return r;
  return hip_status(moe::launch_combine_bwd(dy, yp, dtype == MOE_BF16, T, d, k, cap, topk_w,
                                            inv_perm, dyp, d_topk_w, stream),
                    "moe_combine_bwd");
}

#define LAYER_CALL(fn, ...)            \
  do {                                 \
    const int r_ = fn(__VA_ARGS__);    \
    if (r_ != MOE_OK) {                \
      if (where) *where = #fn;         \
      return r_;                       \
    }                                  \
  } while (0)

int moe_layer_fwd(const moe_layer* l, const char** where, hipStream_t stream) {
  if (where) *where = "moe_layer_fwd";
  REQUIRE(l != nullptr, "layer must not be NULL");
  const moe_ffn_set& f = l->sets[0];
  LAYER_CALL(moe_route_mask, l->x, l->w_router, l->router_bias, l->dtype, l->T, l->d, l->E, l->k,
             l->inv_tau, l->gate, l->resident, l->logits, l->topk_idx, l->topk_w, l->topk_local,
             stream);
  LAYER_CALL(moe_dispatch, l->x, l->dtype, l->T, l->d, l->k, l->E_r, l->topk_local, l->counts,
             l->offsets, l->perm, l->inv_perm, const_cast<void*>(f.xp), l->ws_dispatch,
             l->ws_dispatch_bytes, stream);
  LAYER_CALL(moe_grouped_ffn_fwd_sets, l->sets, l->n_sets, l->dtype, l->d, l->ws_ffn,
             l->ws_ffn_bytes, stream);
  LAYER_CALL(moe_combine_fwd, f.yp, l->dtype, l->T, l->d, l->k, f.cap, l->topk_w, l->inv_perm,
             l->n_sets == 2 ? l->sets[1].yp : nullptr, l->y, stream);
  return ok();
}

int moe_layer_bwd(const moe_layer* l, const char** where, hipStream_t stream) {
  if (where) *where = "moe_layer_bwd";
  REQUIRE(l != nullptr, "layer must not be NULL");
  const moe_ffn_set& f = l->sets[0];
  LAYER_CALL(moe_combine_bwd, l->dy, f.yp, l->dtype, l->T, l->d, l->k, f.cap, l->topk_w,
             l->inv_perm, const_cast<void*>(f.dyp), l->d_topk_w, stream);
  LAYER_CALL(moe_grouped_ffn_bwd_sets, l->sets, l->n_sets, l->dtype, l->d, l->accumulate_dw,
             l->ws_ffn, l->ws_ffn_bytes, stream);
  LAYER_CALL(moe_dispatch_bwd, f.dxp, l->dtype, l->T, l->d, l->k, f.cap, l->inv_perm, l->dx,
             l->n_sets == 2 ? 1 : 0, stream);
  LAYER_CALL(moe_route_bwd, l->x, l->w_router, l->dtype, l->T, l->d, l->E, l->k, l->inv_tau,
             l->gate, l->topk_idx, l->topk_w, l->logits, l->d_topk_w, l->dz, l->dw_router,
             l->d_bias, l->dx, 1, l->ws_route, l->ws_route_bytes, stream);
  return ok();
}

namespace {
int check_norm(int dtype, int T, int d) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(T >= 0 && d >= 1, "bad sizes T = %d, d = %d", T, d);
  SUPPORT(d % 8 == 0, "d = %d must be a multiple of 8", d);
  SUPPORT(d <= moe::kMaxNormWidth, "d = %d: at most %d", d, moe::kMaxNormWidth);
  SUPPORT(T < 1 << 30, "T = %d must be below 2^30", T);
  return MOE_OK;
}
}  // namespace

int moe_layernorm_fwd(const void* x, const float* weight, const float* bias, int dtype, int T,
                      int d, float eps, void* y, float* mean, float* rstd, hipStream_t stream) {
  int r;
  if ((r = check_norm(dtype, T, d)) != MOE_OK) return r;
  REQUIRE(std::isfinite(eps) && eps >= 0.f, "eps must be finite and >= 0");
  REQUIRE(weight, "weight must not be NULL");
  REQUIRE(T == 0 || (x && y && mean && rstd), "x, y, mean and rstd must not be NULL");
  for (const void* p : {x, (const void*)weight, (const void*)bias, (const void*)y})
    SUPPORT(p == nullptr || aligned16(p), "arrays must be 16-byte aligned");
  return hip_status(moe::launch_norm_fwd(x, weight, bias, dtype == MOE_BF16, T, d, eps, y, mean,
                                         rstd, stream),
                    "moe_layernorm_fwd");
}

size_t moe_layernorm_bwd_workspace_size(int T, int d, int dtype) {
  if (check_norm(dtype, T, d) != MOE_OK) return 0;
  return moe::norm_bwd_ws_bytes(T, d, dtype == MOE_BF16);
}

int moe_layernorm_bwd(const void* dy, const void* x, const float* weight, const float* mean,
                      const float* rstd, int dtype, int T, int d, const void* dres, void* dx,
                      float* dw, float* db, int accumulate_dw, void* ws, size_t ws_bytes,
                      hipStream_t stream) {
  int r;
  if ((r = check_norm(dtype, T, d)) != MOE_OK) return r;
  REQUIRE(weight && dw, "weight and dw must not be NULL");
  REQUIRE(T == 0 || (dy && x && mean && rstd && dx), "dy, x, mean, rstd and dx must not be NULL");
  const size_t need = moe::norm_bwd_ws_bytes(T, d, dtype == MOE_BF16);
  REQUIRE(need == 0 || (ws && ws_bytes >= need), "workspace of %zu bytes needed (got %zu)", need,
          ws_bytes);
  for (const void* p : {dy, x, (const void*)weight, dres, (const void*)dx, (const void*)dw,
                        (const void*)db, (const void*)ws})
    SUPPORT(p == nullptr || aligned16(p), "arrays must be 16-byte aligned");
  return hip_status(moe::launch_norm_bwd(dy, x, weight, mean, rstd, dtype == MOE_BF16, T, d, dres,
                                         dx, dw, db, accumulate_dw, ws, stream),
                    "moe_layernorm_bwd");
}

namespace {
int check_block(const moe_block_norm* p, bool fwd) {
  REQUIRE(p != nullptr, "the arguments must not be NULL");
  int r;
  if ((r = check_norm(p->dtype, p->T, p->d)) != MOE_OK) return r;
  REQUIRE(p->gate_kind >= MOE_BLOCK_GATE_NONE && p->gate_kind <= MOE_BLOCK_GATE_TOKEN,
          "gate_kind = %d is none", p->gate_kind);
  const bool channel = p->gate_kind == MOE_BLOCK_GATE_CHANNEL, token = p->gate_kind == MOE_BLOCK_GATE_TOKEN;
  const bool post = p->post_weight != nullptr, pre = p->pre_weight != nullptr, any = p->T > 0;
  REQUIRE(std::isfinite(p->scale), "scale must be finite");
  REQUIRE(post || pre, "post_weight and pre_weight must not both be NULL");
  REQUIRE(post || !p->post_bias, "post_bias without post_weight");
  REQUIRE(pre || !p->pre_bias, "pre_bias without pre_weight");
  REQUIRE(p->gate_kind == MOE_BLOCK_GATE_NONE ? !p->gate : p->gate || (token && !any),
          "gate must be given with its gate_kind, and only then");
  REQUIRE(!any || !post || (p->post_mean && p->post_rstd), "post_mean and post_rstd must not be NULL");
  REQUIRE(!any || !pre || (p->pre_mean && p->pre_rstd), "pre_mean and pre_rstd must not be NULL");
  const float* gate16 = channel ? p->gate : nullptr;
  for (const void* q : {(const void*)p->f, (const void*)p->x_out, (const void*)p->post_weight,
                        (const void*)p->post_bias, (const void*)gate16, (const void*)p->pre_weight,
                        (const void*)p->pre_bias})
    SUPPORT(q == nullptr || aligned16(q), "arrays must be 16-byte aligned");
  if (fwd) {
    REQUIRE(std::isfinite(p->eps) && p->eps >= 0.f, "eps must be finite and >= 0");
    REQUIRE(!any || (p->x && p->f && p->x_out), "x, f and x_out must not be NULL");
    REQUIRE(!any || pre == (p->u != nullptr), "u must be given with pre_weight, and only then");
    SUPPORT(aligned16(p->x) && aligned16(p->u), "arrays must be 16-byte aligned");
    return MOE_OK;
  }
  REQUIRE(!any || (p->f && p->dx && p->df), "f, dx and df must not be NULL");
  REQUIRE(!any || !pre || (p->du && p->x_out), "du and x_out must not be NULL");
  REQUIRE(!any || pre || p->dres, "dres must not be NULL without a pre-norm");
  REQUIRE(!pre || p->d_pre_weight, "d_pre_weight must not be NULL");
  REQUIRE(!post || p->d_post_weight, "d_post_weight must not be NULL");
  REQUIRE(p->gate_kind == MOE_BLOCK_GATE_NONE || p->d_gate || (token && !any), "d_gate must not be NULL");
  const float* d_gate16 = channel ? p->d_gate : nullptr;
  for (const void* q : {p->du, p->dres, (const void*)p->dx, (const void*)p->df,
                        (const void*)p->d_post_weight, (const void*)p->d_post_bias, (const void*)d_gate16,
                        (const void*)p->d_pre_weight, (const void*)p->d_pre_bias, (const void*)p->ws})
    SUPPORT(q == nullptr || aligned16(q), "arrays must be 16-byte aligned");
  const size_t need = moe::block_norm_ws_bytes(p->T, p->d, p->dtype == MOE_BF16);
  REQUIRE(need == 0 || (p->ws && p->ws_bytes >= need), "workspace of %zu bytes needed (got %zu)", need,
          p->ws_bytes);
  return MOE_OK;
}
}  // namespace

int moe_block_norm_fwd(const moe_block_norm* p, hipStream_t stream) {
  const int r = check_block(p, true);
  if (r != MOE_OK) return r;
  return hip_status(moe::launch_block_norm_fwd(p, stream), "moe_block_norm_fwd");
}

size_t moe_block_norm_bwd_workspace_size(int T, int d, int dtype) {
  if (check_norm(dtype, T, d) != MOE_OK) return 0;
  return moe::block_norm_ws_bytes(T, d, dtype == MOE_BF16);
}

int moe_block_norm_bwd(const moe_block_norm* p, hipStream_t stream) {
  const int r = check_block(p, false);
  if (r != MOE_OK) return r;
  return hip_status(moe::launch_block_norm_bwd(p, stream), "moe_block_norm_bwd");
}

namespace {
int check_xent_sizes(const moe_xent* p) {
  REQUIRE(p != nullptr, "the arguments must not be NULL");
  int r;
  if ((r = check_dtype(p->dtype)) != MOE_OK) return r;
  REQUIRE(p->N >= 0 && p->d >= 1 && p->V >= 1, "bad sizes N = %d, d = %d, V = %d", p->N, p->d, p->V);
  SUPPORT(p->N < 1 << 23, "N = %d must be below 2^23", p->N);
  SUPPORT(p->d <= 1 << 16, "d = %d: at most 2^16", p->d);
  SUPPORT(p->V < 1 << 30, "V = %d must be below 2^30", p->V);
  SUPPORT((int64_t)p->N * p->d < (int64_t(1) << 31) - 16, "N d = %lld must be below 2^31 - 16",
          (long long)p->N * p->d);
  if (p->dtype == MOE_BF16) SUPPORT(p->d % 64 == 0, "d = %d must be a multiple of 64 for bf16", p->d);
  else SUPPORT(p->d % 8 == 0, "d = %d must be a multiple of 8", p->d);
  return MOE_OK;
}

int check_xent(const moe_xent* p, bool fwd) {
  int r;
  if ((r = check_xent_sizes(p)) != MOE_OK) return r;
  const bool any = p->N > 0;
  REQUIRE(std::isfinite(p->scale) && p->scale != 0.f && std::isfinite(p->z_coef),
          "scale must be finite and not 0, z_coef finite");
  REQUIRE(!any || (p->x && p->w && p->labels && p->lse), "x, w, labels and lse must not be NULL");
  SUPPORT(aligned16(p->x) && aligned16(p->w), "x and w must be 16-byte aligned");
  if (fwd) {
    REQUIRE(p->total && (!any || p->loss), "loss and total must not be NULL");
  } else {
    SUPPORT(p->dw_dtype == MOE_F32 || p->dw_dtype == p->dtype, "dw_dtype = %d is neither fp32 nor dtype",
            p->dw_dtype);
    REQUIRE(p->dw && (!any || p->dx), "dx and dw must not be NULL");
    SUPPORT(aligned16(p->dx) && aligned16(p->dw), "dx and dw must be 16-byte aligned");
  }
  const size_t need = fwd ? moe::xent_fwd_ws_bytes(p) : moe::xent_bwd_ws_bytes(p);
  REQUIRE(p->ws && p->ws_bytes >= need, "workspace of %zu bytes needed (got %zu)", need, p->ws_bytes);
  SUPPORT((uintptr_t)p->ws % 256 == 0, "ws must be 256-byte aligned");
  return MOE_OK;
}
}  // namespace

size_t moe_xent_fwd_workspace_size(const moe_xent* p) {
  return check_xent_sizes(p) == MOE_OK ? moe::xent_fwd_ws_bytes(p) : 0;
}

int moe_xent_fwd(const moe_xent* p, hipStream_t stream) {
  const int r = check_xent(p, true);
  if (r != MOE_OK) return r;
  return hip_status(moe::launch_xent_fwd(p, stream), "moe_xent_fwd");
}

size_t moe_xent_bwd_workspace_size(const moe_xent* p) {
  return check_xent_sizes(p) == MOE_OK ? moe::xent_bwd_ws_bytes(p) : 0;
}

int moe_xent_bwd(const moe_xent* p, hipStream_t stream) {
  const int r = check_xent(p, false);
  if (r != MOE_OK) return r;
  return hip_status(moe::launch_xent_bwd(p, stream), "moe_xent_bwd");
}

namespace {
int check_mx(int dtype, int rows, int cols, const void* x, const uint8_t* codes,
             const uint8_t* scales) {
  int r;
  if ((r = check_dtype(dtype)) != MOE_OK) return r;
  REQUIRE(rows >= 0 && cols >= 1, "bad sizes rows = %d, cols = %d", rows, cols);
  SUPPORT(cols % moe::MX_BLOCK == 0, "cols = %d must be a multiple of 32", cols);
  SUPPORT((int64_t)rows * (cols / 8) <= moe::kMxWords, "rows = %d of cols = %d are too many", rows,
          cols);
  REQUIRE(rows == 0 || (x && codes && scales), "x, codes and scales must not be NULL");
  SUPPORT(aligned16(x) && aligned16(codes), "x and codes must be 16-byte aligned");
  return MOE_OK;
}
}  // namespace

int moe_mxfp4_scale_stride(int cols) { return cols < 1 ? 0 : moe::mx_stride(cols); }

int moe_mxfp4_quantize(const void* x, int dtype, int rows, int cols, const int32_t* n_rows,
                       uint8_t* codes, uint8_t* scales, hipStream_t stream) {
  const int r = check_mx(dtype, rows, cols, x, codes, scales);
  if (r != MOE_OK) return r;
  return hip_status(
      moe::launch_mx_quantize(x, dtype == MOE_BF16, rows, cols, n_rows, codes, scales, stream),
      "moe_mxfp4_quantize");
}

int moe_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int rows,
                         int cols, const int32_t* n_rows, void* x, hipStream_t stream) {
  const int r = check_mx(dtype, rows, cols, x, codes, scales);
  if (r != MOE_OK) return r;
  return hip_status(
      moe::launch_mx_dequantize(codes, scales, dtype == MOE_BF16, rows, cols, n_rows, x, stream),
      "moe_mxfp4_dequantize");
}

size_t moe_mxfp4_ffn_fwd_workspace_size(int cap, int H) {
  return cap < 0 || H < 1 ? 0 : moe::mx_ffn_ws_bytes(cap, H);
}

int moe_mxfp4_ffn_fwd(const moe_mxfp4_ffn* f, hipStream_t stream) {
  REQUIRE(f != nullptr, "the arguments must not be NULL");
  REQUIRE(f->activation == MOE_ACT_SWIGLU || f->activation == MOE_ACT_SILU,
          "activation = %d is not an expert form", f->activation);
  REQUIRE(f->cap >= 0 && f->d >= 1 && f->H >= 1 && f->n_groups >= 0,
          "bad sizes cap = %d, d = %d, H = %d, n_groups = %d", f->cap, f->d, f->H, f->n_groups);
  SUPPORT(f->n_groups <= moe::kMaxGroups, "n_groups = %d: at most %d groups", f->n_groups,
          moe::kMaxGroups);
  SUPPORT(f->d % 64 == 0 && f->H % 64 == 0, "d = %d and H = %d must be multiples of 64", f->d, f->H);
  SUPPORT((int64_t)f->cap * std::max(f->d, f->H) / 2 < 0xFFFFFFF0L &&
              (int64_t)f->H * f->d < 0xFFFFFFF0L / std::max(f->n_groups, 1),
          "MXFP4 operands must each stay below 4 GiB (cap = %d, H = %d, groups = %d)", f->cap, f->H,
          f->n_groups);
  REQUIRE(f->offsets, "offsets must not be NULL");
  REQUIRE(f->n_groups == 0 ||
              (f->w_gate_up && f->w_gate_up_scales && f->w_down && f->w_down_scales),
          "the experts' codes and scales must not be NULL");
  REQUIRE(f->cap == 0 || (f->x && f->x_scales && f->y), "x, its scales and y must not be NULL");
  for (const void* p : {(const void*)f->x, (const void*)f->w_gate_up, (const void*)f->w_down,
                        (const void*)f->y})
    SUPPORT(p == nullptr || aligned16(p), "codes and y must be 16-byte aligned");
  for (const void* p : {f->x_scales, f->w_gate_up_scales, f->w_down_scales})
    SUPPORT((reinterpret_cast<uintptr_t>(p) & 3u) == 0, "scales must be 4-byte aligned");
  const size_t need = moe::mx_ffn_ws_bytes(f->cap, f->H);
  REQUIRE(need == 0 || (f->ws && f->ws_bytes >= need), "workspace of %zu bytes needed (got %zu)", need,
          f->ws_bytes);
  SUPPORT((reinterpret_cast<uintptr_t>(f->ws) & 255u) == 0, "the workspace must be 256-byte aligned");
  return hip_status(moe::launch_mx_ffn(f, stream), "moe_mxfp4_ffn_fwd");
}

namespace {
// Everything of a moe_few but its pointers.
int check_few_sizes(const moe_few* f) {
  int r;
  REQUIRE(f != nullptr, "the arguments must not be NULL");
  if ((r = check_dtype(f->dtype)) != MOE_OK) return r;
  REQUIRE(f->weights == MOE_W_PLAIN || f->weights == MOE_W_MXFP4, "unknown weights %d", f->weights);
  REQUIRE(f->activation == MOE_ACT_SWIGLU || f->activation == MOE_ACT_SILU,
          "activation = %d is not an expert form", f->activation);
  REQUIRE(f->gate >= MOE_GATE_SOFTMAX_TOPK && f->gate <= MOE_GATE_SIGMOID, "unknown gate %d", f->gate);
  SUPPORT(f->weights == MOE_W_PLAIN || f->dtype == MOE_BF16, "MXFP4 weights need dtype MOE_BF16");
  REQUIRE(f->T >= 0 && f->d >= 1 && f->H >= 1 && f->Hs >= 0, "bad sizes T = %d, d = %d, H = %d, Hs = %d",
          f->T, f->d, f->H, f->Hs);
  SUPPORT(f->T <= moe::kFewTokens, "T = %d: at most %d tokens (moe_layer_fwd takes more)", f->T,
          moe::kFewTokens);
  REQUIRE(f->E >= 1 && f->E <= 256, "E = %d must be in [1, 256]", f->E);
  REQUIRE(f->k >= 1 && f->k <= f->E, "k = %d must be in [1, E = %d]", f->k, f->E);
  SUPPORT(f->k <= moe::kFewRoutes, "k = %d: at most %d routes", f->k, moe::kFewRoutes);
  REQUIRE(f->E_r >= 0 && f->E_r <= f->E, "E_r = %d must be in [0, E = %d]", f->E_r, f->E);
  REQUIRE(std::isfinite(f->inv_tau) && f->inv_tau > 0.f, "inv_tau must be finite and > 0");
  SUPPORT(f->d % 64 == 0 && f->H % 64 == 0 && f->Hs % 64 == 0,
          "d = %d, H = %d and Hs = %d must be multiples of 64", f->d, f->H, f->Hs);
  SUPPORT(2L * std::max(f->H, f->Hs) * f->d < 1L << 31, "an expert's matrix must stay below 2^31 elements");
  // (the kernels address a row of h by a 32-bit byte offset)
  SUPPORT((int64_t)f->T * f->k * std::max(f->H, f->Hs) < int64_t(1) << 29,
          "T = %d: T k max(H, Hs) must stay below 2^29", f->T);
  return MOE_OK;
}
}  // namespace

size_t moe_few_fwd_workspace_size(const moe_few* f) {
  return check_few_sizes(f) == MOE_OK ? moe::few_ws_bytes(f) : 0;
}

int moe_few_fwd(const moe_few* f, hipStream_t stream) {
  int r;
  if ((r = check_few_sizes(f)) != MOE_OK) return r;
  const bool mx = f->weights == MOE_W_MXFP4;
  REQUIRE(f->w_router && f->resident, "w_router and resident must not be NULL");
  REQUIRE(f->T == 0 || (f->x && f->y), "x and y must not be NULL");
  REQUIRE(f->E_r == 0 || (f->w_gate_up && f->w_down), "the experts' weights must not be NULL");
  REQUIRE(f->Hs == 0 || (f->shared_gate_up && f->shared_down),
          "the shared experts' weights must not be NULL");
  REQUIRE(!mx || ((f->E_r == 0 || (f->w_gate_up_scales && f->w_down_scales)) &&
                  (f->Hs == 0 || (f->shared_gate_up_scales && f->shared_down_scales))),
          "MXFP4 weights need their scales");
  for (const void* p : {f->x, f->w_router, f->w_gate_up, f->w_down, f->shared_gate_up,
                        f->shared_down, (const void*)f->y})
    SUPPORT(p == nullptr || aligned16(p), "x, y and the weights must be 16-byte aligned");
  for (const void* p : {f->w_gate_up_scales, f->w_down_scales, f->shared_gate_up_scales,
                        f->shared_down_scales})
    SUPPORT((reinterpret_cast<uintptr_t>(p) & 3u) == 0, "scales must be 4-byte aligned");
  const size_t need = moe::few_ws_bytes(f);
  REQUIRE(need == 0 || (f->ws && f->ws_bytes >= need), "workspace of %zu bytes needed (got %zu)", need,
          f->ws_bytes);
  SUPPORT((reinterpret_cast<uintptr_t>(f->ws) & 255u) == 0, "the workspace must be 256-byte aligned");
  return hip_status(moe::launch_few(f, stream), "moe_few_fwd");
}

int moe_expert_delta(const float* theta_start, const float* theta_now,
                     const float* const* peers, int n_peers, size_t n_params, float* delta_local,
                     float* delta_avg, hipStream_t stream) {
  REQUIRE(n_peers >= 0 && n_peers <= moe::kMaxPeers, "n_peers = %d must be in [0, %d]", n_peers,
          moe::kMaxPeers);
  REQUIRE(n_params == 0 || (theta_start && theta_now && delta_avg),
          "theta_start, theta_now and delta_avg must not be NULL");
  REQUIRE(n_peers == 0 || peers, "peers must not be NULL when n_peers > 0");
  for (int p = 0; p < n_peers; ++p) {
    REQUIRE(n_params == 0 || peers[p], "peers[%d] must not be NULL", p);
    SUPPORT(peers[p] == nullptr || aligned16(peers[p]), "peers[%d] must be 16-byte aligned", p);
  }
  for (const void* p : {(const void*)theta_start, (const void*)theta_now, (const void*)delta_local,
                        (const void*)delta_avg})
    SUPPORT(p == nullptr || aligned16(p), "arrays must be 16-byte aligned");
  return hip_status(moe::launch_expert_delta(theta_start, theta_now, peers, n_peers, n_params,
                                             delta_local, delta_avg, stream),
                    "moe_expert_delta");
}

int moe_adamw_step(float* theta, const float* grad, float* m, float* v, size_t n, int step,
                   float lr, float beta1, float beta2, float eps, float weight_decay,
                   void* theta_bf16, hipStream_t stream) {
  REQUIRE(n == 0 || (theta && grad && m && v), "theta, grad, m and v must not be NULL");
  REQUIRE(step >= 1, "step = %d must be >= 1", step);
  REQUIRE(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f && eps >= 0.f,
          "betas must lie in [0, 1) and eps must be >= 0");
  for (const void* p : {(const void*)theta, (const void*)grad, (const void*)m, (const void*)v,
                        (const void*)theta_bf16})
    SUPPORT(p == nullptr || aligned16(p), "arrays must be 16-byte aligned");
  const float c1 = (float)(1.0 - std::pow((double)beta1, (double)step));
  const float c2 = (float)(1.0 - std::pow((double)beta2, (double)step));
  REQUIRE(c1 > 0.f && c2 > 0.f, "bias corrections must be positive (betas > 0 at step %d)", step);
  return hip_status(moe::launch_adamw(theta, grad, m, v, n, lr, beta1, beta2, eps, weight_decay,
                                      c1, c2, theta_bf16, stream),
                    "moe_adamw_step");
}

namespace {
int check_grads(const moe_grad* g, int n, bool out) {
  REQUIRE(n >= 0, "n_grads = %d must be >= 0", n);
  REQUIRE(n == 0 || g, "grads must not be NULL");
  for (int i = 0; i < n; ++i) {
    int r;
    if ((r = check_dtype(g[i].dtype)) != MOE_OK) return r;
    REQUIRE(g[i].n == 0 || (g[i].grad && (!out || g[i].out)), "tensor %d: grad%s must not be NULL", i,
            out ? " and out" : "");
    SUPPORT(g[i].n < (size_t)1 << 44, "tensor %d: %zu values are too many", i, g[i].n);
    const uintptr_t size = g[i].dtype == MOE_BF16 ? 2 : 4;
    SUPPORT(((uintptr_t)g[i].grad | (out ? (uintptr_t)g[i].out : 0)) % size == 0,
            "tensor %d must be aligned to its type", i);
  }
  return MOE_OK;
}
}  // namespace

size_t moe_grad_norm_workspace_size(const moe_grad* grads, int n_grads) {
  if (check_grads(grads, n_grads, false) != MOE_OK) return 0;
  return moe::grad_norm_ws_bytes(grads, n_grads);
}

int moe_grad_norm(const moe_grad* grads, int n_grads, float max_norm, float* norm, void* ws,
                  size_t ws_bytes, hipStream_t stream) {
  const int r = check_grads(grads, n_grads, false);
  if (r != MOE_OK) return r;
  REQUIRE(max_norm > 0.f, "max_norm must be > 0");
  REQUIRE(norm, "norm must not be NULL");
  SUPPORT((uintptr_t)norm % 4 == 0 && (uintptr_t)ws % 8 == 0, "norm and ws must be aligned");
  const size_t need = moe::grad_norm_ws_bytes(grads, n_grads);
  REQUIRE(need == 0 || (ws && ws_bytes >= need), "workspace of %zu bytes needed (got %zu)", need,
          ws_bytes);
  return hip_status(moe::launch_grad_norm(grads, n_grads, max_norm, norm, ws, stream),
                    "moe_grad_norm");
}

int moe_grad_clip(const moe_grad* grads, int n_grads, const float* norm, hipStream_t stream) {
  const int r = check_grads(grads, n_grads, true);
  if (r != MOE_OK) return r;
  REQUIRE(norm, "norm must not be NULL");
  SUPPORT((uintptr_t)norm % 4 == 0, "norm must be aligned");
  return hip_status(moe::launch_grad_clip(grads, n_grads, norm, stream), "moe_grad_clip");
}

int moe_adamw_steps(const moe_adamw_tensor* tensors, int n_tensors, int step, float lr, float beta1,
                    float beta2, float eps, const float* norm, hipStream_t stream) {
  REQUIRE(n_tensors >= 0, "n_tensors = %d must be >= 0", n_tensors);
  REQUIRE(n_tensors == 0 || tensors, "tensors must not be NULL");
  REQUIRE(step >= 1, "step = %d must be >= 1", step);
  REQUIRE(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f && eps >= 0.f,
          "betas must lie in [0, 1) and eps must be >= 0");
  SUPPORT((uintptr_t)norm % 4 == 0, "norm must be aligned");
  for (int i = 0; i < n_tensors; ++i) {
    const moe_adamw_tensor& p = tensors[i];
    int r;
    if ((r = check_dtype(p.grad_dtype)) != MOE_OK) return r;
    REQUIRE(p.n == 0 || (p.theta && p.grad && p.m && p.v),
            "tensor %d: theta, grad, m and v must not be NULL", i);
    SUPPORT(p.n < (size_t)1 << 43, "tensor %d: %zu values are too many", i, p.n);
    for (const void* q : {(const void*)p.theta, p.grad, (const void*)p.m, (const void*)p.v,
                          (const void*)p.theta_bf16})
      SUPPORT(q == nullptr || aligned16(q), "tensor %d: arrays must be 16-byte aligned", i);
  }
  const float c1 = (float)(1.0 - std::pow((double)beta1, (double)step));
  const float c2 = (float)(1.0 - std::pow((double)beta2, (double)step));
  REQUIRE(c1 > 0.f && c2 > 0.f, "bias corrections must be positive (betas > 0 at step %d)", step);
  return hip_status(moe::launch_adamw_steps(tensors, n_tensors, lr, beta1, beta2, eps, c1, c2, norm,
                                            stream),
                    "moe_adamw_steps");
}

int moe_outer_nesterov(float* theta_start, float* theta_now, const float* delta_avg,
                       float* momentum, size_t n, float lr, float mu, void* theta_bf16,
                       hipStream_t stream) {
  REQUIRE(n == 0 || (theta_start && theta_now && delta_avg && momentum),
          "theta_start, theta_now, delta_avg and momentum must not be NULL");
  for (const void* p : {(const void*)theta_start, (const void*)theta_now,
                        (const void*)delta_avg, (const void*)momentum, (const void*)theta_bf16})
    SUPPORT(p == nullptr || aligned16(p), "arrays must be 16-byte aligned");
  return hip_status(moe::launch_outer_nesterov(theta_start, theta_now, delta_avg, momentum, n, lr,
                                               mu, theta_bf16, stream),
                    "moe_outer_nesterov");
}

int moe_replica_mean(const float* local, const float* const* peers, int n_peers, size_t n,
                     float* out, hipStream_t stream) {
  REQUIRE(n_peers >= 0 && n_peers <= moe::kMaxPeers, "n_peers = %d must be in [0, %d]", n_peers,
          moe::kMaxPeers);
  REQUIRE(n == 0 || (local && out), "local and out must not be NULL");
  REQUIRE(n_peers == 0 || peers, "peers must not be NULL when n_peers > 0");
  for (int p = 0; p < n_peers; ++p) {
    REQUIRE(n == 0 || peers[p], "peers[%d] must not be NULL", p);
    SUPPORT(peers[p] == nullptr || aligned16(peers[p]), "peers[%d] must be 16-byte aligned", p);
  }
  SUPPORT((local == nullptr || aligned16(local)) && (out == nullptr || aligned16(out)),
          "arrays must be 16-byte aligned");
  return hip_status(moe::launch_replica_mean(local, peers, n_peers, n, out, stream),
                    "moe_replica_mean");
}

static bool is_permutation(const int32_t* p, int n) {
  if (!p) return true;
  std::vector<char> seen(n, 0);
  for (int i = 0; i < n; ++i) {
    if (p[i] < 0 || p[i] >= n || seen[p[i]]) return false;
    seen[p[i]] = 1;
  }
  return true;
}

int moe_gen_placement(int N_e, int O_e, int M, const int32_t* expert_perm,
                      const int32_t* worker_perm, int32_t* sets) {
  REQUIRE(sets, "sets must not be NULL");
  REQUIRE(N_e >= 1 && M >= 1 && O_e >= 1 && O_e <= M,
          "need N_e >= 1 and 1 <= O_e <= M (N_e = %d, O_e = %d, M = %d)", N_e, O_e, M);
  REQUIRE(((long)N_e * O_e) % M == 0, "M = %d must divide N_e O_e = %ld", M, (long)N_e * O_e);
  REQUIRE(is_permutation(expert_perm, N_e), "expert_perm is not a permutation of 0..N_e-1");
  REQUIRE(is_permutation(worker_perm, M), "worker_perm is not a permutation of 0..M-1");
  REQUIRE(moe::gen_placement(N_e, O_e, M, expert_perm, worker_perm, sets), "placement failed");
  return MOE_OK;
}

int moe_migration_map(const int32_t* prev_set, int n_prev, const int32_t* new_set, int n_new,
                      int32_t* map) {
  REQUIRE(n_prev >= 0 && n_new >= 0, "set sizes must be >= 0");
  REQUIRE((n_prev == 0 || prev_set) && (n_new == 0 || (new_set && map)),
          "sets and map must not be NULL");
  for (int i = 0; i < n_new; ++i) {
    REQUIRE(i == 0 || new_set[i] > new_set[i - 1], "new_set must be strictly ascending");
    map[i] = -1;
    for (int j = 0; j < n_prev; ++j)
      if (prev_set[j] == new_set[i]) map[i] = j;
  }
  return MOE_OK;
}

int moe_copy_expert_rows(const float* src, const int32_t* src_row, float* dst,
                         const int32_t* dst_row, int n_rows, size_t row_len, void* dst_bf16,
                         hipStream_t stream) {
  REQUIRE(n_rows >= 0 && n_rows <= 256, "n_rows = %d must be in [0, 256]", n_rows);
  REQUIRE(n_rows == 0 || row_len == 0 || (src_row && dst), "src_row and dst must not be NULL");
  bool any_src = false;
  for (int r = 0; r < n_rows; ++r) {
    any_src = any_src || src_row[r] >= 0;
    REQUIRE(src_row[r] >= -1, "src_row[%d] = %d must be >= -1", r, src_row[r]);
    if (dst_row) {
      REQUIRE(dst_row[r] >= 0, "dst_row[%d] = %d must be >= 0", r, dst_row[r]);
      for (int q = 0; q < r; ++q) REQUIRE(dst_row[q] != dst_row[r], "dst_row repeats %d", dst_row[r]);
    }
  }
  REQUIRE(!any_src || src, "src must not be NULL when a row is copied");
  SUPPORT((!src || aligned16(src)) && (!dst || aligned16(dst)) &&
              (!dst_bf16 || aligned16(dst_bf16)) && row_len % 4 == 0,
          "src, dst and dst_bf16 must be 16-byte aligned and row_len a multiple of 4");
  return hip_status(moe::launch_copy_expert_rows(src, src_row, dst, dst_row, n_rows, row_len,
                                                 dst_bf16, stream),
                    "moe_copy_expert_rows");
}

int moe_warmup_lr(const int* steps, int n_rows, double lr, int warmup_steps, float* lr_out) {
  REQUIRE(n_rows >= 0, "n_rows = %d must be >= 0", n_rows);
  REQUIRE(n_rows == 0 || (steps && lr_out), "steps and lr_out must not be NULL");
  REQUIRE(std::isfinite(lr), "lr must be finite");
  for (int r = 0; r < n_rows; ++r) REQUIRE(steps[r] >= 0, "steps[%d] = %d must be >= 0", r, steps[r]);
  for (int r = 0; r < n_rows; ++r) {
    const double f = warmup_steps > 0 ? std::min(1.0, (double)steps[r] / (double)warmup_steps) : 1.0;
    lr_out[r] = (float)(lr * f);
  }
  return MOE_OK;
}

int moe_adamw_step_rows(float* theta, const float* grad, float* m, float* v, int n_rows,
                        size_t row_len, const int* steps, const float* lr, float beta1,
                        float beta2, float eps, float weight_decay, void* theta_bf16,
                        hipStream_t stream) {
  REQUIRE(n_rows >= 0 && (n_rows == 0 || (steps && lr)), "steps and lr must not be NULL");
  REQUIRE(n_rows == 0 || row_len == 0 || (theta && grad && m && v),
          "theta, grad, m and v must not be NULL");
  REQUIRE(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f && eps >= 0.f,
          "betas must lie in [0, 1) and eps must be >= 0");
  SUPPORT(row_len % 4 == 0, "row_len must be a multiple of 4");
  for (const void* p : {(const void*)theta, (const void*)grad, (const void*)m, (const void*)v,
                        (const void*)theta_bf16})
    SUPPORT(p == nullptr || aligned16(p), "arrays must be 16-byte aligned");
  for (int r = 0; r < n_rows; ++r) REQUIRE(steps[r] >= 1, "steps[%d] = %d must be >= 1", r, steps[r]);
  // one launch per run of rows that share (step, lr)
  for (int r0 = 0; r0 < n_rows;) {
    int r1 = r0 + 1;
    while (r1 < n_rows && steps[r1] == steps[r0] && lr[r1] == lr[r0]) ++r1;
    const float c1 = (float)(1.0 - std::pow((double)beta1, (double)steps[r0]));
    const float c2 = (float)(1.0 - std::pow((double)beta2, (double)steps[r0]));
    REQUIRE(c1 > 0.f && c2 > 0.f, "bias corrections must be positive");
    const size_t o = (size_t)r0 * row_len, n = (size_t)(r1 - r0) * row_len;
    void* lp = theta_bf16 ? static_cast<uint16_t*>(theta_bf16) + o : nullptr;  // bf16 elements
    const int st = hip_status(moe::launch_adamw(theta + o, grad + o, m + o, v + o, n, lr[r0],
                                                beta1, beta2, eps, weight_decay, c1, c2, lp,
                                                stream),
                              "moe_adamw_step_rows");
    if (st != MOE_OK) return st;
    r0 = r1;
  }
  return MOE_OK;
}

}  // extern "C"
