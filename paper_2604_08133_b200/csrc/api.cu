// C-ABI entry points (see include/allocmoe.h): argument checks, workspace carve-up, launches.
// Nothing here allocates or synchronises; every launch goes to the caller's stream.
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <cmath>
#include <initializer_list>

#include "allocmoe.h"

#include "adapter.h"
#include "ffn.h"
#include "router_grad.h"
#include "shape_check.h"
#include "train.h"

// launchers defined next to their kernels
moe_status launch_moe_gate(const moe_shape*, const uint16_t*, const uint16_t*, const float*, float*, int32_t*, float*,
                           int32_t*, int, int32_t*, cudaStream_t);
moe_status launch_alloc_t_select(const moe_shape*, const float*, int64_t, int32_t*, int32_t*, cudaStream_t);
moe_status launch_moe_permute(const moe_shape*, const uint16_t*, const int32_t*, const float*, const int32_t*, int64_t,
                              int32_t*, int32_t*, float*, int32_t*, uint16_t*, int32_t*, int32_t*, bool, cudaStream_t);
moe_status launch_gather_rows(const moe_shape*, const uint16_t*, const int32_t*, int64_t, const int32_t*, uint16_t*,
                              int32_t*, cudaStream_t);
bool moe_route_fits(const moe_shape*);
moe_status launch_moe_route(const moe_shape*, const float*, const int32_t*, int64_t, bool, int32_t*, int32_t*, int32_t*,
                            float*, int32_t*, int32_t*, cudaStream_t);
moe_status launch_moe_combine(const moe_shape*, const uint16_t*, const int32_t*, const float*, const int32_t*,
                              const uint16_t*, const uint16_t*, long long, uint16_t*, cudaStream_t);
moe_status launch_rmsnorm(const moe_shape*, const uint16_t*, uint16_t*, cudaStream_t);
moe_status launch_token_rule_select(const moe_shape*, const float*, int, float, int32_t*, int32_t*, int32_t*, cudaStream_t);

namespace {

using allocmoe::aligned16;
using allocmoe::shape_ok;

bool budget_ok(const moe_shape* s, int64_t budget) {
  return budget >= (int64_t)s->K_base * s->T && budget <= (int64_t)s->K_orig * s->T;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool n_seq_ok(int32_t n_seq) { return n_seq >= 1 && n_seq <= (1 << 20); }
constexpr int32_t kMaxRows = 1 << 30;   // row and column numbers of the calls below stay clear of 2^31 when rounded up to a tile
bool router_shape_ok(const moe_shape* s) { return shape_ok(s) && s->T <= kMaxRows; }
bool adapters_ok(int32_t n, int32_t rank) { return n >= 1 && n <= (1 << 20) && rank >= 8 && rank <= 128 && rank % 8 == 0; }
bool adapter_shape_ok(const moe_adapter_shape* s) {
  return s != nullptr && s->flags == 0 && s->T >= 1 && s->T <= kMaxRows && s->K >= 8 && s->K <= kMaxRows && s->K % 8 == 0 &&
         s->M >= 8 && s->M <= kMaxRows && s->M % 8 == 0 && adapters_ok(s->n_adapters, s->rank);
}
bool adapted_shape_ok(const moe_shape* s) {
  return shape_ok(s) && s->S >= 1 && s->T <= kMaxRows && 2 * (int64_t)s->S * s->I <= kMaxRows;
}
size_t shared_adapted_h_bytes(const moe_shape* s) {
  return ((size_t)s->T * s->S * s->I * 2 + 255) & ~(size_t)255;
}

bool all_aligned16(std::initializer_list<const void*> ptrs) {
  for (const void* ptr : ptrs)
    if (!aligned16(ptr)) return false;
  return true;
}
// Outputs, NULL where there is none, none of which may be another.
bool all_different(std::initializer_list<const void*> ptrs) {
  for (auto a = ptrs.begin(); a != ptrs.end(); ++a)
    for (auto b = ptrs.begin(); b != a; ++b)
      if (*a != nullptr && *a == *b) return false;
  return true;
}
bool grouped_shape_ok(const moe_grouped_shape* s, uint32_t flags) {
  if (s == nullptr || (s->flags & ~flags) != 0 || (s->flags & (MOE_GROUPED_DW_FP32 | MOE_GROUPED_DW_ADD)) == MOE_GROUPED_DW_ADD) return false;
  if (s->P < 1 || s->P > kMaxRows || s->K < 8 || s->K > kMaxRows || s->K % 8 != 0 || s->M < 8 || s->M > kMaxRows || s->M % 8 != 0 ||
      s->E < 1 || s->E > 128)
    return false;
  // numbers of tiles, and strides of a group's weight in bytes, stay within what a launch counts in
  const int64_t widest = s->K > s->M ? s->K : s->M;
  return (s->P / 128 + s->E) * (widest / 64 + 1) < (1ll << 31) && (int64_t)s->E * (s->K / 128 + 1) * (s->M / 128 + 1) < (1ll << 31) &&
         (int64_t)s->K * s->M < (1ll << 37);
}
bool ffn_backward_ok(const moe_shape* s, int64_t budget) {
  return shape_ok(s) && s->T <= kMaxRows && budget >= 0 && budget <= (int64_t)s->K_orig * s->T && budget <= kMaxRows &&
         (budget / 128 + s->N) * (int64_t)(2 * s->I / 64 + s->H / 64 + 2) < (1ll << 31) &&
         (int64_t)s->N * (2 * s->I / 128 + 1) * (s->H / 128 + 1) < (1ll << 31) && 2ll * s->I <= kMaxRows && 2ll * s->I * s->H < (1ll << 37);
}
// Workspace of the experts' backward pass: x_perm [B,H], h [B,I], du [B,2I]; regions start on 256-byte boundaries.
struct FfnBackwardWs { size_t x_perm, h, du, total; };
FfnBackwardWs ffn_backward_ws(const moe_shape* s, int64_t budget) {
  const size_t B = (size_t)budget;
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  FfnBackwardWs w{};
  w.h = up(B * s->H * 2);
  w.du = w.h + up(B * s->I * 2);
  w.total = w.du + up(2 * B * s->I * 2) + 256;
  return w;
}
bool shared_backward_ok(const moe_shape* s) {
  return shape_ok(s) && s->S >= 1 && s->T <= kMaxRows && 2ll * s->S * s->I <= kMaxRows && 2ll * s->S * s->I * s->H < (1ll << 37) &&
         (s->T / 128 + 1) * (int64_t)(2ll * s->S * (s->I / 64 + 2) + s->H / 64 + 2) < (1ll << 31) &&
         (2ll * s->S * s->I / 128 + 1) * (s->H / 128 + 1) < (1ll << 31);
}
size_t shared_backward_h_bytes(const moe_shape* s) { return ((size_t)s->T * s->S * s->I * 2 + 255) & ~(size_t)255; }
bool norm_shape_ok(const moe_norm_shape* s) {
  return s != nullptr && (s->flags & ~MOE_NORM_Y_AS_IS) == 0 && s->T >= 1 && s->T <= kMaxRows && s->H >= 8 && s->H <= 8192 && s->H % 8 == 0 &&
         (s->gate_cols == 0 || s->gate_cols == 1 || s->gate_cols == s->H) && std::isfinite(s->eps) && s->eps > 0.f;
}
// Entries of an optimizer's list as far as the host can see them; states8: for the calls that move 8-bit states alone.
bool adamw_entries_ok(const moe_adamw_tensor* t, int32_t count, bool states8) {
  if (t == nullptr || count < 1 || count > (1 << 20)) return false;
  for (int32_t k = 0; k < count; ++k) {
    const uint32_t f = t[k].flags;
    if (t[k].n < 1 || (f & ~(MOE_ADAMW_PARAM_BF16 | MOE_ADAMW_GRAD_BF16 | MOE_ADAMW_STATE8)) != 0 || !t[k].m || !t[k].v) return false;
    if (!all_aligned16({t[k].m, t[k].v})) return false;
    if ((f & MOE_ADAMW_STATE8) != 0 && (!t[k].m_scale || !t[k].v_scale || !aligned4(t[k].m_scale) || !aligned4(t[k].v_scale))) return false;
    if (states8) {
      if ((f & MOE_ADAMW_STATE8) == 0) return false;
    } else if (!t[k].param || !t[k].grad || t[k].param == t[k].grad || !all_aligned16({t[k].param, t[k].grad, t[k].copy}) ||
               !std::isfinite(t[k].weight_decay)) {
      return false;
    }
  }
  return adamw_chunks_ok(t, count);
}

// Fixed carve-up of the workspace; every region starts on a 256-byte boundary.
struct WsLayout {
  size_t topk_idx, topk_score, n_sel, expert_offsets, perm_token, perm_weight, pair_pos, seg_counts;
  size_t x_perm, h, y_perm, h_sh, y_shared, gemm_done, total;
};

WsLayout ws_layout(const moe_shape* s, int64_t budget_max) {
  WsLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    size_t at = off;
    off += (bytes + 255) & ~(size_t)255;
    return at;
  };
  const size_t T = s->T, H = s->H, N = s->N, I = s->I, S = s->S, K = s->K_orig, B = (size_t)budget_max;
  L.topk_idx = take(T * K * 4);
  L.topk_score = take(T * K * 4);
  L.n_sel = take(T * 4);
  L.expert_offsets = take((N + 1) * 4);
  L.perm_token = take(B * 4);
  L.perm_weight = take(B * 4);
  L.pair_pos = take(T * K * 4);
  L.seg_counts = take(N * ((T + 31) / 32) * 4);
  L.x_perm = take(B * H * 2);
  L.h = take(B * I * 2);
  L.y_perm = take(B * H * 2);
  L.h_sh = take(T * S * I * 2);
  L.y_shared = take(T * H * 2);
  L.gemm_done = take(ffn_done_ints(s, budget_max) * 4);
  L.total = off;
  return L;
}

// One NVTX range per C-ABI call (header-only NVTX: a no-op costing a few nanoseconds unless a profiler is
// attached), so that a timeline shows which entry point enqueued which kernels.
struct ApiRange {
  explicit ApiRange(const char* name) { nvtxRangePushA(name); }
  ~ApiRange() { nvtxRangePop(); }
  ApiRange(const ApiRange&) = delete;
  ApiRange& operator=(const ApiRange&) = delete;
};

template <typename T>
T* at(void* ws, size_t off) { return reinterpret_cast<T*>(static_cast<unsigned char*>(ws) + off); }

// Optional stage timing of moe_layer_forward (off by default): events at the stage boundaries.
constexpr int kProfStages = 6;   // gate, route, gather, ffn GEMM-1, ffn GEMM-2, combine
bool g_prof_on = false;
cudaEvent_t g_prof_ev[kProfStages + 1];
void prof_mark(int i, cudaStream_t st) {
  if (g_prof_on) cudaEventRecord(g_prof_ev[i], st);
}

}  // namespace

extern "C" {

const char* moe_status_string(moe_status s) {
  switch (s) {
    case MOE_OK: return "ok";
    case MOE_ERR_ARG: return "invalid argument (null or misaligned pointer, unsupported shape)";
    case MOE_ERR_BUDGET: return "budget outside [K_base*T, K_orig*T] or kept counts do not add up to it";
    case MOE_ERR_WORKSPACE: return "workspace too small";
    case MOE_ERR_CUDA: return "CUDA call failed";
    case MOE_ERR_NONFINITE: return "routing score is NaN, Inf or negative, or an updated value is not finite";
    case MOE_ERR_TIMEOUT: return "bounded device wait gave up";
  }
  return "unknown status";
}

size_t moe_workspace_bytes(const moe_shape* shape, int64_t budget_max) {
  if (!shape_ok(shape) || budget_max < 0 || budget_max > (int64_t)shape->K_orig * shape->T) return 0;
  return ws_layout(shape, budget_max).total;
}

moe_status moe_gate(const moe_shape* shape, const uint16_t* x, const uint16_t* W_gate, const float* gate_bias,
                    float* scores, int32_t* topk_idx, float* topk_score, void* stream) {
  ApiRange nvtx_range("moe_gate");
  if (!shape_ok(shape) || !x || !W_gate || !topk_idx || !topk_score) return MOE_ERR_ARG;
  if (!aligned16(x) || !aligned16(W_gate) || !aligned16(topk_idx) || !aligned16(topk_score)) return MOE_ERR_ARG;
  return launch_moe_gate(shape, x, W_gate, gate_bias, scores, topk_idx, topk_score, nullptr, 0, nullptr,
                         (cudaStream_t)stream);
}

moe_status alloc_t_select(const moe_shape* shape, const float* topk_score, int64_t budget, int32_t* n_sel,
                          int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("alloc_t_select");
  (void)ws;
  (void)ws_bytes;
  if (!shape_ok(shape) || !topk_score || !n_sel || !dev_status) return MOE_ERR_ARG;
  if (!aligned16(topk_score) || !aligned16(n_sel)) return MOE_ERR_ARG;
  if (!budget_ok(shape, budget)) return MOE_ERR_BUDGET;
  return launch_alloc_t_select(shape, topk_score, budget, n_sel, dev_status, (cudaStream_t)stream);
}

moe_status moe_permute(const moe_shape* shape, const uint16_t* x, const int32_t* topk_idx, const float* topk_score,
                       const int32_t* n_sel, int64_t budget, int32_t* expert_offsets, int32_t* perm_token,
                       float* perm_weight, int32_t* pair_pos, uint16_t* x_perm, int32_t* dev_status, void* ws,
                       size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_permute");
  if (!shape_ok(shape) || !topk_idx || !topk_score || !n_sel || !expert_offsets || !perm_token || !perm_weight ||
      !pair_pos || !dev_status || !ws)
    return MOE_ERR_ARG;
  if (x_perm != nullptr && (!x || !aligned16(x) || !aligned16(x_perm))) return MOE_ERR_ARG;
  if (!aligned16(ws)) return MOE_ERR_ARG;
  if (!budget_ok(shape, budget)) return MOE_ERR_BUDGET;
  const WsLayout L = ws_layout(shape, budget);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  return launch_moe_permute(shape, x, topk_idx, topk_score, n_sel, budget, expert_offsets, perm_token, perm_weight,
                            pair_pos, x_perm, dev_status, at<int32_t>(ws, L.seg_counts), true, (cudaStream_t)stream);
}

moe_status moe_route(const moe_shape* shape, const int32_t* topk_idx, const float* topk_score, int64_t budget,
                     int32_t* n_sel, int32_t* expert_offsets, int32_t* perm_token, float* perm_weight, int32_t* pair_pos,
                     int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_route");
  if (!shape_ok(shape) || !topk_idx || !topk_score || !n_sel || !expert_offsets || !perm_token || !perm_weight ||
      !pair_pos || !dev_status)
    return MOE_ERR_ARG;
  if (!aligned16(topk_idx) || !aligned16(topk_score) || !aligned16(n_sel)) return MOE_ERR_ARG;
  if (!moe_route_fits(shape)) return MOE_ERR_ARG;
  if (!budget_ok(shape, budget)) return MOE_ERR_BUDGET;
  return launch_moe_route(shape, topk_score, topk_idx, budget, false, n_sel, expert_offsets, perm_token, perm_weight,
                          pair_pos, dev_status, (cudaStream_t)stream);
}

moe_status moe_grouped_ffn(const moe_shape* shape, const uint16_t* x_or_xperm, const int32_t* perm_token,
                           const int32_t* expert_offsets, int64_t budget, const uint16_t* W13, const uint16_t* W2,
                           uint16_t* y_perm, int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_grouped_ffn");
  if (!shape_ok(shape) || !x_or_xperm || !expert_offsets || !W13 || !W2 || !y_perm || !dev_status || !ws)
    return MOE_ERR_ARG;
  if (!aligned16(x_or_xperm) || !aligned16(W13) || !aligned16(W2) || !aligned16(y_perm) || !aligned16(ws))
    return MOE_ERR_ARG;
  if (budget < 0 || budget > (int64_t)shape->K_orig * shape->T) return MOE_ERR_BUDGET;
  const WsLayout L = ws_layout(shape, budget);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  FfnArgs a;
  a.s = shape;
  a.a_routed = x_or_xperm;
  a.gather_idx = perm_token;
  if (perm_token != nullptr && budget > 0 && !ffn_gathers(shape, budget)) {
    // long expert runs: one copy of the rows into the workspace, then 128-row box loads, is faster than
    // fetching every tile's rows four at a time
    const moe_status r = launch_gather_rows(shape, x_or_xperm, perm_token, budget, nullptr, at<uint16_t>(ws, L.x_perm), dev_status, st);
    if (r != MOE_OK) return r;
    a.a_routed = at<uint16_t>(ws, L.x_perm);
    a.gather_idx = nullptr;
  }
  a.expert_offsets = expert_offsets;
  a.budget = budget;
  a.W13 = W13;
  a.W2 = W2;
  a.h = at<uint16_t>(ws, L.h);
  a.y_perm = y_perm;
  a.dev_status = dev_status;
  a.done = at<int32_t>(ws, L.gemm_done);
  a.stream = st;
  return launch_ffn(a);
}

moe_status moe_shared_ffn(const moe_shape* shape, const uint16_t* x, const uint16_t* Wsh13, const uint16_t* Wsh2,
                          uint16_t* y_shared, int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_shared_ffn");
  if (!shape_ok(shape) || shape->S < 1 || !x || !Wsh13 || !Wsh2 || !y_shared || !dev_status || !ws) return MOE_ERR_ARG;
  if (!aligned16(x) || !aligned16(Wsh13) || !aligned16(Wsh2) || !aligned16(y_shared) || !aligned16(ws)) return MOE_ERR_ARG;
  const WsLayout L = ws_layout(shape, 0);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  FfnArgs a;
  a.s = shape;
  a.x_shared = x;
  a.Wsh13 = Wsh13;
  a.Wsh2 = Wsh2;
  a.h_sh = at<uint16_t>(ws, L.h_sh);
  a.y_shared = y_shared;
  a.dev_status = dev_status;
  a.done = at<int32_t>(ws, L.gemm_done);
  a.stream = (cudaStream_t)stream;
  return launch_ffn(a);
}

moe_status moe_combine(const moe_shape* shape, const uint16_t* y_perm, const int32_t* pair_pos,
                       const float* topk_score, const int32_t* n_sel, const uint16_t* y_shared, uint16_t* out,
                       void* stream) {
  ApiRange nvtx_range("moe_combine");
  if (!shape_ok(shape) || !y_perm || !pair_pos || !topk_score || !n_sel || !out) return MOE_ERR_ARG;
  if (!aligned16(y_perm) || !aligned16(out) || (y_shared && !aligned16(y_shared))) return MOE_ERR_ARG;
  return launch_moe_combine(shape, y_perm, pair_pos, topk_score, n_sel, y_shared, nullptr,
                            (long long)shape->K_orig * shape->T, out, (cudaStream_t)stream);
}

moe_status moe_layer_forward(const moe_shape* shape, const uint16_t* x, const uint16_t* W_gate, const float* gate_bias,
                             const uint16_t* W13, const uint16_t* W2, const uint16_t* Wsh13, const uint16_t* Wsh2,
                             int64_t budget, const uint16_t* residual, uint16_t* out, int32_t* dev_status, void* ws,
                             size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_layer_forward");
  if (!shape_ok(shape) || !x || !W_gate || !W13 || !W2 || !out || !dev_status || !ws) return MOE_ERR_ARG;
  if (shape->S > 0 && (!Wsh13 || !Wsh2)) return MOE_ERR_ARG;
  if (!aligned16(x) || !aligned16(W_gate) || !aligned16(W13) || !aligned16(W2) || !aligned16(out) || !aligned16(ws))
    return MOE_ERR_ARG;
  if (shape->S > 0 && (!aligned16(Wsh13) || !aligned16(Wsh2))) return MOE_ERR_ARG;
  if (residual != nullptr && (!aligned16(residual) || residual == out)) return MOE_ERR_ARG;
  if (!budget_ok(shape, budget)) return MOE_ERR_BUDGET;
  const WsLayout L = ws_layout(shape, budget);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  int32_t* topk_idx = at<int32_t>(ws, L.topk_idx);
  float* topk_score = at<float>(ws, L.topk_score);
  int32_t* n_sel = at<int32_t>(ws, L.n_sel);
  int32_t* expert_offsets = at<int32_t>(ws, L.expert_offsets);
  int32_t* perm_token = at<int32_t>(ws, L.perm_token);
  float* perm_weight = at<float>(ws, L.perm_weight);
  int32_t* pair_pos = at<int32_t>(ws, L.pair_pos);
  uint16_t* x_perm = at<uint16_t>(ws, L.x_perm);
  uint16_t* y_perm = at<uint16_t>(ws, L.y_perm);
  uint16_t* y_shared = shape->S > 0 ? at<uint16_t>(ws, L.y_shared) : nullptr;

  // for short expert runs GEMM-1 fetches the routed tokens' rows from x by index and no permuted copy is made
  if (ffn_gathers(shape, budget)) x_perm = nullptr;

  prof_mark(0, st);
  // the gate launch also clears the expert GEMMs' row-block counters (no memset between kernels of the call)
  moe_status r = launch_moe_gate(shape, x, W_gate, gate_bias, nullptr, topk_idx, topk_score, at<int32_t>(ws, L.gemm_done),
                                 (int)ffn_done_ints(shape, budget), dev_status, st);
  if (r != MOE_OK) return r;
  prof_mark(1, st);
  if (moe_route_fits(shape)) {
    // selection and permutation bookkeeping in one launch, then the row gather
    r = launch_moe_route(shape, topk_score, topk_idx, budget, false, n_sel, expert_offsets, perm_token, perm_weight,
                         pair_pos, dev_status, st);
    if (r != MOE_OK) return r;
    prof_mark(2, st);
    if (budget > 0 && x_perm != nullptr) r = launch_gather_rows(shape, x, perm_token, budget, nullptr, x_perm, dev_status, st);
  } else {
    r = launch_alloc_t_select(shape, topk_score, budget, n_sel, dev_status, st);
    if (r != MOE_OK) return r;
    prof_mark(2, st);
    r = launch_moe_permute(shape, x, topk_idx, topk_score, n_sel, budget, expert_offsets, perm_token, perm_weight,
                           pair_pos, x_perm, dev_status, at<int32_t>(ws, L.seg_counts), true, st);
  }
  if (r != MOE_OK) return r;
  prof_mark(3, st);
  FfnArgs a;
  a.s = shape;
  a.a_routed = x_perm != nullptr ? x_perm : x;
  a.gather_idx = x_perm != nullptr ? nullptr : perm_token;
  a.expert_offsets = expert_offsets;
  a.budget = budget;
  a.W13 = W13;
  a.W2 = W2;
  a.h = at<uint16_t>(ws, L.h);
  a.y_perm = y_perm;
  a.x_shared = shape->S > 0 ? x : nullptr;
  a.Wsh13 = Wsh13;
  a.Wsh2 = Wsh2;
  a.h_sh = at<uint16_t>(ws, L.h_sh);
  a.y_shared = y_shared;
  a.dev_status = dev_status;
  a.done = at<int32_t>(ws, L.gemm_done);
  a.done_is_clear = true;
  a.stream = st;
  a.between = g_prof_on ? g_prof_ev[4] : nullptr;
  r = launch_ffn(a);
  if (r != MOE_OK) return r;
  prof_mark(5, st);
  r = launch_moe_combine(shape, y_perm, pair_pos, topk_score, n_sel, y_shared, residual, budget, out,
                         st);
  prof_mark(6, st);
  return r;
}

moe_status moe_layer_forward_routed(const moe_shape* shape, const uint16_t* x, const int32_t* topk_idx,
                                    const float* topk_score, const int32_t* n_sel, int64_t budget_max,
                                    int64_t budget_hint, const uint16_t* W13, const uint16_t* W2, const uint16_t* Wsh13,
                                    const uint16_t* Wsh2, const uint16_t* residual, uint16_t* out, int32_t* dev_status,
                                    void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_layer_forward_routed");
  if (!shape_ok(shape) || !x || !topk_idx || !topk_score || !n_sel || !W13 || !W2 || !out || !dev_status || !ws)
    return MOE_ERR_ARG;
  if (shape->S > 0 && (!Wsh13 || !Wsh2)) return MOE_ERR_ARG;
  // n_sel is read one int at a time: a slice of a longer array (this rank's part of the pool's counts) is fine
  if (!aligned16(x) || !aligned16(topk_idx) || !aligned16(topk_score) || !aligned16(W13) || !aligned16(W2) ||
      !aligned16(out) || !aligned16(ws) || (reinterpret_cast<uintptr_t>(n_sel) & 3u) != 0)
    return MOE_ERR_ARG;
  if (shape->S > 0 && (!aligned16(Wsh13) || !aligned16(Wsh2))) return MOE_ERR_ARG;
  if (residual != nullptr && (!aligned16(residual) || residual == out)) return MOE_ERR_ARG;
  if (budget_max < 0 || budget_max > (int64_t)shape->K_orig * shape->T) return MOE_ERR_BUDGET;
  if (budget_hint < 0) return MOE_ERR_BUDGET;
  const WsLayout L = ws_layout(shape, budget_max);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  const int64_t expected = (budget_hint > 0 && budget_hint < budget_max) ? budget_hint : budget_max;
  int32_t* expert_offsets = at<int32_t>(ws, L.expert_offsets);
  int32_t* perm_token = at<int32_t>(ws, L.perm_token);
  float* perm_weight = at<float>(ws, L.perm_weight);
  int32_t* pair_pos = at<int32_t>(ws, L.pair_pos);
  uint16_t* x_perm = at<uint16_t>(ws, L.x_perm);
  uint16_t* y_perm = at<uint16_t>(ws, L.y_perm);
  uint16_t* y_shared = shape->S > 0 ? at<uint16_t>(ws, L.y_shared) : nullptr;
  if (ffn_gathers(shape, expected)) x_perm = nullptr;

  moe_status r;
  if (moe_route_fits(shape)) {
    r = launch_moe_route(shape, topk_score, topk_idx, budget_max, true, const_cast<int32_t*>(n_sel), expert_offsets,
                         perm_token, perm_weight, pair_pos, dev_status, st);
    if (r != MOE_OK) return r;
    if (budget_max > 0 && x_perm != nullptr)
      r = launch_gather_rows(shape, x, perm_token, budget_max, expert_offsets + shape->N, x_perm, dev_status, st);
  } else {
    r = launch_moe_permute(shape, x, topk_idx, topk_score, n_sel, budget_max, expert_offsets, perm_token, perm_weight,
                           pair_pos, x_perm, dev_status, at<int32_t>(ws, L.seg_counts), false, st);
  }
  if (r != MOE_OK) return r;
  FfnArgs a;
  a.s = shape;
  a.a_routed = x_perm != nullptr ? x_perm : x;
  a.gather_idx = x_perm != nullptr ? nullptr : perm_token;
  a.expert_offsets = expert_offsets;
  a.budget = budget_max;
  a.budget_hint = expected;
  a.W13 = W13;
  a.W2 = W2;
  a.h = at<uint16_t>(ws, L.h);
  a.y_perm = y_perm;
  a.x_shared = shape->S > 0 ? x : nullptr;
  a.Wsh13 = Wsh13;
  a.Wsh2 = Wsh2;
  a.h_sh = at<uint16_t>(ws, L.h_sh);
  a.y_shared = y_shared;
  a.dev_status = dev_status;
  a.done = at<int32_t>(ws, L.gemm_done);
  a.stream = st;
  r = launch_ffn(a);
  if (r != MOE_OK) return r;
  return launch_moe_combine(shape, y_perm, pair_pos, topk_score, n_sel, y_shared, residual, budget_max, out, st);
}

moe_status moe_selftest_wait_timeout(const moe_shape* shape, const int32_t* expert_offsets, int64_t budget,
                                     const uint16_t* W2, uint16_t* y_perm, int64_t wait_limit_clk, int32_t* dev_status,
                                     void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_selftest_wait_timeout");
  if (!shape_ok(shape) || !expert_offsets || !W2 || !y_perm || !dev_status || !ws) return MOE_ERR_ARG;
  if (!aligned16(W2) || !aligned16(y_perm) || !aligned16(ws)) return MOE_ERR_ARG;
  if (budget < 1 || budget > (int64_t)shape->K_orig * shape->T) return MOE_ERR_BUDGET;
  if (wait_limit_clk < 1000 || wait_limit_clk > 2000000000ll) return MOE_ERR_ARG;
  const WsLayout L = ws_layout(shape, budget);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  FfnArgs a;
  a.s = shape;
  a.a_routed = at<uint16_t>(ws, L.x_perm);   // never read: GEMM-1 is not launched
  a.expert_offsets = expert_offsets;
  a.budget = budget;
  a.W13 = W2;                                 // only a tensor map is built from it
  a.W2 = W2;
  a.h = at<uint16_t>(ws, L.h);
  a.y_perm = y_perm;
  a.dev_status = dev_status;
  a.done = at<int32_t>(ws, L.gemm_done);      // cleared by launch_ffn, then never incremented
  a.wait_limit_clk = wait_limit_clk;
  a.gemm2_only = true;
  a.stream = (cudaStream_t)stream;
  return launch_ffn(a);
}

moe_status moe_select_top_p(const moe_shape* shape, const float* topk_score, float P, int32_t* n_sel, int32_t* total,
                            int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_select_top_p");
  if (!shape_ok(shape) || !topk_score || !n_sel || !dev_status || !(P == P)) return MOE_ERR_ARG;
  return launch_token_rule_select(shape, topk_score, 0, P, n_sel, total, dev_status, (cudaStream_t)stream);
}

moe_status moe_select_rel_threshold(const moe_shape* shape, const float* topk_score, float beta, int32_t* n_sel,
                                    int32_t* total, int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_select_rel_threshold");
  if (!shape_ok(shape) || !topk_score || !n_sel || !dev_status || !(beta >= 0.f)) return MOE_ERR_ARG;
  return launch_token_rule_select(shape, topk_score, 1, beta, n_sel, total, dev_status, (cudaStream_t)stream);
}

size_t moe_router_workspace_bytes(const moe_shape* shape, int32_t n_seq) {
  if (!router_shape_ok(shape) || !n_seq_ok(n_seq)) return 0;
  return router_workspace_bytes(shape, n_seq);
}

moe_status moe_balance_loss(const moe_shape* shape, const float* scores, const int32_t* topk_idx, const int32_t* n_sel,
                            const int32_t* seq_offsets, int32_t n_seq, float alpha, int32_t* counts, float* coef,
                            float* loss, int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_balance_loss");
  if (!router_shape_ok(shape) || !n_seq_ok(n_seq) || (seq_offsets == nullptr && n_seq != 1)) return MOE_ERR_ARG;
  if (!scores || !topk_idx || !counts || !coef || !loss || !dev_status || !ws) return MOE_ERR_ARG;
  if (!aligned16(scores) || !aligned16(topk_idx) || !aligned16(counts) || !aligned16(coef) || !aligned16(ws)) return MOE_ERR_ARG;
  if (!aligned4(n_sel) || !aligned4(seq_offsets) || !aligned4(loss)) return MOE_ERR_ARG;
  if (!std::isfinite(alpha)) return MOE_ERR_ARG;
  if (ws_bytes < router_workspace_bytes(shape, n_seq)) return MOE_ERR_WORKSPACE;
  return launch_balance_loss(shape, scores, topk_idx, n_sel, seq_offsets, n_seq, alpha, counts, coef, loss, dev_status, ws,
                             (cudaStream_t)stream);
}

moe_status moe_gate_backward(const moe_shape* shape, const uint16_t* x, const uint16_t* W_gate, const float* scores,
                             const int32_t* topk_idx, const int32_t* n_sel, const float* d_topk_score, const float* coef,
                             const int32_t* seq_offsets, int32_t n_seq, float* d_logits, uint16_t* dx, float* dW_gate,
                             float* d_bias, int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_gate_backward");
  if (!router_shape_ok(shape) || !n_seq_ok(n_seq) || (seq_offsets == nullptr && n_seq != 1)) return MOE_ERR_ARG;
  if (!scores || !dev_status || !ws || (!d_topk_score && !coef) || (d_topk_score && !topk_idx)) return MOE_ERR_ARG;
  if ((!d_logits && !dx && !dW_gate && !d_bias) || (dx && !W_gate) || (dW_gate && !x)) return MOE_ERR_ARG;
  for (const void* ptr : {(const void*)x, (const void*)W_gate, (const void*)scores, (const void*)topk_idx,
                          (const void*)d_topk_score, (const void*)coef, (const void*)d_logits, (const void*)dx,
                          (const void*)dW_gate, (const void*)d_bias, (const void*)ws})
    if (!aligned16(ptr)) return MOE_ERR_ARG;
  if (!aligned4(n_sel) || !aligned4(seq_offsets)) return MOE_ERR_ARG;
  if ((dx && dx == x) || (d_logits && (d_logits == scores || d_logits == d_topk_score || d_logits == coef))) return MOE_ERR_ARG;
  if (ws_bytes < router_workspace_bytes(shape, n_seq)) return MOE_ERR_WORKSPACE;
  GateBackwardArgs a;
  a.s = shape;
  a.x = x;
  a.W_gate = W_gate;
  a.scores = scores;
  a.topk_idx = topk_idx;
  a.n_sel = n_sel;
  a.d_topk_score = d_topk_score;
  a.coef = coef;
  a.seq_offsets = seq_offsets;
  a.n_seq = n_seq;
  a.d_logits = d_logits;
  a.dx = dx;
  a.dW = dW_gate;
  a.d_bias = d_bias;
  a.dev_status = dev_status;
  a.ws = ws;
  a.stream = (cudaStream_t)stream;
  return launch_gate_backward(a);
}

moe_status moe_combine_backward(const moe_shape* shape, const uint16_t* d_out, const uint16_t* y_perm,
                                const int32_t* pair_pos, const float* topk_score, const int32_t* n_sel, int64_t budget,
                                float* d_topk_score, uint16_t* d_y_perm, void* stream) {
  ApiRange nvtx_range("moe_combine_backward");
  if (!shape_ok(shape) || (int64_t)shape->T * shape->K_orig > INT32_MAX) return MOE_ERR_ARG;   // pair_pos is int32
  if (!d_out || (!y_perm && budget != 0) || !pair_pos || !n_sel || !d_topk_score) return MOE_ERR_ARG;
  if (d_y_perm != nullptr && (!topk_score || d_y_perm == y_perm || d_y_perm == d_out)) return MOE_ERR_ARG;
  if (!aligned16(d_out) || !aligned16(y_perm) || !aligned16(d_y_perm) || !aligned16(pair_pos) || !aligned16(topk_score) ||
      !aligned16(d_topk_score) || !aligned4(n_sel))
    return MOE_ERR_ARG;
  if (budget < 0 || budget > (int64_t)shape->K_orig * shape->T) return MOE_ERR_BUDGET;
  return launch_combine_backward(shape, d_out, y_perm, pair_pos, topk_score, n_sel, budget, d_topk_score, d_y_perm,
                                 (cudaStream_t)stream);
}

size_t moe_adapter_workspace_bytes(const moe_adapter_shape* shape) {
  if (!adapter_shape_ok(shape)) return 0;
  return adapter_workspace_bytes(shape->T, shape->rank);
}

moe_status moe_adapter_linear(const moe_adapter_shape* shape, const uint16_t* x, const uint16_t* W, const uint16_t* A,
                              const uint16_t* B, const float* scale, const int32_t* adapter_id, uint16_t* y,
                              int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_adapter_linear");
  if (!adapter_shape_ok(shape) || !x || !W || !A || !B || !scale || !adapter_id || !y || !dev_status || !ws) return MOE_ERR_ARG;
  if (!aligned16(x) || !aligned16(W) || !aligned16(A) || !aligned16(B) || !aligned16(y) || !aligned16(ws) ||
      !aligned4(scale) || !aligned4(adapter_id) || x == y)
    return MOE_ERR_ARG;
  if (ws_bytes < adapter_workspace_bytes(shape->T, shape->rank)) return MOE_ERR_WORKSPACE;
  AdapterArgs a;
  a.T = shape->T;
  a.K = shape->K;
  a.M = shape->M;
  a.n_adapters = shape->n_adapters;
  a.rank = shape->rank;
  a.x = x;
  a.W = W;
  a.A = A;
  a.B = B;
  a.scale = scale;
  a.adapter_id = adapter_id;
  a.y = y;
  a.dev_status = dev_status;
  a.ws = ws;
  a.stream = (cudaStream_t)stream;
  return launch_adapter_linear(a);
}

size_t moe_shared_adapted_workspace_bytes(const moe_shape* shape, int32_t n_adapters, int32_t rank) {
  if (!adapted_shape_ok(shape) || !adapters_ok(n_adapters, rank)) return 0;
  return shared_adapted_h_bytes(shape) + adapter_workspace_bytes(shape->T, rank);
}

moe_status moe_shared_ffn_adapted(const moe_shape* shape, int32_t n_adapters, int32_t rank, const uint16_t* x,
                                  const uint16_t* Wsh13, const uint16_t* Wsh2, const uint16_t* A13, const uint16_t* B13,
                                  const uint16_t* A2, const uint16_t* B2, const float* scale, const int32_t* adapter_id,
                                  uint16_t* y_shared, int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_shared_ffn_adapted");
  if (!adapted_shape_ok(shape) || !adapters_ok(n_adapters, rank)) return MOE_ERR_ARG;
  for (const void* ptr : {(const void*)x, (const void*)Wsh13, (const void*)Wsh2, (const void*)A13, (const void*)B13,
                          (const void*)A2, (const void*)B2, (const void*)y_shared, (const void*)ws})
    if (!ptr || !aligned16(ptr)) return MOE_ERR_ARG;
  if (!scale || !adapter_id || !dev_status || !aligned4(scale) || !aligned4(adapter_id) || x == y_shared) return MOE_ERR_ARG;
  if (ws_bytes < moe_shared_adapted_workspace_bytes(shape, n_adapters, rank)) return MOE_ERR_WORKSPACE;
  // h first, then what the two adapted projections use one after the other.  h is bf16 as in moe_shared_ffn: the operand type of
  // the second projection, whose W2 is bf16, and without adapters the two calls agree.  Against 64 bits the result is off by
  // 0.0024 of its size (root mean square) where an fp32 h, at twice the products, would leave y's own rounding, 0.0017.
  uint16_t* h = at<uint16_t>(ws, 0);
  AdapterArgs a;
  a.T = shape->T;
  a.K = shape->H;
  a.M = shape->S * shape->I;
  a.swiglu_rows = shape->I;
  a.n_adapters = n_adapters;
  a.rank = rank;
  a.x = x;
  a.W = Wsh13;
  a.A = A13;
  a.B = B13;
  a.scale = scale;
  a.adapter_id = adapter_id;
  a.y = h;
  a.dev_status = dev_status;
  a.ws = at<void>(ws, shared_adapted_h_bytes(shape));
  a.stream = (cudaStream_t)stream;
  const moe_status r = launch_adapter_linear(a);
  if (r != MOE_OK) return r;
  a.K = shape->S * shape->I;
  a.k_per_sub = shape->I;
  a.M = shape->H;
  a.swiglu_rows = 0;
  a.x = h;
  a.W = Wsh2;
  a.A = A2;
  a.B = B2;
  a.y = y_shared;
  return launch_adapter_linear(a);
}

moe_status moe_grouped_gemm(const moe_grouped_shape* shape, const uint16_t* x, const int32_t* offsets, const uint16_t* W, uint16_t* y,
                            int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_grouped_gemm");
  if (!grouped_shape_ok(shape, 0) || !x || !offsets || !W || !y || !dev_status || !all_aligned16({x, W, y}) || !aligned4(offsets) || y == x || y == W)
    return MOE_ERR_ARG;
  return launch_grouped_gemm(shape, x, offsets, W, y, dev_status, (cudaStream_t)stream);
}

moe_status moe_grouped_gemm_dx(const moe_grouped_shape* shape, const uint16_t* dy, const int32_t* offsets, const uint16_t* W, uint16_t* dx,
                               int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_grouped_gemm_dx");
  if (!grouped_shape_ok(shape, 0) || !dy || !offsets || !W || !dx || !dev_status || !all_aligned16({dy, W, dx}) || !aligned4(offsets) || dx == dy || dx == W)
    return MOE_ERR_ARG;
  return launch_grouped_gemm_dx(shape, dy, offsets, W, dx, dev_status, (cudaStream_t)stream);
}

moe_status moe_grouped_gemm_dw(const moe_grouped_shape* shape, const uint16_t* dy, const uint16_t* x, const int32_t* offsets, void* dW,
                               int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_grouped_gemm_dw");
  if (!grouped_shape_ok(shape, MOE_GROUPED_DW_FP32 | MOE_GROUPED_DW_ADD) || !dy || !x || !offsets || !dW || !dev_status ||
      !all_aligned16({dy, x, dW}) || !aligned4(offsets) || dW == dy || dW == x)
    return MOE_ERR_ARG;
  return launch_grouped_gemm_dw(shape, dy, x, offsets, dW, dev_status, (cudaStream_t)stream);
}

size_t moe_ffn_backward_workspace_bytes(const moe_shape* shape, int64_t budget) {
  return ffn_backward_ok(shape, budget) ? ffn_backward_ws(shape, budget).total : 0;
}

moe_status moe_grouped_ffn_backward(const moe_shape* shape, const uint16_t* x_or_xperm, const int32_t* perm_token,
                                    const int32_t* expert_offsets, int64_t budget, const uint16_t* W13, const uint16_t* W2,
                                    const uint16_t* d_y_perm, uint16_t* dx_perm, uint16_t* dW13, uint16_t* dW2, int32_t* dev_status,
                                    void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_grouped_ffn_backward");
  if (!shape_ok(shape) || !expert_offsets || !W13 || !W2 || !dev_status || !ws) return MOE_ERR_ARG;
  if (budget < 0 || budget > (int64_t)shape->K_orig * shape->T) return MOE_ERR_BUDGET;
  if (!ffn_backward_ok(shape, budget) || (budget > 0 && (!x_or_xperm || !d_y_perm)) || (!dx_perm && !dW13 && !dW2)) return MOE_ERR_ARG;
  if (!all_aligned16({x_or_xperm, W13, W2, d_y_perm, dx_perm, dW13, dW2, ws}) || !aligned4(perm_token) || !aligned4(expert_offsets)) return MOE_ERR_ARG;
  for (const void* out : {(const void*)dx_perm, (const void*)dW13, (const void*)dW2})
    if (out != nullptr && (out == x_or_xperm || out == W13 || out == W2 || out == d_y_perm)) return MOE_ERR_ARG;
  if (!all_different({dx_perm, dW13, dW2, ws})) return MOE_ERR_ARG;
  const FfnBackwardWs w = ffn_backward_ws(shape, budget);
  if (ws_bytes < w.total) return MOE_ERR_WORKSPACE;
  FfnBackwardArgs a;
  a.E = shape->N;
  a.H = shape->H;
  a.I = shape->I;
  a.rows = budget;
  a.offsets = expert_offsets;
  a.x = x_or_xperm;
  a.perm_token = perm_token;
  a.T = shape->T;
  a.x_rows = at<uint16_t>(ws, w.x_perm);
  a.W13 = W13;
  a.W2 = W2;
  a.d_y = d_y_perm;
  a.h = at<uint16_t>(ws, w.h);
  a.du = at<uint16_t>(ws, w.du);
  a.dx = dx_perm;
  a.dW13 = dW13;
  a.dW2 = dW2;
  a.dev_status = dev_status;
  a.stream = (cudaStream_t)stream;
  return launch_ffn_backward(a);
}

size_t moe_shared_ffn_backward_workspace_bytes(const moe_shape* shape) {
  return shared_backward_ok(shape) ? shared_backward_h_bytes(shape) * 3 : 0;
}

moe_status moe_shared_ffn_backward(const moe_shape* shape, const uint16_t* x, const uint16_t* Wsh13, const uint16_t* Wsh2,
                                   const uint16_t* d_y_shared, uint16_t* dx, uint16_t* dWsh13, uint16_t* dWsh2, int32_t* dev_status,
                                   void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_shared_ffn_backward");
  if (!shared_backward_ok(shape) || !x || !Wsh13 || !Wsh2 || !d_y_shared || !dev_status || !ws || (!dx && !dWsh13 && !dWsh2)) return MOE_ERR_ARG;
  if (!all_aligned16({x, Wsh13, Wsh2, d_y_shared, dx, dWsh13, dWsh2, ws})) return MOE_ERR_ARG;
  for (const void* out : {(const void*)dx, (const void*)dWsh13, (const void*)dWsh2})
    if (out != nullptr && (out == x || out == Wsh13 || out == Wsh2 || out == d_y_shared)) return MOE_ERR_ARG;
  if (!all_different({dx, dWsh13, dWsh2, ws})) return MOE_ERR_ARG;
  if (ws_bytes < shared_backward_h_bytes(shape) * 3) return MOE_ERR_WORKSPACE;
  FfnBackwardArgs a;
  a.E = 1;
  a.S = shape->S;
  a.H = shape->H;
  a.I = shape->I;
  a.rows = shape->T;
  a.x = x;
  a.W13 = Wsh13;
  a.W2 = Wsh2;
  a.d_y = d_y_shared;
  a.h = at<uint16_t>(ws, 0);
  a.du = at<uint16_t>(ws, shared_backward_h_bytes(shape));
  a.dx = dx;
  a.dW13 = dWsh13;
  a.dW2 = dWsh2;
  a.dev_status = dev_status;
  a.stream = (cudaStream_t)stream;
  return launch_ffn_backward(a);
}

moe_status moe_block_norm(const moe_norm_shape* shape, const uint16_t* r, const uint16_t* y, const float* w_post, const uint16_t* gate,
                          const float* scale, const float* w_pre, uint16_t* r_out, uint16_t* n_out, void* stream) {
  ApiRange nvtx_range("moe_block_norm");
  if (!norm_shape_ok(shape) || !r || (y == nullptr) != (r_out == nullptr) || (!r_out && !n_out) || (gate == nullptr) != (shape->gate_cols == 0))
    return MOE_ERR_ARG;
  if (!all_aligned16({r, y, w_post, w_pre, r_out, n_out}) || !aligned4(scale)) return MOE_ERR_ARG;
  if (shape->gate_cols == 1 ? (reinterpret_cast<uintptr_t>(gate) & 1u) != 0 : !aligned16(gate)) return MOE_ERR_ARG;
  if (n_out != nullptr && (n_out == r_out || n_out == r || n_out == gate)) return MOE_ERR_ARG;
  if (r_out != nullptr && (r_out == y || r_out == gate)) return MOE_ERR_ARG;
  BlockNormArgs a;
  a.s = shape;
  a.r = r;
  a.y = y;
  a.w_post = w_post;
  a.gate = gate;
  a.scale = scale;
  a.w_pre = w_pre;
  a.r_out = r_out;
  a.n_out = n_out;
  a.stream = (cudaStream_t)stream;
  return launch_block_norm(a);
}

size_t moe_norm_workspace_bytes(const moe_norm_shape* shape) { return norm_shape_ok(shape) ? block_norm_workspace_bytes(shape) : 0; }

moe_status moe_block_norm_backward(const moe_norm_shape* shape, const uint16_t* r_out, const uint16_t* y, const float* w_post,
                                   const uint16_t* gate, const float* scale, const float* w_pre, const uint16_t* d_n,
                                   const uint16_t* d_r_out, uint16_t* d_r, uint16_t* d_y, uint16_t* d_gate, float* dw_post, float* dw_pre,
                                   float* d_scale, void* ws, size_t ws_bytes, void* stream) {
  ApiRange nvtx_range("moe_block_norm_backward");
  if (!norm_shape_ok(shape) || (!d_n && !d_r_out) || (d_n && !r_out)) return MOE_ERR_ARG;
  if ((gate == nullptr) != (shape->gate_cols == 0) || (d_gate && !gate) || (!y && (d_y || d_gate || dw_post || d_scale)) || (dw_pre && !d_n))
    return MOE_ERR_ARG;
  if (!d_r && !d_y && !d_gate && !dw_post && !dw_pre && !d_scale) return MOE_ERR_ARG;
  if (!all_aligned16({r_out, y, w_post, w_pre, d_n, d_r_out, d_r, d_y, dw_post, dw_pre, ws}) || !aligned4(scale) || !aligned4(d_scale))
    return MOE_ERR_ARG;
  for (const void* g : {(const void*)gate, (const void*)d_gate})
    if (shape->gate_cols == 1 ? (reinterpret_cast<uintptr_t>(g) & 1u) != 0 : !aligned16(g)) return MOE_ERR_ARG;
  for (const void* in : {(const void*)r_out, (const void*)y, (const void*)gate, (const void*)d_n, (const void*)d_r_out}) {
    if (in == nullptr) continue;
    if ((in == d_r && in != d_n && in != d_r_out) || (in == d_y && in != y) || in == d_gate || in == dw_post || in == dw_pre || in == d_scale)
      return MOE_ERR_ARG;
  }
  const bool sums = dw_post || dw_pre || d_scale;
  if (!all_different({d_r, d_y, d_gate, dw_post, dw_pre, d_scale, sums ? ws : nullptr})) return MOE_ERR_ARG;
  if (sums && !ws) return MOE_ERR_ARG;
  if (sums && ws_bytes < block_norm_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  BlockNormArgs a;
  a.s = shape;
  a.r = r_out;
  a.y = y;
  a.w_post = w_post;
  a.gate = gate;
  a.scale = scale;
  a.w_pre = w_pre;
  a.d_n = d_n;
  a.d_r_out = d_r_out;
  a.d_r = d_r;
  a.d_y = d_y;
  a.d_gate = d_gate;
  a.dw_post = dw_post;
  a.dw_pre = dw_pre;
  a.d_scale = d_scale;
  a.ws = ws;
  a.stream = (cudaStream_t)stream;
  return launch_block_norm_backward(a);
}

moe_status moe_adamw_step(const moe_adamw_tensor* tensors, int32_t count, double beta1, double beta2, double eps, const float* hyper,
                          int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_adamw_step");
  if (!adamw_entries_ok(tensors, count, false) || !hyper || !dev_status || !aligned4(hyper)) return MOE_ERR_ARG;
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0) || !std::isfinite(eps) || !((float)eps > 0.f)) return MOE_ERR_ARG;
  AdamwArgs a;
  a.tensors = tensors;
  a.count = count;
  a.beta1 = beta1;
  a.beta2 = beta2;
  a.eps = eps;
  a.hyper = hyper;
  a.dev_status = dev_status;
  a.stream = (cudaStream_t)stream;
  return launch_adamw_step(a);
}

static moe_status adamw_states(const moe_adamw_tensor* tensors, int32_t count, const float* const* m32, const float* const* v32,
                               int32_t* dev_status, bool write, void* stream) {
  if (!adamw_entries_ok(tensors, count, true) || !m32 || !v32 || (write && !dev_status)) return MOE_ERR_ARG;
  for (int32_t k = 0; k < count; ++k)
    if (!m32[k] || !v32[k] || !all_aligned16({m32[k], v32[k]}) || m32[k] == v32[k]) return MOE_ERR_ARG;
  AdamwArgs a;
  a.tensors = tensors;
  a.count = count;
  a.m32 = m32;
  a.v32 = v32;
  a.dev_status = dev_status;
  a.stream = (cudaStream_t)stream;
  return write ? launch_adamw_write(a) : launch_adamw_read(a);
}

moe_status moe_adamw_states_read(const moe_adamw_tensor* tensors, int32_t count, float* const* m32, float* const* v32, void* stream) {
  ApiRange nvtx_range("moe_adamw_states_read");
  return adamw_states(tensors, count, const_cast<const float* const*>(m32), const_cast<const float* const*>(v32), nullptr, false, stream);
}

moe_status moe_adamw_states_write(const moe_adamw_tensor* tensors, int32_t count, const float* const* m32, const float* const* v32,
                                  int32_t* dev_status, void* stream) {
  ApiRange nvtx_range("moe_adamw_states_write");
  return adamw_states(tensors, count, m32, v32, dev_status, true, stream);
}

moe_status moe_rmsnorm(const moe_shape* shape, const uint16_t* x, uint16_t* out, void* stream) {
  ApiRange nvtx_range("moe_rmsnorm");
  if (!shape_ok(shape) || !x || !out || !aligned16(x) || !aligned16(out)) return MOE_ERR_ARG;
  return launch_rmsnorm(shape, x, out, (cudaStream_t)stream);
}

moe_status moe_profile_enable(int32_t on) {
  if (on && !g_prof_on) {
    for (int i = 0; i <= kProfStages; ++i)
      if (cudaEventCreate(&g_prof_ev[i]) != cudaSuccess) return MOE_ERR_CUDA;
    g_prof_on = true;
  } else if (!on && g_prof_on) {
    g_prof_on = false;
    for (int i = 0; i <= kProfStages; ++i) cudaEventDestroy(g_prof_ev[i]);
  }
  return MOE_OK;
}

moe_status moe_profile_read(float* stage_ms) {
  if (!g_prof_on || !stage_ms) return MOE_ERR_ARG;
  if (cudaEventSynchronize(g_prof_ev[kProfStages]) != cudaSuccess) return MOE_ERR_CUDA;
  for (int i = 0; i < kProfStages; ++i)
    if (cudaEventElapsedTime(&stage_ms[i], g_prof_ev[i], g_prof_ev[i + 1]) != cudaSuccess) return MOE_ERR_CUDA;
  return MOE_OK;
}

moe_status moe_layer_intermediates(const moe_shape* shape, int64_t budget_max, void* ws, size_t ws_bytes,
                                   int32_t** topk_idx, float** topk_score, int32_t** n_sel, int32_t** expert_offsets,
                                   int32_t** perm_token, int32_t** pair_pos, uint16_t** y_perm) {
  if (!shape_ok(shape) || !ws) return MOE_ERR_ARG;
  if (budget_max < 0 || budget_max > (int64_t)shape->K_orig * shape->T) return MOE_ERR_BUDGET;
  const WsLayout L = ws_layout(shape, budget_max);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  if (topk_idx) *topk_idx = at<int32_t>(ws, L.topk_idx);
  if (topk_score) *topk_score = at<float>(ws, L.topk_score);
  if (n_sel) *n_sel = at<int32_t>(ws, L.n_sel);
  if (expert_offsets) *expert_offsets = at<int32_t>(ws, L.expert_offsets);
  if (perm_token) *perm_token = at<int32_t>(ws, L.perm_token);
  if (pair_pos) *pair_pos = at<int32_t>(ws, L.pair_pos);
  if (y_perm) *y_perm = at<uint16_t>(ws, L.y_perm);
  return MOE_OK;
}

}  // extern "C"
