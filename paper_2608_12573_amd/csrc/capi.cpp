// extern "C" entry points of libprofk.so: argument checks, workspace
// carving and launches.  Declarations and contracts are in include/profk.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <mutex>

#include "adjust.h"
#include "launch.h"
#include "linear.h"
#include "logprobs.h"
#include "mx4.h"
#include "norm.h"
#include "plan_internal.h"
#include "profk.h"

namespace {

thread_local int g_last_hip_error = 0;
thread_local hipEvent_t g_ev_before = nullptr;
thread_local hipEvent_t g_ev_after = nullptr;

int hip_fail(hipError_t e) {
  g_last_hip_error = static_cast<int>(e);
  return PROFK_EHIP;
}

bool plan_consistent(const profk_plan_t* p) {
  return p->N >= 1 && p->N <= static_cast<int64_t>(UINT32_MAX) && p->k >= 1 && p->k <= p->N &&
         p->k_req >= 1 && p->k_req <= p->k && p->S >= 1 && p->t >= 1 && p->t <= p->S &&
         p->S <= static_cast<int64_t>(UINT32_MAX) && p->M >= p->k && p->M <= p->N &&
         (p->mode == PROFK_MODE_FILTER || p->mode == PROFK_MODE_DIRECT) &&
         (p->lexicographic == 0 || p->lexicographic == 1);
}

bool dtype_ok(int32_t dt) { return dt == PROFK_F32 || dt == PROFK_BF16; }

size_t elem_size(int32_t dt) { return dt == PROFK_F32 ? 4 : 2; }

// Shared checks of the flat entry points.  Returns PROFK_OK and fills the
// layout when the call may proceed.
int check_flat(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t N, int64_t k,
               const void* out_vals, const int64_t* out_idx, const void* ws, size_t ws_bytes,
               profk::FlatLayout* L) {
  if (!plan || !values || !out_vals || !out_idx || !ws) return PROFK_ENULL;
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (!plan_consistent(plan) || plan->N != N || plan->k != k) return PROFK_EINVAL;
  if (reinterpret_cast<uintptr_t>(values) % elem_size(dtype) != 0) return PROFK_EINVAL;
  *L = profk::flat_layout(*plan, dtype, profk::device_cu_count());
  if (ws_bytes < L->bytes) return PROFK_EWORKSPACE;
  return PROFK_OK;
}

int run_flat(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t N, int64_t k,
             uint64_t seed, uint64_t row, void* out_vals, int64_t* out_idx, void* ws, size_t ws_bytes,
             void* stream, profk_info_t* info, int use_tau, uint32_t tau_key) {
  profk::FlatLayout L;
  const int rc = check_flat(plan, dtype, values, N, k, out_vals, out_idx, ws, ws_bytes, &L);
  if (rc != PROFK_OK) return rc;
  profk::FlatCall c{plan, dtype, values, static_cast<uint32_t>(N), static_cast<uint32_t>(k), seed, row,
                    out_vals, out_idx, static_cast<uint8_t*>(ws), L, static_cast<hipStream_t>(stream),
                    info, use_tau, tau_key, g_ev_before, g_ev_after};
  const hipError_t e = profk::launch_flat(c);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

// Rows of a batch that ws_bytes hold a vector workspace each for (0: not
// even one); a plan with k above the one-block refinement takes one at a
// time.
int64_t rows_at_once(const profk::FlatLayout& L, int64_t B, size_t ws_bytes) {
  const uint64_t n = ws_bytes / L.bytes;
  if (L.big) return n > 0 ? 1 : 0;
  const int64_t most = B < profk::kRowBatch ? B : profk::kRowBatch;
  return n < static_cast<uint64_t>(most) ? static_cast<int64_t>(n) : most;
}

int check_sae_shape(const void* x, const void* w_enc, const float* b_enc, int64_t B, int64_t d_model,
                    int64_t d_dict) {
  if (!x || !w_enc || !b_enc) return PROFK_ENULL;
  if (B < 1 || d_model < 64 || d_model % 64 != 0 || d_dict < 1) return PROFK_EINVAL;
  if (d_model > (1 << 16) || B > static_cast<int64_t>(UINT32_MAX) / d_dict) return PROFK_EINVAL;
  if (reinterpret_cast<uintptr_t>(x) % 16 != 0 || reinterpret_cast<uintptr_t>(w_enc) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(b_enc) % 4 != 0)
    return PROFK_EINVAL;
  return PROFK_OK;
}

}  // namespace

extern "C" {

void profk_default_opts(profk_plan_opts_t* o) {
  if (!o) return;
  o->S_min = 32768;
  o->S_max = 131072;
  o->cost_ratio = 1.0;
  o->eps_split = 0.5;
  o->paper_literal = 0;
  o->force_mode = PROFK_FORCE_AUTO;
  o->lexicographic = 0;
}

void profk_default_row_opts(profk_plan_opts_t* o) {
  profk_default_opts(o);
  if (!o) return;
  o->S_min = 256;
  // tau_B / tau_A measured for the per-row kernel on MI355X: a sampled
  // element costs a scattered line fetch, so fewer draws and a larger buffer
  // are faster than the unit ratio.
  o->cost_ratio = 0.5;
}

int profk_plan(int64_t N, int64_t k, double eps, double recall, const profk_plan_opts_t* opts,
               profk_plan_t* out) {
  profk_plan_opts_t o;
  if (opts) o = *opts; else profk_default_opts(&o);
  return profk::make_plan(N, k, eps, recall, o, out);
}

void profk_default_sae_opts(profk_plan_opts_t* o) {
  profk_default_opts(o);
  if (!o) return;
  // tau_B / tau_A measured for the fused SAE path on MI355X: a draw is a
  // d_model-long dot product on the matrix cores with two row reads, not a
  // single gathered element, so fewer draws and a larger buffer are faster.
  o->cost_ratio = 1.0 / 64.0;
}

int profk_plan_rows(int64_t D, int64_t k, double eps, double recall, const profk_plan_opts_t* opts,
                    profk_plan_t* out) {
  profk_plan_opts_t o;
  if (opts) o = *opts; else profk_default_row_opts(&o);
  return profk::make_plan(D, k, eps, recall, o, out);
}

size_t profk_workspace_size(const profk_plan_t* plan, int32_t dtype, int64_t batch) {
  if (!plan || !dtype_ok(dtype) || !plan_consistent(plan) || batch < 1) return 0;
  // The row kernel keeps everything in LDS; rows outside its envelope run the
  // vector kernels, at least one row at a time (profk_rows_workspace_size).
  if (batch > 1 && profk::rows_fit_block(*plan, dtype)) return 256;
  return profk::flat_layout(*plan, dtype, profk::device_cu_count()).bytes;
}

size_t profk_rows_workspace_size(const profk_plan_t* plan, int32_t dtype, int64_t B) {
  const size_t least = profk_workspace_size(plan, dtype, B);
  if (least == 0 || B < 2) return least;
  const int cus = profk::device_cu_count();
  const profk::FlatLayout L = profk::flat_layout(*plan, dtype, cus);
  const size_t cap = profk::kRowBatchBytes > L.bytes ? static_cast<size_t>(profk::kRowBatchBytes) : L.bytes;
  const int64_t R = rows_at_once(L, B, cap);
  return profk::rows_block_threads(*plan, dtype, B, R, cus) == 0 ? static_cast<size_t>(R) * L.bytes : least;
}

int profk_topk(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t N, int64_t k,
               uint64_t seed, void* out_vals, int64_t* out_idx, void* ws, size_t ws_bytes,
               void* stream, profk_info_t* info_dev) {
  return run_flat(plan, dtype, values, N, k, seed, 0, out_vals, out_idx, ws, ws_bytes, stream,
                  info_dev, 0, 0);
}

int profk_topk_tau(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t N, int64_t k,
                   uint32_t tau_key, void* out_vals, int64_t* out_idx, void* ws, size_t ws_bytes,
                   void* stream, profk_info_t* info_dev) {
  return run_flat(plan, dtype, values, N, k, 0, 0, out_vals, out_idx, ws, ws_bytes, stream, info_dev,
                  1, tau_key);
}

int profk_batchtopk(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t B, int64_t D,
                    int64_t k_row, uint64_t seed, void* out_vals, int64_t* out_flat_idx, void* ws,
                    size_t ws_bytes, void* stream, profk_info_t* info_dev) {
  if (B < 1 || D < 1 || k_row < 1 || k_row > D) return PROFK_EINVAL;
  if (B > static_cast<int64_t>(UINT32_MAX) / D) return PROFK_EINVAL;
  return run_flat(plan, dtype, values, B * D, B * k_row, seed, 0, out_vals, out_flat_idx, ws, ws_bytes,
                  stream, info_dev, 0, 0);
}

// ---- BatchTopK SAE layer ----

size_t profk_sae_workspace_size(const profk_plan_t* plan, int64_t B, int64_t d_dict) {
  if (!plan || !plan_consistent(plan) || B < 1 || d_dict < 1 || plan->N != B * d_dict) return 0;
  return profk::sae_layout(*plan, static_cast<uint32_t>(B), static_cast<uint32_t>(d_dict),
                           profk::device_cu_count())
      .bytes;
}

int profk_sae_encode_topk(const profk_plan_t* plan, const void* x, const void* w_enc, const float* b_enc,
                          int64_t B, int64_t d_model, int64_t d_dict, int64_t k_row, uint64_t seed,
                          float* out_vals, int64_t* out_flat_idx, void* ws, size_t ws_bytes, void* stream,
                          profk_info_t* info_dev) {
  if (!plan || !out_vals || !out_flat_idx || !ws) return PROFK_ENULL;
  int rc = check_sae_shape(x, w_enc, b_enc, B, d_model, d_dict);
  if (rc != PROFK_OK) return rc;
  if (k_row < 1 || k_row > d_dict) return PROFK_EINVAL;
  if (!plan_consistent(plan) || plan->N != B * d_dict || plan->k != B * k_row || plan->lexicographic)
    return PROFK_EINVAL;
  const profk::SaeLayout L = profk::sae_layout(*plan, static_cast<uint32_t>(B), static_cast<uint32_t>(d_dict),
                                               profk::device_cu_count());
  if (ws_bytes < L.bytes) return PROFK_EWORKSPACE;
  profk::SaeCall c{plan, x, w_enc, b_enc, static_cast<uint32_t>(B), static_cast<uint32_t>(d_model),
                   static_cast<uint32_t>(d_dict), static_cast<uint32_t>(B * k_row), seed, out_vals, out_flat_idx,
                   static_cast<uint8_t*>(ws), L, static_cast<hipStream_t>(stream), info_dev, nullptr,
                   g_ev_before, g_ev_after};
  const hipError_t e = profk::launch_sae_topk(c);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_sae_encode_dense(const void* x, const void* w_enc, const float* b_enc, int64_t B, int64_t d_model,
                           int64_t d_dict, float* out, void* stream) {
  if (!out) return PROFK_ENULL;
  int rc = check_sae_shape(x, w_enc, b_enc, B, d_model, d_dict);
  if (rc != PROFK_OK) return rc;
  profk::SaeCall c{};
  c.x = x;
  c.w = w_enc;
  c.bias = b_enc;
  c.B = static_cast<uint32_t>(B);
  c.d_model = static_cast<uint32_t>(d_model);
  c.d_dict = static_cast<uint32_t>(d_dict);
  c.stream = static_cast<hipStream_t>(stream);
  const hipError_t e = profk::launch_sae_dense(c, out);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_debug_sae_sample(const profk_plan_t* plan, const void* x, const void* w_enc, const float* b_enc,
                           int64_t B, int64_t d_model, int64_t d_dict, uint64_t seed, uint32_t* keys_dev,
                           void* ws, size_t ws_bytes, void* stream) {
  if (!plan || !keys_dev || !ws) return PROFK_ENULL;
  int rc = check_sae_shape(x, w_enc, b_enc, B, d_model, d_dict);
  if (rc != PROFK_OK) return rc;
  if (!plan_consistent(plan) || plan->N != B * d_dict || plan->mode != PROFK_MODE_FILTER) return PROFK_EINVAL;
  const profk::SaeLayout L = profk::sae_layout(*plan, static_cast<uint32_t>(B), static_cast<uint32_t>(d_dict),
                                               profk::device_cu_count());
  if (ws_bytes < L.bytes) return PROFK_EWORKSPACE;
  profk::SaeCall c{plan, x, w_enc, b_enc, static_cast<uint32_t>(B), static_cast<uint32_t>(d_model),
                   static_cast<uint32_t>(d_dict), static_cast<uint32_t>(plan->k), seed, nullptr, nullptr,
                   static_cast<uint8_t*>(ws), L, static_cast<hipStream_t>(stream), nullptr, keys_dev};
  const hipError_t e = profk::launch_sae_sample(c);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

size_t profk_sae_decode_workspace_size(int64_t B, int64_t K) {
  if (B < 1 || K < 0 || B > static_cast<int64_t>(INT32_MAX) || K > static_cast<int64_t>(UINT32_MAX)) return 0;
  return profk::sae_decode_workspace(static_cast<uint32_t>(B), static_cast<uint32_t>(K));
}

int profk_sae_decode(const float* vals, const int64_t* flat_idx, int64_t K, const void* w_dec,
                     const float* b_dec, int64_t B, int64_t d_model, int64_t d_dict, float* out, void* ws,
                     size_t ws_bytes, void* stream) {
  if (!vals || !flat_idx || !w_dec || !b_dec || !out || !ws) return PROFK_ENULL;
  if (K < 1 || B < 1 || d_model < 1 || d_dict < 1 || d_dict > static_cast<int64_t>(profk::sae_decode_max_dict()))
    return PROFK_EINVAL;
  if (B > static_cast<int64_t>(UINT32_MAX) / d_dict || K > B * d_dict || d_model > (1 << 16)) return PROFK_EINVAL;
  if (reinterpret_cast<uintptr_t>(w_dec) % 2 != 0) return PROFK_EINVAL;
  if (ws_bytes < profk_sae_decode_workspace_size(B, K)) return PROFK_EWORKSPACE;
  profk::SaeDecodeCall c{vals, flat_idx, static_cast<uint32_t>(K), static_cast<uint32_t>(B),
                         static_cast<uint32_t>(d_model), static_cast<uint32_t>(d_dict), w_dec, b_dec, out, ws,
                         static_cast<hipStream_t>(stream)};
  const hipError_t e = profk::launch_sae_decode(c);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_topk_rows(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t B, int64_t D,
                    int64_t row_stride, int64_t k, uint64_t seed, void* out_vals, int64_t* out_idx,
                    void* ws, size_t ws_bytes, void* stream, profk_info_t* info_dev) {
  if (!plan || !values || !out_vals || !out_idx) return PROFK_ENULL;
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (!plan_consistent(plan) || plan->N != D || plan->k != k) return PROFK_EINVAL;
  if (B < 1 || B > static_cast<int64_t>(INT32_MAX) || row_stride < D) return PROFK_EINVAL;
  if (reinterpret_cast<uintptr_t>(values) % elem_size(dtype) != 0) return PROFK_EINVAL;
  const int cus = profk::device_cu_count();
  const profk::FlatLayout FL = profk::flat_layout(*plan, dtype, cus);
  const bool small = profk::rows_fit_block(*plan, dtype);
  if (!small && !ws) return PROFK_ENULL;
  if (!small && ws_bytes < FL.bytes) return PROFK_EWORKSPACE;
  // A workspace that is not needed is used where the vector path can: its
  // regions take 32-bit atomics and 16-byte loads, which want them aligned.
  const bool usable = ws && (!small || reinterpret_cast<uintptr_t>(ws) % 16 == 0);
  const int64_t R = rows_at_once(FL, B, usable ? ws_bytes : 0);
  const int threads = profk::rows_block_threads(*plan, dtype, B, R, cus);
  // Rows of one launch: of the vector path (sample, filter, refinement or
  // fallback) the R that the workspace holds, reused in stream order; of row
  // blocks (launch_rows, and launch_small, which needs no workspace) what a
  // grid takes.  Each row has its own Philox stream (counter word 1 = row).
  const int64_t step = threads > 0 ? profk::rows_per_launch(threads)
                       : threads == profk::kRowsSmall ? profk::rows_per_launch(profk::kSmallBS) : R;
  const uint64_t es = elem_size(dtype);
  (void)hipGetLastError();
  for (int64_t r = 0; r < B; r += step) {
    const uint32_t n = static_cast<uint32_t>(B - r < step ? B - r : step);
    const void* const x = static_cast<const uint8_t*>(values) + static_cast<uint64_t>(r) * row_stride * es;
    void* const v = static_cast<uint8_t*>(out_vals) + static_cast<uint64_t>(r) * k * es;
    int64_t* const i = out_idx + r * k;
    profk_info_t* const info = info_dev ? info_dev + r : nullptr;
    hipError_t e;
    if (threads > 0) {
      const profk::RowCall c{plan, dtype, x, static_cast<uint32_t>(r), n, static_cast<uint32_t>(D),
                             static_cast<uint32_t>(k), static_cast<uint64_t>(row_stride), seed, v, i,
                             info, threads, static_cast<hipStream_t>(stream)};
      e = profk::launch_rows(c);
    } else {
      profk::FlatCall fc{plan, dtype, x, static_cast<uint32_t>(D), static_cast<uint32_t>(k), seed,
                         static_cast<uint64_t>(r), v, i, static_cast<uint8_t*>(ws), FL,
                         static_cast<hipStream_t>(stream), info, 0, 0};
      fc.rows = n;
      fc.stride = {static_cast<uint64_t>(row_stride) * es, FL.bytes};
      e = profk::launch_flat(fc);
    }
    if (e != hipSuccess) return hip_fail(e);
  }
  return PROFK_OK;
}

// ---- Token log probabilities ----

namespace {

// Shapes of the log probability calls; T = 0 is a call without rows.
int check_logits(int32_t dtype, int64_t T, int64_t V, int64_t row_stride, int64_t n_top) {
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (T < 0 || T > static_cast<int64_t>(INT32_MAX) || V < 1 || V > static_cast<int64_t>(INT32_MAX)) return PROFK_EINVAL;
  if (row_stride < V || n_top < 0 || n_top > profk::kLpMaxTop) return PROFK_EINVAL;
  // the rows' byte offsets fit 63 bits
  if (row_stride > INT64_MAX / 8 / (T > 0 ? T : 1)) return PROFK_EINVAL;
  return PROFK_OK;
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

size_t profk_token_logprobs_workspace_size(int64_t T, int64_t V, int64_t n_top) {
  if (T < 1 || check_logits(PROFK_F32, T, V, V, n_top) != PROFK_OK) return 0;
  return profk::lp_layout(T, V, n_top, profk::device_cu_count()).bytes;
}

int profk_token_logprobs(int32_t dtype, const void* logits, int64_t T, int64_t V, int64_t row_stride,
                         const int64_t* tokens, int64_t n_top, float* out_logprob, float* out_entropy,
                         float* out_lse, float* out_top_logprob, int64_t* out_top_idx, void* ws, size_t ws_bytes,
                         void* stream) {
  return profk_token_logprobs_ex(dtype, logits, T, V, row_stride, tokens, n_top, out_logprob, out_entropy, out_lse,
                                 nullptr, out_top_logprob, out_top_idx, ws, ws_bytes, stream);
}

int profk_token_logprobs_ex(int32_t dtype, const void* logits, int64_t T, int64_t V, int64_t row_stride,
                            const int64_t* tokens, int64_t n_top, float* out_logprob, float* out_entropy,
                            float* out_lse, float* out_lse_low, float* out_top_logprob, int64_t* out_top_idx,
                            void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_logits(dtype, T, V, row_stride, n_top);
  if (rc != PROFK_OK || T == 0) return rc;
  if (!logits || !tokens || !out_logprob || !out_entropy || !out_lse) return PROFK_ENULL;
  if (n_top > 0 && (!out_top_logprob || !out_top_idx)) return PROFK_ENULL;
  if (!aligned(logits, elem_size(dtype)) || !aligned(ws, 16)) return PROFK_EINVAL;
  const profk::LpLayout L = profk::lp_layout(T, V, n_top, profk::device_cu_count());
  if (L.bytes > 0 && !ws) return PROFK_ENULL;
  if (ws_bytes < L.bytes) return PROFK_EWORKSPACE;
  profk::LpCall c{};
  c.dtype = dtype;
  c.T = T;
  c.a.x = logits;
  c.a.stride = static_cast<uint64_t>(row_stride);
  c.a.V = static_cast<uint32_t>(V);
  c.a.n = static_cast<uint32_t>(n_top);
  c.a.tokens = tokens;
  c.a.logprob = out_logprob;
  c.a.entropy = out_entropy;
  c.a.lse = out_lse;
  c.a.lse_low = out_lse_low;
  c.a.top = out_top_logprob;
  c.a.top_idx = out_top_idx;
  c.L = L;
  c.ws = static_cast<uint8_t*>(ws);
  c.stream = static_cast<hipStream_t>(stream);
  const hipError_t e = profk::launch_logprobs(c);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_token_logprobs_grad(int32_t dtype, const void* logits, int64_t T, int64_t V, int64_t row_stride,
                              const int64_t* tokens, const float* lse, const float* entropy,
                              const float* g_logprob, const float* g_entropy, int64_t n_top,
                              const int64_t* top_idx, const float* g_top, void* out, int64_t out_stride,
                              void* stream) {
  return profk_token_logprobs_grad_ex(dtype, logits, T, V, row_stride, tokens, lse, nullptr, entropy, g_logprob,
                                      g_entropy, nullptr, n_top, top_idx, g_top, out, out_stride, stream);
}

int profk_token_logprobs_grad_ex(int32_t dtype, const void* logits, int64_t T, int64_t V, int64_t row_stride,
                                 const int64_t* tokens, const float* lse, const float* lse_low, const float* entropy,
                                 const float* g_logprob, const float* g_entropy, const float* g_lse, int64_t n_top,
                                 const int64_t* top_idx, const float* g_top, void* out, int64_t out_stride,
                                 void* stream) {
  const int rc = check_logits(dtype, T, V, row_stride, n_top);
  if (rc != PROFK_OK) return rc;
  if (check_logits(dtype, T, V, out_stride, n_top) != PROFK_OK) return PROFK_EINVAL;
  if (T == 0) return PROFK_OK;
  if (!logits || !lse || !out || (g_logprob && !tokens) || (g_entropy && !entropy)) return PROFK_ENULL;
  if (n_top > 0 && (!top_idx || !g_top)) return PROFK_ENULL;
  if (!aligned(logits, elem_size(dtype)) || !aligned(out, elem_size(dtype))) return PROFK_EINVAL;
  const auto extent = [&](int64_t stride) {
    return static_cast<uintptr_t>(((T - 1) * stride + V) * static_cast<int64_t>(elem_size(dtype)));
  };
  const uintptr_t xb = reinterpret_cast<uintptr_t>(logits), ob = reinterpret_cast<uintptr_t>(out);
  if (xb < ob + extent(out_stride) && ob < xb + extent(row_stride)) return PROFK_EINVAL;
  profk::LpGradArgs a{};
  a.x = logits;
  a.stride = static_cast<uint64_t>(row_stride);
  a.V = static_cast<uint32_t>(V);
  a.n = static_cast<uint32_t>(n_top);
  a.tokens = g_logprob ? tokens : nullptr;
  a.lse = lse;
  a.lse_low = lse_low;
  a.entropy = entropy;
  a.g_logprob = g_logprob;
  a.g_entropy = g_entropy;
  a.g_lse = g_lse;
  a.g_top = g_top;
  a.top_idx = top_idx;
  a.out = out;
  a.out_stride = static_cast<uint64_t>(out_stride);
  const hipError_t e = profk::launch_logprobs_grad(a, dtype, T, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

// ---- Microscaled 4-bit values ----

namespace {

int check_mx(int64_t R, int64_t K) {
  return R < 0 || R > static_cast<int64_t>(INT32_MAX) || K < 1 || K > profk::kMxMaxK ? PROFK_EINVAL : PROFK_OK;
}
bool mx_aligned(const void* codes, const void* scales) { return aligned(codes, 16) && aligned(scales, 4); }
size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t profk_mx4_codes_size(int64_t R, int64_t K) {
  return check_mx(R, K) == PROFK_OK ? static_cast<size_t>(R) * profk::mx_steps(K) * 64 : 0;
}

size_t profk_mx4_scales_size(int64_t R, int64_t K) {
  return check_mx(R, K) == PROFK_OK ? (static_cast<size_t>(R) + 31) / 32 * profk::mx_steps(K) * 128 : 0;
}

int profk_mx4_quantize(int32_t dtype, const void* x, int64_t R, int64_t K, int64_t row_stride, uint8_t* codes,
                       uint8_t* scales, void* stream) {
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (check_mx(R, K) != PROFK_OK || row_stride < K || row_stride > INT64_MAX / 8 / (R > 0 ? R : 1)) return PROFK_EINVAL;
  if (R == 0) return PROFK_OK;
  if (!x || !codes || !scales) return PROFK_ENULL;
  if (!aligned(x, elem_size(dtype)) || !mx_aligned(codes, scales)) return PROFK_EINVAL;
  const hipError_t e = profk::launch_mx_quantize(dtype, x, static_cast<uint64_t>(row_stride), R, K, codes, scales,
                                                 static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_mx4_dequantize(int32_t dtype, const uint8_t* codes, const uint8_t* scales, int64_t R, int64_t K, void* out,
                         void* stream) {
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (check_mx(R, K) != PROFK_OK) return PROFK_EINVAL;
  if (R == 0) return PROFK_OK;
  if (!codes || !scales || !out) return PROFK_ENULL;
  if (!aligned(out, elem_size(dtype)) || !mx_aligned(codes, scales)) return PROFK_EINVAL;
  const hipError_t e =
      profk::launch_mx_dequantize(dtype, codes, scales, R, K, out, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_mx4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, int64_t M, const uint8_t* b_codes,
                     const uint8_t* b_scales, int64_t N, int64_t K, int32_t out_dtype, void* out, void* stream) {
  if (!dtype_ok(out_dtype)) return PROFK_EDTYPE;
  if (check_mx(M, K) != PROFK_OK || check_mx(N, K) != PROFK_OK) return PROFK_EINVAL;
  if (M == 0 || N == 0) return PROFK_OK;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return PROFK_ENULL;
  if (!mx_aligned(a_codes, a_scales) || !mx_aligned(b_codes, b_scales) || !aligned(out, elem_size(out_dtype)))
    return PROFK_EINVAL;
  const profk::MxMatmulCall c{a_codes, a_scales, b_codes, b_scales, M, N, K, out_dtype, out,
                              static_cast<hipStream_t>(stream), nullptr, 0, 0};
  const hipError_t e = profk::launch_mx_matmul(c);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

size_t profk_mx4_linear_workspace_size(int64_t M, int64_t K, int64_t N) {
  if (check_mx(M, K) != PROFK_OK || check_mx(N, K) != PROFK_OK || M == 0 || N == 0) return 0;
  if (profk::mx_quantizes_x(M, K)) return 0;
  return align256(profk_mx4_codes_size(M, K)) + profk_mx4_scales_size(M, K);
}

int profk_mx4_linear(int32_t dtype, const void* x, int64_t M, int64_t K, int64_t row_stride, const uint8_t* w_codes,
                     const uint8_t* w_scales, int64_t N, int32_t out_dtype, void* out, void* ws, size_t ws_bytes,
                     void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return PROFK_EDTYPE;
  if (check_mx(M, K) != PROFK_OK || check_mx(N, K) != PROFK_OK) return PROFK_EINVAL;
  if (row_stride < K || row_stride > INT64_MAX / 8 / (M > 0 ? M : 1)) return PROFK_EINVAL;
  if (M == 0 || N == 0) return PROFK_OK;
  const size_t need = profk_mx4_linear_workspace_size(M, K, N);
  if (!x || !w_codes || !w_scales || !out || (need && !ws)) return PROFK_ENULL;
  if (!aligned(x, elem_size(dtype)) || !mx_aligned(w_codes, w_scales) || !aligned(out, elem_size(out_dtype)) ||
      !aligned(ws, 16))
    return PROFK_EINVAL;
  if (ws_bytes < need) return PROFK_EWORKSPACE;
  if (need == 0) {
    const profk::MxMatmulCall c{nullptr, nullptr, w_codes, w_scales, M, N, K, out_dtype, out,
                                static_cast<hipStream_t>(stream), x, static_cast<uint64_t>(row_stride), dtype};
    const hipError_t e = profk::launch_mx_matmul(c);
    return e == hipSuccess ? PROFK_OK : hip_fail(e);
  }
  uint8_t* const codes = static_cast<uint8_t*>(ws);
  uint8_t* const scales = codes + align256(profk_mx4_codes_size(M, K));
  const int rc = profk_mx4_quantize(dtype, x, M, K, row_stride, codes, scales, stream);
  if (rc != PROFK_OK) return rc;
  return profk_mx4_matmul(codes, scales, M, w_codes, w_scales, N, K, out_dtype, out, stream);
}

// ---- Layer norm ----

namespace {

// Rows of C elements, row_stride apart, whose byte offsets fit 63 bits.
bool rows_ok(int64_t R, int64_t C, int64_t stride) {
  return R >= 0 && R <= static_cast<int64_t>(INT32_MAX) && C >= 0 && stride >= C &&
         stride <= INT64_MAX / 8 / (R > 0 ? R : 1);
}

// A matrix in memory, from its first element to its last.
struct Span {
  uintptr_t at, bytes;
  Span(const void* p, int64_t R, int64_t C, int64_t stride, int32_t dtype)
      : at(reinterpret_cast<uintptr_t>(p)),
        bytes(p && R > 0 && C > 0 ? static_cast<uintptr_t>((R - 1) * stride + C) * elem_size(dtype) : 0) {}
  Span(const void* p, size_t n) : at(reinterpret_cast<uintptr_t>(p)), bytes(p ? n : 0) {}
};
bool overlap(const Span& a, const Span& b) {
  return a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes;
}

// An output that overlaps an input or another output.
bool any_overlap(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span* o = outs.begin(); o != outs.end(); ++o) {
    for (const Span& i : ins)
      if (overlap(*o, i)) return true;
    for (const Span* p = o + 1; p != outs.end(); ++p)
      if (overlap(*o, *p)) return true;
  }
  return false;
}

bool norm_ok(int64_t T, int64_t D) { return T >= 0 && T <= static_cast<int64_t>(INT32_MAX) && D >= 1 && D <= profk::kNormMaxD; }

}  // namespace

int profk_layer_norm(int32_t dtype, const void* x, int64_t T, int64_t D, int64_t x_stride, int32_t param_dtype,
                     const void* weight, const void* bias, float eps, int32_t out_dtype, void* out,
                     int64_t out_stride, float* mean, float* rstd, void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(param_dtype) || !dtype_ok(out_dtype)) return PROFK_EDTYPE;
  if (!norm_ok(T, D) || !rows_ok(T, D, x_stride) || !rows_ok(T, D, out_stride)) return PROFK_EINVAL;
  if (!(eps > 0.0f) || std::isinf(eps)) return PROFK_EINVAL;
  if (T == 0) return PROFK_OK;
  if (!x || !out) return PROFK_ENULL;
  if (!aligned(x, elem_size(dtype)) || !aligned(out, elem_size(out_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4) ||
      !aligned(weight, elem_size(param_dtype)) || !aligned(bias, elem_size(param_dtype)))
    return PROFK_EINVAL;
  const bool same = x == out && dtype == out_dtype && (x_stride == out_stride || T == 1);
  const Span sx(x, T, D, x_stride, dtype), so(out, T, D, out_stride, out_dtype), sm(mean, 1, T, T, PROFK_F32),
      sr(rstd, 1, T, T, PROFK_F32), sw(weight, 1, D, D, param_dtype), sb(bias, 1, D, D, param_dtype);
  if ((!same && overlap(sx, so)) || any_overlap({so, sm, sr}, {sw, sb}) || any_overlap({sm, sr}, {sx})) return PROFK_EINVAL;
  const profk::NormArgs a{x, static_cast<uint64_t>(x_stride), static_cast<uint64_t>(out_stride),
                          static_cast<uint32_t>(T), static_cast<uint32_t>(D), weight, bias, param_dtype, eps, out,
                          mean, rstd};
  const hipError_t e = profk::launch_norm(a, dtype, out_dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

size_t profk_layer_norm_grad_workspace_size(int64_t T, int64_t D) {
  if (!norm_ok(T, D)) return 0;
  return align256(static_cast<size_t>(profk::norm_grad_parts(T, D, profk::device_cu_count())) * 2 * static_cast<size_t>(D) * 4);
}

int profk_layer_norm_grad(int32_t dtype, const void* x, int64_t T, int64_t D, int64_t x_stride, int32_t dy_dtype,
                          const void* dy, int64_t dy_stride, int32_t param_dtype, const void* weight,
                          const float* mean, const float* rstd, void* dx, int64_t dx_stride, void* dweight,
                          void* dbias, void* ws, size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(param_dtype) || !dtype_ok(dy_dtype)) return PROFK_EDTYPE;
  if (!norm_ok(T, D) || !rows_ok(T, D, x_stride) || !rows_ok(T, D, dy_stride) || !rows_ok(T, D, dx_stride))
    return PROFK_EINVAL;
  const bool sums = dweight || dbias;
  if ((T == 0 && !sums) || (!sums && !dx)) return PROFK_OK;
  if ((T > 0 && (!x || !dy || !mean || !rstd)) || (sums && !ws)) return PROFK_ENULL;
  if (!aligned(x, elem_size(dtype)) || !aligned(dx, elem_size(dtype)) || !aligned(dy, elem_size(dy_dtype)) ||
      !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, elem_size(param_dtype)) ||
      !aligned(dweight, elem_size(param_dtype)) || !aligned(dbias, elem_size(param_dtype)) || !aligned(ws, 16))
    return PROFK_EINVAL;
  const Span out(dx, T, D, dx_stride, dtype);
  if (overlap(out, Span(x, T, D, x_stride, dtype)) || overlap(out, Span(dy, T, D, dy_stride, dy_dtype)))
    return PROFK_EINVAL;
  const size_t need = sums ? profk_layer_norm_grad_workspace_size(T, D) : 0;
  if (ws_bytes < need) return PROFK_EWORKSPACE;
  if (any_overlap({out, Span(dweight, 1, D, D, param_dtype), Span(dbias, 1, D, D, param_dtype), Span(ws, need)},
                  {Span(x, T, D, x_stride, dtype), Span(dy, T, D, dy_stride, dy_dtype), Span(weight, 1, D, D, param_dtype),
                   Span(mean, 1, T, T, PROFK_F32), Span(rstd, 1, T, T, PROFK_F32)}))
    return PROFK_EINVAL;
  const profk::NormGradArgs a{x, dy, static_cast<uint64_t>(x_stride), static_cast<uint64_t>(dy_stride),
                              static_cast<uint64_t>(dx_stride), static_cast<uint32_t>(T), static_cast<uint32_t>(D),
                              weight, param_dtype, mean, rstd, dx, dweight, dbias,
                              sums ? static_cast<float*>(ws) : nullptr,
                              profk::norm_grad_parts(T, D, profk::device_cu_count())};
  const hipError_t e = profk::launch_norm_grad(a, dtype, dy_dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

// ---- Dense product ----

namespace {

int check_linear(int64_t M, int64_t K, int64_t x_stride, int64_t N, int64_t w_stride, int32_t act) {
  if (K < 1 || K > profk::kLinMaxK || !rows_ok(M, K, x_stride) || !rows_ok(N, K, w_stride)) return PROFK_EINVAL;
  if (act < PROFK_ACT_NONE || act > PROFK_ACT_SILU) return PROFK_EINVAL;
  return PROFK_OK;
}

}  // namespace

size_t profk_linear_workspace_size(int64_t M, int64_t K, int64_t N) {
  if (check_linear(M, K, K, N, K, PROFK_ACT_NONE) != PROFK_OK || M == 0 || N == 0) return 0;
  return profk::lin_workspace(M, N, K, profk::device_cu_count());
}

int profk_linear(const void* x, int64_t M, int64_t K, int64_t x_stride, const void* w, int64_t N, int64_t w_stride,
                 const float* bias, int32_t activation, int32_t out_dtype, const void* residual,
                 int64_t residual_stride, void* out, void* pre, void* ws, size_t ws_bytes, void* stream) {
  if (!dtype_ok(out_dtype)) return PROFK_EDTYPE;
  if (check_linear(M, K, x_stride, N, w_stride, activation) != PROFK_OK) return PROFK_EINVAL;
  if (residual && !rows_ok(M, N, residual_stride)) return PROFK_EINVAL;
  if (M == 0 || N == 0) return PROFK_OK;
  const size_t need = profk_linear_workspace_size(M, K, N);
  if (!x || !w || !out || (need && !ws)) return PROFK_ENULL;
  const size_t es = elem_size(out_dtype);
  if (!aligned(x, 2) || !aligned(w, 2) || !aligned(bias, 4) || !aligned(residual, es) || !aligned(out, es) ||
      !aligned(pre, es) || !aligned(ws, 16))
    return PROFK_EINVAL;
  const Span sx(x, M, K, x_stride, PROFK_BF16), sw(w, N, K, w_stride, PROFK_BF16), so(out, M, N, N, out_dtype),
      sp(pre, M, N, N, out_dtype), sr(residual, M, N, residual_stride, out_dtype), sb(bias, 1, N, N, PROFK_F32);
  const bool same = residual == out && (residual_stride == N || M == 1);
  if (any_overlap({so, sp}, {sx, sw, sb}) || overlap(sp, sr) || (!same && overlap(so, sr))) return PROFK_EINVAL;
  if (ws_bytes < need) return PROFK_EWORKSPACE;
  if (any_overlap({Span(ws, need)}, {sx, sw, sb, sr, so, sp})) return PROFK_EINVAL;
  const profk::LinCall c{x, w, static_cast<uint64_t>(x_stride), static_cast<uint64_t>(w_stride), M, N, K, bias,
                         activation, out_dtype, residual, static_cast<uint64_t>(residual_stride), out, pre, ws};
  const hipError_t e = profk::launch_linear(c, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

size_t profk_linear_grad_workspace_size(int64_t M, int64_t K, int64_t N) {
  if (check_linear(M, K, K, N, K, PROFK_ACT_NONE) != PROFK_OK) return 0;
  return profk::lin_grad_workspace(M, N, K, profk::device_cu_count());
}

int profk_linear_grad(int32_t dtype, const void* dy, int64_t dy_stride, const void* pre, int32_t activation,
                      const void* x, int64_t M, int64_t K, int64_t x_stride, const void* w, int64_t N,
                      int64_t w_stride, void* dx, void* dw, float* dbias, void* ws, size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  const bool round_dz = activation >= 0 && activation & PROFK_DZ_BF16;
  if (round_dz) activation &= ~PROFK_DZ_BF16;
  if (check_linear(M, K, x_stride, N, w_stride, activation) != PROFK_OK || !rows_ok(M, N, dy_stride)) return PROFK_EINVAL;
  if ((!dx || M == 0) && ((!dw && !dbias) || N == 0)) return PROFK_OK;
  if (M > 0 && N > 0 && (!dy || (activation != PROFK_ACT_NONE && !pre) || (dw && !x) || (dx && !w))) return PROFK_ENULL;
  const size_t need = profk_linear_grad_workspace_size(M, K, N);
  if (need && !ws) return PROFK_ENULL;
  if (!aligned(x, 2) || !aligned(w, 2) || !aligned(dy, elem_size(dtype)) || !aligned(pre, elem_size(dtype)) ||
      !aligned(dx, 2) || !aligned(dw, 2) || !aligned(dbias, 4) || !aligned(ws, 16))
    return PROFK_EINVAL;
  const Span sx(x, M, K, x_stride, PROFK_BF16), sw(w, N, K, w_stride, PROFK_BF16), sd(dy, M, N, dy_stride, dtype),
      sp(pre, M, N, N, dtype), s1(dx, M, K, K, PROFK_BF16), s2(dw, N, K, K, PROFK_BF16), s3(dbias, 1, N, N, PROFK_F32);
  if (any_overlap({s1, s2, s3}, {sx, sw, sd, sp})) return PROFK_EINVAL;
  if (ws_bytes < need) return PROFK_EWORKSPACE;
  if (any_overlap({Span(ws, need)}, {sx, sw, sd, sp, s1, s2, s3})) return PROFK_EINVAL;
  const profk::LinGradCall c{dy, pre, static_cast<uint64_t>(dy_stride), dtype, activation, round_dz, x, w,
                             static_cast<uint64_t>(x_stride), static_cast<uint64_t>(w_stride), M, N, K, dx, dw, dbias,
                             ws};
  const hipError_t e = profk::launch_linear_grad(c, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

// ---- Penalties, biases and masks ----

namespace {

// The parts that both calls have; returns PROFK_OK for a call with rows.
int check_adjust(int32_t dtype, const void* logits, int64_t T, int64_t V, int64_t x_stride, const int64_t* tokens,
                 const int64_t* token_offsets, int64_t n_tokens, const float* repetition, const uint32_t* allowed,
                 int64_t n_masks, int64_t allowed_stride, const int64_t* mask, const void* out, int64_t out_stride,
                 profk::AdjustArgs* a) {
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (V < 1 || V > static_cast<int64_t>(INT32_MAX) || !rows_ok(T, V, x_stride) || !rows_ok(T, V, out_stride))
    return PROFK_EINVAL;
  if (tokens && (n_tokens < 0 || n_tokens > profk::kAdjMaxList)) return PROFK_EINVAL;
  if (allowed) {
    if (n_masks < 1 || allowed_stride < (V + 31) / 32 || allowed_stride > INT64_MAX / 8 / n_masks) return PROFK_EINVAL;
    if (!mask && n_masks != 1 && n_masks != T) return PROFK_EINVAL;
  }
  if (T == 0) return PROFK_OK;
  if (!logits || !out || (tokens && !token_offsets)) return PROFK_ENULL;
  if (!aligned(logits, elem_size(dtype)) || !aligned(out, elem_size(dtype)) || !aligned(tokens, 8) ||
      !aligned(token_offsets, 8) || !aligned(repetition, 4) || !aligned(allowed, 4) || !aligned(mask, 8))
    return PROFK_EINVAL;
  const size_t rows = static_cast<size_t>(T);
  if (any_overlap({Span(out, T, V, out_stride, dtype)},
                  {Span(tokens, static_cast<size_t>(n_tokens) * 8), Span(token_offsets, (rows + 1) * 8),
                   Span(repetition, rows * 4), Span(mask, rows * 8),
                   Span(allowed, allowed ? ((static_cast<size_t>(n_masks) - 1) * static_cast<size_t>(allowed_stride) +
                                            (static_cast<size_t>(V) + 31) / 32) * 4 : 0)}))
    return PROFK_EINVAL;
  a->x = logits;
  a->out = const_cast<void*>(out);
  a->stride = static_cast<uint64_t>(x_stride);
  a->out_stride = static_cast<uint64_t>(out_stride);
  a->V = static_cast<uint32_t>(V);
  a->tokens = tokens;
  a->offsets = token_offsets;
  a->n_tokens = n_tokens;
  a->repetition = repetition;
  a->allowed = allowed;
  a->allowed_stride = static_cast<uint64_t>(allowed_stride);
  a->n_masks = n_masks;
  a->mask = mask;
  return PROFK_OK;
}

}  // namespace

int profk_adjust_logits(int32_t dtype, const void* logits, int64_t T, int64_t V, int64_t x_stride,
                        const int64_t* tokens, const int64_t* token_offsets, int64_t n_tokens,
                        const int64_t* n_prompt, const float* repetition, const float* presence,
                        const float* frequency, const int64_t* bias_ids, const float* bias_values,
                        const int64_t* bias_offsets, int64_t n_bias, const uint32_t* allowed, int64_t n_masks,
                        int64_t allowed_stride, const int64_t* mask, void* out, int64_t out_stride, void* stream) {
  profk::AdjustArgs a{};
  const int rc = check_adjust(dtype, logits, T, V, x_stride, tokens, token_offsets, n_tokens, repetition, allowed,
                              n_masks, allowed_stride, mask, out, out_stride, &a);
  if (rc != PROFK_OK) return rc;
  if (bias_ids && (n_bias < 0 || n_bias > profk::kAdjMaxList)) return PROFK_EINVAL;
  if (T == 0) return PROFK_OK;
  if (bias_ids && (!bias_values || !bias_offsets)) return PROFK_ENULL;
  if (!aligned(n_prompt, 8) || !aligned(presence, 4) || !aligned(frequency, 4) || !aligned(bias_ids, 8) ||
      !aligned(bias_values, 4) || !aligned(bias_offsets, 8))
    return PROFK_EINVAL;
  const bool same = logits == out && (x_stride == out_stride || T == 1);
  const Span so(out, T, V, out_stride, dtype);
  const size_t rows = static_cast<size_t>(T), biases = bias_ids ? static_cast<size_t>(n_bias) : 0;
  if ((!same && overlap(Span(logits, T, V, x_stride, dtype), so)) ||
      any_overlap({so}, {Span(n_prompt, rows * 8), Span(presence, rows * 4), Span(frequency, rows * 4),
                         Span(bias_ids, biases * 8), Span(bias_values, biases * 4), Span(bias_offsets, (rows + 1) * 8)}))
    return PROFK_EINVAL;
  a.n_prompt = n_prompt;
  a.presence = presence;
  a.frequency = frequency;
  a.bias_ids = bias_ids;
  a.bias_values = bias_values;
  a.bias_offsets = bias_offsets;
  a.n_bias = n_bias;
  const hipError_t e = profk::launch_adjust(a, dtype, T, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_adjust_logits_grad(int32_t dtype, const void* d_out, int64_t d_stride, const void* logits, int64_t T,
                             int64_t V, int64_t x_stride, const int64_t* tokens, const int64_t* token_offsets,
                             int64_t n_tokens, const float* repetition, const uint32_t* allowed, int64_t n_masks,
                             int64_t allowed_stride, const int64_t* mask, void* out, int64_t out_stride,
                             void* stream) {
  profk::AdjustArgs a{};
  const int rc = check_adjust(dtype, logits, T, V, x_stride, tokens, token_offsets, n_tokens, repetition, allowed,
                              n_masks, allowed_stride, mask, out, out_stride, &a);
  if (rc != PROFK_OK) return rc;
  if (!rows_ok(T, V, d_stride)) return PROFK_EINVAL;
  if (T == 0) return PROFK_OK;
  if (!d_out) return PROFK_ENULL;
  if (!aligned(d_out, elem_size(dtype))) return PROFK_EINVAL;
  const Span so(out, T, V, out_stride, dtype);
  const bool same = d_out == out && (d_stride == out_stride || T == 1);
  if (overlap(so, Span(logits, T, V, x_stride, dtype)) || (!same && overlap(so, Span(d_out, T, V, d_stride, dtype))))
    return PROFK_EINVAL;
  // (without a repetition penalty the history has no part in the gradient)
  if (!repetition) a.tokens = nullptr;
  a.dy = d_out;
  a.dy_stride = static_cast<uint64_t>(d_stride);
  const hipError_t e = profk::launch_adjust(a, dtype, T, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_debug_sample_indices(uint64_t seed, int64_t row, int64_t S, int64_t N, int64_t* out_dev,
                               void* stream) {
  if (!out_dev) return PROFK_ENULL;
  if (S < 1 || S > static_cast<int64_t>(UINT32_MAX) || N < 1 || row < 0) return PROFK_EINVAL;
  const hipError_t e = profk::launch_sample_indices(seed, static_cast<uint64_t>(row),
                                                    static_cast<uint32_t>(S), static_cast<uint64_t>(N),
                                                    out_dev, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

int profk_debug_filter(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t N,
                       uint32_t tau_key, uint32_t* buf_key, uint32_t* buf_idx, uint32_t* count_dev,
                       void* ws, size_t ws_bytes, void* stream) {
  if (!plan || !values || !buf_key || !buf_idx || !count_dev || !ws) return PROFK_ENULL;
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (!plan_consistent(plan) || plan->N != N) return PROFK_EINVAL;
  if (reinterpret_cast<uintptr_t>(values) % elem_size(dtype) != 0) return PROFK_EINVAL;
  const profk::FlatLayout L = profk::flat_layout(*plan, dtype, profk::device_cu_count());
  if (ws_bytes < L.bytes) return PROFK_EWORKSPACE;
  profk::FlatCall c{plan, dtype, values, static_cast<uint32_t>(N), static_cast<uint32_t>(plan->k), 0, 0,
                    nullptr, nullptr, static_cast<uint8_t*>(ws), L, static_cast<hipStream_t>(stream),
                    nullptr, 1, tau_key};
  const hipError_t e = profk::launch_debug_filter(c, buf_key, buf_idx, count_dev);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

// ---- Entry point that allocates nothing ----
//
// profk_topk_noalloc runs profk_topk's kernels on a fixed device array
// instead of a caller's workspace.  In host code `scratch` names a host-side
// stand-in, not device memory: its device address is looked up once per
// device with hipGetSymbolAddress and only that address is passed on.
static __device__ __align__(256) uint8_t scratch[PROFK_NOALLOC_SCRATCH_BYTES];

namespace {
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_dev[kMaxDevices] = {};

// The current device's copy of `scratch`, looked up on the first call on
// that device (with it current); NULL with *err set when the lookup fails.
void* device_scratch(hipError_t* err) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) { *err = e; return nullptr; }
  if (dev < 0 || dev >= kMaxDevices) { *err = hipErrorInvalidDevice; return nullptr; }
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_dev[dev]) {
    void* ptr = nullptr;
    e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !ptr) { *err = e != hipSuccess ? e : hipErrorInvalidSymbol; return nullptr; }
    g_scratch_dev[dev] = ptr;
  }
  return g_scratch_dev[dev];
}
}  // namespace

int profk_topk_noalloc(const profk_plan_t* plan, int32_t dtype, const void* values, int64_t N, int64_t k,
                       uint64_t seed, void* out_vals, int64_t* out_idx, void* stream, profk_info_t* info_dev) {
  if (!plan || !values || !out_vals || !out_idx) return PROFK_ENULL;
  if (!dtype_ok(dtype)) return PROFK_EDTYPE;
  if (!plan_consistent(plan) || plan->N != N || plan->k != k) return PROFK_EINVAL;
  const size_t need = profk_workspace_size(plan, dtype, 1);
  if (need == 0) return PROFK_EINVAL;
  if (need > static_cast<size_t>(PROFK_NOALLOC_SCRATCH_BYTES)) return PROFK_EWORKSPACE;
  hipError_t e = hipSuccess;
  void* ws = device_scratch(&e);
  if (!ws) return hip_fail(e);
  return run_flat(plan, dtype, values, N, k, seed, 0, out_vals, out_idx, ws, PROFK_NOALLOC_SCRATCH_BYTES,
                  stream, info_dev, 0, 0);
}

int profk_debug_read_probe(const void* values, uint64_t bytes, int32_t blocks_per_cu, int32_t loads_per_lane,
                           uint32_t* out_dev, uint32_t* grid, void* stream) {
  if (!values || !out_dev || !grid) return PROFK_ENULL;
  // the probe's vector indices and its grid stride (at most 2^21 vectors)
  // stay below 2^32
  if (bytes < 16 || bytes % 16 != 0 || bytes / 16 > static_cast<uint64_t>(UINT32_MAX) - (1u << 22))
    return PROFK_EINVAL;
  if (reinterpret_cast<uintptr_t>(values) % 16 != 0) return PROFK_EINVAL;
  if (blocks_per_cu < 1 || blocks_per_cu > 8 || (loads_per_lane != 4 && loads_per_lane != 8)) return PROFK_EINVAL;
  const hipError_t e = profk::launch_read_probe(values, bytes / 16, blocks_per_cu, loads_per_lane, out_dev, grid,
                                                static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

namespace {
std::mutex g_simple_mu;
void* g_simple_ws = nullptr;
size_t g_simple_bytes = 0;
}  // namespace

int profk_topk_simple(const float* values, int64_t N, int64_t k, uint64_t seed, float* out_vals,
                      int64_t* out_idx) {
  profk_plan_t plan;
  int rc = profk_plan(N, k, 1e-6, 1.0, nullptr, &plan);
  if (rc != PROFK_OK) return rc;
  std::lock_guard<std::mutex> lock(g_simple_mu);
  const size_t need = profk_workspace_size(&plan, PROFK_F32, 1);
  if (need == 0) return PROFK_EINVAL;
  if (need > g_simple_bytes) {
    if (g_simple_ws) (void)hipFree(g_simple_ws);
    g_simple_ws = nullptr;
    g_simple_bytes = 0;
    hipError_t e = hipMalloc(&g_simple_ws, need);
    if (e != hipSuccess) return hip_fail(e);
    g_simple_bytes = need;
  }
  rc = profk_topk(&plan, PROFK_F32, values, N, k, seed, out_vals, out_idx, g_simple_ws, g_simple_bytes,
                  nullptr, nullptr);
  if (rc != PROFK_OK) return rc;
  const hipError_t e = hipStreamSynchronize(nullptr);
  return e == hipSuccess ? PROFK_OK : hip_fail(e);
}

void profk_release(void) {
  std::lock_guard<std::mutex> lock(g_simple_mu);
  if (g_simple_ws) (void)hipFree(g_simple_ws);
  g_simple_ws = nullptr;
  g_simple_bytes = 0;
}

const char* profk_status_string(int code) {
  switch (code) {
    case PROFK_OK: return "ok";
    case PROFK_EINVAL: return "invalid argument";
    case PROFK_EDTYPE: return "unsupported dtype";
    case PROFK_EWORKSPACE: return "workspace too small";
    case PROFK_ENULL: return "null pointer";
    case PROFK_EHIP: return "HIP runtime error";
    default: return "unknown status";
  }
}

int profk_last_hip_error(void) { return g_last_hip_error; }

void profk_set_trace_events(void* before, void* after) {
  g_ev_before = static_cast<hipEvent_t>(before);
  g_ev_after = static_cast<hipEvent_t>(after);
}

}  // extern "C"
