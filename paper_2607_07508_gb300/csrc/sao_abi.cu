// extern "C" entry points of libsao: argument checks, workspace carving and
// dispatch to the kernel launchers. See include/sao.h for the contract.
#include <math.h>
#include <stdint.h>

#include <atomic>

#include <nvtx3/nvToolsExt.h>

#include "balance.cuh"
#include "distill.cuh"
#include "grads.cuh"
#include "logprobs_common.cuh"
#include "norm.cuh"
#include "route.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"

namespace sao {

static std::atomic<size_t> g_dz_budget{size_t(4) << 30};
void set_dz_budget(size_t bytes) { g_dz_budget.store(bytes < (size_t(1) << 20) ? (size_t(1) << 20) : bytes); }
size_t dz_budget() { return g_dz_budget.load(); }

static std::atomic<int> g_cta_pairs{0};
void set_cta_pairs(int on) { g_cta_pairs.store(on ? 1 : 0); }
int cta_group() { return g_cta_pairs.load() ? 2 : 1; }

static std::atomic<uint64_t> g_scan_wait_ns{kWaitLimitNs};
static std::atomic<int> g_scan_skip{0};
uint64_t scan_wait_ns() { return g_scan_wait_ns.load(); }
int scan_skip() { return g_scan_skip.load(); }

// O(N) kernels size their grids from N alone (deterministic on any device).
size_t on_ws_bytes(int64_t N) {
  size_t w = elementwise_ws_bytes(N, 0);
  const size_t g = gae_ws_bytes(N, N + 1);
  const size_t st = step_gae_ws_bytes(N, N + 1);
  const size_t bl = baselines_ws_bytes(N, N + 1);
  if (g > w) w = g;
  if (st > w) w = st;
  if (bl > w) w = bl;
  return w;
}

size_t logprobs_ws_bytes(int64_t N, int32_t h, int32_t V, sao_dtype dt) {
  if (h <= 0 || V <= 0) return 0;
  return dt == SAO_BF16 ? tc_ws_bytes(N, h, V) : f32_ws_bytes(N, h, V);
}

}  // namespace sao

using namespace sao;

namespace {

// An NVTX range around every entry point, so a profiler timeline shows the
// ABI calls with their kernels (header-only NVTX: no cost without a tool).
struct NvtxRange {
  explicit NvtxRange(const char *name) { nvtxRangePushA(name); }
  ~NvtxRange() { nvtxRangePop(); }
  NvtxRange(const NvtxRange &) = delete;
  NvtxRange &operator=(const NvtxRange &) = delete;
};
#define SAO_RANGE() NvtxRange sao_nvtx_range_(__func__)

struct Ws {
  unsigned int *err;
  void *body;
  size_t body_bytes;
};

sao_status take_ws(void *ws, size_t ws_bytes, size_t need_body, Ws *out) {
  if (ws == nullptr) return fail(SAO_ERR_INVALID_ARG, "workspace is NULL");
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return fail(SAO_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
  if (ws_bytes < kWsHeader + need_body)
    return fail(SAO_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, kWsHeader + need_body);
  out->err = static_cast<unsigned int *>(ws);
  out->body = static_cast<char *>(ws) + kWsHeader;
  out->body_bytes = ws_bytes - kWsHeader;
  return SAO_OK;
}

bool bad_dtype(sao_dtype dt) { return dt != SAO_F32 && dt != SAO_BF16; }

sao_status check_logprob_shapes(sao_dtype dt, int64_t N, int32_t h, int32_t V) {
  if (bad_dtype(dt)) return fail(SAO_ERR_UNSUPPORTED, "unknown dtype %d", int(dt));
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (h < 1 || V < 1) return fail(SAO_ERR_SHAPE, "h = %d and V = %d must be >= 1", h, V);
  if (dt == SAO_BF16 && (h % 8) != 0) return fail(SAO_ERR_SHAPE, "bf16 needs h %% 8 == 0 (h = %d)", h);
  return SAO_OK;
}

sao_status check_tc_device(sao_dtype dt) {
  if (dt != SAO_BF16) return SAO_OK;
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  if (di.cc_major != 10 || di.cc_minor != 3)
    return fail(SAO_ERR_UNSUPPORTED, "the bf16 tensor-core path needs an sm_103 device (found sm_%d%d)",
                di.cc_major, di.cc_minor);
  return SAO_OK;
}

}  // namespace

extern "C" {

int sao_version(void) { return 100; }

const char *sao_last_error_string(void) { return last_error(); }

void sao_set_checked(int on) { set_checked(on); }
int sao_get_checked(void) { return checked_mode() ? 1 : 0; }

void sao_set_dz_budget_bytes(size_t bytes) { set_dz_budget(bytes); }
size_t sao_get_dz_budget_bytes(void) { return dz_budget(); }

void sao_set_cta_pairs(int on) { set_cta_pairs(on); }
int sao_get_cta_pairs(void) { return cta_group() == 2 ? 1 : 0; }

void sao_debug_set_scan_hooks(uint64_t wait_ns, int32_t skip_chunks) {
  g_scan_wait_ns.store(wait_ns == 0 ? kWaitLimitNs : (wait_ns > kWaitLimitNs ? kWaitLimitNs : wait_ns));
  g_scan_skip.store(skip_chunks > 0 ? skip_chunks : 0);
}

size_t sao_workspace_bytes(int64_t N, int32_t h, int32_t V, sao_dtype dt) {
  if (N < 0 || h < 0 || V < 0 || bad_dtype(dt)) return 0;
  size_t body = on_ws_bytes(N);
  const size_t lp = logprobs_ws_bytes(N, h, V, dt);
  if (lp > body) body = lp;
  return kWsHeader + body;
}

sao_status sao_token_logprobs_fwd(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                  const uint8_t *row_mask, int64_t N, int32_t h, int32_t V, float *logp,
                                  float *lse, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_logprob_shapes(dt, N, h, V));
  if (N == 0) return SAO_OK;
  if (!H || !W || !y || !logp || !lse) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  SAO_TRY(check_tc_device(dt));
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, logprobs_ws_bytes(N, h, V, dt), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  if (dt == SAO_BF16)
    SAO_TRY(tc_fwd(H, W, y, row_mask, N, h, V, logp, lse, w.err, w.body, w.body_bytes, nullptr, s));
  else
    SAO_TRY(f32_fwd(static_cast<const float *>(H), static_cast<const float *>(W), y, row_mask, N, h, V, logp,
                     lse, w.err, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_token_logprobs_bwd(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                  const float *lse, const float *grad_logp, int64_t N, int32_t h, int32_t V,
                                  void *dH, float *dW, int accumulate_dW, void *ws, size_t ws_bytes,
                                  sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_logprob_shapes(dt, N, h, V));
  if (!W || !dW) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (N == 0) {
    if (!accumulate_dW) SAO_CUDA_TRY(cudaMemsetAsync(dW, 0, sizeof(float) * size_t(V) * size_t(h), s));
    return SAO_OK;
  }
  if (!H || !y || !lse || !grad_logp || !dH) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  SAO_TRY(check_tc_device(dt));
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, logprobs_ws_bytes(N, h, V, dt), &w));
  SAO_TRY(begin_call(ws, s));
  if (dt == SAO_BF16)
    SAO_TRY(tc_bwd(H, W, y, lse, grad_logp, N, h, V, dH, dW, accumulate_dW, w.err, w.body, w.body_bytes, nullptr,
                   s));
  else
    SAO_TRY(f32_bwd(static_cast<const float *>(H), static_cast<const float *>(W), y, lse, grad_logp, N, h, V,
                     static_cast<float *>(dH), dW, accumulate_dW, w.err, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

size_t sao_logprob_cache_bytes(int64_t N, int32_t V) {
  if (N <= 0 || V <= 0) return 0;
  return logprob_cache_view(nullptr, N, V).bytes;
}

// The cache must hold sao_logprob_cache_bytes(N, V) bytes at a 256-byte
// aligned address (its parts are TMA operands and 16-byte vector streams).
static sao_status take_cache(const void *cache, size_t cache_bytes, int64_t N, int32_t V, LogprobCache *out) {
  if (!cache) return fail(SAO_ERR_INVALID_ARG, "NULL probability cache");
  if ((reinterpret_cast<uintptr_t>(cache) & 255u) != 0)
    return fail(SAO_ERR_INVALID_ARG, "probability cache not 256-byte aligned");
  *out = logprob_cache_view(const_cast<void *>(cache), N, V);
  if (cache_bytes < out->bytes)
    return fail(SAO_ERR_WORKSPACE, "probability cache too small: %zu bytes, need %zu", cache_bytes, out->bytes);
  return SAO_OK;
}

sao_status sao_token_logprobs_fwd_cached(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                         const uint8_t *row_mask, int64_t N, int32_t h, int32_t V, float *logp,
                                         float *lse, void *cache, size_t cache_bytes, void *ws, size_t ws_bytes,
                                         sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_logprob_shapes(dt, N, h, V));
  if (dt != SAO_BF16) return fail(SAO_ERR_UNSUPPORTED, "the probability cache is for bf16 only");
  if (N == 0) return SAO_OK;
  if (!H || !W || !y || !logp || !lse) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  SAO_TRY(check_tc_device(dt));
  LogprobCache k;
  SAO_TRY(take_cache(cache, cache_bytes, N, V, &k));
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, logprobs_ws_bytes(N, h, V, dt), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(tc_fwd(H, W, y, row_mask, N, h, V, logp, lse, w.err, w.body, w.body_bytes, &k, s));
  return finish_call(ws, s);
}

sao_status sao_token_logprobs_bwd_cached(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                         const float *lse, const float *grad_logp, int64_t N, int32_t h, int32_t V,
                                         void *dH, float *dW, int accumulate_dW, const void *cache,
                                         size_t cache_bytes, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_logprob_shapes(dt, N, h, V));
  if (dt != SAO_BF16) return fail(SAO_ERR_UNSUPPORTED, "the probability cache is for bf16 only");
  if (!W || !dW) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (N == 0) {
    if (!accumulate_dW) SAO_CUDA_TRY(cudaMemsetAsync(dW, 0, sizeof(float) * size_t(V) * size_t(h), s));
    return SAO_OK;
  }
  if (!H || !y || !lse || !grad_logp || !dH) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  SAO_TRY(check_tc_device(dt));
  LogprobCache k;
  SAO_TRY(take_cache(cache, cache_bytes, N, V, &k));
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, logprobs_ws_bytes(N, h, V, dt), &w));
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(tc_bwd(H, W, y, lse, grad_logp, N, h, V, dH, dW, accumulate_dW, w.err, w.body, w.body_bytes, &k, s));
  return finish_call(ws, s);
}

sao_status sao_advantages(const float *values, const float *rewards, const uint8_t *loss_mask,
                          const int32_t *cu_seqlens, int32_t B, int64_t N, float gamma, float lambda_policy,
                          float lambda_critic, float len_adaptive_alpha, float *adv, float *ret, void *ws,
                          size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (B < 0) return fail(SAO_ERR_SHAPE, "B = %d < 0", B);
  if (N > 0 && B == 0) return fail(SAO_ERR_SHAPE, "N > 0 tokens need at least one trajectory");
  if (!(gamma >= 0.f && gamma <= 1.f) || !(lambda_policy >= 0.f && lambda_policy <= 1.f) ||
      !(lambda_critic >= 0.f && lambda_critic <= 1.f) || !isfinite(len_adaptive_alpha))
    return fail(SAO_ERR_INVALID_ARG, "gamma and lambdas must lie in [0, 1] and alpha be finite");
  if (N == 0) return SAO_OK;
  if (!values || !rewards || !loss_mask || !cu_seqlens || !adv || !ret)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, gae_ws_bytes(N, B), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(gae_launch(values, rewards, loss_mask, cu_seqlens, B, N, gamma, lambda_policy, lambda_critic,
                     len_adaptive_alpha, adv, ret, w.err, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_step_advantages(const float *values, const float *rewards, const uint8_t *loss_mask,
                               const int32_t *cu_seqlens, int32_t B, int64_t N, float gamma, float lambda_policy,
                               float lambda_critic, float len_adaptive_alpha, int mode, float *adv, float *ret,
                               uint8_t *value_mask, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (B < 0) return fail(SAO_ERR_SHAPE, "B = %d < 0", B);
  if (N > 0 && B == 0) return fail(SAO_ERR_SHAPE, "N > 0 tokens need at least one trajectory");
  if (mode != SAO_STEP_AVERAGE && mode != SAO_STEP_LAST) return fail(SAO_ERR_INVALID_ARG, "unknown step mode %d", mode);
  if (!(gamma >= 0.f && gamma <= 1.f) || !(lambda_policy >= 0.f && lambda_policy <= 1.f) ||
      !(lambda_critic >= 0.f && lambda_critic <= 1.f) || !isfinite(len_adaptive_alpha))
    return fail(SAO_ERR_INVALID_ARG, "gamma and lambdas must lie in [0, 1] and alpha be finite");
  if (N == 0) return SAO_OK;
  if (!values || !rewards || !loss_mask || !cu_seqlens || !adv || !ret)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, step_gae_ws_bytes(N, B), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(step_gae_launch(values, rewards, loss_mask, cu_seqlens, B, N, gamma, lambda_policy, lambda_critic,
                          len_adaptive_alpha, mode, adv, ret, value_mask, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

static sao_status check_eps(float eps_low, float eps_high) {
  if (!(eps_low >= 0.f) || !(eps_high >= 0.f) || isnan(eps_low) || isnan(eps_high))
    return fail(SAO_ERR_INVALID_ARG, "clip bounds must be >= 0 (eps_low = %g, eps_high = %g)", eps_low, eps_high);
  return SAO_OK;
}

sao_status sao_policy_loss_fwd(const float *logp, const float *old_logp, const float *adv,
                               const uint8_t *loss_mask, int64_t N, float eps_low, float eps_high, int64_t n_norm,
                               float *loss, float *coef, uint8_t *flags, int64_t *counts, void *ws,
                               size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0) return fail(SAO_ERR_SHAPE, "N < 0");
  SAO_TRY(check_eps(eps_low, eps_high));
  if (!loss || !counts) return fail(SAO_ERR_INVALID_ARG, "NULL loss or counts");
  if (N > 0 && (!logp || !old_logp || !adv || !loss_mask)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, elementwise_ws_bytes(N, 0), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(policy_loss_launch(logp, old_logp, adv, loss_mask, N, eps_low, eps_high, n_norm, loss, coef, flags,
                             counts, nullptr, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_policy_loss_bwd(const float *logp, const float *old_logp, const float *adv,
                               const uint8_t *loss_mask, int64_t N, float eps_low, float eps_high, int64_t n_norm,
                               const float *grad_loss, float *grad_logp, void *ws, size_t ws_bytes,
                               sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0) return fail(SAO_ERR_SHAPE, "N < 0");
  SAO_TRY(check_eps(eps_low, eps_high));
  if (N == 0) return SAO_OK;
  if (!logp || !old_logp || !adv || !loss_mask || !grad_loss || !grad_logp)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, elementwise_ws_bytes(N, 0), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(policy_loss_launch(logp, old_logp, adv, loss_mask, N, eps_low, eps_high, n_norm, nullptr, grad_logp,
                             nullptr, nullptr, grad_loss, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

static sao_status check_band(float w_low, float w_high) {
  if (!(w_low >= 0.f) || !(w_high > w_low) || isnan(w_low) || isnan(w_high))
    return fail(SAO_ERR_INVALID_ARG, "mismatch band needs 0 <= w_low < w_high (w_low = %g, w_high = %g)", w_low,
                w_high);
  return SAO_OK;
}

sao_status sao_decoupled_loss_fwd(const float *logp, const float *prox_logp, const float *rollout_logp,
                                  const float *adv, const uint8_t *loss_mask, int64_t N, float eps_low,
                                  float eps_high, float w_low, float w_high, int64_t n_norm, float *loss,
                                  float *coef, uint8_t *flags, int64_t *counts, void *ws, size_t ws_bytes,
                                  sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0) return fail(SAO_ERR_SHAPE, "N < 0");
  SAO_TRY(check_eps(eps_low, eps_high));
  SAO_TRY(check_band(w_low, w_high));
  if (!loss || !counts) return fail(SAO_ERR_INVALID_ARG, "NULL loss or counts");
  if (N > 0 && (!logp || !prox_logp || !rollout_logp || !adv || !loss_mask))
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, elementwise_ws_bytes(N, 0), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(decoupled_loss_launch(logp, prox_logp, rollout_logp, adv, loss_mask, N, eps_low, eps_high, w_low, w_high,
                                n_norm, loss, coef, flags, counts, nullptr, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_decoupled_loss_bwd(const float *logp, const float *prox_logp, const float *rollout_logp,
                                  const float *adv, const uint8_t *loss_mask, int64_t N, float eps_low,
                                  float eps_high, float w_low, float w_high, int64_t n_norm, const float *grad_loss,
                                  float *grad_logp, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0) return fail(SAO_ERR_SHAPE, "N < 0");
  SAO_TRY(check_eps(eps_low, eps_high));
  SAO_TRY(check_band(w_low, w_high));
  if (N == 0) return SAO_OK;
  if (!logp || !prox_logp || !rollout_logp || !adv || !loss_mask || !grad_loss || !grad_logp)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, elementwise_ws_bytes(N, 0), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(decoupled_loss_launch(logp, prox_logp, rollout_logp, adv, loss_mask, N, eps_low, eps_high, w_low, w_high,
                                n_norm, nullptr, grad_logp, nullptr, nullptr, grad_loss, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_value_loss(const float *values, const float *ret, const uint8_t *loss_mask, int64_t N, int64_t n_norm,
                          float *loss, float *grad_values, double *ev_sums, void *ws, size_t ws_bytes,
                          sao_stream_t stream) {
  SAO_RANGE();
  if (N < 0) return fail(SAO_ERR_SHAPE, "N < 0");
  if (!loss) return fail(SAO_ERR_INVALID_ARG, "NULL loss");
  if (N > 0 && (!values || !ret || !loss_mask || !grad_values)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, elementwise_ws_bytes(N, 0), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(value_loss_launch(values, ret, loss_mask, N, n_norm, loss, grad_values, ev_sums, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

static sao_status check_traj(int32_t B, int64_t N, const int32_t *cu) {
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (B < 0) return fail(SAO_ERR_SHAPE, "B = %d < 0", B);
  if (N > 0 && (B == 0 || !cu)) return fail(SAO_ERR_SHAPE, "N > 0 tokens need at least one trajectory");
  return SAO_OK;
}

sao_status sao_clip_loss_fwd(const float *logp, const float *old_logp, const float *adv, const uint8_t *loss_mask,
                             const int32_t *cu_seqlens, int32_t B, int64_t N, float eps_low, float eps_high, int norm,
                             float *loss, float *coef, uint8_t *flags, int64_t *counts, void *ws, size_t ws_bytes,
                             sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_traj(B, N, cu_seqlens));
  SAO_TRY(check_eps(eps_low, eps_high));
  if (norm != SAO_NORM_TOKEN && norm != SAO_NORM_SEQUENCE) return fail(SAO_ERR_INVALID_ARG, "unknown norm %d", norm);
  if (!loss || !counts) return fail(SAO_ERR_INVALID_ARG, "NULL loss or counts");
  if (N > 0 && (!logp || !old_logp || !adv || !loss_mask)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, baselines_ws_bytes(N, B), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(clip_loss_launch(logp, old_logp, adv, loss_mask, cu_seqlens, B, N, eps_low, eps_high, norm, loss, coef,
                           flags, counts, nullptr, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_clip_loss_bwd(const float *logp, const float *old_logp, const float *adv, const uint8_t *loss_mask,
                             const int32_t *cu_seqlens, int32_t B, int64_t N, float eps_low, float eps_high, int norm,
                             const float *grad_loss, float *grad_logp, void *ws, size_t ws_bytes,
                             sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_traj(B, N, cu_seqlens));
  SAO_TRY(check_eps(eps_low, eps_high));
  if (norm != SAO_NORM_TOKEN && norm != SAO_NORM_SEQUENCE) return fail(SAO_ERR_INVALID_ARG, "unknown norm %d", norm);
  if (N == 0) return SAO_OK;
  if (!logp || !old_logp || !adv || !loss_mask || !grad_loss || !grad_logp)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, baselines_ws_bytes(N, B), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(clip_loss_launch(logp, old_logp, adv, loss_mask, cu_seqlens, B, N, eps_low, eps_high, norm, nullptr,
                           grad_logp, nullptr, nullptr, grad_loss, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_group_advantages(const float *rewards, const int32_t *group_ids, int32_t B, const uint8_t *loss_mask,
                                const int32_t *cu_seqlens, int64_t N, float eps_stab, float *adv, void *ws,
                                size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_traj(B, N, cu_seqlens));
  if (!(eps_stab >= 0.f) || !isfinite(eps_stab)) return fail(SAO_ERR_INVALID_ARG, "eps_stab must be >= 0");
  if (N == 0) return SAO_OK;
  if (!rewards || !group_ids || !loss_mask || !adv) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, baselines_ws_bytes(N, B), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(group_adv_launch(rewards, group_ids, B, loss_mask, cu_seqlens, N, eps_stab, adv, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_running_mean_advantages(const float *rewards, const int32_t *prompt_ids, int32_t B,
                                       int32_t num_prompts, float *history, int64_t *seen, int32_t window,
                                       const uint8_t *loss_mask, const int32_t *cu_seqlens, int64_t N, float *adv,
                                       void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_traj(B, N, cu_seqlens));
  if (window < 1 || num_prompts < 1) return fail(SAO_ERR_INVALID_ARG, "window and num_prompts must be >= 1");
  if (B > 0 && (!rewards || !prompt_ids || !history || !seen)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  if (N > 0 && (!loss_mask || !adv)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, baselines_ws_bytes(N, B), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(running_mean_launch(rewards, prompt_ids, B, num_prompts, history, seen, window, loss_mask, cu_seqlens, N,
                              adv, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

static sao_status check_distill(sao_dtype dt, sao_dtype top_dt, int64_t N, int32_t h, int32_t V, int32_t K,
                                float temperature) {
  SAO_TRY(check_logprob_shapes(dt, N, h, V));
  if (bad_dtype(top_dt)) return fail(SAO_ERR_UNSUPPORTED, "unknown dtype %d of the teacher's logits", int(top_dt));
  if (K < 1 || K > SAO_DISTILL_MAX_K) return fail(SAO_ERR_SHAPE, "K = %d not in 1..%d", K, SAO_DISTILL_MAX_K);
  // tiles of 128 rows x 256 columns are numbered in 32 bits
  if (((N + 127) / 128) * ((int64_t(V) + 255) / 256) >= (int64_t(1) << 31))
    return fail(SAO_ERR_SHAPE, "N = %lld rows of V = %d are too many tiles", (long long)N, V);
  if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature))
    return fail(SAO_ERR_INVALID_ARG, "temperature must be positive and finite (%g)", temperature);
  return SAO_OK;
}

size_t sao_distill_workspace_bytes(int64_t N, int32_t h, int32_t V, int32_t K, sao_dtype dt) {
  if (N < 0 || h < 1 || V < 1 || K < 1 || K > SAO_DISTILL_MAX_K || bad_dtype(dt)) return 0;
  return kWsHeader + distill_ws_most(N, h, V, K, dt);
}

sao_status sao_distill_loss_fwd(const void *H, const void *W, sao_dtype dt, const int32_t *top_ids,
                                const void *top_logits, sao_dtype top_dt, const float *teacher_lse,
                                const uint8_t *row_mask, int64_t N, int32_t h, int32_t V, int32_t K,
                                float temperature, float *loss, float *lse, float *lse_rest, float *z_top, void *ws,
                                size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_distill(dt, top_dt, N, h, V, K, temperature));
  if (N == 0) return SAO_OK;
  if (!H || !W || !top_ids || !top_logits || !loss || !lse || !lse_rest || !z_top)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  if (dt == SAO_BF16 && (!aligned16(H) || !aligned16(W)))
    return fail(SAO_ERR_INVALID_ARG, "H and W of a bf16 head must be 16-byte aligned");
  SAO_TRY(check_tc_device(dt));
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, distill_ws_bytes(N, h, V, K, dt), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(distill_fwd_launch(H, W, dt, top_ids, top_logits, top_dt, teacher_lse, row_mask, N, h, V, K, temperature,
                             loss, lse, lse_rest, z_top, w.err, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_distill_loss_bwd(const void *H, const void *W, sao_dtype dt, const int32_t *top_ids,
                                const void *top_logits, sao_dtype top_dt, const float *teacher_lse, const float *lse,
                                const float *lse_rest, const float *z_top, const float *grad_loss, int64_t N,
                                int32_t h, int32_t V, int32_t K, float temperature, void *dH, void *dW,
                                sao_dtype dw_dt, int accumulate_dW, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_distill(dt, top_dt, N, h, V, K, temperature));
  if (bad_dtype(dw_dt) || (dw_dt == SAO_BF16 && dt != SAO_BF16))
    return fail(SAO_ERR_UNSUPPORTED, "dW is fp32, or bf16 for a bf16 head");
  if (dw_dt == SAO_BF16 && accumulate_dW)
    return fail(SAO_ERR_UNSUPPORTED, "a bf16 dW is overwritten: only an fp32 one can be added to");
  if (!W || !dW) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (N == 0) {
    if (!accumulate_dW) SAO_CUDA_TRY(cudaMemsetAsync(dW, 0, (dw_dt == SAO_BF16 ? 2 : 4) * size_t(V) * size_t(h), s));
    return SAO_OK;
  }
  if (!H || !top_ids || !top_logits || !lse || !lse_rest || !z_top || !grad_loss || !dH)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  if (dt == SAO_BF16 && (!aligned16(H) || !aligned16(W) || !aligned16(dH) || !aligned16(dW)))
    return fail(SAO_ERR_INVALID_ARG, "H, W, dH and dW of a bf16 head must be 16-byte aligned");
  SAO_TRY(check_tc_device(dt));
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, distill_ws_bytes(N, h, V, K, dt), &w));
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(distill_bwd_launch(H, W, dt, top_ids, top_logits, top_dt, teacher_lse, lse, lse_rest, z_top, grad_loss, N, h,
                             V, K, temperature, dH, dW, dw_dt, accumulate_dW, w.err, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

static sao_status check_balance(sao_dtype dt, const int32_t *cu, int32_t B, int64_t N, int32_t E, int32_t k,
                                int score) {
  if (bad_dtype(dt)) return fail(SAO_ERR_UNSUPPORTED, "unknown dtype %d", int(dt));
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (E < 1 || E > SAO_BALANCE_MAX_EXPERTS || k < 1 || k > E)
    return fail(SAO_ERR_SHAPE, "E = %d experts, k = %d: 1 <= k <= E <= %d", E, k, SAO_BALANCE_MAX_EXPERTS);
  if (cu && (B < 0 || (N > 0 && B == 0))) return fail(SAO_ERR_SHAPE, "N > 0 tokens need at least one trajectory");
  if (cu && int64_t(B) * ((E + 31) / 32) >= (int64_t(1) << 31))
    return fail(SAO_ERR_SHAPE, "B = %d trajectories of %d experts are too many", B, E);
  if (score != SAO_SCORE_SOFTMAX && score != SAO_SCORE_SIGMOID)
    return fail(SAO_ERR_INVALID_ARG, "unknown score %d", score);
  return SAO_OK;
}

size_t sao_balance_workspace_bytes(int64_t N, int32_t E, int32_t B) {
  if (N < 0 || E < 1 || E > SAO_BALANCE_MAX_EXPERTS || B < 0) return 0;
  return kWsHeader + balance_ws_bytes(N, E, B < 1 ? 1 : B);
}

sao_status sao_balance_loss_fwd(const void *logits, sao_dtype dt, const int32_t *expert_ids, const uint8_t *row_mask,
                                const int32_t *cu_seqlens, int32_t B, int64_t N, int32_t E, int32_t k, int score,
                                float *loss, int64_t *counts, float *prob_sums, int64_t *rows, void *ws,
                                size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_balance(dt, cu_seqlens, B, N, E, k, score));
  if (!loss) return fail(SAO_ERR_INVALID_ARG, "NULL loss");
  const int32_t segments = cu_seqlens ? B : 1;
  if (segments > 0 && (!counts || !prob_sums || !rows)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  if (N > 0 && (!logits || !expert_ids)) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (N == 0) {
    SAO_CUDA_TRY(cudaMemsetAsync(loss, 0, sizeof(float), s));
    if (segments > 0) {
      SAO_CUDA_TRY(cudaMemsetAsync(counts, 0, sizeof(int64_t) * size_t(segments) * size_t(E), s));
      SAO_CUDA_TRY(cudaMemsetAsync(prob_sums, 0, sizeof(float) * size_t(segments) * size_t(E), s));
      SAO_CUDA_TRY(cudaMemsetAsync(rows, 0, sizeof(int64_t) * size_t(segments), s));
    }
    return SAO_OK;
  }
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, balance_ws_bytes(N, E, segments), &w));
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(balance_fwd_launch(logits, dt, expert_ids, row_mask, cu_seqlens, segments, N, E, k, score, loss, counts,
                             prob_sums, rows, w.err, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_balance_loss_bwd(const void *logits, sao_dtype dt, const uint8_t *row_mask, const int32_t *cu_seqlens,
                                int32_t B, int64_t N, int32_t E, int32_t k, int score, const int64_t *counts,
                                const int64_t *rows, const float *grad_loss, void *grad_logits, void *ws,
                                size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_balance(dt, cu_seqlens, B, N, E, k, score));
  if (N == 0) return SAO_OK;
  if (!logits || !counts || !rows || !grad_loss || !grad_logits)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, 0, &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(balance_bwd_launch(logits, dt, row_mask, cu_seqlens, cu_seqlens ? B : 1, N, E, k, score, counts, rows,
                             grad_loss, grad_logits, w.err, s));
  return finish_call(ws, s);
}

static sao_status check_route(sao_dtype dt, int64_t N, int32_t E, int32_t k, int score, float scale) {
  if (bad_dtype(dt)) return fail(SAO_ERR_UNSUPPORTED, "unknown dtype %d", int(dt));
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (E < 1 || E > SAO_ROUTE_MAX_EXPERTS) return fail(SAO_ERR_SHAPE, "E = %d: 1 <= E <= %d", E, SAO_ROUTE_MAX_EXPERTS);
  if (k < 1 || k > SAO_ROUTE_MAX_K || k > E)
    return fail(SAO_ERR_SHAPE, "k = %d of %d experts: 1 <= k <= %d", k, E, SAO_ROUTE_MAX_K);
  if (score != SAO_SCORE_SOFTMAX && score != SAO_SCORE_SIGMOID)
    return fail(SAO_ERR_INVALID_ARG, "unknown score %d", score);
  if (!isfinite(scale)) return fail(SAO_ERR_INVALID_ARG, "scale must be finite (%g)", scale);
  return SAO_OK;
}

static bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

size_t sao_route_workspace_bytes(int64_t N, int32_t E) {
  if (N < 0 || E < 1 || E > SAO_ROUTE_MAX_EXPERTS) return 0;
  return kWsHeader;
}

sao_status sao_route_fwd(const void *logits, sao_dtype dt, const float *bias, const uint8_t *row_mask, int64_t N,
                         int32_t E, int32_t k, int score, int32_t groups, int32_t groups_kept, int group_score,
                         int renormalise, float scale, int replay, int32_t *expert_ids, float *weights, void *ws,
                         size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_route(dt, N, E, k, score, scale));
  if (!replay) {
    if (groups < 1 || groups > SAO_ROUTE_MAX_GROUPS || E % groups != 0 || groups_kept < 1 || groups_kept > groups)
      return fail(SAO_ERR_SHAPE, "%d of %d groups of %d experts", groups_kept, groups, E);
    if (k > groups_kept * (E / groups))
      return fail(SAO_ERR_SHAPE, "k = %d of %d experts that stay", k, groups_kept * (E / groups));
    if (group_score != SAO_GROUP_MAX && group_score != SAO_GROUP_TOP2)
      return fail(SAO_ERR_INVALID_ARG, "unknown group_score %d", group_score);
  }
  if (N == 0) return SAO_OK;
  if (!logits || !expert_ids || !weights) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  if (!aligned_to(logits, dt == SAO_BF16 ? 2 : 4) || !aligned_to(bias, 4) || !aligned_to(expert_ids, 4) ||
      !aligned_to(weights, 4))
    return fail(SAO_ERR_INVALID_ARG, "an array is not aligned to its elements");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, 0, &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(route_fwd_launch({logits, bias, row_mask, N, E, k, score, groups, groups_kept, group_score == SAO_GROUP_TOP2,
                            renormalise, scale, replay, expert_ids, weights, w.err}, dt, s));
  return finish_call(ws, s);
}

sao_status sao_route_bwd(const void *logits, sao_dtype dt, const uint8_t *row_mask, int64_t N, int32_t E, int32_t k,
                         int score, int renormalise, float scale, const int32_t *expert_ids, const float *weights,
                         const float *grad_weights, void *grad_logits, int accumulate, void *ws, size_t ws_bytes,
                         sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_route(dt, N, E, k, score, scale));
  if (N == 0) return SAO_OK;
  if (!logits || !expert_ids || !weights || !grad_weights || !grad_logits)
    return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  if (!aligned_to(logits, dt == SAO_BF16 ? 2 : 4) || !aligned_to(grad_logits, dt == SAO_BF16 ? 2 : 4) ||
      !aligned_to(expert_ids, 4) || !aligned_to(weights, 4) || !aligned_to(grad_weights, 4))
    return fail(SAO_ERR_INVALID_ARG, "an array is not aligned to its elements");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, 0, &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(route_bwd_launch({logits, row_mask, N, E, k, score, renormalise, scale, expert_ids, weights, grad_weights,
                            grad_logits, accumulate, w.err}, dt, s));
  return finish_call(ws, s);
}

static sao_status check_norm(sao_dtype dt, sao_dtype w_dt, int64_t N, int32_t h) {
  if (bad_dtype(dt) || bad_dtype(w_dt)) return fail(SAO_ERR_UNSUPPORTED, "unknown dtype %d or %d", int(dt), int(w_dt));
  if (N < 0 || N >= (int64_t(1) << 31)) return fail(SAO_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (h < 1 || h > SAO_NORM_MAX_H) return fail(SAO_ERR_SHAPE, "h = %d: 1 <= h <= %d", h, SAO_NORM_MAX_H);
  return SAO_OK;
}

size_t sao_norm_workspace_bytes(int64_t N, int32_t h) {
  if (N < 0 || h < 1 || h > SAO_NORM_MAX_H) return 0;
  return kWsHeader + norm_ws_bytes(N, h);
}

sao_status sao_rms_norm_fwd(const void *x, const void *residual, sao_dtype dt, const void *weight, sao_dtype w_dt,
                            float eps, int64_t N, int32_t h, void *sum, void *y, float *rstd, uint8_t *y8,
                            void *scales, int scaling, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_norm(dt, w_dt, N, h));
  if (!(eps >= 0.f) || isinf(eps)) return fail(SAO_ERR_INVALID_ARG, "eps must be finite and not negative (%g)", eps);
  if (scaling < SAO_SCALE_NONE || scaling > SAO_SCALE_MX32)
    return fail(SAO_ERR_INVALID_ARG, "unknown scaling %d", scaling);
  if (N == 0) return SAO_OK;
  if (!x || !weight || (!y && !y8)) return fail(SAO_ERR_INVALID_ARG, "NULL x, weight, or neither y nor y8");
  if (!residual != !sum) return fail(SAO_ERR_INVALID_ARG, "residual and sum are given together or not at all");
  if (!y8 != !scales || !y8 != (scaling == SAO_SCALE_NONE))
    return fail(SAO_ERR_INVALID_ARG, "y8, scales and a scaling are given together or not at all");
  const unsigned unit = dt == SAO_BF16 ? 2 : 4;
  if (!aligned_to(x, unit) || !aligned_to(residual, unit) || !aligned_to(sum, unit) || !aligned_to(y, unit) ||
      !aligned_to(weight, w_dt == SAO_BF16 ? 2 : 4) || !aligned_to(rstd, 4) ||
      (scaling != SAO_SCALE_MX32 && !aligned_to(scales, 4)))
    return fail(SAO_ERR_INVALID_ARG, "an array is not aligned to its elements");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, 0, &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(norm_fwd_launch({x, residual, weight, sum, y, rstd, y8, scales, scaling, eps, N, h}, dt, w_dt, s));
  return finish_call(ws, s);
}

sao_status sao_rms_norm_bwd(const void *sum, sao_dtype dt, const void *weight, sao_dtype w_dt, const float *rstd,
                            const void *dy, const void *dsum, int64_t N, int32_t h, void *dx, float *dweight,
                            int accumulate, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_norm(dt, w_dt, N, h));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (N == 0) {
    if (dweight && !accumulate) SAO_CUDA_TRY(cudaMemsetAsync(dweight, 0, sizeof(float) * size_t(h), s));
    return SAO_OK;
  }
  if (!sum || !weight || !rstd || !dy || !dx) return fail(SAO_ERR_INVALID_ARG, "NULL array argument");
  const unsigned unit = dt == SAO_BF16 ? 2 : 4;
  if (!aligned_to(sum, unit) || !aligned_to(dy, unit) || !aligned_to(dsum, unit) || !aligned_to(dx, unit) ||
      !aligned_to(weight, w_dt == SAO_BF16 ? 2 : 4) || !aligned_to(rstd, 4) || !aligned_to(dweight, 4))
    return fail(SAO_ERR_INVALID_ARG, "an array is not aligned to its elements");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, dweight ? norm_ws_bytes(N, h) : 0, &w));
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(norm_bwd_launch({sum, weight, rstd, dy, dsum, dx, dweight, accumulate, N, h}, dt, w_dt, w.body,
                          w.body_bytes, s));
  return finish_call(ws, s);
}

static sao_status check_tensors(const sao_tensor *t, int32_t count, const char *what) {
  for (int32_t i = 0; i < count; ++i) {
    if (bad_dtype(t[i].dt)) return fail(SAO_ERR_UNSUPPORTED, "%s[%d]: unknown dtype %d", what, i, int(t[i].dt));
    if (t[i].n < 0 || t[i].n >= (int64_t(1) << 48))
      return fail(SAO_ERR_SHAPE, "%s[%d]: %lld elements", what, i, (long long)t[i].n);
    if (t[i].n > 0 && !t[i].data) return fail(SAO_ERR_INVALID_ARG, "%s[%d] is NULL", what, i);
    if (!aligned_to(t[i].data, t[i].dt == SAO_BF16 ? 2 : 4))
      return fail(SAO_ERR_INVALID_ARG, "%s[%d] is not aligned to its elements", what, i);
  }
  return SAO_OK;
}

static sao_status check_lists(const sao_tensor *grads, const sao_tensor *out, int32_t count) {
  if (count < 0) return fail(SAO_ERR_SHAPE, "count = %d", count);
  if (count > 0 && !grads) return fail(SAO_ERR_INVALID_ARG, "NULL list");
  SAO_TRY(check_tensors(grads, count, "grads"));
  if (out) {
    SAO_TRY(check_tensors(out, count, "out"));
    for (int32_t i = 0; i < count; ++i)
      if (out[i].n != grads[i].n)
        return fail(SAO_ERR_SHAPE, "out[%d] has %lld elements, grads[%d] %lld", i, (long long)out[i].n, i,
                    (long long)grads[i].n);
  }
  return check_disjoint(grads, out, count);
}

size_t sao_grad_workspace_bytes(void) { return kWsHeader + grad_ws_bytes(); }

sao_status sao_grad_sumsq(const sao_tensor *grads, int32_t count, double *sumsq, void *ws, size_t ws_bytes,
                          sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_lists(grads, nullptr, count));
  if (!sumsq) return fail(SAO_ERR_INVALID_ARG, "NULL sumsq");
  if (!aligned_to(sumsq, 8)) return fail(SAO_ERR_INVALID_ARG, "sumsq is not aligned to its elements");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, grad_ws_bytes(), &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(grad_sumsq_launch(grads, count, sumsq, w.body, w.body_bytes, s));
  return finish_call(ws, s);
}

sao_status sao_grad_clip(const sao_tensor *grads, const sao_tensor *out, int32_t count, const double *sumsq,
                         float max_norm, float *norm, float *coef, void *ws, size_t ws_bytes, sao_stream_t stream) {
  SAO_RANGE();
  SAO_TRY(check_lists(grads, out, count));
  if (!(max_norm > 0.f)) return fail(SAO_ERR_INVALID_ARG, "max_norm must be positive (%g)", max_norm);
  if (!sumsq || !norm || !coef) return fail(SAO_ERR_INVALID_ARG, "NULL sumsq, norm or coef");
  if (!aligned_to(sumsq, 8) || !aligned_to(norm, 4) || !aligned_to(coef, 4))
    return fail(SAO_ERR_INVALID_ARG, "sumsq, norm or coef is not aligned to its elements");
  Ws w;
  SAO_TRY(take_ws(ws, ws_bytes, 0, &w));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  SAO_TRY(begin_call(ws, s));
  SAO_TRY(grad_clip_launch(grads, out, count, sumsq, max_norm, norm, coef, s));
  return finish_call(ws, s);
}

void sao_profile_enable(int on) { profile_enable(on); }
void sao_profile_reset(void) { profile_reset(); }
int sao_profile_read(const char **names, int64_t *launches, double *total_ms, int cap) {
  return profile_read(names, launches, total_ms, cap);
}

}  // extern "C"
