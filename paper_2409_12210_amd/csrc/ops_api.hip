// C ABI of the operators around the layer: argument checks, workspace carving, launches.  As in api.hip nothing here allocates
// or synchronises, and all checks come before the first launch.
#include <cmath>
#include <cstring>

#include "ops.h"
#include "ortho.h"

namespace {
modse_status check_dtype(const modse_dtype& dtype) {
  int32_t bits;  // (read as an integer: a caller may have put any value there)
  static_assert(sizeof(modse_dtype) == sizeof(int32_t), "enumeration stored as a 32-bit integer");
  std::memcpy(&bits, &dtype, sizeof bits);
  return bits == (int32_t)MODSE_F32 || bits == (int32_t)MODSE_BF16 ? MODSE_OK : MODSE_ERR_UNSUPPORTED;
}
modse_status check_set(const modse_matrix_set* set) {
  if (!set || set->n_matrices < 0) return MODSE_ERR_INVALID_ARG;
  if (check_dtype(set->dtype) != MODSE_OK || set->n_matrices > modse_ortho::MAX_MATS) return MODSE_ERR_UNSUPPORTED;
  if (set->n_matrices && (!set->rows || !set->cols)) return MODSE_ERR_INVALID_ARG;
  return MODSE_OK;
}
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
modse_status hip_status(hipError_t e) { return e == hipSuccess ? MODSE_OK : MODSE_ERR_HIP; }

constexpr int64_t MAX_ROWS = (int64_t)1 << 31;
modse_status check_norm(int64_t T, int32_t d, const modse_dtype& dtype) {
  if (T < 0 || d < 1) return MODSE_ERR_INVALID_ARG;
  if (check_dtype(dtype) != MODSE_OK || d > MODSE_NORM_MAX_D || T >= MAX_ROWS) return MODSE_ERR_UNSUPPORTED;
  return MODSE_OK;
}
modse_status check_logprobs(int64_t T, int32_t vocab, const modse_dtype& dtype, int32_t top) {
  if (T < 0 || vocab < 1 || top < 0) return MODSE_ERR_INVALID_ARG;
  if (check_dtype(dtype) != MODSE_OK || top > MODSE_LOGPROBS_MAX_TOP) return MODSE_ERR_UNSUPPORTED;
  // (a launch has fewer than 2^32 threads, 256 of them for a row, or for 8192 of its entries)
  if (vocab > 1 << 30 || T >= 1 << 24 || T * ((vocab + 8191) / 8192) >= 1 << 24) return MODSE_ERR_UNSUPPORTED;
  return MODSE_OK;
}
struct LogprobsLayout {
  size_t part, keys, total;
};
LogprobsLayout logprobs_layout(int64_t T, int splits, int top) {
  LogprobsLayout w = {0, 0, 0};
  if (splits == 1) return w;
  w.keys = align_up((size_t)T * splits * sizeof(f32x4), 256);
  w.total = w.keys + align_up((size_t)T * splits * top * sizeof(uint64_t), 256);
  return w;
}
}  // namespace

extern "C" {

modse_status modse_norm_fwd(int64_t T, int32_t d_model, modse_dtype dtype, const void* x, const void* residual,
                            const void* gamma, float eps, void* y, void* h, float* rstd, void* q, float* scale,
                            int32_t group, void* hip_stream) {
  const modse_status st = check_norm(T, d_model, dtype);
  if (st != MODSE_OK) return st;
  if (!(eps >= 0.f) || std::isinf(eps)) return MODSE_ERR_INVALID_ARG;
  if (group != 0 && group != 32 && group != 64 && group != 128) return MODSE_ERR_UNSUPPORTED;
  if (T == 0) return MODSE_OK;
  if (!x || !gamma || !q != !scale || (group && !q) || (!y && !h && !rstd && !q)) return MODSE_ERR_INVALID_ARG;
  const NormFwdArgs a = {x, residual, gamma, y, h, rstd, static_cast<uint8_t*>(q), scale, T, d_model, group, eps};
  return hip_status(launch_norm_fwd(dtype, a, static_cast<hipStream_t>(hip_stream)));
}

modse_status modse_norm_bwd_workspace_size(int64_t T, int32_t d_model, modse_dtype dtype, size_t* bytes) {
  if (!bytes) return MODSE_ERR_INVALID_ARG;
  const modse_status st = check_norm(T, d_model, dtype);
  if (st != MODSE_OK) return st;
  *bytes = (size_t)norm_bwd_blocks(T, d_model) * d_model * sizeof(float);
  return MODSE_OK;
}

modse_status modse_norm_bwd(int64_t T, int32_t d_model, modse_dtype dtype, const void* h, const void* gamma,
                            const float* rstd, const void* dY, const void* dH, void* dX, float* dgamma, int accumulate,
                            void* ws, size_t ws_bytes, void* hip_stream) {
  const modse_status st = check_norm(T, d_model, dtype);
  if (st != MODSE_OK) return st;
  if (T == 0) return MODSE_OK;
  if (!h || !gamma || !rstd || !dY || !dX || !dgamma || !ws || !aligned16(ws)) return MODSE_ERR_INVALID_ARG;
  if (ws_bytes < (size_t)norm_bwd_blocks(T, d_model) * d_model * sizeof(float)) return MODSE_ERR_WORKSPACE;
  const NormBwdArgs a = {h, gamma, rstd, dY, dH, dX, dgamma, static_cast<float*>(ws), T, d_model, accumulate};
  return hip_status(launch_norm_bwd(dtype, a, static_cast<hipStream_t>(hip_stream)));
}

modse_status modse_logprobs_workspace_size(int64_t T, int32_t vocab, modse_dtype dtype, int32_t top, size_t* bytes) {
  if (!bytes) return MODSE_ERR_INVALID_ARG;
  const modse_status st = check_logprobs(T, vocab, dtype, top);
  if (st != MODSE_OK) return st;
  // (fewer rows are cut finer: the most of all calls of at most T rows)
  size_t most = 0;
  for (int64_t t = 1; t <= T; ++t) {
    const int splits = logprobs_split(t, vocab, top).splits;
    if (splits == 1) break;
    const size_t total = logprobs_layout(t, splits, top).total;
    if (total > most) most = total;
  }
  *bytes = most;
  return MODSE_OK;
}

modse_status modse_logprobs_fwd(int64_t T, int32_t vocab, modse_dtype dtype, const void* logits, int64_t ld_logits,
                                const int32_t* targets, float* logp, float* stats, float* entropy, int32_t top,
                                int32_t* top_idx, float* top_logp, void* ws, size_t ws_bytes, void* hip_stream) {
  const modse_status st = check_logprobs(T, vocab, dtype, top);
  if (st != MODSE_OK) return st;
  if (T == 0) return MODSE_OK;
  if (!logits || ld_logits < vocab || !targets != !logp || (top && (!top_idx || !top_logp)) ||
      (!logp && !stats && !entropy && !top))
    return MODSE_ERR_INVALID_ARG;
  const LogprobsSplit split = logprobs_split(T, vocab, top);
  const LogprobsLayout w = logprobs_layout(T, split.splits, top);
  if (w.total && (!ws || !aligned16(ws))) return MODSE_ERR_INVALID_ARG;
  if (ws_bytes < w.total) return MODSE_ERR_WORKSPACE;
  char* const wsb = static_cast<char*>(ws);
  const LogprobsFwdArgs a = {logits, ld_logits, targets, logp, stats, entropy, top_idx, top_logp,
                             reinterpret_cast<f32x4*>(wsb + w.part), reinterpret_cast<uint64_t*>(wsb + w.keys), T, vocab, top};
  return hip_status(launch_logprobs_fwd(dtype, a, split, static_cast<hipStream_t>(hip_stream)));
}

modse_status modse_logprobs_bwd(int64_t T, int32_t vocab, modse_dtype dtype, const void* logits, int64_t ld_logits,
                                const int32_t* targets, const float* stats, const float* entropy, const float* d_logp,
                                const float* d_entropy, void* d_logits, int64_t ld_d_logits, void* hip_stream) {
  const modse_status st = check_logprobs(T, vocab, dtype, 0);
  if (st != MODSE_OK) return st;
  if (T == 0) return MODSE_OK;
  if (!logits || ld_logits < vocab || ld_d_logits < vocab || !stats || !d_logits || !targets != !d_logp ||
      (d_entropy && !entropy) || (d_logits == logits && ld_logits != ld_d_logits))
    return MODSE_ERR_INVALID_ARG;
  const LogprobsBwdArgs a = {logits, ld_logits, targets, stats, entropy, d_logp, d_entropy, d_logits, ld_d_logits, T, vocab};
  return hip_status(launch_logprobs_bwd(dtype, a, static_cast<hipStream_t>(hip_stream)));
}

modse_status modse_orthogonalize_workspace_size(const modse_matrix_set* set, size_t* bytes) {
  if (!bytes) return MODSE_ERR_INVALID_ARG;
  modse_status st = check_set(set);
  if (st != MODSE_OK) return st;
  OrthoLayout w;
  if ((st = ortho_layout(set, nullptr, 0, w)) != MODSE_OK) return st;
  *bytes = w.total;
  return MODSE_OK;
}

modse_status modse_orthogonalize(const modse_matrix_set* set, const float* coeffs, int32_t steps, float eps, void* ws,
                                 size_t ws_bytes, void* hip_stream) {
  using namespace modse_ortho;
  modse_status st = check_set(set);
  if (st != MODSE_OK) return st;
  if (!coeffs || steps < 1 || !(eps >= 0.f) || std::isinf(eps)) return MODSE_ERR_INVALID_ARG;
  if (steps > MAX_STEPS) return MODSE_ERR_UNSUPPORTED;
  double bound = 1;  // of singular values
  for (int i = 0; i < steps; ++i) {
    bound = quintic_bound(coeffs[3 * i], coeffs[3 * i + 1], coeffs[3 * i + 2], bound);
    if (!(bound <= 0x1p40)) return MODSE_ERR_UNSUPPORTED;  // (NaN too)
  }
  OrthoLayout w;
  if ((st = ortho_layout(set, coeffs, steps, w)) != MODSE_OK) return st;
  if (set->n_matrices == 0) return MODSE_OK;
  if (!set->G || !set->U || !ws || reinterpret_cast<uintptr_t>(ws) % 256) return MODSE_ERR_INVALID_ARG;
  for (int i = 0; i < set->n_matrices; ++i)
    if (!set->G[i] || !set->U[i]) return MODSE_ERR_INVALID_ARG;
  if (ws_bytes < w.total) return MODSE_ERR_WORKSPACE;
  return hip_status(launch_orthogonalize(set, w, coeffs, eps, static_cast<char*>(ws), static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
