// C ABI of the operators around the expert layer: argument checks ahead of any launch.
#include <cmath>
#include <new>

#include "kernels.h"

using namespace spes;

namespace {

bool dtype_ok(int dtype) { return dtype == SPES_F32 || dtype == SPES_BF16; }
bool element_aligned(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == SPES_F32 ? 3u : 1u)) == 0; }

constexpr int kMaxNormCols = 16384;      // a row in the registers of 256 lanes

constexpr int kMaxRouterExperts = 512, kMaxRouterChoice = 16;      // a token's logits in the registers of sixteen lanes, a chosen expert to a lane

int router_supported(int T, int M, int k, const spes_router_opts* o) {
  if (o == nullptr || T < 0 || M < 1 || k < 1 || (o->score != SPES_SCORE_SOFTMAX && o->score != SPES_SCORE_SIGMOID) || !std::isfinite(o->scale))
    return SPES_EINVAL;
  if (o->groups < 1 || o->kept_groups < 1 || o->kept_groups > o->groups || M % o->groups != 0) return SPES_EINVAL;
  if (k > (long)o->kept_groups * (M / o->groups)) return SPES_EINVAL;
  if (M > kMaxRouterExperts || k > kMaxRouterChoice || o->groups > 16) return SPES_ESHAPE;
  return SPES_OK;
}

constexpr int kMaxSide = 16384;      // of a matrix: 32-bit byte offsets into it
constexpr float kCoef[3] = {3.4445f, -4.7750f, 2.0315f};

int matrices_supported(long n, int rows, int cols, int dtype) {
  if (n < 1 || rows < 1 || cols < 1 || !dtype_ok(dtype)) return SPES_EINVAL;
  if (rows > kMaxSide || cols > kMaxSide) return SPES_ESHAPE;
  if (n > 65535) return SPES_ESHAPE;      // a grid dimension
  // a launch has one block for 128 x 128 elements and more of a matrix
  if (n * (((long)rows + 127) / 128) * (((long)cols + 127) / 128) > (1L << 28)) return SPES_ESHAPE;
  return SPES_OK;
}
bool coef_ok(const float* c) { return c == nullptr || (std::isfinite(c[0]) && std::isfinite(c[1]) && std::isfinite(c[2])); }
bool steps_ok(int steps) { return steps >= 1 && steps <= 64; }

}  // namespace

extern "C" {

SPES_API size_t spes_norm_scratch_bytes(int32_t rows, int32_t cols) {
  if (rows < 0 || cols < 1 || cols > kMaxNormCols) return 0;
  return norm_scratch_bytes(rows, cols);
}

SPES_API int spes_norm_fwd(int32_t kind, int32_t rows, int32_t cols, int32_t dtype, const void* x, int64_t x_stride, const void* add,
                           int64_t add_stride, const void* weight, const void* bias, float eps, void* sum, void* y, float* mean, float* rstd,
                           void* stream) {
  if ((kind != SPES_NORM_LAYER && kind != SPES_NORM_RMS) || rows < 0 || cols < 1 || !dtype_ok(dtype) || !(eps >= 0.f)) return SPES_EINVAL;
  if (cols > kMaxNormCols) return SPES_ESHAPE;
  if (rows == 0) return SPES_OK;
  if (!x || !weight || !y || !rstd || (kind == SPES_NORM_LAYER) != (mean != nullptr) || (add != nullptr) != (sum != nullptr)) return SPES_EINVAL;
  if (x_stride < cols || (add && add_stride < cols)) return SPES_EINVAL;
  if (!element_aligned(x, dtype) || !element_aligned(add, dtype) || !aligned16(weight) || !aligned16(bias) || !aligned16(sum) || !aligned16(y) ||
      !aligned16(mean) || !aligned16(rstd))
    return SPES_EALIGN;
  return launch_norm_fwd(dtype, kind, rows, cols, x, x_stride, add, add_stride, weight, bias, eps, sum, y, mean, rstd, static_cast<hipStream_t>(stream));
}

SPES_API int spes_norm_bwd(int32_t kind, int32_t rows, int32_t cols, int32_t dtype, const void* dy, int64_t dy_stride, const void* x,
                           int64_t x_stride, const void* weight, const float* mean, const float* rstd, const void* dres, int64_t dres_stride,
                           void* dx, float* d_weight, float* d_bias, int32_t accumulate, void* scratch, void* stream) {
  if ((kind != SPES_NORM_LAYER && kind != SPES_NORM_RMS) || rows < 0 || cols < 1 || !dtype_ok(dtype)) return SPES_EINVAL;
  if (cols > kMaxNormCols) return SPES_ESHAPE;
  if ((d_bias && !d_weight) || (d_weight && !scratch && rows > 0)) return SPES_EINVAL;
  if (rows > 0) {
    if (!dy || !x || !weight || !rstd || !dx || (kind == SPES_NORM_LAYER) != (mean != nullptr)) return SPES_EINVAL;
    if (dy_stride < cols || x_stride < cols || (dres && dres_stride < cols)) return SPES_EINVAL;
  }
  if (!element_aligned(dy, dtype) || !element_aligned(x, dtype) || !element_aligned(dres, dtype) || !aligned16(weight) || !aligned16(mean) ||
      !aligned16(rstd) || !aligned16(dx) || !aligned16(d_weight) || !aligned16(d_bias) || !aligned16(scratch))
    return SPES_EALIGN;
  return launch_norm_bwd(dtype, kind, rows, cols, dy, dy_stride, x, x_stride, weight, mean, rstd, dres, dres_stride, dx, d_weight, d_bias,
                         accumulate != 0, static_cast<float*>(scratch), static_cast<hipStream_t>(stream));
}

SPES_API int spes_router_fwd(int32_t T, int32_t n_experts, int32_t top_k, const spes_router_opts* opts, const float* logits, const float* bias,
                             int32_t* idx, float* gate, int32_t* count, void* stream) {
  const int rc = router_supported(T, n_experts, top_k, opts);
  if (rc != SPES_OK) return rc;
  if (!count || (T > 0 && (!logits || !idx || !gate))) return SPES_EINVAL;
  if (!aligned16(logits) || !aligned16(bias) || !aligned16(idx) || !aligned16(gate) || !aligned16(count)) return SPES_EALIGN;
  return launch_router_fwd(T, n_experts, top_k, *opts, logits, bias, idx, gate, count, static_cast<hipStream_t>(stream));
}

SPES_API int spes_router_bwd(int32_t T, int32_t n_experts, int32_t top_k, const spes_router_opts* opts, const float* logits, const int32_t* idx,
                             const float* dgate, float* dlogits, void* stream) {
  const int rc = router_supported(T, n_experts, top_k, opts);
  if (rc != SPES_OK) return rc;
  if (T == 0) return SPES_OK;
  if (!logits || !idx || !dgate || !dlogits) return SPES_EINVAL;
  if (!aligned16(logits) || !aligned16(idx) || !aligned16(dgate) || !aligned16(dlogits)) return SPES_EALIGN;
  return launch_router_bwd(T, n_experts, top_k, *opts, logits, idx, dgate, dlogits, static_cast<hipStream_t>(stream));
}

SPES_API size_t spes_orthogonalize_scratch_bytes(int32_t n, int32_t rows, int32_t cols, int32_t dtype) {
  return matrices_supported(n, rows, cols, dtype) == SPES_OK ? orthogonalize_scratch_bytes(n, rows, cols, dtype) : 0;
}

SPES_API int spes_orthogonalize(int32_t n, int32_t rows, int32_t cols, int32_t dtype, const void* src, void* out, int32_t steps, const float* coef,
                                void* scratch, void* stream) {
  const int rc = matrices_supported(n, rows, cols, dtype);
  if (rc != SPES_OK) return rc;
  if (!src || !out || !scratch || !steps_ok(steps) || !coef_ok(coef)) return SPES_EINVAL;
  if (!aligned16(src) || !aligned16(out) || !aligned16(scratch)) return SPES_EALIGN;
  return launch_orthogonalize(dtype, n, rows, cols, src, out, steps, coef ? coef : kCoef, scratch, static_cast<hipStream_t>(stream));
}

SPES_API int spes_masked_muon(int32_t n_experts, int32_t rows, int32_t cols, int32_t dtype, void* param, const uint8_t* trainable_mask, float* master,
                              float* m, const float* grad, float lr, float beta, int32_t nesterov, float weight_decay, float update_scale, int32_t steps,
                              const float* coef, float grad_scale, void* scratch, void* stream) {
  if (n_experts < 1 || !param || !trainable_mask || !(beta >= 0.f && beta < 1.f) || !steps_ok(steps) || !coef_ok(coef)) return SPES_EINVAL;
  int n = 0;
  for (int e = 0; e < n_experts; ++e) n += trainable_mask[e] != 0;
  const int rc = matrices_supported(n > 0 ? n : 1, rows, cols, dtype);
  if (rc != SPES_OK) return rc;
  if (n == 0) return SPES_OK;
  if (!m || !grad || !scratch || (!master && dtype != SPES_F32)) return SPES_EINVAL;
  if (!aligned16(param) || !aligned16(m) || !aligned16(grad) || !aligned16(master) || !aligned16(scratch)) return SPES_EALIGN;
  long* const param_at = new (std::nothrow) long[n];
  if (param_at == nullptr) return SPES_EINVAL;
  for (int e = 0, i = 0; e < n_experts; ++e)
    if (trainable_mask[e]) param_at[i++] = (long)e * rows * cols;
  const int status = launch_masked_muon(dtype, n, rows, cols, param, param_at, master, m, grad, lr, beta, nesterov, weight_decay, update_scale, steps,
                                        coef ? coef : kCoef, grad_scale, scratch, static_cast<hipStream_t>(stream));
  delete[] param_at;
  return status;
}

}  // extern "C"
