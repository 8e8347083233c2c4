// C ABI of the operators around the expert layer: argument checks ahead of any launch.
#include <cmath>

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

}  // extern "C"
