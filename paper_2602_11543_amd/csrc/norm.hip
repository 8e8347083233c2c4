// Layer norm and root-mean-square norm in front of a block, with the residual stream's addition on the way in and the residual
// gradient's on the way back.  With v = x (+ add, rounded to the storage type, as the stream is stored), per row of N columns
//      mean = sum v / N (layer norm; 0 otherwise)     rstd = (sum (v - mean)^2 / N + eps)^-1/2     hat = (v - mean) rstd     y = hat w + b
//      dx = rstd (h - hat (sum h hat / N) - sum h / N) + dres      with h = dy w; the last sum for layer norm only
//      dw = sum over rows of dy hat     db = sum over rows of dy
// Every sum is fp32.  One pass over memory: a row stays in the registers of its 16, 64 or 256 lanes, eight columns to a lane
// and unit, so the mean is subtracted before anything is squared.
#include <type_traits>

#include "kernels.h"
#include "units.h"

namespace spes {
namespace {

// Sums of N values at once over the LPR lanes of a row, in all of them.  256 lanes: through LDS, in one of two places in turn, so that
// one barrier a call is enough (a wavefront that is a call ahead writes the other place).
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float* v, float (*red)[N][4], int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = LPR == 16 ? lane_group_sum<16>(v[i]) : wave_sum(v[i]);
  if (LPR == 256) {
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[turn][i][threadIdx.x >> 6] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (red[turn][i][0] + red[turn][i][1]) + (red[turn][i][2] + red[turn][i][3]);
  }
}

struct FwdArgs {
  int rows, cols;
  const void *x, *add, *weight, *bias;
  long x_stride, add_stride;
  float eps;
  void *sum, *y;
  float *mean, *rstd;
};

template <typename T, int LPR, int NU, bool LAYER>
__global__ __launch_bounds__(256) void norm_fwd_kernel(const FwdArgs a) {
  constexpr int RPB = 256 / LPR;
  __shared__ float red[2][1][4];
  int turn = 0;
  const int l = threadIdx.x % LPR;
  const T* const x = static_cast<const T*>(a.x);
  const T* const add = static_cast<const T*>(a.add);
  T* const y = static_cast<T*>(a.y);
  T* const sum = static_cast<T*>(a.sum);
  int left[NU];
  Unit<T> w[NU], b[NU];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = (l + i * LPR) * 8;
    left[i] = a.cols - c;
    w[i].load(static_cast<const T*>(a.weight) + (left[i] > 0 ? c : 0), left[i]);
    b[i].load(static_cast<const T*>(a.bias) + (left[i] > 0 ? c : 0), a.bias ? left[i] : 0);
  }
  const float n = (float)a.cols;
  for (long row = (long)blockIdx.x * RPB + threadIdx.x / LPR; row < a.rows; row += (long)gridDim.x * RPB) {
    Unit<T> in[NU], more[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = left[i] > 0 ? (l + i * LPR) * 8 : 0;
      in[i].load(x + row * a.x_stride + c, left[i]);
      if (add) more[i].load(add + row * a.add_stride + c, left[i]);
    }
    float v[NU][8], s = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      in[i].get(v[i]);
      if (add) {
        float o[8];
        more[i].get(o);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] += o[e];
        in[i].set(v[i]);
        in[i].store(sum + row * a.cols + (l + i * LPR) * 8, left[i]);
        in[i].get(v[i]);                  // normalised is what is stored
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[i][e];
    }
    float mean = 0.f;
    if (LAYER) {
      row_sums<LPR, 1>(&s, red, turn);
      mean = s / n;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (LAYER) v[i][e] = e < left[i] ? v[i][e] - mean : 0.f;
        q = fmaf(v[i][e], v[i][e], q);
      }
    row_sums<LPR, 1>(&q, red, turn);
    const float rstd = 1.f / sqrtf(q / n + a.eps);
    if (l == 0) {
      a.rstd[row] = rstd;
      if (LAYER) a.mean[row] = mean;
    }
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float wf[8], bf[8];
      w[i].get(wf);
      b[i].get(bf);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e] * rstd, wf[e], bf[e]);
      in[i].set(v[i]);
      in[i].store(y + row * a.cols + (l + i * LPR) * 8, left[i]);
    }
  }
}

struct BwdArgs {
  int rows, cols;
  const void *dy, *x, *weight, *dres;
  long dy_stride, x_stride, dres_stride;
  const float *mean, *rstd;
  void* dx;
  float* part;          // [blocks][cols] of dw, then of db; NULL: no gradient of the weight
  bool bias;
};

template <typename T, int LPR, int NU, bool LAYER>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const BwdArgs a) {
  constexpr int RPB = 256 / LPR, N = LAYER ? 2 : 1;
  __shared__ float red[2][N][4];
  __shared__ float across[RPB > 1 ? 256 * 8 : 1];
  int turn = 0;
  const int l = threadIdx.x % LPR;
  const T* const dy = static_cast<const T*>(a.dy);
  const T* const x = static_cast<const T*>(a.x);
  const T* const dres = static_cast<const T*>(a.dres);
  T* const dx = static_cast<T*>(a.dx);
  int left[NU];
  Unit<T> w[NU];
  float dw[NU][8], db[NU][8];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = (l + i * LPR) * 8;
    left[i] = a.cols - c;
    w[i].load(static_cast<const T*>(a.weight) + (left[i] > 0 ? c : 0), left[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.f;
  }
  const float inv_n = 1.f / (float)a.cols;
  for (long row = (long)blockIdx.x * RPB + threadIdx.x / LPR; row < a.rows; row += (long)gridDim.x * RPB) {
    Unit<T> g[NU], in[NU], res[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = left[i] > 0 ? (l + i * LPR) * 8 : 0;
      g[i].load(dy + row * a.dy_stride + c, left[i]);
      in[i].load(x + row * a.x_stride + c, left[i]);
      if (dres) res[i].load(dres + row * a.dres_stride + c, left[i]);
    }
    const float rstd = a.rstd[row], mean = LAYER ? a.mean[row] : 0.f;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float gf[8], xf[8], wf[8];
      g[i].get(gf);
      in[i].get(xf);
      w[i].get(wf);
#pragma unroll
      for (int e = 0; e < 8; ++e) {        // (columns beyond the row: dy and w are zero)
        const float hat = (xf[e] - mean) * rstd, h = gf[e] * wf[e];
        dw[i][e] = fmaf(gf[e], hat, dw[i][e]);
        db[i][e] += gf[e];
        s[0] = fmaf(h, hat, s[0]);
        s[1] += h;
      }
    }
    row_sums<LPR, N>(s, red, turn);
    const float c0 = s[0] * inv_n, c1 = LAYER ? s[1] * inv_n : 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float gf[8], xf[8], wf[8], o[8];
      g[i].get(gf);
      in[i].get(xf);
      w[i].get(wf);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hat = (xf[e] - mean) * rstd, h = gf[e] * wf[e];
        o[e] = (h - fmaf(hat, c0, c1)) * rstd;
      }
      if (dres) {
        float rf[8];
        res[i].get(rf);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += rf[e];
      }
      in[i].set(o);
      in[i].store(dx + row * a.cols + (l + i * LPR) * 8, left[i]);
    }
  }
  if (a.part == nullptr) return;
  // the block's rows side by side, added in their order
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which == 1 && !a.bias) break;
    float* const out = a.part + ((long)which * gridDim.x + blockIdx.x) * a.cols;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float (&d)[8] = which ? db[i] : dw[i];
      if (RPB > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) across[e * 256 + threadIdx.x] = d[e];
        __syncthreads();
        if (threadIdx.x < LPR)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            for (int r = 1; r < RPB; ++r) d[e] += across[e * 256 + r * LPR + threadIdx.x];
      }
      if (threadIdx.x < LPR) {
        Unit<float> u;
        u.set(d);
        u.store(out + (l + i * LPR) * 8, left[i]);
      }
    }
  }
}

// out[c] (+)= sum over p, ascending within each of eight slices and then over these, of part[p][c]: 32 columns to a block
__global__ __launch_bounds__(256) void norm_columns_kernel(const float* __restrict__ part, int n_part, int cols, float* __restrict__ d_weight,
                                                           float* __restrict__ d_bias, int accumulate) {
  __shared__ float acc[8][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  const float* const src = part + (long)blockIdx.y * n_part * cols;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int p = slice; p < n_part; p += 8) s += src[(long)p * cols + c];
  }
  acc[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice == 0 && c < cols) {
    for (int i = 1; i < 8; ++i) s += acc[i][threadIdx.x];
    float* const out = blockIdx.y ? d_bias : d_weight;
    out[c] = accumulate ? out[c] + s : s;
  }
}

int lanes_per_row(int cols) { return cols <= 256 ? 16 : cols <= 1024 ? 64 : 256; }

// blocks of the backward pass, each with a partial sum of the weight's gradient
int bwd_blocks(int rows, int cols) {
  const int need = cdiv(rows, 256 / lanes_per_row(cols));
  return need < 512 ? need : 512;
}

template <typename F>
int with_rows(int dtype, int kind, int cols, F launch) {
  auto typed = [&](auto t) {
    using T = decltype(t);
    auto shaped = [&](auto layer) {
      using L = decltype(layer);
      if (cols <= 128) return launch(t, std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}, L{});
      if (cols <= 256) return launch(t, std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{}, L{});
      if (cols <= 512) return launch(t, std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{}, L{});
      if (cols <= 1024) return launch(t, std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{}, L{});
      if (cols <= 2048) return launch(t, std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{}, L{});
      if (cols <= 4096) return launch(t, std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{}, L{});
      if (cols <= 8192) return launch(t, std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{}, L{});
      return launch(t, std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{}, L{});
    };
    return kind == SPES_NORM_LAYER ? shaped(std::true_type{}) : shaped(std::false_type{});
  };
  return dtype == SPES_F32 ? typed(float{}) : typed(bf16_t{});
}

}  // namespace

size_t norm_scratch_bytes(int rows, int cols) { return (size_t)2 * (rows > 0 ? bwd_blocks(rows, cols) : 1) * cols * 4; }

int launch_norm_fwd(int dtype, int kind, int rows, int cols, const void* x, long x_stride, const void* add, long add_stride, const void* weight,
                    const void* bias, float eps, void* sum, void* y, float* mean, float* rstd, hipStream_t s) {
  if (rows == 0) return SPES_OK;
  FwdArgs a = {rows, cols, x, add, weight, bias, x_stride, add_stride, eps, sum, y, mean, rstd};
  return with_rows(dtype, kind, cols, [&](auto t, auto lpr, auto nu, auto layer) {
    constexpr int LPR = decltype(lpr)::value, RPB = 256 / LPR;
    const int need = cdiv(rows, RPB), grid = need < 2048 ? need : 2048;
    hipLaunchKernelGGL((norm_fwd_kernel<decltype(t), LPR, decltype(nu)::value, decltype(layer)::value>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
  });
}

int launch_norm_bwd(int dtype, int kind, int rows, int cols, const void* dy, long dy_stride, const void* x, long x_stride, const void* weight,
                    const float* mean, const float* rstd, const void* dres, long dres_stride, void* dx, float* d_weight, float* d_bias,
                    int accumulate, float* scratch, hipStream_t s) {
  const int grid = rows > 0 ? bwd_blocks(rows, cols) : 0;
  if (grid > 0) {
    BwdArgs a = {rows, cols, dy, x, weight, dres, dy_stride, x_stride, dres_stride, mean, rstd, dx, d_weight ? scratch : nullptr, d_bias != nullptr};
    const int rc = with_rows(dtype, kind, cols, [&](auto t, auto lpr, auto nu, auto layer) {
      constexpr int LPR = decltype(lpr)::value;
      hipLaunchKernelGGL((norm_bwd_kernel<decltype(t), LPR, decltype(nu)::value, decltype(layer)::value>), dim3(grid), dim3(256), 0, s, a);
      return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
    });
    if (rc != SPES_OK) return rc;
  }
  if (d_weight == nullptr || (grid == 0 && accumulate)) return SPES_OK;
  hipLaunchKernelGGL(norm_columns_kernel, dim3(cdiv(cols, 32), d_bias ? 2 : 1), dim3(256), 0, s, scratch, grid, cols, d_weight, d_bias, accumulate);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

}  // namespace spes
