// Layer norm and root-mean-square norm in front of a block, with the residual stream's addition on the way in and the residual
// gradient's on the way back.  With v = x (+ add, rounded to the storage type, as the stream is stored), per row of N columns
//      mean = sum v / N (layer norm; 0 otherwise)     rstd = (sum (v - mean)^2 / N + eps)^-1/2     hat = (v - mean) rstd     y = hat w + b
//      dx = rstd (h - hat (sum h hat / N) - sum h / N) + dres      with h = dy w; the last sum for layer norm only
//      dw = sum over rows of dy hat     db = sum over rows of dy
// Every sum is fp32.  One pass over memory: a row stays in the registers of its 16, 64 or 256 lanes, 16 bytes to a lane
// and unit, so the mean is subtracted before anything is squared.
#include <type_traits>

#include "kernels.h"
#include "plan.h"
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

// How the rows end: with a whole unit; inside one, which is then read from where it ends with the row and shifted (guarded loads are
// waited for where they stand: 32768 x 4095 703 us, so 504); or they are shorter than one, and read element by element.
enum Ends { kWhole, kInside, kNarrow };
template <typename T, int LPR, int NU, Ends ENDS>
struct RowUnits {
  static constexpr int W = 16 / (int)sizeof(T);
  int cols, l;
  __device__ __forceinline__ int left(int i) const { return cols - (l + i * LPR) * W; }          // elements of the row from the unit's first on
  __device__ __forceinline__ int from(int i) const { return min((l + i * LPR) * W, cols - W); }
  template <bool ONCE> __device__ __forceinline__ void request(Unit<T> (&u)[NU], const T* row) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if constexpr (ENDS == kNarrow) u[i].load(row, left(i));
      else u[i].template load<ONCE>(row + from(i));
    }
  }
  template <bool ONCE> __device__ __forceinline__ void put(const Unit<T>& u, int i, T* row) const {
    T* const p = row + (l + i * LPR) * W;
    if constexpr (ENDS != kWhole) u.template store<ONCE>(p, left(i));
    else if (left(i) > 0) u.template store<ONCE>(p);
  }
  // before they are used: units beyond the row are zeros
  __device__ __forceinline__ void cut(Unit<T> (&u)[NU]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if constexpr (ENDS == kInside) u[i].drop((l + i * LPR) * W - from(i));
      if constexpr (ENDS == kWhole) u[i].keep(left(i) > 0);
    }
  }
};

struct FwdArgs {
  int rows, cols;
  const void *x, *add, *weight, *bias;
  long x_stride, add_stride;
  float eps;
  void *sum, *y;
  float *mean, *rstd;
};

// Bound by memory where there are many rows: 32768 x 4096 bf16, both residual streams, 197 us, 1.07 GB at 5.4 TB/s (a copy of 2 GiB runs at 4.9).  4096 x
// 768 6.7 us, 200 x 2048 3.8, most of it the launch and one way to memory and back.
template <typename T, int LPR, int NU, Ends ENDS, bool LAYER, bool ONCE>
__global__ __launch_bounds__(256) void norm_fwd_kernel(const FwdArgs a) {
  constexpr int RPB = 256 / LPR, W = 16 / (int)sizeof(T);
  __shared__ float red[2][1][4];
  int turn = 0;
  const int l = threadIdx.x % LPR;
  const T* const x = static_cast<const T*>(a.x);
  const T* const add = static_cast<const T*>(a.add);
  T* const y = static_cast<T*>(a.y);
  T* const sum = static_cast<T*>(a.sum);
  const RowUnits<T, LPR, NU, ENDS> at = {a.cols, l};
  Unit<T> w[NU], b[NU];
  at.template request<false>(w, static_cast<const T*>(a.weight));
  at.cut(w);
  if (a.bias) {
    at.template request<false>(b, static_cast<const T*>(a.bias));
    at.cut(b);
  } else {
#pragma unroll
    for (int i = 0; i < NU; ++i) b[i].keep(false);
  }
  const float n = (float)a.cols;
  for (long row = (long)blockIdx.x * RPB + threadIdx.x / LPR; row < a.rows; row += (long)gridDim.x * RPB) {
    Unit<T> in[NU], more[NU];
    at.template request<ONCE>(in, x + row * a.x_stride);
    if (add) at.template request<ONCE>(more, add + row * a.add_stride);
    at.cut(in);
    if (add) at.cut(more);
    float v[NU][W], s = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      in[i].get(v[i]);
      if (add) {
        float o[W];
        more[i].get(o);
#pragma unroll
        for (int e = 0; e < W; ++e) v[i][e] += o[e];
        in[i].set(v[i]);
        at.template put<ONCE>(in[i], i, sum + row * a.cols);
        in[i].get(v[i]);                  // normalised is what is stored
      }
#pragma unroll
      for (int e = 0; e < W; ++e) s += v[i][e];
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
      for (int e = 0; e < W; ++e) {
        if (LAYER) v[i][e] = e < at.left(i) ? v[i][e] - mean : 0.f;
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
      float wf[W], bf[W];
      w[i].get(wf);
      b[i].get(bf);
#pragma unroll
      for (int e = 0; e < W; ++e) v[i][e] = fmaf(v[i][e] * rstd, wf[e], bf[e]);
      in[i].set(v[i]);
      at.template put<ONCE>(in[i], i, y + row * a.cols);
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

// At most 512 blocks, each with its sums of dw and db in registers until its rows are done: 32768 x 4096 bf16, 176 us, 1.07 GB at 6.1 TB/s; 4096 x 768 7.1 us.
// Then norm_columns_kernel adds the blocks' sums in a fixed order, 3.6 us of 768 columns, 4.8 of 4096: atomics would save that launch and give
// another gradient every time.  Its loop has sixteen loads in flight from 481 partial sums on, below one: 383 of 1001 columns 5.6 us.
// Wide rows take registers from each other's latency, 278 to 512 of a lane, spilled ones among them above 8192 columns: 8192 x 8192 fp32 5.1 TB/s, 4096 x 16384 3.9,
// 8192 x 16384 bf16 3.3 (layer norm; the other kind 5.6, 4.1, 4.4).
template <typename T, int LPR, int NU, Ends ENDS, bool LAYER, bool ONCE>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const BwdArgs a) {
  constexpr int RPB = 256 / LPR, N = LAYER ? 2 : 1, W = 16 / (int)sizeof(T);
  __shared__ float red[2][N][4];
  __shared__ float across[RPB > 1 ? 256 * W : 1];
  int turn = 0;
  const int l = threadIdx.x % LPR;
  const T* const dy = static_cast<const T*>(a.dy);
  const T* const x = static_cast<const T*>(a.x);
  const T* const dres = static_cast<const T*>(a.dres);
  T* const dx = static_cast<T*>(a.dx);
  const RowUnits<T, LPR, NU, ENDS> at = {a.cols, l};
  Unit<T> w[NU];
  at.template request<false>(w, static_cast<const T*>(a.weight));
  at.cut(w);
  float dw[NU][W], db[NU][W];
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < W; ++e) dw[i][e] = db[i][e] = 0.f;
  const float inv_n = 1.f / (float)a.cols;
  for (long row = (long)blockIdx.x * RPB + threadIdx.x / LPR; row < a.rows; row += (long)gridDim.x * RPB) {
    Unit<T> g[NU], in[NU], res[NU];
    at.template request<ONCE>(g, dy + row * a.dy_stride);
    at.template request<ONCE>(in, x + row * a.x_stride);
    if (dres) at.template request<ONCE>(res, dres + row * a.dres_stride);
    at.cut(g);
    at.cut(in);
    if (dres) at.cut(res);
    const float rstd = a.rstd[row], mean = LAYER ? a.mean[row] : 0.f;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float gf[W], xf[W], wf[W];
      g[i].get(gf);
      in[i].get(xf);
      w[i].get(wf);
#pragma unroll
      for (int e = 0; e < W; ++e) {        // (columns beyond the row: dy and w are zero)
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
      float gf[W], xf[W], wf[W], o[W];
      g[i].get(gf);
      in[i].get(xf);
      w[i].get(wf);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float hat = (xf[e] - mean) * rstd, h = gf[e] * wf[e];
        o[e] = (h - fmaf(hat, c0, c1)) * rstd;
      }
      if (dres) {
        float rf[W];
        res[i].get(rf);
#pragma unroll
        for (int e = 0; e < W; ++e) o[e] += rf[e];
      }
      in[i].set(o);
      at.template put<ONCE>(in[i], i, dx + row * a.cols);
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
      float (&d)[W] = which ? db[i] : dw[i];
      if (RPB > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < W; ++e) across[e * 256 + threadIdx.x] = d[e];
        __syncthreads();
        if (threadIdx.x < LPR)
#pragma unroll
          for (int e = 0; e < W; ++e)
            for (int r = 1; r < RPB; ++r) d[e] += across[e * 256 + r * LPR + threadIdx.x];
      }
      if (threadIdx.x < LPR) {
#pragma unroll
        for (int h = 0; h < W / 4; ++h) {
          Unit<float> u;
          u.set(d + 4 * h);
          u.store(out + (l + i * LPR) * W + 4 * h, at.left(i) - 4 * h);
        }
      }
    }
  }
}

// out[c] (+)= sum over p, ascending within each of 32 slices and then over these, of part[p][c]: 32 columns to a block
__global__ __launch_bounds__(1024) void norm_columns_kernel(const float* __restrict__ part, int n_part, int cols, float* __restrict__ d_weight,
                                                            float* __restrict__ d_bias, int accumulate) {
  __shared__ float acc[32][33];
  const int x = threadIdx.x & 31, c = blockIdx.x * 32 + x, slice = threadIdx.x >> 5;
  const float* const src = part + (long)blockIdx.y * n_part * cols;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 16
    for (int p = slice; p < n_part; p += 32) s += src[(long)p * cols + c];
  }
  acc[slice][x] = s;
  __syncthreads();
  if (slice == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += acc[i][x];
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
int with_rows(int dtype, int kind, int cols, bool once, F launch) {
  auto typed = [&](auto t) {
    using T = decltype(t);
    constexpr int W = 16 / (int)sizeof(T), UNITS = (int)sizeof(T) / 2;          // fp32: twice as many units
    auto shaped = [&](auto layer) {
      auto with = [&](auto lpr, auto nu) {
        constexpr std::integral_constant<int, decltype(nu)::value * UNITS> units;
        if (cols % W != 0) return launch(t, lpr, units, std::integral_constant<Ends, kInside>{}, layer, std::false_type{});
        if (once) return launch(t, lpr, units, std::integral_constant<Ends, kWhole>{}, layer, std::true_type{});
        return launch(t, lpr, units, std::integral_constant<Ends, kWhole>{}, layer, std::false_type{});
      };
      if (cols < W) return launch(t, std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}, std::integral_constant<Ends, kNarrow>{}, layer, std::false_type{});
      if (cols <= 128) return with(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
      if (cols <= 256) return with(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
      if (cols <= 512) return with(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
      if (cols <= 1024) return with(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
      if (cols <= 2048) return with(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
      if (cols <= 4096) return with(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
      if (cols <= 8192) return with(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
      return with(std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{});
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
  const bool once = plan::norm_streams(dtype == SPES_F32 ? 4 : 2, rows, cols, add ? 4 : 2, x_stride, add ? add_stride : 0, 0);
  FwdArgs a = {rows, cols, x, add, weight, bias, x_stride, add_stride, eps, sum, y, mean, rstd};
  return with_rows(dtype, kind, cols, once, [&](auto t, auto lpr, auto nu, auto ends, auto layer, auto streaming) {
    constexpr int LPR = decltype(lpr)::value, RPB = 256 / LPR;
    const int need = cdiv(rows, RPB), grid = need < 2048 ? need : 2048;
    constexpr int NU = decltype(nu)::value;
    constexpr bool LAYER = decltype(layer)::value;
    hipLaunchKernelGGL((norm_fwd_kernel<decltype(t), LPR, NU, decltype(ends)::value, LAYER, decltype(streaming)::value>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
  });
}

int launch_norm_bwd(int dtype, int kind, int rows, int cols, const void* dy, long dy_stride, const void* x, long x_stride, const void* weight,
                    const float* mean, const float* rstd, const void* dres, long dres_stride, void* dx, float* d_weight, float* d_bias,
                    int accumulate, float* scratch, hipStream_t s) {
  const int grid = rows > 0 ? bwd_blocks(rows, cols) : 0;
  if (grid > 0) {
    const bool once = plan::norm_streams(dtype == SPES_F32 ? 4 : 2, rows, cols, dres ? 4 : 3, x_stride, dy_stride, dres ? dres_stride : 0);
    BwdArgs a = {rows, cols, dy, x, weight, dres, dy_stride, x_stride, dres_stride, mean, rstd, dx, d_weight ? scratch : nullptr, d_bias != nullptr};
    const int rc = with_rows(dtype, kind, cols, once, [&](auto t, auto lpr, auto nu, auto ends, auto layer, auto streaming) {
      constexpr int LPR = decltype(lpr)::value;
      constexpr int NU = decltype(nu)::value;
    constexpr bool LAYER = decltype(layer)::value;
    hipLaunchKernelGGL((norm_bwd_kernel<decltype(t), LPR, NU, decltype(ends)::value, LAYER, decltype(streaming)::value>), dim3(grid), dim3(256), 0, s, a);
      return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
    });
    if (rc != SPES_OK) return rc;
  }
  if (d_weight == nullptr || (grid == 0 && accumulate)) return SPES_OK;
  hipLaunchKernelGGL(norm_columns_kernel, dim3(cdiv(cols, 32), d_bias ? 2 : 1), dim3(1024), 0, s, scratch, grid, cols, d_weight, d_bias, accumulate);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

}  // namespace spes
