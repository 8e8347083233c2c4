// Queries and keys ahead of attention: the root-mean-square norm of every head and the rotation by the token's position, in one pass.  Per head x of D elements
//      rstd = (sum x^2 / D + eps)^-1/2      hat = x rstd      y = hat w        pairs (a, b) of the first `rot` elements of y -> (a c - b s, a s + b c)
// and for the gradient dz, with every pair turned back into dy,
//      dw = sum over tokens and heads of dy hat      h = dy w      dx = rstd (h - hat (sum h hat / D))
// Sums are fp32, a result is rounded once.  A lane holds two chunks of eight elements which are one another's partners in the rotation, so that it
// takes no exchange between lanes, and 2, 4, 8 or 16 lanes hold a head.
#include <algorithm>

#include "kernels.h"

namespace spes {
namespace {

constexpr int kMaxBlocks = 1024;         // of the backward: one partial sum each

struct Side {                            // queries or keys
  const void *dy, *x, *weight;           // dy: backward only
  void* out;
  float *part, *d_weight;
  long row;                              // of x, in the backward of out as well
  int heads, blocks;
};
struct QkArgs {
  Side side[2];
  const float* table;
  const int* pos;
  int T, dim, rot, interleaved, n_pos, accumulate;
  float eps;
};

template <int LG>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (LG >= 8) return lane_group_sum<LG>(v);
  v += dpp_move<0xB1>(v);                // quad_perm [1,0,3,2]
  if constexpr (LG == 4) v += dpp_move<0x4E>(v);      // quad_perm [2,3,0,1]
  return v;
}

// Which elements lane p of a head holds
struct Place {
  int a, b;                              // first elements of its chunks
  bool has_a, has_b, turned;
  int pair;                              // first of its eight pairs
};
__device__ __forceinline__ Place place(const QkArgs& g, int p) {
  const int turned = g.rot / 16;
  if (p < turned) return g.interleaved ? Place{16 * p, 16 * p + 8, true, true, true, 8 * p} : Place{8 * p, 8 * p + g.rot / 2, true, true, true, 8 * p};
  const int at = g.rot + 16 * (p - turned);
  return Place{at, at + 8, at < g.dim, at + 8 < g.dim, false, 0};
}

template <typename T> __device__ __forceinline__ void get8(float* v, const T* p, bool there);
template <> __device__ __forceinline__ void get8<bf16_t>(float* v, const bf16_t* p, bool there) {
  Vec16<bf16_t> u;
  u.raw = make_uint4(0, 0, 0, 0);
  if (there) u.load(p);
  u.unpack(v);
}
template <> __device__ __forceinline__ void get8<float>(float* v, const float* p, bool there) {
  Vec16<float> u, w;
  u.raw = w.raw = make_float4(0.f, 0.f, 0.f, 0.f);
  if (there) {
    u.load(p);
    w.load(p + 4);
  }
  u.unpack(v);
  w.unpack(v + 4);
}
__device__ __forceinline__ void put8(bf16_t* p, const float* v) {
  Vec16<bf16_t> u;
  u.pack(v);
  u.store(p);
}
__device__ __forceinline__ void put8(float* p, const float* v) {
  Vec16<float> u, w;
  u.pack(v);
  w.pack(v + 4);
  u.store(p);
  w.store(p + 4);
}

// Cosines and sines of a lane's pairs; a position that the table does not have gives NaN
__device__ __forceinline__ void angles(const QkArgs& g, const Place& at, int token, float* c, float* s) {
  if (!at.turned) return;
  const int pos = g.pos ? g.pos[token] : token;
  if ((unsigned)pos >= (unsigned)g.n_pos) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s[i] = NAN;
    return;
  }
  const float* const row = g.table + (long)pos * g.rot + at.pair;
  get8<float>(c, row, true);
  // (rot / 2 is a multiple of eight)
  get8<float>(s, row + g.rot / 2, true);
}

// v: sixteen elements, pairs as (v[i], v[8 + i]), or of neighbours
__device__ __forceinline__ void turn(float* v, const float* c, const float* s, bool neighbours, float sign) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = neighbours ? v[2 * i] : v[i], b = neighbours ? v[2 * i + 1] : v[8 + i];
    const float x = a * c[i] - b * (sign * s[i]), y = a * (sign * s[i]) + b * c[i];
    if (neighbours) {
      v[2 * i] = x;
      v[2 * i + 1] = y;
    } else {
      v[i] = x;
      v[8 + i] = y;
    }
  }
}

template <typename T, int LG, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_rope_fwd_kernel(const QkArgs g) {
  const bool keys = (int)blockIdx.x >= g.side[0].blocks;
  const Side d = keys ? g.side[1] : g.side[0];
  const Place at = place(g, threadIdx.x % LG);
  float w[16];
  if (d.weight) {
    get8<T>(w, static_cast<const T*>(d.weight) + at.a, at.has_a);
    get8<T>(w + 8, static_cast<const T*>(d.weight) + at.b, at.has_b);
  }
  const long n = (long)g.T * d.heads;
  for (long u = (long)(blockIdx.x - (keys ? g.side[0].blocks : 0)) * (256 / LG) + threadIdx.x / LG; u < n; u += (long)d.blocks * (256 / LG)) {
    const int token = (int)((unsigned)u / (unsigned)d.heads), head = (int)((unsigned)u - (unsigned)token * (unsigned)d.heads);
    const T* const x = static_cast<const T*>(d.x) + token * d.row + (long)head * g.dim;
    float v[16], c[8], s[8];
    get8<T>(v, x + at.a, at.has_a);
    get8<T>(v + 8, x + at.b, at.has_b);
    angles(g, at, token, c, s);
    if (d.weight) {
      float q = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) q = fmaf(v[i], v[i], q);
      const float rstd = 1.f / sqrtf(group_sum<LG>(q) / (float)g.dim + g.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = v[i] * rstd * w[i];
    }
    if (at.turned) turn(v, c, s, NEIGHBOURS, 1.f);
    T* const y = static_cast<T*>(d.out) + u * g.dim;
    if (at.has_a) put8(y + at.a, v);
    if (at.has_b) put8(y + at.b, v + 8);
  }
}

template <typename T, int LG, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_rope_bwd_kernel(const QkArgs g) {
  __shared__ float red[4][16 * LG];
  const bool keys = (int)blockIdx.x >= g.side[0].blocks;
  const Side d = keys ? g.side[1] : g.side[0];
  const int p = threadIdx.x % LG, block = (int)blockIdx.x - (keys ? g.side[0].blocks : 0);
  const Place at = place(g, p);
  float w[16], dw[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[i] = 0.f;
  if (d.weight) {
    get8<T>(w, static_cast<const T*>(d.weight) + at.a, at.has_a);
    get8<T>(w + 8, static_cast<const T*>(d.weight) + at.b, at.has_b);
  }
  const long n = (long)g.T * d.heads;
  for (long u = (long)block * (256 / LG) + threadIdx.x / LG; u < n; u += (long)d.blocks * (256 / LG)) {
    const int token = (int)((unsigned)u / (unsigned)d.heads), head = (int)((unsigned)u - (unsigned)token * (unsigned)d.heads);
    const long to = token * d.row + (long)head * g.dim;
    const T* const dy = static_cast<const T*>(d.dy) + u * g.dim;
    float v[16], h[16], c[8], s[8];
    get8<T>(h, dy + at.a, at.has_a);
    get8<T>(h + 8, dy + at.b, at.has_b);
    if (d.weight) {
      const T* const x = static_cast<const T*>(d.x) + to;
      get8<T>(v, x + at.a, at.has_a);
      get8<T>(v + 8, x + at.b, at.has_b);
    }
    angles(g, at, token, c, s);
    if (at.turned) turn(h, c, s, NEIGHBOURS, -1.f);
    if (d.weight) {
      float q = 0.f, t = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) q = fmaf(v[i], v[i], q);
      const float rstd = 1.f / sqrtf(group_sum<LG>(q) / (float)g.dim + g.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[i] *= rstd;
        dw[i] = fmaf(h[i], v[i], dw[i]);
        h[i] *= w[i];
        t = fmaf(h[i], v[i], t);
      }
      t = group_sum<LG>(t) / (float)g.dim;
#pragma unroll
      for (int i = 0; i < 16; ++i) h[i] = rstd * (h[i] - v[i] * t);
    }
    T* const dx = static_cast<T*>(d.out) + to;
    if (at.has_a) put8(dx + at.a, h);
    if (at.has_b) put8(dx + at.b, h + 8);
  }
  if (!d.d_weight) return;
  // over the wavefront's heads, then over the block's four wavefronts
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int o = LG; o < kWave; o <<= 1) dw[i] += __shfl_xor(dw[i], o, kWave);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane < LG)
#pragma unroll
    for (int i = 0; i < 16; ++i) red[wave][16 * p + i] = dw[i];
  __syncthreads();
  if ((int)threadIdx.x < 16 * LG) {
    const int i = threadIdx.x % 16;
    const Place to = place(g, threadIdx.x / 16);
    const float sum = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
    if (i < 8 ? to.has_a : to.has_b) d.part[(long)block * g.dim + (i < 8 ? to.a + i : to.b + i - 8)] = sum;
  }
}

// The weights' gradients from the blocks' partial sums: 32 lanes to a column, in a fixed order
__global__ __launch_bounds__(256) void qk_rope_columns_kernel(const QkArgs g) {
  __shared__ float red[32][9];
  const Side d = blockIdx.y ? g.side[1] : g.side[0];
  if (!d.d_weight) return;
  const int col = blockIdx.x * 8 + threadIdx.x % 8, r = threadIdx.x / 8;
  float sum = 0.f;
#pragma unroll 8
  for (int b = r; b < d.blocks; b += 32) sum += d.part[(long)b * g.dim + col];
  red[r][threadIdx.x % 8] = sum;
  __syncthreads();
  if (threadIdx.x < 8) {
    float all = 0.f;
    for (int i = 0; i < 32; ++i) all += red[i][threadIdx.x];
    d.d_weight[col] = g.accumulate ? d.d_weight[col] + all : all;
  }
}

int lanes_of(int dim, int rot) {
  const int pairs = rot / 16 + ((dim - rot) / 8 + 1) / 2;
  return pairs <= 2 ? 2 : pairs <= 4 ? 4 : pairs <= 8 ? 8 : 16;
}

// blocks of a side: its share of `limit`, at most one for every block's worth of heads
int side_blocks(const QkShape& a, int heads, int limit) {
  const long need = cdiv((long)a.T * heads, 256 / lanes_of(a.dim, a.rot));
  return (int)std::max<long>(1, std::min<long>(need, (long)limit * heads / (a.heads + a.kv_heads)));
}

template <typename T, int LG>
int run(const QkArgs& g, bool backward, hipStream_t s) {
  const dim3 grid((unsigned)(g.side[0].blocks + g.side[1].blocks)), block(256);
  if (backward) {
    if (g.interleaved) qk_rope_bwd_kernel<T, LG, true><<<grid, block, 0, s>>>(g);
    else qk_rope_bwd_kernel<T, LG, false><<<grid, block, 0, s>>>(g);
    if (g.side[0].d_weight) qk_rope_columns_kernel<<<dim3(g.dim / 8, 2), block, 0, s>>>(g);
  } else {
    if (g.interleaved) qk_rope_fwd_kernel<T, LG, true><<<grid, block, 0, s>>>(g);
    else qk_rope_fwd_kernel<T, LG, false><<<grid, block, 0, s>>>(g);
  }
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}
template <typename T>
int run(const QkArgs& g, bool backward, hipStream_t s) {
  switch (lanes_of(g.dim, g.rot)) {
    case 2: return run<T, 2>(g, backward, s);
    case 4: return run<T, 4>(g, backward, s);
    case 8: return run<T, 8>(g, backward, s);
    default: return run<T, 16>(g, backward, s);
  }
}
int run(int dtype, const QkArgs& g, bool backward, hipStream_t s) { return dtype == SPES_BF16 ? run<bf16_t>(g, backward, s) : run<float>(g, backward, s); }

}  // namespace

int launch_qk_rope_fwd(int dtype, const QkShape& a, const void* q, const void* k, const void* q_weight, const void* k_weight, const float* table,
                       const int* pos, void* q_out, void* k_out, hipStream_t s) {
  constexpr int kLimit = 4096;
  QkArgs g = {{{nullptr, q, q_weight, q_out, nullptr, nullptr, a.q_row, a.heads, side_blocks(a, a.heads, kLimit)},
               {nullptr, k, k_weight, k_out, nullptr, nullptr, a.k_row, a.kv_heads, side_blocks(a, a.kv_heads, kLimit)}},
              table, pos, a.T, a.dim, a.rot, a.interleaved, a.n_pos, 0, a.eps};
  return run(dtype, g, false, s);
}

size_t qk_rope_scratch_bytes(const QkShape& a) {
  return (size_t)(side_blocks(a, a.heads, kMaxBlocks) + side_blocks(a, a.kv_heads, kMaxBlocks)) * a.dim * sizeof(float);
}

int launch_qk_rope_bwd(int dtype, const QkShape& a, const void* dq, const void* dk, const void* q, const void* k, const void* q_weight,
                       const void* k_weight, const float* table, const int* pos, void* dq_in, void* dk_in, float* d_q_weight, float* d_k_weight,
                       int accumulate, float* scratch, hipStream_t s) {
  const int nq = side_blocks(a, a.heads, kMaxBlocks), nk = side_blocks(a, a.kv_heads, kMaxBlocks);
  QkArgs g = {{{dq, q, q_weight, dq_in, scratch, d_q_weight, a.q_row, a.heads, nq},
               {dk, k, k_weight, dk_in, scratch + (d_q_weight ? (long)nq * a.dim : 0), d_k_weight, a.k_row, a.kv_heads, nk}},
              table, pos, a.T, a.dim, a.rot, a.interleaved, a.n_pos, accumulate, a.eps};
  return run(dtype, g, true, s);
}

}  // namespace spes
