// Queries and keys ahead of attention: the root-mean-square norm of every head and the rotation by the token's position, in one pass.  Per head x of D elements
//      rstd = (sum x^2 / D + eps)^-1/2      hat = x rstd      y = hat w        pairs (a, b) of the first `rot` elements of y -> (a c - b s, a s + b c)
// and for the gradient dz, with every pair turned back into dy,
//      dw = sum over tokens and heads of dy hat      h = dy w      dx = rstd (h - hat (sum h hat / D))
// Sums are fp32, a result is rounded once.  A lane holds two chunks of eight elements which are one another's partners in the rotation, so that it
// takes no exchange between lanes, and 2, 4, 8 or 16 lanes hold a head.
#include <algorithm>

#include "kernels.h"
#include "plan.h"

namespace spes {
namespace {

constexpr int kMaxBlocks = 1024;         // of the backward: partial sums of queries or keys, one each

struct Side {                            // queries or keys
  const void *dy, *x, *weight;           // dy: backward only
  void* out;
  float *part, *d_weight;
  long row;                              // of x, in the backward of out as well
  int heads, blocks;                     // blocks: that have partial sums of this side
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

// Sum over the wavefront's heads, the lanes LG apart, in all of them
template <int LG>
__device__ __forceinline__ float heads_sum(float v) {
  if (LG <= 2) v += dpp_move<0x122>(v);        // row_ror:2
  if (LG <= 4) v += dpp_move<0x124>(v);        // row_ror:4
  if (LG <= 8) v += dpp_move<0x128>(v);        // row_ror:8
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(h[0]) + __uint_as_float(h[1]);
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

// Eight elements as they are loaded; ONCE: with the non-temporal hint
template <typename T, bool ONCE> struct Eight {
  static constexpr int N = 8 / Vec16<T>::N;
  Vec16<T> u[N];
  __device__ __forceinline__ void load(const T* p, bool there) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u[i].raw = {};
      if (there) {
        if (ONCE) u[i].load_once(p + i * Vec16<T>::N);
        else u[i].load(p + i * Vec16<T>::N);
      }
    }
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int i = 0; i < N; ++i) u[i].unpack(v + i * Vec16<T>::N);
  }
  static __device__ __forceinline__ void put(T* p, const float* v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      Vec16<T> w;
      w.pack(v + i * Vec16<T>::N);
      if (ONCE) w.store_once(p + i * Vec16<T>::N);
      else w.store(p + i * Vec16<T>::N);
    }
  }
};
template <typename T>
__device__ __forceinline__ void get8(float* v, const T* p, bool there) {
  Eight<T, false> e;
  e.load(p, there);
  e.get(v);
}

// Cosines and sines of a lane's pairs; a position that the table does not have gives NaN
__device__ __forceinline__ void angles(const QkArgs& g, const Place& at, int pos, float* c, float* s) {
  if (!at.turned) return;
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

// Tensors that pass through the caches (and so carry the non-temporal hint): a wavefront goes over a token's heads, 64 / LG at a time, U such rounds at
// once, with the angles in registers: queries' rounds first, then keys'.  32768 tokens, 32 + 8 heads of 128 in bf16: 116 to 119 us (5.7 TB/s) and
// 183 to 200 (5.0 to 5.5), memory; the whole step 304 us, with a head to LG lanes as below 341.
template <typename T, int LG, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_rope_fwd_kernel(const QkArgs g) {
  constexpr int NG = kWave / LG, U = sizeof(T) == 2 ? 4 : 2;
  const int lane = threadIdx.x & 63, group = lane / LG;
  const Place at = place(g, lane % LG);
  const bool norm = g.side[0].weight != nullptr;
  float w[2][16];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (norm) {
      get8<T>(w[i], static_cast<const T*>(g.side[i].weight) + at.a, at.has_a);
      get8<T>(w[i] + 8, static_cast<const T*>(g.side[i].weight) + at.b, at.has_b);
    }
  const int q_rounds = cdiv(g.side[0].heads, NG), rounds = q_rounds + cdiv(g.side[1].heads, NG);
  // (a scalar, as is then the position)
  const int first = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  for (int token = first; token < g.T; token += gridDim.x * 4) {
    const int pos = g.pos ? g.pos[token] : token;
    Eight<T, true> in[U][2];
    auto request = [&](int r0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const bool keys = r0 + i >= q_rounds;
        const int head = (r0 + i - (keys ? q_rounds : 0)) * NG + group;
        const bool there = r0 + i < rounds && head < (keys ? g.side[1].heads : g.side[0].heads);
        const T* const x = static_cast<const T*>(keys ? g.side[1].x : g.side[0].x) + (long)token * (keys ? g.side[1].row : g.side[0].row) + (long)head * g.dim;
        in[i][0].load(x + at.a, there && at.has_a);
        in[i][1].load(x + at.b, there && at.has_b);
      }
    };
    float c[8], s[8];
    angles(g, at, pos, c, s);
    for (int r0 = 0; r0 < rounds; r0 += U) {
      request(r0);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (r0 + i >= rounds) break;
        const bool keys = r0 + i >= q_rounds;
        const int head = (r0 + i - (keys ? q_rounds : 0)) * NG + group, heads = keys ? g.side[1].heads : g.side[0].heads;
        float v[16];
        in[i][0].get(v);
        in[i][1].get(v + 8);
        if (norm) {
          float q = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) q = fmaf(v[e], v[e], q);
          const float rstd = 1.f / sqrtf(group_sum<LG>(q) / (float)g.dim + g.eps);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = v[e] * rstd * (keys ? w[1][e] : w[0][e]);
        }
        if (at.turned) turn(v, c, s, NEIGHBOURS, 1.f);
        T* const y = static_cast<T*>(keys ? g.side[1].out : g.side[0].out) + ((long)token * heads + head) * g.dim;
        if (head < heads && at.has_a) Eight<T, true>::put(y + at.a, v);
        if (head < heads && at.has_b) Eight<T, true>::put(y + at.b, v + 8);
      }
    }
  }
}

template <typename T, int LG, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_rope_bwd_kernel(const QkArgs g) {
  constexpr int NG = kWave / LG, U = sizeof(T) == 2 ? 2 : 1;
  __shared__ float red[4][2][16 * LG];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane / LG, p = lane % LG;
  const Place at = place(g, p);
  const bool norm = g.side[0].weight != nullptr;
  float w[2][16], dw[2][16];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = 0.f;
    if (norm) {
      get8<T>(w[i], static_cast<const T*>(g.side[i].weight) + at.a, at.has_a);
      get8<T>(w[i] + 8, static_cast<const T*>(g.side[i].weight) + at.b, at.has_b);
    }
  }
  const int q_rounds = cdiv(g.side[0].heads, NG), rounds = q_rounds + cdiv(g.side[1].heads, NG);
  // (a scalar, as is then the position)
  const int first = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  for (int token = first; token < g.T; token += gridDim.x * 4) {
    const int pos = g.pos ? g.pos[token] : token;
    Eight<T, true> up[U][2], in[U][2];
    auto request = [&](int r0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const bool keys = r0 + i >= q_rounds;
        const int head = (r0 + i - (keys ? q_rounds : 0)) * NG + group, heads = keys ? g.side[1].heads : g.side[0].heads;
        const bool there = r0 + i < rounds && head < heads;
        const T* const dy = static_cast<const T*>(keys ? g.side[1].dy : g.side[0].dy) + ((long)token * heads + head) * g.dim;
        const T* const x = static_cast<const T*>(keys ? g.side[1].x : g.side[0].x) + (long)token * (keys ? g.side[1].row : g.side[0].row) + (long)head * g.dim;
        up[i][0].load(dy + at.a, there && at.has_a);
        up[i][1].load(dy + at.b, there && at.has_b);
        in[i][0].load(x + at.a, norm && there && at.has_a);
        in[i][1].load(x + at.b, norm && there && at.has_b);
      }
    };
    float c[8], s[8];
    angles(g, at, pos, c, s);
    for (int r0 = 0; r0 < rounds; r0 += U) {
      request(r0);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (r0 + i >= rounds) break;
        const bool keys = r0 + i >= q_rounds;
        const int head = (r0 + i - (keys ? q_rounds : 0)) * NG + group, heads = keys ? g.side[1].heads : g.side[0].heads;
        float h[16];
        up[i][0].get(h);
        up[i][1].get(h + 8);
        if (at.turned) turn(h, c, s, NEIGHBOURS, -1.f);
        if (norm) {
          float v[16], q = 0.f, t = 0.f;
          in[i][0].get(v);
          in[i][1].get(v + 8);
#pragma unroll
          for (int e = 0; e < 16; ++e) q = fmaf(v[e], v[e], q);
          const float rstd = 1.f / sqrtf(group_sum<LG>(q) / (float)g.dim + g.eps);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            v[e] *= rstd;
            // (heads that are not there are zeros, but a position that the table lacks turns these into NaN)
            const float more = head < heads ? h[e] * v[e] : 0.f;
            if (keys) dw[1][e] += more;
            else dw[0][e] += more;
            h[e] *= keys ? w[1][e] : w[0][e];
            t = fmaf(h[e], v[e], t);
          }
          t = group_sum<LG>(t) / (float)g.dim;
#pragma unroll
          for (int e = 0; e < 16; ++e) h[e] = rstd * (h[e] - v[e] * t);
        }
        T* const dx = static_cast<T*>(keys ? g.side[1].out : g.side[0].out) + (long)token * (keys ? g.side[1].row : g.side[0].row) + (long)head * g.dim;
        if (head < heads && at.has_a) Eight<T, true>::put(dx + at.a, h);
        if (head < heads && at.has_b) Eight<T, true>::put(dx + at.b, h + 8);
      }
    }
  }
  if (!g.side[0].d_weight) return;
  // over the wavefront's heads, then over the block's four wavefronts
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = heads_sum<LG>(dw[i][e]);
  if (lane < LG)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) red[wave][i][16 * p + e] = dw[i][e];
  __syncthreads();
  for (int n = threadIdx.x; n < 32 * LG; n += 256) {
    const int i = n / (16 * LG), m = n % (16 * LG), e = m % 16;
    const Place to = place(g, m / 16);
    const float sum = (red[0][i][m] + red[1][i][m]) + (red[2][i][m] + red[3][i][m]);
    if (e < 8 ? to.has_a : to.has_b) (i ? g.side[1].part : g.side[0].part)[(long)blockIdx.x * g.dim + (e < 8 ? to.a + e : to.b + e - 8)] = sum;
  }
}

// Tensors that the caches hold: LG lanes to a head, heads one behind the other, blocks of queries and blocks of keys.  Short launches, in which what
// counts is how little a wavefront has to fetch before its first store (4096 tokens, 12 + 12 heads of 64: 7.9 and 11.0 us, 3.2 and 3.4 TB/s out of the Infinity
// Cache; the whole step 21.7 to 24.5 us, with the kernels above 27).
template <typename T, int LG, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_flat_fwd_kernel(const QkArgs g) {
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
    angles(g, at, g.pos ? g.pos[token] : token, c, s);
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
    if (at.has_a) Eight<T, false>::put(y + at.a, v);
    if (at.has_b) Eight<T, false>::put(y + at.b, v + 8);
  }
}

template <typename T, int LG, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_flat_bwd_kernel(const QkArgs g) {
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
    angles(g, at, g.pos ? g.pos[token] : token, c, s);
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
    if (at.has_a) Eight<T, false>::put(dx + at.a, h);
    if (at.has_b) Eight<T, false>::put(dx + at.b, h + 8);
  }
  if (!d.d_weight) return;
  // over the wavefront's heads, then over the block's four wavefronts
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[i] = heads_sum<LG>(dw[i]);
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

// The weights' gradients from the blocks' partial sums: 32 lanes to a column, in a fixed order; 4 to 5 us, two trips to memory
__global__ __launch_bounds__(256) void qk_rope_columns_kernel(const QkArgs g) {
  __shared__ float red[32][9];
  const float* const part = blockIdx.y ? g.side[1].part : g.side[0].part;
  const int blocks = blockIdx.y ? g.side[1].blocks : g.side[0].blocks;
  float* const out = blockIdx.y ? g.side[1].d_weight : g.side[0].d_weight;
  const int col = blockIdx.x * 8 + threadIdx.x % 8, r = threadIdx.x / 8;
  float sum = 0.f;
#pragma unroll 8
  for (int b = r; b < blocks; b += 32) sum += part[(long)b * g.dim + col];
  red[r][threadIdx.x % 8] = sum;
  __syncthreads();
  if (threadIdx.x < 8) {
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) all += red[i][threadIdx.x];
    out[col] = g.accumulate ? out[col] + all : all;
  }
}

int lanes_of(int dim, int rot) {
  const int pairs = rot / 16 + ((dim - rot) / 8 + 1) / 2;
  return pairs <= 2 ? 2 : pairs <= 4 ? 4 : pairs <= 8 ? 8 : 16;
}

// How a call runs: as tensors that pass through the caches, or flat; blocks of queries and of keys (passing: the same blocks have both)
struct Plan { bool once; int blocks[2]; };
Plan plan_of(int dtype, const QkShape& a, int tensors, int limit) {
  if (plan::norm_streams(dtype == SPES_BF16 ? 2 : 4, a.T, (a.heads + a.kv_heads) * a.dim, tensors, a.dim, a.q_row, a.k_row)) {
    const int n = std::max(1, std::min(cdiv(a.T, 4), limit / 2));
    return {true, {n, n}};
  }
  Plan p = {false, {1, 1}};
  const int heads[2] = {a.heads, a.kv_heads};
  for (int i = 0; i < 2; ++i)
    p.blocks[i] = (int)std::max<long>(1, std::min<long>(cdiv((long)a.T * heads[i], 256 / lanes_of(a.dim, a.rot)), (long)limit * heads[i] / (a.heads + a.kv_heads)));
  return p;
}
constexpr int kForward = 2, kBackward = 3, kForwardBlocks = 8192;      // tensors that pass; blocks at most (of the backward: kMaxBlocks)

template <typename T, int LG, bool NEIGHBOURS>
void start(const QkArgs& g, const Plan& p, bool backward, hipStream_t s) {
  const dim3 grid((unsigned)(p.once ? p.blocks[0] : p.blocks[0] + p.blocks[1])), block(256);
  if (p.once) {
    if (backward) qk_rope_bwd_kernel<T, LG, NEIGHBOURS><<<grid, block, 0, s>>>(g);
    else qk_rope_fwd_kernel<T, LG, NEIGHBOURS><<<grid, block, 0, s>>>(g);
  } else {
    if (backward) qk_flat_bwd_kernel<T, LG, NEIGHBOURS><<<grid, block, 0, s>>>(g);
    else qk_flat_fwd_kernel<T, LG, NEIGHBOURS><<<grid, block, 0, s>>>(g);
  }
}
template <typename T, int LG>
void start(const QkArgs& g, const Plan& p, bool backward, hipStream_t s) {
  if (g.interleaved) start<T, LG, true>(g, p, backward, s);
  else start<T, LG, false>(g, p, backward, s);
}
template <typename T>
int run(const QkArgs& g, const Plan& p, bool backward, hipStream_t s) {
  switch (lanes_of(g.dim, g.rot)) {
    case 2: start<T, 2>(g, p, backward, s); break;
    case 4: start<T, 4>(g, p, backward, s); break;
    case 8: start<T, 8>(g, p, backward, s); break;
    default: start<T, 16>(g, p, backward, s);
  }
  if (backward && g.side[0].d_weight) qk_rope_columns_kernel<<<dim3(g.dim / 8, 2), dim3(256), 0, s>>>(g);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

}  // namespace

int launch_qk_rope_fwd(int dtype, const QkShape& a, const void* q, const void* k, const void* q_weight, const void* k_weight, const float* table,
                       const int* pos, void* q_out, void* k_out, hipStream_t s) {
  const Plan p = plan_of(dtype, a, kForward, kForwardBlocks);
  const QkArgs g = {{{nullptr, q, q_weight, q_out, nullptr, nullptr, a.q_row, a.heads, p.blocks[0]},
                     {nullptr, k, k_weight, k_out, nullptr, nullptr, a.k_row, a.kv_heads, p.blocks[1]}},
                    table, pos, a.T, a.dim, a.rot, a.interleaved, a.n_pos, 0, a.eps};
  return dtype == SPES_BF16 ? run<bf16_t>(g, p, false, s) : run<float>(g, p, false, s);
}

size_t qk_rope_scratch_bytes(const QkShape& a) {
  // (either way of running, whatever the strides and the type)
  return (size_t)kMaxBlocks * a.dim * sizeof(float);
}

int launch_qk_rope_bwd(int dtype, const QkShape& a, const void* dq, const void* dk, const void* q, const void* k, const void* q_weight,
                       const void* k_weight, const float* table, const int* pos, void* dq_in, void* dk_in, float* d_q_weight, float* d_k_weight,
                       int accumulate, float* scratch, hipStream_t s) {
  const Plan p = plan_of(dtype, a, kBackward, kMaxBlocks);
  const QkArgs g = {{{dq, q, q_weight, dq_in, scratch, d_q_weight, a.q_row, a.heads, p.blocks[0]},
                     {dk, k, k_weight, dk_in, d_q_weight ? scratch + (long)p.blocks[0] * a.dim : nullptr, d_k_weight, a.k_row, a.kv_heads, p.blocks[1]}},
                    table, pos, a.T, a.dim, a.rot, a.interleaved, a.n_pos, accumulate, a.eps};
  return dtype == SPES_BF16 ? run<bf16_t>(g, p, true, s) : run<float>(g, p, true, s);
}

}  // namespace spes
