// Routing to experts from given scores, and its gradient.  Per token with logits l
//      s = softmax(l) or sigmoid(l)            c = s + bias                    (the bias steers the choice and nothing else)
//      c = -inf where l masks the expert (-inf or the type's lowest value: no bias brings it back) and where it would be NaN
//      groups: of equal size; a group counts the sum of its two largest c that are not -inf; only the `kept` best groups are open
//      idx = the k largest c in open groups, equal ones to the lower expert    gate = scale s[idx] (/ sum of s[idx], renorm)
// Sixteen lanes hold a token, four consecutive experts to a lane and quad, so a wavefront works on four tokens and every
// reduction stays within a row of lanes, in data-parallel-primitive steps.  What bounds it is the choice, not the 4 M
// bytes of a token: 32768 tokens over 64 experts, top-8, 13.6 us for 10 MB, vector instructions in 72 % of the CUs' cycles; 16384 over 256 in 8 groups of which
// 4 are open, 18.5 us for 18 MB, 59 % (each with 1.2 to 2.3 us for the launch that clears the counts); 48 over 64 4.2 us.  Wavefronts wait half of their time: for the
// bias, which is asked for quad by quad, for the row and for the chosen logits, which are read again; two or four of them to a SIMD cover only part of it.
//
// Gradient, the choice held fixed, with g the gates' share (scale taken out) and u = scale dgate.  Every difference is between gradients, weighted by
// shares, so nothing cancels when one expert takes all:
//      renorm:   D_j = sum_i g_i (u_j - u_i);  softmax: dl_j = g_j D_j (the other scores do not matter);  sigmoid: dl_j = g_j (1 - s_j) D_j
//      otherwise sigmoid: dl_j = u_j s_j (1 - s_j);   softmax: dl_j = s_j (sum_i s_i (u_j - u_i) + u_j sum of the s not chosen),
//                and dl_e = -s_e sum_i s_i u_i for an expert that is not chosen
#include <cfloat>
#include <type_traits>

#include "kernels.h"
#include "lds_load.h"
#include "units.h"

namespace spes {
namespace {

constexpr int kRow = 16;                       // lanes of a token
// Every block adds its counts to all experts' at its end, and what is added to one address waits in line.  16384 tokens over 256 experts in blocks of
// 256 threads: 1024 of them 33 us, 512 26; in blocks of 512: 256 of them 23, 128 29.
constexpr int kBlocks = 256;
constexpr int kSkew = 20;                      // floats: one more for every group ahead, so that groups of 32 start in different banks

template <int CTRL> __device__ __forceinline__ int dpp_int(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ unsigned row_max(unsigned v) {
  v = max(v, (unsigned)dpp_int<0x128>((int)v));       // row_ror 8, 4, 2, 1
  v = max(v, (unsigned)dpp_int<0x124>((int)v));
  v = max(v, (unsigned)dpp_int<0x122>((int)v));
  return max(v, (unsigned)dpp_int<0x121>((int)v));
}
__device__ __forceinline__ int row_min(int v) {
  v = min(v, dpp_int<0x128>(v));
  v = min(v, dpp_int<0x124>(v));
  v = min(v, dpp_int<0x122>(v));
  return min(v, dpp_int<0x121>(v));
}
__device__ __forceinline__ float row_max_f(float v) {
  v = fmaxf(v, dpp_move<0x128>(v));
  v = fmaxf(v, dpp_move<0x124>(v));
  v = fmaxf(v, dpp_move<0x122>(v));
  return fmaxf(v, dpp_move<0x121>(v));
}
__device__ __forceinline__ float row_sum(float v) { return lane_group_sum<16>(v); }

// A choice is a double: the score's value, which leaves the low 29 bits of the mantissa free, and in these the expert, such that equal scores are in
// the order of the experts.  Then one comparison decides, and a sorting step is v_max_f64 and v_min_f64, two full-rate instructions instead of the
// five of a pair (a compare and four selects).  -inf becomes the lowest finite value, +inf the highest.
constexpr double kAbove = 0x1p130, kBelow = -0x1p130, kClosed = -0x1p140;      // beyond all floats
constexpr int kExpertBits = 511;
__device__ __forceinline__ double with_low(double v, unsigned low) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  return __builtin_bit_cast(double, make_uint2(w.x | low, w.y));
}
__device__ __forceinline__ double choice_of(float c, unsigned e) {
  const double v = fmin(fmax((double)c, kBelow), kAbove);
  const unsigned sign = (unsigned)((int)__builtin_bit_cast(uint2, v).y >> 31);          // larger low bits: larger, of a negative number smaller
  return with_low(v, e ^ (kExpertBits & ~sign));
}
__device__ __forceinline__ int expert_of(double v) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  return (int)((w.x & kExpertBits) ^ (kExpertBits & ~(unsigned)((int)w.y >> 31)));
}
// (as instructions: the compiler, which does not know that none of these is a signalling NaN, adds one to quieten each operand that came from another lane)
__device__ __forceinline__ double larger(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double smaller(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ void order(double& a, double& b) {          // the larger one first
  const double hi = larger(a, b);
  b = smaller(a, b);
  a = hi;
}
// descending: a bitonic sequence of N (a power of two), or any sequence
template <int N> __device__ __forceinline__ void sort_bitonic(double* v) {
#pragma unroll
  for (int d = N / 2; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((i & d) == 0) order(v[i], v[i + d]);
}
template <int N> __device__ __forceinline__ void sort(double* v) {
  if constexpr (N > 1) {
    sort<N / 2>(v);
    sort<N / 2>(v + N / 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) order(v[i], v[N - 1 - i]);          // both halves descend: the first half gets the largest, either is bitonic now
    sort_bitonic<N / 2>(v);
    sort_bitonic<N / 2>(v + N / 2);
  }
}
// the K largest of two descending lists, in `a`
template <int K> __device__ __forceinline__ void merge(double* a, const double* b) {
  double hi[K];
#pragma unroll
  for (int i = 0; i < K; ++i) hi[i] = larger(a[i], b[K - 1 - i]);
  sort_bitonic<K>(hi);
#pragma unroll
  for (int i = 0; i < K; ++i) a[i] = hi[i];
}
template <int CTRL> __device__ __forceinline__ double dpp_double(double v) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  return __builtin_bit_cast(double, make_uint2((unsigned)dpp_int<CTRL>((int)w.x), (unsigned)dpp_int<CTRL>((int)w.y)));
}
// The K largest of a row of lanes, from L descending values in each: lists of neighbours, of pairs, of halves are merged, and grow until they
// have K.  Every lane ends with the whole list.
template <int K, int L, int CTRL> __device__ __forceinline__ void merge_lanes(double* v) {
  double o[K];
#pragma unroll
  for (int i = 0; i < L; ++i) o[i] = dpp_double<CTRL>(v[i]);
  if constexpr (L < K) {
#pragma unroll
    for (int i = 0; i < L; ++i) {          // the L largest, and the rest, either bitonic
      v[L + i] = smaller(v[i], o[L - 1 - i]);
      v[i] = larger(v[i], o[L - 1 - i]);
    }
    sort_bitonic<L>(v);
    sort_bitonic<L>(v + L);
  } else {
    merge<K>(v, o);
  }
}
template <int K, int L> __device__ __forceinline__ void merge_row(double* v) {
  constexpr int L1 = L < K ? 2 * L : K, L2 = L1 < K ? 2 * L1 : K, L3 = L2 < K ? 2 * L2 : K;
  merge_lanes<K, L, 0xB1>(v);         // quad_perm [1,0,3,2]
  merge_lanes<K, L1, 0x4E>(v);        // quad_perm [2,3,0,1]
  merge_lanes<K, L2, 0x141>(v);       // row_half_mirror
  merge_lanes<K, L3, 0x140>(v);       // row_mirror
}

// group scores (no NaN among them), in the order of their values: unsigned keys, 0 below all
__device__ __forceinline__ unsigned order_key(float f) {
  const unsigned u = __float_as_uint(f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

// a logit that keeps its expert from the token
__device__ __forceinline__ bool masks(float l) { return l <= -FLT_MAX; }

// 1 / d, within a step, of 1 <= d <= 2: the hardware's and one Newton step, where a division takes three times as many instructions
__device__ __forceinline__ float inverse(float d) {
  const float r = __builtin_amdgcn_rcpf(d);
  return fmaf(fmaf(-d, r, 1.f), r, r);
}
// The choice is made from the same bits as the gates: with the hardware's exponential and reciprocal for every expert and these for the chosen ones, scores a
// few steps apart came out in another order than their gates.
__device__ __forceinline__ float sigmoid(float l) {
  const float small = expf(-fabsf(l)), big = inverse(1.f + small);
  return l < 0.f ? small * big : big;
}

struct RouterArgs {
  int T, M, k, groups, kept, size, parts;      // parts: lanes that look through a group, a power of two; groups * parts <= 16
  unsigned inv_size;                           // e / size = e inv_size >> 20 for e < 512
  bool renorm;
  float scale;
  const float *logits, *bias;
  int* idx;
  float* gate;
  int* count;
  bool one_block;                              // count is written, not added to
  const float* dgate;
  float* dlogits;
};

// four logits from expert e on, -inf beyond the last one
__device__ __forceinline__ void load4(const float* row, int e, int M, float* v) {
  if (e + 4 <= M) {
    const f32x4_any q = *reinterpret_cast<const f32x4_any*>(row + e);
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = q[c];
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = e + c < M ? row[e + c] : -INFINITY;
  }
}

// softmax of one token: the largest logit, the inverse of the sum, and exponentials in place of the logits, MARK: -inf of masked ones.  A row of -inf alone
// has no largest one: its scores are 0.
template <int NQ, bool MARK>
__device__ __forceinline__ void softmax_terms(float (&v)[NQ * 4], float& mx, float& inv) {
  mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < NQ * 4; ++i) mx = fmaxf(mx, v[i]);
  mx = row_max_f(mx);
  if (mx == -INFINITY) mx = 0.f;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NQ * 4; ++i) {
    const float e = expf(v[i] - mx);
    sum += e;
    v[i] = MARK && masks(v[i]) ? -INFINITY : e;
  }
  sum = row_sum(sum);
  inv = sum == 0.f ? 0.f : 1.f / sum;
}

// Score of a token's chosen expert, one to a lane, and what it lacks to 1 (of softmax: 1), for the gates and for their gradient.  RENORM: up to a factor that
// all of them have, so that shares keep their bits where the scores underflow: a softmax over the chosen ones alone; sigmoids times e to the
// power of -top, top the largest logit between 0 and -100.  What is 0 here has neither gate nor gradient.
struct Score { float s, other; };
template <bool SOFTMAX, bool RENORM>
__device__ __forceinline__ Score chosen_score(float x, bool has) {
  const float largest = RENORM ? row_max_f(has ? x : -INFINITY) : 0.f;
  if (SOFTMAX) return {has ? expf(x - (largest == -INFINITY ? 0.f : largest)) : 0.f, 1.f};
  const float small = expf(-fabsf(x)), big = inverse(1.f + small), top = fmaxf(fminf(largest, 0.f), -100.f);
  return {!has ? 0.f : x < 0.f ? (RENORM ? expf(x - top) : small) * big : big, x < 0.f ? big : small * big};
}

// K: a power of two, k at least
template <int NQ, int K, bool SOFTMAX, bool GROUPS, int BLOCK>
__global__ __launch_bounds__(BLOCK) void router_fwd_kernel(const RouterArgs a) {
  constexpr int V = NQ * 4, TOKENS = BLOCK / kRow;
  __shared__ int hist[NQ * 64];
  __shared__ float choice[GROUPS ? TOKENS : 1][NQ * 64 + kSkew];
  const int l = threadIdx.x % kRow, at = threadIdx.x / kRow;
  for (int e = threadIdx.x; e < NQ * 64; e += BLOCK) hist[e] = 0;
  __syncthreads();
  float bias[V];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    if (a.bias) load4(a.bias, q * 64 + l * 4, a.M, bias + q * 4);
    else bias[q * 4] = bias[q * 4 + 1] = bias[q * 4 + 2] = bias[q * 4 + 3] = 0.f;
  }
  for (long t0 = (long)blockIdx.x * TOKENS; t0 < a.T; t0 += (long)gridDim.x * TOKENS) {
    const long t = t0 + at < a.T ? t0 + at : a.T - 1;          // (surplus rows of lanes repeat the last token and store nothing)
    const bool live = t0 + at < a.T;
    const float* const row = a.logits + t * a.M;
    float v[V];
#pragma unroll
    for (int q = 0; q < NQ; ++q) load4(row, q * 64 + l * 4, a.M, v + q * 4);
    float mx = 0.f, inv = 1.f;
    if constexpr (SOFTMAX) softmax_terms<NQ, true>(v, mx, inv);
    double best[V > K ? V : K];
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e = q * 64 + l * 4 + c, i = q * 4 + c;
        float x = (SOFTMAX ? v[i] * inv : sigmoid(v[i])) + bias[i];
        x = masks(v[i]) || x != x ? -INFINITY : x;           // (of a minimum with a NaN the other one is left: a NaN would stand for it in the scan below)
        const double mine = choice_of(x, (unsigned)e);
        best[i] = e < a.M ? mine : kClosed;
        if (GROUPS) choice[at][e < a.M ? e + (int)((unsigned)e * a.inv_size >> 20) : NQ * 64 + kSkew - 1] = x;          // (the last one is nobody's)
      }
    if (GROUPS) {
      // lanes g parts .. look through group g; the first of them ranks it among the others
      wave_lds_order();
      const int g = l / a.parts, part = l % a.parts;
      float first = -INFINITY, second = -INFINITY;
      if (g < a.groups) {
        const float* const own = choice[at] + g * (a.size + 1);
        for (int n = part; n < a.size; n += a.parts) {
          const float x = own[n];
          second = fmaxf(second, fminf(first, x));
          first = fmaxf(first, x);
        }
      }
      for (int d = 1; d < a.parts; d *= 2) {
        const float f2 = __shfl_xor(first, d, kWave), s2 = __shfl_xor(second, d, kWave);
        second = fmaxf(fmaxf(second, s2), fminf(first, f2));
        first = fmaxf(first, f2);
      }
      wave_lds_order();
      const unsigned mine = part == 0 && g < a.groups ? order_key(second == -INFINITY ? first : first + second) : 0u;
      int rank = 0;
      auto against = [&](unsigned other, int lane) { rank += other > mine || (other == mine && lane < l) ? 1 : 0; };
#define SPES_TURN(r) against((unsigned)dpp_int<0x120 + r>((int)mine), dpp_int<0x120 + r>(l))
      SPES_TURN(1); SPES_TURN(2); SPES_TURN(3); SPES_TURN(4); SPES_TURN(5); SPES_TURN(6); SPES_TURN(7); SPES_TURN(8);
      SPES_TURN(9); SPES_TURN(10); SPES_TURN(11); SPES_TURN(12); SPES_TURN(13); SPES_TURN(14); SPES_TURN(15);
#undef SPES_TURN
      const unsigned open = (unsigned)(__ballot(mine != 0 && rank < a.kept) >> (threadIdx.x & 48)) & 0xffffu;
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const unsigned e = (unsigned)(q * 64 + l * 4 + c);
          if ((open >> ((e * a.inv_size >> 20) * a.parts) & 1u) == 0) best[q * 4 + c] = kClosed;
        }
    }
    // the K largest of the lane, then of the token
    constexpr int L = V < K ? V : K;
    sort<L>(best);
#pragma unroll
    for (int i = L; i < V; i += L) {
      sort<L>(best + i);
      merge<L>(best, best + i);
    }
    merge_row<K, L>(best);
    double pick = best[0];              // of lane j: the j-th
#pragma unroll
    for (int j = 1; j < K; ++j) pick = l == j ? best[j] : pick;
    const int chosen = expert_of(pick);
    const bool mine = l < a.k;
    const float x = mine ? row[chosen] : 0.f;
    float share;
    if (a.renorm) {
      const float s = chosen_score<SOFTMAX, true>(x, mine).s, total = row_sum(s);
      share = total == 0.f ? 0.f : s / total;
      if (SOFTMAX && inv != inv) share = inv;               // (a NaN or +inf anywhere in the row)
    } else {
      share = !mine ? 0.f : SOFTMAX ? expf(x - mx) * inv : sigmoid(x);
    }
    if (mine && live) {
      a.idx[t * a.k + l] = chosen;
      a.gate[t * a.k + l] = share * a.scale;
      atomicAdd(&hist[chosen], 1);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.M; e += BLOCK) {
    if (a.one_block) a.count[e] = hist[e];
    else if (hist[e] != 0) atomicAdd(&a.count[e], hist[e]);      // (integers: any order gives the same)
  }
}

__global__ __launch_bounds__(512) void zero_kernel(int* __restrict__ p, int n) {
  if (threadIdx.x < n) p[threadIdx.x] = 0;
}

// sum over the chosen i of w_i (u - u_i), in every lane for its own u
__device__ __forceinline__ float weighted_differences(float w, float u) {
  float d = 0.f;
#define SPES_TURN(r) d = fmaf(dpp_move<0x120 + r>(w), u - dpp_move<0x120 + r>(u), d)
  SPES_TURN(1); SPES_TURN(2); SPES_TURN(3); SPES_TURN(4); SPES_TURN(5); SPES_TURN(6); SPES_TURN(7); SPES_TURN(8);
  SPES_TURN(9); SPES_TURN(10); SPES_TURN(11); SPES_TURN(12); SPES_TURN(13); SPES_TURN(14); SPES_TURN(15);
#undef SPES_TURN
  return d;
}

// WHOLE: softmax without renormalisation, where every score has a gradient.  Otherwise only the k chosen ones are read, and
// the row of dlogits is put together in LDS and goes out whole: 16384 x 256 5.9 us, 32768 x 64 4.8 (17 and 8 MB written).
template <int NQ, bool SOFTMAX, bool WHOLE>
__global__ __launch_bounds__(256) void router_bwd_kernel(const RouterArgs a) {
  constexpr int V = NQ * 4;
  __shared__ __align__(16) float out[16][NQ * 64];
  const int l = threadIdx.x % kRow, at = threadIdx.x / kRow;
  float* const mine = out[at];
  for (long t0 = (long)blockIdx.x * 16; t0 < a.T; t0 += (long)gridDim.x * 16) {
    const long t = t0 + at < a.T ? t0 + at : a.T - 1;
    const bool live = t0 + at < a.T;
    const float* const row = a.logits + t * a.M;
    int e = -1;
    float u = 0.f, x = 0.f;
    if (l < a.k) {
      e = a.idx[t * a.k + l];
      if (e < 0 || e >= a.M) e = -1;                       // (no expert: no gradient)
      else { u = a.dgate[t * a.k + l] * a.scale; x = row[e]; }
    }
    const bool has = e >= 0;
    float p[WHOLE ? V : 1], mx = 0.f, inv = 1.f;
    if (WHOLE) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) load4(row, q * 64 + l * 4, a.M, p + q * 4);
      if constexpr (WHOLE) softmax_terms<NQ, false>(p, mx, inv);
#pragma unroll
      for (int i = 0; i < (WHOLE ? V : 1); ++i) p[i] *= inv;
    }
    // marks of the chosen ones, then results
    wave_lds_order();
#pragma unroll
    for (int q = 0; q < NQ; ++q) *reinterpret_cast<float4*>(mine + q * 64 + l * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
    wave_lds_order();
    float d;
    if (WHOLE) {
      if (has) mine[e] = 1.f;
      wave_lds_order();
      float rest = 0.f;
#pragma unroll
      for (int i = 0; i < (WHOLE ? V : 1); ++i) rest += mine[(i / 4) * 64 + l * 4 + i % 4] == 0.f ? p[i] : 0.f;
      rest = row_sum(rest);
      wave_lds_order();
      const float s = has ? expf(x - mx) * inv : 0.f;
      d = s * (weighted_differences(s, u) + u * rest);
      const float dot = row_sum(s * u);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        float* const o = mine + q * 64 + l * 4;
        const float* const pq = p + (WHOLE ? q * 4 : 0);
        *reinterpret_cast<float4*>(o) = make_float4(-pq[0] * dot, -pq[WHOLE ? 1 : 0] * dot, -pq[WHOLE ? 2 : 0] * dot, -pq[WHOLE ? 3 : 0] * dot);
      }
      wave_lds_order();
    } else {
      if (SOFTMAX || a.renorm) {
        const Score c = chosen_score<SOFTMAX, true>(x, has);
        const float total = row_sum(c.s), g = total == 0.f ? 0.f : c.s / total;
        d = g * c.other * weighted_differences(g, u);
      } else {
        const Score c = chosen_score<false, false>(x, has);
        d = c.s * c.other * u;
      }
    }
    if (has) mine[e] = d;
    wave_lds_order();
    if (live) {
      float* const dst = a.dlogits + t * a.M;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int e0 = q * 64 + l * 4;
        const float4 o = *reinterpret_cast<const float4*>(mine + e0);
        if (e0 + 4 <= a.M) {
          *reinterpret_cast<f32x4_any*>(dst + e0) = f32x4_any{o.x, o.y, o.z, o.w};
        } else {
          if (e0 < a.M) dst[e0] = o.x;
          if (e0 + 1 < a.M) dst[e0 + 1] = o.y;
          if (e0 + 2 < a.M) dst[e0 + 2] = o.z;
        }
      }
    }
  }
}

RouterArgs router_args(int T, int M, int k, const spes_router_opts& o) {
  RouterArgs a = {};
  a.T = T; a.M = M; a.k = k; a.groups = o.groups; a.kept = o.kept_groups; a.size = M / o.groups;
  a.parts = 1;
  while (a.parts * 2 * a.groups <= kRow) a.parts *= 2;
  a.inv_size = ((1u << 20) + (unsigned)a.size - 1) / (unsigned)a.size;
  a.renorm = o.renorm != 0;
  a.scale = o.scale;
  return a;
}

template <typename F>
int with_quads(int M, F launch) {
  if (M <= 64) return launch(std::integral_constant<int, 1>{});
  if (M <= 128) return launch(std::integral_constant<int, 2>{});
  if (M <= 256) return launch(std::integral_constant<int, 4>{});
  return launch(std::integral_constant<int, 8>{});
}

}  // namespace

int launch_router_fwd(int T, int M, int k, const spes_router_opts& o, const float* logits, const float* bias, int* idx, float* gate, int* count,
                      hipStream_t s) {
  RouterArgs a = router_args(T, M, k, o);
  a.logits = logits; a.bias = bias; a.idx = idx; a.gate = gate; a.count = count;
  // A single block counts by itself; several need a launch ahead of theirs that clears the counts.
  a.one_block = T <= 128;
  if (!a.one_block) hipLaunchKernelGGL(zero_kernel, dim3(1), dim3(512), 0, s, count, M);
  const bool groups = o.groups > 1;
  return with_quads(M, [&](auto nq) {
    constexpr int NQ = decltype(nq)::value;
    auto go = [&](auto choice, auto softmax, auto grouped) {
      constexpr bool SM = decltype(softmax)::value, GR = decltype(grouped)::value;
      constexpr int K = decltype(choice)::value;
      constexpr int ONE = NQ <= 2 ? 1024 : 512;          // (of more experts, a block of 1024 would spill registers)
      const int need = cdiv(T, ONE / kRow);
      hipLaunchKernelGGL((router_fwd_kernel<NQ, K, SM, GR, ONE>), dim3(a.one_block ? 1 : need < kBlocks ? need : kBlocks), dim3(ONE), 0, s, a);
      return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
    };
    auto kind = [&](auto choice) {
      if (o.score == SPES_SCORE_SOFTMAX) return groups ? go(choice, std::true_type{}, std::true_type{}) : go(choice, std::true_type{}, std::false_type{});
      return groups ? go(choice, std::false_type{}, std::true_type{}) : go(choice, std::false_type{}, std::false_type{});
    };
    if (k <= 2) return kind(std::integral_constant<int, 2>{});
    if (k <= 4) return kind(std::integral_constant<int, 4>{});
    if (k <= 8) return kind(std::integral_constant<int, 8>{});
    return kind(std::integral_constant<int, 16>{});
  });
}

int launch_router_bwd(int T, int M, int k, const spes_router_opts& o, const float* logits, const int* idx, const float* dgate, float* dlogits,
                      hipStream_t s) {
  RouterArgs a = router_args(T, M, k, o);
  a.logits = logits; a.idx = const_cast<int*>(idx); a.dgate = dgate; a.dlogits = dlogits;
  const int grid = cdiv(T, 16) < 4096 ? cdiv(T, 16) : 4096;
  return with_quads(M, [&](auto nq) {
    constexpr int NQ = decltype(nq)::value;
    if (o.score == SPES_SCORE_SIGMOID) hipLaunchKernelGGL((router_bwd_kernel<NQ, false, false>), dim3(grid), dim3(256), 0, s, a);
    else if (o.renorm) hipLaunchKernelGGL((router_bwd_kernel<NQ, true, false>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((router_bwd_kernel<NQ, true, true>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
  });
}

}  // namespace spes
