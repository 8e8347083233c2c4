// Newton-Schulz orthogonalisation of a stack of matrices, and the optimizer step built on it.
//
// A matrix U is scaled to Frobenius norm 1 and taken through the odd polynomial x -> a x + b x^3 + c x^5 of its singular values, `steps` times.
// With X the scaled matrix, its shorter side lo along the rows (a tall one is turned on the way in and out)
//      G = X X^T      P = b G + c G G      X <- a X + P X
// so a step is three matrix products of lo^2 hi, lo^3 and 2 lo^2 hi operations, of the symmetric ones half the tiles.
//
// The products run on the matrix cores on fp16 operands with fp32 sums.  fp16 because its step, 2^-11, is what the polynomial forgives: it
// grows small singular values 3.4-fold a step, and what rounding adds to them grows alike.  Against 64 bits, on gradients with 16 strong
// directions above a broad floor, 512 x 1024: bf16 operands leave 1.3e-2 of the result's norm, fp16 ones 1.6e-3; nearly all of that is the
// rounding of X itself in the first two steps, in the term a X, so while it matters X is carried with its remainder (a second fp16
// plane, 22 bits together): 1.0e-3.  In the later steps, where singular values are near 1 and P near (b + c) I, what is rounded is P - (b + c) I, and
// the step is X <- (a + b + c) X + (P - (b + c) I) X: 0.8e-3.  fp32 storage takes every operand as such a pair and every product as three,
// lo hi + hi lo + hi hi: 3e-7.  Range: X stands scaled by 2^12, G and P by 2^11, which holds singular values below 5, G below 25
// and P below 31; after the first scaling they are at most 1.21 with the default coefficients.
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "lds_load.h"
#include "units.h"

namespace spes {
namespace {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr int kXcds = 8;
constexpr int kXBits = 12, kGBits = 11;        // X, and G and P, as they are stored, are scaled by these powers of two
constexpr int kPad = 64;                       // stored matrices have sides that are multiples of this, zeros beyond the matrix
constexpr int kSumBlocks = 256;                // partial sums of squares of a matrix, at most
constexpr int kSlots = 64;                     // matrices of an optimizer launch

enum Epi { kGram, kPoly, kStep, kLast, kUpdate };

struct NsArgs {
  const f16 *A, *B, *E;
  f16* C;
  long a_ms, b_ms, e_ms, c_ms;                 // elements from one matrix to the next
  long a_lo, b_lo, e_lo, c_lo;                 // elements from a matrix to its plane of remainders; 0: it has none here
  int lda, ldb, lde, ldc;
  int M, N, K, n;                              // of the products, padded; matrices
  int passes;                                  // 1: hi hi; 3: lo hi, hi lo, hi hi
  float alpha, beta;                           // result = (alpha product + beta E) factor
  float diagonal;                              // kPoly: added to the diagonal
  const float* factor;                         // of each matrix, NULL: 1.  kGram: squared
  // the end: rows x cols as the caller has them
  void *out, *param;
  float* master;
  int rows, cols;
  bool tall;
  float keep, rate;                            // w <- keep w - rate o
  long param_at[kSlots];                       // of each matrix, in elements
};

// x as the sum of two fp16 values; 8 at a time.  (x is pinned as it is in 32 bits: a product that is rounded straight to fp16 for one of
// the two uses and by way of fp32 for the other comes out a step apart where the fp32 value lies half way between two, and the remainder is then
// that of the other one.)
__device__ __forceinline__ void split8(const float* x, uint4& hi, uint4& lo) {
  f16x8 h, r;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = x[e];
    asm("" : "+v"(v));
    h[e] = (f16)v;
    r[e] = (f16)(v - (float)h[e]);
  }
  hi = __builtin_bit_cast(uint4, h);
  lo = __builtin_bit_cast(uint4, r);
}
__device__ __forceinline__ void add8(float* x, const uint4& v) {
  const f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += (float)h[e];
}

template <typename T>
__device__ __forceinline__ void put_result(const NsArgs& g, int i, long row, int col, const float* o) {
  if (row >= g.rows || col >= g.cols) return;
  Unit<T> u;
  u.set(o);
  u.store(static_cast<T*>(g.out) + ((long)i * g.rows + row) * g.cols + col, g.cols - col);
}
// w <- keep w - rate o in 32 bits, and its copy in the expert store
template <typename T>
__device__ __forceinline__ void update(const NsArgs& g, int i, long row, int col, const float* o) {
  if (row >= g.rows || col >= g.cols) return;
  const int left = g.cols - col;
  T* const p = static_cast<T*>(g.param) + g.param_at[i] + row * g.cols + col;
  float* const m = g.master ? g.master + ((long)i * g.rows + row) * g.cols + col : reinterpret_cast<float*>(p);
  Unit<float> w;
  w.load(m, left);
#pragma unroll
  for (int e = 0; e < 8; ++e) w.w[e] = fmaf(-g.rate, o[e], g.keep * w.w[e]);
  w.store(m, left);
  if (g.master) {
    Unit<T> u;
    u.set(w.w);
    u.store(p, left);
  }
}

// One BM x BN tile of one product, of a symmetric one (kGram, kPoly) with its mirror image.  Four wavefronts, each a quarter of the tile.
// Operands come straight into LDS as in gemm_mfma.hip: A, and B with B_KC, as [row][k], else B as [k][column].
template <Epi EPI, bool B_KC, typename T, int BM, int BN, int NS>
__global__ __launch_bounds__(256, 2) void ns_gemm_kernel(const NsArgs g) {
  constexpr int BK = 64, TM = BM / 32, TN = BN / 32, NA = BM / 32, NB = BN / 32, NP = NA + NB;
  constexpr int A_VEC = BM * 8, B_VEC = BN * 8, STAGE = A_VEC + B_VEC;
  constexpr int PITCH = BN / 2 + 4, SLAB = 32 * PITCH;
  constexpr bool SYM = EPI == kGram || EPI == kPoly;
  static_assert(BM == BN, "mirror images of square tiles");
  __shared__ uint4 smem[NS * STAGE > SLAB ? NS * STAGE : SLAB];
  static_assert(NS * STAGE * 16 >= 4 * SLAB * 4, "a slab for every wavefront");
  const int tid = threadIdx.x, lane = tid & 63, wave = (int)uniform(tid >> 6);
  const int l16 = lane & 15, lq = lane >> 4, wm = wave >> 1, wn = wave & 1;

  const unsigned mt = (unsigned)cdiv(g.M, BM), nt = (unsigned)cdiv(g.N, BN), per = SYM ? mt * (mt + 1) / 2 : mt * nt;
  const unsigned total = per * (unsigned)g.n, per_xcd = (total + kXcds - 1) / kXcds;
  const unsigned slot = blockIdx.x / kXcds, t = (blockIdx.x % kXcds) * per_xcd + slot;
  if (slot >= per_xcd || t >= total) return;
  const int mat = (int)(t / per);
  unsigned in = t - (unsigned)mat * per, mi, ni;
  if (SYM) {
    mi = (unsigned)((sqrtf(8.f * (float)in + 1.f) - 1.f) * 0.5f);
    if (mi * (mi + 1) / 2 > in) --mi;
    if ((mi + 1) * (mi + 2) / 2 <= in) ++mi;
    ni = in - mi * (mi + 1) / 2;
  } else {
    mi = in / nt;
    ni = in - mi * nt;
  }
  const int m0 = (int)mi * BM, n0 = (int)ni * BN;

  // ---- operands ----
  const int nk = g.K / BK, nsteps = nk * g.passes;
  auto base_of = [](const f16* p, long elems) -> unsigned long {
    const unsigned long v = reinterpret_cast<unsigned long>(p + elems);
    return (unsigned long)uniform((unsigned)(v >> 32)) << 32 | uniform((unsigned)v);
  };
  const unsigned long a_base = base_of(g.A, mat * g.a_ms), b_base = base_of(g.B, mat * g.b_ms);
  const unsigned a_bytes = uniform((unsigned)g.M * (unsigned)g.lda * 2u), b_bytes = uniform((unsigned)(B_KC ? g.N : g.K) * (unsigned)g.ldb * 2u);
  const unsigned a_step = 128u, b_step = uniform(B_KC ? 128u : (unsigned)g.ldb * 128u);       // bytes per K-tile
  const int kc_chunk = (lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7);
  constexpr int BCH = BN / 8;
  unsigned aoff[NA], boff[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i) aoff[i] = ((unsigned)(m0 + wave * 8 + (lane >> 3) + 32 * i) * (unsigned)g.lda + (unsigned)kc_chunk * 8u) * 2u;
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (B_KC) {
      boff[i] = ((unsigned)(n0 + wave * 8 + (lane >> 3) + 32 * i) * (unsigned)g.ldb + (unsigned)kc_chunk * 8u) * 2u;
    } else {
      const int k = wave * (64 / BCH) + lane / BCH + i * (64 / NB);
      boff[i] = ((unsigned)k * (unsigned)g.ldb + (unsigned)n0 + (unsigned)((lane % BCH) ^ (2 * (k & 3))) * 8u) * 2u;
    }
  }
  const unsigned lds0 = (unsigned)(unsigned long)(__attribute__((address_space(3))) uint4*)smem + (unsigned)wave * 1024u;
  auto load_tile = [&](int step, int s) {
    const int pass = step / nk, k = step - pass * nk;
    const bool alive = step < nsteps;
    const unsigned long a = a_base + (g.passes == 3 && pass == 0 ? (unsigned long)g.a_lo * 2 : 0) + (unsigned)k * a_step;
    const unsigned long b = b_base + (g.passes == 3 && pass == 1 ? (unsigned long)g.b_lo * 2 : 0) + (unsigned long)((unsigned)k * b_step);
    const rsrc_t ra = make_rsrc(a, alive ? a_bytes - (unsigned)k * a_step : 0u), rb = make_rsrc(b, alive ? b_bytes - (unsigned)k * b_step : 0u);
    const unsigned dst = lds0 + (unsigned)s * (STAGE * 16u);
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const unsigned d = set_lds_dest(dst + (unsigned)i * 4096u);
      one_instruction();
      load_to_lds(ra, aoff[i], d);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const unsigned d = set_lds_dest(dst + A_VEC * 16u + (unsigned)i * 4096u);
      one_instruction();
      load_to_lds(rb, boff[i], d);
    }
  };

  f32x4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int kc_pos = lq ^ (l16 >> 1);
  const uint4* const a_kc = smem + (wm * (BM / 2) + l16) * 8;
  const uint4* const b_kc = smem + A_VEC + (wn * (BN / 2) + l16) * 8;
  const bf16_t* const b_tr = reinterpret_cast<const bf16_t*>(smem + A_VEC) + (lq * 8 + (l16 >> 2)) * BN + (lane & 3) * 4 + wn * (BN / 2);
  auto tr_pos = [&](int i) { return (i & ~3) * 16 + ((i & 3) ^ (l16 >> 2)) * 16; };
  for (int s = 0; s < NS - 1; ++s) load_tile(s, s);
  int cur = 0, fill = NS - 1;
  for (int step = 0; step < nsteps; ++step) {
    wait_and_meet<(NS - 2) * NP>();
    load_tile(step + NS - 1, fill);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      f16x8 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = __builtin_bit_cast(f16x8, a_kc[cur * STAGE + i * 128 + (kc_pos ^ (ks * 4))]);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        if (B_KC) {
          fb[j] = __builtin_bit_cast(f16x8, b_kc[cur * STAGE + j * 128 + (kc_pos ^ (ks * 4))]);
        } else {
          const bf16_t* p = b_tr + cur * (STAGE * 8) + ks * 32 * BN + tr_pos(j);
          const uint2 lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * BN);
          fb[j] = __builtin_bit_cast(f16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
        }
      }
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j], fa[i], acc[j][i], 0, 0, 0);
    }
    cur = cur + 1 == NS ? 0 : cur + 1;
    fill = fill + 1 == NS ? 0 : fill + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // no load may still write the LDS that the slabs use
  __syncthreads();

  // ---- epilogue: 32 rows of the wavefront's quarter at a time, turned through LDS so that lanes lie along the columns ----
  float* const slab = reinterpret_cast<float*>(smem) + wave * SLAB;
  const float f1 = g.factor ? g.factor[mat] : 1.f, f = EPI == kGram ? f1 * f1 : f1;
  const bool mirror = SYM ? mi != ni : (EPI == kLast || EPI == kUpdate) && g.tall;
  const bool direct = SYM || EPI == kStep || !g.tall;
  const f16* const E = g.E + mat * g.e_ms;
  f16* const C = g.C + mat * g.c_ms;
  auto put = [&](int row, int col, const float* v) {
    if (EPI == kLast || EPI == kUpdate) {
      if (EPI == kLast) put_result<T>(g, mat, row, col, v);
      else update<T>(g, mat, row, col, v);
    } else {
      uint4 hi, lo;
      split8(v, hi, lo);
      *reinterpret_cast<uint4*>(C + (long)row * g.ldc + col) = hi;
      if (g.c_lo != 0) *reinterpret_cast<uint4*>(C + g.c_lo + (long)row * g.ldc + col) = lo;
    }
  };
#pragma unroll
  for (int i = 0; i < BM / 64; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int ii = 0; ii < 2; ++ii)
        *reinterpret_cast<f32x4*>(slab + (ii * 16 + l16) * PITCH + j * 16 + lq * 4) = acc[j][2 * i + ii];
    wave_lds_order();
    constexpr int CPR = BN / 16, RPI = 64 / CPR;         // lanes per row, rows at a time
#pragma unroll
    for (int st = 0; st < 32 / RPI; ++st) {
      const int r = st * RPI + lane / CPR, c = lane % CPR * 8;
      const int row = m0 + wm * (BM / 2) + i * 32 + r, col = n0 + wn * (BN / 2) + c;
      float v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(slab + r * PITCH + c + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = q[e];
      }
      const bool in_range = row < g.M && col < g.N;
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (EPI != kGram && in_range) {
        add8(x, *reinterpret_cast<const uint4*>(E + (long)row * g.lde + col));
        if (g.e_lo != 0) add8(x, *reinterpret_cast<const uint4*>(E + g.e_lo + (long)row * g.lde + col));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf(g.alpha, v[e], g.beta * x[e]) * f;
      if (EPI == kPoly) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += row == col + e ? g.diagonal : 0.f;
      }
      if (direct && in_range) put(row, col, v);
      if (mirror) {
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(slab + r * PITCH + c + 4 * h) = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
      }
    }
    wave_lds_order();
    if (mirror) {
#pragma unroll
      for (int st = 0; st < BN / 32; ++st) {             // lanes: sixteen columns by four runs of eight rows
        const int c = st * 16 + l16, r = lq * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = slab[(r + e) * PITCH + c];
        const int row = n0 + wn * (BN / 2) + c, col = m0 + wm * (BM / 2) + i * 32 + r;
        if (row < g.N && col < g.M) put(row, col, v);
      }
      wave_lds_order();
    }
  }
}

// ---- into the scaled form, and the momentum ----

struct PrepArgs {
  const void* src;                   // orthogonalisation: [n, rows, cols]
  float* m;                          // optimizer step: momentum and gradient; the matrix is nesterov ? g + beta m : m
  const float* grad;
  float beta, grad_scale;
  bool nesterov;
  int rows, cols, n;
  double* part;                      // [n][blocks] partial sums of squares
  int blocks;
  float* factor;
  f16* X;
  long ms, lo_plane;                 // lo_plane 0: no remainders
  int lo, hi, ld;                    // of X, the matrix's sides and the stored rows' length
  int lo_p;
  bool tall;
};

// Squares are summed in 64 bits: those of a small gradient are below what 32 bits hold, and the sum scales everything that follows.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void ns_sum_kernel(const PrepArgs a) {
  __shared__ double red[4];
  const long elems = (long)a.rows * a.cols, first = (long)blockIdx.y * elems;
  double s = 0;
  for (long u = (long)blockIdx.x * 256 + threadIdx.x; u * 8 < elems; u += (long)a.blocks * 256) {
    const long at = first + u * 8, rest = elems - u * 8;
    const int left = rest < 8 ? (int)rest : 8;
    float v[8];
    if (MUON) {
      Unit<float> m, g;
      m.load(a.m + at, left);
      g.load(a.grad + at, left);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ge = g.w[e] * a.grad_scale;
        m.w[e] = fmaf(a.beta, m.w[e], ge);
        v[e] = a.nesterov ? fmaf(a.beta, m.w[e], ge) : m.w[e];
      }
      m.store(a.m + at, left);
    } else {
      Unit<T> x;
      x.load(static_cast<const T*>(a.src) + at, left);
      x.get(v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (double)v[e] * (double)v[e];          // (beyond the end: zeros)
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.part[(long)blockIdx.y * a.blocks + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// A 64 x 64 tile of X: U 2^e, so that a bf16 matrix is held exactly; what the power of two leaves of 1 / |U| is the factor of
// the first step's products.  A matrix of zeros stays one; infinities and NaN make all of it NaN.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void ns_scale_kernel(const PrepArgs a) {
  __shared__ double red[4];
  __shared__ float turn[64][65];
  const int tid = threadIdx.x, mat = blockIdx.y, tiles_h = a.ld / 64;
  double s = tid < a.blocks ? a.part[(long)mat * a.blocks + tid] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  s = (red[0] + red[1]) + (red[2] + red[3]);
  int exponent = 0;
  float factor = 0.f;
  if (s != 0.0) {
    const double part = frexp(sqrt(s), &exponent);               // |U| = part 2^exponent, part in [1/2, 1)
    factor = isfinite(s) ? (float)(1.0 / part) : NAN;
    if (!isfinite(s)) exponent = 0;
  }
  if (blockIdx.x == 0 && tid == 0) a.factor[mat] = factor;
  const int shift = kXBits - exponent;
  const int l0 = (blockIdx.x / tiles_h) * 64, h0 = (blockIdx.x % tiles_h) * 64;
  const long first = (long)mat * a.rows * a.cols;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r = half * 32 + tid / 8, c = tid % 8 * 8;
    const int row = (a.tall ? h0 : l0) + r, col = (a.tall ? l0 : h0) + c;       // of the caller's matrix
    const int left = row < a.rows ? a.cols - col : 0;
    const long at = first + (left > 0 ? (long)row * a.cols + col : 0);
    float v[8];
    if (MUON) {
      Unit<float> m;
      m.load(a.m + at, left);
      m.get(v);
      if (a.nesterov) {
        Unit<float> g;
        g.load(a.grad + at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(a.beta, v[e], g.w[e] * a.grad_scale);
      }
    } else {
      Unit<T> x;
      x.load(static_cast<const T*>(a.src) + at, left);
      x.get(v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = ldexpf(v[e], shift);
    if (!a.tall) {
      uint4 hi, lo;
      split8(v, hi, lo);
      f16* const p = a.X + mat * a.ms + (long)row * a.ld + col;
      *reinterpret_cast<uint4*>(p) = hi;
      if (a.lo_plane != 0) *reinterpret_cast<uint4*>(p + a.lo_plane) = lo;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) turn[r][c + e] = v[e];
    }
  }
  if (!a.tall) return;
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r = half * 32 + tid / 8, c = tid % 8 * 8;                         // of X's tile
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = turn[c + e][r];
    uint4 hi, lo;
    split8(v, hi, lo);
    f16* const p = a.X + mat * a.ms + (long)(l0 + r) * a.ld + h0 + c;
    *reinterpret_cast<uint4*>(p) = hi;
    if (a.lo_plane != 0) *reinterpret_cast<uint4*>(p + a.lo_plane) = lo;
  }
}

struct Buffers {
  int lo, hi, lo_p, hi_p, planes;     // planes of G and P; X has two
  int sum_blocks;
  size_t part, factor, x[2], g, p, total;
};

Buffers buffers(int n, int rows, int cols, int dtype) {
  Buffers b;
  b.lo = rows < cols ? rows : cols; b.hi = rows < cols ? cols : rows;
  b.lo_p = (int)round_up(b.lo, kPad); b.hi_p = (int)round_up(b.hi, kPad);
  b.planes = dtype == SPES_F32 ? 2 : 1;
  const long units = ((long)rows * cols + 7) / 8;
  b.sum_blocks = (int)(units / 1024 < 1 ? 1 : units / 1024 > kSumBlocks ? kSumBlocks : units / 1024);
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += round_up(bytes, 256); return o; };
  b.part = take((size_t)n * kSumBlocks * 8);
  b.factor = take((size_t)n * 4);
  for (int i = 0; i < 2; ++i) b.x[i] = take((size_t)n * 2 * b.lo_p * b.hi_p * 2);
  b.g = take((size_t)n * b.planes * b.lo_p * b.lo_p * 2);
  b.p = take((size_t)n * b.planes * b.lo_p * b.lo_p * 2);
  b.total = off;
  return b;
}

template <Epi EPI, bool B_KC, typename T>
int launch_product(const NsArgs& g, hipStream_t s) {
  constexpr int BM = 128;
  const long mt = cdiv(g.M, BM), nt = cdiv(g.N, BM);
  const long total = (EPI == kGram || EPI == kPoly ? mt * (mt + 1) / 2 : mt * nt) * g.n;
  hipLaunchKernelGGL((ns_gemm_kernel<EPI, B_KC, T, BM, BM, 2>), dim3((unsigned)((total + kXcds - 1) / kXcds * kXcds)), dim3(256), 0, s, g);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

// carried: steps that take X with its remainder, in bf16 storage
constexpr int kCarried = 2;

template <typename T>
int run(const Buffers& b, int steps, const float* coef, bool exact_start, bool muon, PrepArgs a, NsArgs end, const long* param_at, char* scratch, hipStream_t s) {
  const bool f32 = sizeof(T) == 4;
  const long xs = (long)b.lo_p * b.hi_p, gs = (long)b.lo_p * b.lo_p;
  f16* X[2] = {reinterpret_cast<f16*>(scratch + b.x[0]), reinterpret_cast<f16*>(scratch + b.x[1])};
  f16 *G = reinterpret_cast<f16*>(scratch + b.g), *P = reinterpret_cast<f16*>(scratch + b.p);
  a.part = reinterpret_cast<double*>(scratch + b.part); a.blocks = b.sum_blocks;
  a.factor = reinterpret_cast<float*>(scratch + b.factor);
  a.X = X[0]; a.ms = 2 * xs; a.lo = b.lo; a.hi = b.hi; a.ld = b.hi_p; a.lo_p = b.lo_p; a.tall = a.rows > a.cols;
  const bool first_lo = f32 || !exact_start;
  a.lo_plane = first_lo ? xs : 0;
  const dim3 sums((unsigned)b.sum_blocks, (unsigned)a.n), tiles((unsigned)(b.lo_p / 64 * (b.hi_p / 64)), (unsigned)a.n);
  if (muon) {
    hipLaunchKernelGGL((ns_sum_kernel<T, true>), sums, dim3(256), 0, s, a);
    hipLaunchKernelGGL((ns_scale_kernel<T, true>), tiles, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((ns_sum_kernel<T, false>), sums, dim3(256), 0, s, a);
    hipLaunchKernelGGL((ns_scale_kernel<T, false>), tiles, dim3(256), 0, s, a);
  }
  if (hipGetLastError() != hipSuccess) return SPES_EHIP;
  NsArgs g = end;
  g.n = a.n; g.passes = f32 ? 3 : 1;
  for (int i = 0; i < steps; ++i) {
    const bool last = i + 1 == steps, x_lo = f32 || (i == 0 ? first_lo : i < kCarried), next_lo = f32 || i + 1 < kCarried;
    f16 *x = X[i & 1], *y = X[(i + 1) & 1];
    const float* factor = i == 0 ? a.factor : nullptr;
    NsArgs q = g;
    q.A = q.B = x; q.a_ms = q.b_ms = 2 * xs; q.a_lo = q.b_lo = xs; q.lda = q.ldb = b.hi_p;
    q.M = q.N = b.lo_p; q.K = b.hi_p;
    q.C = G; q.c_ms = b.planes * gs; q.c_lo = f32 ? gs : 0; q.ldc = b.lo_p;
    q.alpha = ldexpf(1.f, kGBits - 2 * kXBits); q.beta = 0.f; q.factor = factor;
    q.E = G; q.e_ms = 0; q.e_lo = 0; q.lde = b.lo_p;
    int rc = launch_product<kGram, true, T>(q, s);
    if (rc != SPES_OK) return rc;
    q.A = q.B = q.E = G; q.a_ms = q.b_ms = q.e_ms = b.planes * gs; q.a_lo = q.b_lo = gs; q.e_lo = f32 ? gs : 0; q.lda = q.ldb = b.lo_p;
    q.K = b.lo_p; q.C = P;
    q.alpha = coef[2] * ldexpf(1.f, -kGBits); q.beta = coef[1]; q.factor = nullptr;
    const float shift = f32 || i < kCarried ? 0.f : -(coef[1] + coef[2]);
    q.diagonal = ldexpf(shift, kGBits);
    rc = launch_product<kPoly, true, T>(q, s);
    if (rc != SPES_OK) return rc;
    q.A = P; q.B = q.E = x; q.b_ms = q.e_ms = 2 * xs; q.b_lo = xs; q.e_lo = x_lo ? xs : 0; q.ldb = q.lde = b.hi_p;
    q.M = b.lo_p; q.N = b.hi_p; q.K = b.lo_p;
    q.C = y; q.c_ms = 2 * xs; q.c_lo = next_lo ? xs : 0; q.ldc = b.hi_p;
    q.alpha = ldexpf(1.f, -kGBits); q.beta = coef[0] - shift; q.factor = factor;
    if (!last) {
      rc = launch_product<kStep, false, T>(q, s);
      if (rc != SPES_OK) return rc;
      continue;
    }
    // out of the scaled form
    q.alpha = ldexpf(q.alpha, -kXBits); q.beta = ldexpf(q.beta, -kXBits);
    if (!muon) return launch_product<kLast, false, T>(q, s);
    for (int first = 0; first < a.n; first += kSlots) {
      NsArgs u = q;
      u.n = a.n - first < kSlots ? a.n - first : kSlots;
      u.A += first * u.a_ms; u.B += first * u.b_ms; u.E += first * u.e_ms;
      if (u.factor) u.factor += first;
      if (u.master) u.master += (long)first * a.rows * a.cols;
      for (int k = 0; k < u.n; ++k) u.param_at[k] = param_at[first + k];
      rc = launch_product<kUpdate, false, T>(u, s);
      if (rc != SPES_OK) return rc;
    }
  }
  return SPES_OK;
}

}  // namespace

size_t orthogonalize_scratch_bytes(int n, int rows, int cols, int dtype) { return buffers(n, rows, cols, dtype).total; }

int launch_orthogonalize(int dtype, int n, int rows, int cols, const void* src, void* out, int steps, const float* coef, void* scratch, hipStream_t s) {
  const Buffers b = buffers(n, rows, cols, dtype);
  PrepArgs a = {};
  a.src = src; a.rows = rows; a.cols = cols; a.n = n;
  NsArgs end = {};
  end.out = out; end.rows = rows; end.cols = cols; end.tall = rows > cols;
  return dtype == SPES_F32 ? run<float>(b, steps, coef, false, false, a, end, nullptr, static_cast<char*>(scratch), s)
                           : run<bf16_t>(b, steps, coef, true, false, a, end, nullptr, static_cast<char*>(scratch), s);
}

int launch_masked_muon(int dtype, int n, int rows, int cols, void* param, const long* param_at, float* master, float* m, const float* grad, float lr,
                       float beta, int nesterov, float weight_decay, float update_scale, int steps, const float* coef, float grad_scale, void* scratch,
                       hipStream_t s) {
  const Buffers b = buffers(n, rows, cols, dtype);
  PrepArgs a = {};
  a.m = m; a.grad = grad; a.beta = beta; a.grad_scale = grad_scale; a.nesterov = nesterov != 0; a.rows = rows; a.cols = cols; a.n = n;
  NsArgs end = {};
  end.param = param; end.master = master; end.rows = rows; end.cols = cols; end.tall = rows > cols;
  end.keep = 1.f - lr * weight_decay; end.rate = lr * update_scale;
  return dtype == SPES_F32 ? run<float>(b, steps, coef, false, true, a, end, param_at, static_cast<char*>(scratch), s)
                           : run<bf16_t>(b, steps, coef, false, true, a, end, param_at, static_cast<char*>(scratch), s);
}

}  // namespace spes
