// Newton-Schulz orthogonalisation of a stack of matrices, and the optimizer step built on it.
//
// A matrix U is scaled to Frobenius norm 1 and taken through the odd polynomial x -> a x + b x^3 + c x^5 of its singular values, `steps` times.
// With X the scaled matrix, its shorter side lo along the rows (a tall one is turned on the way in and out)
//      G = X X^T      P = b G + c G G      X <- a X + P X
// so a step is three matrix products of lo^2 hi, lo^3 and 2 lo^2 hi operations, of the symmetric ones half the tiles.
//
// The products run on the matrix cores on fp16 operands with fp32 sums.  What limits them is not the directions that the matrix has but those that it
// lacks: the polynomial grows small singular values 3.4-fold a step, and rounding noise in empty directions alike.  An expert that got
// few tokens has a gradient of low rank, and there the fp16 rounding of X alone, 2e-4 of its norm, would end as 1.4e-2 (512 x 1024, rank 1; bf16
// operands leave 1.3e-2 even of a broad spectrum).  So X goes from step to step with its remainder (a second fp16 plane, 22 bits together), which is added, times a, at the
// step's end.  The term a X itself stands in P, X <- (P + a I) X + a remainder: where singular values are near 1, P is near (b + c) I and
// P + a I is rounded to finer steps; what its diagonal loses in that, up to 2^-10, is kept in 32 bits and multiplied with X at the step's end too
// (without: 2.3e-3).  The last step, behind which nothing grows, does without both.  Left are, against 64 bits after five steps, in the update
// of fp32 weights: rank 1 1.4e-3, 8 0.7e-3, 128 1.2e-3, full rank 1.1e-3, 16 strong directions above a broad floor 0.8e-3 (512 x 1024; rank 1 of 96 x 96
// 1.6e-3, of sides below 64 up to 2.1e-3).  fp32 storage takes every operand as such a pair and every product as three,
// lo hi + hi lo + hi hi: full rank 2e-6, rank 1 1.2e-4, as products in fp32.  Range: X stands scaled by 2^12, G and P by 2^11, which holds singular values below 5, G below 25
// and P below 31; after the first scaling they are at most 1.21 with the default coefficients.
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "lds_load.h"
#include "plan.h"
#include "units.h"

namespace spes {
namespace {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr int kXcds = 8;
constexpr int kXBits = 12, kGBits = 11;        // X, and G and P, as they are stored, are scaled by these powers of two
constexpr int kPad = 64;                       // stored matrices have sides that are multiples of this, zeros beyond the matrix
constexpr int kFewRows = 32;                   // up to so many, operands are pairs in bf16 storage too: rounding is of one sign in a single direction (a
                                               // 1 x 16 matrix came out 4.4e-3 off), and such matrices wait for launches, not for products
constexpr int kSumBlocks = 256;                // partial sums of squares of a matrix, at most
constexpr int kSlots = 64;                     // matrices of an optimizer launch

enum Epi { kGram, kPoly, kStep, kLast, kUpdate, kPart };      // kLast, kUpdate: a step whose result is the caller's, or his weights' update; kPart: a
                                                              // part of kGram's sum, of K-tiles that blockIdx.y says

struct NsArgs {
  const f16 *A, *B, *E;
  f16* C;
  long a_ms, b_ms, e_ms, c_ms;                 // elements from one matrix to the next
  long a_lo, b_lo, e_lo, c_lo;                 // elements from a matrix to its plane of remainders; 0: it has none here
  int lda, ldb, lde, ldc;
  int M, N, K, n;                              // of the products, padded; matrices
  float alpha, beta;                           // result = (alpha product + beta E) factor
  float diagonal;                              // kPoly: added to the diagonal
  float* rest;                                 // [n][M], operands that are not pairs: what P's diagonal lost when it was rounded
  const float* factor;                         // of each matrix, NULL: 1.  kGram: squared
  float* part;                                 // kPart: [parts][n][M][M]
  int k_tiles;                                 // kPart: of a part
  // the end: rows x cols as the caller has them
  void *out, *param;
  float* master;
  int rows, cols;
  bool tall;
  float keep, rate;                            // w <- keep w - rate o
  long param_at[kSlots];                       // of each matrix, in elements
};

// x as the sum of two fp16 values.  (x is pinned as it is in 32 bits: a product that is rounded straight to fp16 for one of
// the two uses and by way of fp32 for the other comes out a step apart where the fp32 value lies half way between two, and the remainder is then
// that of the other one.)
template <int N>
__device__ __forceinline__ void split(const float* x, f16* hi, f16* lo) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float v = x[e];
    asm("" : "+v"(v));
    hi[e] = (f16)v;
    lo[e] = (f16)(v - (float)hi[e]);
  }
}
__device__ __forceinline__ void split8(const float* x, uint4& hi, uint4& lo) {
  f16 h[8], r[8];
  split<8>(x, h, r);
  hi = __builtin_bit_cast(uint4, *reinterpret_cast<f16x8*>(h));
  lo = __builtin_bit_cast(uint4, *reinterpret_cast<f16x8*>(r));
}
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;

template <int BM_, int BN_, int NSA_, int NSB_, int MINB_>
struct Cfg {
  static constexpr int BM = BM_, BN = BN_, MINB = MINB_;
  static constexpr int NSA = NSA_, NSB = NSB_;              // LDS slots of each operand, one K-tile each
  static constexpr int WM = BM < 64 ? 1 : 2, QM = BM / WM, QN = BN * WM / 4;      // wavefronts along m, and the part of the tile that each has
  static constexpr int BK = 64, TM = QM / 16, TN = QN / 16; // 16 x 16 MFMA tiles per wavefront along m, n
  static constexpr int NA = BM / 32, NB = BN / 32;          // 1 KB loads per wavefront and K-tile
  static constexpr int A_VEC = BM * 8, B_VEC = BN * 8;      // 16-byte units of a slot
  // epilogue slabs, 32 rows of a wavefront's quarter: floats, or bytes of fp16 (rows 4 or 36 banks apart: the sixteen rows of a write miss each other)
  static constexpr int PITCH = QN + 4, SLAB = 32 * PITCH, PITCH16 = 2 * QN + 16, SLAB16 = 32 * PITCH16;
  static constexpr bool STAGED = BN == 64 && (BM < 64 || MINB == 1);      // both planes of a pair, or two K-tiles, side by side in a slot, see the main loop
  static constexpr int UNITS = (NSA * A_VEC + NSB * B_VEC) * (STAGED ? 2 : 1);
  static_assert(4 * SLAB * 4 <= UNITS * 16 && 4 * 4 * SLAB16 <= UNITS * 16, "a float slab, or four of fp16, for every wavefront");
  static_assert(BM == BN || 2 * BM == BN, "square tiles, and halves of them");
};
// one block per CU: all 160 KB of LDS, 256 accumulators per lane; half of such a tile
typedef Cfg<256, 256, 3, 2, 1> Tile;
typedef Cfg<128, 256, 3, 3, 1> TileHalf;
// two blocks per CU; half of such a tile
typedef Cfg<128, 128, 3, 2, 2> TileSmall;
typedef Cfg<64, 128, 4, 3, 2> TileSmallHalf;
// few tiles; on pairs
typedef Cfg<64, 64, 5, 5, 2> TileTiny;
typedef Cfg<32, 64, 3, 3, 2> TileTinyHalf;
typedef Cfg<64, 64, 4, 4, 1> TileTinyPairs;
typedef Cfg<32, 64, 4, 4, 1> TileTinyPairsHalf;

// One BM x BN tile of one product, of a symmetric one (kGram, kPoly) with its mirror image.  Four wavefronts, each a quarter of the tile (QM x QN) as TM x TN
// MFMA tiles of 16 x 16.  Operands come straight into LDS, K-tiles of 64, three or two of them at a time: A, and B with B_KC, as
// [row][k], else B as [k][column], read through the transposing read; both permuted within a row against bank conflicts.  The main loop is
// that of gemm_mfma.hip without its masks and index tables: stored matrices are padded, so every K-tile is whole.  Fragments are read a
// k-step ahead of their MFMAs, and loads, reads and the scalars of the next K-tiles are dealt out over the gaps between MFMAs.
// Bound by the matrix cores at the clock that their power allows where there are many tiles: 8 of 3584 x 4864, 842 us of a step are 1.19 PFLOP/s, 895 with X in two
// planes read and written beside it 1.12, 465 of G 1.15 (a library product of 8192^3 in fp16: 1.24).  With few tiles by operands on their way, which every die fetches for itself: one of
// 1280 x 1536, 210 tiles of 64 x 64, 9.3 us of G for 2.1 of multiplying.
// SPLIT: operands are pairs.  IN, OUT: planes of what is read beside the product and of the result
// Tile `in` of matrix `mat`, in squares of BN, of which `half` is the upper or the lower half if BM is less
template <Epi EPI, bool B_KC, bool SPLIT, int IN, int OUT, typename T, typename C>
__device__ __forceinline__ void ns_tile(const NsArgs& g, uint4* const smem, const int mat, const unsigned in, const int half) {
  constexpr int BM = C::BM, BN = C::BN, QM = C::QM, QN = C::QN, BK = C::BK, TM = C::TM, TN = C::TN, NSA = C::NSA, NSB = C::NSB, NA = C::NA, NB = C::NB, NP = NA + NB;
  constexpr int A_VEC = C::A_VEC, B_VEC = C::B_VEC, PITCH = C::PITCH;
  constexpr bool SYM = EPI == kGram || EPI == kPoly || EPI == kPart;
  const int tid = threadIdx.x, lane = tid & 63, wave = (int)uniform(tid >> 6);
  const int l16 = lane & 15, lq = lane >> 4, wm = C::WM == 1 ? 0 : wave >> 1, wn = C::WM == 1 ? wave : wave & 1;
  unsigned mi, ni;
  if (SYM) {
    mi = (unsigned)((sqrtf(8.f * (float)in + 1.f) - 1.f) * 0.5f);
    if (mi * (mi + 1) / 2 > in) --mi;
    if ((mi + 1) * (mi + 2) / 2 <= in) ++mi;
    ni = in - mi * (mi + 1) / 2;
  } else {
    // row tiles four at a time, the column tiles inside: what an XCD works on at once shares four row panels
    const unsigned mt = (unsigned)cdiv(g.M, BN), nt = (unsigned)cdiv(g.N, BN);
    const unsigned group = in / (4 * nt), within = in - group * 4 * nt, left = mt - group * 4, rows = left < 4 ? left : 4;
    ni = within / rows;
    mi = group * 4 + (within - ni * rows);
  }
  const int m0 = (int)uniform(mi * BN + (unsigned)half * BM), n0 = (int)uniform(ni * BN);
  if (BM != BN && m0 >= g.M) return;

  // ---- operands: buffer resources whose base moves with the K-tile and that end with the operand, behind which loads deliver zeros; a lane's
  // byte offsets are fixed ----
  static_assert(EPI != kPart || B_KC, "parts along the rows of both operands");
  const int k0 = EPI == kPart ? (int)blockIdx.y * g.k_tiles : 0;
  const int nk = (int)uniform(EPI == kPart ? (unsigned)min(g.k_tiles, g.K / BK - k0) : (unsigned)g.K / BK), nsteps = SPLIT ? 3 * nk : nk;
  auto base_of = [](const f16* p, long elems) -> unsigned long {
    const unsigned long v = reinterpret_cast<unsigned long>(p + elems);
    return (unsigned long)uniform((unsigned)(v >> 32)) << 32 | uniform((unsigned)v);
  };
  const unsigned long a_base = base_of(g.A, mat * g.a_ms + k0 * BK), b_base = base_of(g.B, mat * g.b_ms + k0 * BK);
  const unsigned a_bytes = uniform(((unsigned)g.M * (unsigned)g.lda - (unsigned)(k0 * BK)) * 2u);
  const unsigned b_bytes = uniform(((unsigned)(B_KC ? g.N : g.K) * (unsigned)g.ldb - (unsigned)(k0 * BK)) * 2u);
  const unsigned a_step = BK * 2u, b_step = uniform(B_KC ? BK * 2u : (unsigned)g.ldb * (BK * 2u));       // bytes per K-tile
  const int kc_chunk = (lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7);
  constexpr int BCH = BN / 8;       // 16-byte chunks per k-row
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

  f32x4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      // (zeros that the compiler takes for different values)
      if (C::MINB == 1) asm("" : "+a"(acc[j][i]));
      else asm("" : "+v"(acc[j][i]));
    }

  if constexpr (C::STAGED) {
    // On the smallest tiles a wavefront has four or eight MFMAs in a K-tile, less than its meeting and its reads take.  So all four planes of
    // a K-tile are loaded at once, which is 24 MFMAs of a wavefront for one meeting and four loads in place of six, in four stages of LDS; where operands
    // are not pairs, two K-tiles, in the order of the loop below.  Against that loop, over the pairs one after the other: 4 matrices of 512 x 256 in
    // fp32, products of 10.2, 6.9 and 7.3 us 7.8, 6.2 and 6.5, the call 122 -> 105.  (On squares of 64 without pairs it takes 9.7 us for that one's 8.9, 210 tiles.)
    static_assert(NSA == NSB, "whole stages");
    constexpr int STAGE = 2 * (A_VEC + B_VEC), STAGES = NSA;
    const unsigned a_lo = uniform((unsigned)g.a_lo * 2u), b_lo = uniform((unsigned)g.b_lo * 2u);
    const unsigned lds0 = (unsigned)(unsigned long)(__attribute__((address_space(3))) uint4*)smem + (unsigned)wave * 1024u;
    auto load_stage = [&](int k, int s) {
#pragma unroll
      for (int two = 0; two < 2; ++two) {
        const int t = SPLIT ? k : 2 * k + two;
        const unsigned inside = t < nk ? ~0u : 0u, ahead = (unsigned)t;
        const unsigned a_dst = lds0 + (unsigned)(s * STAGE + two * A_VEC) * 16u, b_dst = lds0 + (unsigned)(s * STAGE + 2 * A_VEC + two * B_VEC) * 16u;
        const rsrc_t ra = make_rsrc(a_base + (SPLIT && two ? a_lo : 0u) + (unsigned long)(ahead * a_step), (a_bytes - ahead * a_step) & inside);
        const rsrc_t rb = make_rsrc(b_base + (SPLIT && two ? b_lo : 0u) + (unsigned long)(ahead * b_step), (b_bytes - ahead * b_step) & inside);
#pragma unroll
        for (int i = 0; i < NA; ++i) {
          const unsigned d = set_lds_dest(a_dst + (unsigned)i * 4096u);
          one_instruction();
          load_to_lds(ra, aoff[i], d);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const unsigned d = set_lds_dest(b_dst + (unsigned)i * 4096u);
          one_instruction();
          load_to_lds(rb, boff[i], d);
        }
      }
    };
    const int kc_pos = lq ^ (l16 >> 1);
    const uint4* const a_kc = smem + (wm * QM + l16) * 8;
    const uint4* const b_kc = smem + 2 * A_VEC + (wn * QN + l16) * 8;
    const bf16_t* const b_tr = reinterpret_cast<const bf16_t*>(smem + 2 * A_VEC) + (lq * 8 + (l16 >> 2)) * BN + (lane & 3) * 4;
    for (int s = 0; s < STAGES - 1; ++s) load_stage(s, s);
    int cur = 0, fill = STAGES - 1;
    const int ns = SPLIT ? nk : (nk + 1) / 2;
    for (int k = 0; k < ns; ++k) {
      wait_and_meet<(STAGES - 2) * 2 * NP>();
      load_stage(k + STAGES - 1, fill);
#pragma unroll
      for (int turn = 0; turn < 2; ++turn) {
        f16x8 fa[2][TM], fb[2][TN];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int two = SPLIT ? x : turn, ks = SPLIT ? turn : x;         // both planes at a k-step, or both k-steps of a K-tile
#pragma unroll
          for (int i = 0; i < TM; ++i) fa[x][i] = __builtin_bit_cast(f16x8, a_kc[cur * STAGE + two * A_VEC + i * 128 + (kc_pos ^ (ks * 4))]);
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            if (B_KC) {
              fb[x][j] = __builtin_bit_cast(f16x8, b_kc[cur * STAGE + two * B_VEC + j * 128 + (kc_pos ^ (ks * 4))]);
            } else {
              const bf16_t* p = b_tr + (cur * STAGE + two * B_VEC) * 8 + ks * 32 * BN + ((wn * TN + j) ^ (l16 >> 2)) * 16;
              const uint2 lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * BN);
              fb[x][j] = __builtin_bit_cast(f16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
            }
          }
        }
#pragma unroll
        for (int pass = 0; pass < (SPLIT ? 3 : 2); ++pass)          // lo hi, hi lo, hi hi; or the k-steps
#pragma unroll
          for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
              acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[pass == 1][j], fa[SPLIT ? pass == 0 : pass][i], acc[j][i], 0, 0, 0);
      }
      cur = cur + 1 == STAGES ? 0 : cur + 1;
      fill = fill + 1 == STAGES ? 0 : fill + 1;
    }
  } else {
    // ---- the K-tiles being loaded; with SPLIT the pairs lo hi, hi lo, hi hi one after the other ----
    const unsigned lds0 = (unsigned)(unsigned long)(__attribute__((address_space(3))) uint4*)smem + (unsigned)wave * 1024u;
    struct Src { unsigned lo, hi, bytes, k, dst; };
    Src as = {0, 0, 0, 0, 0}, bs = as;
    struct At { int k, pass; };                         // K-tile within its pass, and the pass
    auto after = [&](At x) {
      if (!SPLIT) return At{x.k + 1, 0};
      int k, end;          // (on the scalar unit, where the compiler would not keep it)
      asm("s_cmp_eq_u32 %2, %3\n\ts_cselect_b32 %0, 0, %2\n\ts_cselect_b32 %1, 1, 0" : "=&s"(k), "=&s"(end) : "s"(x.k + 1), "s"(nk) : "scc");
      return At{k, x.pass + end};
    };
    // in steps, so that the main loop can deal them out: 0 the k, 1 the base, 2 the size, 3 where to
    auto next_src = [&](Src& x, int step, At at, unsigned per_tile, unsigned long base, unsigned lo_plane, int lo_pass, unsigned bytes, unsigned dst) {
      if (step == 0) {
        x.k = (unsigned)at.k;
        pin(x.k);
      } else if (step == 1) {
        const unsigned plane = SPLIT ? lo_plane & (unsigned)(((at.pass ^ lo_pass) - 1) >> 31) : 0u;
        const unsigned long v = base + (unsigned long)plane + (unsigned long)(x.k * per_tile);
        x.lo = (unsigned)v; x.hi = (unsigned)(v >> 32);
        pin(x.lo); pin(x.hi);
      } else if (step == 2) {
        x.bytes = (bytes - x.k * per_tile) & (unsigned)((SPLIT ? at.pass - 3 : at.k - nk) >> 31);
        pin(x.bytes);
      } else {
        x.dst = dst;
        pin(x.dst);
      }
    };
    const unsigned a_lo = uniform((unsigned)g.a_lo * 2u), b_lo = uniform((unsigned)g.b_lo * 2u);
    auto next_a = [&](int step, At at, int s) { next_src(as, step, at, a_step, a_base, a_lo, 0, a_bytes, lds0 + (unsigned)s * (A_VEC * 16u)); };
    auto next_b = [&](int step, At at, int s) {
      next_src(bs, step, at, b_step, b_base, b_lo, 1, b_bytes, lds0 + NSA * A_VEC * 16u + (unsigned)s * (B_VEC * 16u));
    };
    unsigned lds_dest = 0;
    auto aim = [&](int p) { lds_dest = set_lds_dest((p < NB ? bs.dst + (unsigned)p * 4096u : as.dst + (unsigned)(p - NB) * 4096u)); };
    auto load = [&](int p) {
      if (p < NB) load_to_lds(rsrc_t{bs.lo, bs.hi, bs.bytes, 0x00020000u}, boff[p], lds_dest);
      else load_to_lds(rsrc_t{as.lo, as.hi, as.bytes, 0x00020000u}, aoff[p - NB], lds_dest);
    };

    f16x8 fa[2][TM], fb[2][TN];
    const int kc_pos = lq ^ (l16 >> 1);
    const uint4* const a_kc = smem + (wm * QM + l16) * 8;
    const uint4* const b_kc = smem + NSA * A_VEC + (wn * QN + l16) * 8;
    const bf16_t* const b_tr = reinterpret_cast<const bf16_t*>(smem + NSA * A_VEC) + (lq * 8 + (l16 >> 2)) * BN + (lane & 3) * 4;
    // (sixteen columns u of a k-row stand at position u ^ (k & 3) of their four)
    auto tr_pos = [&](int j) { return ((wn * TN + j) ^ (l16 >> 2)) * 16; };
    auto read_frag_b = [&](int s, int ks, int set, int j) {
      if (B_KC) {
        fb[set][j] = __builtin_bit_cast(f16x8, b_kc[s * B_VEC + j * 128 + (kc_pos ^ (ks * 4))]);
      } else {
        const bf16_t* p = b_tr + s * (B_VEC * 8) + ks * 32 * BN + tr_pos(j);
        const uint2 lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * BN);
        fb[set][j] = __builtin_bit_cast(f16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
      }
    };
    // fragment w of a k-step in the order the MFMAs first need them: B0, A0 .. A(TM-1), B1 .. B(TN-1)
    auto read_frag = [&](int sa, int sb, int ks, int set, int w) {
      if (w == 0) read_frag_b(sb, ks, set, 0);
      else if (w <= TM) fa[set][w - 1] = __builtin_bit_cast(f16x8, a_kc[sa * A_VEC + (w - 1) * 128 + (kc_pos ^ (ks * 4))]);
      else read_frag_b(sb, ks, set, w - TM);
    };

    // ---- schedule, in gaps between the 2 MF MFMAs of a K-tile (gemm_mfma.hip) ----
    constexpr int MF = TM * TN, NF = TM + TN;
    constexpr bool WIDE = MF >= 32;                   // room for a second meeting point
    constexpr int F0 = MF >= 64 ? 2 : 1;              // gaps per fragment
    constexpr int QF = NF * F0 + 8 < MF ? NF * F0 + 8 : MF;          // K-tile t is in registers: its slots may be overwritten
    constexpr int QL = WIDE ? 2 * MF - NF * F0 - (MF >= 64 ? 12 : 6) : QF;    // K-tile t+1 is in LDS: its first fragments may be read
    constexpr int DG_ALL = 2 * MF / NP, DG_B = (2 * MF - QF) / NB, DG = DG_ALL < DG_B ? DG_ALL : DG_B;      // gaps per load
    constexpr int R0 = QL < MF ? MF : QL;
    constexpr int F1 = (2 * MF - R0) / NF < 4 ? (2 * MF - R0) / NF : 4;
    constexpr int SS = MF >= 32 ? 2 : 1;              // gaps per step of the scalars
    static_assert(DG >= 1 && F1 >= 1 && QF + NB * DG <= 2 * MF && R0 + NF * F1 <= 2 * MF && QF >= 4 * SS && NB * DG >= 4 * SS, "more fragments or loads than MFMA gaps");
    constexpr int LATE = QF + NP * DG > 2 * MF ? (QF + NP * DG - 2 * MF + DG - 1) / DG : 0;      // loads of an iteration that the next one issues
    constexpr int LOADED = QL > QF ? ((QL - QF) / DG < NP ? (QL - QF) / DG : NP) : 0;
    constexpr int AFTER_A = (NSA - 2) * NP, AFTER_B = NA + (NSB - 2) * NP, AHEAD = AFTER_A < AFTER_B ? AFTER_A : AFTER_B;
    static_assert(AHEAD + NP < 64, "the counter of outstanding loads");
    constexpr int FAR = NSA > NSB ? NSA : NSB;
    At at_a = {0, 0}, at_b = {0, 0};                    // to be loaded next
#pragma unroll
    for (int u = -FAR; u < 0; ++u) {
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        if (u + NSB >= 0) next_b(st, at_b, u + NSB);
        if (u + NSA >= 0) next_a(st, at_a, u + NSA);
      }
      if (u + NSB >= 0) at_b = after(at_b);
      if (u + NSA >= 0) at_a = after(at_a);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if ((p < NB ? u + NSB : u + NSA) < 0 || (u == -1 && p >= NP - LATE)) continue;
        aim(p); one_instruction(); load(p);
      }
    }
    wait_and_meet<AHEAD + NP - LATE>();
#pragma unroll
    for (int w = 0; w < NF; ++w) read_frag(0, 0, 0, 0, w);
    int t = 0, sa = 0, sb = 0;
    do {
      const int sa1 = sa + 1 == NSA ? 0 : sa + 1, sb1 = sb + 1 == NSB ? 0 : sb + 1;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < 2 * MF; ++q) {
        const int ks = q / MF, j = (q % MF) / TM, i = q % TM;
        if (q == QF) {
          wait_and_meet<(WIDE ? 63 : AHEAD)>();
          __builtin_amdgcn_sched_barrier(0);
        }
        if (WIDE && q == QL) {
          wait_and_meet<AHEAD + LOADED>();
          __builtin_amdgcn_sched_barrier(0);
        }
        acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[ks][j], fa[ks][i], acc[j][i], 0, 0, 0);
        // (a use in this gap: the product has no side effects, and the compiler gathers those of many gaps in one place else.  No instruction)
        if (C::MINB == 1) asm volatile("" :: "a"(acc[j][i]));
        else asm volatile("" :: "v"(acc[j][i]));
        if (q < MF && q % F0 == 0 && q / F0 < NF) read_frag(sa, sb, 1, 1, q / F0);
        if (q >= R0 && (q - R0) % F1 == 0 && (q - R0) / F1 < NF) read_frag(sa1, sb1, 0, 0, (q - R0) / F1);
        if (q >= QF - 4 * SS && q < QF && (QF - 1 - q) % SS == 0) next_b((q - (QF - 4 * SS)) / SS, at_b, sb);
        if (q >= QF && q < QF + 4 * SS && (q - QF) % SS == 0) next_a((q - QF) / SS, at_a, sa);
        {
          const int at = q >= QF ? q - QF : q - QF + 2 * MF, p = at / DG;
          if (p < NP && (q >= QF || p >= NP - LATE)) {
            // (a gap ahead of the load, but in the same iteration)
            const bool alone = DG == 1 || (q == 0 && at % DG == DG - 1);
            if (alone || (at % DG == DG - 2 && q < 2 * MF - 1)) aim(p);
            if (alone) one_instruction();
            if (at % DG == DG - 1) load(p);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      sa = sa1; sb = sb1;
      at_a = after(at_a); at_b = after(at_b);
      ++t;
    } while (t < nsteps);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // no load may still write the LDS that the slabs use

  // ---- epilogue: 32 rows of the wavefront's quarter at a time, turned through LDS so that lanes lie along the columns ----
  const float f1 = g.factor ? g.factor[mat] : 1.f, f = EPI == kGram ? f1 * f1 : f1;
  constexpr int CPR = QN / 8, RPI = 64 / CPR, NST = 32 / RPI;         // lanes per row (eight columns each), rows at a time
  const int e_row = m0 + wm * QM + lane / CPR, e_col = n0 + wn * QN + lane % CPR * 8;
  if constexpr (EPI == kPart) {
    float* const out = g.part + ((long)blockIdx.y * g.n + mat) * g.M * g.M + (long)(m0 + wm * QM + l16) * g.M + n0 + wn * QN + lq * 4;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int i = 0; i < TM; ++i) *reinterpret_cast<f32x4*>(out + (long)(i * 16) * g.M + j * 16) = acc[j][i];
  } else if constexpr (EPI == kLast || EPI == kUpdate) {
    // The result goes to the caller's matrix, turned if it is tall: W columns of a row of it to a lane.  kUpdate: w <- keep w - rate o in 32 bits, and
    // its copy in the expert store; the weights of 32 rows are requested ahead of the stores of those before.  Tiles inside the
    // matrix (WHOLE) have no guards, behind which every load would be waited for by itself: 16 of 1024 x 2048, the last step 132 -> 107 us, 8 of
    // 4864 x 3584 1152 -> 990.  (On 256-wide tiles the weights and results of 32 rows, beside 256 accumulators, spill 26 registers of bf16 storage, 31 of fp32.)
    const float alpha = g.alpha * f;
    float* const slab = reinterpret_cast<float*>(smem) + wave * C::SLAB;
    constexpr int W = EPI == kUpdate ? 4 : 16 / (int)sizeof(T);
    constexpr int LPR = QN / W, RUNS = 32 / W;       // lanes per row; turned: runs of W rows, which are columns of the result
    constexpr int STEPS = QN * 32 / W / 64;
    const long first = (long)mat * g.rows * g.cols;
    __syncthreads();
    auto finish = [&](auto whole_c, auto tall_c) {
      constexpr bool WHOLE = decltype(whole_c)::value, TALL = decltype(tall_c)::value;
      auto row_of = [&](int i, int st) { return TALL ? n0 + wn * QN + st * (64 / RUNS) + lane / RUNS : m0 + wm * QM + i * 32 + st * (64 / LPR) + lane / LPR; };
      auto col_of = [&](int i) { return TALL ? m0 + wm * QM + i * 32 + lane % RUNS * W : n0 + wn * QN + lane % LPR * W; };
      auto left_of = [&](int i, int st) { return WHOLE ? W : row_of(i, st) < g.rows ? g.cols - col_of(i) : 0; };
      auto at = [&](int i, int st) { return left_of(i, st) > 0 ? (long)row_of(i, st) * g.cols + col_of(i) : 0l; };
      T* const param = static_cast<T*>(g.param) + (EPI == kUpdate ? g.param_at[mat] : 0l);
      float* const weight = g.master ? g.master + first : reinterpret_cast<float*>(param);
      Unit<float, 4> w[EPI == kUpdate ? STEPS : 1];
      auto load_w = [&](int i) {
        if constexpr (EPI == kUpdate) {
#pragma unroll
          for (int st = 0; st < STEPS; ++st) w[st].load(weight + at(i, st), left_of(i, st));
        }
      };
      load_w(0);
#pragma unroll
      for (int i = 0; i < QM / 32; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int ii = 0; ii < 2; ++ii) {
            f32x4 v = acc[j][2 * i + ii];
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] *= alpha;
            *reinterpret_cast<f32x4*>(slab + (ii * 16 + l16) * PITCH + j * 16 + lq * 4) = v;
          }
        wave_lds_order();
        float o[STEPS][W];
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          if (TALL) {
#pragma unroll
            for (int e = 0; e < W; ++e) o[st][e] = slab[(lane % RUNS * W + e) * PITCH + st * (64 / RUNS) + lane / RUNS];
          } else {
#pragma unroll
            for (int h = 0; h < W / 4; ++h) {
              const f32x4 q = *reinterpret_cast<const f32x4*>(slab + (st * (64 / LPR) + lane / LPR) * PITCH + lane % LPR * W + 4 * h);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[st][4 * h + e] = q[e];
            }
          }
          if constexpr (EPI == kUpdate) {
            float x[W];
            w[st].get(x);
#pragma unroll
            for (int e = 0; e < W; ++e) o[st][e] = fmaf(-g.rate, o[st][e], g.keep * x[e]);
          }
        }
        if (i + 1 < QM / 32) load_w(i + 1);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          if constexpr (EPI == kUpdate) {
            Unit<float, W> u;
            u.set(o[st]);
            u.store(weight + at(i, st), left_of(i, st));
            if (g.master) {
              Unit<T, W> c;
              c.set(o[st]);
              c.store(param + at(i, st), left_of(i, st));
            }
          } else {
            Unit<T, W> u;
            u.set(o[st]);
            u.store(static_cast<T*>(g.out) + first + at(i, st), left_of(i, st));
          }
        }
        wave_lds_order();
      }
    };
    const bool whole = g.tall ? m0 + BM <= g.cols && n0 + BN <= g.rows : m0 + BM <= g.rows && n0 + BN <= g.cols;
    if (whole) g.tall ? finish(std::true_type{}, std::true_type{}) : finish(std::true_type{}, std::false_type{});
    else g.tall ? finish(std::false_type{}, std::true_type{}) : finish(std::false_type{}, std::false_type{});
  } else {
    // All of it on fp16 in LDS, a slab for each plane of what is read beside the product (kPoly: G, kStep: X and its remainder) and of the result.  The
    // arithmetic is done where the products are, four columns to a lane, and rounded there.  Loads and stores go through buffer resources that end
    // with the matrix: a lane beyond it asks for nothing, and there are no branches.
    constexpr int PITCH16 = C::PITCH16, SLAB16 = C::SLAB16;
    char* const slab = reinterpret_cast<char*>(smem) + wave * (4 * SLAB16);
    const unsigned plane_bytes = uniform((unsigned)g.M * (unsigned)g.ldc * 2u), row_bytes = (unsigned)g.ldc * 2u;
    const __amdgpu_buffer_rsrc_t in_rs[2] = {tile_rsrc(base_of(g.E, mat * g.e_ms), plane_bytes), tile_rsrc(base_of(g.E, mat * g.e_ms + g.e_lo), plane_bytes)};
    const __amdgpu_buffer_rsrc_t out_rs[2] = {tile_rsrc(base_of(g.C, mat * g.c_ms), plane_bytes), tile_rsrc(base_of(g.C, mat * g.c_ms + g.c_lo), plane_bytes)};
    // (a matrix has less than 2^30 bytes, and what is added below stays far from 2^31)
    const unsigned off0 = e_col < g.N ? (unsigned)e_row * row_bytes + (unsigned)e_col * 2u : 1u << 31;
    auto off = [&](int i, int st) { return off0 + (unsigned)(i * 32 + st * RPI) * row_bytes; };
    rsrc_t in0[IN > 0 ? NST : 1], in1[IN > 1 ? NST : 1];
    auto load_in = [&](int i) {
#pragma unroll
      for (int st = 0; st < NST; ++st) {
        if constexpr (IN > 0) in0[st] = __builtin_amdgcn_raw_buffer_load_b128(in_rs[0], (int)off(i, st), 0, 0);
        if constexpr (IN > 1) in1[st] = __builtin_amdgcn_raw_buffer_load_b128(in_rs[1], (int)off(i, st), 0, 0);
      }
    };
    load_in(0);
    const float alpha = g.alpha * f, beta = g.beta * f;
    constexpr bool KEEPS = EPI == kPoly && OUT == 1, TAKES = EPI == kStep && IN > 0;        // the rest of P's diagonal, which kStep multiplies X with
    const __amdgpu_buffer_rsrc_t rest_rs = tile_rsrc(base_of(reinterpret_cast<const f16*>(g.rest), 2l * mat * g.M), KEEPS || TAKES ? (unsigned)g.M * 4u : 0u);
    const unsigned rest_row = (unsigned)(m0 + wm * QM + l16) * 4u;
    float rest[TAKES ? TM : 1];
    if constexpr (TAKES) {
#pragma unroll
      for (int i = 0; i < TM; ++i) rest[i] = load4(rest_rs, rest_row + (unsigned)i * 64u) * alpha;
    }
    // (the diagonal passes through the MFMA tiles i, j with j - i = tile_d, in a lane's element r through r = in_d)
    const int tile_d = (m0 + wm * QM - n0 - wn * QN) / 16, in_d = l16 - lq * 4;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < QM / 32; ++i) {
      if constexpr (IN > 0) {
#pragma unroll
        for (int st = 0; st < NST; ++st) {
          char* const p = slab + (st * RPI + lane / CPR) * PITCH16 + lane % CPR * 16;
          *reinterpret_cast<rsrc_t*>(p) = in0[st];
          if constexpr (IN > 1) *reinterpret_cast<rsrc_t*>(p + SLAB16) = in1[st];
        }
        wave_lds_order();
        if (i + 1 < QM / 32) load_in(i + 1);          // ahead of the stores, behind which they would wait
      }
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
          char* const p = slab + (ii * 16 + l16) * PITCH16 + (j * 16 + lq * 4) * 2;
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = acc[j][2 * i + ii][r] * alpha;
          if constexpr (IN > 0) {
            const f16x4 x = *reinterpret_cast<const f16x4*>(p);
            const float times = TAKES ? rest[TAKES ? 2 * i + ii : 0] : beta;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = fmaf((float)x[r], times, v[r]);
          }
          if constexpr (IN > 1) {
            const f16x4 x = *reinterpret_cast<const f16x4*>(p + SLAB16);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = fmaf((float)x[r], beta, v[r]);
          }
          const bool diagonal = EPI == kPoly && j - 2 * i - ii == tile_d;
          if (diagonal) {
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] += in_d == r ? g.diagonal : 0.f;
          }
          // (pinned in 32 bits for every tile alike: see split)
          f16 hi[4], lo[4];
          split<4>(v, hi, lo);
          if constexpr (OUT > 1) *reinterpret_cast<f16x4*>(p + (IN + 1) * SLAB16) = f16x4{lo[0], lo[1], lo[2], lo[3]};
          if (KEEPS && diagonal) {
            float lost = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) lost = in_d == r ? v[r] - (float)hi[r] : lost;
            store4(rest_rs, (unsigned)in_d < 4u ? rest_row + (unsigned)(2 * i + ii) * 64u : 1u << 31, lost);
          }
          *reinterpret_cast<f16x4*>(p + IN * SLAB16) = f16x4{hi[0], hi[1], hi[2], hi[3]};
        }
      wave_lds_order();
#pragma unroll
      for (int two = 0; two < OUT; ++two) {
        const char* const from = slab + (IN + two) * SLAB16;
#pragma unroll
        for (int st = 0; st < NST; ++st)
          store16(out_rs[two], off(i, st), *reinterpret_cast<const rsrc_t*>(from + (st * RPI + lane / CPR) * PITCH16 + lane % CPR * 16));
        if (SYM && mi != ni) {
          // the mirror image through the transposing read: sixteen columns by four runs of eight rows
          const int col = m0 + wm * QM + i * 32 + lq * 8;
          const unsigned at = col < g.M ? (unsigned)(n0 + wn * QN + l16) * row_bytes + (unsigned)col * 2u : 1u << 31;
#pragma unroll
          for (int st = 0; st < TN; ++st) {
            const bf16_t* const p = reinterpret_cast<const bf16_t*>(from + (lq * 8 + (l16 >> 2)) * PITCH16 + (st * 16 + (lane & 3) * 4) * 2);
            const uint2 x = lds_read_tr(p), y = lds_read_tr(p + 4 * (PITCH16 / 2));
            store16(out_rs[two], at + (unsigned)(st * 16) * row_bytes, rsrc_t{x.x, x.y, y.x, y.y});
          }
        }
      }
      wave_lds_order();
    }
  }
}

// Every XCD (workgroups go round the eight) gets one contiguous range of the tiles.  A last round of tiles that leaves half of the CUs or more
// without one runs on halves of them (CH, plan::square_cut), dealt out by themselves: 8 of 3584 x 4864, 840 tiles of G 498 -> 465 us, of P
// 387 -> 366; one of 1280 x 1536, 120 tiles of the step 13.9 -> 11.4; 4 of 512 x 256, 40, 40 and 128 tiles of 64,
// fp32 8.2, 6.2, 6.2 -> 6.4, 4.9, 5.6, the call 106 -> 88, bf16 5.2, 4.5, 4.4 -> 4.4, 3.9, 3.9.
template <Epi EPI, bool B_KC, bool SPLIT, int IN, int OUT, typename T, typename C, typename CH>
__global__ __launch_bounds__(256, C::MINB) void ns_gemm_kernel(const NsArgs g) {
  __shared__ uint4 smem[C::UNITS > CH::UNITS ? C::UNITS : CH::UNITS];
  constexpr bool SYM = EPI == kGram || EPI == kPoly || EPI == kPart;
  const unsigned mt = (unsigned)cdiv(g.M, C::BN), nt = (unsigned)cdiv(g.N, C::BN), per = SYM ? mt * (mt + 1) / 2 : mt * nt;
  const unsigned total = per * (unsigned)g.n, cut = C::BM != CH::BM ? (unsigned)plan::square_cut(C::BM, total) : 0, whole = total - cut;
  const unsigned first_half = (whole + kXcds - 1) / kXcds * kXcds;
  const bool halves = C::BM != CH::BM && blockIdx.x >= first_half;
  const unsigned block = halves ? blockIdx.x - first_half : blockIdx.x, count = halves ? 2 * cut : whole;
  const unsigned per_xcd = (count + kXcds - 1) / kXcds, slot = block / kXcds, at = (block % kXcds) * per_xcd + slot;
  if (slot >= per_xcd || at >= count) return;
  const unsigned tile = halves ? whole + at / 2 : at;
  const int mat = (int)uniform(tile / per);
  const unsigned in = tile - (unsigned)mat * per;
  if constexpr (C::BM != CH::BM) {
    if (halves) {
      ns_tile<EPI, B_KC, SPLIT, IN, OUT, T, CH>(g, smem, mat, in, (int)(at & 1));
      return;
    }
  }
  if constexpr (EPI != kPart) ns_tile<EPI, B_KC, SPLIT, IN, OUT, T, C>(g, smem, mat, in, 0);      // (parts are of few tiles: halves)
}

// kGram from its parts, added in their order: four columns of a row to a thread, eight parts requested at once (beyond the last one through the
// buffer's end: zeros).  Below the diagonal's tiles the mirror image is written too.
template <int OUT>
__global__ __launch_bounds__(256) void ns_join_kernel(const NsArgs g, int parts) {
  const int at = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4, size = g.M * g.M, mat = blockIdx.y;
  const int r = at / g.M, c = at - r * g.M;
  if (at >= size || r / 64 < c / 64) return;
  const unsigned step = (unsigned)(g.n * size) * 4u;
  const __amdgpu_buffer_rsrc_t rs = tile_rsrc(reinterpret_cast<unsigned long>(g.part + (long)mat * size), (unsigned)(parts * g.n - mat) * (unsigned)size * 4u);
  float v[4] = {};
  for (int first = 0; first < parts; first += 8) {
    f32x4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)((unsigned)at * 4u + (unsigned)(first + k) * step), 0, 0));
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[k][e];
  }
  const float f = g.factor ? g.factor[mat] : 1.f, alpha = g.alpha * (f * f);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= alpha;
  f16 plane[2][4];
  split<4>(v, plane[0], plane[1]);
#pragma unroll
  for (int two = 0; two < OUT; ++two) {
    f16* const out = g.C + mat * g.c_ms + two * g.c_lo;
    *reinterpret_cast<f16x4*>(out + (long)r * g.ldc + c) = f16x4{plane[two][0], plane[two][1], plane[two][2], plane[two][3]};
    if (r / 64 > c / 64)
#pragma unroll
      for (int e = 0; e < 4; ++e) out[(long)(c + e) * g.ldc + r] = plane[two][e];
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
// Momentum of 16 matrices of 1024 x 2048: 70 us for 403 MB, 5.7 TB/s; of 8 of 4864 x 3584 310 us, 5.4.
template <typename T, bool MUON, bool ONCE>
__global__ __launch_bounds__(256) void ns_sum_kernel(const PrepArgs a) {
  __shared__ double red[4];
  constexpr int W = MUON ? 4 : 16 / (int)sizeof(T);
  const long elems = (long)a.rows * a.cols, first = (long)blockIdx.y * elems;
  double s = 0;
#pragma unroll 2
  for (long u = (long)blockIdx.x * 256 + threadIdx.x; u * W < elems; u += (long)a.blocks * 256) {
    const long at = first + u * W, rest = elems - u * W;
    const int left = rest < W ? (int)rest : W;
    float v[W];
    if constexpr (MUON) {
      Unit<float> m, g;
      float mf[W], gf[W];
      m.template load<ONCE>(a.m + at, left);
      g.template load<ONCE>(a.grad + at, left);
      m.get(mf);
      g.get(gf);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float ge = gf[e] * a.grad_scale;
        mf[e] = fmaf(a.beta, mf[e], ge);
        v[e] = a.nesterov ? fmaf(a.beta, mf[e], ge) : mf[e];
      }
      m.set(mf);
      m.template store<ONCE>(a.m + at, left);
    } else {
      Unit<T> x;
      x.template load<ONCE>(static_cast<const T*>(a.src) + at, left);
      x.get(v);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) s += (double)v[e] * (double)v[e];          // (beyond the end: zeros)
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.part[(long)blockIdx.y * a.blocks + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// A 64 x 64 tile of X: U 2^e, so that a bf16 matrix is held exactly; what the power of two leaves of 1 / |U| is the factor of
// the first step's products.  A matrix of zeros stays one; infinities and NaN make all of it NaN.
// It reads again what ns_sum_kernel read, since the norm is known only now: 16 of 1024 x 2048, 72 us for 403 MB; 8 of 4864 x 3584, 208 us
// for 1.12 GB, 5.4 TB/s.  (Going over the matrices from the last one back, for what the Infinity Cache still holds, changed nothing.)
template <typename T, bool MUON, bool ONCE>
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
  // X's tile, eight columns to a thread; a tile inside the matrix without guards
  auto stored = [&](int r, int c, const float* v) {
    uint4 hi, lo;
    split8(v, hi, lo);
    f16* const p = a.X + mat * a.ms + (long)(l0 + r) * a.ld + h0 + c;
    *reinterpret_cast<uint4*>(p) = hi;
    if (a.lo_plane != 0) *reinterpret_cast<uint4*>(p + a.lo_plane) = lo;
  };
  auto tile = [&](auto whole_c) {
    constexpr bool WHOLE = decltype(whole_c)::value;
    // everything is requested before anything is used
    constexpr int N = MUON ? 2 : (int)sizeof(T) / 2, W = 8 / N;          // 16-byte units of eight columns
    using S = std::conditional_t<MUON, float, T>;
    Unit<S> x[2][N], grad[2][MUON ? N : 1];
    auto load = [&](const S* from, Unit<S> (&u)[2][N]) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int row = (a.tall ? h0 : l0) + half * 32 + tid / 8, col = (a.tall ? l0 : h0) + tid % 8 * 8;       // of the caller's matrix
        const int left = WHOLE ? 8 : row < a.rows ? a.cols - col : 0;
        const S* const p = from + first + (left > 0 ? (long)row * a.cols + col : 0);
#pragma unroll
        for (int h = 0; h < N; ++h) u[half][h].template load<ONCE>(p + W * h, left - W * h);
      }
    };
    float v[2][8];
    if constexpr (MUON) {
      load(a.m, x);
      if (a.nesterov) load(a.grad, grad);
    } else {
      load(static_cast<const T*>(a.src), x);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int h = 0; h < N; ++h) {
        x[half][h].get(v[half] + W * h);
        if constexpr (MUON) {
          if (a.nesterov) {
            float gf[W];
            grad[half][h].get(gf);
#pragma unroll
            for (int e = 0; e < W; ++e) v[half][W * h + e] = fmaf(a.beta, v[half][W * h + e], gf[e] * a.grad_scale);
          }
        }
      }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = half * 32 + tid / 8, c = tid % 8 * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[half][e] = ldexpf(v[half][e], shift);
      if (!a.tall) {
        stored(r, c, v[half]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn[r][c + e] = v[half][e];
      }
    }
  };
  const bool whole = a.tall ? h0 + 64 <= a.rows && l0 + 64 <= a.cols : l0 + 64 <= a.rows && h0 + 64 <= a.cols;
  if (whole) tile(std::true_type{});
  else tile(std::false_type{});
  if (!a.tall) return;
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r = half * 32 + tid / 8, c = tid % 8 * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = turn[c + e][r];
    stored(r, c, v);
  }
}

struct Buffers {
  int lo, hi, lo_p, hi_p;
  bool pairs;                         // every operand with its remainder
  int planes;                         // of G and P; X has two
  int sum_blocks, gram_parts;
  size_t part, factor, x[2], g, p, rest, gram, total;
};

Buffers buffers(int n, int rows, int cols, int dtype) {
  Buffers b;
  b.lo = rows < cols ? rows : cols; b.hi = rows < cols ? cols : rows;
  b.lo_p = (int)round_up(b.lo, kPad); b.hi_p = (int)round_up(b.hi, kPad);
  b.pairs = dtype == SPES_F32 || b.lo <= kFewRows;
  b.planes = b.pairs ? 2 : 1;
  const long units = ((long)rows * cols + 7) / 8;
  b.sum_blocks = (int)(units / 1024 < 1 ? 1 : units / 1024 > kSumBlocks ? kSumBlocks : units / 1024);
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += round_up(bytes, 256); return o; };
  b.part = take((size_t)n * kSumBlocks * 8);
  b.factor = take((size_t)n * 4);
  for (int i = 0; i < 2; ++i) b.x[i] = take((size_t)n * 2 * b.lo_p * b.hi_p * 2);
  b.g = take((size_t)n * b.planes * b.lo_p * b.lo_p * 2);
  b.p = take((size_t)n * b.planes * b.lo_p * b.lo_p * 2);
  b.rest = take(b.pairs ? 0 : (size_t)n * b.lo_p * 4);
  b.gram_parts = plan::gram_parts(b.lo_p, b.hi_p, n, b.pairs);
  b.gram = take(b.gram_parts > 1 ? (size_t)b.gram_parts * n * b.lo_p * b.lo_p * 4 : 0);
  b.total = off;
  return b;
}

template <Epi EPI, bool B_KC, bool SPLIT, int IN, int OUT, typename T, typename C, typename CH = C>
int launch_tiles(const NsArgs& g, hipStream_t s, int parts = 1) {
  const long mt = cdiv(g.M, C::BN), nt = cdiv(g.N, C::BN);
  const long total = (EPI == kGram || EPI == kPoly || EPI == kPart ? mt * (mt + 1) / 2 : mt * nt) * g.n, cut = C::BM != CH::BM ? plan::square_cut(C::BM, total) : 0;
  const long blocks = (long)round_up(total - cut, kXcds) + (long)round_up(2 * cut, kXcds);
  hipLaunchKernelGGL((ns_gemm_kernel<EPI, B_KC, SPLIT, IN, OUT, T, C, CH>), dim3((unsigned)blocks, (unsigned)parts), dim3(256), 0, s, g);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}
// of: matrices of the whole product, where a launch has only some of them.  One tile for all: in pairs the order of the sums goes by it.
template <Epi EPI, bool B_KC, bool SPLIT, int IN, int OUT, typename T>
int launch_product(const NsArgs& g, int of, hipStream_t s) {
  const int side = plan::square_tile(g.M, g.N, of, EPI == kGram || EPI == kPoly);
  if (side == Tile::BM) return launch_tiles<EPI, B_KC, SPLIT, IN, OUT, T, Tile, TileHalf>(g, s);
  if (side == TileSmall::BM) return launch_tiles<EPI, B_KC, SPLIT, IN, OUT, T, TileSmall, TileSmallHalf>(g, s);
  return launch_tiles<EPI, B_KC, SPLIT, IN, OUT, T, std::conditional_t<SPLIT, TileTinyPairs, TileTiny>, std::conditional_t<SPLIT, TileTinyPairsHalf, TileTinyHalf>>(g, s);
}
// a last step; matrices of few rows in bf16 storage, the only ones on pairs there, have few tiles
template <Epi EPI, typename T>
int launch_end(bool pairs, const NsArgs& g, int of, hipStream_t s) {
  if constexpr (sizeof(T) == 4) return launch_product<EPI, false, true, 0, 0, T>(g, of, s);
  else return pairs ? launch_tiles<EPI, false, true, 0, 0, T, TileTinyPairs, TileTinyPairsHalf>(g, s) : launch_product<EPI, false, false, 0, 0, T>(g, of, s);
}

template <bool SPLIT, int OUT>
int launch_gram_parts(const NsArgs& g, int parts, hipStream_t s) {
  const int rc = launch_tiles<kPart, true, SPLIT, 0, 0, float, std::conditional_t<SPLIT, TileTinyPairs, TileTiny>, std::conditional_t<SPLIT, TileTinyPairsHalf, TileTinyHalf>>(g, s, parts);
  if (rc != SPES_OK) return rc;
  hipLaunchKernelGGL((ns_join_kernel<OUT>), dim3((unsigned)(g.M * g.M / 1024), (unsigned)g.n), dim3(256), 0, s, g, parts);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

template <typename T>
int run(const Buffers& b, int steps, const float* coef, bool exact_start, bool muon, PrepArgs a, NsArgs end, const long* param_at, char* scratch, hipStream_t s) {
  const long xs = (long)b.lo_p * b.hi_p, gs = (long)b.lo_p * b.lo_p;
  f16* X[2] = {reinterpret_cast<f16*>(scratch + b.x[0]), reinterpret_cast<f16*>(scratch + b.x[1])};
  f16 *G = reinterpret_cast<f16*>(scratch + b.g), *P = reinterpret_cast<f16*>(scratch + b.p);
  a.part = reinterpret_cast<double*>(scratch + b.part); a.blocks = b.sum_blocks;
  a.factor = reinterpret_cast<float*>(scratch + b.factor);
  a.X = X[0]; a.ms = 2 * xs; a.lo = b.lo; a.hi = b.hi; a.ld = b.hi_p; a.lo_p = b.lo_p; a.tall = a.rows > a.cols;
  const bool first_lo = b.pairs || !exact_start;
  a.lo_plane = first_lo ? xs : 0;
  const dim3 sums((unsigned)b.sum_blocks, (unsigned)a.n), tiles((unsigned)(b.lo_p / 64 * (b.hi_p / 64)), (unsigned)a.n);
  auto prepare = [&](auto of_muon, auto streaming) {
    constexpr bool MUON = decltype(of_muon)::value, ONCE = decltype(streaming)::value;
    hipLaunchKernelGGL((ns_sum_kernel<T, MUON, ONCE>), sums, dim3(256), 0, s, a);
    hipLaunchKernelGGL((ns_scale_kernel<T, MUON, ONCE>), tiles, dim3(256), 0, s, a);
  };
  // The non-temporal hint where the Infinity Cache does not hold gradient and momentum: 8 matrices of 4864 x 3584, scaling 231 -> 193 us; 16 of
  // 1024 x 2048, which just fit, 74 -> 87 with it.
  const bool once = (long)a.n * a.rows * a.cols * (muon ? 8 : (long)sizeof(T)) > (256l << 20);
  if (muon) once ? prepare(std::true_type{}, std::true_type{}) : prepare(std::true_type{}, std::false_type{});
  else once ? prepare(std::false_type{}, std::true_type{}) : prepare(std::false_type{}, std::false_type{});
  if (hipGetLastError() != hipSuccess) return SPES_EHIP;
  NsArgs g = end;
  g.n = a.n;
  for (int i = 0; i < steps; ++i) {
    const bool last = i + 1 == steps, x_lo = i > 0 || first_lo, next_lo = b.pairs || i + 2 < steps;         // X's remainder; the last step has none
    f16 *x = X[i & 1], *y = X[(i + 1) & 1];
    const float* factor = i == 0 ? a.factor : nullptr;
    NsArgs q = g;
    q.A = q.B = x; q.a_ms = q.b_ms = 2 * xs; q.a_lo = q.b_lo = xs; q.lda = q.ldb = b.hi_p;
    q.M = q.N = b.lo_p; q.K = b.hi_p;
    q.C = G; q.c_ms = b.planes * gs; q.c_lo = b.pairs ? gs : 0; q.ldc = b.lo_p;
    q.alpha = ldexpf(1.f, kGBits - 2 * kXBits); q.beta = 0.f; q.factor = factor;
    q.E = G; q.e_ms = 0; q.e_lo = 0; q.lde = b.lo_p;
    int rc;
    if (b.gram_parts > 1) {
      q.part = reinterpret_cast<float*>(scratch + b.gram);
      q.k_tiles = cdiv(b.hi_p / 64, b.gram_parts);
      rc = b.pairs ? launch_gram_parts<true, 2>(q, b.gram_parts, s) : launch_gram_parts<false, 1>(q, b.gram_parts, s);
    } else {
      rc = b.pairs ? launch_product<kGram, true, true, 0, 2, float>(q, a.n, s) : launch_product<kGram, true, false, 0, 1, float>(q, a.n, s);
    }
    if (rc != SPES_OK) return rc;
    q.A = q.B = q.E = G; q.a_ms = q.b_ms = q.e_ms = b.planes * gs; q.a_lo = q.b_lo = gs; q.e_lo = b.pairs ? gs : 0; q.lda = q.ldb = b.lo_p;
    q.K = b.lo_p; q.C = P;
    q.alpha = coef[2] * ldexpf(1.f, -kGBits); q.beta = coef[1]; q.factor = nullptr;
    q.diagonal = ldexpf(coef[0], kGBits); q.rest = reinterpret_cast<float*>(scratch + b.rest);
    rc = b.pairs ? launch_product<kPoly, true, true, 2, 2, float>(q, a.n, s) : launch_product<kPoly, true, false, 1, 1, float>(q, a.n, s);
    if (rc != SPES_OK) return rc;
    q.A = P; q.B = x; q.b_ms = 2 * xs; q.b_lo = xs; q.ldb = b.hi_p;
    q.E = x; q.e_ms = 2 * xs; q.e_lo = xs; q.lde = b.hi_p;
    q.M = b.lo_p; q.N = b.hi_p; q.K = b.lo_p;
    q.C = y; q.c_ms = 2 * xs; q.c_lo = next_lo ? xs : 0; q.ldc = b.hi_p;
    q.alpha = ldexpf(1.f, -kGBits); q.beta = coef[0]; q.factor = factor;
    if (!last) {
      rc = b.pairs           ? launch_product<kStep, false, true, 0, 2, float>(q, a.n, s)
           : x_lo && next_lo ? launch_product<kStep, false, false, 2, 2, float>(q, a.n, s)
           : x_lo            ? launch_product<kStep, false, false, 2, 1, float>(q, a.n, s)
           : next_lo         ? launch_product<kStep, false, false, 1, 2, float>(q, a.n, s)
                             : launch_product<kStep, false, false, 1, 1, float>(q, a.n, s);
      if (rc != SPES_OK) return rc;
      continue;
    }
    // out of the scaled form
    q.alpha = ldexpf(q.alpha, -kXBits);
    if (!muon) return launch_end<kLast, T>(b.pairs, q, a.n, s);
    for (int first = 0; first < a.n; first += kSlots) {
      NsArgs u = q;
      u.n = a.n - first < kSlots ? a.n - first : kSlots;
      u.A += first * u.a_ms; u.B += first * u.b_ms; u.E += first * u.e_ms;
      if (u.factor) u.factor += first;
      if (u.master) u.master += (long)first * a.rows * a.cols;
      for (int k = 0; k < u.n; ++k) u.param_at[k] = param_at[first + k];
      rc = launch_end<kUpdate, T>(b.pairs, u, a.n, s);
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
