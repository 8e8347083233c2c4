// Attention over sequences of unequal length, forward.  Per query and head, over the keys that the query sees,
//      s = scale q k^T      m = max s      l = sum exp(s - m)      o = sum exp(s - m) v / l      lse = m + ln l
// in one pass over the keys: running maximum and sum per row, scores and probabilities never leave the registers.
#include <algorithm>

#include "attention.h"

namespace spes {
namespace {

using namespace attn;

struct FwdArgs {
  AttnShape a;
  const void *q, *k, *v;
  void* o;
  float *lse, *part_o, *part_lse;
  int parts, per;       // parts that a tile's keys are cut into at most, and steps of keys to a part (for few rows: see FewPlan)
  float c;              // scale log2 e: exponentials are of base two
};

constexpr int kFewRows = 32, kFewStep = 32, kMaxParts = 64;
constexpr float kLazy = 8.f;      // the running maximum is raised, and what has been summed is scaled, once a score passes it by 2^8

// Steps [from, to) of the n that part `part` has; false for a part that there is no work for, but for the first one
__device__ __forceinline__ bool part_of(const FwdArgs& g, int part, int n, int& from, int& to) {
  from = min((int)min((long)part * g.per, (long)n), n);
  to = part == g.parts - 1 ? n : min((int)min((long)(part + 1) * g.per, (long)n), n);
  return part == 0 || from < n;
}
__device__ __forceinline__ int parts_used(const FwdArgs& g, int n) { return min(max(cdiv(n, g.per), 1), g.parts); }

// A row's result: part of one, or the whole.  acc: DB tiles of O^T, the lane's column is the row
template <typename T, int DB>
__device__ __forceinline__ void put_row(const FwdArgs& g, int part, long token, int head, int half, const f32x16 (&acc)[DB], float sum, float m) {
  const AttnShape& a = g.a;
  const float inv = sum == 0.f ? 0.f : 1.f / sum, lse = (m + log2f(sum)) * kLn2;
  const bool whole = g.parts == 1;
  float* const po = g.part_o + (((long)part * a.q_rows + token) * a.heads + head) * a.dim;
  T* const op = static_cast<T*>(g.o) + (token * a.heads + head) * a.dim;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 32 * d + 8 * i + 4 * half;
      const float4 v = make_float4(acc[d][4 * i] * inv, acc[d][4 * i + 1] * inv, acc[d][4 * i + 2] * inv, acc[d][4 * i + 3] * inv);
      if (at < a.dim) {
        if (whole) put4(op + at, v.x, v.y, v.z, v.w);
        else put4(po + at, v.x, v.y, v.z, v.w);
      }
    }
  if (half == 0) (whole ? g.lse : g.part_lse + (long)part * a.heads * a.q_rows)[(long)head * a.q_rows + token] = lse;
}

// 128 rows, 32 to each of four wavefronts.  With KS = 2 there are four more, and the two sets take every second step of keys and join what they have at the end:
// half the steps one behind the other for launches that leave CUs empty.
template <typename T, int DC, int KS>
__global__ __launch_bounds__(256 * KS, sizeof(T) == 2 ? 2 : 1) void attn_fwd_kernel(const FwdArgs g) {
  constexpr int DH = tile_dim(DC);
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = DC / 16, DB = DC / 32, SLOT = kStep * L::kRowBytes;
  __shared__ __align__(1024) char smem[4 * KS * SLOT];       // keys and values, two of each for each set
  __shared__ float2 stats[KS == 1 ? 1 : kRows];
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6) & 3, ks = (int)uniform(threadIdx.x >> 8), x = lane & 31, half = lane >> 5;
  const int part = blockIdx.x % g.parts, item = blockIdx.x / g.parts, kvh = item % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, item / a.kv_heads, kRows, lane, s, tile, tiles)) return;
  tile = tiles - 1 - tile;                                   // the longest first

  // this lane's row, and what the block and the wavefront see between them
  const int G = a.group, n_rows = s.lq * G, r0 = tile * kRows, row = r0 + wave * 32 + x;
  const int query = min(row, n_rows - 1) / G, head = kvh * G + min(row, n_rows - 1) % G;
  const bool real = row < n_rows;
  const Reach mine = reach(a, s, query);
  const int last = min(r0 + kRows, n_rows) - 1;
  const int lo = reach(a, s, r0 / G).lo, hi = reach(a, s, last / G).hi;
  const int w_first = min(r0 + wave * 32, n_rows - 1) / G, w_last = min(r0 + wave * 32 + 31, n_rows - 1) / G;
  const Reach w0 = reach(a, s, w_first), w1 = reach(a, s, w_last);       // [w0.lo, w1.hi) is seen by some row, [w1.lo, w0.hi) by all
  const bool w_real = r0 + wave * 32 < n_rows;
  int j0 = lo / kStep, j1;
  {
    int from, to;
    if (!part_of(g, part, hi > lo ? cdiv(hi, kStep) - j0 : 0, from, to)) return;
    j1 = j0 + to;
    j0 += from;
  }

  // queries: the operand with the rows across, in registers
  Frag qf[KC];
  {
    const T* const qp = static_cast<const T*>(g.q) + (long)(s.q0 + query) * a.q_row + (long)head * a.q_head + 8 * half;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[kc] = real && 16 * kc + 8 * half < a.dim ? Mma<T>::load(qp + 16 * kc) : Mma<T>::zero();
  }

  // keys and values on their way into LDS
  const long stride[2] = {a.k_row * ES, a.v_row * ES};
  const unsigned long base[2] = {(unsigned long)g.k + (unsigned long)(s.k0 * stride[0] + (long)kvh * a.k_head * ES),
                                 (unsigned long)g.v + (unsigned long)(s.k0 * stride[1] + (long)kvh * a.v_head * ES)};
  const unsigned lds0 = lds_address(smem);
  unsigned off[2][L::kLoads];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < L::kLoads; ++n) off[i][n] = L::load_off(wave, n, lane, stride[i], a.dim);
  TileStream stream(base, stride, j0 + ks, min(s.lk, j1 * kStep), KS);
  auto fetch = [&](int slot) {
    const rsrc_t k = stream.next(0), v = stream.next(1);
    return PairLoad<T, DH>(off, k, v, lds0 + (unsigned)((slot * KS + ks) * 2 * SLOT), wave);
  };
  constexpr int PIECES = PairLoad<T, DH>::kPieces;

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  float m = -INFINITY, l[4] = {0.f, 0.f, 0.f, 0.f};             // of this lane's row, in units of log2; l: this half's share
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
  settle(qf);
  if (j0 < j1) fetch(0).all();
  int slot = 0;
  for (int first = j0; first < j1; first += KS, slot ^= 1) {
    wait_and_meet<0>();
    const int j = first + ks, key0 = j * kStep;
    const PairLoad<T, DH> next = fetch(slot ^ 1);
    if (!w_real || (KS > 1 && j >= j1) || key0 >= w1.hi || key0 + kStep <= w0.lo) {
      next.all();
      continue;
    }
    const char* const kt = smem + (slot * KS + ks) * 2 * SLOT;
    const char* const vt = kt + SLOT;
    f32x16 sc[2] = {f32x16{}, f32x16{}};
    Frag kf[3][2];             // read two steps ahead
#pragma unroll
    for (int kc = 0; kc < 2; ++kc)
#pragma unroll
      for (int n = 0; n < 2; ++n) kf[kc][n] = L::row_frag(kt, rb, n, kc);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      if (kc + 2 < KC)
#pragma unroll
        for (int n = 0; n < 2; ++n) kf[(kc + 2) % 3][n] = L::row_frag(kt, rb, n, kc + 2);
#pragma unroll
      for (int n = 0; n < 2; ++n) sc[n] = Mma<T>::mma(kf[kc % 3][n], qf[kc], sc[n]);
#pragma unroll
      for (int p = PIECES * kc / KC; p < PIECES * (kc + 1) / KC; ++p) next.piece(p);
    }
    if (key0 < w1.lo || key0 + kStep > w0.hi) {
      const int from = mine.lo - key0 - 4 * half, to = mine.hi - key0 - 4 * half;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 32 * n + 8 * (i / 4) + i % 4;
          if (at < from || at >= to) sc[n][i] = -INFINITY;
        }
    }
    float tops[4] = {sc[0][0], sc[0][8], sc[1][0], sc[1][8]};          // (four chains of eight, as the sums below: one chain would be waited for)
#pragma unroll
    for (int i = 1; i < 8; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) tops[u] = fmaxf(tops[u], sc[u / 2][8 * (u % 2) + i]);
    const float top = both_max(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))) * g.c;
    if (__any(top > m + kLazy)) {
      const bool raise = top > m + kLazy;
      const float f = raise ? exp2_(m - top) : 1.f;
      if (raise) m = top;
#pragma unroll
      for (int u = 0; u < 4; ++u) l[u] *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[n][i] = exp2_(fmaf(sc[n][i], g.c, -base));
        l[2 * n + i / 8] += sc[n][i];
      }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const Frag p = Mma<T>::of(sc[kk / 2], kk % 2);
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] = Mma<T>::mma(L::col_frag(vt, cb, d, kk), p, acc[d]);
    }
  }

  drain();
  float sum = both_sum((l[0] + l[1]) + (l[2] + l[3]));
  if constexpr (KS == 2) {
    // the second set's to the first, both scaled to their common maximum
    float4* const other = reinterpret_cast<float4*>(smem) + wave * DB * 4 * kWave + lane;
    wait_and_meet<0>();
    if (ks == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) other[(d * 4 + i) * kWave] = make_float4(acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]);
      if (half == 0) stats[wave * 32 + x] = make_float2(m, sum);
    }
    wait_and_meet<0>();
    if (ks == 1) return;
    const float2 st = stats[wave * 32 + x];
    const float top = fmaxf(m, st.x), low = top == -INFINITY ? 0.f : top, f = exp2_(m - low), f1 = exp2_(st.x - low);
    sum = sum * f + st.y * f1;
    m = top;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 u = other[(d * 4 + i) * kWave];
        acc[d][4 * i] = acc[d][4 * i] * f + u.x * f1;
        acc[d][4 * i + 1] = acc[d][4 * i + 1] * f + u.y * f1;
        acc[d][4 * i + 2] = acc[d][4 * i + 2] * f + u.z * f1;
        acc[d][4 * i + 3] = acc[d][4 * i + 3] * f + u.w * f1;
      }
  }
  if (real) put_row<T, DB>(g, part, s.q0 + query, head, half, acc, sum, m);
}

// Few rows of a sequence (up to 32) against many keys: every wavefront goes over keys of its own, steps of 32, through LDS of its own, so nothing is waited
// for but the wavefront's own loads, of which the next step's are always on their way.  The wavefronts' sums meet in LDS at the end.
template <typename T, int DH>
struct Few {
  typedef Tile<T, DH> L;
  static constexpr int kSlot = kFewStep * L::kRowBytes, kLoads = kFewStep / L::kRowsPerLoad;      // of keys or values
  static constexpr int kWaves = 64 * 1024 / (4 * kSlot) < 4 ? 64 * 1024 / (4 * kSlot) : 4;          // two slots of both each; two blocks to a CU
};
// What the blocks of that kernel make of the descriptors, every one for itself: items of (tile of rows, part of its sequence's keys), all parts of one size
// `per`, such that there are about kFewItems of them, so the work is even however unequal the sequences are.
constexpr int kFewItems = 1024, kFewLeast = 8, kFewBlocks = 512;      // kFewLeast: steps to a part at least; kFewBlocks: what the chip holds
struct Span { int tiles, j0, n; };      // of a sequence: tiles of rows, first step of keys that its queries see, steps
__device__ __forceinline__ Span span_of(const AttnShape& a, const Seq& s) {
  if (s.lq == 0) return Span{0, 0, 0};
  const int lo = reach(a, s, 0).lo, hi = reach(a, s, s.lq - 1).hi;
  return Span{cdiv((long)s.lq * a.group, kFewRows), lo / kFewStep, hi > lo ? cdiv(hi, kFewStep) - lo / kFewStep : 0};
}
struct FewPlan {
  Seq seq;              // of lane b, where there are at most 64 sequences
  int per;
  __device__ __forceinline__ Seq lanes(const AttnShape& a, int b0, int lane) const {
    if (a.n_seq <= kWave) return seq;
    return b0 + lane < a.n_seq ? sequence(a, b0 + lane) : Seq{0, 0, 0, 0};
  }
  __device__ __forceinline__ FewPlan(const AttnShape& a, int parts, int lane) : seq(lane < a.n_seq ? sequence(a, lane) : Seq{0, 0, 0, 0}), per(1 << 30) {
    if (parts == 1) return;
    long steps = 0;
    int most = 0;
    for (int b0 = 0; b0 < a.n_seq; b0 += kWave) {
      const Span p = span_of(a, lanes(a, b0, lane));
      steps += (long)p.tiles * p.n;
      most = max(most, p.n);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      steps += __shfl_xor(steps, o, kWave);
      most = max(most, __shfl_xor(most, o, kWave));
    }
    per = __builtin_amdgcn_readfirstlane(max(max((int)((steps * a.kv_heads + kFewItems - 1) / kFewItems), cdiv(most, parts)), kFewLeast));
  }
  // item t: its sequence, tile, steps [from, to) of the sequence and part; false beyond the last item
  __device__ __forceinline__ bool find(const AttnShape& a, int t, int lane, Seq& s, int& tile, int& part, int& from, int& to) const {
    int before = 0;
    for (int b0 = 0; b0 < a.n_seq; b0 += kWave) {
      const Seq mine = lanes(a, b0, lane);
      const Span p = span_of(a, mine);
      const int cuts = max(cdiv(p.n, per), 1);
      int sum = p.tiles * cuts;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int up = __shfl_up(sum, d, kWave);
        if (lane >= d) sum += up;
      }
      const unsigned long has = __ballot(t < before + sum);
      if (has) {
        const int at = __builtin_ctzl(has);
        auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        s = Seq{pick(mine.q0), pick(mine.lq), pick(mine.k0), pick(mine.lk)};
        const int c = pick(cuts), i = t - before - (pick(sum) - pick(p.tiles) * c), n = pick(p.n), j0 = pick(p.j0);
        tile = i / c;
        part = i - tile * c;
        from = j0 + part * per;
        to = j0 + (part == c - 1 ? n : (part + 1) * per);
        return true;
      }
      before += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    return false;
  }
};

template <typename T, int DC>
__global__ __launch_bounds__((64 * Few<T, tile_dim(DC)>::kWaves)) void attn_few_kernel(const FwdArgs g) {
  constexpr int DH = tile_dim(DC);
  typedef Tile<T, DH> L;
  typedef Few<T, DH> W;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = DC / 16, DB = DC / 32;
  __shared__ __align__(1024) char smem[W::kWaves * 4 * W::kSlot];
  __shared__ float2 stats[W::kWaves][kFewRows];
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 31, half = lane >> 5;
  const FewPlan plan(a, g.parts, lane);
  char* const mem = smem + wave * 4 * W::kSlot;
  const unsigned lds0 = lds_address(mem);
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
  for (int item = blockIdx.x;; item += gridDim.x) {
  Seq s;
  int tile, part, j0, j1;
  const int kvh = item % a.kv_heads;
  if (!plan.find(a, item / a.kv_heads, lane, s, tile, part, j0, j1)) return;
  const int G = a.group, n_rows = s.lq * G, r0 = tile * kFewRows, row = r0 + x, last = min(r0 + kFewRows, n_rows) - 1;
  const int query = min(row, last) / G, head = kvh * G + min(row, last) % G;
  const bool real = row <= last;
  const Reach mine = reach(a, s, query), first = reach(a, s, r0 / G), final = reach(a, s, last / G);
  // (of its sequence's steps, those that the tile sees)
  j0 = max(j0, first.lo / kFewStep);
  j1 = final.hi > first.lo ? min(j1, cdiv(final.hi, kFewStep)) : j0;

  const long stride[2] = {a.k_row * ES, a.v_row * ES};
  const unsigned long base[2] = {(unsigned long)g.k + (unsigned long)(s.k0 * stride[0] + (long)kvh * a.k_head * ES),
                                 (unsigned long)g.v + (unsigned long)(s.k0 * stride[1] + (long)kvh * a.v_head * ES)};
  unsigned off[2][W::kLoads];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < W::kLoads; ++i) {
      const int r = i * L::kRowsPerLoad + lane / L::kChunks, ch = L::load_chunk(r, lane);
      off[t][i] = ch * (16 / ES) < a.dim ? (unsigned)(r * stride[t] + ch * 16) : kOutOfRange;
    }
  auto load = [&](int j, int slot) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const unsigned long at = base[t] + (unsigned long)((long)j * kFewStep * stride[t]);
      const rsrc_t rs = rsrc_for_lds(at, (unsigned)(j < j1 ? min(s.lk - j * kFewStep, kFewStep) * stride[t] : 0));
#pragma unroll
      for (int i = 0; i < W::kLoads; ++i) {
        const unsigned m = set_lds_dest(uniform(lds0 + (unsigned)((slot * 2 + t) * W::kSlot + i * 1024)));
        one_instruction();
        load_to_lds(rs, off[t][i], m);
      }
    }
  };
  int j = j0 + wave;
  // queries first: they are waited for by number of loads behind them
  Frag qf[KC];
  {
    const T* const qp = static_cast<const T*>(g.q) + (long)(s.q0 + query) * a.q_row + (long)head * a.q_head + 8 * half;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[kc] = real && 16 * kc + 8 * half < a.dim ? Mma<T>::load(qp + 16 * kc) : Mma<T>::zero();
  }
  load(j, 0);
  settle(qf);

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  float m = -INFINITY, l[2] = {0.f, 0.f};
  int slot = 0;
  for (; j < j1; j += W::kWaves, slot ^= 1) {
    load(j + W::kWaves, slot ^ 1);
    wait_for<2 * W::kLoads>();
    const int key0 = j * kFewStep;
    const char* const ks = mem + slot * 2 * W::kSlot;
    const char* const vs = ks + W::kSlot;
    f32x16 sc = f32x16{};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) sc = Mma<T>::mma(L::row_frag(ks, rb, 0, kc), qf[kc], sc);
    if (key0 < final.lo || key0 + kFewStep > first.hi) {
      const int from = mine.lo - key0 - 4 * half, to = mine.hi - key0 - 4 * half;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = 8 * (i / 4) + i % 4;
        if (at < from || at >= to) sc[i] = -INFINITY;
      }
    }
    float tops[2] = {sc[0], sc[8]};
#pragma unroll
    for (int i = 1; i < 8; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) tops[u] = fmaxf(tops[u], sc[8 * u + i]);
    const float top = both_max(fmaxf(tops[0], tops[1])) * g.c;
    if (__any(top > m + kLazy)) {
      const bool raise = top > m + kLazy;
      const float f = raise ? exp2_(m - top) : 1.f;
      if (raise) m = top;
      l[0] *= f;
      l[1] *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] *= f;
    }
    const float low = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[i] = exp2_(fmaf(sc[i], g.c, -low));
      l[i / 8] += sc[i];
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const Frag p = Mma<T>::of(sc, kk);
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] = Mma<T>::mma(L::col_frag(vs, cb, d, kk), p, acc[d]);
    }
    wait_for_reads();         // ahead of the loads that overwrite them
  }
  drain();

  // the wavefronts' sums, scaled to their common maximum
  const float sum = both_sum(l[0] + l[1]);
  if (half == 0) stats[wave][x] = make_float2(m, sum);
  wait_and_meet<0>();
  float top = -INFINITY, all = 0.f;
#pragma unroll
  for (int w = 0; w < W::kWaves; ++w) top = fmaxf(top, stats[w][x].x);
  const float low = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < W::kWaves; ++w) all += stats[w][x].y * exp2_(stats[w][x].x - low);
  const float f = exp2_(m - low);
  // slice DB / kWaves of the elements is joined by one wavefront: [wave][d][i][lane]
  float4* const shared = reinterpret_cast<float4*>(smem);
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    acc[d] *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      shared[((wave * DB + d) * 4 + i) * kWave + lane] = make_float4(acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]);
  }
  wait_and_meet<0>();
  const bool whole = g.parts == 1;
  const float inv = all == 0.f ? 0.f : 1.f / all;
  const long token = s.q0 + query;
  float* const po = g.part_o + (((long)part * a.q_rows + token) * a.heads + head) * a.dim;
  T* const op = static_cast<T*>(g.o) + (token * a.heads + head) * a.dim;
  for (int t = wave; t < 4 * DB; t += W::kWaves) {
    float4 v = shared[t * kWave + lane];
#pragma unroll
    for (int w = 1; w < W::kWaves; ++w) {
      const float4 u = shared[(w * DB * 4 + t) * kWave + lane];
      v = make_float4(v.x + u.x, v.y + u.y, v.z + u.z, v.w + u.w);
    }
    const int at = 32 * (t / 4) + 8 * (t % 4) + 4 * half;
    if (real && at < a.dim) {
      if (whole) put4(op + at, v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      else put4(po + at, v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    }
  }
  if (real && wave == 0 && half == 0) (whole ? g.lse : g.part_lse + (long)part * a.heads * a.q_rows)[(long)head * a.q_rows + token] = (top + log2f(all)) * kLn2;
  wait_and_meet<0>();           // the next item's loads overwrite what has been read here
  }
}

// The parts of a row's keys joined: weights exp(lse_p - lse).  LANES lanes to a row: 32 hold four elements each, and each 32 go over every
// (LANES / 32)th part.
template <typename T, int LANES, bool FEW>
__global__ __launch_bounds__(256) void attn_join_kernel(const FwdArgs g) {
  constexpr int GROUPS = LANES / 32, PER_BLOCK = 256 / LANES;
  __shared__ float4 red[256];
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, kvh = blockIdx.x % a.kv_heads, t = threadIdx.x % LANES, group = t / 32, d = 4 * (t % 32);
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, blockIdx.x / a.kv_heads, PER_BLOCK, lane, s, tile, tiles)) return;
  const int n_rows = s.lq * a.group, row = tile * PER_BLOCK + (int)threadIdx.x / LANES;
  const bool real = row < n_rows;
  const int r = min(row, n_rows - 1), head = kvh * a.group + r % a.group;
  const long token = s.q0 + r / a.group;
  // as many parts as there were for the row's tile
  int used;
  if constexpr (FEW) {
    used = max(cdiv(span_of(a, s).n, FewPlan(a, g.parts, lane).per), 1);
  } else {
    const int r0 = r / kRows * kRows, from = reach(a, s, r0 / a.group).lo, to = reach(a, s, (min(r0 + kRows, n_rows) - 1) / a.group).hi;
    used = parts_used(g, to > from ? cdiv(to, kStep) - from / kStep : 0);
  }
  const float* const lse = g.part_lse + (long)head * a.q_rows + token;
  const long lse_step = (long)a.heads * a.q_rows, step = (long)a.q_rows * a.heads * a.dim;
  constexpr int MINE = kMaxParts / GROUPS < 8 ? kMaxParts / GROUPS : 8;          // parts of a lane that are requested at once, ahead of their weights
  const float* const op = g.part_o + (token * a.heads + head) * a.dim + d;
  const bool in = d < a.dim;
  float4 o[MINE];
  auto request = [&](int p0) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int p = p0 + i * GROUPS + group;
      o[i] = p < used && in ? *reinterpret_cast<const float4*>(op + p * step) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  request(0);
  float mine[kMaxParts / 32], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxParts / 32; ++i) {
    const int p = t % 32 + 32 * i;
    mine[i] = p < used ? lse[p * lse_step] : -INFINITY;
    top = fmaxf(top, mine[i]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  const float low = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int i = 0; i < kMaxParts / 32; ++i) sum += mine[i] = exp2_((mine[i] - low) * kLog2e);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < used; p0 += MINE * GROUPS) {
    if (p0 > 0) request(p0);
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int p = p0 + i * GROUPS + group;
      const float w0 = __shfl(mine[0], (lane & 32) + (p & 31), kWave), w1 = __shfl(mine[1], (lane & 32) + (p & 31), kWave), w = p < 32 ? w0 : w1;
      if (p < used) y = make_float4(fmaf(w, o[i].x, y.x), fmaf(w, o[i].y, y.y), fmaf(w, o[i].z, y.z), fmaf(w, o[i].w, y.w));
    }
  }
  if constexpr (GROUPS > 1) {
    red[threadIdx.x] = y;
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) {
      const float4 o = red[threadIdx.x + 32 * i];
      y = make_float4(y.x + o.x, y.y + o.y, y.z + o.z, y.w + o.w);
    }
  }
  if (!real) return;
  if (t == 0) g.lse[(long)head * a.q_rows + token] = top + log2f(sum) * kLn2;
  if (in) put4(static_cast<T*>(g.o) + (token * a.heads + head) * a.dim + d, y.x * inv, y.y * inv, y.z * inv, y.w * inv);
}
static_assert(kMaxParts == 64, "two parts to a lane");

// How a call is cut.  few: 32 rows at most to a sequence on the average, by the kernel for these.  Parts: so that few rows against many keys fill the chip.
struct Cut { bool few; int parts, per; };
Cut cut_of(int dtype, const AttnShape& a) {
  if (a.n_seq == 0 || a.q_rows == 0) return {false, 1, 1};
  const long rows = (long)a.q_rows * a.group, keys = a.k_rows / a.n_seq;
  if (rows <= (long)kFewRows * a.n_seq) {
    const long tiles = std::max<long>(cdiv(rows, kFewRows), std::min(a.n_seq, a.q_rows)) * a.kv_heads;
    return {true, (int)std::max<long>(1, std::min<long>({kMaxParts, 4 * kFewItems / tiles, a.k_rows / (kFewLeast * kFewStep)})), 1};
  }
  const long tiles = std::max<long>(cdiv(rows, kRows), std::min(a.n_seq, a.q_rows)) * a.kv_heads;
  const long held = dtype == SPES_F32 && a.dim > 64 ? 256 : 512;      // blocks that the chip holds: two to a CU, or one
  const int parts = (int)std::max<long>(1, std::min<long>({kMaxParts, held / tiles, keys / 256}));
  return {false, parts, (int)cdiv(cdiv(std::max<long>(keys, 1), kStep), parts)};
}

template <typename T, int DC>
int fwd(const FwdArgs& g, bool few, hipStream_t s) {
  const AttnShape& a = g.a;
  const long n = (long)a.q_rows * a.group;
  auto grid = [&](long per, int parts) { return dim3((unsigned)((n / per + a.n_seq) * a.kv_heads * parts)); };
  if (few) {
    attn_few_kernel<T, DC><<<std::min<unsigned>(grid(kFewRows, g.parts).x, kFewBlocks), dim3(64 * Few<T, tile_dim(DC)>::kWaves), 0, s>>>(g);
    if (g.parts > 1) attn_join_kernel<T, 256, true><<<grid(1, 1), dim3(256), 0, s>>>(g);
  } else {
    bool two = false;
    if constexpr (kTwoSets<T, DC>) two = g.parts == 1 && two_sets(n / kRows * a.kv_heads, 512, a.k_rows, a.n_seq);
    if constexpr (kTwoSets<T, DC>)
      if (two) attn_fwd_kernel<T, DC, 2><<<grid(kRows, g.parts), dim3(512), 0, s>>>(g);
    if (!two) attn_fwd_kernel<T, DC, 1><<<grid(kRows, g.parts), dim3(256), 0, s>>>(g);
    if (g.parts > 1) attn_join_kernel<T, 32, false><<<grid(8, 1), dim3(256), 0, s>>>(g);
  }
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}
template <typename T>
int fwd(const FwdArgs& g, bool few, hipStream_t s) {
  const int dim = g.a.dim;
  return dim <= 32 ? fwd<T, 32>(g, few, s) : dim <= 64 ? fwd<T, 64>(g, few, s) : dim <= 96 ? fwd<T, 96>(g, few, s) : fwd<T, 128>(g, few, s);
}

}  // namespace

size_t attn_fwd_scratch_bytes(int dtype, const AttnShape& a) {
  const int parts = cut_of(dtype, a).parts;
  return parts == 1 ? 16 : (size_t)parts * a.q_rows * a.heads * (a.dim + 1) * sizeof(float) + 16;
}

int launch_attn_fwd(int dtype, const AttnShape& a, const void* q, const void* k, const void* v, void* o, float* lse, void* scratch, hipStream_t s) {
  const Cut cut = cut_of(dtype, a);
  FwdArgs g = {a, q, k, v, o, lse, nullptr, nullptr, cut.parts, cut.per, a.scale * kLog2e};
  g.part_o = static_cast<float*>(scratch);
  g.part_lse = g.part_o + (size_t)g.parts * a.q_rows * a.heads * a.dim;
  return dtype == SPES_BF16 ? fwd<bf16_t>(g, cut.few, s) : fwd<float>(g, cut.few, s);
}

}  // namespace spes
