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
  int items;            // of few rows whose keys are not cut: places of tiles
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

// A row's result: part of one, or the whole.  The row is the lane's column j of the DC elements in acc
template <typename T, int DC>
__device__ __forceinline__ void put_row(const FwdArgs& g, int part, long token, int head, int quad, const Acc (&acc)[kFrags<DC>], int j, float sum, float m) {
  const AttnShape& a = g.a;
  const float inv = sum == 0.f ? 0.f : 1.f / sum, lse = (m + log2f(sum)) * kLn2;
  const bool whole = g.parts == 1;
  float* const po = g.part_o + (((long)part * a.q_rows + token) * a.heads + head) * a.dim;
  T* const op = static_cast<T*>(g.o) + (token * a.heads + head) * a.dim;
#pragma unroll
  for (int d = 0; d < kFrags<DC>; ++d)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!has_tile<DC>(d, i)) continue;
      const int at = 32 * d + 16 * i + 4 * quad;
      const f32x4 v = acc[d].t[i][j] * inv;
      if (at < a.dim) {
        if (whole) put4(op + at, v[0], v[1], v[2], v[3]);
        else put4(po + at, v[0], v[1], v[2], v[3]);
      }
    }
  if (quad == 0) (whole ? g.lse : g.part_lse + (long)part * a.heads * a.q_rows)[(long)head * a.q_rows + token] = lse;
}

// 128 rows, 32 to each of four wavefronts, whose queries stay in registers; 64 keys and values at a time pass through LDS, the next ones on their way meanwhile.
// With KS = 2 there are four more wavefronts, and the two sets take every second step of keys and join what they have at the end: half the steps one behind
// the other for launches that leave CUs empty.
// Two wavefronts to a SIMD in bf16 (220 registers with heads of 128): one's matrix instructions run beside the other's exponentials.  32 heads of 128 (8 of
// keys), 8 x 4096 tokens, causal: 1.10 to 1.19 ms, 0.92 to 1.00 PFLOP/s of what the mask leaves, bound by power (with zeros for data 0.89 ms; a library product of
// 8192^3 1.22 to 1.27 PFLOP/s).  512 queries against 16000 keys: 147 to 160 us, 0.83 to 0.90 PFLOP/s.  12 heads of 64, 2 x 2048 tokens: 31 us; there exponentials and
// maxima take longer than the products.  fp32, 10 heads of 80, 2760 tokens, window of 700: 76 us, one wavefront to a SIMD (263 registers, and LDS for one set, with rows
// of 80 laid out as 128); the matrix instructions of the longest block 55 of them.
template <typename T, int DC, int KS>
__global__ __launch_bounds__(256 * KS, sizeof(T) == 2 ? 2 : 1) void attn_fwd_kernel(const FwdArgs g) {
  constexpr int DH = tile_dim(DC);
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = kFrags<DC>, DB = kFrags<DC>, SLOT = kStep * L::kRowBytes;
  __shared__ __align__(1024) char smem[4 * KS * SLOT];       // keys and values, two of each for each set
  __shared__ float2 stats[KS == 1 ? 1 : kRows];
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6) & 3, ks = (int)uniform(threadIdx.x >> 8), x = lane & 15, quad = lane >> 4;
  const int part = blockIdx.x % g.parts, item = blockIdx.x / g.parts, kvh = item % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, item / a.kv_heads, kRows, lane, s, tile, tiles)) return;
  tile = tiles - 1 - tile;                                   // the longest first

  // this lane's two rows, and what the block and the wavefront see between them
  const int G = a.group, n_rows = s.lq * G, r0 = tile * kRows, w_row = r0 + wave * 32;
  const Row row[2] = {Row(w_row + x, n_rows, G, kvh), Row(w_row + 16 + x, n_rows, G, kvh)};
  const Reach mine[2] = {reach(a, s, row[0].query), reach(a, s, row[1].query)};
  const int last = min(r0 + kRows, n_rows) - 1;
  const int lo = reach(a, s, r0 / G).lo, hi = reach(a, s, last / G).hi;
  const int w_first = min(w_row, n_rows - 1) / G, w_last = min(w_row + 31, n_rows - 1) / G;
  const Reach w0 = reach(a, s, w_first), w1 = reach(a, s, w_last);       // [w0.lo, w1.hi) is seen by some row, [w1.lo, w0.hi) by all
  const bool w_real = w_row < n_rows;
  int j0 = lo / kStep, j1;
  {
    int from, to;
    if (!part_of(g, part, hi > lo ? cdiv(hi, kStep) - j0 : 0, from, to)) return;
    j1 = j0 + to;
    j0 += from;
  }

  // queries: the operand with the rows across, in registers
  Frag qf[KC][2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const T* const qp = static_cast<const T*>(g.q) + (long)(s.q0 + row[j].query) * a.q_row + (long)row[j].head * a.q_head;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[kc][j] = head_frag<T, DC>(qp, kc, quad, a.dim, row[j].real);
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
  constexpr int PIECES = PairLoad<T, DH>::kPieces, NS = 2 * KC;      // NS: steps of 32 keys and 32 elements

  Acc acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = Acc{};
  float m[2] = {-INFINITY, -INFINITY}, l[2][2] = {{0.f, 0.f}, {0.f, 0.f}};      // of the lane's rows, m in units of log2; l: this lane's share
  const typename L::Base rb = L::row_base(lane);
  const unsigned cb = L::col_base(lane);
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
    Acc sc[2] = {Acc{}, Acc{}};          // of 32 keys each
    Frag kf[3][2];                       // read two steps ahead
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) kf[t][i] = L::row_frag(kt, rb, 2 * (t % 2) + i, t / 2, last_half<DC>(t / 2));
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      if (t + 2 < NS)
#pragma unroll
        for (int i = 0; i < 2; ++i) kf[(t + 2) % 3][i] = L::row_frag(kt, rb, 2 * ((t + 2) % 2) + i, (t + 2) / 2, last_half<DC>((t + 2) / 2));
#pragma unroll
      for (int i = 0; i < 2; ++i) mma<T>(kf[t % 3][i], qf[t / 2], sc[t % 2].t[i], last_half<DC>(t / 2));
#pragma unroll
      for (int p = PIECES * t / NS; p < PIECES * (t + 1) / NS; ++p) next.piece(p);
    }
    if (key0 < w1.lo || key0 + kStep > w0.hi) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int from = mine[c].lo - key0 - 4 * quad, to = mine[c].hi - key0 - 4 * quad;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = 32 * n + 16 * i + e;
              if (at < from || at >= to) sc[n].t[i][c][e] = -INFINITY;
            }
      }
    }
    float top[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float half[2];                     // (two chains, as the sums below: one would be waited for)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        half[n] = sc[n].t[0][c][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) half[n] = fmaxf(half[n], sc[n].t[e / 4][c][e % 4]);
      }
      top[c] = quad_max(fmaxf(half[0], half[1])) * g.c;
    }
    if (__any(top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bool raise = top[c] > m[c] + kLazy;
        const float f = raise ? exp2_(m[c] - top[c]) : 1.f;
        if (raise) m[c] = top[c];
        l[c][0] *= f;
        l[c][1] *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (has_tile<DC>(d, i)) acc[d].t[i][c] *= f;
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float low = m[c] == -INFINITY ? 0.f : m[c];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = exp2_(fmaf(sc[n].t[e / 4][c][e % 4], g.c, -low));
          sc[n].t[e / 4][c][e % 4] = v;
          l[c][n] += v;
        }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const Frag p[2] = {Mma<T>::of(sc[n].t[0][0], sc[n].t[1][0]), Mma<T>::of(sc[n].t[0][1], sc[n].t[1][1])};
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (has_tile<DC>(d, i)) mma<T>(L::col_frag(vt, cb, 2 * d + i, n), p, acc[d].t[i]);
    }
  }

  drain();
  float sum[2] = {quad_sum(l[0][0] + l[0][1]), quad_sum(l[1][0] + l[1][1])};
  if constexpr (KS == 2) {
    // the second set's to the first, both scaled to their common maximum
    f32x4* const other = reinterpret_cast<f32x4*>(smem) + wave * DB * 4 * kWave + lane;
    wait_and_meet<0>();
    if (ks == 1) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 2; ++i) other[(d * 4 + i * 2 + c) * kWave] = acc[d].t[i][c];
        if (quad == 0) stats[wave * 32 + 16 * c + x] = make_float2(m[c], sum[c]);
      }
    }
    wait_and_meet<0>();
    if (ks == 1) return;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float2 st = stats[wave * 32 + 16 * c + x];
      const float top = fmaxf(m[c], st.x), low = top == -INFINITY ? 0.f : top, f = exp2_(m[c] - low), f1 = exp2_(st.x - low);
      sum[c] = sum[c] * f + st.y * f1;
      m[c] = top;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[d].t[i][c] = acc[d].t[i][c] * f + other[(d * 4 + i * 2 + c) * kWave] * f1;
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (row[c].real) put_row<T, DC>(g, part, s.q0 + row[c].query, row[c].head, quad, acc, c, sum[c], m[c]);
}

// Few rows of a sequence (up to 32) against many keys, so bound by memory: every wavefront goes over keys of its own, steps of 32, through LDS of its own, so nothing is waited
// for but the wavefront's own loads, of which the next step's are always on their way.  The wavefronts' sums meet in LDS at the end.
// One token each of 32 sequences over 1 to 8192 keys, 32 / 8 heads of 128: 44 us, 5.2 TB/s, and 6 for joining the parts; one over 131071 keys, 16 / 4 heads:
// 48 us, 5.6 TB/s, and 6 (a copy of 2 GiB 4.9 TB/s).  With the kernel above in its place 83 and 56 us in all instead of 50 and 53: its parts are cut for
// sequences of average length, and all of a block waits for every step.  fp32, where LDS holds one wavefront to a block and two to a CU: 126 us in all (3.6 TB/s)
// and 203 (2.6), 256 sequences of 500 233 (4.5).
template <typename T, int DH>
struct Few {
  typedef Tile<T, DH> L;
  static constexpr int kSlot = kFewStep * L::kRowBytes, kLoads = kFewStep / L::kRowsPerLoad;      // of keys or values
  // two slots of both each; two blocks to a CU: in bf16 up to 64 elements two wavefronts to a SIMD, else one or none
  static constexpr int kWaves = 64 * 1024 / (4 * kSlot) < 4 ? 64 * 1024 / (4 * kSlot) : 4;
};
// What the blocks of that kernel make of the descriptors, every one for itself: items of (tile of rows, part of its sequence's keys), all parts of one size
// `per`, such that there are about kFewItems of them, so the work is even however unequal the sequences are.
// With that many tiles their keys are not cut: the tiles are looked up, by up to eight times the blocks, which even out unequal sequences, and nothing is joined
// (one token each of 256 sequences, 32 / 8 heads of 128, 500 keys: 145 us cut, 109 whole; 1024 of 250 298 -> 234; 128 of 1 to 4096 302 -> 271; with
// the chip's blocks alone 115, 227 and 308; by attn_fwd_kernel 128, 225 and 288).
// (The 32 sequences above: 50 us in all with 1024 items, two for each block, 52 with 512, 56 with 2048; with at least 4 or 16 steps to a part the same as with 8.)
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
  constexpr int ES = sizeof(T), KC = kFrags<DC>, DB = kFrags<DC>;
  __shared__ __align__(1024) char smem[W::kWaves * 4 * W::kSlot];
  __shared__ float2 stats[W::kWaves][kFewRows];
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 15, quad = lane >> 4;
  const FewPlan plan(a, g.parts, lane);
  char* const mem = smem + wave * 4 * W::kSlot;
  const unsigned lds0 = lds_address(mem);
  const typename L::Base rb = L::row_base(lane);
  const unsigned cb = L::col_base(lane);
  for (int item = blockIdx.x;; item += gridDim.x) {
  Seq s;
  int tile, part = 0, j0 = 0, j1 = 1 << 30;
  const int kvh = item % a.kv_heads;
  if (g.parts > 1) {
    if (!plan.find(a, item / a.kv_heads, lane, s, tile, part, j0, j1)) return;
  } else {
    int tiles;
    if (item >= g.items) return;
    if (!find_tile<false>(a, item / a.kv_heads, kFewRows, lane, s, tile, tiles)) continue;
  }
  const int G = a.group, n_rows = s.lq * G, r0 = tile * kFewRows, last = min(r0 + kFewRows, n_rows) - 1;
  const Row row[2] = {Row(r0 + x, n_rows, G, kvh), Row(r0 + 16 + x, n_rows, G, kvh)};
  const Reach mine[2] = {reach(a, s, row[0].query), reach(a, s, row[1].query)}, first = reach(a, s, r0 / G), final = reach(a, s, last / G);
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
  Frag qf[KC][2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const T* const qp = static_cast<const T*>(g.q) + (long)(s.q0 + row[c].query) * a.q_row + (long)row[c].head * a.q_head;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[kc][c] = head_frag<T, DC>(qp, kc, quad, a.dim, row[c].real);
  }
  load(j, 0);
  settle(qf);

  // (rows beyond sixteen, where there are any, are the lane's second)
  const bool both = last - r0 >= 16;
  Acc acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = Acc{};
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  int slot = 0;
  for (; j < j1; j += W::kWaves, slot ^= 1) {
    load(j + W::kWaves, slot ^ 1);
    wait_for<2 * W::kLoads>();
    const int key0 = j * kFewStep;
    const char* const kt = mem + slot * 2 * W::kSlot;
    const char* const vt = kt + W::kSlot;
    Acc sc = Acc{};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool half = last_half<DC>(kc);
        const Frag f = L::row_frag(kt, rb, i, kc, half);
        sc.t[i][0] = Mma<T>::mma(f, qf[kc][0], sc.t[i][0], half);
        if (both) sc.t[i][1] = Mma<T>::mma(f, qf[kc][1], sc.t[i][1], half);
      }
    const bool cut = key0 < final.lo || key0 + kFewStep > first.hi;
    Frag p[2] = {Mma<T>::zero(), Mma<T>::zero()};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (c == 1 && !both) break;
      if (cut) {
        const int from = mine[c].lo - key0 - 4 * quad, to = mine[c].hi - key0 - 4 * quad;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int at = 16 * (e / 4) + e % 4;
          if (at < from || at >= to) sc.t[e / 4][c][e % 4] = -INFINITY;
        }
      }
      float top = sc.t[0][c][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, sc.t[e / 4][c][e % 4]);
      top = quad_max(top) * g.c;
      if (__any(top > m[c] + kLazy)) {
        const bool raise = top > m[c] + kLazy;
        const float f = raise ? exp2_(m[c] - top) : 1.f;
        if (raise) m[c] = top;
        l[c] *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (has_tile<DC>(d, i)) acc[d].t[i][c] *= f;
      }
      const float low = m[c] == -INFINITY ? 0.f : m[c];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = exp2_(fmaf(sc.t[e / 4][c][e % 4], g.c, -low));
        sc.t[e / 4][c][e % 4] = v;
        l[c] += v;
      }
      p[c] = Mma<T>::of(sc.t[0][c], sc.t[1][c]);
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!has_tile<DC>(d, i)) continue;
        const Frag f = L::col_frag(vt, cb, 2 * d + i, 0);
        acc[d].t[i][0] = Mma<T>::mma(f, p[0], acc[d].t[i][0]);
        if (both) acc[d].t[i][1] = Mma<T>::mma(f, p[1], acc[d].t[i][1]);
      }
    wait_for_reads();         // ahead of the loads that overwrite them
  }
  drain();

  // the wavefronts' sums, scaled to their common maximum
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const float sum = quad_sum(l[c]);
    if (quad == 0) stats[wave][16 * c + x] = make_float2(m[c], sum);
  }
  wait_and_meet<0>();
  f32x4* const shared = reinterpret_cast<f32x4*>(smem) + lane;      // [wave][c][d][i][lane]
  float low[2], all[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W::kWaves; ++w) top = fmaxf(top, stats[w][16 * c + x].x);
    low[c] = top == -INFINITY ? 0.f : top;
    all[c] = 0.f;
#pragma unroll
    for (int w = 0; w < W::kWaves; ++w) all[c] += stats[w][16 * c + x].y * exp2_(stats[w][16 * c + x].x - low[c]);
    const float f = exp2_(m[c] - low[c]);
    if (c == 0 || both)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 2; ++i) shared[(((wave * 2 + c) * DB + d) * 2 + i) * kWave] = acc[d].t[i][c] * f;
  }
  wait_and_meet<0>();
  // each of the sixteen elements' quads of a column is joined by one wavefront
  const bool whole = g.parts == 1;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    if (c == 1 && !both) break;
    const float inv = all[c] == 0.f ? 0.f : 1.f / all[c];
    const long token = s.q0 + row[c].query;
    float* const po = g.part_o + (((long)part * a.q_rows + token) * a.heads + row[c].head) * a.dim;
    T* const op = static_cast<T*>(g.o) + (token * a.heads + row[c].head) * a.dim;
    for (int t = wave; t < 2 * DB; t += W::kWaves) {
      f32x4 v = shared[(c * DB * 2 + t) * kWave];
#pragma unroll
      for (int w = 1; w < W::kWaves; ++w) v += shared[((w * 2 + c) * DB * 2 + t) * kWave];
      v *= inv;
      const int at = 16 * t + 4 * quad;
      if (row[c].real && at < a.dim) {
        if (whole) put4(op + at, v[0], v[1], v[2], v[3]);
        else put4(po + at, v[0], v[1], v[2], v[3]);
      }
    }
    // (a row without keys: its sum is nothing, and so is what its maximum is)
    if (row[c].real && wave == 0 && quad == 0)
      (whole ? g.lse : g.part_lse + (long)part * a.heads * a.q_rows)[(long)row[c].head * a.q_rows + token] = (low[c] + log2f(all[c])) * kLn2;
  }
  wait_and_meet<0>();           // the next item's loads overwrite what has been read here
  }
}

// The parts of a row's keys joined: weights exp(lse_p - lse).  LANES lanes to a row: 32 hold four elements each, and each 32 go over every
// (LANES / 32)th part.  A launch of its own, so no block waits for another: 6 us for one token of 32 sequences (1024 rows of up to 19 parts), which is two
// trips to memory one behind the other, and 11 for 512 queries of 32 heads in 4 parts (34 MB).
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

// How a call is cut.  few: 32 rows at most to a sequence on the average, by the kernel for these.  Parts: so that few rows against many keys fill the chip
// (512 queries of 32 heads against 16000 keys, 128 tiles: 219 us whole, 150 in 4 parts with the launch that joins them).
// The host knows averages and the room of a cache, not lengths.  What that costs: the 512 queries in a cache with room for 131072 have all of their keys in the first part
// and take 449 us; beside 512 on 512 keys, 512 on 120000 take 1670 in place of 985; 31 single tokens of the 32 sequences above take 45 us, a prompt of 1000 on 8192 keys 148, and
// both in one batch 222.
struct Cut { bool few; int parts, per; };
Cut cut_of(int dtype, const AttnShape& a) {
  if (a.n_seq == 0 || a.q_rows == 0) return {false, 1, 1};
  const long rows = (long)a.q_rows * a.group, keys = a.k_rows / a.n_seq;
  if (rows <= (long)kFewRows * a.n_seq) {
    const long tiles = std::max<long>(cdiv(rows, kFewRows), std::min(a.n_seq, a.q_rows)) * a.kv_heads;
    const long parts = tiles >= kFewItems ? 1 : std::min<long>({kMaxParts, 4 * kFewItems / tiles, a.k_rows / (kFewLeast * kFewStep)});
    return {true, (int)std::max<long>(1, parts), 1};
  }
  const long tiles = std::max<long>(cdiv(rows, kRows), std::min(a.n_seq, a.q_rows)) * a.kv_heads;
  const long held = dtype == SPES_F32 && a.dim > 64 ? 256 : 512;      // blocks that the chip holds: two to a CU, or one
  const int parts = (int)std::max<long>(1, std::min<long>({kMaxParts, held / tiles, keys / 256}));
  return {false, parts, (int)cdiv(cdiv(std::max<long>(keys, 1), kStep), parts)};
}

template <typename T, int DC>
int fwd(FwdArgs g, bool few, hipStream_t s) {
  const AttnShape& a = g.a;
  const long n = (long)a.q_rows * a.group;
  auto grid = [&](long per, int parts) { return dim3((unsigned)((n / per + a.n_seq) * a.kv_heads * parts)); };
  if (few) {
    g.items = (int)grid(kFewRows, 1).x;
    attn_few_kernel<T, DC><<<std::min<unsigned>(grid(kFewRows, g.parts).x, g.parts > 1 ? kFewBlocks : 8 * kFewBlocks), dim3(64 * Few<T, tile_dim(DC)>::kWaves), 0, s>>>(g);
    if (g.parts > 1) attn_join_kernel<T, 256, true><<<grid(1, 1), dim3(256), 0, s>>>(g);
  } else {
    bool two = false;
    if constexpr (kTwoSets<T, DC>) two = g.parts == 1 && two_sets(n / kRows * a.kv_heads, a.k_rows, a.n_seq);
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
  if constexpr (sizeof(T) == 4) {
    if (dim > 32 && dim <= 48) return fwd<T, 48>(g, few, s);
    if (dim > 64 && dim <= 80) return fwd<T, 80>(g, few, s);
    if (dim > 96 && dim <= 112) return fwd<T, 112>(g, few, s);
  }
  return dim <= 32 ? fwd<T, 32>(g, few, s) : dim <= 64 ? fwd<T, 64>(g, few, s) : dim <= 96 ? fwd<T, 96>(g, few, s) : fwd<T, 128>(g, few, s);
}

}  // namespace

size_t attn_fwd_scratch_bytes(int dtype, const AttnShape& a) {
  const int parts = cut_of(dtype, a).parts;
  return parts == 1 ? 16 : (size_t)parts * a.q_rows * a.heads * (a.dim + 1) * sizeof(float) + 16;
}

int launch_attn_fwd(int dtype, const AttnShape& a, const void* q, const void* k, const void* v, void* o, float* lse, void* scratch, hipStream_t s) {
  const Cut cut = cut_of(dtype, a);
  FwdArgs g = {a, q, k, v, o, lse, nullptr, nullptr, cut.parts, cut.per, a.scale * kLog2e, 0};
  g.part_o = static_cast<float*>(scratch);
  g.part_lse = g.part_o + (size_t)g.parts * a.q_rows * a.heads * a.dim;
  return dtype == SPES_BF16 ? fwd<bf16_t>(g, cut.few, s) : fwd<float>(g, cut.few, s);
}

}  // namespace spes
