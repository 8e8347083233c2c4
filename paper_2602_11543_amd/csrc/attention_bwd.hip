// Attention, backward: the probabilities are formed again from q, k and the forward's lse,
//      p = exp(scale q k^T - lse)      delta = sum do o      ds = p (do v^T - delta)
//      dv = p^T do      dk = scale ds^T q      dq = scale ds k
// Two kernels, so that every sum has one owner and one order: by queries (delta and dq) and by keys (dk and dv, over the rows of all heads that share
// them).  That is 14 D operations a pair for the 10 D of the formulas: s and do v^T are formed twice.  Few blocks of both run as one launch.
// delta is formed from o as it is stored.
#include <type_traits>

#include "attention.h"

namespace spes {
namespace {

using namespace attn;

struct BwdArgs {
  AttnShape a;
  const void *d_o, *q, *k, *v, *o;
  const float* lse;
  void *dq, *dk, *dv;
  float* delta;         // [heads, q_rows]
  float c;
  int q_tiles, k_tiles; // of rows and keys, each for all heads that share keys, at most
};

// delta = sum do o of a lane's row c, whose upstream gradient is in d
template <typename T, int DC>
__device__ __forceinline__ float delta_of(const typename Mma<T>::Frag (&d)[kFrags<DC>][2], int c, const T* o, int quad, int dim, bool real) {
  float sum = 0.f;
#pragma unroll
  for (int kc = 0; kc < kFrags<DC>; ++kc) {
    const typename Mma<T>::Frag of = head_frag<T, DC>(o, kc, quad, dim, real);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(Mma<T>::get(d[kc][c], e), Mma<T>::get(of, e), sum);
  }
  return quad_sum(sum);
}

// 128 rows; KS sets of four wavefronts as in the forward.  Queries and upstream gradients stay in registers, keys and values pass through LDS: each key tile is
// read as rows for the scores and as columns for dq.  8 x 4096 tokens, 32 / 8 heads of 128, causal: 1.43 to 1.47 ms, 1.12 to 1.16 PFLOP/s of the 6 D operations a
// pair, bound by power; 2 x 2048 tokens, 12 heads of 64: 37 us.
template <typename T, int DC, int KS, bool KEEP>
__device__ __forceinline__ void bwd_q(const BwdArgs& g, int item, int kvh, char* smem) {
  constexpr int DH = tile_dim(DC);
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = kFrags<DC>, DB = kFrags<DC>, SLOT = kStep * L::kRowBytes;
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6) & 3, ks = (int)uniform(threadIdx.x >> 8), x = lane & 15, quad = lane >> 4;
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, item, kRows, lane, s, tile, tiles)) return;
  tile = tiles - 1 - tile;                                   // the longest first

  const int G = a.group, n_rows = s.lq * G, r0 = tile * kRows, w_row = r0 + wave * 32;
  const Row row[2] = {Row(w_row + x, n_rows, G, kvh), Row(w_row + 16 + x, n_rows, G, kvh)};
  const Reach mine[2] = {reach(a, s, row[0].query), reach(a, s, row[1].query)};
  const int last = min(r0 + kRows, n_rows) - 1;
  const int lo = reach(a, s, r0 / G).lo, hi = reach(a, s, last / G).hi;
  const int w_first = min(w_row, n_rows - 1) / G, w_last = min(w_row + 31, n_rows - 1) / G;
  const Reach w0 = reach(a, s, w_first), w1 = reach(a, s, w_last);
  const bool w_real = w_row < n_rows;
  const int j0 = lo / kStep, j1 = hi > lo ? cdiv(hi, kStep) : j0;

  Frag qf[KC][2], df[KC][2];
  float delta[2], base[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const long token = s.q0 + row[c].query, at = (token * a.heads + row[c].head) * a.dim;
    const T* const qp = static_cast<const T*>(g.q) + token * a.q_row + (long)row[c].head * a.q_head;
    const T* const dp = static_cast<const T*>(g.d_o) + at;
    const T* const op = static_cast<const T*>(g.o) + at;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      qf[kc][c] = head_frag<T, DC>(qp, kc, quad, a.dim, row[c].real);
      df[kc][c] = head_frag<T, DC>(dp, kc, quad, a.dim, row[c].real);
    }
    base[c] = g.lse[(long)row[c].head * a.q_rows + token] * kLog2e;
    delta[c] = delta_of<T, DC>(df, c, op, quad, a.dim, row[c].real);
    if (KEEP && row[c].real && quad == 0 && ks == 0) g.delta[(long)row[c].head * a.q_rows + token] = delta[c];
  }

  const long stride[2] = {a.k_row * ES, a.v_row * ES};
  const unsigned long source[2] = {(unsigned long)g.k + (unsigned long)(s.k0 * stride[0] + (long)kvh * a.k_head * ES),
                                   (unsigned long)g.v + (unsigned long)(s.k0 * stride[1] + (long)kvh * a.v_head * ES)};
  const unsigned lds0 = lds_address(smem);
  unsigned off[2][L::kLoads];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < L::kLoads; ++n) off[i][n] = L::load_off(wave, n, lane, stride[i], a.dim);
  TileStream stream(source, stride, j0 + ks, min(s.lk, j1 * kStep), KS);
  auto fetch = [&](int slot) {
    const rsrc_t k = stream.next(0), v = stream.next(1);
    return PairLoad<T, DH>(off, k, v, lds0 + (unsigned)((slot * KS + ks) * 2 * SLOT), wave);
  };
  constexpr int PIECES = PairLoad<T, DH>::kPieces, kAhead = 2;

  Acc acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = Acc{};
  const typename L::Base rb = L::row_base(lane);
  const unsigned cb = L::col_base(lane);
  settle(qf);
  settle(df);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    settle(base[c]);
    settle(delta[c]);
  }
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
    const bool cut = key0 < w1.lo || key0 + kStep > w0.hi;
    const char* const kt = smem + (slot * KS + ks) * 2 * SLOT;
    const char* const vt = kt + SLOT;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      Acc sc = Acc{}, ds;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) ds.t[i][c] = f32x4{-delta[c], -delta[c], -delta[c], -delta[c]};
      // operands from LDS in the order of their use, two of them on their way
      constexpr int ALL = 4 * KC;
      auto line = [&](int t) { return L::row_frag(t % 2 ? vt : kt, rb, 2 * n + t / 2 % 2, t / 4, last_half<DC>(t / 4)); };
      Frag r[kAhead + 1];
#pragma unroll
      for (int t = 0; t < kAhead; ++t) r[t] = line(t);
#pragma unroll
      for (int t = 0; t < ALL; ++t) {
        if (t + kAhead < ALL) r[(t + kAhead) % (kAhead + 1)] = line(t + kAhead);
        mma<T>(r[t % (kAhead + 1)], (t % 2 ? df : qf)[t / 4], (t % 2 ? ds : sc).t[t / 2 % 2], last_half<DC>(t / 4));
        if (n == 0)
#pragma unroll
          for (int p = PIECES * t / ALL; p < PIECES * (t + 1) / ALL; ++p) next.piece(p);
      }
      Frag f[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) ds.t[e / 4][c][e % 4] *= exp2_(fmaf(sc.t[e / 4][c][e % 4], g.c, -base[c]));
        if (cut) {
          const int from = mine[c].lo - key0 - 4 * quad, to = mine[c].hi - key0 - 4 * quad;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = 32 * n + 16 * (e / 4) + e % 4;
            if (at < from || at >= to) ds.t[e / 4][c][e % 4] = 0.f;
          }
        }
        f[c] = Mma<T>::of(ds.t[0][c], ds.t[1][c]);
      }
      Frag k[kAhead + 1];
#pragma unroll
      for (int d = 0; d < kAhead; ++d) k[d] = L::col_frag(kt, cb, d, n);
#pragma unroll
      for (int d = 0; d < DC / 16; ++d) {
        if (d + kAhead < DC / 16) k[(d + kAhead) % (kAhead + 1)] = L::col_frag(kt, cb, d + kAhead, n);
        mma<T>(k[d % (kAhead + 1)], f, acc[d / 2].t[d % 2]);
      }
    }
  }
  drain();
  if constexpr (KS == 2) {
    f32x4* const other = reinterpret_cast<f32x4*>(smem) + wave * DB * 4 * kWave + lane;
    wait_and_meet<0>();
    if (ks == 1)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) other[(d * 4 + i) * kWave] = acc[d].t[i / 2][i % 2];
    wait_and_meet<0>();
    if (ks == 1) return;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[d].t[i / 2][i % 2] += other[(d * 4 + i) * kWave];
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    if (!row[c].real) continue;
    T* const dq = static_cast<T*>(g.dq) + (long)(s.q0 + row[c].query) * a.q_row + (long)row[c].head * a.q_head;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = 32 * d + 16 * i + 4 * quad;
        const f32x4 v = acc[d].t[i][c] * a.scale;
        if (at < a.dim) put4(dq + at, v[0], v[1], v[2], v[3]);
      }
  }
}

// Four wavefronts: two groups of 32 keys, and in each one wavefront for the first 32 of the 64 rows that are in LDS and one for the others, whose sums are
// joined at the end.  The rows are gone over from the last one down: the blocks of a sequence's keys then begin at the same rows and find each other's in L2,
// where from each block's first row on they are all over a sequence of which L2 holds half (8 x 4096 tokens, 32 / 8 heads of 128: 8 MB).
// The same problems as above: 2.07 to 2.14 ms, 1.03 to 1.06 PFLOP/s of the 8 D operations a pair (a wavefront's sums, keys and values take 192 of its 256 registers, which
// leaves little for operands ahead of their use: with 128 elements in bf16 26 registers are spilled, 100 bytes a lane); 44 us.  (Four groups, 64 rows each: half the loads into LDS, but the second 32 rows cost
// more registers than there are, with 128 elements all of the backward took 12.6 ms in place of 4.1 then; 64 elements: 97 us in place of 83.)
constexpr int kKeys = 64;
template <int KS> struct Stats { float of[2][KS][2][kStep]; };       // of each slot's rows: -lse / scale (fp32: -lse log2 e), -delta
template <typename T, int DC, int KS>
__device__ __forceinline__ void bwd_kv(const BwdArgs& g, int item, int kvh, char* smem, Stats<KS>& stats) {
  constexpr int DH = tile_dim(DC);
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = kFrags<DC>, DB = kFrags<DC>, SLOT = kStep * L::kRowBytes;
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6) & 3, ks = (int)uniform(threadIdx.x >> 8), x = lane & 15, quad = lane >> 4;
  const int kw = wave % 2, rw = wave / 2;
  Seq s;
  int tile, tiles;
  if (!find_tile<true>(a, item, kKeys, lane, s, tile, tiles)) return;

  const int G = a.group, n_rows = s.lq * G, key0 = tile * kKeys, first = key0 + kw * 32, tail = s.lk - 1;
  // Rows [from, to) see a key: with causal masks r / G + lk - lq >= key, hence r >= (key - (lk - lq)) G, and likewise for the window
  auto rows_of = [&](int at) {
    Reach r = {0, n_rows};
    if (a.causal) {
      const long first_query = (long)min(at, tail) - (s.lk - s.lq), end = a.window > 0 ? min(first_query + a.window, (long)s.lq) : (long)s.lq;
      r.lo = (int)max(first_query, 0l) * G;
      r.hi = (int)max(end, 0l) * G;
    }
    return r;
  };
  const int lo = rows_of(key0).lo, hi = rows_of(key0 + kKeys - 1).hi;
  const int j0 = lo / kStep, j1 = hi > lo ? cdiv(hi, kStep) : j0;

  Frag kf[KC][2], vf[KC][2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int key = first + 16 * c + x;
    const T* const kp = static_cast<const T*>(g.k) + (long)(s.k0 + min(key, tail)) * a.k_row + (long)kvh * a.k_head;
    const T* const vp = static_cast<const T*>(g.v) + (long)(s.k0 + min(key, tail)) * a.v_row + (long)kvh * a.v_head;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      kf[kc][c] = head_frag<T, DC>(kp, kc, quad, a.dim, true);
      vf[kc][c] = head_frag<T, DC>(vp, kc, quad, a.dim, true);
    }
  }

  // rows on their way into LDS: row r of a tile is query r / G, head r % G.  Rows behind the last one repeat it (their probabilities are nothing)
  const unsigned long q_base = (unsigned long)g.q + (unsigned long)((long)s.q0 * a.q_row + (long)kvh * G * a.q_head) * ES;
  const unsigned long d_base = (unsigned long)g.d_o + (unsigned long)(((long)s.q0 * a.heads + (long)kvh * G) * a.dim) * ES;
  const unsigned lds0 = lds_address(smem);
  const unsigned magic = (1u << 22) / (unsigned)G + 1;       // n / G = n magic >> 22 for n < 64 + G, G <= 1024
  unsigned off[2][L::kLoads];
#pragma unroll
  for (int i = 0; i < L::kLoads; ++i) off[0][i] = off[1][i] = kOutOfRange;
  auto aim = [&](int rem, int left) {
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      const int r = L::load_row(wave, i, lane), ch = L::load_chunk(r, lane);
      const unsigned n = (unsigned)(min(r, left - 1) + rem), q = n * magic >> 22, h = n - q * G;
      const bool in = ch * (16 / ES) < a.dim;
      off[0][i] = in ? q * (unsigned)(a.q_row * ES) + h * (unsigned)(a.q_head * ES) + ch * 16 : kOutOfRange;
      off[1][i] = in ? q * (unsigned)(a.heads * a.dim * ES) + h * (unsigned)(a.dim * ES) + ch * 16 : kOutOfRange;
    }
  };
  // the tile that is next, from the last one down: its first row is head `rem` of a query; both are carried on by subtractions, as in TileStream by
  // additions.  A set's last tile may be ahead of the first one: it is not there, and brings rows without probabilities.
  const int by = KS * kStep, by_query = by / G, by_rem = by - by_query * G;
  const long q_bytes = a.q_row * ES, d_bytes = (long)a.heads * a.dim * ES;
  int row0 = (j1 - 1 - ks) * kStep, query0 = max(row0, 0) / G, rem0 = max(row0, 0) - query0 * G;
  unsigned long q_at = q_base + (unsigned long)(query0 * q_bytes), d_at = d_base + (unsigned long)(query0 * d_bytes);
  aim(rem0, n_rows - row0);
  auto fetch = [&](int slot) {
    const bool there = row0 >= j0 * kStep;
    if (there && (by_rem != 0 || row0 + by + kStep > n_rows)) aim(rem0, n_rows - row0);
    const PairLoad<T, DH> load(off, rsrc_for_lds(q_at, there ? kOpen : 0u), rsrc_for_lds(d_at, there ? kOpen : 0u), lds0 + (unsigned)((slot * KS + ks) * 2 * SLOT), wave);
    const int less = rem0 < by_rem, queries = by_query + less;
    row0 -= by;
    query0 -= queries;
    rem0 += less * G - by_rem;
    q_at -= (unsigned long)(queries * q_bytes);
    d_at -= (unsigned long)(queries * d_bytes);
    return load;
  };
  // one row's number of that tile to a lane of the first two wavefronts, on its way while the step before is worked on
  const float* const numbers = wave == 0 ? g.lse : g.delta;
  const float factor = wave == 1 ? -1.f : ES == 2 ? -1.f / a.scale : -kLog2e;
  auto number = [&]() {
    const unsigned n = (unsigned)(lane + rem0), q = n * magic >> 22, h = n - q * G;
    return row0 >= j0 * kStep && row0 + lane < n_rows ? numbers[(long)(kvh * G + (int)h) * a.q_rows + s.q0 + query0 + (int)q] : wave == 0 ? -INFINITY : 0.f;
  };
  auto keep = [&](int slot, float v) {
    if (wave < 2) stats.of[slot][ks][wave][lane] = wave == 0 && v == -INFINITY ? -INFINITY : v * factor;      // a row without keys has no probabilities
  };

  Acc dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = dv[d] = Acc{};
  const typename L::Base rb = L::row_base(lane);
  const unsigned cb = L::col_base(lane);
  settle(kf);
  settle(vf);
  if (j0 < j1) {
    float v = 0.f;
    if (wave < 2) v = number();
    fetch(0).all();
    keep(0, v);
  }
  const Reach mine[2] = {rows_of(first + x), rows_of(first + 16 + x)};

  // the wavefront's 32 of the rows in LDS, the first of them the sequence's r0, against its keys.  The loads of the next rows go out on the way
  auto step = [&](auto cut_, int slot, int r0, const PairLoad<T, DH>& next) {
    constexpr bool CUT = decltype(cut_)::value;
    constexpr int PIECES = PairLoad<T, DH>::kPieces;
    const char* const qs = smem + (slot * KS + ks) * 2 * SLOT;
    const char* const dos = qs + SLOT;
    const float* const st = &stats.of[slot][ks][0][32 * rw + 4 * quad];
    Acc p = Acc{}, ds;
    f32x4 lse[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lse[i] = *reinterpret_cast<const f32x4*>(st + 16 * i);
      const f32x4 w = *reinterpret_cast<const f32x4*>(st + kStep + 16 * i);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (ES == 2) p.t[i][c] = lse[i];
        ds.t[i][c] = w;
      }
    }
    // operands from LDS in the order of their use, some of them on their way: sums and what is summed leave room for one in the first half, for three in the second
    constexpr int HALF = 2 * KC;
    auto row = [&](int t) { return L::row_frag(t < HALF ? qs : dos, rb, 2 * rw + t % 2, t % HALF / 2, last_half<DC>(t % HALF / 2)); };
    Frag r[2] = {row(0), row(1)};
#pragma unroll
    for (int t = 0; t < 2 * HALF; ++t) {
      mma<T>(r[t % 2], (t < HALF ? kf : vf)[t % HALF / 2], (t < HALF ? p : ds).t[t % 2], last_half<DC>(t % HALF / 2));
      if (t + 2 < 2 * HALF) r[t % 2] = row(t + 2);
#pragma unroll
      for (int n = PIECES * t / HALF; n < min(PIECES * (t + 1) / HALF, PIECES); ++n) next.piece(n);
    }
    Frag pf[2], sf[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      // (bf16: the products are summed on top of -lse / scale; in fp32 storage that would round them to its magnitude)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = p.t[e / 4][c][e % 4], u = ES == 2 ? exp2_(v * g.c) : exp2_(fmaf(v, g.c, lse[e / 4][e % 4]));
        p.t[e / 4][c][e % 4] = u;
        ds.t[e / 4][c][e % 4] *= u;
      }
      if constexpr (CUT) {
        const int from = mine[c].lo - r0 - 4 * quad, to = mine[c].hi - r0 - 4 * quad;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int at = 16 * (e / 4) + e % 4;
          if (at < from || at >= to) p.t[e / 4][c][e % 4] = ds.t[e / 4][c][e % 4] = 0.f;
        }
      }
      pf[c] = Mma<T>::of(p.t[0][c], p.t[1][c]);
      sf[c] = Mma<T>::of(ds.t[0][c], ds.t[1][c]);
    }
    constexpr int kAhead = 3, COLS = DC / 16;
    auto column = [&](int t) { return L::col_frag(t < COLS ? dos : qs, cb, t % COLS, rw); };
    Frag f[kAhead + 1];
#pragma unroll
    for (int t = 0; t < kAhead; ++t) f[t] = column(t);
#pragma unroll
    for (int t = 0; t < 2 * COLS; ++t) {
      if (t + kAhead < 2 * COLS) f[(t + kAhead) % (kAhead + 1)] = column(t + kAhead);
      mma<T>(f[t % (kAhead + 1)], t < COLS ? pf : sf, (t < COLS ? dv : dk)[t % COLS / 2].t[t % COLS % 2]);
    }
  };
  int slot = 0, n = 0;           // n: tiles done, from the last one down
  auto run = [&](auto cut_, int to) {
    for (; n < to; n += KS, slot ^= 1) {
      wait_and_meet<0>();
      float number_next = 0.f;
      if (wave < 2) number_next = number();
      const PairLoad<T, DH> next = fetch(slot ^ 1);
      step(cut_, slot, (j1 - 1 - n - ks) * kStep + 32 * rw, next);
      keep(slot ^ 1, number_next);
    }
  };
  // rows that some key does not see only at either end
  const int all_from = cdiv(rows_of(key0 + kKeys - 1).lo, kStep), all_to = rows_of(key0).hi / kStep;
  run(std::true_type{}, min(j1 - all_to, j1 - j0));
  run(std::false_type{}, min(j1 - all_from, j1 - j0) - (KS - 1));
  run(std::true_type{}, j1 - j0);

  drain();
  // the other rows' sums: dk, then dv, through LDS
  f32x4* const shared = reinterpret_cast<f32x4*>(smem) + lane;
  auto place = [&](int set, int d, int i) { return ((set * 2 + kw) * DB * 4 + d * 4 + i) * kWave; };      // set: of the 2 KS - 1 others
  const int set = ks * 2 + rw;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    wait_and_meet<0>();
    if (set > 0)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) shared[place(set - 1, d, i)] = (t ? dv[d] : dk[d]).t[i / 2][i % 2];
    wait_and_meet<0>();
    if (set == 0)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int key = first + 16 * c + x;
        T* const out = t ? static_cast<T*>(g.dv) + (long)(s.k0 + key) * a.v_row + (long)kvh * a.v_head
                         : static_cast<T*>(g.dk) + (long)(s.k0 + key) * a.k_row + (long)kvh * a.k_head;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            f32x4 y = (t ? dv[d] : dk[d]).t[i][c];
#pragma unroll
            for (int o = 0; o < 2 * KS - 1; ++o) y += shared[place(o, d, 2 * i + c)];
            if (t == 0) y *= a.scale;
            const int at = 32 * d + 16 * i + 4 * quad;
            if (key < s.lk && at < a.dim) put4(out + at, y[0], y[1], y[2], y[3]);
          }
      }
  }
}

template <typename T, int DC, int KS> constexpr int kLds = 4 * KS * kStep * Tile<T, tile_dim(DC)>::kRowBytes;
template <typename T, int DC, int KS>
__global__ __launch_bounds__(256 * KS, sizeof(T) == 2 ? 2 : 1) void attn_bwd_q_kernel(const BwdArgs g) {
  __shared__ __align__(1024) char smem[kLds<T, DC, KS>];
  bwd_q<T, DC, KS, true>(g, blockIdx.x / g.a.kv_heads, blockIdx.x % g.a.kv_heads, smem);
}
template <typename T, int DC, int KS>
__global__ __launch_bounds__(256 * KS, sizeof(T) == 2 ? 2 : 1) void attn_bwd_kv_kernel(const BwdArgs g) {
  __shared__ __align__(1024) char smem[kLds<T, DC, KS>];
  __shared__ __align__(16) Stats<KS> stats;
  bwd_kv<T, DC, KS>(g, blockIdx.x / g.a.kv_heads, blockIdx.x % g.a.kv_heads, smem, stats);
}

// Both in one launch, behind one that forms delta: where each by itself leaves CUs empty towards its end, or all along.  Tiles of rows and of keys are dealt out
// evenly, the longest of a sequence first.  fp32, 2760 tokens, 10 / 5 heads of 80, window of 700: 222 to 225 us behind 5 (106 and 135 one after the other); 16 documents
// of 1 to 6011 tokens, 16 / 4 heads of 128: 813 to 879 behind 23, as a profiler sees them one by one; both launches 770 to 825 in a row of calls.
template <typename T, int DC>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attn_bwd_both_kernel(const BwdArgs g) {
  __shared__ __align__(1024) char smem[kLds<T, DC, 1>];
  __shared__ __align__(16) Stats<1> stats;
  const int item = blockIdx.x / g.a.kv_heads, kvh = blockIdx.x % g.a.kv_heads;
  const long all = (long)g.q_tiles + g.k_tiles;
  const int keys = (int)(item * (long)g.k_tiles / all), more = (int)((item + 1) * (long)g.k_tiles / all);      // key tiles ahead of this one, and with it
  if (more > keys) bwd_kv<T, DC, 1>(g, keys, kvh, smem, stats);
  else bwd_q<T, DC, 1, false>(g, item - keys, kvh, smem);
}
// (the same sums in the same order as in bwd_q)
template <typename T, int DC>
__global__ __launch_bounds__(256) void attn_bwd_delta_kernel(const BwdArgs g) {
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 15, quad = lane >> 4, kvh = blockIdx.x % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, blockIdx.x / a.kv_heads, kRows, lane, s, tile, tiles)) return;
  typename Mma<T>::Frag df[kFrags<DC>][2];
  float delta[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const Row row(tile * kRows + wave * 32 + 16 * c + x, s.lq * a.group, a.group, kvh);
    const long token = s.q0 + row.query, at = (token * a.heads + row.head) * a.dim;
#pragma unroll
    for (int kc = 0; kc < kFrags<DC>; ++kc) df[kc][c] = head_frag<T, DC>(static_cast<const T*>(g.d_o) + at, kc, quad, a.dim, row.real);
    delta[c] = delta_of<T, DC>(df, c, static_cast<const T*>(g.o) + at, quad, a.dim, row.real);
    if (row.real && quad == 0) g.delta[(long)row.head * a.q_rows + token] = delta[c];
  }
}

// How many blocks, of both kernels, are launched as one.  The whole backward in two launches takes so many times what it takes in one (means over batches of equal and of
// unequal sequences, 16 / 4 heads of 128 in both types, in fp32 also 10 / 5 of 80 and 12 of 64; the chip holds 256 or 512 blocks):
//      blocks                                        256    512   1024   2048   4000
//      averages of 64 to 768 tokens                 1.35   1.10   1.06   0.97   0.92   (0.45 to 1.36 at 4000: 125 x 128 tokens in fp32 547 in place of 1218 us, where
//                                                                                       tiles of one kind all come to the same CUs)
//      1024 and 2048                                1.38   1.22   1.14   1.05   0.99
//      fp32, 16 heads of 32, 64 to 1024             1.40   1.27   1.17   1.11   1.07
// 1001, 1500 and 259 tokens, 10 / 5 heads of 80 in fp32, window of 700: 247 us in two, 226 in one; 16 documents of 1 to 6011 tokens, 16 / 4 heads of 128 (3200 blocks)
// 820 and 788; 64 of up to 512 (3600) 209 and 224; 16 x 2000, 16 / 4 of 80 in fp32 5640 and 5340; 8 x 4096, 32 / 8 of 128 (12400) 3390 and 3500.
// Short heads in bf16, whose queries' kernel alone has three wavefronts to a SIMD: 2 x 150, 12 heads of 64 (120 blocks) 18 and 15; 8 x 200 (636) 22.5 and 23.3; 32
// documents of up to 1024 158 and 175.
constexpr long kLongAverage = 1000;
template <typename T, int DC>
long together(const AttnShape& a) {
  if (sizeof(T) == 2 && DC <= 64) return 512;
  if (DC > 48 && a.q_rows < kLongAverage * a.n_seq) return 1536;
  return sizeof(T) == 4 ? 1l << 23 : 4096;         // (fp32: what a launch can have)
}

template <typename T, int DC>
int bwd(BwdArgs g, hipStream_t s) {
  const AttnShape& a = g.a;
  const long rows = (long)a.q_rows * a.group;
  g.q_tiles = (int)(a.q_rows > 0 ? rows / kRows + a.n_seq : 0);
  g.k_tiles = (int)(a.k_rows > 0 ? (long)a.k_rows / kKeys + a.n_seq : 0);
  auto grid = [&](long tiles) { return dim3((unsigned)(tiles * a.kv_heads)); };
  if (g.q_tiles > 0 && g.k_tiles > 0 && ((long)g.q_tiles + g.k_tiles) * a.kv_heads <= together<T, DC>(a)) {
    attn_bwd_delta_kernel<T, DC><<<grid(g.q_tiles), dim3(256), 0, s>>>(g);
    attn_bwd_both_kernel<T, DC><<<grid((long)g.q_tiles + g.k_tiles), dim3(256), 0, s>>>(g);
    return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
  }
  // (two sets where launches above the limit can be short of blocks)
  constexpr bool kTwo = kTwoSets<T, DC> && sizeof(T) == 2 && DC <= 64;
  bool two_q = false, two_k = false;
  if constexpr (kTwo) {
    two_q = two_sets(rows / kRows * a.kv_heads, a.k_rows, a.n_seq);
    two_k = two_sets((long)a.k_rows / kKeys * a.kv_heads, rows, a.n_seq);
    if (two_q && g.q_tiles > 0) attn_bwd_q_kernel<T, DC, 2><<<grid(g.q_tiles), dim3(512), 0, s>>>(g);
  }
  if (!two_q && g.q_tiles > 0) attn_bwd_q_kernel<T, DC, 1><<<grid(g.q_tiles), dim3(256), 0, s>>>(g);
  if constexpr (kTwo)
    if (two_k && g.k_tiles > 0) attn_bwd_kv_kernel<T, DC, 2><<<grid(g.k_tiles), dim3(512), 0, s>>>(g);
  if (!two_k && g.k_tiles > 0) attn_bwd_kv_kernel<T, DC, 1><<<grid(g.k_tiles), dim3(256), 0, s>>>(g);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}
template <typename T>
int bwd(const BwdArgs& g, hipStream_t s) {
  const int dim = g.a.dim;
  if constexpr (sizeof(T) == 4) {
    if (dim > 32 && dim <= 48) return bwd<T, 48>(g, s);
    if (dim > 64 && dim <= 80) return bwd<T, 80>(g, s);
    if (dim > 96 && dim <= 112) return bwd<T, 112>(g, s);
  }
  return dim <= 32 ? bwd<T, 32>(g, s) : dim <= 64 ? bwd<T, 64>(g, s) : dim <= 96 ? bwd<T, 96>(g, s) : bwd<T, 128>(g, s);
}

}  // namespace

size_t attn_bwd_scratch_bytes(int, const AttnShape& a) { return (size_t)a.q_rows * a.heads * sizeof(float) + 16; }

int launch_attn_bwd(int dtype, const AttnShape& a, const void* d_o, const void* q, const void* k, const void* v, const void* o, const float* lse, void* dq,
                    void* dk, void* dv, void* scratch, hipStream_t s) {
  const BwdArgs g = {a, d_o, q, k, v, o, lse, dq, dk, dv, static_cast<float*>(scratch), a.scale * kLog2e, 0, 0};
  return dtype == SPES_BF16 ? bwd<bf16_t>(g, s) : bwd<float>(g, s);
}

}  // namespace spes
