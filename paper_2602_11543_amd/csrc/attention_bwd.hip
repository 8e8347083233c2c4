// Attention, backward: the probabilities are formed again from q, k and the forward's lse,
//      p = exp(scale q k^T - lse)      delta = sum do o      ds = p (do v^T - delta)
//      dv = p^T do      dk = scale ds^T q      dq = scale ds k
// Two kernels, so that every sum has one owner and one order: by queries (delta and dq) and by keys (dk and dv, over the rows of all heads that share
// them).  That is 14 D operations a pair for the 10 D of the formulas: s and do v^T are formed twice.
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
};

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attn_bwd_q_kernel(const BwdArgs g) {
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = DH / 16, DB = DH / 32, SLOT = kStep * L::kRowBytes;
  __shared__ __align__(1024) char smem[4 * SLOT];
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, blockIdx.x / a.kv_heads, kRows, lane, s, tile, tiles)) return;
  tile = tiles - 1 - tile;                                   // the longest first

  const int G = a.group, n_rows = s.lq * G, r0 = tile * kRows, row = r0 + wave * 32 + x;
  const int query = min(row, n_rows - 1) / G, head = kvh * G + min(row, n_rows - 1) % G;
  const bool real = row < n_rows;
  const Reach mine = reach(a, s, query);
  const int last = min(r0 + kRows, n_rows) - 1;
  const int lo = reach(a, s, r0 / G).lo, hi = reach(a, s, last / G).hi;
  const int w_first = min(r0 + wave * 32, n_rows - 1) / G, w_last = min(r0 + wave * 32 + 31, n_rows - 1) / G;
  const Reach w0 = reach(a, s, w_first), w1 = reach(a, s, w_last);
  const bool w_real = r0 + wave * 32 < n_rows;
  const int j0 = lo / kStep, j1 = hi > lo ? cdiv(hi, kStep) : j0;
  const long token = s.q0 + query;

  Frag qf[KC], df[KC];
  float delta = 0.f;
  {
    const T* const qp = static_cast<const T*>(g.q) + token * a.q_row + (long)head * a.q_head + 8 * half;
    const long at = (token * a.heads + head) * a.dim + 8 * half;
    const T* const dp = static_cast<const T*>(g.d_o) + at;
    const T* const op = static_cast<const T*>(g.o) + at;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const bool in = real && 16 * kc + 8 * half < a.dim;
      qf[kc] = in ? Mma<T>::load(qp + 16 * kc) : Mma<T>::zero();
      df[kc] = in ? Mma<T>::load(dp + 16 * kc) : Mma<T>::zero();
    }
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const Frag of = real && 16 * kc + 8 * half < a.dim ? Mma<T>::load(op + 16 * kc) : Mma<T>::zero();
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(Mma<T>::get(df[kc], j), Mma<T>::get(of, j), delta);
    }
  }
  delta = both_sum(delta);
  if (real && half == 0) g.delta[(long)head * a.q_rows + token] = delta;

  const long stride[2] = {a.k_row * ES, a.v_row * ES};
  const unsigned long source[2] = {(unsigned long)g.k + (unsigned long)(s.k0 * stride[0] + (long)kvh * a.k_head * ES),
                                   (unsigned long)g.v + (unsigned long)(s.k0 * stride[1] + (long)kvh * a.v_head * ES)};
  const unsigned lds0 = lds_address(smem);
  unsigned off[2][L::kLoads];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < L::kLoads; ++n) off[i][n] = L::load_off(wave, n, lane, stride[i], a.dim);
  auto fetch = [&](int j, int slot) { return PairLoad<T, DH>(off, source, stride, s.lk, j, lds0 + (unsigned)(slot * 2 * SLOT), wave); };
  constexpr int PER = PairLoad<T, DH>::kPieces / KC;

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
  float base = g.lse[(long)head * a.q_rows + token] * kLog2e;
  settle(qf);
  settle(df);
  settle(base);
  settle(delta);
  if (j0 < j1) fetch(j0, 0).all();
  int slot = 0;
  for (int j = j0; j < j1; ++j, slot ^= 1) {
    wait_and_meet<0>();
    const int key0 = j * kStep;
    const PairLoad<T, DH> next = fetch(j + 1 < j1 ? j + 1 : kNone, slot ^ 1);
    if (!w_real || key0 >= w1.hi || key0 + kStep <= w0.lo) {
      next.all();
      continue;
    }
    const bool cut = key0 < w1.lo || key0 + kStep > w0.hi;
    const int from = mine.lo - key0 - 4 * half, to = mine.hi - key0 - 4 * half;
    const char* const ks = smem + slot * 2 * SLOT;
    const char* const vs = ks + SLOT;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      f32x16 sc = f32x16{}, ds;
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] = -delta;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        sc = Mma<T>::mma(L::row_frag(ks, rb, n, kc), qf[kc], sc);
        ds = Mma<T>::mma(L::row_frag(vs, rb, n, kc), df[kc], ds);
        if (n == 0)
#pragma unroll
          for (int p = 0; p < PER; ++p) next.piece(PER * kc + p);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] *= exp2_(fmaf(sc[i], g.c, -base));
      if (cut) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 32 * n + 8 * (i / 4) + i % 4;
          if (at < from || at >= to) ds[i] = 0.f;
        }
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const Frag f = Mma<T>::of(ds, kk);
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = Mma<T>::mma(L::col_frag(ks, cb, d, 2 * n + kk), f, acc[d]);
      }
    }
  }
  drain();
  if (!real) return;
  T* const dq = static_cast<T*>(g.dq) + token * a.q_row + (long)head * a.q_head;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 32 * d + 8 * i + 4 * half;
      if (at < a.dim) put4(dq + at, acc[d][4 * i] * a.scale, acc[d][4 * i + 1] * a.scale, acc[d][4 * i + 2] * a.scale, acc[d][4 * i + 3] * a.scale);
    }
}

// Four wavefronts, two by two: two groups of NB x 32 keys, and in each one wavefront for the first 32 of the 64 rows that are in LDS and one for the
// others, whose sums are joined at the end.
template <typename T, int DH>
struct KvTile {
  static constexpr int NB = 1, kKeys = 2 * NB * 32;
  static constexpr bool kValuesInLds = false;      // dk, dv and the keys take 320 of a lane's 512 registers, the values would take 64
};

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attn_bwd_kv_kernel(const BwdArgs g) {
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = DH / 16, DB = DH / 32, SLOT = kStep * L::kRowBytes, NB = KvTile<T, DH>::NB, KEYS = KvTile<T, DH>::kKeys;
  __shared__ __align__(1024) char smem[4 * SLOT];
  constexpr bool V_LDS = KvTile<T, DH>::kValuesInLds;
  __shared__ __align__(1024) char values[V_LDS ? KEYS * L::kRowBytes : 16];
  __shared__ __align__(16) float stats[2][2][kStep];         // of each slot's rows: -lse / scale (fp32: -lse log2 e), -delta
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 31, half = lane >> 5, kw = wave & 1, rw = wave >> 1;
  const int kvh = blockIdx.x % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<true>(a, blockIdx.x / a.kv_heads, KEYS, lane, s, tile, tiles)) return;

  const int G = a.group, n_rows = s.lq * G, key0 = tile * KEYS, first = key0 + kw * NB * 32, tail = s.lk - 1;
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
  const int lo = rows_of(key0).lo, hi = rows_of(key0 + KEYS - 1).hi;
  const int j0 = lo / kStep, j1 = hi > lo ? cdiv(hi, kStep) : j0;

  Frag kf[NB][KC], vf[NB][V_LDS ? 1 : KC];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int key = min(first + 32 * b + x, tail);
    const T* const kp = static_cast<const T*>(g.k) + (long)(s.k0 + key) * a.k_row + (long)kvh * a.k_head + 8 * half;
    const T* const vp = static_cast<const T*>(g.v) + (long)(s.k0 + key) * a.v_row + (long)kvh * a.v_head + 8 * half;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const bool in = 16 * kc + 8 * half < a.dim;
      kf[b][kc] = in ? Mma<T>::load(kp + 16 * kc) : Mma<T>::zero();
      if constexpr (!V_LDS) vf[b][kc] = in ? Mma<T>::load(vp + 16 * kc) : Mma<T>::zero();
    }
  }

  // rows on their way into LDS: row r of a tile is query r / G, head r % G.  Rows behind the last one repeat it (their probabilities are nothing)
  const unsigned long q_base = (unsigned long)g.q + (unsigned long)((long)s.q0 * a.q_row + (long)kvh * G * a.q_head) * ES;
  const unsigned long d_base = (unsigned long)g.d_o + (unsigned long)(((long)s.q0 * a.heads + (long)kvh * G) * a.dim) * ES;
  const unsigned lds0 = lds_address(smem);
  const unsigned magic = (1u << 22) / (unsigned)G + 1;       // n / G = n magic >> 22 for n < 64 + G, G <= 1024
  unsigned off[2][L::kLoads];
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
  auto fetch = [&](int j, int slot, bool there) {
    const int r0 = j * kStep, query = r0 / G, rem = r0 - query * G;
    if (there && (j == j0 || rem != 0 || kStep % G != 0 || r0 + kStep > n_rows)) aim(rem, n_rows - r0);
    return PairLoad<T, DH>(off, rsrc_for_lds(q_base + (unsigned long)((long)query * a.q_row * ES), there ? kOpen : 0u),
                           rsrc_for_lds(d_base + (unsigned long)((long)query * a.heads * a.dim * ES), there ? kOpen : 0u), lds0 + (unsigned)(slot * 2 * SLOT), wave);
  };
  constexpr int PER = PairLoad<T, DH>::kPieces / KC;
  // one row's number to a lane of the first two wavefronts, on its way while the step before is worked on
  auto number = [&](int j) {
    const int r = j * kStep + lane;
    if (r >= n_rows) return wave == 0 ? -INFINITY : 0.f;
    const long at = (long)(kvh * G + r % G) * a.q_rows + s.q0 + r / G;
    return wave == 0 ? g.lse[at] : -g.delta[at];
  };
  auto keep = [&](int slot, float v) {
    if (wave == 0) v = v == -INFINITY ? -INFINITY : ES == 2 ? -v / a.scale : -v * kLog2e;      // a row without keys has no probabilities
    if (wave < 2) stats[slot][wave][lane] = v;
  };

  f32x16 dk[NB][DB], dv[NB][DB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[b][d] = dv[b][d] = f32x16{};
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    settle(kf[b]);
    if constexpr (!V_LDS) settle(vf[b]);
  }
  if constexpr (V_LDS)
#pragma unroll
    for (int t = 0; t < KEYS / kStep; ++t)
      L::load_rows((unsigned long)g.v + (unsigned long)(((long)(s.k0 + key0 + t * kStep) * a.v_row + (long)kvh * a.v_head) * ES), a.v_row * ES,
                   s.lk - key0 - t * kStep, a.dim, lds_address(values) + (unsigned)(t * SLOT), wave, lane);
  if (j0 < j1) {
    fetch(j0, 0, true).all();
    if (wave < 2) keep(0, number(j0));
  }

  // 32 rows against the wavefront's keys
  auto step = [&](auto cut_, int slot, int r0, const PairLoad<T, DH>& next) {
    constexpr bool CUT = decltype(cut_)::value;
    const char* const qs = smem + slot * 2 * SLOT;
    const char* const dos = qs + SLOT;
    const float* const st = &stats[slot][0][32 * rw + 4 * half];
    f32x16 p[NB], ds[NB];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 u = *reinterpret_cast<const float4*>(st + 8 * i), w = *reinterpret_cast<const float4*>(st + kStep + 8 * i);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (ES == 2) { p[b][4 * i] = u.x; p[b][4 * i + 1] = u.y; p[b][4 * i + 2] = u.z; p[b][4 * i + 3] = u.w; }
        ds[b][4 * i] = w.x; ds[b][4 * i + 1] = w.y; ds[b][4 * i + 2] = w.z; ds[b][4 * i + 3] = w.w;
      }
    }
    if (ES != 2)
#pragma unroll
      for (int b = 0; b < NB; ++b) p[b] = f32x16{};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const Frag f = L::row_frag(qs, rb, rw, kc);
#pragma unroll
      for (int b = 0; b < NB; ++b) p[b] = Mma<T>::mma(f, kf[b][kc], p[b]);
#pragma unroll
      for (int i = 0; i < PER; ++i) next.piece(PER * kc + i);
    }
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const Frag f = L::row_frag(dos, rb, rw, kc);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if constexpr (V_LDS) ds[b] = Mma<T>::mma(f, L::row_frag(values, rb, kw * NB + b, kc), ds[b]);
        else ds[b] = Mma<T>::mma(f, vf[b][kc], ds[b]);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      // (bf16: the products are summed on top of -lse / scale; in fp32 storage that would round them to its magnitude)
      if constexpr (ES == 2) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[b][i] = exp2_(p[b][i] * g.c);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 u = *reinterpret_cast<const float4*>(st + 8 * i);
          p[b][4 * i] = exp2_(fmaf(p[b][4 * i], g.c, u.x));
          p[b][4 * i + 1] = exp2_(fmaf(p[b][4 * i + 1], g.c, u.y));
          p[b][4 * i + 2] = exp2_(fmaf(p[b][4 * i + 2], g.c, u.z));
          p[b][4 * i + 3] = exp2_(fmaf(p[b][4 * i + 3], g.c, u.w));
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[b][i] *= p[b][i];
      if constexpr (CUT) {
        const Reach mine = rows_of(first + 32 * b + x);
        const int from = mine.lo - r0 - 4 * half, to = mine.hi - r0 - 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 8 * (i / 4) + i % 4;
          if (at < from || at >= to) p[b][i] = ds[b][i] = 0.f;
        }
      }
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      Frag f[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) f[b] = Mma<T>::of(p[b], kk);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const Frag c = L::col_frag(dos, cb, d, 2 * rw + kk);
#pragma unroll
        for (int b = 0; b < NB; ++b) dv[b][d] = Mma<T>::mma(c, f[b], dv[b][d]);
      }
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      Frag f[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) f[b] = Mma<T>::of(ds[b], kk);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const Frag c = L::col_frag(qs, cb, d, 2 * rw + kk);
#pragma unroll
        for (int b = 0; b < NB; ++b) dk[b][d] = Mma<T>::mma(c, f[b], dk[b][d]);
      }
    }
  };
  int slot = 0, j = j0;
  auto run = [&](auto cut_, int to) {
    for (; j < to; ++j, slot ^= 1) {
      wait_and_meet<0>();
      const bool more = j + 1 < j1;
      float number_next = 0.f;
      if (more && wave < 2) number_next = number(j + 1);
      step(cut_, slot, j * kStep + 32 * rw, fetch(j + 1, slot ^ 1, more));
      if (more && wave < 2) keep(slot ^ 1, number_next);
    }
  };
  // rows that some key does not see only at either end
  const int all_from = cdiv(rows_of(key0 + KEYS - 1).lo, kStep), all_to = rows_of(key0).hi / kStep;
  run(std::true_type{}, min(max(all_from, j0), j1));
  run(std::false_type{}, min(max(all_to, j), j1));
  run(std::true_type{}, j1);

  // the other rows' sums: dk, then dv, through LDS
  const float scale = a.scale;
  T* const out[2] = {static_cast<T*>(g.dk) + (long)s.k0 * a.k_row + (long)kvh * a.k_head, static_cast<T*>(g.dv) + (long)s.k0 * a.v_row + (long)kvh * a.v_head};
  const long row[2] = {a.k_row, a.v_row};
  float4* const other = reinterpret_cast<float4*>(smem) + kw * NB * DB * 4 * kWave + lane;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    wait_and_meet<0>();
    if (rw == 1)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x16& v = t ? dv[b][d] : dk[b][d];
            other[((b * DB + d) * 4 + i) * kWave] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
    wait_and_meet<0>();
    if (rw == 0)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int key = first + 32 * b + x;
        T* const to = out[t] + key * row[t];
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x16& v = t ? dv[b][d] : dk[b][d];
            const float4 u = other[((b * DB + d) * 4 + i) * kWave];
            const float f = t ? 1.f : scale;
            const int at = 32 * d + 8 * i + 4 * half;
            if (key < s.lk && at < a.dim) put4(to + at, (v[4 * i] + u.x) * f, (v[4 * i + 1] + u.y) * f, (v[4 * i + 2] + u.z) * f, (v[4 * i + 3] + u.w) * f);
          }
      }
  }
}

template <typename T, int DH>
int bwd(const BwdArgs& g, hipStream_t s) {
  const AttnShape& a = g.a;
  if (a.q_rows > 0) attn_bwd_q_kernel<T, DH><<<dim3((unsigned)(((long)a.q_rows * a.group / kRows + a.n_seq) * a.kv_heads)), dim3(256), 0, s>>>(g);
  if (a.k_rows > 0) attn_bwd_kv_kernel<T, DH><<<dim3((unsigned)(((long)a.k_rows / KvTile<T, DH>::kKeys + a.n_seq) * a.kv_heads)), dim3(256), 0, s>>>(g);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

}  // namespace

size_t attn_bwd_scratch_bytes(int, const AttnShape& a) { return (size_t)a.q_rows * a.heads * sizeof(float) + 16; }

int launch_attn_bwd(int dtype, const AttnShape& a, const void* d_o, const void* q, const void* k, const void* v, const void* o, const float* lse, void* dq,
                    void* dk, void* dv, void* scratch, hipStream_t s) {
  const BwdArgs g = {a, d_o, q, k, v, o, lse, dq, dk, dv, static_cast<float*>(scratch), a.scale * kLog2e};
  if (dtype == SPES_BF16) return a.dim <= 64 ? bwd<bf16_t, 64>(g, s) : bwd<bf16_t, 128>(g, s);
  return a.dim <= 64 ? bwd<float, 64>(g, s) : bwd<float, 128>(g, s);
}

}  // namespace spes
