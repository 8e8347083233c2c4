// Attention, backward: the probabilities are formed again from q, k and the forward's lse,
//      p = exp(scale q k^T - lse)      delta = sum do o      ds = p (do v^T - delta)
//      dv = p^T do      dk = scale ds^T q      dq = scale ds k
// Two kernels, so that every sum has one owner and one order: by queries (delta and dq) and by keys (dk and dv, over the rows of all heads that share
// them).  That is 14 D operations a pair for the 10 D of the formulas: s and do v^T are formed twice.
#include <algorithm>

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
  const float base = g.lse[(long)head * a.q_rows + token] * kLog2e;

  const unsigned long k_base = (unsigned long)g.k + (unsigned long)((long)s.k0 * a.k_row + (long)kvh * a.k_head) * ES;
  const unsigned long v_base = (unsigned long)g.v + (unsigned long)((long)s.k0 * a.v_row + (long)kvh * a.v_head) * ES;
  const unsigned lds0 = lds_address(smem);
  unsigned k_off[L::kLoads], v_off[L::kLoads];
#pragma unroll
  for (int i = 0; i < L::kLoads; ++i) {
    k_off[i] = L::load_off(wave, i, lane, a.k_row, a.dim);
    v_off[i] = L::load_off(wave, i, lane, a.v_row, a.dim);
  }
  auto load = [&](int j, int slot) {
    L::load_rows(k_base, j, a.k_row, s.lk, k_off, lds0 + (unsigned)(slot * 2 * SLOT), wave, lane);
    L::load_rows(v_base, j, a.v_row, s.lk, v_off, lds0 + (unsigned)(slot * 2 * SLOT + SLOT), wave, lane);
  };

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
  if (j0 < j1) load(j0, 0);
  int slot = 0;
  for (int j = j0; j < j1; ++j, slot ^= 1) {
    wait_and_meet<0>();
    if (j + 1 < j1) load(j + 1, slot ^ 1);
    const int key0 = j * kStep;
    if (!w_real || key0 >= w1.hi || key0 + kStep <= w0.lo) continue;
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

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attn_bwd_kv_kernel(const BwdArgs g) {
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = DH / 16, DB = DH / 32, SLOT = kStep * L::kRowBytes;
  __shared__ __align__(1024) char smem[4 * SLOT];
  __shared__ __align__(16) float stats[2][2][kStep];         // of each slot's rows: -lse / scale, -delta
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<true>(a, blockIdx.x / a.kv_heads, kRows, lane, s, tile, tiles)) return;

  const int G = a.group, n_rows = s.lq * G, key0 = tile * kRows, first = key0 + wave * 32, key = first + x;
  const bool real = key < s.lk;
  // Rows [from, to) see a key: with causal masks r / G + lk - lq >= key, hence r >= (key - (lk - lq)) G, and likewise for the window
  auto rows_of = [&](int at) {
    Reach r = {0, n_rows};
    if (a.causal) {
      const long first_query = (long)at - (s.lk - s.lq), end = a.window > 0 ? min(first_query + a.window, (long)s.lq) : (long)s.lq;
      r.lo = (int)max(first_query, 0l) * G;
      r.hi = (int)max(end, 0l) * G;
    }
    return r;
  };
  const int tail = s.lk - 1;
  const Reach mine = rows_of(min(key, tail)), w0 = rows_of(min(first, tail)), w1 = rows_of(min(first + 31, tail));      // some: [w0.lo, w1.hi), all: [w1.lo, w0.hi)
  const int lo = rows_of(key0).lo, hi = rows_of(min(key0 + kRows - 1, tail)).hi;
  const bool w_real = first < s.lk;
  const int j0 = lo / kStep, j1 = hi > lo ? cdiv(hi, kStep) : j0;

  Frag kf[KC], vf[KC];
  {
    const T* const kp = static_cast<const T*>(g.k) + (long)(s.k0 + min(key, tail)) * a.k_row + (long)kvh * a.k_head + 8 * half;
    const T* const vp = static_cast<const T*>(g.v) + (long)(s.k0 + min(key, tail)) * a.v_row + (long)kvh * a.v_head + 8 * half;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const bool in = real && 16 * kc + 8 * half < a.dim;
      kf[kc] = in ? Mma<T>::load(kp + 16 * kc) : Mma<T>::zero();
      vf[kc] = in ? Mma<T>::load(vp + 16 * kc) : Mma<T>::zero();
    }
  }

  const unsigned long q_base = (unsigned long)g.q + (unsigned long)((long)s.q0 * a.q_row + (long)kvh * G * a.q_head) * ES;
  const unsigned long d_base = (unsigned long)g.d_o + (unsigned long)(((long)s.q0 * a.heads + (long)kvh * G) * a.dim) * ES;
  const unsigned lds0 = lds_address(smem);
  const unsigned magic = (1u << 22) / (unsigned)G + 1;       // n / G = n magic >> 22 for n < 64 + G, G <= 1024
  const unsigned q_row = (unsigned)(a.q_row * ES), q_head = (unsigned)(a.q_head * ES), d_row = (unsigned)(a.heads * a.dim * ES), d_head = (unsigned)(a.dim * ES);
  auto load = [&](int j, int slot) {
    const int r0 = j * kStep, query = r0 / G, rem = r0 - query * G;
    const rsrc_t rq = open_rsrc(q_base + (unsigned long)((long)query * a.q_row * ES)), rd = open_rsrc(d_base + (unsigned long)((long)query * a.heads * a.dim * ES));
    const unsigned dst = lds0 + (unsigned)(slot * 2 * SLOT + wave * L::kLoads * 1024);
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      const int r = L::load_row(wave, i, lane), ch = L::load_chunk(r, lane);
      const unsigned n = (unsigned)(r + rem), q = n * magic >> 22, h = n - q * G;
      const bool in = r0 + r < n_rows && ch * (16 / ES) < a.dim;
      const unsigned q_off = in ? q * q_row + h * q_head + ch * 16 : kOutOfRange, d_off = in ? q * d_row + h * d_head + ch * 16 : kOutOfRange;
      const unsigned m = set_lds_dest(uniform(dst + i * 1024));
      one_instruction();
      load_to_lds(rq, q_off, m);
      const unsigned m2 = set_lds_dest(uniform(dst + SLOT + i * 1024));
      one_instruction();
      load_to_lds(rd, d_off, m2);
    }
  };
  // one row's number to a lane of the first two wavefronts, on its way while the step before is worked on
  auto number = [&](int j) {
    const int r = j * kStep + lane;
    if (r >= n_rows) return wave == 0 ? -INFINITY : 0.f;
    const long at = (long)(kvh * G + r % G) * a.q_rows + s.q0 + r / G;
    return wave == 0 ? -g.lse[at] / a.scale : -g.delta[at];
  };

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = dv[d] = f32x16{};
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
  if (j0 < j1) {
    load(j0, 0);
    if (wave < 2) {
      const float v = number(j0);
      stats[0][wave][lane] = wave == 0 && v == INFINITY ? -INFINITY : v;      // a row without keys has no probabilities
    }
  }
  int slot = 0;
  for (int j = j0; j < j1; ++j, slot ^= 1) {
    wait_and_meet<0>();
    float next = 0.f;
    if (j + 1 < j1) {
      if (wave < 2) next = number(j + 1);
      load(j + 1, slot ^ 1);
    }
    const int r0 = j * kStep;
    if (w_real && r0 < w1.hi && r0 + kStep > w0.lo) {
      const bool cut = r0 < w1.lo || r0 + kStep > w0.hi;
      const int from = mine.lo - r0 - 4 * half, to = mine.hi - r0 - 4 * half;
      const char* const qs = smem + slot * 2 * SLOT;
      const char* const dos = qs + SLOT;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        f32x16 p, ds;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 u = *reinterpret_cast<const float4*>(&stats[slot][0][32 * n + 8 * i + 4 * half]);
          const float4 w = *reinterpret_cast<const float4*>(&stats[slot][1][32 * n + 8 * i + 4 * half]);
          p[4 * i] = u.x; p[4 * i + 1] = u.y; p[4 * i + 2] = u.z; p[4 * i + 3] = u.w;
          ds[4 * i] = w.x; ds[4 * i + 1] = w.y; ds[4 * i + 2] = w.z; ds[4 * i + 3] = w.w;
        }
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          p = Mma<T>::mma(L::row_frag(qs, rb, n, kc), kf[kc], p);
          ds = Mma<T>::mma(L::row_frag(dos, rb, n, kc), vf[kc], ds);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          p[i] = exp2_(p[i] * g.c);
          ds[i] *= p[i];
        }
        if (cut) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int at = 32 * n + 8 * (i / 4) + i % 4;
            if (at < from || at >= to) p[i] = ds[i] = 0.f;
          }
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const Frag pf = Mma<T>::of(p, kk), sf = Mma<T>::of(ds, kk);
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            dv[d] = Mma<T>::mma(L::col_frag(dos, cb, d, 2 * n + kk), pf, dv[d]);
            dk[d] = Mma<T>::mma(L::col_frag(qs, cb, d, 2 * n + kk), sf, dk[d]);
          }
        }
      }
    }
    if (j + 1 < j1 && wave < 2) stats[slot ^ 1][wave][lane] = wave == 0 && next == INFINITY ? -INFINITY : next;
  }
  if (!real) return;
  T* const dkp = static_cast<T*>(g.dk) + (long)(s.k0 + key) * a.k_row + (long)kvh * a.k_head;
  T* const dvp = static_cast<T*>(g.dv) + (long)(s.k0 + key) * a.v_row + (long)kvh * a.v_head;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 32 * d + 8 * i + 4 * half;
      if (at < a.dim) {
        put4(dkp + at, dk[d][4 * i] * a.scale, dk[d][4 * i + 1] * a.scale, dk[d][4 * i + 2] * a.scale, dk[d][4 * i + 3] * a.scale);
        put4(dvp + at, dv[d][4 * i], dv[d][4 * i + 1], dv[d][4 * i + 2], dv[d][4 * i + 3]);
      }
    }
}

template <typename T, int DH>
int bwd(const BwdArgs& g, hipStream_t s) {
  const AttnShape& a = g.a;
  if (a.q_rows > 0) attn_bwd_q_kernel<T, DH><<<dim3((unsigned)(((long)a.q_rows * a.group / kRows + a.n_seq) * a.kv_heads)), dim3(256), 0, s>>>(g);
  if (a.k_rows > 0) attn_bwd_kv_kernel<T, DH><<<dim3((unsigned)(((long)a.k_rows / kRows + a.n_seq) * a.kv_heads)), dim3(256), 0, s>>>(g);
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
