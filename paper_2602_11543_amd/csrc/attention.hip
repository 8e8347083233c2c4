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
  int parts;
  float c;              // scale log2 e: exponentials are of base two
};

constexpr int kJoinRows = 4, kMaxParts = 32;
constexpr float kLazy = 8.f;      // the running maximum is raised, and what has been summed is scaled, once a score passes it by 2^8

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attn_fwd_kernel(const FwdArgs g) {
  typedef Tile<T, DH> L;
  typedef typename Mma<T>::Frag Frag;
  constexpr int ES = sizeof(T), KC = DH / 16, DB = DH / 32, SLOT = kStep * L::kRowBytes;
  __shared__ __align__(1024) char smem[4 * SLOT];            // keys and values, two of each
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), x = lane & 31, half = lane >> 5;
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
  int j0 = lo / kStep, j1 = hi > lo ? cdiv(hi, kStep) : j0;
  {
    const int n = j1 - j0, from = (int)((long)n * part / g.parts), to = (int)((long)n * (part + 1) / g.parts);
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
  auto fetch = [&](int j, int slot) { return PairLoad<T, DH>(off, base, stride, s.lk, j, lds0 + (unsigned)(slot * 2 * SLOT), wave); };
  constexpr int PER = PairLoad<T, DH>::kPieces / KC;

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  float m = -INFINITY, l[4] = {0.f, 0.f, 0.f, 0.f};             // of this lane's row, in units of log2; l: this half's share
  const unsigned rb = L::row_base(lane), cb = L::col_base(lane);
  settle(qf);
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
    const char* const ks = smem + slot * 2 * SLOT;
    const char* const vs = ks + SLOT;
    f32x16 sc[2] = {f32x16{}, f32x16{}};
    Frag kf[3][2];             // read two steps ahead
#pragma unroll
    for (int kc = 0; kc < 2; ++kc)
#pragma unroll
      for (int n = 0; n < 2; ++n) kf[kc][n] = L::row_frag(ks, rb, n, kc);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      if (kc + 2 < KC)
#pragma unroll
        for (int n = 0; n < 2; ++n) kf[(kc + 2) % 3][n] = L::row_frag(ks, rb, n, kc + 2);
#pragma unroll
      for (int n = 0; n < 2; ++n) sc[n] = Mma<T>::mma(kf[kc % 3][n], qf[kc], sc[n]);
#pragma unroll
      for (int p = 0; p < PER; ++p) next.piece(PER * kc + p);
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
      for (int d = 0; d < DB; ++d) acc[d] = Mma<T>::mma(L::col_frag(vs, cb, d, kk), p, acc[d]);
    }
  }

  drain();
  const float sum = both_sum((l[0] + l[1]) + (l[2] + l[3]));
  if (!real) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum, lse = (m + log2f(sum)) * kLn2;
  const long token = s.q0 + query;
  if (g.parts > 1) {
    float* const op = g.part_o + (((long)part * a.q_rows + token) * a.heads + head) * a.dim;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 32 * d + 8 * i + 4 * half;
        if (at < a.dim) *reinterpret_cast<float4*>(op + at) = make_float4(acc[d][4 * i] * inv, acc[d][4 * i + 1] * inv, acc[d][4 * i + 2] * inv, acc[d][4 * i + 3] * inv);
      }
    if (half == 0) g.part_lse[((long)part * a.heads + head) * a.q_rows + token] = lse;
    return;
  }
  T* const op = static_cast<T*>(g.o) + (token * a.heads + head) * a.dim;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 32 * d + 8 * i + 4 * half;
      if (at < a.dim) put4(op + at, acc[d][4 * i] * inv, acc[d][4 * i + 1] * inv, acc[d][4 * i + 2] * inv, acc[d][4 * i + 3] * inv);
    }
  if (half == 0) g.lse[(long)head * a.q_rows + token] = lse;
}

// The parts of a row's keys joined: weights exp(lse_p - lse).  A wavefront to a row, two elements to a lane.
template <typename T>
__global__ __launch_bounds__(256) void attn_join_kernel(const FwdArgs g) {
  const AttnShape& a = g.a;
  const int lane = threadIdx.x & 63, kvh = blockIdx.x % a.kv_heads;
  Seq s;
  int tile, tiles;
  if (!find_tile<false>(a, blockIdx.x / a.kv_heads, kJoinRows, lane, s, tile, tiles)) return;
  const int row = tile * kJoinRows + (int)(threadIdx.x >> 6);
  if (row >= s.lq * a.group) return;
  const int head = kvh * a.group + row % a.group;
  const long token = s.q0 + row / a.group;
  const float mine = lane < g.parts ? g.part_lse[((long)lane * a.heads + head) * a.q_rows + token] : -INFINITY;
  const float top = wave_max(mine), w = top == -INFINITY ? 0.f : exp2_((mine - top) * kLog2e), sum = wave_sum(w);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (lane == 0) g.lse[(long)head * a.q_rows + token] = top + log2f(sum) * kLn2;
  const int d = 2 * lane;
  if (d >= a.dim) return;
  const float* const op = g.part_o + (token * a.heads + head) * a.dim + d;
  const long step = (long)a.q_rows * a.heads * a.dim;
  float y0 = 0.f, y1 = 0.f;
  for (int p = 0; p < g.parts; ++p) {
    const float2 o = *reinterpret_cast<const float2*>(op + p * step);
    const float f = lane_value(w, p);
    y0 = fmaf(f, o.x, y0);
    y1 = fmaf(f, o.y, y1);
  }
  put2(static_cast<T*>(g.o) + (token * a.heads + head) * a.dim + d, y0 * inv, y1 * inv);
}

// Parts that the keys of every tile are cut into, so that few rows against many keys fill the chip: two blocks to a CU, 256 keys at least to a part
int key_parts(const AttnShape& a) {
  if (a.n_seq == 0 || a.q_rows == 0) return 1;
  const long tiles = std::max<long>(cdiv((long)a.q_rows * a.group, kRows), std::min(a.n_seq, a.q_rows)) * a.kv_heads, keys = a.k_rows / a.n_seq;
  return (int)std::max<long>(1, std::min<long>({kMaxParts, 512 / tiles, keys / 256}));
}

template <typename T, int DH>
int fwd(const FwdArgs& g, hipStream_t s) {
  const AttnShape& a = g.a;
  const long n = (long)a.q_rows * a.group;
  attn_fwd_kernel<T, DH><<<dim3((unsigned)((n / kRows + a.n_seq) * a.kv_heads * g.parts)), dim3(256), 0, s>>>(g);
  if (g.parts > 1) attn_join_kernel<T><<<dim3((unsigned)((n / kJoinRows + a.n_seq) * a.kv_heads)), dim3(256), 0, s>>>(g);
  return hipGetLastError() == hipSuccess ? SPES_OK : SPES_EHIP;
}

}  // namespace

size_t attn_fwd_scratch_bytes(int, const AttnShape& a) {
  const int parts = key_parts(a);
  return parts == 1 ? 16 : (size_t)parts * a.q_rows * a.heads * (a.dim + 1) * sizeof(float) + 16;
}

int launch_attn_fwd(int dtype, const AttnShape& a, const void* q, const void* k, const void* v, void* o, float* lse, void* scratch, hipStream_t s) {
  FwdArgs g = {a, q, k, v, o, lse, nullptr, nullptr, key_parts(a), a.scale * kLog2e};
  g.part_o = static_cast<float*>(scratch);
  g.part_lse = g.part_o + (size_t)g.parts * a.q_rows * a.heads * a.dim;
  if (dtype == SPES_BF16) return a.dim <= 64 ? fwd<bf16_t, 64>(g, s) : fwd<bf16_t, 128>(g, s);
  return a.dim <= 64 ? fwd<float, 64>(g, s) : fwd<float, 128>(g, s);
}

}  // namespace spes
