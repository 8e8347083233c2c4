// What the attention kernels share: how a problem is cut into tiles, tiles in LDS, operand fragments of the 16 x 16 matrix instructions.
//
// Rows.  The heads that share keys stand side by side: row r of a sequence is query r / G under head kvh * G + r % G, G = heads / kv_heads, so a tile of rows
// meets every key once for all of them, and a sum over the rows is one over the heads as well.
//
// Orientation.  Scores are formed as S^T = K Q^T (queries' kernels: keys down, rows across) or S = Q K^T (keys' kernel), 32 x 32 at a time as two by two
// tiles, so that a lane (x = lane % 16, quad = lane / 16) holds of two columns, 16 j + x, the eight scores 16 i + 4 quad + 0..3.  The contraction that follows
// runs over just these: as its order is free, a column's eight are the lane's operand fragment as they stand, and the other operand is read from
// LDS in the same order.
//
// Why 16 x 16 x 32 and not 32 x 32 x 16: what bounds the large cases is power (32 heads of 128, 8 x 4096 tokens, call after call: the clock falls from 2.4 to
// 1.5 GHz), and the smaller form moves half as many accumulators per multiply-add: backward of that, when it was taken, 3.75 -> 3.65 ms, forward 1.13 -> 1.12;
// 2 x 2048 tokens, 12 heads of 64, forward 33 -> 30 us.
//
// Operands in bf16 storage are bf16: probabilities and their gradient are rounded once, by at most 2^-8 of each, on their way into the products that sum them in
// fp32, for the rate of bf16 products, which is eight times that of fp32 ones.  o is then 1.9e-3 to 2.4e-3 off (in norm), dq and dk 2.5e-3, where rounding the exact
// ones to bf16 leaves 1.7e-3; nearly all of it is the one rounding of the gradient.
#pragma once
#include <algorithm>

#include "lds_load.h"
#include "kernels.h"

namespace spes {
namespace attn {

constexpr int kRows = 128;       // rows of a block of four wavefronts, 32 each
constexpr int kStep = 64;        // keys (rows, in the keys' kernel) that pass through LDS at a time
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct f32x8 { float v[8]; };
struct Acc { f32x4 t[2][2]; };       // 32 x 32: tile (i, j)

// Sixteen bytes of device memory; the address space is said, since a flat load would be waited for as a read of LDS as well
__device__ __forceinline__ f32x4 load_global(const void* p) { return *(const __attribute__((address_space(1))) f32x4*)p; }

// A fragment is 32 of the contraction for one row or column of sixteen: eight elements of each quarter of the lanes
template <typename T> struct Mma;
template <> struct Mma<bf16_t> {
  typedef bf16x8 Frag;
  static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, const f32x4& c, bool = false) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ Frag zero() { return __builtin_bit_cast(Frag, make_uint4(0, 0, 0, 0)); }
  static __device__ __forceinline__ Frag load(const bf16_t* p) { return __builtin_bit_cast(Frag, load_global(p)); }
  // a column's eight results, rounded to the operands' type
  static __device__ __forceinline__ Frag of(const f32x4& a, const f32x4& b) {
    return __builtin_bit_cast(Frag, make_uint4(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])));
  }
  static __device__ __forceinline__ float get(const Frag& f, int j) { return (float)f[j]; }
};
template <> struct Mma<float> {
  typedef f32x8 Frag;
  static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c, bool half = false) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!half || j < 4) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ Frag zero() { return Frag{}; }
  static __device__ __forceinline__ Frag load(const float* p) {
    const f32x4 x = load_global(p), y = load_global(p + 4);
    return Frag{{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]}};
  }
  static __device__ __forceinline__ Frag load_half(const float* p) {
    const f32x4 x = load_global(p);
    return Frag{{x[0], x[1], x[2], x[3], 0.f, 0.f, 0.f, 0.f}};
  }
  static __device__ __forceinline__ Frag of(const f32x4& a, const f32x4& b) { return Frag{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}}; }
  static __device__ __forceinline__ float get(const Frag& f, int j) { return f.v[j]; }
};
// row i of tiles: one fragment of the rows with both of the columns
template <typename T>
__device__ __forceinline__ void mma(const typename Mma<T>::Frag& a, const typename Mma<T>::Frag (&b)[2], f32x4 (&c)[2], bool half = false) {
#pragma unroll
  for (int j = 0; j < 2; ++j) c[j] = Mma<T>::mma(a, b[j], c[j], half);
}

// A head is computed as DC elements: 32, 64, 96 or 128, and in fp32 also 48, 80 or 112, whose last fragment is a half: four elements of each quarter of the
// lanes.  (fp32 products are what those kernels take their time for: heads of 80 in place of 96, 10 of them on 5 of keys, 2760 tokens, window of 700: 84 + 277 us
// -> 74 + 236.)
template <int DC> constexpr int kFrags = (DC + 31) / 32;
template <int DC> constexpr bool last_half(int kc) { return DC % 32 != 0 && kc == kFrags<DC> - 1; }
template <int DC> constexpr bool has_tile(int d, int i) { return 32 * d + 16 * i < DC; }       // of a head's columns, in Acc
// fragment kc of the row at p
template <typename T, int DC>
__device__ __forceinline__ typename Mma<T>::Frag head_frag(const T* p, int kc, int quad, int dim, bool real) {
  const bool half = last_half<DC>(kc);
  const int at = 32 * kc + (half ? 4 : 8) * quad;
  if (!real || at >= dim) return Mma<T>::zero();
  if constexpr (DC % 32 != 0)
    if (half) return Mma<T>::load_half(p + at);
  return Mma<T>::load(p + at);
}

__device__ __forceinline__ unsigned lds_address(void* p) { return uniform((unsigned)(unsigned long)(__attribute__((address_space(3))) char*)p); }
// The resource of `bytes` bytes from `base` on for loads that stand in assembly.  Where one of its scalars comes out of a vector register, five wait states
// have to pass before a load reads it; the compiler does not know that the load does, so they stand here (tests/test_lds_load_hazards.py looks at what is built).
__device__ __forceinline__ rsrc_t rsrc_for_lds(unsigned long base, unsigned bytes) {
  rsrc_t r = {uniform((unsigned)base), uniform((unsigned)(base >> 32)), uniform(bytes), 0x00020000u};
  asm volatile("s_nop 4" : "+s"(r));
  return r;
}
constexpr unsigned kOpen = 0x80000000u;      // bytes of a resource that is not to end: offsets are below 2^31

// in rows of 64 or 128 elements in LDS
constexpr int tile_dim(int dim) { return dim <= 64 ? 64 : 128; }

// Whether two sets of four wavefronts have room in LDS, and whether a launch of so many blocks is to have them: where they leave half of the chip empty or
// hold it for long steps one behind the other (512 blocks), and steps enough for both.  2 x 2048 tokens, 12 heads of 64: forward (384 blocks)
// 42 -> 31 us, gradients of queries (384 blocks) and keys (768, which keep one set) 87 -> 79; with two sets for the 768 as well 95.  Steps: one sequence of 200
// tokens, 12 heads of 64, forward 9.0 us, with two sets 9.7.  (Eight wavefronts with more than 128 registers, 140 and 164 there, are alone on a CU, so
// 384 blocks are one and a half rounds.)
template <typename T, int DC> constexpr bool kTwoSets = 2 * 4 * kStep * tile_dim(DC) * (int)sizeof(T) <= 144 * 1024;
inline bool two_sets(long blocks, long steps_rows, int n_seq) { return std::max<long>(blocks, n_seq) <= 512 && steps_rows >= 4l * kStep * n_seq; }

// A tile in LDS: rows of DH elements, chunk c (16 bytes) of row r at position c ^ turn(r).  LDS has 64 banks of four bytes.  A read of 16 bytes a lane is
// served sixteen lanes at a time, 0-3, 12-15, 20-27 and so on: eight rows at one chunk and the other eight at the next one.  The transposing reads take
// eight rows of 32 bytes, and in fp32 64 lanes read four rows of 64 bytes, four rows apart.  Each of them meets every bank once (counted: no conflicts; with
// rows 0-7 at even turns and 8-15 at odd ones in their order, every second read of 16 bytes was one).
template <typename T, int DH>
struct Tile {
  static constexpr int kRowBytes = DH * (int)sizeof(T), kChunks = kRowBytes / 16, kRowsPerLoad = 64 / kChunks;
  static __device__ __forceinline__ int turn(int r) {
    if (sizeof(T) == 4) return r & 15;
    const int far = (r >> 3) & 1;
    return DH == 64 ? (((r >> 1) & 3) ^ 2 * far) << 1 | far : ((r & 7) ^ 4 * far) << 1 | far;
  }
  // fragments of rows: lane (x, quad) takes elements 32 kc + 8 quad .. + 7 of row 16 n + x, of half a fragment 32 kc + 4 quad .. + 3
  struct Base { unsigned whole, half; };
  static __device__ __forceinline__ Base row_base(int lane) {
    const int x = lane & 15, quad = lane >> 4;
    auto at = [&](int chunk) { return (unsigned)(x * kRowBytes + ((chunk ^ turn(x)) << 4)); };
    return Base{at(sizeof(T) == 4 ? 2 * quad : quad), at(quad)};
  }
  static __device__ __forceinline__ typename Mma<T>::Frag row_frag(const char* slot, const Base& base, int n, int kc, bool half = false) {
    if constexpr (sizeof(T) == 2) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(slot + (base.whole ^ (unsigned)(kc << 6)) + n * 16 * kRowBytes));
    } else {
      const float4 p = *reinterpret_cast<const float4*>(slot + ((half ? base.half : base.whole) ^ (unsigned)((8 * kc) << 4)) + n * 16 * kRowBytes);
      if (half) return f32x8{{p.x, p.y, p.z, p.w, 0.f, 0.f, 0.f, 0.f}};
      const float4 q = *reinterpret_cast<const float4*>(slot + (base.whole ^ (unsigned)((8 * kc + 1) << 4)) + n * 16 * kRowBytes);
      return f32x8{{p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w}};
    }
  }
  // fragments of columns: lane (x, quad) takes column 16 n + x of rows 32 kk + 4 quad + 0..3 and 32 kk + 16 + 4 quad + 0..3
  static __device__ __forceinline__ unsigned col_base(int lane) {
    const int x = lane & 15, quad = lane >> 4;
    if (sizeof(T) == 4) return (unsigned)(4 * quad * kRowBytes + (((x >> 2) ^ (quad << 2)) << 4) + (x & 3) * 4);
    const int r = 4 * quad + (x >> 2);
    return (unsigned)(r * kRowBytes + ((((x & 3) >> 1) ^ turn(r)) << 4) + (x & 1) * 8);
  }
  static __device__ __forceinline__ typename Mma<T>::Frag col_frag(const char* slot, unsigned base, int n, int kk) {
    if constexpr (sizeof(T) == 2) {
      const char* const at = slot + (base ^ (unsigned)(n << 5)) + 32 * kk * kRowBytes;
      const uint2 p = lds_read_tr(reinterpret_cast<const bf16_t*>(at)), q = lds_read_tr(reinterpret_cast<const bf16_t*>(at + 16 * kRowBytes));
      return __builtin_bit_cast(bf16x8, make_uint4(p.x, p.y, q.x, q.y));
    } else {
      f32x8 f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        f.v[j] = *reinterpret_cast<const float*>(slot + (base ^ (unsigned)((4 * n ^ (j & 3)) << 4)) + (32 * kk + (j & 3) + 16 * (j >> 2)) * kRowBytes);
      return f;
    }
  }
  // one wavefront's load i of a slot: lane l brings the chunk that belongs at position l % kChunks of row `row(i, l)`
  static constexpr int kLoads = kStep / (4 * kRowsPerLoad);                 // of each of four wavefronts for kStep rows
  static __device__ __forceinline__ int load_row(int wave, int i, int lane) { return (wave * kLoads + i) * kRowsPerLoad + lane / kChunks; }
  static __device__ __forceinline__ int load_chunk(int row, int lane) { return (lane % kChunks) ^ turn(row); }
  // byte offset from a slot's first row in memory, rows `stride` bytes apart, of `dim` elements
  static __device__ __forceinline__ unsigned load_off(int wave, int i, int lane, long stride, int dim) {
    const int r = load_row(wave, i, lane), ch = load_chunk(r, lane);
    return ch * (16 / (int)sizeof(T)) < dim ? (unsigned)(r * stride + ch * 16) : kOutOfRange;
  }
};

// Two tensors' tiles on their way into a slot, one wavefront's load at a time: the vector-memory path takes a load of a wavefront in sixteen clocks, and a
// wavefront that issues one behind the other stands still (eight in a row: 440 clocks), so callers deal them out over their matrix instructions
template <typename T, int DH>
struct PairLoad {
  typedef Tile<T, DH> L;
  static constexpr int kPieces = 2 * L::kLoads;
  const unsigned (&off)[2][L::kLoads];
  rsrc_t rs[2];
  unsigned dst;
  __device__ __forceinline__ PairLoad(const unsigned (&off_)[2][L::kLoads], const rsrc_t& first, const rsrc_t& second, unsigned slot, int wave)
      : off(off_), rs{first, second}, dst(slot + (unsigned)(wave * L::kLoads * 1024)) {}
  __device__ __forceinline__ void piece(int p) const {
    const int i = p / L::kLoads, n = p % L::kLoads;
    const unsigned m = set_lds_dest(uniform(dst + (unsigned)((i * kStep * L::kRowBytes) + n * 1024)));
    one_instruction();
    load_to_lds(rs[i], off[i][n], m);
  }
  __device__ __forceinline__ void all() const {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) piece(p);
  }
};

// Where the tiles of two tensors stand in memory, one after the other.  All of it in scalars that are carried on by additions: formed anew
// for every tile, with the products and limits that this takes, they cost a step of 64 keys and 64 elements a tenth of its time.
struct TileStream {
  unsigned long at[2];
  long left[2], step[2];       // bytes: from the tile to the last row's end, and to the next tile
  // tile j of rows `stride` bytes apart from `base`, of `rows` rows in all; `by` tiles ahead with every one
  __device__ __forceinline__ TileStream(const unsigned long (&base)[2], const long (&stride)[2], int j, int rows, int by) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      at[i] = base[i] + (unsigned long)((long)j * kStep * stride[i]);
      left[i] = ((long)rows - (long)j * kStep) * stride[i];
      step[i] = (long)by * kStep * stride[i];
    }
  }
  // of the tile that is next; it ends with the last row, and behind it loads bring zeros: loops issue them to their end, without a branch among the
  // matrix instructions
  __device__ __forceinline__ rsrc_t next(int i) {
    const long bytes = left[i];
    const rsrc_t r = rsrc_for_lds(at[i], bytes <= 0 ? 0u : bytes < (long)kOpen ? (unsigned)bytes : kOpen);
    at[i] += (unsigned long)step[i];
    left[i] -= step[i];
    return r;
  }
};

// The last loads into LDS, before a block may end
__device__ __forceinline__ void drain() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// This wavefront's loads but the newest N; its LDS reads
template <int N>
__device__ __forceinline__ void wait_for() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }
__device__ __forceinline__ void wait_for_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// over the four lanes of a column, in all of them
__device__ __forceinline__ float quad_max(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// Fragments loaded from memory are waited for here, not at their first use inside a loop, where the wait would be for the loads into LDS behind them as well
template <typename F, int N>
__device__ __forceinline__ void settle(F (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(F) == 16) {
      rsrc_t r = __builtin_bit_cast(rsrc_t, f[i]);
      asm volatile("" : "+v"(r));
      f[i] = __builtin_bit_cast(F, r);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(f[i].v[j]));
    }
  }
}
template <typename F, int M, int N>
__device__ __forceinline__ void settle(F (&f)[M][N]) {
#pragma unroll
  for (int i = 0; i < M; ++i) settle(f[i]);
}
__device__ __forceinline__ void settle(float& v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ void put4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void put4(bf16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}
// A sequence as the descriptors give it, cut to the rows that there are, so that whatever they hold no access leaves the tensors
struct Seq { int q0, lq, k0, lk; };
__device__ __forceinline__ Seq sequence(const AttnShape& a, int b) {
  Seq s;
  s.q0 = min(max(a.q_start[b], 0), a.q_rows);
  s.lq = min(max(a.q_start[b + 1], s.q0), a.q_rows) - s.q0;
  s.k0 = min(max(a.k_start[b], 0), a.k_rows);
  const int len = a.k_len ? a.k_len[b] : max(a.k_start[b + 1], s.k0) - s.k0;
  s.lk = min(max(len, 0), a.k_rows - s.k0);
  return s;
}

// Slot t of the list of all sequences' tiles, `per` rows (or keys) each: the sequence, and which of its tiles.  Starts are ascending, so sequence b has the slots from
// start[b] group / per + b on, which are as many as its tiles or one more, and is looked for by every wavefront for itself, 64 places at a time: once up to
// 64 sequences, twice up to 4096.  (Sums over all sequences ahead: 2048 of 16 tokens, 16 / 4 heads of 128, 396 + 841 us ->
// 140 + 384; 2 of 2048, 12 heads of 64, forward 31 -> 29.)  A cache's
// starts have any order, so there these sums it is (only the keys' gradients ask).  False for a slot without a tile.
template <bool KEYS>
__device__ __forceinline__ bool find_tile(const AttnShape& a, int t, int per, int lane, Seq& seq, int& tile, int& tiles) {
  auto tiles_of = [&](const Seq& s) { return KEYS ? cdiv(s.lk, per) : cdiv(s.lq * a.group, per); };
  Seq s = {0, 0, 0, 0};
  int from, at;
  if (KEYS && a.k_len) {
    int b0 = 0, all = 0;
    do {
      t -= all;
      if (b0 >= a.n_seq) return false;
      s = b0 + lane < a.n_seq ? sequence(a, b0 + lane) : Seq{0, 0, 0, 0};
      const int n = tiles_of(s);
      int sum = n;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int up = __shfl_up(sum, d, kWave);
        if (lane >= d) sum += up;
      }
      all = __builtin_amdgcn_readlane(sum, kWave - 1);
      from = sum - n;
      at = __builtin_ctzl(__ballot(t < sum) | 1ul << 63);
      b0 += kWave;
    } while (t >= all);
  } else {
    const int* const start = KEYS ? a.k_start : a.q_start;
    auto slot = [&](int b) { return KEYS ? min(max(start[b], 0), a.k_rows) / per + b : min(max(start[b], 0), a.q_rows) * a.group / per + b; };
    int lo = 0, hi = a.n_seq;
    while (hi - lo > kWave) {
      const int step = cdiv(hi - lo, kWave), b = lo + lane * step;
      const unsigned long before = __ballot(b < hi && slot(b) <= t);
      if (before == 0) return false;
      lo += (63 - __builtin_clzl(before)) * step;
      hi = min(lo + step, hi);
    }
    if (lo + lane < hi) s = sequence(a, lo + lane);
    from = (KEYS ? s.k0 : s.q0 * a.group) / per + lo + lane;
    const unsigned long before = __ballot(lo + lane < hi && from <= t);
    if (before == 0) return false;
    at = 63 - __builtin_clzl(before);
  }
  auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
  seq = Seq{pick(s.q0), pick(s.lq), pick(s.k0), pick(s.lk)};
  tiles = tiles_of(seq);
  tile = t - pick(from);
  return tile < tiles;
}

// One of the two rows of a lane in the queries' kernels; a row behind the last one stands for that one, but is not real
struct Row {
  bool real;
  int query, head;
  __device__ __forceinline__ Row(int r, int rows, int G, int kvh) : real(r < rows) {
    r = min(r, rows - 1);
    query = r / G;
    head = kvh * G + (r - query * G);
  }
};

// Keys [lo, hi) that query i of a sequence sees
struct Reach { int lo, hi; };
__device__ __forceinline__ Reach reach(const AttnShape& a, const Seq& s, int i) {
  if (!a.causal) return Reach{0, s.lk};
  const int end = min(max(i - s.lq + 1 + s.lk, 0), s.lk);      // (in this order no sum passes 32 bits, with 2^31 keys either)
  return Reach{a.window > 0 ? max(end - a.window, 0) : 0, end};
}

}  // namespace attn
}  // namespace spes
