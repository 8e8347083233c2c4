// A few columns of a row at a time, wherever the row begins.
#pragma once
#include "common.h"

namespace spes {

// 16 or 8 bytes at any address that the element type allows: rows begin wherever their stride puts them
template <typename T, int WORDS> struct AnyVec;
template <> struct AnyVec<bf16_t, 4> { typedef __attribute__((ext_vector_type(4), aligned(2), may_alias)) unsigned int type; };
template <> struct AnyVec<bf16_t, 2> { typedef __attribute__((ext_vector_type(2), aligned(2), may_alias)) unsigned int type; };
template <> struct AnyVec<float, 4> { typedef __attribute__((ext_vector_type(4), aligned(4), may_alias)) unsigned int type; };
typedef __attribute__((ext_vector_type(4), aligned(4), may_alias)) float f32x4_any;
typedef __attribute__((aligned(2), may_alias)) unsigned int u32_any;

// W columns of a row, 16 bytes unless said otherwise, `left` of them inside it.  Lanes side by side make one run of it: with 32 bytes of
// fp32 to a lane a stream of 16384 x 4096 went at 4.5 TB/s, with 16 at 6.0.  ONCE: with the non-temporal hint
template <typename T, int W = 16 / (int)sizeof(T)>
struct Unit {
  static constexpr int WORDS = W * (int)sizeof(T) / 4;
  typedef typename AnyVec<T, WORDS>::type vec;
  vec w;
  template <bool ONCE = false> __device__ __forceinline__ void load(const T* p, int left) {
    if (left >= W) {
      w = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const vec*>(p)) : *reinterpret_cast<const vec*>(p);
    } else {
      // 4, 2 and 1 elements, as many as there are
#pragma unroll
      for (int i = 0; i < WORDS; ++i) w[i] = 0u;
      if (left <= 0) return;
      if constexpr (sizeof(T) == 4) {
        if (left & 2) { w[0] = __float_as_uint(p[0]); w[1] = __float_as_uint(p[1]); }
        if (left & 1) {
          const unsigned one = __float_as_uint(p[left - 1]);
          if (left & 2) w[2] = one;
          else w[0] = one;
        }
      } else {
        if (W == 8 && (left & 4)) {
          const typename AnyVec<bf16_t, 2>::type q = *reinterpret_cast<const typename AnyVec<bf16_t, 2>::type*>(p);
          w[0] = q[0]; w[1] = q[1];
        }
        const int at = W == 8 ? left & 4 : 0;
        unsigned pair = 0, one = 0;
        if (left & 2) pair = *reinterpret_cast<const u32_any*>(p + at);
        if (left & 1) one = p[left - 1];
        const unsigned first = left & 2 ? pair : one, second = left & 2 ? one : 0u;
        if (W == 8 && at) { w[2] = first; w[WORDS - 1] = second; }
        else { w[0] = first; w[1] = second; }
      }
    }
  }
  // all W of them; then, of a run that was begun `back` elements ahead of its first one to end with its row, those from there on, zeros behind
  template <bool ONCE = false> __device__ __forceinline__ void load(const T* p) {
    w = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const vec*>(p)) : *reinterpret_cast<const vec*>(p);
  }
  __device__ __forceinline__ void keep(bool yes) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = yes ? w[i] : 0u;
  }
  __device__ __forceinline__ void drop(int back) {
    static_assert(WORDS == 4, "16 bytes");
    unsigned long long lo = (unsigned long long)w[1] << 32 | w[0], hi = (unsigned long long)w[3] << 32 | w[2];
    int bits = back * 8 * (int)sizeof(T);
    const bool far = bits >= 64, none = bits >= 128;
    lo = far ? hi : lo;
    hi = far ? 0ull : hi;
    bits &= 63;
    lo = lo >> bits | hi << 1 << (63 - bits);
    hi >>= bits;
    lo = none ? 0ull : lo;
    hi = none ? 0ull : hi;
    w = vec{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
  }
  template <bool ONCE = false> __device__ __forceinline__ void store(T* p) const {
    if (ONCE) __builtin_nontemporal_store(w, reinterpret_cast<vec*>(p));
    else *reinterpret_cast<vec*>(p) = w;
  }
  template <bool ONCE = false> __device__ __forceinline__ void store(T* p, int left) const {
    if (left >= W) {
      if (ONCE) __builtin_nontemporal_store(w, reinterpret_cast<vec*>(p));
      else *reinterpret_cast<vec*>(p) = w;
    } else if (left > 0) {
      if constexpr (sizeof(T) == 4) {
        if (left & 2) { p[0] = __uint_as_float(w[0]); p[1] = __uint_as_float(w[1]); }
        if (left & 1) p[left - 1] = __uint_as_float(left & 2 ? w[2] : w[0]);
      } else {
        const int at = W == 8 ? left & 4 : 0;
        if (at) *reinterpret_cast<typename AnyVec<bf16_t, 2>::type*>(p) = typename AnyVec<bf16_t, 2>::type{w[0], w[1]};
        const unsigned first = at ? w[WORDS / 2] : w[0], second = at ? w[WORDS - 1] : w[1];
        if (left & 2) *reinterpret_cast<u32_any*>(p + at) = first;
        if (left & 1) p[left - 1] = (bf16_t)(left & 2 ? second : first);
      }
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(T) == 4) {
        f[i] = __uint_as_float(w[i]);
      } else {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
      else w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
  }
};

}  // namespace spes
