// Eight columns of a row at a time, wherever the row begins.
#pragma once
#include "common.h"

namespace spes {

// Rows begin wherever their stride puts them: 16-byte accesses at any address that the element type allows.
typedef __attribute__((ext_vector_type(4), aligned(2), may_alias)) unsigned int u32x4_any;
typedef __attribute__((ext_vector_type(4), aligned(4), may_alias)) float f32x4_any;

// Eight columns of a row, `left` of them inside it
template <typename T> struct Unit;
template <> struct Unit<bf16_t> {
  unsigned int w[4];
  __device__ __forceinline__ void load(const bf16_t* p, int left) {
    if (left >= 8) {
      const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = 2 * i < left ? (unsigned)p[2 * i] : 0u;
        if (2 * i + 1 < left) w[i] |= (unsigned)p[2 * i + 1] << 16;
      }
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ void store(bf16_t* p, int left) const {
    if (left >= 8) {
      *reinterpret_cast<u32x4_any*>(p) = u32x4_any{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) p[e] = (bf16_t)(w[e / 2] >> (16 * (e & 1)));
    }
  }
};
template <> struct Unit<float> {
  float w[8];
  __device__ __forceinline__ void load(const float* p, int left) {
    if (left >= 8) {
      const f32x4_any a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) { w[i] = a[i]; w[4 + i] = b[i]; }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = e < left ? p[e] : 0.f;
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = w[e];
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = f[e];
  }
  __device__ __forceinline__ void store(float* p, int left) const {
    if (left >= 8) {
      *reinterpret_cast<f32x4_any*>(p) = f32x4_any{w[0], w[1], w[2], w[3]};
      *reinterpret_cast<f32x4_any*>(p + 4) = f32x4_any{w[4], w[5], w[6], w[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) p[e] = w[e];
    }
  }
};

}  // namespace spes
