// Consecutive values of a row: eight, moved 16 bytes at a time, or N in one or two accesses; and the conversions between
// storage types and fp32.
#pragma once

#include "pctc_internal.h"

namespace pctc {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(signed char v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T>
struct Vec8;
template <>
struct Vec8<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const unsigned*>(&b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) { *reinterpret_cast<uint4*>(p) = pack(v); }
};
template <>
struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
};
// N = 1, 2, 4 or 8 values, N * sizeof(T) bytes aligned (16 where that is more): fp32, bf16, or 8 bits (to be read).
template <typename T, int N>
struct VecN {
  static constexpr int BYTES = N * (int)sizeof(T), WORDS = BYTES < 4 ? 1 : BYTES / 4;
  unsigned u[WORDS];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i];
        u[4 * i] = v.x; u[4 * i + 1] = v.y; u[4 * i + 2] = v.z; u[4 * i + 3] = v.w;
      }
    } else if constexpr (BYTES == 8) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      u[0] = v.x; u[1] = v.y;
    } else if constexpr (BYTES == 4) {
      u[0] = *reinterpret_cast<const unsigned*>(p);
    } else if constexpr (BYTES == 2) {
      u[0] = *reinterpret_cast<const unsigned short*>(p);
    } else {
      u[0] = *reinterpret_cast<const unsigned char*>(p);
    }
  }
  // what another SM has written during this kernel: not from this SM's cache
  __device__ __forceinline__ void load_l2(const T* p) {
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) {
        const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p) + i);
        u[4 * i] = v.x; u[4 * i + 1] = v.y; u[4 * i + 2] = v.z; u[4 * i + 3] = v.w;
      }
    } else if constexpr (BYTES == 8) {
      const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p));
      u[0] = v.x; u[1] = v.y;
    } else if constexpr (BYTES == 4) {
      u[0] = __ldcg(reinterpret_cast<const unsigned*>(p));
    } else {
      u[0] = __ldcg(reinterpret_cast<const unsigned short*>(p));
    }
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
    else if constexpr (sizeof(T) == 1) return (float)(signed char)(u[i >> 2] >> (8 * (i & 3)));
    else return __uint_as_float((i & 1) ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16);
  }
  __device__ __forceinline__ void add_to(float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += value(i);
  }
  static __device__ __forceinline__ void store(T* p, const float (&x)[N]) {
    unsigned w[WORDS];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(x[i]);
    } else if constexpr (N == 1) {
      *p = from_float<T>(x[0]);
      return;
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&b);
      }
    }
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i)
        reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else if constexpr (BYTES == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
      *reinterpret_cast<unsigned*>(p) = w[0];
    }
  }
};

}  // namespace pctc
