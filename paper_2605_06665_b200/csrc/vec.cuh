// Rows of a tensor, 16 bytes at a time.
#pragma once

#include "common.cuh"

namespace unipool {

// V consecutive elements as they lie in memory: 16 bytes, or two or one element where those do not fit.
template <typename E, int V> struct Vec;
template <> struct Vec<__nv_bfloat16, 8> {
  uint4 raw;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { raw = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Vec<float, 4> {
  float4 raw;
  __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void zero() { raw = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = raw.x; v[1] = raw.y; v[2] = raw.z; v[3] = raw.w; }
  __device__ __forceinline__ static void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <> struct Vec<__nv_bfloat16, 2> {
  uint32_t raw;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { raw = *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ void zero() { raw = 0u; }
  __device__ __forceinline__ void get(float (&v)[2]) const {
    v[0] = __uint_as_float(raw << 16);
    v[1] = __uint_as_float(raw & 0xffff0000u);
  }
  __device__ __forceinline__ static void store(__nv_bfloat16* p, const float (&v)[2]) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v[0], v[1]);
  }
};
template <> struct Vec<float, 2> {
  float2 raw;
  __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float2*>(p); }
  __device__ __forceinline__ void zero() { raw = make_float2(0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[2]) const { v[0] = raw.x; v[1] = raw.y; }
  __device__ __forceinline__ static void store(float* p, const float (&v)[2]) { *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]); }
};
template <typename E> struct Vec<E, 1> {
  E raw;
  __device__ __forceinline__ void load(const E* p) { raw = *p; }
  __device__ __forceinline__ void zero() { raw = from_f32<E>(0.f); }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f32(raw); }
  __device__ __forceinline__ static void store(E* p, const float (&v)[1]) { *p = from_f32<E>(v[0]); }
};

}  // namespace unipool
