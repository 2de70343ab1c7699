// Element access of the streaming kernels (network glue, training operators) for the two storage types.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "rotconv_bf16.h"

namespace rotconv {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Element access for the two storage types: fp32, and bfloat16 kept in uint16_t (arithmetic is fp32 in
// both cases; a bf16 result is rounded once, to nearest even).  V = elements of one 16-byte access.
template <typename T> struct Elt;
template <> struct Elt<float> {
  static constexpr int V = 4;
  static __device__ __forceinline__ float ld(const float* p) { return *p; }
  static __device__ __forceinline__ void st(float* p, float v) { *p = v; }
  static __device__ __forceinline__ void ldv(const float* p, float* v) {
    const f4 a = *reinterpret_cast<const f4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = a[k];
  }
  static __device__ __forceinline__ void stv(float* p, const float* v) {
    *reinterpret_cast<f4*>(p) = f4{v[0], v[1], v[2], v[3]};
  }
  static __device__ __forceinline__ void ldh(const float* p, float* v) {   // half a vector: 8 bytes
    const float2 a = *reinterpret_cast<const float2*>(p);
    v[0] = a.x; v[1] = a.y;
  }
  static __device__ __forceinline__ void sth(float* p, const float* v) {
    *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  }
};
template <> struct Elt<uint16_t> {
  static constexpr int V = 8;
  static __device__ __forceinline__ float ld(const uint16_t* p) { return bf16_to_f32(*p); }
  static __device__ __forceinline__ void st(uint16_t* p, float v) { *p = f32_to_bf16(v); }
  static __device__ __forceinline__ void ldv(const uint16_t* p, float* v) {
    const u4 a = *reinterpret_cast<const u4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(a[k] << 16);
      v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void stv(uint16_t* p, const float* v) {
    u4 a;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = (uint32_t)f32_to_bf16(v[2 * k]) | ((uint32_t)f32_to_bf16(v[2 * k + 1]) << 16);
    *reinterpret_cast<u4*>(p) = a;
  }
  static __device__ __forceinline__ void ldh(const uint16_t* p, float* v) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xffff0000u);
    v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xffff0000u);
  }
  static __device__ __forceinline__ void sth(uint16_t* p, const float* v) {
    *reinterpret_cast<uint2*>(p) = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                                              (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
  }
};

}  // namespace
}  // namespace rotconv
