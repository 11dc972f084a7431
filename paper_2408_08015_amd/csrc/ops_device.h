// Device-side pieces that the operators of ops.h share: rows of any alignment, read and written 16 bytes at a time.
#pragma once
#include "device_utils.h"

namespace ast {

// (The hardware takes global accesses of 16 bytes at any address that is a multiple of the element size.)
struct __attribute__((packed, aligned(1))) Raw16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(1))) Raw8 { uint32_t w[2]; };

// eight consecutive values as fp32
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const Raw16 a = *reinterpret_cast<const Raw16*>(p), b = *reinterpret_cast<const Raw16*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = __uint_as_float(a.w[i]);
    v[4 + i] = __uint_as_float(b.w[i]);
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  const Raw16 a = *reinterpret_cast<const Raw16*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(a.w[i] << 16);
    v[2 * i + 1] = __uint_as_float(a.w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return bf2f(*p); }
// the first n (< 8) of them, 0 behind
template <typename T>
__device__ __forceinline__ void load8_part(const T* p, int n, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? load1(p + i) : 0.f;
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = (bf16_t)(f2bf_pk(v, 0.f) & 0xffffu); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  Raw16 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a.w[i] = __float_as_uint(v[i]);
    b.w[i] = __float_as_uint(v[4 + i]);
  }
  *reinterpret_cast<Raw16*>(p) = a;
  *reinterpret_cast<Raw16*>(p + 4) = b;
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  Raw16 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) a.w[i] = f2bf_pk(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<Raw16*>(p) = a;
}
template <typename T>
__device__ __forceinline__ void store8_part(T* p, int n, const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) store1(p + i, v[i]);
}

}  // namespace ast
