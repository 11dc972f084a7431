// Device-side pieces that the operators of ops.h share: rows of any alignment, read and written 16 bytes at a time.
#pragma once
#include "device_utils.h"

namespace ast {

// (The hardware takes global accesses of 16 bytes at any address that is a multiple of the element size.)
struct __attribute__((packed, aligned(1))) Raw16 { uint32_t w[4]; };

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
// Eight consecutive values as they are loaded, to be asked for early and worked on late.  EVEN: from a 16-byte address.
// Otherwise the aligned 16-byte groups that the values lie in are read and shifted (an unaligned read takes the memory pipeline
// several times as long); every group that is read holds some of the values, so no granule is touched that the tensor is not in.
__device__ __forceinline__ uint32_t either(uint32_t mask, uint32_t a, uint32_t b) { return (a & mask) | (b & ~mask); }
template <typename T, int W>
__device__ __forceinline__ void eight_values(const uint32_t (&w)[W], float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (sizeof(T) == 4) {
      f[i] = __uint_as_float(w[i]);
    } else {
      f[(2 * i) % 8] = __uint_as_float(w[i] << 16);
      f[(2 * i + 1) % 8] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
// the W words that begin `bytes` (even, below 4 W) behind the first byte of lo, hi one after the other
template <int W>
__device__ __forceinline__ void funnel(uint32_t (&lo)[W], const uint32_t (&hi)[W], uint32_t bytes) {
  uint32_t z[2 * W + 1];
#pragma unroll
  for (int i = 0; i < W; ++i) z[i] = lo[i], z[W + i] = hi[i];
  z[2 * W] = 0;
#pragma unroll
  for (int s = W / 2; s > 0; s /= 2) {
    const uint32_t mask = bytes & (4 * s) ? 0xffffffffu : 0;
#pragma unroll
    for (int i = 0; i < W + s; ++i) z[i] = either(mask, z[(i + s) % (2 * W)], z[i]);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) lo[i] = __builtin_amdgcn_alignbyte(z[i + 1], z[i], bytes & 2);
}
template <typename T, bool EVEN>
struct Eight {
  static constexpr int W = (int)sizeof(T) * 2, N = EVEN ? W : W + 4;  // words
  uint32_t v[N], m;
  __device__ __forceinline__ void load(const T* p) {
    m = EVEN ? 0 : (uint32_t)reinterpret_cast<uintptr_t>(p) & 15;
    // (not an address made from a number: that would be read through the slower path for any memory)
    const uint4* const g = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) - m);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 a = g[i == W / 4 && m == 0 ? 0 : i];
      v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w;
    }
  }
  __device__ __forceinline__ void words(uint32_t (&w)[W]) const {
    if (EVEN) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = v[i];
      return;
    }
    const uint32_t by8 = 0u - (m >> 3 & 1), by4 = 0u - (m >> 2 & 1);
    uint32_t a[N], b[N];
#pragma unroll
    for (int i = 0; i < W + 2; ++i) a[i] = either(by8, v[(i + 2) % N], v[i]);
#pragma unroll
    for (int i = 0; i < W + 1; ++i) b[i] = either(by4, a[(i + 1) % N], a[i]);
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = __builtin_amdgcn_alignbyte(b[(i + 1) % N], b[i], m & 2);
  }
  __device__ __forceinline__ void values(float (&f)[8]) const {
    uint32_t w[W];
    words(w);
    eight_values<T>(w, f);
  }
};
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return bf2f(*p); }
// the first n (< 8) of them, 0 behind
template <typename T>
__device__ __forceinline__ void load8_part(const T* p, int n, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? load1(p + i) : 0.f;
}
// values c .. c + 7 of a row of `cols`, 0 behind its end; EVEN: rows start at 16-byte addresses
template <typename T, bool EVEN>
__device__ __forceinline__ void load8_row(const T* row, int c, int cols, float (&v)[8]) {
  const int over = c + 8 - cols;
  if (EVEN && over <= 0) {
    load8(row + c, v);
  } else if (cols >= 8) {  // (the last eight, moved down)
    Eight<T, false> e;
    e.load(row + c - max(over, 0));
    uint32_t w[Eight<T, false>::W];
    e.words(w);
    if (over > 0) {
      const uint32_t zero[Eight<T, false>::W] = {};
      funnel(w, zero, (uint32_t)over * (uint32_t)sizeof(T));
    }
    eight_values<T>(w, v);
  } else {
    load8_part(row + c, cols - c, v);
  }
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
