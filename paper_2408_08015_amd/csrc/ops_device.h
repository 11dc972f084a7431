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


// ---- a block of 32 values in 8 bits (op_stash8.hip): eight of them a lane, four neighbouring lanes a block, all four active.
// The lane's eight codes, and the block's byte (its exponent + 127, or 255), which all four lanes get.
__device__ __forceinline__ uint32_t stash8_code(float steps) {
  return (uint32_t)(int)rintf(fminf(fmaxf(steps, -127.f), 127.f)) & 0xffu;
}
__device__ __forceinline__ uint8_t stash8_block(const float (&v)[8], uint2& w) {
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
  // maximum over the block's four lanes, as bits (those of a NaN are above all others)
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_QUAD_SWAP1, 0xF, 0xF, true));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_QUAD_SWAP2, 0xF, 0xF, true));
  const bool finite = top < 0x7f800000u;
  const int e = min(max((int)((top + 0x01ffffu) >> 23) - 127 - 6, -126), 121);
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  w = make_uint2(0, 0);
  if (finite) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w.x |= stash8_code(v[k] * inv) << (8 * k);
      w.y |= stash8_code(v[4 + k] * inv) << (8 * k);
    }
  }
  return (uint8_t)(finite ? e + 127 : 255);
}

// Eight values of a row of `cols`, from place c on, as they are loaded (0 behind the row's end), to be asked for early; EVEN: rows
// start at 16-byte addresses and hold a multiple of eight values.
template <typename T, bool EVEN>
struct RowEight {
  Eight<T, EVEN> e;
  int over;  // places behind the row's end: the last eight values were read
  __device__ __forceinline__ void load(const T* row, int c, int cols) {
    over = 0;
    if (EVEN) {
      e.load(row + c);
    } else if (cols >= 8) {
      over = max(c + 8 - cols, 0);
      e.load(row + c - over);
    } else {  // (c is 0)
      e.m = 0;
#pragma unroll
      for (int i = 0; i < Eight<T, EVEN>::N; ++i) e.v[i] = 0;
#pragma unroll
      for (int i = 0; i < 7; ++i) {
        if (i >= cols) break;
        if (sizeof(T) == 4) e.v[i] = reinterpret_cast<const uint32_t*>(row)[i];
        else e.v[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(row)[i] << (i % 2 * 16);
      }
    }
  }
  __device__ __forceinline__ void values(float (&f)[8]) const {
    uint32_t w[Eight<T, EVEN>::W];
    e.words(w);
    if (!EVEN && over > 0) {
      const uint32_t zero[Eight<T, EVEN>::W] = {};
      funnel(w, zero, (uint32_t)over * (uint32_t)sizeof(T));
    }
    eight_values<T>(w, f);
  }
};
template <typename T, bool EVEN>
__device__ __forceinline__ void store_row8(T* row, int c, int cols, const float (&v)[8]) {
  if (EVEN || cols - c >= 8) store8(row + c, v);
  else store8_part(row + c, cols - c, v);
}

// ---- rows (heads) of 2^ls lanes each, ls <= 6: sum over the lanes of a row, valid in each of them
__device__ __forceinline__ float row_sum(float v, int ls) {
  if (ls > 0) v += dpp_move<DPP_QUAD_SWAP1>(v);
  if (ls > 1) v += dpp_move<DPP_QUAD_SWAP2>(v);
  if (ls > 2) v += dpp_move<DPP_HALF_MIRROR>(v);
  if (ls > 3) v += dpp_move<DPP_ROW_MIRROR>(v);
  if (ls > 4) v += __shfl_xor(v, 16, 64);
  if (ls > 5) v += __shfl_xor(v, 32, 64);
  return v;
}

// ... and over the lanes that hold the same place of the wavefront's rows (rotations inside 16 lanes, then across them)
__device__ __forceinline__ float places_sum(float v, int ls) {
  if (ls < 4) v += dpp_move<0x128>(v);
  if (ls < 3) v += dpp_move<0x124>(v);
  if (ls < 2) v += dpp_move<0x122>(v);
  if (ls < 1) v += dpp_move<0x121>(v);
  if (ls < 5) v += __shfl_xor(v, 16, 64);
  if (ls < 6) v += __shfl_xor(v, 32, 64);
  return v;
}

}  // namespace ast
