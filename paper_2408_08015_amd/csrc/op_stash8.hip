// Activations in 8 bits: blocks of 32 values of a row share a power of two 2^e, the least with 127 * 2^e >= max |x|
// (-126 <= e <= 121), and are kept as round-to-nearest-even(x / 2^e) in a signed byte.  The power of two makes the quotient exact,
// so the only rounding is the one to the step, and a restored value (7 bits and a sign) is exact in bf16.
//
// e comes from the bits of the maximum m * 2^E: 127 = 1.984375 * 2^6, so e = E - 6, one more where the fraction bits of m
// exceed those of 1.984375 (0x7e0000).  Past 127 * 2^121 it would be 122 and the values +-64, which fp32 has no room for: such
// values stay at +-127 steps of 2^121.  A block with an infinity or a NaN keeps zeros and the byte 255, which as a float's
// exponent is an infinity: 0 * inf restores NaN.
//
// (16384 x 2048 bf16 values packed and restored 40 us, 101 + 101 MB; GELU's gradient of 12289 x 1500 19 us, 93 MB: 4.9 TB/s; in fp32,
// with erfcf and expf a value, 40 us, 167 MB: 4.2 TB/s.)
// All three kernels move bytes: a lane takes eight values (16 bytes of bf16, 8 of the kept ones), four lanes a block.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

__device__ __forceinline__ float scale_of(uint8_t b) { return __uint_as_float((uint32_t)b << 23); }

__device__ __forceinline__ void restore8(uint2 q, float s, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (float)(int)(int8_t)(q.x >> (8 * i)) * s;
    v[4 + i] = (float)(int)(int8_t)(q.y >> (8 * i)) * s;
  }
}

template <typename T, bool EVEN>
__global__ __launch_bounds__(256) void stash8_pack_kernel(const T* __restrict__ x, int64_t rows, int cols, int pitch,
                                                          uint8_t* __restrict__ q, uint8_t* __restrict__ scales) {
  const int per_row = pitch / 8;
  const int64_t n = rows * per_row;  // (a multiple of four: the lanes of a block stay together)
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row;
    const int c = (int)(i - r * per_row) * 8;
    float v[8];
    if (c < cols) load8_row<T, EVEN>(x + r * cols, c, cols, v);
    else load8_part(x, 0, v);
    uint2 w;
    const uint8_t scale = stash8_block(v, w);
    *reinterpret_cast<uint2*>(q + r * pitch + c) = w;
    if ((threadIdx.x & 3) == 0) scales[r * (pitch / kStash8Block) + c / kStash8Block] = scale;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void stash8_unpack_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scales,
                                                            int64_t rows, int cols, int pitch, T* __restrict__ x) {
  const int per_row = (cols + 7) / 8;
  const int64_t n = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row;
    const int c = (int)(i - r * per_row) * 8;
    float v[8];
    restore8(*reinterpret_cast<const uint2*>(q + r * pitch + c),
             scale_of(scales[r * (pitch / kStash8Block) + c / kStash8Block]), v);
    T* dst = x + r * cols + c;
    if (cols - c >= 8) store8(dst, v);
    else store8_part(dst, cols - c, v);
  }
}

// GELU'(z) = Phi(z) + z phi(z)
template <bool EXACT>
__device__ __forceinline__ float gelu_slope(float z) {
  if (!EXACT) return gelu_grad_fast(z);  // (bf16 results: within 3e-7 of Phi)
  return 0.5f * erfcf(z * -0.70710678118f) + z * 0.3989422804f * expf(-0.5f * z * z);
}

template <typename T, bool EVEN>
__global__ __launch_bounds__(256) void gelu_bwd_stash8_kernel(const T* dy, const uint8_t* __restrict__ q,
                                                              const uint8_t* __restrict__ scales, int64_t rows, int cols,
                                                              int pitch, T* dz) {  // (dz may be dy)
  const int per_row = (cols + 7) / 8;
  const int64_t n = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row;
    const int c = (int)(i - r * per_row) * 8;
    const int live = cols - c;
    float z[8], g[8];
    restore8(*reinterpret_cast<const uint2*>(q + r * pitch + c),
             scale_of(scales[r * (pitch / kStash8Block) + c / kStash8Block]), z);
    load8_row<T, EVEN>(dy + r * cols, c, cols, g);  // (in place: what it reads of others' places is not used)
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] *= gelu_slope<sizeof(T) == 4>(z[k]);
    if (live >= 8) store8(dz + r * cols + c, g);
    else store8_part(dz + r * cols + c, live, g);
  }
}

bool rows_even(const void* p, int64_t cols, bool bf16) {  // every row starts at a 16-byte address
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols * (bf16 ? 2 : 4) % 16 == 0;
}
unsigned blocks_for(int64_t chunks) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((chunks + 255) / 256, 1 << 20)); }

}  // namespace

void stash8_pack(hipStream_t st, const void* x, bool bf16, int64_t rows, int64_t cols, void* stash) {
  if (rows <= 0) return;
  const int pitch = (int)stash8_pitch(cols);
  uint8_t* q = static_cast<uint8_t*>(stash);
  uint8_t* sc = q + rows * pitch;
  const dim3 grid(blocks_for(rows * (pitch / 8)));
  auto go = [&](auto kernel, auto* p) { KLAUNCH_NAMED("stash8_pack_kernel", kernel, grid, dim3(256), 0, st, p, rows, (int)cols, pitch, q, sc); };
  const bool even = rows_even(x, cols, bf16);
  if (bf16) go(even ? stash8_pack_kernel<bf16_t, true> : stash8_pack_kernel<bf16_t, false>, static_cast<const bf16_t*>(x));
  else go(even ? stash8_pack_kernel<float, true> : stash8_pack_kernel<float, false>, static_cast<const float*>(x));
}

void stash8_unpack(hipStream_t st, const void* stash, int64_t rows, int64_t cols, void* x, bool bf16) {
  if (rows <= 0) return;
  const int pitch = (int)stash8_pitch(cols);
  const uint8_t* q = static_cast<const uint8_t*>(stash);
  const uint8_t* sc = q + rows * pitch;
  const dim3 grid(blocks_for(rows * ((cols + 7) / 8)));
  if (bf16) KLAUNCH(stash8_unpack_kernel<bf16_t>, grid, dim3(256), 0, st, q, sc, rows, (int)cols, pitch, static_cast<bf16_t*>(x));
  else KLAUNCH(stash8_unpack_kernel<float>, grid, dim3(256), 0, st, q, sc, rows, (int)cols, pitch, static_cast<float*>(x));
}

void gelu_bwd_stash8(hipStream_t st, const void* dy, bool bf16, const void* stash, int64_t rows, int64_t cols, void* dz) {
  if (rows <= 0) return;
  const int pitch = (int)stash8_pitch(cols);
  const uint8_t* q = static_cast<const uint8_t*>(stash);
  const uint8_t* sc = q + rows * pitch;
  const dim3 grid(blocks_for(rows * ((cols + 7) / 8)));
  auto go = [&](auto kernel, auto* p, auto* out) {
    KLAUNCH_NAMED("gelu_bwd_stash8_kernel", kernel, grid, dim3(256), 0, st, p, q, sc, rows, (int)cols, pitch, out);
  };
  const bool even = rows_even(dy, cols, bf16);
  if (bf16)
    go(even ? gelu_bwd_stash8_kernel<bf16_t, true> : gelu_bwd_stash8_kernel<bf16_t, false>, static_cast<const bf16_t*>(dy), static_cast<bf16_t*>(dz));
  else
    go(even ? gelu_bwd_stash8_kernel<float, true> : gelu_bwd_stash8_kernel<float, false>, static_cast<const float*>(dy), static_cast<float*>(dz));
}

}  // namespace ast
