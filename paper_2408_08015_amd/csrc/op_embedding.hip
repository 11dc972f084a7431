// Token embedding: y[t] = scale * W[ids[t]] and its gradient dW[v] = scale * sum of dy[t] over the tokens t of id v.
//
// Both move bytes and compute next to nothing.  The gradient orders the tokens by id first (stably, ids outside the table
// last), so that the tokens of a row lie next to each other and one wavefront adds them in their order: no atomics, equal
// calls give equal bits.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

// Forward: L = 2^ls lanes per row, eight values each at a time.
template <typename TW, typename TY>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const int32_t* __restrict__ ids, int64_t tokens,
                                                            const TW* __restrict__ table, uint32_t rows, int width,
                                                            float scale, TY* __restrict__ y, int ls) {
  const int lane = threadIdx.x & ((1 << ls) - 1);
  const int per = 256 >> ls;  // rows of a block at a time
  for (int64_t t = (int64_t)blockIdx.x * per + (threadIdx.x >> ls); t < tokens; t += (int64_t)gridDim.x * per) {
    const uint32_t id = (uint32_t)ids[t];
    const bool live = id < rows;
    const TW* src = table + (size_t)(live ? id : 0) * width;
    TY* dst = y + (size_t)t * width;
    for (int c = lane * 8; c < width; c += 8 << ls) {
      float v[8];
      const int n = width - c;
      if (n >= 8) load8(src + c, v);
      else load8_part(src + c, n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = live ? v[i] * scale : 0.f;
      if (n >= 8) store8(dst + c, v);
      else store8_part(dst + c, n, v);
    }
  }
}

// ids outside the table sort behind every row
__device__ __forceinline__ uint32_t sort_key(int32_t id, uint32_t rows) { return min((uint32_t)id, rows); }

__global__ __launch_bounds__(256) void embedding_zero_kernel(float4* __restrict__ p, size_t n4, float* __restrict__ tail, int rest) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (size_t)gridDim.x * 256)
    p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (blockIdx.x == 0 && (int)threadIdx.x < rest) tail[threadIdx.x] = 0.f;
}

// Place of every token in the order: the number of tokens in front of it, counted.
__global__ __launch_bounds__(256) void embedding_rank_kernel(const int32_t* __restrict__ ids, int64_t tokens, uint32_t rows,
                                                             uint32_t* __restrict__ key, uint32_t* __restrict__ order) {
  __shared__ uint32_t sk[1024];
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t mine = t < tokens ? sort_key(ids[t], rows) : 0xffffffffu;
  uint32_t rank = 0;
  for (int64_t u0 = 0; u0 < tokens; u0 += 1024) {
    __syncthreads();
    for (int i = threadIdx.x; i < 1024; i += 256) sk[i] = u0 + i < tokens ? sort_key(ids[u0 + i], rows) : 0xffffffffu;
    __syncthreads();
    const int n = (int)min((int64_t)1024, tokens - u0);
    for (int i = 0; i < n; ++i) rank += sk[i] < mine || (sk[i] == mine && u0 + i < t);
  }
  if (t < tokens) {
    key[rank] = mine;
    order[rank] = (uint32_t)t;
  }
}

// One wavefront per run of equal ids.
template <typename T>
__global__ __launch_bounds__(256) void embedding_runs_kernel(const uint32_t* __restrict__ key, const uint32_t* __restrict__ order,
                                                             int64_t tokens, uint32_t rows, int width, const T* __restrict__ dy,
                                                             float scale, int accumulate, float* __restrict__ dtable) {
  const int lane = threadIdx.x & 63;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < tokens; i += (int64_t)gridDim.x * 4) {
    const uint32_t k = key[i];
    if (k >= rows || (i > 0 && key[i - 1] == k)) continue;
    for (int c = lane; c < width; c += 64) {
      double s = 0;
      for (int64_t j = i; j < tokens && key[j] == k; ++j) s += load1(dy + (size_t)order[j] * width + c);
      float* out = dtable + (size_t)k * width + c;
      *out = (accumulate ? *out : 0.f) + (float)s * scale;
    }
  }
}

int row_lanes_log2(int64_t width) {  // lanes that share a row's chunks of eight
  int ls = 0;
  while (ls < 8 && (8 << ls) < width) ++ls;
  return ls;
}

}  // namespace

void embedding_fwd(hipStream_t st, const int32_t* ids, int64_t tokens, const void* table, bool table_bf16, int64_t rows,
                   int64_t width, float scale, void* y, bool y_bf16) {
  if (tokens <= 0) return;
  const int ls = row_lanes_log2(width), per = 256 >> ls;
  const unsigned blocks = (unsigned)std::min<int64_t>((tokens + per - 1) / per, 1 << 20);
#define LAUNCH(TW, TY)                                                                                                        \
  KLAUNCH((embedding_fwd_kernel<TW, TY>), dim3(blocks), dim3(256), 0, st, ids, tokens, static_cast<const TW*>(table), (uint32_t)rows, \
          (int)width, scale, static_cast<TY*>(y), ls)
  if (table_bf16) {
    if (y_bf16) LAUNCH(bf16_t, bf16_t); else LAUNCH(bf16_t, float);
  } else {
    if (y_bf16) LAUNCH(float, bf16_t); else LAUNCH(float, float);
  }
#undef LAUNCH
}

size_t embedding_bwd_ws_bytes(int64_t tokens, int64_t, int64_t) { return ((size_t)tokens * 8 + 15) / 16 * 16; }

void embedding_bwd(hipStream_t st, const int32_t* ids, int64_t tokens, const void* dy, bool dy_bf16, int64_t rows,
                   int64_t width, float scale, bool accumulate, float* dtable, void* ws) {
  uint32_t* key = static_cast<uint32_t*>(ws);
  uint32_t* order = key + tokens;
  if (!accumulate) {
    const size_t n = (size_t)rows * width;
    // (16-byte writes from the first address that allows them)
    size_t head = std::min<size_t>((16 - (reinterpret_cast<uintptr_t>(dtable) & 15)) / 4 % 4, n);
    const size_t n4 = (n - head) / 4;
    const unsigned blocks = (unsigned)std::min<size_t>(n4 / 256 + 1, 8192);
    KLAUNCH(embedding_zero_kernel, dim3(blocks), dim3(256), 0, st, reinterpret_cast<float4*>(dtable + head), n4,
            dtable + head + 4 * n4, (int)(n - head - 4 * n4));
    if (head) KLAUNCH(embedding_zero_kernel, dim3(1), dim3(256), 0, st, nullptr, 0, dtable, (int)head);
  }
  if (tokens <= 0) return;
  KLAUNCH(embedding_rank_kernel, dim3((unsigned)((tokens + 255) / 256)), dim3(256), 0, st, ids, tokens, (uint32_t)rows, key, order);
  const unsigned blocks = (unsigned)std::min<int64_t>((tokens + 3) / 4, 1 << 16);
  if (dy_bf16)
    KLAUNCH(embedding_runs_kernel<bf16_t>, dim3(blocks), dim3(256), 0, st, key, order, tokens, (uint32_t)rows, (int)width,
            static_cast<const bf16_t*>(dy), scale, (int)accumulate, dtable);
  else
    KLAUNCH(embedding_runs_kernel<float>, dim3(blocks), dim3(256), 0, st, key, order, tokens, (uint32_t)rows, (int)width,
            static_cast<const float*>(dy), scale, (int)accumulate, dtable);
}

}  // namespace ast
