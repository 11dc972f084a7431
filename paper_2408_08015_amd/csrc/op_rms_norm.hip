// RMS norm with the residual's addition, forward and backward, one pass over the rows each.
//
//   s = x + r, rounded to the stream's type;  rho = 1 / sqrt(mean(s^2) + eps);  y = s rho g, rounded;  kept = y in 8 bits
//   h = dy g;  n = s rho;  ds = rho (h - n mean(h n)) + dsum = rho h - s rho^3 mean(h s) + dsum;  dg = sum of dy n
//
// The norm is that of the sum as it is written, so the backward pass, which forms rho again from it, is the gradient of what the
// forward pass computed; what is kept in 8 bits is y as it is written, the same bytes that a pack of y gives.
// Bound by the bytes of the rows.  A row stays in the registers of its lanes (8 values a group, IT groups a lane): 2^ls
// lanes of a wavefront for up to 1024 values, a block for more, so it is read once and both sums of the backward pass are of
// values at hand.  A lane keeps its columns from row to row: gains are loaded once, and the gains' gradients are summed in
// registers, then over the wavefronts, then over the blocks in 64 bits, in a fixed order.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

struct NormArgs {
  const void *x, *r;         // forward: x and the residual (or nullptr); backward: dy and dsum (or nullptr)
  const void* s;             // backward: the sum
  const float* gain;
  void *y, *sum;             // forward: y and the sum (or nullptr); backward: dx and ds (either may be nullptr)
  uint8_t *q, *scales;       // y in 8 bits, or nullptr
  float* part;               // backward: [blocks][cols] sums of dy n
  int64_t rows;
  int cols, pitch;
  float eps, inv;
  int ls;                    // log2 of a row's lanes (rows inside a wavefront)
};

__device__ __forceinline__ void round_to(float (&)[8], const float*) {}
__device__ __forceinline__ void round_to(float (&v)[8], const bf16_t*) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = f2bf_pk(v[2 * i], v[2 * i + 1]);
    v[2 * i] = __uint_as_float(w << 16);
    v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
  }
}

__device__ __forceinline__ void gains(const NormArgs& g, int c, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < g.cols ? g.gain[c + e] : 0.f;
}
__device__ __forceinline__ void copy8(const float (&a)[8], float (&b)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = a[e];
}

// Sums over the lanes of a row: inside a wavefront, or (THREADS > 0) over a block; two at once, valid in every lane.  sh: two
// buffers of 2 x 16 values that calls use in turn, so one barrier a call is enough.
template <int THREADS>
__device__ __forceinline__ void row_sums(float& a, float& b, bool two, int ls, float (*sh)[32], int turn) {
  if (THREADS == 0) {
    a = row_sum(a, ls);
    if (two) b = row_sum(b, ls);
    return;
  }
  a = wave_sum(a);
  if (two) b = wave_sum(b);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh[turn][wave] = a;
    sh[turn][16 + wave] = b;
  }
  __syncthreads();
  a = b = 0.f;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) {
    a += sh[turn][i];
    if (two) b += sh[turn][16 + i];
  }
}

// BLOCK: threads that take one row together, 0: 2^ls lanes do (blocks of 256 threads).
template <typename T, typename S, bool EVEN, int IT, int BLOCK>
__global__ __launch_bounds__(BLOCK ? BLOCK : 256) void rms_norm_kernel(const NormArgs g) {
  __shared__ float sh[2][32];
  const int lanes = BLOCK ? BLOCK : 1 << g.ls;
  const int lane = threadIdx.x & (lanes - 1);
  const int64_t step = (int64_t)gridDim.x * (BLOCK ? 1 : 256 >> g.ls);
  int64_t row = BLOCK ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (256 >> g.ls) + (threadIdx.x >> g.ls);
  constexpr bool AHEAD = BLOCK < 1024;  // the next row is asked for before this one is worked on, and gains stay in registers
  float kept[AHEAD ? IT : 1][8];
#pragma unroll
  for (int i = 0; i < (AHEAD ? IT : 0); ++i) gains(g, (lane + i * lanes) * 8, kept[i]);
  struct Row {
    RowEight<T, EVEN> x[IT];
    RowEight<S, EVEN> r[IT];
  };
  auto fetch = [&](int64_t at, Row& w) __attribute__((always_inline)) {
    if (at >= g.rows) return;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
      if (c >= g.cols) continue;
      w.x[i].load(static_cast<const T*>(g.x) + at * g.cols, c, g.cols);
      if (g.r) w.r[i].load(static_cast<const S*>(g.r) + at * g.cols, c, g.cols);
    }
  };
  Row cur;
  if (AHEAD) fetch(row, cur);
  for (int turn = 0; row < g.rows; row += step, turn ^= 1) {
    Row next;
    if (AHEAD) fetch(row + step, next);
    else fetch(row, cur);
    float v[IT][8], ss = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
      if (c < g.cols) {
        cur.x[i].values(v[i]);
        if (g.r) {
          float r[8];
          cur.r[i].values(r);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] += r[e];
          round_to(v[i], static_cast<const S*>(nullptr));
          store_row8<S, EVEN>(static_cast<S*>(g.sum) + row * g.cols, c, g.cols, v[i]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += v[i][e] * v[i][e];
    }
    row_sums<BLOCK>(ss, none, false, g.ls, sh, turn);
    const float rho = rsqrtf(ss * g.inv + g.eps);
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
      float gain[8];
      if (AHEAD) copy8(kept[AHEAD ? i : 0], gain);
      else gains(g, c, gain);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * rho * gain[e];
      if (c < g.cols) store_row8<T, EVEN>(static_cast<T*>(g.y) + row * g.cols, c, g.cols, v[i]);
      if (g.q && c < g.pitch) {  // (a block of 32 values is four lanes' groups, all inside the pitch or none)
        if (!EVEN) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] = c + e < g.cols ? v[i][e] : 0.f;  // (0 times an infinite rho is no zero)
        }
        round_to(v[i], static_cast<const T*>(nullptr));
        uint2 w;
        const uint8_t scale = stash8_block(v[i], w);
        *reinterpret_cast<uint2*>(g.q + row * g.pitch + c) = w;
        if ((lane & 3) == 0) g.scales[row * (g.pitch / kStash8Block) + c / kStash8Block] = scale;
      }
    }
    if (AHEAD) cur = next;
  }
}

template <typename T, typename S, bool EVEN, int IT, int BLOCK>
__global__ __launch_bounds__(BLOCK ? BLOCK : 256) void rms_norm_bwd_kernel(const NormArgs g) {
  __shared__ float sh[2][32];
  const int lanes = BLOCK ? BLOCK : 1 << g.ls;
  const int lane = threadIdx.x & (lanes - 1);
  const int64_t step = (int64_t)gridDim.x * (BLOCK ? 1 : 256 >> g.ls);
  int64_t row = BLOCK ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (256 >> g.ls) + (threadIdx.x >> g.ls);
  constexpr bool AHEAD = BLOCK < 1024;
  float kept[AHEAD ? IT : 1][8], acc[IT][8];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    if (AHEAD) gains(g, (lane + i * lanes) * 8, kept[AHEAD ? i : 0]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
  }
  struct Row {
    RowEight<T, EVEN> d[IT];
    RowEight<S, EVEN> s[IT], r[IT];
  };
  auto fetch = [&](int64_t at, Row& w) __attribute__((always_inline)) {
    if (at >= g.rows) return;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
      if (c >= g.cols) continue;
      w.d[i].load(static_cast<const T*>(g.x) + at * g.cols, c, g.cols);
      w.s[i].load(static_cast<const S*>(g.s) + at * g.cols, c, g.cols);
      if (g.r) w.r[i].load(static_cast<const S*>(g.r) + at * g.cols, c, g.cols);
    }
  };
  Row cur;
  if (AHEAD) fetch(row, cur);
  for (int turn = 0; row < g.rows; row += step, turn ^= 1) {
    Row next;
    if (AHEAD) fetch(row + step, next);
    else fetch(row, cur);
    float s[IT][8], d[IT][8], ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
      if (c < g.cols) {
        cur.s[i].values(s[i]);
        cur.d[i].values(d[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = d[i][e] = 0.f;
      }
      float gain[8];
      if (AHEAD) copy8(kept[AHEAD ? i : 0], gain);
      else gains(g, c, gain);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss += s[i][e] * s[i][e];
        dot += d[i][e] * gain[e] * s[i][e];
      }
    }
    row_sums<BLOCK>(ss, dot, true, g.ls, sh, turn);
    const float rho = rsqrtf(ss * g.inv + g.eps);
    const float m = rho * rho * dot * g.inv;  // mean(h n) rho = rho^2 mean(h s)
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
      if (c >= g.cols) continue;
      float r[8] = {}, gain[8];
      if (AHEAD) copy8(kept[AHEAD ? i : 0], gain);
      else gains(g, c, gain);
      if (g.r) cur.r[i].values(r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[i][e] += d[i][e] * (s[i][e] * rho);
        s[i][e] = rho * (d[i][e] * gain[e] - s[i][e] * m) + r[e];
      }
      if (g.y) store_row8<T, EVEN>(static_cast<T*>(g.y) + row * g.cols, c, g.cols, s[i]);
      if (g.sum) store_row8<S, EVEN>(static_cast<S*>(g.sum) + row * g.cols, c, g.cols, s[i]);
    }
    if (AHEAD) cur = next;
  }
  // the gains' gradients: over the rows of a wavefront, then over the wavefronts
  float* const part = g.part + (int64_t)blockIdx.x * g.cols;
  if (BLOCK) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = (lane + i * lanes) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < g.cols) part[c + e] = acc[i][e];
    }
    return;
  }
  constexpr int WIDE = IT * 64 * 8;
  __shared__ float red[BLOCK ? 1 : 4 * WIDE];
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = (lane + i * lanes) * 8 + e;
      const float v = places_sum(acc[i][e], g.ls);
      if ((threadIdx.x & 63) >> g.ls == 0 && c < g.cols) red[wave * WIDE + c] = v;
    }
  __syncthreads();
  for (int c = threadIdx.x; c < g.cols; c += 256)
    part[c] = red[c] + red[WIDE + c] + red[2 * WIDE + c] + red[3 * WIDE + c];
}

// dgain[c] (+)= sum over the blocks, in 64 bits: 32 columns a block, 32 rows of it at a time
__global__ __launch_bounds__(1024) void rms_norm_gain_sum_kernel(const float* __restrict__ part, int blocks, int cols, float* out,
                                                                 int accumulate) {
  __shared__ double sh[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  double s = 0;
  if (c < cols) {
#pragma unroll 8
    for (int b = y; b < blocks; b += 32) s += part[(int64_t)b * cols + c];
  }
  sh[y][x] = s;
  __syncthreads();
  for (int half = 16; half > 0; half /= 2) {
    if (y < half) sh[y][x] += sh[y + half][x];
    __syncthreads();
  }
  if (y == 0 && c < cols) out[c] = (accumulate ? out[c] : 0.f) + (float)sh[0][x];
}

struct Shape { int it, block, ls; };

// Lanes of a row: one group of eight values a lane up to 512 values, two up to 1024; then a block's of 256, 512, 1024 threads, two
// groups a lane.
Shape shape_of(int cols, bool keep) {
  const int groups = (cols + 7) / 8;
  Shape s = {1, 0, keep ? 2 : 0};  // (8 bits: four lanes a block of 32 values)
  if (groups <= 128) {
    if (groups > 64) s.it = 2;
    while ((s.it << s.ls) < groups) ++s.ls;
    return s;
  }
  s.block = groups <= 512 ? 256 : groups <= 1024 ? 512 : 1024;
  s.it = groups <= s.block ? 1 : 2;  // (16384 values at most)
  return s;
}

constexpr int kMostPartials = 1024;
int64_t bwd_blocks(int64_t rows, const Shape& s) {
  const int64_t at_once = s.block ? 1 : 256 >> s.ls;
  return std::max<int64_t>(1, std::min<int64_t>((rows + at_once - 1) / at_once, s.block == 1024 ? kMostPartials / 2 : kMostPartials));
}

template <bool BWD, typename T, typename S, bool EVEN, int IT, int BLOCK>
void go(hipStream_t st, int64_t blocks, const NormArgs& g) {
  const dim3 grid((unsigned)blocks), block(BLOCK ? BLOCK : 256);
  if (BWD) KLAUNCH_NAMED("rms_norm_bwd_kernel", (rms_norm_bwd_kernel<T, S, EVEN, IT, BLOCK>), grid, block, 0, st, g);
  else KLAUNCH_NAMED("rms_norm_kernel", (rms_norm_kernel<T, S, EVEN, IT, BLOCK>), grid, block, 0, st, g);
}
template <bool BWD, typename T, typename S, bool EVEN>
void pick(hipStream_t st, int64_t blocks, const Shape& s, const NormArgs& g) {
  if (s.block == 0) {
    if (s.it == 1) go<BWD, T, S, EVEN, 1, 0>(st, blocks, g);
    else go<BWD, T, S, EVEN, 2, 0>(st, blocks, g);
  } else if (s.block == 256) {
    if (s.it == 1) go<BWD, T, S, EVEN, 1, 256>(st, blocks, g);
    else go<BWD, T, S, EVEN, 2, 256>(st, blocks, g);
  } else if (s.block == 512) {
    go<BWD, T, S, EVEN, 2, 512>(st, blocks, g);
  } else {
    go<BWD, T, S, EVEN, 2, 1024>(st, blocks, g);
  }
}
template <bool BWD>
void launch(hipStream_t st, const ast_norm_cfg& c, const Shape& s, int64_t blocks, const NormArgs& g) {
  bool even = c.width % 8 == 0;
  for (const void* p : {g.x, g.r, g.s, (const void*)g.y, (const void*)g.sum}) even = even && reinterpret_cast<uintptr_t>(p) % 16 == 0;
  const bool tb = c.dtype != AST_F32, sb = c.sum_dtype != AST_F32;
#define PICK(T, S) (even ? pick<BWD, T, S, true>(st, blocks, s, g) : pick<BWD, T, S, false>(st, blocks, s, g))
  if (tb && sb) PICK(bf16_t, bf16_t);
  else if (tb) PICK(bf16_t, float);
  else PICK(float, float);
#undef PICK
}

NormArgs args_of(const ast_norm_cfg& c, const Shape& s, const float* gain) {
  NormArgs g = {};
  g.gain = gain;
  g.rows = c.rows;
  g.cols = (int)c.width;
  g.eps = c.eps;
  g.inv = 1.f / (float)c.width;
  g.ls = s.ls;
  return g;
}

}  // namespace

void rms_norm_fwd(hipStream_t st, const ast_norm_cfg& c, const void* x, const void* residual, const float* gain, void* y,
                  void* sum, void* stash) {
  if (c.rows <= 0) return;
  const Shape s = shape_of((int)c.width, stash != nullptr);
  NormArgs g = args_of(c, s, gain);
  g.x = x;
  g.r = residual;
  g.y = y;
  g.sum = sum;
  g.pitch = (int)stash8_pitch(c.width);
  if (stash) {
    g.q = static_cast<uint8_t*>(stash);
    g.scales = g.q + c.rows * g.pitch;
  }
  const int64_t at_once = s.block ? 1 : 256 >> s.ls;
  launch<false>(st, c, s, std::min<int64_t>((c.rows + at_once - 1) / at_once, 2048), g);
}

size_t rms_norm_bwd_ws_bytes(int64_t rows, int64_t width) {
  return (size_t)bwd_blocks(rows, shape_of((int)width, false)) * (size_t)width * sizeof(float);
}

void rms_norm_bwd(hipStream_t st, const ast_norm_cfg& c, const void* dy, const void* sum, const float* gain, const void* dsum,
                  void* dx, void* ds, float* dgain, bool accumulate, void* ws) {
  const Shape s = shape_of((int)c.width, false);
  const int64_t blocks = c.rows > 0 ? bwd_blocks(c.rows, s) : 0;
  NormArgs g = args_of(c, s, gain);
  g.x = dy;
  g.s = sum;
  g.r = dsum;
  g.y = dx;
  g.sum = ds;
  g.part = static_cast<float*>(ws);
  if (blocks) launch<true>(st, c, s, blocks, g);
  KLAUNCH(rms_norm_gain_sum_kernel, dim3((unsigned)((c.width + 31) / 32)), dim3(1024), 0, st, g.part, (int)blocks, (int)c.width,
          dgain, (int)accumulate);
}

}  // namespace ast
