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
// Rows whose length is no multiple of eight begin anywhere in a group of eight of the tensor, at the same place of it in every eighth
// row.  So a wavefront takes every eighth row (or a multiple of that), in the tensor's groups: loads and stores stay aligned, and its
// lanes keep their columns; only the groups at a row's ends, which it shares with its neighbours, are written value by value.
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

// How a row is read and written.  EVEN: its length is a multiple of eight and every tensor begins at a 16-byte address; GROUPS: the
// tensors do, in the tensor's groups of eight; ANY: from any address, shifted into place.
enum Way : int { ANY = 0, EVEN = 1, GROUPS = 2 };
template <typename T, Way W>
struct Part {  // eight values of a row from place c on (GROUPS: c may lie in front of the row)
  RowEight<T, W == EVEN> e;
  __device__ __forceinline__ void load(const void* base, int64_t row, int c, int cols, int64_t all) {
    const T* const p = static_cast<const T*>(base) + row * cols;
    e.load(p, c, cols);
  }
  __device__ __forceinline__ void values(float (&f)[8], int, int) const { e.values(f); }
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) asm volatile("" : "+v"(e.e.v[i]));
  }
};
template <typename T>
struct Part<T, GROUPS> {
  uint32_t v[2 * sizeof(T)];
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) asm volatile("" : "+v"(v[i]));
  }
  __device__ __forceinline__ void load(const void* base, int64_t row, int c, int cols, int64_t all) {
    const int64_t at = row * cols + c;  // (a multiple of eight; the tensor's last 16 bytes are read again where nothing follows them)
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const T*>(base) + at + (i == 0 || at + 4 < all ? 4 * i : 0));
      v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w;
    }
  }
  __device__ __forceinline__ void values(float (&f)[8], int c, int cols) const {
    eight_values<T>(v, f);
    if (c < 0 || c + 8 > cols) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (unsigned)(c + i) < (unsigned)cols ? f[i] : 0.f;
    }
  }
};
template <typename T, Way W>
__device__ __forceinline__ void store_part(void* base, int64_t row, int c, int cols, const float (&v)[8]) {
  T* const p = static_cast<T*>(base) + row * cols;
  if (W != GROUPS) {
    store_row8<T, W == EVEN>(p, c, cols, v);
  } else if (c >= 0 && c + 8 <= cols) {
    store8(p + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((unsigned)(c + i) < (unsigned)cols) store1(p + c + i, v[i]);
  }
}
__device__ __forceinline__ void gains(const NormArgs& g, int c, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (unsigned)(c + e) < (unsigned)g.cols ? g.gain[c + e] : 0.f;
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

// The rows of a group of lanes: the first one, how far it is to the next, and where it begins in a group of eight.
// BLOCK: threads that take one row together; 0: 2^ls lanes do, of 256 threads (GROUPS: 512, a wavefront for every row modulo eight).
template <Way W, int BLOCK>
struct Rows {
  static constexpr int THREADS = BLOCK ? BLOCK : W == GROUPS ? 512 : 256;
  int lanes, lane, shift;
  int64_t row, step;
  __device__ __forceinline__ Rows(const NormArgs& g) {
    lanes = BLOCK ? BLOCK : 1 << g.ls;
    lane = threadIdx.x & (lanes - 1);
    const int some = BLOCK ? 1 : THREADS >> g.ls;  // (by the block)
    if (BLOCK) {
      row = blockIdx.x;  // (the same for the block: rows have scalar addresses)
    } else if (W != GROUPS) {
      row = (int64_t)blockIdx.x * some + (threadIdx.x >> g.ls);
    } else {
      const int wave = threadIdx.x >> 6, of = (threadIdx.x & 63) >> g.ls;
      row = ((int64_t)blockIdx.x * (some / 8) + of) * 8 + wave;
    }
    step = (int64_t)gridDim.x * some;  // (GROUPS: a multiple of eight)
    shift = W == GROUPS ? (int)(row * g.cols & 7) : 0;
  }
  __device__ __forceinline__ int place(int i) const { return (lane + i * lanes) * 8 - shift; }
};

template <typename T, typename S, Way W, int IT, int BLOCK>
__global__ __launch_bounds__((Rows<W, BLOCK>::THREADS)) void rms_norm_kernel(const NormArgs g) {
  __shared__ float sh[2][32];
  Rows<W, BLOCK> at(g);
  const int64_t all = g.rows * g.cols;
  float gain[IT][8];
#pragma unroll
  for (int i = 0; i < IT; ++i) gains(g, at.place(i), gain[i]);
  struct Row {
    Part<T, W> x[IT];
    Part<S, W> r[IT];
  };
  auto fetch = [&](int64_t row, Row& w) __attribute__((always_inline)) {
    if (row >= g.rows) return;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = at.place(i);
      if (c >= g.cols) continue;
      w.x[i].load(g.x, row, c, g.cols, all);
      if (g.r) w.r[i].load(g.r, row, c, g.cols, all);
    }
  };
  Row cur;
  fetch(at.row, cur);
  int turn = 0;
  for (int64_t row = at.row; row < g.rows; row += at.step, turn ^= 1) {
    Row next;  // (asked for before this one is worked on)
    fetch(row + at.step, next);
    float v[IT][8], ss = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = at.place(i);
      if (c < g.cols) {
        cur.x[i].values(v[i], c, g.cols);
        if (g.r) {
          float r[8];
          cur.r[i].values(r, c, g.cols);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] += r[e];
          round_to(v[i], static_cast<const S*>(nullptr));
          store_part<S, W>(g.sum, row, c, g.cols, v[i]);
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
      const int c = at.place(i);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * rho * gain[i][e];
      if (c < g.cols) store_part<T, W>(g.y, row, c, g.cols, v[i]);
      if (W != GROUPS && g.q && c < g.pitch) {  // (a block of 32 values is four lanes' groups, all inside the pitch or none; values behind
                                                // the row are 0 times a finite rho, or their block has a NaN anyway)
        round_to(v[i], static_cast<const T*>(nullptr));
        uint2 w;
        const uint8_t scale = stash8_block(v[i], w);
        *reinterpret_cast<uint2*>(g.q + row * g.pitch + c) = w;
        if ((at.lane & 3) == 0) g.scales[row * (g.pitch / kStash8Block) + c / kStash8Block] = scale;
      }
    }
    cur = next;
  }
}

template <typename T, typename S, Way W, int IT, int BLOCK>
__global__ __launch_bounds__((Rows<W, BLOCK>::THREADS)) void rms_norm_bwd_kernel(const NormArgs g) {
  __shared__ float sh[2][32];
  Rows<W, BLOCK> at(g);
  const int64_t all = g.rows * g.cols;
  // Four groups a lane: the next row is not asked for early, and values are formed from the loaded words again behind the sums, or
  // the rows do not fit the registers.
  constexpr bool AHEAD = IT < 4, AGAIN = IT == 4;
  float gain[IT][8], acc[IT][8];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    gains(g, at.place(i), gain[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
  }
  struct Row {
    Part<T, W> d[IT];
    Part<S, W> s[IT], r[IT];
  };
  auto fetch = [&](int64_t row, Row& w) __attribute__((always_inline)) {
    if (row >= g.rows) return;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = at.place(i);
      if (c >= g.cols) continue;
      w.d[i].load(g.x, row, c, g.cols, all);
      w.s[i].load(g.s, row, c, g.cols, all);
      if (g.r) w.r[i].load(g.r, row, c, g.cols, all);
    }
  };
  Row cur;
  if (AHEAD) fetch(at.row, cur);
  int turn = 0;
  for (int64_t row = at.row; row < g.rows; row += at.step, turn ^= 1) {
    Row next;
    if (AHEAD) fetch(row + at.step, next);
    else fetch(row, cur);
    float s[IT][8], d[IT][8], ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = at.place(i);
      if (c < g.cols) {
        cur.s[i].values(s[i], c, g.cols);
        cur.d[i].values(d[i], c, g.cols);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = d[i][e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss += s[i][e] * s[i][e];
        dot += d[i][e] * gain[i][e] * s[i][e];
      }
    }
    row_sums<BLOCK>(ss, dot, true, g.ls, sh, turn);
    const float rho = rsqrtf(ss * g.inv + g.eps);
    const float m = rho * rho * dot * g.inv;  // mean(h n) rho = rho^2 mean(h s)
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = at.place(i);
      if (c >= g.cols) continue;
      float r[8] = {};
      if (AGAIN) {  // (pinned, or the compiler keeps the values of before)
        cur.s[i].pin();
        cur.d[i].pin();
        cur.s[i].values(s[i], c, g.cols);
        cur.d[i].values(d[i], c, g.cols);
      }
      if (g.r) cur.r[i].values(r, c, g.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[i][e] += d[i][e] * (s[i][e] * rho);
        s[i][e] = rho * (d[i][e] * gain[i][e] - s[i][e] * m) + r[e];
      }
      if (g.y) store_part<T, W>(g.y, row, c, g.cols, s[i]);
      if (g.sum) store_part<S, W>(g.sum, row, c, g.cols, s[i]);
    }
    if (AHEAD) cur = next;
  }
  // the gains' gradients: over the rows of a wavefront, then over the wavefronts
  float* const part = g.part + (int64_t)blockIdx.x * g.cols;
  if (BLOCK) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int c = at.place(i);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((unsigned)(c + e) < (unsigned)g.cols) part[c + e] = acc[i][e];
    }
    return;
  }
  constexpr int WIDE = IT * 64 * 8, WAVES = Rows<W, BLOCK>::THREADS / 64;
  __shared__ float red[BLOCK ? 1 : WAVES * WIDE];
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = at.place(i) + e;
      const float v = places_sum(acc[i][e], g.ls);
      if ((threadIdx.x & 63) >> g.ls == 0 && (unsigned)c < (unsigned)g.cols) red[wave * WIDE + c] = v;
    }
  __syncthreads();
  for (int c = threadIdx.x; c < g.cols; c += WAVES * 64) {
    float v = red[c];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += red[i * WIDE + c];
    part[c] = v;
  }
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

struct Shape { int it, block, ls, groups; };

// Lanes of a row: one group of eight values a lane up to 512 values, two up to 1024; then a block's of 256, 512 threads, two groups a
// lane, and four in 512 threads: their registers hold 2048 groups where those of 1024 threads spill (us of 2048 rows of 16384 in bf16
// and of 4096 of 10001: forward 88, 85, backward 74, 84; with 1024 threads 96, 119, 152, 209).
Shape shape_of(int cols, bool keep, Way way) {
  const int groups = (cols + (way == GROUPS ? 14 : 7)) / 8;
  Shape s = {1, 0, keep ? 2 : 0, groups};  // (8 bits: four lanes a block of 32 values)
  if (groups <= 128) {
    if (groups > 64) s.it = 2;
    while ((s.it << s.ls) < groups) ++s.ls;
    return s;
  }
  s.block = groups <= 512 ? 256 : 512;
  s.it = groups <= s.block ? 1 : groups <= 2 * s.block ? 2 : 4;
  return s;
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
Way way_of(int cols, bool aligned, bool keep, bool wide) {  // wide: backward on an fp32 stream
  if (!aligned) return ANY;
  if (cols % 8 == 0) return EVEN;
  // (8 bits lie in groups of a row's own; and where the one group more, that of a row which begins inside one, takes four groups a lane
  // instead of two, the backward pass on an fp32 stream loses: 4096 rows of 8191, bf16 on fp32: 153 us, 117 shifted into place; bf16:
  // 71 and 103; forward 96 and 104, 73 and 97)
  const bool over = wide && (cols + 14) / 8 > 1024 && cols <= 8192;
  return keep || over || cols > 16376 ? ANY : GROUPS;
}

// Blocks of a call: as many as rows need, at most 2048 forward.  Backward every block leaves partial sums; us of 12288 rows of 1504,
// bf16 on an fp32 stream, of 32768 of 1024, and of 4096 of 8192 in bf16: 1024 blocks 63.6, 61.0, 84.5; 512 57.9, 56.2, 68.2;
// 256 74.1, 65.7, 60.7.  On a bf16 stream 512 leave too little under way where a row leaves lanes without a group: so many more (32 M values
// in rows of 24, 40, 200, 1025, 1201, 1600: 53, 57, 54, 63, 65, 54 us, with 512 63, 71, 64, 93, 82, 64; not where rows are full, 2048 57
// for 55.5 with 768, nor for two groups a lane, 700 74 for 68).  Rows that are shifted into place keep more of them busy (12289 of 1501 so: 68.7, 74.4, 127).
constexpr int kMostPartials = 1024;
int64_t blocks_of(int64_t rows, const Shape& s, Way way, bool bwd, bool wide) {
  const int64_t at_once = s.block ? 1 : (way == GROUPS ? 512 : 256) >> s.ls;
  int64_t most = !bwd ? 2048 : way == ANY && s.block < 512 ? kMostPartials : s.block < 512 ? 512 : 256;
  if (bwd && !wide && s.it == 1 && (way == EVEN || (way == GROUPS && s.block)))
    most = (512 * (s.block ? s.block : 1 << s.ls) / s.groups + 128) / 256 * 256;
  int64_t n = std::max<int64_t>(1, std::min<int64_t>((rows + at_once - 1) / at_once, most));
  if (bwd && s.block) n = std::min(n, std::max<int64_t>(256, rows / 4));  // (1024 bf16 rows of 4096: 512 blocks 20.1 us, 256 16.7)
  return s.block && way == GROUPS ? (n + 7) / 8 * 8 : n;  // (a block's rows begin at one place of a group)
}

template <bool BWD, typename T, typename S, Way W, int IT, int BLOCK>
void go(hipStream_t st, int64_t blocks, const NormArgs& g) {
  const dim3 grid((unsigned)blocks), block(Rows<W, BLOCK>::THREADS);
  if (BWD) KLAUNCH_NAMED("rms_norm_bwd_kernel", (rms_norm_bwd_kernel<T, S, W, IT, BLOCK>), grid, block, 0, st, g);
  else KLAUNCH_NAMED("rms_norm_kernel", (rms_norm_kernel<T, S, W, IT, BLOCK>), grid, block, 0, st, g);
}
template <bool BWD, typename T, typename S, Way W>
void pick(hipStream_t st, int64_t blocks, const Shape& s, const NormArgs& g) {
  if (s.block == 0) {
    if (s.it == 1) go<BWD, T, S, W, 1, 0>(st, blocks, g);
    else go<BWD, T, S, W, 2, 0>(st, blocks, g);
  } else if (s.block == 256) {
    if (s.it == 1) go<BWD, T, S, W, 1, 256>(st, blocks, g);
    else go<BWD, T, S, W, 2, 256>(st, blocks, g);
  } else if (s.it == 2) {
    go<BWD, T, S, W, 2, 512>(st, blocks, g);
  } else {
    go<BWD, T, S, W, 4, 512>(st, blocks, g);
  }
}
template <bool BWD>
void launch(hipStream_t st, const ast_norm_cfg& c, Way way, const Shape& s, int64_t blocks, const NormArgs& g) {
  const bool tb = c.dtype != AST_F32, sb = c.sum_dtype != AST_F32;
#define PICK(T, S)                                                  \
  (way == EVEN ? pick<BWD, T, S, EVEN>(st, blocks, s, g)            \
               : way == GROUPS ? pick<BWD, T, S, GROUPS>(st, blocks, s, g) : pick<BWD, T, S, ANY>(st, blocks, s, g))
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
  const int cols = (int)c.width;
  const Way way = way_of(cols, aligned16(x) && aligned16(residual) && aligned16(y) && aligned16(sum), stash != nullptr,
                         false);
  const Shape s = shape_of(cols, stash != nullptr, way);
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
  launch<false>(st, c, way, s, blocks_of(c.rows, s, way, false, false), g);
}

size_t rms_norm_bwd_ws_bytes(int64_t rows, int64_t width) {  // (whatever the tensors' addresses and types: fp32 streams take no more)
  int64_t most = 0;
  for (const Way way : {ANY, EVEN, GROUPS}) most = std::max(most, blocks_of(rows, shape_of((int)width, false, way), way, true, false));
  return (size_t)most * (size_t)width * sizeof(float);
}

void rms_norm_bwd(hipStream_t st, const ast_norm_cfg& c, const void* dy, const void* sum, const float* gain, const void* dsum,
                  void* dx, void* ds, float* dgain, bool accumulate, void* ws) {
  const int cols = (int)c.width;
  const Way way = way_of(cols, aligned16(dy) && aligned16(sum) && aligned16(dsum) && aligned16(dx) && aligned16(ds), false,
                         c.sum_dtype == AST_F32);
  const Shape s = shape_of(cols, false, way);
  const int64_t blocks = c.rows > 0 ? blocks_of(c.rows, s, way, true, c.sum_dtype == AST_F32) : 0;
  NormArgs g = args_of(c, s, gain);
  g.x = dy;
  g.s = sum;
  g.r = dsum;
  g.y = dx;
  g.sum = ds;
  g.part = static_cast<float*>(ws);
  if (blocks) launch<true>(st, c, way, s, blocks, g);
  KLAUNCH(rms_norm_gain_sum_kernel, dim3((unsigned)((c.width + 31) / 32)), dim3(1024), 0, st, g.part, (int)blocks, (int)c.width,
          dgain, (int)accumulate);
}

}  // namespace ast
