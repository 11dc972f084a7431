// Distillation from a teacher's top logits: the loss of a row of logits, and its gradient.
//
//   p = softmax over the row's valid entries of t / tau,  q = softmax(z / tau),  q1 = softmax(z)
//   loss = (1 - l) tau^2 sum_k p_k (log p_k - log q_{id_k}) - l log q1_label
//   dz_v = dloss [ (1 - l) tau (q_v - sum over k with id_k = v of p_k) + l (q1_v - [v = label]) ]
//
// Bound by the bytes of the logits.  One pass gives the largest logit m and the sums of exp((z - m) / tau) and exp(z - m), each
// thread with a running maximum of its own; they are kept as they are (m, sum, sum), not as logarithms: exp((z - m) / tau) / sum
// is good to a few roundings however large the logits are.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

struct DistillArgs {
  const void* z;
  void* dz;
  int64_t z_stride, dz_stride;
  const int32_t *ids, *labels;
  const void* t;
  const float *dloss, *stats_in;
  float *loss, *stats;
  int vocab, entries, teacher_bf16;
  float scale, inv_tau;      // log2(e) / tau; 1 / tau
  float kl, rate, mix;       // (1 - l) tau^2, (1 - l) tau, l
};

constexpr float kLog2e = 1.44269504f;
constexpr float kLowest = -3.402823466e38f;  // where a running maximum starts (an infinity would give NaN for -inf - -inf)
constexpr int kMostEntries = 1024;

__device__ __forceinline__ float exp_scaled(float x, float s) { return __builtin_amdgcn_exp2f(x * s); }

struct Sums { float m, a, b; };  // maximum, sum at the temperature, sum without it
template <bool TWO>
__device__ __forceinline__ void merge(Sums& s, float m, float a, float b, float scale) {
  const float top = fmaxf(s.m, m), x = exp_scaled(s.m - top, scale), y = exp_scaled(m - top, scale);
  s.a = s.a * x + a * y;
  if (TWO) s.b = s.b * exp_scaled(s.m - top, kLog2e) + b * exp_scaled(m - top, kLog2e);
  s.m = top;
}

template <int THREADS, bool TWO>
__device__ __forceinline__ Sums block_sums(Sums s, float scale, float (*sh)[16]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    merge<TWO>(s, __shfl_xor(s.m, d, 64), __shfl_xor(s.a, d, 64), TWO ? __shfl_xor(s.b, d, 64) : 0.f, scale);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh[0][wave] = s.m;
    sh[1][wave] = s.a;
    if (TWO) sh[2][wave] = s.b;
  }
  __syncthreads();
  s.m = sh[0][0], s.a = sh[1][0], s.b = TWO ? sh[2][0] : 0.f;
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) merge<TWO>(s, sh[0][w], sh[1][w], TWO ? sh[2][w] : 0.f, scale);
  return s;
}

// The teacher's side of a row, by one wavefront: p and log p of every entry, the student's logits at their places.
struct Entries {
  int id[kMostEntries];
  float p[kMostEntries], logp[kMostEntries], z[kMostEntries];
  bool any;  // one of them counts
};
template <typename T>
__device__ __forceinline__ void teacher(const DistillArgs& g, int64_t row, const T* z, Entries& e, int lane) {
  float top = -INFINITY;
  for (int k = lane; k < g.entries; k += 64) {
    const int64_t at = row * g.entries + k;
    int id = g.ids[at];
    const float t = g.teacher_bf16 ? bf2f(static_cast<const bf16_t*>(g.t)[at]) : static_cast<const float*>(g.t)[at];
    if (id < 0 || id >= g.vocab || t == -INFINITY) id = -1;
    e.id[k] = id;
    e.logp[k] = t;
    e.z[k] = id >= 0 ? load1(z + id) : 0.f;
    if (id >= 0) top = t > top || t != t ? t : top;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const float o = __shfl_xor(top, d, 64);
    top = o > top || o != o ? o : top;
  }
  if (lane == 0) e.any = top != -INFINITY;
  float sum = 0.f;
  for (int k = lane; k < g.entries; k += 64) {
    const float l = (e.logp[k] - top) * g.inv_tau, p = e.id[k] >= 0 ? expf(l) : 0.f;
    e.logp[k] = l;
    e.p[k] = p;
    sum += p;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  const float inv = 1.f / sum, ls = logf(sum);
  for (int k = lane; k < g.entries; k += 64) {
    if (e.id[k] < 0) continue;
    e.p[k] *= inv;
    e.logp[k] -= ls;
  }
}

template <typename T, bool EVEN, int THREADS, bool TWO>
__device__ __forceinline__ Sums row_stats(const DistillArgs& g, const T* z, float (*sh)[16]) {
  constexpr int U = 4;  // groups of eight that are asked for together
  Sums s = {kLowest, 0.f, 0.f};
  const int groups = g.vocab / 8;
  for (int at = threadIdx.x; at < groups; at += U * THREADS) {
    Eight<T, EVEN> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + u * THREADS < groups) e[u].load(z + (at + u * THREADS) * 8);
    float v[U][8], top = s.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = -INFINITY;
      if (at + u * THREADS < groups) e[u].values(v[u]);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, v[u][i]);
    }
    s.a *= exp_scaled(s.m - top, g.scale);
    if (TWO) s.b *= exp_scaled(s.m - top, kLog2e);
    s.m = top;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = v[u][i] - top;
        s.a += exp_scaled(d, g.scale);
        if (TWO) s.b += exp_scaled(d, kLog2e);
      }
  }
  if (groups * 8 + (int)threadIdx.x < g.vocab) {  // (the last values, fewer than eight)
    const float v = load1(z + groups * 8 + threadIdx.x), top = fmaxf(s.m, v);
    s.a = s.a * exp_scaled(s.m - top, g.scale) + exp_scaled(v - top, g.scale);
    if (TWO) s.b = s.b * exp_scaled(s.m - top, kLog2e) + exp_scaled(v - top, kLog2e);
    s.m = top;
  }
  return block_sums<THREADS, TWO>(s, g.scale, sh);
}

// the loss of a row, by one wavefront
__device__ __forceinline__ float row_loss(const DistillArgs& g, const Entries& e, const Sums& s, float zl, bool label, int lane) {
  float loss = 0.f;
  if (g.kl != 0.f) {
    const float ls = logf(s.a);
    for (int k = lane; k < g.entries; k += 64)
      if (e.id[k] >= 0 && e.p[k] != 0.f) loss += e.p[k] * (e.logp[k] - ((e.z[k] - s.m) * g.inv_tau - ls));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) loss += __shfl_xor(loss, d, 64);
    loss *= g.kl;
  }
  if (label) loss -= g.mix * ((zl - s.m) - logf(s.b));
  return loss;
}

// MODE 0: loss and statistics; 1: the gradient from them; 2: loss and gradient.
template <typename T, bool EVEN, int THREADS, bool TWO, int MODE>
__global__ __launch_bounds__(THREADS) void distill_kernel(const DistillArgs g) {
  __shared__ Entries e;
  __shared__ float sh[3][16];
  __shared__ float zl_sh;
  const int64_t row = blockIdx.x;
  const T* const z = static_cast<const T*>(g.z) + row * g.z_stride;
  const int lane = threadIdx.x & 63;
  int label = g.labels && g.mix != 0.f ? g.labels[row] : -1;
  if (label < 0 || label >= g.vocab) label = -1;
  const float w = MODE ? g.dloss[row] : 1.f;
  if (threadIdx.x < 64) {
    teacher(g, row, z, e, lane);
    if (lane == 0) zl_sh = label >= 0 ? load1(z + label) : 0.f;
  }
  Sums s;
  if (MODE == 1) {
    s = {g.stats_in[row * 3], g.stats_in[row * 3 + 1], g.stats_in[row * 3 + 2]};
    __syncthreads();
  } else {
    s = row_stats<T, EVEN, THREADS, TWO>(g, z, sh);
    if (!TWO) s.b = s.a;  // (no label, or a temperature of 1)
    if (threadIdx.x < 64) {
      const float loss = row_loss(g, e, s, zl_sh, label >= 0, lane);
      if (lane == 0) {
        g.loss[row] = loss;
        if (MODE == 0) {
          g.stats[row * 3] = s.m;
          g.stats[row * 3 + 1] = s.a;
          g.stats[row * 3 + 2] = g.labels && g.mix != 0.f ? s.b : 0.f;
        }
      }
    }
  }
  if (MODE == 0) return;

  T* const dz = static_cast<T*>(g.dz) + row * g.dz_stride;
  const float rate = e.any && g.rate != 0.f ? w * g.rate : 0.f, mix = label >= 0 ? w * g.mix : 0.f;
  const float ca = rate != 0.f ? rate / s.a : 0.f, cb = mix != 0.f ? mix / s.b : 0.f;
  auto slope = [&](float v) __attribute__((always_inline)) {  // dloss (rate q + mix q1)
    const float d = v - s.m;
    float x = 0.f;
    if (ca != 0.f) x = ca * exp_scaled(d, g.scale);
    if (cb != 0.f) x += cb * exp_scaled(d, kLog2e);
    return x;
  };
  const int groups = g.vocab / 8;
  for (int at = threadIdx.x; at < groups; at += THREADS) {
    Eight<T, EVEN> r;
    r.load(z + at * 8);
    float v[8];
    r.values(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = slope(v[i]);
    store8(dz + at * 8, v);
  }
  if (groups * 8 + (int)threadIdx.x < g.vocab) {
    const int at = groups * 8 + threadIdx.x;
    store1(dz + at, slope(load1(z + at)));
  }
  __syncthreads();
  // the places of the teacher's entries and of the label: the first of equal ones writes the whole
  for (int k = threadIdx.x; k <= g.entries; k += THREADS) {
    const int id = k < g.entries ? e.id[k] : label;
    if (id < 0) continue;
    float p = 0.f;
    bool first = true;
    for (int j = 0; j < g.entries; ++j)
      if (e.id[j] == id) {
        p += e.p[j];
        first = first && j >= k;
      }
    if (!first) continue;
    const float d = (k < g.entries ? e.z[k] : zl_sh) - s.m;
    float x = 0.f;
    if (rate != 0.f) x = rate * (exp_scaled(d, g.scale) / s.a - p);
    if (mix != 0.f) x += mix * (exp_scaled(d, kLog2e) / s.b - (id == label ? 1.f : 0.f));
    store1(dz + id, x);
  }
}

template <int MODE, typename T, bool EVEN>
void go(hipStream_t st, int64_t rows, const DistillArgs& g, bool two) {
  auto run = [&](auto kernel, int threads) { KLAUNCH_NAMED(MODE == 0 ? "distill_kernel" : MODE == 1 ? "distill_bwd_kernel" : "distill_step_kernel", kernel, dim3((unsigned)rows), dim3(threads), 0, st, g); };
  if (MODE == 1 || !two) run(distill_kernel<T, EVEN, 512, false, MODE>, 512);
  else run(distill_kernel<T, EVEN, 512, true, MODE>, 512);
}
template <int MODE>
void launch(hipStream_t st, const ast_distill_cfg& c, DistillArgs g) {
  const int es = c.dtype == AST_F32 ? 4 : 2;
  bool even = reinterpret_cast<uintptr_t>(g.z) % 16 == 0 && g.z_stride * es % 16 == 0;
  if (MODE) even = even && reinterpret_cast<uintptr_t>(g.dz) % 16 == 0 && g.dz_stride * es % 16 == 0;
  const bool two = g.labels && g.mix != 0.f && c.temperature != 1.f;
  if (c.dtype == AST_F32) even ? go<MODE, float, true>(st, c.rows, g, two) : go<MODE, float, false>(st, c.rows, g, two);
  else even ? go<MODE, bf16_t, true>(st, c.rows, g, two) : go<MODE, bf16_t, false>(st, c.rows, g, two);
}

DistillArgs args_of(const ast_distill_cfg& c, const void* z, const int32_t* ids, const void* t) {
  DistillArgs g = {};
  g.z = z;
  g.z_stride = c.logits_stride;
  g.ids = ids;
  g.labels = c.labels_dev;
  g.t = t;
  g.vocab = (int)c.vocab;
  g.entries = c.entries;
  g.teacher_bf16 = c.teacher_dtype != AST_F32;
  g.inv_tau = 1.f / c.temperature;
  g.scale = kLog2e / c.temperature;
  g.mix = c.labels_dev ? c.label_weight : 0.f;
  g.rate = (1.f - g.mix) * c.temperature;
  g.kl = g.rate * c.temperature;
  return g;
}

}  // namespace

void distill_fwd(hipStream_t st, const ast_distill_cfg& c, const void* z, const int32_t* ids, const void* t, float* loss, float* stats) {
  DistillArgs g = args_of(c, z, ids, t);
  g.loss = loss;
  g.stats = stats;
  launch<0>(st, c, g);
}

void distill_bwd(hipStream_t st, const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t,
                 const float* stats, void* dz, int64_t dz_stride) {
  DistillArgs g = args_of(c, z, ids, t);
  g.dloss = dloss;
  g.stats_in = stats;
  g.dz = dz;
  g.dz_stride = dz_stride;
  launch<1>(st, c, g);
}

void distill_step(hipStream_t st, const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t,
                  float* loss, void* dz, int64_t dz_stride) {
  DistillArgs g = args_of(c, z, ids, t);
  g.dloss = dloss;
  g.loss = loss;
  g.dz = dz;
  g.dz_stride = dz_stride;
  launch<2>(st, c, g);
}

}  // namespace ast
