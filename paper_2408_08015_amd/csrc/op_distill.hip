// Distillation from a teacher's top logits: the loss of a row of logits, and its gradient.
//
//   p = softmax over the row's valid entries of t / tau,  q = softmax(z / tau),  q1 = softmax(z)
//   loss = (1 - l) tau^2 sum_k p_k (log p_k - log q_{id_k}) - l log q1_label
//   dz_v = dloss [ (1 - l) tau (q_v - sum over k with id_k = v of p_k) + l (q1_v - [v = label]) ]
//
// Bound by the bytes of the logits.  One pass gives the largest logit m and the sums of exp((z - m) / tau) and exp(z - m), each
// thread with a running maximum of its own; they are kept as they are (m, sum, sum), not as logarithms: what exp((z - m) / tau) / sum is
// off by goes by the distance from m, not by the size of the logits.  It is up to 2 (m - z) / tau steps of 2^-24, 0.6 in the mean
// square: one for the rounding of z - m, which any form in fp32 has, the other for that of the product with log2(e) / tau.  (The
// difference alone: 1 and 0.4.  The smallest normal values, at a distance of 87, are off by 1e-5 of themselves.)
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
  float *parts, *places_z;   // few rows, loss and gradient: sums of a row's slices [rows][slices][3]; logits at the entries' places [rows][entries + 1]
  int64_t row0;              // of the launch
  int vocab, entries, teacher_bf16, slices;
  float scale, inv_tau;      // log2(e) / tau; 1 / tau
  float kl, rate, mix;       // (1 - l) tau^2, (1 - l) tau, l
};

constexpr float kLog2e = 1.44269504f;
constexpr float kLowest = -3.402823466e38f;  // where a running maximum starts (an infinity would give NaN for -inf - -inf)
// A row of few values is a wavefront's: several times as many rows are under way, and none waits for another wavefront of its own.
constexpr int kFewValues = 4096, kFewEntries = 256;

__device__ __forceinline__ float exp_scaled(float x, float s) { return __builtin_amdgcn_exp2f(x * s); }

// How the two exponentials of a value are formed.  ONE: there is one only (no label counts, or the temperature is 1); SQUARE,
// FOURTH: the temperature is 2 or 4, and exp(x) is a power of exp(x / T); BOTH: any other temperature.  (us of loss and gradient in bf16
// with labels, at 2 as a square and as two exponentials: 4096 x 131072 457, 496, 2001 x 50021 100, 111, 8192 x 1000 18.7, 20.3; at 4: 478,
// 498, 105, 111, 19.3, 20.5; fp32 4096 x 32768 214, 216 and 216, 215.  Each product takes half of the gain, so no further powers.)
enum Exps : int { ONE = 0, SQUARE = 1, FOURTH = 2, BOTH = 3 };
template <Exps E>
__device__ __forceinline__ void exps(float d, float scale, float& a, float& b) {
  a = exp_scaled(d, scale);
  b = E == BOTH ? exp_scaled(d, kLog2e) : a;
  if (E == SQUARE || E == FOURTH) b *= b;
  if (E == FOURTH) b *= b;
}

struct Sums { float m, a, b; };  // maximum, sum at the temperature, sum without it
template <Exps E>
__device__ __forceinline__ void merge(Sums& s, float m, float a, float b, float scale) {
  const float top = fmaxf(s.m, m);
  float xa, xb, ya, yb;
  exps<E>(s.m - top, scale, xa, xb);
  exps<E>(m - top, scale, ya, yb);
  s.a = s.a * xa + a * ya;
  if (E != ONE) s.b = s.b * xb + b * yb;
  s.m = top;
}

template <Exps E>
__device__ __forceinline__ Sums wave_sums(Sums s, float scale) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    merge<E>(s, __shfl_xor(s.m, d, 64), __shfl_xor(s.a, d, 64), E != ONE ? __shfl_xor(s.b, d, 64) : 0.f, scale);
  return s;
}
template <int THREADS, Exps E>
__device__ __forceinline__ Sums block_sums(Sums s, float scale, float (*sh)[16]) {
  s = wave_sums<E>(s, scale);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh[0][wave] = s.m;
    sh[1][wave] = s.a;
    if (E != ONE) sh[2][wave] = s.b;
  }
  __syncthreads();
  s.m = sh[0][0], s.a = sh[1][0], s.b = E != ONE ? sh[2][0] : 0.f;
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) merge<E>(s, sh[0][w], sh[1][w], E != ONE ? sh[2][w] : 0.f, scale);
  if (E == ONE) s.b = s.a;
  return s;
}

// The teacher's side of a row, and the student's logits at its places.
template <int THREADS>
struct Entries {
  static constexpr int MOST = THREADS == 64 ? kFewEntries : 1024;
  __attribute__((aligned(16))) int id[MOST];  // -1: does not count
  float p[MOST], logp[MOST], z[MOST];
  float z_label;
};
template <int THREADS>
struct Places {  // of the ids' lowest bits: stand in the row, stand more than once
  static constexpr int SEEN = THREADS == 64 ? kFewValues : 32768;  // places that these bits tell apart
  uint32_t seen[SEEN / 32], twice[SEEN / 32];
};
// Every one of THREADS threads its entries; returns whether it has one that counts.  Logits are read from z where they lie in
// [lo, hi), or all of them from saved (a row's places_z).
template <int THREADS, typename T, typename E>
__device__ __forceinline__ bool gather(const DistillArgs& g, int64_t row, const T* z, const float* saved, int lo, int hi, int label, E& e) {
  bool any = false;
  for (int k = threadIdx.x; k < g.entries; k += THREADS) {
    const int64_t at = row * g.entries + k;
    int id = g.ids[at];
    const float t = g.teacher_bf16 ? bf2f(static_cast<const bf16_t*>(g.t)[at]) : static_cast<const float*>(g.t)[at];
    if (id < 0 || id >= g.vocab || t == -INFINITY) id = -1;
    e.id[k] = id;
    e.logp[k] = t;
    if (id >= 0) {
      if (saved) e.z[k] = saved[k];
      else if (id >= lo && id < hi) e.z[k] = load1(z + id);
      any = true;
    }
  }
  if (threadIdx.x < 3)  // (what a group of four reads behind the last entry)
    if (g.entries + (int)threadIdx.x < E::MOST) e.id[g.entries + threadIdx.x] = -1;
  if (threadIdx.x == THREADS - 1 && label >= 0) {
    if (saved) e.z_label = saved[g.entries];
    else if (label >= lo && label < hi) e.z_label = load1(z + label);
  }
  return any;
}
// p and log p, by one wavefront, once all entries are there; and which ids may stand several times
template <int THREADS>
__device__ __forceinline__ void teacher(const DistillArgs& g, Entries<THREADS>& e, int lane, Places<THREADS>* places) {
  float top = -INFINITY;
  for (int k = lane; k < g.entries; k += 64) {
    const float t = e.logp[k];
    if (e.id[k] >= 0) top = t > top || t != t ? t : top;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const float o = __shfl_xor(top, d, 64);
    top = o > top || o != o ? o : top;
  }
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
    const int id = e.id[k];
    if (id < 0) continue;
    e.p[k] *= inv;
    e.logp[k] -= ls;
    if (!places) continue;
    const uint32_t at = (uint32_t)id % Places<THREADS>::SEEN, bit = 1u << (at & 31);
    if (atomicOr(&places->seen[at / 32], bit) & bit) atomicOr(&places->twice[at / 32], bit);
  }
}

// A row in groups of eight from its first 16-byte address on; `head` values in front of them and `tail` behind, fewer than eight.
struct Split { int head, groups, tail; };
template <typename T>
__device__ __forceinline__ Split split_row(const T* z, int vocab) {
  Split s;
  s.head = min((int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(z)) & 15) / (int)sizeof(T), vocab);
  s.groups = (vocab - s.head) / 8;
  s.tail = vocab - s.head - s.groups * 8;
  return s;
}

// the sums of N groups at a time, each thread's own
template <typename T, Exps E, int N>
__device__ __forceinline__ void add_groups(Sums& s, const Eight<T, true> (&e)[N], float scale) {
  float v[N][8], top = s.m;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    e[u].values(v[u]);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, v[u][i]);
  }
  float a, b;
  exps<E>(s.m - top, scale, a, b);
  s.a *= a;
  if (E != ONE) s.b *= b;
  s.m = top;
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      exps<E>(v[u][i] - top, scale, a, b);
      s.a += a;
      if (E != ONE) s.b += b;
    }
}
// group `at` of a row, or -inf behind its last one
template <typename T>
__device__ __forceinline__ void load_group(Eight<T, true>& e, const T* z, int at, int groups, bool all) {
  e.load(z + (all ? at : min(at, groups - 1)) * 8);
  if (!all) {
#pragma unroll
    for (int i = 0; i < Eight<T, true>::N; ++i) e.v[i] = at < groups ? e.v[i] : sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  }
}

// the loss of a row, by one wavefront
template <int THREADS>
__device__ __forceinline__ float row_loss(const DistillArgs& g, const Entries<THREADS>& e, const Sums& s, bool label, int lane) {
  float loss = 0.f;
  if (g.kl != 0.f) {
    const float ls = logf(s.a);
    for (int k = lane; k < g.entries; k += 64)
      if (e.id[k] >= 0 && e.p[k] != 0.f) loss += e.p[k] * (e.logp[k] - ((e.z[k] - s.m) * g.inv_tau - ls));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) loss += __shfl_xor(loss, d, 64);
    loss *= g.kl;
  }
  if (label) loss -= g.mix * ((e.z_label - s.m) - logf(s.b));
  return loss;
}

// What a launch does.  A row is a block's, or, where there are few rows, cut into slices: PART sums a slice (and the first slice
// saves the logits at the entries' places: others may be writing the gradient in place of them later), JOIN_STEP adds the slices up.
enum Mode : int {
  LOSS = 0,           // loss and statistics
  GRADIENT = 1,       // the gradient from them (a slice)
  STEP = 2,           // loss and gradient
  PART = 3,
  JOIN_STEP = 4       // STEP from the sums of the slices
};
// KEEP: with STEP a thread keeps the first KEEP groups that it reads in registers, and the next STORE in shared memory; what a row has
// more is read again (from the caches, where it stayed there).
template <typename T, int THREADS, int KEEP, int STORE, Exps E, Mode MODE>
__global__ __launch_bounds__(THREADS, 4) void distill_kernel(const DistillArgs g) {
  constexpr bool SUMS = MODE == LOSS || MODE == STEP || MODE == PART, JOIN = MODE == JOIN_STEP;
  constexpr bool GRAD = MODE == GRADIENT || MODE == STEP || MODE == JOIN_STEP;
  constexpr bool CUT = MODE != LOSS && MODE != STEP;  // blockIdx.y: a slice
  constexpr int U = 4, K = KEEP ? KEEP : 1;  // U: groups that are asked for together
  __shared__ Entries<THREADS> e;
  __shared__ float sh[3][16];
  const int64_t row = g.row0 + blockIdx.x;
  const T* const z = static_cast<const T*>(g.z) + row * g.z_stride;
  const int tid = threadIdx.x, lane = tid & 63;
  Split sp = split_row(z, g.vocab);
  const int slice = CUT ? blockIdx.y : 0, slices = CUT ? gridDim.y : 1;
  const int per = CUT ? (sp.groups + slices - 1) / slices : sp.groups, g0 = min(slice * per, sp.groups);
  const bool lowest = slice == 0, highest = slice == slices - 1;
  const int lo = lowest ? 0 : sp.head + g0 * 8, hi = highest ? g.vocab : sp.head + min(g0 + per, sp.groups) * 8;
  const T* const zg = z + sp.head + g0 * 8;
  // the value in front of or behind the groups that falls to this thread
  const int behind = tid - (lowest ? sp.head : 0);
  const int odd = lowest && tid < sp.head ? tid : highest && behind >= 0 && behind < sp.tail ? sp.head + sp.groups * 8 + behind : -1;
  sp.groups = min(per, sp.groups - g0);

  int label = g.labels && g.mix != 0.f ? g.labels[row] : -1;
  if (label < 0 || label >= g.vocab) label = -1;
  const float w = GRAD ? g.dloss[row] : 1.f;
  constexpr int W = sizeof(T) / 2;  // 16 bytes each of a group
  __shared__ uint4 stored[STORE ? STORE * W : 1][STORE ? THREADS : 1];  // (a thread reads what it wrote)
  Eight<T, true> kept[K];
#pragma unroll
  for (int u = 0; u < KEEP; ++u)
    if (u * THREADS < sp.groups) load_group(kept[u], zg, tid + u * THREADS, sp.groups, (u + 1) * THREADS <= sp.groups);
  const float zodd = odd >= 0 ? load1(z + odd) : -INFINITY;
  bool any = false;  // an entry of the teacher's counts
  const float* const saved = JOIN ? g.places_z + row * (g.entries + 1) : nullptr;
  typedef Places<THREADS> Seen;
  Seen* places = nullptr;
  if constexpr (GRAD) {  // (what may be written in place of the logits waits for their values at the entries' places)
    __shared__ Seen store;
    places = &store;
    for (int i = tid; i < Seen::SEEN / 32; i += THREADS) places->seen[i] = places->twice[i] = 0;
    any = __syncthreads_or(gather<THREADS>(g, row, z, saved, lo, hi, label, e));
    if (tid < 64) teacher<THREADS>(g, e, lane, places);
  } else if constexpr (MODE == PART) {
    if (lowest) {
      float* const to = g.places_z + row * (g.entries + 1);
      for (int k = tid; k <= g.entries; k += THREADS) {
        const int id = k < g.entries ? g.ids[row * g.entries + k] : label;
        to[k] = id >= 0 && id < g.vocab ? load1(z + id) : 0.f;
      }
    }
  } else {  // (the others go on to the row; many entries are gathered by all: 8192 x 2000 with 512 47 us from 65, 2001 x 50021 with
            // 100 would take 53.7 from 51.8)
    if (g.entries > 128) {
      gather<THREADS>(g, row, z, saved, lo, hi, label, e);
      __syncthreads();
    } else if (tid < 64) {
      gather<64>(g, row, z, saved, lo, hi, label, e);
    }
    if (tid < 64) teacher<THREADS>(g, e, lane, nullptr);
  }

  Sums s = {kLowest, 0.f, 0.f};
  if constexpr (MODE == GRADIENT) s = {g.stats_in[row * 3], g.stats_in[row * 3 + 1], g.stats_in[row * 3 + 2]};
  if constexpr (JOIN) {
    const float* const p = g.parts + (row * g.slices + lane) * 3;
    if (lane < g.slices) s = {p[0], p[1], p[2]};
    s = wave_sums<E>(s, g.scale);
    if (E == ONE) s.b = s.a;
  }
  if constexpr (SUMS) {
    for (int at = tid + KEEP * THREADS; at - tid < sp.groups; at += U * THREADS) {
      Eight<T, true> r[U];
      const bool all = at - tid + U * THREADS <= sp.groups;
#pragma unroll
      for (int u = 0; u < U; ++u) load_group(r[u], zg, at + u * THREADS, sp.groups, all);
      if (STORE) {
        const int n = (at - tid) / THREADS - KEEP;  // (the same in all threads)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (n + u < STORE) {
#pragma unroll
            for (int w = 0; w < W; ++w) stored[(n + u) * W + w][tid] = reinterpret_cast<const uint4*>(r[u].v)[w];
          }
      }
      add_groups<T, E>(s, r, g.scale);
    }
#pragma unroll
    for (int u = 0; u < KEEP; u += 2)  // (the last slots may be empty)
      if ((u + 1) * THREADS < sp.groups) {
        const Eight<T, true> two[2] = {kept[u], kept[u + 1 < K ? u + 1 : u]};
        add_groups<T, E>(s, two, g.scale);
      } else if (u * THREADS < sp.groups) {
        const Eight<T, true> one[1] = {kept[u]};
        add_groups<T, E>(s, one, g.scale);
      }
    float oa, ob;
    exps<E>(zodd - fmaxf(zodd, kLowest), g.scale, oa, ob);
    merge<E>(s, fmaxf(zodd, kLowest), oa, ob, g.scale);
    s = block_sums<THREADS, E>(s, g.scale, sh);
  }
  if constexpr (MODE == PART) {
    if (tid < 3) g.parts[(row * g.slices + slice) * 3 + tid] = tid == 0 ? s.m : tid == 1 ? s.a : s.b;
    return;
  }
  if (MODE != GRADIENT && lowest && tid < 64) {
    const float loss = row_loss(g, e, s, label >= 0, lane);
    if (lane == 0) {
      g.loss[row] = loss;
      if (!GRAD) {
        g.stats[row * 3] = s.m;
        g.stats[row * 3 + 1] = s.a;
        g.stats[row * 3 + 2] = g.labels && g.mix != 0.f ? s.b : 0.f;
      }
    }
  }
  if constexpr (GRAD) {

  T* const dz = static_cast<T*>(g.dz) + row * g.dz_stride;
  T* const dg = dz + (zg - z);
  const float rate = any && g.rate != 0.f ? w * g.rate : 0.f, mix = label >= 0 ? w * g.mix : 0.f;
  const float ca = rate != 0.f ? rate / s.a : 0.f, cb = mix != 0.f ? mix / s.b : 0.f;
  auto slope = [&](float v) __attribute__((always_inline)) {  // dloss (rate q + mix q1)
    float a, b;
    exps<E>(v - s.m, g.scale, a, b);
    return E == ONE ? (ca + cb) * a : E == SQUARE ? a * fmaf(cb, a, ca) : ca * a + cb * b;
  };
  auto write = [&](const Eight<T, true>& r, int at) __attribute__((always_inline)) {
    float v[8];
    r.values(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = slope(v[i]);
    store8(dg + at * 8, v);
  };
  if (rate == 0.f && mix == 0.f) {  // (a token that does not count: zeros, whatever its logits are)
    const float zero[8] = {};
    for (int at = tid; at < sp.groups; at += THREADS) store8(dg + at * 8, zero);
    if (odd >= 0) store1(dz + odd, 0.f);
    return;
  }
#pragma unroll
  for (int u = 0; u < KEEP; ++u)
    if (tid + u * THREADS < sp.groups) write(kept[u], tid + u * THREADS);
  if (STORE) {
#pragma unroll
    for (int u = 0; u < STORE; ++u)
      if (tid + (KEEP + u) * THREADS < sp.groups) {
        Eight<T, true> r;
#pragma unroll
        for (int w = 0; w < W; ++w) reinterpret_cast<uint4*>(r.v)[w] = stored[u * W + w][tid];
        write(r, tid + (KEEP + u) * THREADS);
      }
  }
  for (int at = tid + (KEEP + STORE) * THREADS; at < sp.groups; at += U * THREADS) {
    Eight<T, true> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + u * THREADS < sp.groups) r[u].load(zg + (at + u * THREADS) * 8);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + u * THREADS < sp.groups) write(r[u], at + u * THREADS);
  }
  if (odd >= 0) store1(dz + odd, slope(zodd));
  __syncthreads();
  // The places of the teacher's entries and of the label: the first of equal ids writes the whole.  Few ids share their lowest bits
  // with another: only those look through the row for equal ones.
  for (int k = tid; k <= g.entries; k += THREADS) {
    const int id = k < g.entries ? e.id[k] : label;
    if (id < 0 || id < lo || id >= hi) continue;
    float p = k < g.entries ? e.p[k] : 0.f;
    bool first = true;
    const uint32_t at = (uint32_t)id % Seen::SEEN;
    if ((k < g.entries ? places->twice : places->seen)[at / 32] >> (at & 31) & 1) {
      p = 0.f;
      for (int j = 0; j < g.entries; j += 4) {
        const int4 q = *reinterpret_cast<const int4*>(e.id + j);
        if (q.x == id) p += e.p[j], first = first && j >= k;
        if (q.y == id) p += e.p[j + 1], first = first && j + 1 >= k;
        if (q.z == id) p += e.p[j + 2], first = first && j + 2 >= k;
        if (q.w == id) p += e.p[j + 3], first = first && j + 3 >= k;
      }
    }
    if (!first) continue;
    float a, b;
    exps<E>((k < g.entries ? e.z[k] : e.z_label) - s.m, g.scale, a, b);
    float x = 0.f;
    if (rate != 0.f) x = rate * (a / s.a - p);
    if (mix != 0.f) x += mix * (b / s.b - (id == label ? 1.f : 0.f));
    store1(dz + id, x);
  }
  }
}

// Slices of a row: of 8192 values or more where rows alone would leave compute units without a block.  The loss alone is never cut (16 bf16
// rows of 131072: 15.6 us in two launches, 11.5 in one).  us in slices and in one, 64 entries, a pass among others (8 us are the call's):
//                      gradient                                             loss and gradient (two launches in slices)
//             16384     32768     49152      65536      131072      16384      32768       49152       65536       131072    values
//   bf16  4   8.1, 8.2  8.1, 7.8  9.1, 9.3   9.4, 12.3  8.3, 15.5   13.0, 9.1  13.0, 8.9   12.8, 10.6  13.2, 16.3  12.5, 23.6
//        16   7.9, 8.0  8.0, 8.1  8.6, 10.5  9.3, 12.8  8.3, 16.0   12.5, 9.0  12.5, 8.8   12.9, 10.9  13.5, 16.7  13.3, 24.3
//        64   8.0, 8.1  8.0, 8.1  9.6, 9.3   10.5, 14.1 12.1, 18.2  12.3, 9.0  12.3, 9.8   13.7, 12.0  16.6, 17.9  18.1, 26.8
//   fp32 64   7.9, 7.9  8.1, 9.2  9.5, 11.7  12.7, 17.7 24.2, 42.7  12.3, 8.7  13.3, 10.3  15.7, 14.3  19.6, 21.2  30.8, 40.6
// The gradient gains or stays; loss and gradient gain from 65536 values on and lose up to 4 us below.  More than 64 rows, in 8 slices and
// in one: 128 x 131072 bf16 19.2, 24.1 and 28.9, 31.4, fp32 34.6, 48.8 and 48.4, 47.5; 200 x 131072 bf16 29.0, 29.9 and 40.4, 37.7.
int slices_of(int64_t rows, int64_t vocab) {
  if (rows > 64) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({64, vocab / 8192, 512 / std::max<int64_t>(rows, 1)}));
}

constexpr int64_t kRowsAtOnce = 1 << 22;  // (a launch has fewer than 2^32 threads)
template <Mode MODE, typename T, int THREADS, int KEEP, int STORE = 0>
void go(hipStream_t st, int64_t rows, int slices, DistillArgs g, Exps e) {
  const char* const name = MODE == GRADIENT ? "distill_bwd_kernel" : MODE == STEP || MODE == JOIN_STEP ? "distill_step_kernel" : "distill_kernel";
  auto run = [&](auto kernel) {
    for (g.row0 = 0; g.row0 < rows; g.row0 += kRowsAtOnce)
      KLAUNCH_NAMED(name, kernel, dim3((unsigned)std::min<int64_t>(rows - g.row0, kRowsAtOnce), (unsigned)slices), dim3(THREADS), 0, st, g);
  };
  if (e == ONE) run(distill_kernel<T, THREADS, KEEP, STORE, ONE, MODE>);
  else if (e == SQUARE) run(distill_kernel<T, THREADS, KEEP, STORE, SQUARE, MODE>);
  else if (e == FOURTH) run(distill_kernel<T, THREADS, KEEP, STORE, FOURTH, MODE>);
  else run(distill_kernel<T, THREADS, KEEP, STORE, BOTH, MODE>);
}
template <Mode MODE, typename T>
void pick(hipStream_t st, const ast_distill_cfg& c, const DistillArgs& g, Exps e) {
  const int64_t r = c.rows, v = c.vocab;
  // (us of 8192 rows with 32 entries, loss, gradient, both: 1000 bf16 13, 13, 17, in blocks of 256 threads 25, 27, 33; 4096 bf16 19, 34, 37
  // and 32, 39, 43; fp32 of 2048 17, 35, 34 and 32, 39, 39, of 4096 28, 65, 64 and 36, 57, 63)
  if (v <= (sizeof(T) == 2 || MODE == LOSS ? kFewValues : kFewValues / 2) && c.entries <= kFewEntries) {
    go<MODE, T, 64, MODE == STEP ? 8 : 0>(st, r, 1, g, e);
    return;
  }
  if constexpr (MODE == GRADIENT) {
    if (v <= 8192) go<MODE, T, 256, 0>(st, r, 1, g, e);
    else go<MODE, T, 512, 0>(st, r, g.slices, g, e);
  } else if constexpr (MODE == STEP) {
    if (g.slices > 1) {
      go<PART, T, 512, 0>(st, r, g.slices, g, e);
      go<JOIN_STEP, T, 512, 0>(st, r, g.slices, g, e);
    } else if (v <= 8192) go<MODE, T, 256, 4>(st, r, 1, g, e);
    else if (v <= 16384) go<MODE, T, 256, 8>(st, r, 1, g, e);
    // (what a row has more than 512 threads keep beside their work is read again; with shared memory for a part of it two blocks share
    // a unit as without.  us of 4096 rows, 131072 bf16 at temperatures of 2 and 1: 16 groups a thread 485, 481, and 4 in shared memory 472,
    // 467, 20 and 6 462, 452, 22 and 6 466, 446, but 100021 392 for 374; spilled from there on.  fp32, 40000 and 65536: 8 286, 467, 10 and 3
    // 268, 459)
    else if (v <= (sizeof(T) == 4 ? 8 : 16) * 512 * 8) go<MODE, T, 512, sizeof(T) == 4 ? 8 : 16>(st, r, 1, g, e);
    else go<MODE, T, 512, sizeof(T) == 4 ? 10 : 20, sizeof(T) == 4 ? 3 : 6>(st, r, 1, g, e);
  } else {
    if (v <= 8192) go<MODE, T, 256, 0>(st, r, 1, g, e);
    else go<MODE, T, 512, 0>(st, r, 1, g, e);
  }
}
template <Mode MODE>
void launch(hipStream_t st, const ast_distill_cfg& c, DistillArgs g, void* ws) {
  const float tau = c.temperature;
  const Exps e = !g.labels || g.mix == 0.f || tau == 1.f ? ONE : tau == 2.f ? SQUARE : tau == 4.f ? FOURTH : BOTH;
  g.slices = slices_of(c.rows, c.vocab);
  g.parts = static_cast<float*>(ws);
  g.places_z = g.parts + c.rows * g.slices * 3;
  if (c.dtype == AST_F32) pick<MODE, float>(st, c, g, e);
  else pick<MODE, bf16_t>(st, c, g, e);
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

size_t distill_step_ws_bytes(const ast_distill_cfg& c) {
  const int slices = slices_of(c.rows, c.vocab);
  return slices > 1 ? (size_t)c.rows * (size_t)(slices * 3 + c.entries + 1) * sizeof(float) : 0;
}

void distill_fwd(hipStream_t st, const ast_distill_cfg& c, const void* z, const int32_t* ids, const void* t, float* loss, float* stats) {
  DistillArgs g = args_of(c, z, ids, t);
  g.loss = loss;
  g.stats = stats;
  launch<LOSS>(st, c, g, nullptr);
}

void distill_bwd(hipStream_t st, const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t,
                 const float* stats, void* dz, int64_t dz_stride) {
  DistillArgs g = args_of(c, z, ids, t);
  g.dloss = dloss;
  g.stats_in = stats;
  g.dz = dz;
  g.dz_stride = dz_stride;
  launch<GRADIENT>(st, c, g, nullptr);
}

void distill_step(hipStream_t st, const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t,
                  float* loss, void* dz, int64_t dz_stride, void* ws) {
  DistillArgs g = args_of(c, z, ids, t);
  g.dloss = dloss;
  g.loss = loss;
  g.dz = dz;
  g.dz_stride = dz_stride;
  launch<STEP>(st, c, g, ws);
}

}  // namespace ast
