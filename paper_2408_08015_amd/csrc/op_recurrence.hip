// Gated linear recurrence, forward and backward, one pass over the tokens each.
//
//   a = sigmoid(f),  h_t = a_t h_{t-1} + (1 - a_t) z_t,  y_t = h_t swish(o_t)
//   G_t = dy_t swish(o_t) + K_{t+1},  K_t = a_t G_t      (G: the gradient that reaches h_t; K: what it passes on to h_{t-1})
//   dz = (1 - a) G,  df = a (1 - a) (h_{t-1} - z) G,  do = dy h swish'(o)
//
// Both are scans of affine maps, x -> A x + U for a run of tokens, and bound by the bytes of the tokens' rows.  So the rows are read
// once: a wavefront holds TOK tokens of 64 (fp32) or 128 (bf16) channels in registers, forms their map, learns what comes in
// and finishes.  WAVES wavefronts of a block join their maps through LDS, blocks through the workspace:
//
//   a block leaves the map of its tokens in one 64-bit word a channel (A, U) as soon as it has it; 32 blocks in a row make a
//   group, and the last of them leaves the value behind the group.  What comes in to a block is the value in front of its group and the
//   maps of the group's earlier blocks, joined in their order: the result does not depend on which block ran when.
//
// A word is its own flag: the preparing launch fills them with a pattern that no map has, and a word is written once, by
// one atomic store.  Blocks take their place in the chain from a counter when they start, so a block only waits for ones that
// have started before it and wait for none behind them: every wait ends.
// A run in which a sequence starts passes nothing through: its A is -0 (products with it stay -0, and none of a sequence's
// infinities or NaN reach the next one).
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

constexpr int FWD_WAVES = 8, BWD_WAVES = 8;
constexpr int GROUP = 32;               // blocks of a chain whose maps are joined one by one
constexpr int FWD_TOK = 16, BWD_TOK = 8;  // tokens of a wavefront: 48 and 32 registers of loads (16 bits: two channels a register)
constexpr int COUNTER = 64;              // a counter's words: no two in one cache line
static_assert(BWD_TOK * BWD_WAVES == AST_RECURRENCE_CHUNK, "a block of the backward pass starts where a state was kept");
static_assert(FWD_TOK * FWD_WAVES % AST_RECURRENCE_CHUNK == 0 && AST_RECURRENCE_CHUNK % FWD_TOK == 0, "kept states are a wavefront's first");

constexpr uint32_t NOT_YET = 0xffffffffu;  // a NaN with a sign: maps are made without it

struct Rows { const void* p; int64_t stride; };

struct RecArgs {
  Rows f, z, o, dy;             // o.p may be nullptr
  void *y;                      // forward
  void *df, *dz, *dgo;          // backward
  int64_t df_stride, dz_stride, do_stride;
  const float *state, *dfinal;  // [sequences][channels] or nullptr
  float *final, *dstate;
  float* saved;                 // state in front of every AST_RECURRENCE_CHUNK-th token
  const int32_t* seq;           // a token's sequence, -1: none; nullptr: by offsets or t / period
  const int32_t* offsets;       // of a call of one chunk and fewer than 64 sequences, which prepares nothing; or nullptr
  int sequences;                // (where offsets is given)
  int64_t tokens, period;
  unsigned long long *maps, *heads;  // the chain: [chunk][channels], [group][channels]; nullptr: chunks on their own
  unsigned* counters;           // [columns], COUNTER apart
  int channels, columns, chunks;
};

// Consecutive channels of a lane, one register of a row.  Lanes behind the last channel read the last ones, and a lane that has
// one channel where others have two reads a pair and takes its upper half, so that no load waits for a condition.
struct Lane32 {
  typedef float T;
  static constexpr int V = 1;
  uint32_t at;  // bytes from a row's first value
  __device__ __forceinline__ Lane32(int c, int channels) : at(4u * (uint32_t)min(c, channels - 1)) {}
  __device__ __forceinline__ uint32_t load(const void* row) const { return *reinterpret_cast<const uint32_t*>(static_cast<const char*>(row) + at); }
  __device__ __forceinline__ void values(uint32_t w, float (&v)[1]) const { v[0] = __uint_as_float(w); }
  template <bool FULL> __device__ __forceinline__ void store(void* row, const float (&v)[1]) const {
    *reinterpret_cast<float*>(static_cast<char*>(row) + at) = v[0];
  }
};
struct __attribute__((packed, aligned(2))) Raw4 { uint32_t w; };
struct Lane16 {  // (two channels or more)
  typedef bf16_t T;
  static constexpr int V = 2;
  uint32_t at, first;  // first: the bytes that become the first value (v_perm_b32)
  __device__ __forceinline__ Lane16(int c, int channels)
      : at(2u * (uint32_t)min(c, channels - 2)), first(c < channels - 1 ? 0x01000c0cu : 0x03020c0cu) {}
  __device__ __forceinline__ uint32_t load(const void* row) const { return reinterpret_cast<const Raw4*>(static_cast<const char*>(row) + at)->w; }
  __device__ __forceinline__ void values(uint32_t w, float (&v)[2]) const {
    v[0] = __uint_as_float(__builtin_amdgcn_perm(w, w, first));
    v[1] = __uint_as_float(w & 0xffff0000u);
  }
  template <bool FULL> __device__ __forceinline__ void store(void* row, const float (&v)[2]) const {
    const uint32_t w = f2bf_pk(v[0], v[1]);
    char* const p = static_cast<char*>(row) + at;
    if (FULL || first == 0x01000c0cu) reinterpret_cast<Raw4*>(p)->w = w;
    else *reinterpret_cast<bf16_t*>(p + 2) = (bf16_t)w;
  }
};
struct Lane16One {  // one channel a lane: rows of a single one, and calls that would leave compute units without a block
  typedef bf16_t T;
  static constexpr int V = 1;
  uint32_t at;
  __device__ __forceinline__ Lane16One(int c, int channels) : at(2u * (uint32_t)min(c, channels - 1)) {}
  __device__ __forceinline__ uint32_t load(const void* row) const { return *reinterpret_cast<const bf16_t*>(static_cast<const char*>(row) + at); }
  __device__ __forceinline__ void values(uint32_t w, float (&v)[1]) const { v[0] = __uint_as_float(w << 16); }
  template <bool FULL> __device__ __forceinline__ void store(void* row, const float (&v)[1]) const {
    store1(reinterpret_cast<bf16_t*>(static_cast<char*>(row) + at), v[0]);
  }
};
// the rows of a wavefront's tokens, one after the other; behind the last token: that one again
template <int TOK>
struct RowsFrom {
  const char* p;
  int64_t step;
  int left;
  __device__ __forceinline__ RowsFrom(const Rows& r, int64_t t0, int64_t tokens, int esize)
      : p(static_cast<const char*>(r.p) + min(t0, tokens - 1) * r.stride * esize), step(r.stride * esize), left((int)min((int64_t)TOK, tokens - t0)) {}
  __device__ __forceinline__ const void* next() {
    const void* const at = p;
    if (--left > 0) p += step;
    return at;
  }
};
// a lane's channels of a row of fp32 states
template <int V>
__device__ __forceinline__ void load_state(const float* rows, int64_t row, int c, int channels, float (&v)[V]) {
  const float* const p = rows + row * channels;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = p[(uint32_t)min(c + i, channels - 1)];
}
template <int V>
__device__ __forceinline__ void store_state(float* rows, int64_t row, int c, int channels, const float (&v)[V]) {
  float* const p = rows + row * channels;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (c + i < channels) p[(uint32_t)(c + i)] = v[i];
}

// exp(-|x|), within about 2^-22 of it for fp32 tensors (the rest of the product with log2 e is added behind the exponential:
// 2^-24 of an argument of 20 would be 1e-6 of the result), with a product alone for bf16 ones: off by up to 1.3 |x| steps of 2^-24, 1e-6 at 12.
// That is far below a step of their results and reaches the fp32 states only; the rest would cost 65536 x 1024 in sequences of 64 115 us
// forward instead of 108, as one sequence 144 to 147 instead of 132 to 140, backward 232 instead of 223.
template <bool EXACT>
__device__ __forceinline__ float exp_neg(float x) {
  const float n = -fabsf(x), t = n * 1.44269504f;
  const float e = __builtin_amdgcn_exp2f(t);
  if (!EXACT) return e;
  const float rest = fmaf(n, 1.44269504f, -t) + n * 1.925963033e-8f;  // (log2 e in two parts)
  return n < -100.f ? 0.f : fmaf(e, rest * 0.69314718f, e);
}
// sigmoid(x) and 1 - sigmoid(x), each to the relative precision of the exponential; 0 and 1 at the infinities
template <bool EXACT>
__device__ __forceinline__ void gates(float x, float& a, float& b) {
  const float e = exp_neg<EXACT>(x);
  float r = __builtin_amdgcn_rcpf(1.f + e);
  if (EXACT) r = fmaf(r, fmaf(-(1.f + e), r, 1.f), r);  // (a step of Newton's method: the reciprocal is good to an ulp)
  const float s = e * r;
  a = x >= 0.f ? r : s;
  b = x >= 0.f ? s : r;
  asm volatile("" : "+v"(a), "+v"(b));  // (chosen here: kept for later, each choice would hold two more registers and a mask)
}

// Both in one register: the smaller one, which a subtraction from 1 gives the larger one of to its full precision, with the sign
// bit where it is sigmoid(x).
template <bool EXACT>
__device__ __forceinline__ float small_gate(float x) {
  const float e = exp_neg<EXACT>(x);
  float r = __builtin_amdgcn_rcpf(1.f + e);
  if (EXACT) r = fmaf(r, fmaf(-(1.f + e), r, 1.f), r);
  float s = __builtin_copysignf(e * r, x);
  asm volatile("" : "+v"(s));
  return s;
}
// a h + (1 - a) z, and A a
__device__ __forceinline__ float step(float s, float h, float z) {
  const float m = fabsf(s), big = 1.f - m;
  const bool neg = (int)__float_as_uint(s) < 0;
  return fmaf(m, neg ? h : z, big * (neg ? z : h));
}
__device__ __forceinline__ float keep(float s, float A) {
  const float m = fabsf(s);
  return A * ((int)__float_as_uint(s) < 0 ? m : 1.f - m);
}

__device__ __forceinline__ bool cut(float A) { return (int)__float_as_uint(A) < 0; }  // nothing passes through
// (A, U) behind (a, u): x -> A (a x + u) + U
__device__ __forceinline__ void join(float& a, float& u, float A, float U) {
  u = cut(A) ? U : fmaf(A, u, U);
  a = cut(A) ? A : a * A;
}

__device__ __forceinline__ unsigned long long map_word(float A, float U) {
  const uint32_t a = A != A ? 0x7fc00000u : __float_as_uint(A);
  return (unsigned long long)__float_as_uint(U) << 32 | a;
}
__device__ __forceinline__ void leave(unsigned long long* p, unsigned long long w) {
  __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long look(unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// What a wavefront's tokens are (the same in all its lanes): bit i stands for token i.
template <int TOK, bool FEW>  // FEW: g.offsets may be given
struct Tokens {
  unsigned live, start, last;  // belongs to a sequence; is its first; its last
  int32_t at;                  // lane i: the sequence of token i (0: with the token in front) or, by period, of token 0
  bool listed;
  __device__ __forceinline__ Tokens(const RecArgs& g, int64_t t0, int lane)
      : live(0), start(0), last(0), at(0), listed(g.seq != nullptr || (FEW && g.offsets != nullptr)) {
    if (t0 >= g.tokens) return;
    const int n = (int)min((int64_t)TOK, g.tokens - t0);
    if (listed) {
      const int64_t t = t0 - 1 + lane;  // (lanes 0 .. TOK + 1 count)
      if (FEW && g.offsets) {  // (lane i holds offsets[i]; counted: the sequences that begin at the token or in front of it)
        const int32_t o = g.offsets[min(lane, g.sequences)];
        for (int s = 0; s < g.sequences; ++s) at += __builtin_amdgcn_readlane(o, s) <= t ? 1 : 0;
        const bool in = t >= __builtin_amdgcn_readlane(o, 0) && t < __builtin_amdgcn_readlane(o, g.sequences);
        at = in && t < g.tokens && lane <= TOK + 1 ? at - 1 : -1;
      } else {
        at = t >= 0 && t < g.tokens && lane <= TOK + 1 ? g.seq[t] : -1;
      }
      const int32_t next = __builtin_amdgcn_update_dpp(-1, at, DPP_WAVE_SHL1, 0xF, 0xF, false);
      const bool differ = at != next;
      const unsigned long long all = (1ull << n) - 1, change = __ballot(differ);  // bit i: tokens i - 1 and i differ
      live = (unsigned)(__ballot(at >= 0) >> 1 & all);
      start = (unsigned)(change & live);
      last = (unsigned)(change >> 1 & live);
    } else {
      live = (1u << n) - 1;
      const unsigned period = (unsigned)g.period, s = (unsigned)t0 / period, into = (unsigned)t0 - s * period;  // (tokens < 2^31)
      at = (int32_t)s;
      if (into == 0) start |= 1;
      for (unsigned i = period - into; i < (unsigned)n; i += period) start |= 1u << i;
      for (unsigned i = period - into - 1; i < (unsigned)n; i += period) last |= 1u << i;
      if (t0 + n == g.tokens) last |= 1u << (n - 1);
    }
  }
  __device__ __forceinline__ int64_t sequence(int i) const {
    return (int64_t)__builtin_amdgcn_readlane(at, listed ? i + 1 : 0) + (listed ? 0 : __popc(start & ((2u << i) - 2)));
  }
};

// What comes out of sequences without tokens (copied, or 0 where nothing is passed in), by the wavefront of the call's one block
// of these channels.
template <int V>
__device__ __forceinline__ void pass_on(const RecArgs& g, const float* in, float* out, int c) {
  for (int s = 0; s < g.sequences; ++s) {
    if (g.offsets[s] != g.offsets[s + 1]) continue;
    float x[V] = {};
    if (in) load_state(in, s, c, g.channels, x);
    store_state(out, s, c, g.channels, x);
  }
}

// The chain.  Lane i takes the block's channels i, i + 64 here (words side by side), whichever it computes with.
// A block leaves its map: that of its wavefronts' maps in the order of the scan (`back`: from the last).
template <int V, int WAVES>
__device__ __forceinline__ void leave_map(const RecArgs& g, int at, int first, int lane, bool back, const float2 (*mine)[64 * V],
                                          float (&A)[V], float (&U)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = first + lane + 64 * v;
    A[v] = 1.f, U[v] = 0.f;
#pragma unroll 2
    for (int i = 0; i < WAVES; ++i) {
      const float2 m = mine[back ? WAVES - 1 - i : i][lane + 64 * v];
      join(A[v], U[v], m.x, m.y);
    }
    if (c < g.channels) leave(g.maps + (int64_t)at * g.channels + c, map_word(A[v], U[v]));
  }
}
// What comes in to a block whose place in the chain is `at`, in x[channel]; all threads of the block call it.  Every wavefront joins
// the maps of SHARE blocks in front; the first one joins theirs, steps from the value in front of the group, and leaves the
// next group's value if this block is its group's last ((A, U): what leave_map gave it).
template <int V, int WAVES>
__device__ __forceinline__ void come_in(const RecArgs& g, int at, int first, int wave, int lane, float2 (*got)[64 * V], const float (&A)[V],
                                        const float (&U)[V], float* x) {
  constexpr int SHARE = GROUP / WAVES;
  const int group = at / GROUP, r = at % GROUP;
  unsigned long long* const maps = g.maps + ((int64_t)group * GROUP + wave * SHARE) * g.channels;
  unsigned long long w[V][SHARE];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < SHARE; ++j) {  // (all asked for at once)
      const int c = first + lane + 64 * v;
      w[v][j] = wave * SHARE + j < r && c < g.channels ? look(maps + (int64_t)j * g.channels + c) : 0x3f800000u;  // (1, 0) from nobody
    }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float a = 1.f, b = 0.f;
#pragma unroll
    for (int j = 0; j < SHARE; ++j) {
      while ((uint32_t)w[v][j] == NOT_YET) {
        __builtin_amdgcn_s_sleep(1);
        w[v][j] = look(maps + (int64_t)j * g.channels + first + lane + 64 * v);
      }
      join(a, b, __uint_as_float((uint32_t)w[v][j]), __uint_as_float((uint32_t)(w[v][j] >> 32)));
    }
    got[wave][lane + 64 * v] = make_float2(a, b);
  }
  __syncthreads();
  if (wave == 0) {
    unsigned long long h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = first + lane + 64 * v;
      h[v] = group > 0 && c < g.channels ? look(g.heads + (int64_t)group * g.channels + c) : 0;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = first + lane + 64 * v;
      float a = 1.f, b = 0.f;
#pragma unroll 2
      for (int i = 0; i < WAVES; ++i) {
        const float2 m = got[i][lane + 64 * v];
        join(a, b, m.x, m.y);
      }
      while ((uint32_t)h[v] == NOT_YET && !cut(a)) {
        __builtin_amdgcn_s_sleep(1);
        h[v] = look(g.heads + (int64_t)group * g.channels + c);
      }
      const float in = cut(a) ? b : fmaf(a, __uint_as_float((uint32_t)(h[v] >> 32)), b);
      if (r == GROUP - 1 && at + 1 < g.chunks && c < g.channels)
        leave(g.heads + (int64_t)(group + 1) * g.channels + c, map_word(0.f, cut(A[v]) ? U[v] : fmaf(A[v], in, U[v])));
      x[lane + 64 * v] = in;
    }
  }
  __syncthreads();
}

// A block's channels and its place in their chain: in the order in which the blocks of these channels start where they wait for each
// other (one counter for all channels would be the call's bound: 8 to 10 ns a block).  Blocks go to the eight XCDs in turn: where
// blocks do not wait, every eighth one takes the next channels of the same tokens, so that the cache lines of rows which do not begin
// at one, shared by two blocks, meet in one L2 (20011 x 777 fp32 in sequences of 64: 53 us forward, 101 backward; next to each
// other 63 and 125).  In a chain the order of starting decides, and the blocks of one XCD take the same channels forward, which the
// last 3 % speak for (65536 x 1024 bf16: 137 against 141 us), and neighbouring ones backward (223 against 226, without o 176 against 193).
struct Place { int at, column; };
template <bool BACK>
__device__ __forceinline__ Place place(const RecArgs& g) {
  const bool apart = BACK || !g.maps;
  const unsigned k = apart ? blockIdx.x >> 3 : blockIdx.x, n = k / (unsigned)g.columns, column = k - n * (unsigned)g.columns;
  if (!g.maps) return {(int)(n * 8 + (blockIdx.x & 7)), (int)column};
  __shared__ int p;
  if (threadIdx.x == 0) p = (int)atomicAdd(g.counters + column * COUNTER, 1u);
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(p), (int)column};  // (the same in all lanes: rows have scalar addresses)
}

template <typename L, bool GATE>
__global__ __launch_bounds__(64 * FWD_WAVES, 4) void recurrence_kernel(const RecArgs g) {
  typedef typename L::T T;
  constexpr int V = L::V, TOK = FWD_TOK, WAVES = FWD_WAVES, ES = sizeof(T);
  constexpr bool EXACT = sizeof(T) == 4;
  __shared__ float2 mine[WAVES][64 * V];
  __shared__ float2 got[WAVES][64 * V];
  __shared__ float head[64 * V];
  const Place p = place<false>(g);
  if (p.at >= g.chunks) return;
  const int chunk = p.at, column = p.column;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (column * 64 + lane) * V;
  const L at(c, g.channels);
  const int64_t t0 = ((int64_t)chunk * WAVES + wave) * TOK;

  uint32_t rf[TOK], rz[TOK], ro[GATE ? TOK : 1];
  {
    RowsFrom<TOK> f(g.f, t0, g.tokens, ES), z(g.z, t0, g.tokens, ES), o(GATE ? g.o : g.z, t0, g.tokens, ES);
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      rf[i] = at.load(f.next());
      rz[i] = at.load(z.next());
      if (GATE) ro[GATE ? i : 0] = at.load(o.next());
    }
  }
  const Tokens<TOK, V == 1> tk(g, t0, lane);
  if (V == 1 && g.offsets && g.final && wave == FWD_WAVES - 1) pass_on<V>(g, g.state, g.final, c);
  // the gates, and the wavefront's map
  float s[TOK][V], A[V], U[V];
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    float f[V];
    at.values(rf[i], f);
#pragma unroll
    for (int v = 0; v < V; ++v) s[i][v] = small_gate<EXACT>(f[v]);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) A[v] = 1.f, U[v] = 0.f;
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    float z[V];
    at.values(rz[i], z);
    if (tk.start >> i & 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) U[v] = 0.f;
      if (g.state) load_state(g.state, tk.sequence(i), c, g.channels, U);
    }
    if (tk.live >> i & 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        U[v] = step(s[i][v], U[v], z[v]);
        A[v] = keep(s[i][v], A[v]);
        // (a first token's gate gives way to its state: the one in front, which may have been replaced by then, is read once)
        if (tk.start >> i & 1) s[i][v] = U[v];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i) asm volatile("" : "+v"(rz[i]));  // (what is formed of z and the gates is formed again below, not kept)
#pragma unroll
  for (int v = 0; v < V; ++v) mine[wave][lane * V + v] = make_float2(tk.start ? -0.f : A[v], U[v]);  // (a NaN gate is no way through)
  __syncthreads();
  if (g.maps && wave == 0) leave_map<V, WAVES>(g, chunk, column * 64 * V, lane, false, mine, A, U);
  // the output gates, while the map is under way
  float w[GATE ? TOK : 1][V];
  if (GATE) {
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      float o[V];
      at.values(ro[GATE ? i : 0], o);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float a, b;
        gates<EXACT>(o[v], a, b);
        w[GATE ? i : 0][v] = o[v] * a;
        asm volatile("" : "+v"(w[GATE ? i : 0][v]));
      }
    }
  }
  float in[V] = {}, x[V];
  if (g.maps) {
    come_in<V, WAVES>(g, chunk, column * 64 * V, wave, lane, got, A, U, head);
#pragma unroll
    for (int v = 0; v < V; ++v) in[v] = head[lane * V + v];
  }
  // through the wavefronts in front of this one
#pragma unroll
  for (int v = 0; v < V; ++v) {
    x[v] = in[v];
#pragma unroll 2
    for (int i = 0; i < wave; ++i) {
      const float2 m = mine[i][lane * V + v];
      x[v] = cut(m.x) ? m.y : fmaf(m.x, x[v], m.y);
    }
  }
  if (c >= g.channels || t0 >= g.tokens) return;
  if (g.saved && t0 % AST_RECURRENCE_CHUNK == 0) store_state(g.saved, t0 / AST_RECURRENCE_CHUNK, c, g.channels, x);
  auto finish = [&](auto full) __attribute__((always_inline)) {
    constexpr bool FULL = decltype(full)::value;
    char* row = static_cast<char*>(g.y) + t0 * g.channels * ES;
#pragma unroll
    for (int i = 0; i < TOK; ++i, row += (int64_t)g.channels * ES) {
      if (!(tk.live >> i & 1)) continue;
      float z[V], y[V];
      at.values(rz[i], z);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        x[v] = tk.start >> i & 1 ? s[i][v] : step(s[i][v], x[v], z[v]);
        y[v] = GATE ? x[v] * w[GATE ? i : 0][v] : x[v];
      }
      at.template store<FULL>(row, y);
      if (g.final && (tk.last >> i & 1)) store_state(g.final, tk.sequence(i), c, g.channels, x);
    }
  };
  if ((column + 1) * 64 * V <= g.channels) finish(std::true_type{});
  else finish(std::false_type{});
}

template <typename L, bool GATE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void recurrence_bwd_kernel(const RecArgs g) {
  typedef typename L::T T;
  constexpr int V = L::V, TOK = BWD_TOK, ES = sizeof(T);
  constexpr bool EXACT = sizeof(T) == 4;
  __shared__ float2 mine[WAVES][64 * V];
  __shared__ float2 mine_k[WAVES][64 * V];
  __shared__ float2 got[WAVES][64 * V];
  __shared__ float head[64 * V];
  const Place p = place<true>(g);
  if (p.at >= g.chunks) return;
  const int chunk = g.chunks - 1 - p.at, column = p.column;  // (the scan runs from the last token to the first)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (column * 64 + lane) * V;
  const L at(c, g.channels);
  const bool full = (column + 1) * 64 * V <= g.channels;
  const int64_t t0 = ((int64_t)chunk * WAVES + wave) * TOK;

  uint32_t rf[TOK], rz[TOK], rd[TOK], ro[GATE ? TOK : 1];
  {
    RowsFrom<TOK> f(g.f, t0, g.tokens, ES), z(g.z, t0, g.tokens, ES), d(g.dy, t0, g.tokens, ES), o(GATE ? g.o : g.z, t0, g.tokens, ES);
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      rf[i] = at.load(f.next());
      rd[i] = at.load(d.next());
      if (GATE) ro[GATE ? i : 0] = at.load(o.next());
      rz[i] = at.load(z.next());
    }
  }
  float h[V];  // the state in front of the block
  load_state(g.saved, (int64_t)chunk * (WAVES / BWD_WAVES), c, g.channels, h);
  const Tokens<TOK, V == 1> tk(g, t0, lane);
  if (V == 1 && g.offsets && g.dstate && wave == WAVES - 1) pass_on<V>(g, g.dfinal, g.dstate, c);

  // the gates, and the gradients at the tokens
  float a[TOK][V], b[TOK][V], d[TOK][V], q[GATE ? TOK : 1][V], A[V], U[V], K[V];
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    float f[V], o[V];
    at.values(rf[i], f);
    at.values(rd[i], d[i]);
    if (GATE) at.values(ro[GATE ? i : 0], o);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      gates<EXACT>(f[v], a[i][v], b[i][v]);
      if (GATE) {
        float s, n;
        gates<EXACT>(o[v], s, n);
        q[GATE ? i : 0][v] = d[i][v] * fmaf(o[v] * s, n, s);  // dy swish'(o)
        d[i][v] *= o[v] * s;
        asm volatile("" : "+v"(d[i][v]), "+v"(q[GATE ? i : 0][v]));
      }
    }
  }
  // forwards: the map of the states
#pragma unroll
  for (int v = 0; v < V; ++v) A[v] = 1.f, U[v] = 0.f;
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    float z[V];
    at.values(rz[i], z);
    if (tk.start >> i & 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) U[v] = 0.f;
      if (g.state) load_state(g.state, tk.sequence(i), c, g.channels, U);
    }
    if (tk.live >> i & 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        U[v] = fmaf(a[i][v], U[v], b[i][v] * z[v]);
        A[v] *= a[i][v];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i) asm volatile("" : "+v"(rz[i]));  // (the products with z are formed again below, not kept)
  // backwards: what the tokens pass on to the ones in front of them, without what comes in from behind
#pragma unroll
  for (int v = 0; v < V; ++v) K[v] = 0.f;
#pragma unroll
  for (int i = TOK - 1; i >= 0; --i) {
    if (!(tk.live >> i & 1)) continue;
    if (tk.last >> i & 1) {  // (what reaches the state behind a sequence is read once: dstate may be the same tensor)
#pragma unroll
      for (int v = 0; v < V; ++v) K[v] = 0.f;
      if (g.dfinal) {
        load_state(g.dfinal, tk.sequence(i), c, g.channels, K);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          d[i][v] += K[v];
          K[v] = 0.f;
        }
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) K[v] = tk.start >> i & 1 ? 0.f : a[i][v] * (d[i][v] + K[v]);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    mine[wave][lane * V + v] = make_float2(tk.start ? -0.f : A[v], U[v]);  // (a NaN gate is no way through)
    mine_k[wave][lane * V + v] = make_float2(tk.start ? -0.f : A[v], K[v]);
  }
  __syncthreads();
  if (g.maps && wave == 0) leave_map<V, WAVES>(g, p.at, column * 64 * V, lane, true, mine_k, A, K);
  // the state in front of this wavefront
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll 2
    for (int w = 0; w < wave; ++w) {
      const float2 m = mine[w][lane * V + v];
      h[v] = cut(m.x) ? m.y : fmaf(m.x, h[v], m.y);
    }
  // forwards again, with the states: the output gate's gradient; w: a (h_{t-1} - z)
  float w[TOK][V];
  auto states = [&](auto whole) __attribute__((always_inline)) {
    char* row = GATE ? static_cast<char*>(g.dgo) + t0 * g.do_stride * ES : nullptr;
#pragma unroll
    for (int i = 0; i < TOK; ++i, row += g.do_stride * ES) {
      float z[V], e[V];
      at.values(rz[i], z);
      if (tk.start >> i & 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = 0.f;
        if (g.state) load_state(g.state, tk.sequence(i), c, g.channels, h);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        w[i][v] = a[i][v] * (h[v] - z[v]);
        asm volatile("" : "+v"(w[i][v]));
        h[v] = fmaf(a[i][v], h[v], b[i][v] * z[v]);
        if (GATE) e[v] = q[GATE ? i : 0][v] * h[v];
      }
      if (GATE && (tk.live >> i & 1) && (decltype(whole)::value || c < g.channels)) at.template store<decltype(whole)::value>(row, e);
    }
  };
  if (full) states(std::true_type{});
  else states(std::false_type{});
  float x[V] = {};
  if (g.maps) {
    come_in<V, WAVES>(g, p.at, column * 64 * V, wave, lane, got, A, K, head);
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = head[lane * V + v];
  }
  if (c >= g.channels || t0 >= g.tokens) return;
#pragma unroll
  for (int v = 0; v < V; ++v)  // through the wavefronts behind this one
#pragma unroll 2
    for (int i = WAVES - 1; i > wave; --i) {
      const float2 m = mine_k[i][lane * V + v];
      x[v] = cut(m.x) ? m.y : fmaf(m.x, x[v], m.y);
    }
  // and backwards with what comes in
  auto finish = [&](auto whole) __attribute__((always_inline)) {
    char* fr = static_cast<char*>(g.df) + (t0 + TOK - 1) * g.df_stride * ES;
    char* zr = static_cast<char*>(g.dz) + (t0 + TOK - 1) * g.dz_stride * ES;
#pragma unroll
    for (int i = TOK - 1; i >= 0; --i, fr -= g.df_stride * ES, zr -= g.dz_stride * ES) {
      if (!(tk.live >> i & 1)) continue;
      if (tk.last >> i & 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = 0.f;
      }
      float df[V], dz[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float G = d[i][v] + x[v];
        dz[v] = b[i][v] * G;
        df[v] = w[i][v] * dz[v];
        x[v] = a[i][v] * G;
      }
      at.template store<decltype(whole)::value>(fr, df);
      at.template store<decltype(whole)::value>(zr, dz);
      if (tk.start >> i & 1) {
        if (g.dstate) store_state(g.dstate, tk.sequence(i), c, g.channels, x);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = 0.f;
      }
    }
  };
  if (full) finish(std::true_type{});
  else finish(std::false_type{});
}

// Sequences of one token each, forward, in calls that are not large: nothing is scanned.  Four channels a thread.
template <typename T, bool GATE>
__global__ __launch_bounds__(256) void recurrence_token_kernel(const RecArgs g) {
  constexpr bool EXACT = sizeof(T) == 4;
  const int per_row = (g.channels + 3) / 4;
  const int64_t n = g.tokens * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / per_row;
    const int c = (int)(i - t * per_row) * 4, some = min(4, g.channels - c);
    const T* const f = static_cast<const T*>(g.f.p) + t * g.f.stride + c;
    const T* const z = static_cast<const T*>(g.z.p) + t * g.z.stride + c;
    const T* const o = GATE ? static_cast<const T*>(g.o.p) + t * g.o.stride + c : nullptr;
    const int64_t at = t * g.channels + c;
    float fv[4], zv[4], ov[4], h[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = min(k, some - 1);
      fv[k] = load1(f + e);
      zv[k] = load1(z + e);
      if (GATE) ov[k] = load1(o + e);
      h[k] = g.state ? g.state[at + e] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k >= some) break;
      const float x = step(small_gate<EXACT>(fv[k]), h[k], zv[k]);
      float y = x;
      if (GATE) {
        float a, b;
        gates<EXACT>(ov[k], a, b);
        y *= ov[k] * a;
      }
      store1(static_cast<T*>(g.y) + at + k, y);
      if (g.final) g.final[at + k] = x;
      if (g.saved && t % AST_RECURRENCE_CHUNK == 0) g.saved[t / AST_RECURRENCE_CHUNK * g.channels + c + k] = 0.f;  // (the token begins a sequence)
    }
  }
}

// In front of a scan: the words of its chain and its counters, the tokens' sequences, and what comes out of sequences without
// tokens (copied, or 0 where nothing is passed in).
__global__ __launch_bounds__(256) void recurrence_prepare_kernel(unsigned long long* words, int64_t n_words, unsigned* counters, int columns,
                                                                 const int32_t* offsets, int64_t sequences, int64_t tokens,
                                                                 int32_t* seq, const float* in, float* out, int channels) {
  const int64_t me = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)gridDim.x * 256;
  if (counters)
    for (int64_t i = me; i < columns; i += all) counters[i * COUNTER] = 0;
  for (int64_t i = me; i < n_words; i += all) words[i] = ~0ull;
  if (!offsets) return;
  const int32_t first = offsets[0], end = offsets[sequences];
  for (int64_t t = me; t < tokens; t += all) {  // the last sequence that begins at the token or in front of it
    int64_t lo = 0, hi = sequences;             // offsets[lo] <= t < offsets[hi]
    if (t < first || t >= end) {
      seq[t] = -1;
      continue;
    }
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) / 2;
      if (offsets[mid] <= t) lo = mid;
      else hi = mid;
    }
    seq[t] = (int32_t)lo;
  }
  if (!out) return;
  const int64_t wave = me >> 6, waves = all >> 6;
  for (int64_t s = wave; s < sequences; s += waves) {
    if (offsets[s] != offsets[s + 1]) continue;
    for (int64_t c = threadIdx.x & 63; c < channels; c += 64) out[s * channels + c] = in ? in[s * channels + c] : 0.f;
  }
}

// The workspace: words of the chain, the counters, the tokens' sequences.
struct Layout { size_t maps, heads, counters, seq, end; int64_t words; int chunks, columns; bool chained, pairs; };
Layout layout_of(const ast_recurrence_cfg& c, int per) {
  Layout l = {};
  l.chunks = (int)((c.tokens + per - 1) / per);
  l.pairs = c.dtype != AST_F32 && c.channels > 1 && (int64_t)l.chunks * ((c.channels + 127) / 128) >= 1024;
  const int width = l.pairs ? 128 : 64;  // channels of a block
  l.columns = (int)((c.channels + width - 1) / width);
  // (chunks that each begin with a sequence's first token need nothing from each other)
  l.chained = l.chunks > 1 && (c.offsets_dev || per % c.period != 0);
  size_t at = 0;
  if (l.chained) {
    l.words = ((int64_t)l.chunks + (l.chunks + GROUP - 1) / GROUP) * c.channels;
    l.heads = (size_t)l.chunks * c.channels * 8;
    at = l.counters = (size_t)l.words * 8;
    at += (size_t)l.columns * COUNTER * 4;
  }
  l.seq = at;
  if (c.offsets_dev) at += ((size_t)c.tokens * 4 + 15) / 16 * 16;
  l.end = at;
  return l;
}

void prepare(hipStream_t st, const ast_recurrence_cfg& c, const Layout& l, void* ws, const float* in, float* out, RecArgs& g) {
  char* const w = static_cast<char*>(ws);
  g.tokens = c.tokens;
  g.period = c.period;
  g.channels = (int)c.channels;
  g.columns = l.columns;
  g.chunks = l.chunks;
  if (l.chained) {
    g.maps = reinterpret_cast<unsigned long long*>(w + l.maps);
    g.heads = reinterpret_cast<unsigned long long*>(w + l.heads);
    g.counters = reinterpret_cast<unsigned*>(w + l.counters);
  }
  if (!l.chained && !c.offsets_dev) return;
  // Nothing to prepare: the wavefronts of a block look their tokens' sequences up among fewer than 64 (64 x 512 bf16 in five: 10.5 us
  // forward, 12 backward, after a launch that prepares 14.2 and 14.8).
  if (l.chunks == 1 && !l.pairs && c.sequences < 64) {
    g.offsets = c.offsets_dev;
    g.sequences = (int)c.sequences;
    return;
  }
  if (c.offsets_dev) g.seq = reinterpret_cast<int32_t*>(w + l.seq);
  const int64_t most = std::max<int64_t>({l.words / 4, c.offsets_dev ? c.tokens : 0, c.offsets_dev && out ? 64 * c.sequences : 0, 1});
  KLAUNCH(recurrence_prepare_kernel, dim3((unsigned)std::min<int64_t>((most + 255) / 256, 2048)), dim3(256), 0, st, g.maps, l.words,
          g.counters, l.columns, c.offsets_dev, c.sequences, c.tokens, reinterpret_cast<int32_t*>(w + l.seq), in, out, (int)c.channels);
}

}  // namespace

// Backward in blocks of twice as many wavefronts: where sequences of that many tokens then need nothing from another block, in small
// calls (sequences of 128 tokens: 4096 x 512 bf16 10.7 us, in a chain 15.6; 8192 x 1024 39.2 and 38.4: one such block fills a compute
// unit).
static bool bwd_wide(const ast_recurrence_cfg& c) {
  const int per = BWD_TOK * BWD_WAVES;
  return !c.offsets_dev && c.tokens > per && per % c.period != 0 && 2 * per % c.period == 0 &&
         (c.tokens + per - 1) / per * ((c.channels + 63) / 64) <= 1024;
}

size_t recurrence_ws_bytes(const ast_recurrence_cfg& c) {
  return std::max(layout_of(c, FWD_TOK * FWD_WAVES).end, layout_of(c, (bwd_wide(c) ? 2 : 1) * BWD_TOK * BWD_WAVES).end);
}

void recurrence_fwd(hipStream_t st, const ast_recurrence_cfg& c, const ast_rows& f, const ast_rows& z, const ast_rows* o,
                    const float* state, void* y, float* final, float* saved, void* ws) {
  const Layout l = layout_of(c, FWD_TOK * FWD_WAVES);
  RecArgs g = {};
  g.f = {f.dev, f.stride};
  g.z = {z.dev, z.stride};
  if (o) g.o = {o->dev, o->stride};
  g.state = state;
  g.y = y;
  g.final = final;
  g.saved = saved;
  prepare(st, c, l, ws, state, final, g);
  if (l.chunks == 0) return;
  // (many tokens fill the blocks of a scan: bf16, 512 x 4096 9 us here, 11.8 there; 1024 x 4096 12.5 both; 8192 x 4096 80, 57)
  if (!c.offsets_dev && c.period == 1 && c.tokens * c.channels <= 1 << 22) {
    const int64_t n = c.tokens * ((c.channels + 3) / 4);
    const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16));
    auto go = [&](auto kernel) { KLAUNCH_NAMED("recurrence_token_kernel", kernel, grid, dim3(256), 0, st, g); };
    if (c.dtype == AST_F32) go(o ? recurrence_token_kernel<float, true> : recurrence_token_kernel<float, false>);
    else go(o ? recurrence_token_kernel<bf16_t, true> : recurrence_token_kernel<bf16_t, false>);
    return;
  }
  const dim3 grid((unsigned)(l.chunks + 7) / 8 * 8 * (unsigned)l.columns), block(64 * FWD_WAVES);
  auto go = [&](auto kernel) { KLAUNCH_NAMED("recurrence_kernel", kernel, grid, block, 0, st, g); };
  if (c.dtype == AST_F32) go(o ? recurrence_kernel<Lane32, true> : recurrence_kernel<Lane32, false>);
  else if (l.pairs) go(o ? recurrence_kernel<Lane16, true> : recurrence_kernel<Lane16, false>);
  else go(o ? recurrence_kernel<Lane16One, true> : recurrence_kernel<Lane16One, false>);
}

void recurrence_bwd(hipStream_t st, const ast_recurrence_cfg& c, const ast_rows& dy, const ast_rows& f, const ast_rows& z,
                    const ast_rows* o, const float* state, const float* saved, const float* dfinal, const ast_rows& df,
                    const ast_rows& dz, const ast_rows* dgo, float* dstate, void* ws) {
  const bool wide = bwd_wide(c);
  const Layout l = layout_of(c, (wide ? 2 : 1) * BWD_TOK * BWD_WAVES);
  RecArgs g = {};
  g.f = {f.dev, f.stride};
  g.z = {z.dev, z.stride};
  if (o) g.o = {o->dev, o->stride};
  g.dy = {dy.dev, dy.stride};
  g.df = const_cast<void*>(df.dev);
  g.dz = const_cast<void*>(dz.dev);
  g.df_stride = df.stride;
  g.dz_stride = dz.stride;
  if (dgo) {
    g.dgo = const_cast<void*>(dgo->dev);
    g.do_stride = dgo->stride;
  }
  g.state = state;
  g.saved = const_cast<float*>(saved);
  g.dfinal = dfinal;
  g.dstate = dstate;
  prepare(st, c, l, ws, dfinal, dstate, g);
  if (l.chunks == 0) return;
  const dim3 grid((unsigned)(l.chunks + 7) / 8 * 8 * (unsigned)l.columns), block(64 * (wide ? 2 : 1) * BWD_WAVES);
  auto go = [&](auto kernel) { KLAUNCH_NAMED("recurrence_bwd_kernel", kernel, grid, block, 0, st, g); };
#define PICK(L) (o ? go(recurrence_bwd_kernel<L, true, BWD_WAVES>) : go(recurrence_bwd_kernel<L, false, BWD_WAVES>))
#define PICK_WIDE(L) (o ? go(recurrence_bwd_kernel<L, true, 2 * BWD_WAVES>) : go(recurrence_bwd_kernel<L, false, 2 * BWD_WAVES>))
  if (c.dtype == AST_F32) wide ? PICK_WIDE(Lane32) : PICK(Lane32);
  else if (l.pairs) PICK(Lane16);  // (wide calls, of more than 64 tokens and at most 1024 blocks of 64 tokens and channels, have fewer than 1024 of 128)
  else wide ? PICK_WIDE(Lane16One) : PICK(Lane16One);
#undef PICK
#undef PICK_WIDE
}

}  // namespace ast
