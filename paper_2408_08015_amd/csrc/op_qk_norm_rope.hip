// Norm and rotation of queries and keys, forward and backward, one pass over the heads each.
//
//   n = x r,  r = 1 / sqrt(mean(x^2) + eps);  u = gain * n;  (y_a, y_b) = (u_a c - u_b s, u_a s + u_b c)
//   du = the rotation backwards of dy;  dgain += du * n;  h = gain * du;  dx = r (h - n mean(h n))
//
// Both are bound by the bytes of the heads where there are many of them: 32768 tokens of 32 + 8 heads of 128 in bf16 take 134 us
// forward, 5.0 TB/s, what a large copy reaches; 10007 tokens of 12 + 3 fp32 heads of 80 29 us backward, 5.0 TB/s.  Few tokens cost
// the chain of position, angle, head, sums: 128 tokens of 8 + 8 heads of 64 4.8 us, 4096 12 us backward (25 MB).  A lane holds both values of its pairs: VEC values from place a and VEC from
// place b of a head (half split: a and a + rotary / 2; neighbouring pairs, and values that are not rotated: 2 VEC in a row),
// so the rotation needs no exchange, and 2^ls lanes make a head.  The angles of a token serve all its heads: a block forms
// cos and sin of its tokens once, in LDS, 64-bit turns reduced to half a turn before they are rounded.
#include <algorithm>
#include <cmath>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

struct HeadsAt { const void* p; int64_t ts, hs; };

struct QkArgs {
  HeadsAt x[2], dy[2], y[2];  // queries, keys; y: the result, or dx
  const float* gain[2];
  const int32_t* pos;
  float* part;                // backward: [blocks][head_dim] sums of du * n
  int64_t tokens;
  double log2_theta;
  float eps, inv_dim, inv_heads[2];
  int period, heads[2], dim, rotary;
  int units, rot_units;       // units (a lane's places) of a head, and how many of them rotate
  int ls;                     // log2 of the lanes of a head
  int tb[2];                  // tokens a block takes at a time
  unsigned blocks_q;          // the first blocks take queries, the others keys
};

constexpr int QK_TRIG = 2048;  // pairs (cos, sin) of a block's tokens

// VEC consecutive values: as they are loaded, and as numbers
template <typename T, int VEC> struct Vec;
template <> struct Vec<bf16_t, 8> {
  typedef uint4 Raw;
  static __device__ __forceinline__ void expand(const Raw& a, float (&v)[8]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(f2bf_pk(v[0], v[1]), f2bf_pk(v[2], v[3]), f2bf_pk(v[4], v[5]), f2bf_pk(v[6], v[7]));
  }
};
template <> struct Vec<float, 4> {
  typedef float4 Raw;
  static __device__ __forceinline__ void expand(const Raw& a, float (&v)[4]) { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <> struct Vec<bf16_t, 2> {
  typedef uint32_t Raw;
  static __device__ __forceinline__ void expand(const Raw& a, float (&v)[2]) {
    v[0] = __uint_as_float(a << 16);
    v[1] = __uint_as_float(a & 0xffff0000u);
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[2]) { *reinterpret_cast<uint32_t*>(p) = f2bf_pk(v[0], v[1]); }
};
template <> struct Vec<float, 2> {
  typedef float2 Raw;
  static __device__ __forceinline__ void expand(const Raw& a, float (&v)[2]) { v[0] = a.x; v[1] = a.y; }
  static __device__ __forceinline__ void store(float* p, const float (&v)[2]) { *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]); }
};
template <typename T> struct Vec<T, 1> {
  typedef T Raw;
  static __device__ __forceinline__ void expand(const Raw& a, float (&v)[1]) { v[0] = load1(&a); }
  static __device__ __forceinline__ void store(T* p, const float (&v)[1]) { store1(p, v[0]); }
};

// sum over the 2^ls lanes of a head, valid in each of them
__device__ __forceinline__ float head_sum(float v, int ls) {
  if (ls > 0) v += dpp_move<DPP_QUAD_SWAP1>(v);
  if (ls > 1) v += dpp_move<DPP_QUAD_SWAP2>(v);
  if (ls > 2) v += dpp_move<DPP_HALF_MIRROR>(v);
  if (ls > 3) v += dpp_move<DPP_ROW_MIRROR>(v);
  if (ls > 4) v += __shfl_xor(v, 16, 64);
  if (ls > 5) v += __shfl_xor(v, 32, 64);
  return v;
}

// ... and over the lanes that hold the same place of the wavefront's heads (rotations inside the rows of 16, then across them)
__device__ __forceinline__ float places_sum(float v, int ls) {
  if (ls < 4) v += dpp_move<0x128>(v);
  if (ls < 3) v += dpp_move<0x124>(v);
  if (ls < 2) v += dpp_move<0x122>(v);
  if (ls < 1) v += dpp_move<0x121>(v);
  if (ls < 5) v += __shfl_xor(v, 16, 64);
  if (ls < 6) v += __shfl_xor(v, 32, 64);
  return v;
}

// One lane's share of a head: IT units of 2 x VEC values.
template <typename T, int VEC, int IT, bool INTER, bool BWD>
__global__ __launch_bounds__(256, 4) void qk_norm_rope_kernel(const QkArgs g) {
  typedef Vec<T, VEC> V;
  __shared__ __attribute__((aligned(16))) float2 trig[QK_TRIG];
  __shared__ float red[BWD ? 4 * 256 : 1];
  const int tid = threadIdx.x, lane = tid & ((1 << g.ls) - 1), group = tid >> g.ls, groups = 256 >> g.ls;
  const int half = g.rotary / 2;
  const int w = blockIdx.x >= g.blocks_q;
  const unsigned block = blockIdx.x - (w ? g.blocks_q : 0), blocks = w ? gridDim.x - g.blocks_q : g.blocks_q;
  const int H = g.heads[w], tb = g.tb[w];
  const HeadsAt X = g.x[w], D = g.dy[w], Y = g.y[w];

  // this lane's places in a head, and their gains
  int pa[IT], pb[IT], pair[IT];
  bool on_a[IT], on_b[IT], rot[IT];
  float gain[IT][2][VEC], acc[IT][2][VEC];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int u = lane + (i << g.ls);
    rot[i] = u < g.rot_units;
    pair[i] = u * VEC;
    if (INTER) {
      pa[i] = u * 2 * VEC;
      pb[i] = pa[i] + VEC;
    } else {
      pa[i] = rot[i] ? u * VEC : g.rotary + (u - g.rot_units) * 2 * VEC;
      pb[i] = rot[i] ? pa[i] + half : pa[i] + VEC;
    }
    on_a[i] = u < g.units;  // (a unit's first place always exists)
    on_b[i] = on_a[i] && pb[i] < g.dim;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      gain[i][0][e] = on_a[i] ? g.gain[w][pa[i] + e] : 0.f;
      gain[i][1][e] = on_b[i] ? g.gain[w][pb[i] + e] : 0.f;
      acc[i][0][e] = acc[i][1][e] = 0.f;
    }
  }
  // this thread's share of the angles: one pair of every few tokens
  double turn = 0;
  const int tpass = half ? 256 / half : 1;  // tokens at a time (half <= 128)
  const int ti = half ? tid / half : 0, tp = half ? tid - ti * half : 0;
  if (half) turn = exp2(-(double)(2 * tp) / (double)g.rotary * g.log2_theta) * 0.15915494309189533577;

  for (int64_t t0 = (int64_t)block * tb; t0 < g.tokens; t0 += (int64_t)blocks * tb) {
    const int nt = (int)min((int64_t)tb, g.tokens - t0);
    const int rows = nt * H;
    struct Row {  // a head: where it lies, and its values as they were loaded
      int token, head;
      typename V::Raw x[IT][2], d[BWD ? IT : 1][2];
    };
    auto fetch = [&](int row, Row& r) __attribute__((always_inline)) {
      r.token = row < rows ? (int)(((float)row + 0.5f) * g.inv_heads[w]) : -1;  // row / H (exact: tb * H <= 2^20)
      r.head = row - r.token * H;
      if (r.token < 0) return;
      const T* src = static_cast<const T*>(X.p) + (t0 + r.token) * X.ts + r.head * X.hs;
      const T* dsrc = static_cast<const T*>(D.p) + (t0 + r.token) * D.ts + r.head * D.hs;
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int place = z ? pb[i] : pa[i];
          r.x[i][z] = typename V::Raw{};
          if (BWD) r.d[BWD ? i : 0][z] = typename V::Raw{};
          if (z ? on_b[i] : on_a[i]) {
            r.x[i][z] = *reinterpret_cast<const typename V::Raw*>(src + place);
            if (BWD) r.d[BWD ? i : 0][z] = *reinterpret_cast<const typename V::Raw*>(dsrc + place);
          }
        }
    };
    Row cur;
    fetch(group, cur);
    if (half) {
      __syncthreads();  // the last tokens' angles have been read
      if (ti < tpass)
        for (int t = ti; t < nt; t += tpass) {
          const int32_t p = g.pos ? g.pos[t0 + t] : (int32_t)((t0 + t) % g.period);
          double a = (double)p * turn;
          a -= rint(a);
          float s, c;
          sincospif(2.f * (float)a, &s, &c);
          trig[t * half + tp] = make_float2(c, s);
        }
      __syncthreads();
    }
    for (int row = group; row < rows; row += groups) {
      Row next;  // requested before this head is worked on
      fetch(row + groups, next);
      float x[IT][2][VEC], d[IT][2][VEC];
      float ss = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          V::expand(cur.x[i][z], x[i][z]);
          if (BWD) V::expand(cur.d[BWD ? i : 0][z], d[i][z]);
#pragma unroll
          for (int e = 0; e < VEC; ++e) ss += x[i][z][e] * x[i][z][e];
        }
      // the rotation of the pairs (u, v) in place, forwards or (BWD) backwards
      auto rotate = [&](int i, float (&a)[VEC], float (&b)[VEC]) __attribute__((always_inline)) {
        if (!rot[i]) return;
        const float2* cs = trig + cur.token * half + pair[i];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          // (a head that ends inside a unit has no second place: nothing there turns)
          const float2 f = !INTER || 2 * e < VEC || on_b[i] ? cs[e] : make_float2(1.f, 0.f);
          const float s = BWD ? -f.y : f.y;
          // pair e: (a_e, b_e), or neighbours: pairs 0 .. VEC/2 - 1 in a, the others in b
          float& p = INTER && VEC > 1 ? (2 * e < VEC ? a[(2 * e) % VEC] : b[(2 * e) % VEC]) : a[e];
          float& q = INTER && VEC > 1 ? (2 * e < VEC ? a[(2 * e + 1) % VEC] : b[(2 * e + 1) % VEC]) : b[e];
          const float u = p, v = q;
          p = u * f.x - v * s;
          q = u * s + v * f.x;
        }
      };
      if (BWD) {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          rotate(i, d[i][0], d[i][1]);
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < VEC; ++e) dot += d[i][z][e] * gain[i][z][e] * x[i][z][e];
        }
        dot = head_sum(dot, g.ls);
      }
      ss = head_sum(ss, g.ls);
      const float r = rsqrtf(ss * g.inv_dim + g.eps);
      if (BWD) {
        const float m = r * r * dot * g.inv_dim;  // r mean(h n) = r^2 mean(h x)
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              acc[i][z][e] += d[i][z][e] * (x[i][z][e] * r);
              x[i][z][e] = r * (d[i][z][e] * gain[i][z][e] - x[i][z][e] * m);
            }
      } else {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i][z][e] = x[i][z][e] * r * gain[i][z][e];
          rotate(i, x[i][0], x[i][1]);
        }
      }
      T* dst = static_cast<T*>(const_cast<void*>(Y.p)) + (t0 + cur.token) * Y.ts + cur.head * Y.hs;
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        if (on_a[i]) V::store(dst + pa[i], x[i][0]);
        if (on_b[i]) V::store(dst + pb[i], x[i][1]);
      }
      cur = next;
    }
  }

  if (BWD) {  // sums of the gains' gradients: over the heads of a wavefront, then over the wavefronts, in a fixed order
    const int wave = tid >> 6;
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float v = places_sum(acc[i][z][e], g.ls);
          if ((tid & 63) >> g.ls == 0 && (z ? on_b[i] : on_a[i])) red[wave * 256 + (z ? pb[i] : pa[i]) + e] = v;
        }
    __syncthreads();
    if (tid < g.dim) g.part[(int64_t)blockIdx.x * g.dim + tid] = red[tid] + red[256 + tid] + red[512 + tid] + red[768 + tid];
  }
}

// dgain[i] (+)= sum over the blocks, in 64 bits: 16 columns a block, 64 rows of it at a time
__global__ __launch_bounds__(1024) void qk_gain_sum_kernel(const float* __restrict__ part, int blocks_q, int blocks_k, int dim,
                                                           float* dq, float* dk, int accumulate) {
  __shared__ double sh[64][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4, w = blockIdx.y;
  const float* p = part + (w ? (int64_t)blocks_q * dim : 0) + col;
  const int blocks = w ? blocks_k : blocks_q;
  double s = 0;
  if (col < dim) {
#pragma unroll 8
    for (int b = row; b < blocks; b += 64) s += p[(int64_t)b * dim];
  }
  sh[row][threadIdx.x & 15] = s;
  __syncthreads();
  if (row < 8) {
    for (int r = row + 8; r < 64; r += 8) s += sh[r][threadIdx.x & 15];
    sh[row][threadIdx.x & 15] = s;
  }
  __syncthreads();
  if (row == 0 && col < dim) {
    for (int r = 1; r < 8; ++r) s += sh[r][threadIdx.x];
    float* out = (w ? dk : dq) + col;
    *out = (accumulate ? *out : 0.f) + (float)s;
  }
}

bool steps_of(const ast_heads& h, int bytes, int esize) {  // every head starts at a multiple of `bytes`
  return reinterpret_cast<uintptr_t>(h.dev) % bytes == 0 && h.token_stride * esize % bytes == 0 && h.head_stride * esize % bytes == 0;
}

constexpr int QK_MOST_BLOCKS = 1024;  // of a backward pass and of queries or keys: partial sums of the gains' gradients

struct Shape { int vec, it, ls, units, rot_units, tb[2]; unsigned blocks[2]; };

// Lanes and blocks of a call.  About 2048 blocks of queries and as many of keys forward, 1024 backward (whose blocks each leave
// partial sums): a block forms its angles and waits for its first loads once.  us, forward of 32768 tokens, 32 + 8 heads of
// 128, and backward of 10007 tokens, 12 + 3 fp32 heads of 80: 1024 blocks 145 and 38.4, 2048 blocks 140 and 42.2, blocks that
// take a token of every lane group 199 and 46.7.
Shape shape_of(const ast_qk_cfg& c, const int heads[2], int vec, bool bwd) {
  Shape s = {};
  s.vec = vec;
  s.it = vec == 1 ? 4 : vec == 2 ? 2 : 1;
  if (c.interleaved) {
    s.units = (c.head_dim + 2 * s.vec - 1) / (2 * s.vec);
    s.rot_units = (c.rotary + 2 * s.vec - 1) / (2 * s.vec);
  } else {
    s.rot_units = c.rotary / 2 / s.vec;
    s.units = s.rot_units + ((c.head_dim - c.rotary) / s.vec + 1) / 2;
  }
  while ((s.it << s.ls) < s.units) ++s.ls;  // (at most 128 units: no more than 32 lanes)
  const int groups = 256 >> s.ls;  // heads at a time
  for (int w = 0; w < 2; ++w) {
    const int most = bwd ? QK_MOST_BLOCKS : 2048;
    // (two heads a lane backward, one forward, where that leaves 128 and 256 blocks)
    const int64_t fill = bwd ? std::min<int64_t>((2 * groups + heads[w] - 1) / heads[w], c.tokens / 128)
                             : std::min<int64_t>((groups + heads[w] - 1) / heads[w], c.tokens / 256);
    int64_t tb = std::max<int64_t>((c.tokens + most - 1) / most, fill);
    if (c.rotary) tb = std::min<int64_t>(tb, QK_TRIG / (c.rotary / 2));
    tb = std::max<int64_t>(1, std::min<int64_t>({tb, 64, (1 << 20) / heads[w]}));
    s.tb[w] = (int)tb;
    const int64_t need = (c.tokens + tb - 1) / tb;
    s.blocks[w] = (unsigned)std::min<int64_t>(need, bwd ? QK_MOST_BLOCKS : 1 << 20);
  }
  return s;
}

void launch(hipStream_t st, const ast_qk_cfg& c, const ast_heads* dy, const ast_heads* x, const float* gq, const float* gk,
            const ast_heads* y, float* part, unsigned* blocks) {
  const bool bwd = dy != nullptr, bf = c.dtype == AST_BF16_F32ACC;
  QkArgs g = {};
  const int esize = bf ? 2 : 4;
  // values that are read and written at a time: 16 bytes, two, or one, as the head's parts and its addresses allow
  auto fits = [&](int v) {
    if (c.head_dim % v || !(c.interleaved ? c.rotary % (2 * v) == 0 || c.rotary == c.head_dim : c.rotary / 2 % v == 0)) return false;
    for (int w = 0; w < 2; ++w)
      if (!steps_of(x[w], v * esize, esize) || !steps_of(y[w], v * esize, esize) || (bwd && !steps_of(dy[w], v * esize, esize))) return false;
    return true;
  };
  const int vec = fits(16 / esize) ? 16 / esize : fits(2) ? 2 : 1;
  for (int w = 0; w < 2; ++w) {
    g.x[w] = {x[w].dev, x[w].token_stride, x[w].head_stride};
    g.y[w] = {y[w].dev, y[w].token_stride, y[w].head_stride};
    if (bwd) g.dy[w] = {dy[w].dev, dy[w].token_stride, dy[w].head_stride};
    g.heads[w] = x[w].heads;
    g.inv_heads[w] = 1.f / (float)x[w].heads;
  }
  const Shape s = shape_of(c, g.heads, vec, bwd);
  g.gain[0] = gq;
  g.gain[1] = gk;
  g.pos = c.positions_dev;
  g.period = c.period;
  g.part = part;
  g.tokens = c.tokens;
  g.log2_theta = std::log2(c.theta);
  g.eps = c.eps;
  g.inv_dim = 1.f / (float)c.head_dim;
  g.dim = c.head_dim;
  g.rotary = c.rotary;
  g.units = s.units;
  g.rot_units = s.rot_units;
  g.ls = s.ls;
  for (int w = 0; w < 2; ++w) {
    g.tb[w] = s.tb[w];
    blocks[w] = s.blocks[w];
  }
  g.blocks_q = s.blocks[0];
  const dim3 grid(s.blocks[0] + s.blocks[1]);
#define GO(T, VEC, IT)                                                                                                        \
  do {                                                                                                                        \
    if (bwd) {                                                                                                                \
      if (c.interleaved) KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, true, true>), grid, dim3(256), 0, st, g);                   \
      else KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, false, true>), grid, dim3(256), 0, st, g);                                \
    } else {                                                                                                                  \
      if (c.interleaved) KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, true, false>), grid, dim3(256), 0, st, g);                  \
      else KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, false, false>), grid, dim3(256), 0, st, g);                               \
    }                                                                                                                         \
  } while (0)
  if (bf) {
    if (vec == 8) GO(bf16_t, 8, 1);
    else if (vec == 2) GO(bf16_t, 2, 2);
    else GO(bf16_t, 1, 4);
  } else {
    if (vec == 4) GO(float, 4, 1);
    else if (vec == 2) GO(float, 2, 2);
    else GO(float, 1, 4);
  }
#undef GO
}

}  // namespace

void qk_norm_rope_fwd(hipStream_t st, const ast_qk_cfg& c, const ast_heads& q, const ast_heads& k, const float* gq,
                      const float* gk, const ast_heads& yq, const ast_heads& yk) {
  if (c.tokens <= 0) return;
  const ast_heads x[2] = {q, k}, y[2] = {yq, yk};
  unsigned blocks[2];
  launch(st, c, nullptr, x, gq, gk, y, nullptr, blocks);
}

size_t qk_norm_rope_bwd_ws_bytes(int64_t tokens, int head_dim) {  // (whatever the blocks' shape: at most one block a token)
  return (size_t)std::min<int64_t>(std::max<int64_t>(tokens, 1), QK_MOST_BLOCKS) * 2 * head_dim * sizeof(float);
}

void qk_norm_rope_bwd(hipStream_t st, const ast_qk_cfg& c, const ast_heads& dyq, const ast_heads& dyk, const ast_heads& q,
                      const ast_heads& k, const float* gq, const float* gk, const ast_heads& dq, const ast_heads& dk,
                      float* dgq, float* dgk, bool accumulate, void* ws) {
  const ast_heads dy[2] = {dyq, dyk}, x[2] = {q, k}, y[2] = {dq, dk};
  float* part = static_cast<float*>(ws);
  unsigned blocks[2] = {0, 0};
  if (c.tokens > 0) launch(st, c, dy, x, gq, gk, y, part, blocks);
  KLAUNCH(qk_gain_sum_kernel, dim3((unsigned)((c.head_dim + 15) / 16), 2), dim3(1024), 0, st, part, (int)blocks[0], (int)blocks[1],
          c.head_dim, dgq, dgk, (int)accumulate);
}

}  // namespace ast
