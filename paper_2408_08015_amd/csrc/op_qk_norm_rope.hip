// Norm and rotation of queries and keys, forward and backward, one pass over the heads each.
//
//   n = x r,  r = 1 / sqrt(mean(x^2) + eps);  u = gain * n;  (y_a, y_b) = (u_a c - u_b s, u_a s + u_b c)
//   du = the rotation backwards of dy;  dgain += du * n;  h = gain * du;  dx = r (h - n mean(h n))
//
// Both are bound by the bytes of the heads.  A lane holds both values of its pairs: VEC values from place a and VEC from
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

struct HeadsIn { const void* p; int64_t ts, hs; };
struct HeadsOut { void* p; int64_t ts, hs; };

struct QkArgs {
  HeadsIn x[2], dy[2];  // queries, keys
  HeadsOut y[2];        // y, or dx
  const float* gain[2];
  const int32_t* pos;
  float* part;          // backward: [blocks][2][head_dim] sums of du * n
  int64_t tokens;
  double log2_theta;
  float eps, inv_dim;
  int period, heads[2], dim, rotary;
  int units, rot_units; // units (a lane's places) of a head, and how many of them rotate
  int ls;               // log2 of the lanes of a head
  int tb;               // tokens a block takes at a time
};

constexpr int QK_TRIG = 2048;  // pairs (cos, sin) of a block's tokens

template <typename T, int VEC> struct Vec;
template <> struct Vec<bf16_t, 8> {
  static __device__ __forceinline__ void load(const bf16_t* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
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
  static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <typename T> struct Vec<T, 1> {
  static __device__ __forceinline__ void load(const T* p, float (&v)[1]) { v[0] = load1(p); }
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

// One lane's share of a head: IT units of 2 x VEC values.
template <typename T, int VEC, int IT, bool INTER, bool BWD>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const QkArgs g) {
  __shared__ __attribute__((aligned(16))) float2 trig[QK_TRIG];
  __shared__ float red[BWD ? 4 * 256 : 1];
  const int tid = threadIdx.x, lane = tid & ((1 << g.ls) - 1), group = tid >> g.ls, groups = 256 >> g.ls;
  const int half = g.rotary / 2;

  // this lane's places in a head
  int pa[IT], pb[IT], pair[IT];
  bool on_a[IT], on_b[IT], rot[IT];
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
  }
  // this thread's share of the angles: one pair of every few tokens
  double turn = 0;
  const int tpass = half ? 256 / half : 1;  // tokens at a time (half <= 128)
  const int ti = half ? tid / half : 0, tp = half ? tid - ti * half : 0;
  if (half) turn = exp2(-(double)(2 * tp) / (double)g.rotary * g.log2_theta) * 0.15915494309189533577;

  float acc[2][BWD ? IT : 1][BWD ? 2 * VEC : 1];
  if (BWD) {
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) acc[w][BWD ? i : 0][BWD ? e : 0] = 0.f;
  }

  for (int64_t t0 = (int64_t)blockIdx.x * g.tb; t0 < g.tokens; t0 += (int64_t)gridDim.x * g.tb) {
    const int nt = (int)min((int64_t)g.tb, g.tokens - t0);
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
#pragma unroll
    for (int w = 0; w < 2; ++w) {  // queries, keys
      const int H = g.heads[w];
      float gain[IT][2 * VEC];
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          gain[i][e] = on_a[i] ? g.gain[w][pa[i] + e] : 0.f;
          gain[i][VEC + e] = on_b[i] ? g.gain[w][pb[i] + e] : 0.f;
        }
      int t = group / H, h = group - t * H;
      const int dt = groups / H, dh = groups - dt * H;
      while (t < nt) {
        const T* src = static_cast<const T*>(g.x[w].p) + (t0 + t) * g.x[w].ts + h * g.x[w].hs;
        float x[IT][2][VEC], d[BWD ? IT : 1][2][VEC];
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[i][0][e] = x[i][1][e] = 0.f;
          if (on_a[i]) Vec<T, VEC>::load(src + pa[i], x[i][0]);
          if (on_b[i]) Vec<T, VEC>::load(src + pb[i], x[i][1]);
        }
        if (BWD) {
          const T* dsrc = static_cast<const T*>(g.dy[w].p) + (t0 + t) * g.dy[w].ts + h * g.dy[w].hs;
#pragma unroll
          for (int i = 0; i < IT; ++i) {
            const int k = BWD ? i : 0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[k][0][e] = d[k][1][e] = 0.f;
            if (on_a[i]) Vec<T, VEC>::load(dsrc + pa[i], d[k][0]);
            if (on_b[i]) Vec<T, VEC>::load(dsrc + pb[i], d[k][1]);
          }
        }
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int e = 0; e < VEC; ++e) ss += x[i][0][e] * x[i][0][e] + x[i][1][e] * x[i][1][e];
        // the rotation of the pairs (u, v) in place, forwards or (BWD) backwards
        auto rotate = [&](int i, float (&a)[VEC], float (&b)[VEC]) __attribute__((always_inline)) {
          if (!rot[i]) return;
          const float2* cs = trig + t * half + pair[i];
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
            const int k = BWD ? i : 0;
            rotate(i, d[k][0], d[k][1]);
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int e = 0; e < VEC; ++e) dot += d[k][z][e] * gain[i][z * VEC + e] * x[i][z][e];
          }
          dot = head_sum(dot, g.ls);
        }
        ss = head_sum(ss, g.ls);
        const float r = rsqrtf(ss * g.inv_dim + g.eps);
        T* dst = static_cast<T*>(g.y[w].p) + (t0 + t) * g.y[w].ts + h * g.y[w].hs;
        if (BWD) {
          const float m = r * r * dot * g.inv_dim;  // r mean(h n) = r^2 mean(h x)
#pragma unroll
          for (int i = 0; i < IT; ++i) {
            const int k = BWD ? i : 0;
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int e = 0; e < VEC; ++e) {
                acc[w][k][BWD ? z * VEC + e : 0] += d[k][z][e] * (x[i][z][e] * r);
                x[i][z][e] = r * (d[k][z][e] * gain[i][z * VEC + e] - x[i][z][e] * m);
              }
          }
        } else {
#pragma unroll
          for (int i = 0; i < IT; ++i) {
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int e = 0; e < VEC; ++e) x[i][z][e] = x[i][z][e] * r * gain[i][z * VEC + e];
            rotate(i, x[i][0], x[i][1]);
          }
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          if (on_a[i]) Vec<T, VEC>::store(dst + pa[i], x[i][0]);
          if (on_b[i]) Vec<T, VEC>::store(dst + pb[i], x[i][1]);
        }
        t += dt;
        h += dh;
        if (h >= H) { h -= H; ++t; }
      }
    }
  }

  if (BWD) {  // sums of the gains' gradients: over the heads of a wavefront, then over the wavefronts, in a fixed order
    const int wave = tid >> 6;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) {
          float v = acc[w][BWD ? i : 0][BWD ? e : 0];
          for (int o = 1 << g.ls; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
          const int place = e < VEC ? pa[i] + e : pb[i] + e - VEC;
          if ((tid & 63) >> g.ls == 0 && (e < VEC ? on_a[i] : on_b[i])) red[wave * 256 + place] = v;
        }
      __syncthreads();
      if (tid < g.dim)
        g.part[((int64_t)blockIdx.x * 2 + w) * g.dim + tid] = red[tid] + red[256 + tid] + red[512 + tid] + red[768 + tid];
    }
  }
}

// dgain[i] (+)= sum over the blocks, in 64 bits: 16 columns a block, 16 rows of it at a time
__global__ __launch_bounds__(256) void qk_gain_sum_kernel(const float* __restrict__ part, int blocks, int dim, float* dq,
                                                          float* dk, int accumulate) {
  __shared__ double sh[16][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4;
  double s = 0;
  if (col < 2 * dim)
    for (int b = row; b < blocks; b += 16) s += part[(int64_t)b * 2 * dim + col];
  sh[row][threadIdx.x & 15] = s;
  __syncthreads();
  if (row == 0 && col < 2 * dim) {
    for (int r = 1; r < 16; ++r) s += sh[r][threadIdx.x];
    float* out = col < dim ? dq + col : dk + (col - dim);
    *out = (accumulate ? *out : 0.f) + (float)s;
  }
}

bool wide(const ast_heads& h, int vec_bytes, int esize) {
  return (reinterpret_cast<uintptr_t>(h.dev) % vec_bytes) == 0 && (h.token_stride * esize) % vec_bytes == 0 &&
         (h.head_stride * esize) % vec_bytes == 0;
}

constexpr int QK_MOST_BLOCKS = 1024;  // of a backward pass: partial sums of the gains' gradients

int backward_blocks(int64_t tokens) { return (int)std::min<int64_t>(std::max<int64_t>(tokens, 1), QK_MOST_BLOCKS); }

void launch(hipStream_t st, const ast_qk_cfg& c, const ast_heads* dy, const ast_heads* x, const float* gq, const float* gk,
            const ast_heads* y, float* part) {
  const bool bwd = dy != nullptr, bf = c.dtype == AST_BF16_F32ACC;
  QkArgs g = {};
  const int full = bf ? 8 : 4;
  bool vec = c.head_dim % full == 0 && (c.interleaved ? c.rotary % (2 * full) == 0 || c.rotary == c.head_dim : c.rotary / 2 % full == 0);
  for (int w = 0; w < 2; ++w) {
    g.x[w] = {x[w].dev, x[w].token_stride, x[w].head_stride};
    g.y[w] = {const_cast<void*>(y[w].dev), y[w].token_stride, y[w].head_stride};
    if (bwd) g.dy[w] = {dy[w].dev, dy[w].token_stride, dy[w].head_stride};
    g.heads[w] = x[w].heads;
    vec = vec && wide(x[w], 16, bf ? 2 : 4) && wide(y[w], 16, bf ? 2 : 4) && (!bwd || wide(dy[w], 16, bf ? 2 : 4));
  }
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
  const int V = vec ? full : 1;
  if (c.interleaved) {
    g.units = (c.head_dim + 2 * V - 1) / (2 * V);
    g.rot_units = (c.rotary + 2 * V - 1) / (2 * V);
  } else {
    g.rot_units = c.rotary / 2 / V;
    g.units = g.rot_units + ((c.head_dim - c.rotary) / V + 1) / 2;
  }
  while (g.ls < 6 && (1 << g.ls) < g.units) ++g.ls;
  g.tb = 1;
  const int most = std::min(16, c.rotary ? QK_TRIG / (c.rotary / 2) : 16);
  while (2 * g.tb <= most && (int64_t)g.tb * 2 * 1024 <= c.tokens) g.tb *= 2;
  const int64_t need = (c.tokens + g.tb - 1) / g.tb;
  const unsigned blocks = bwd ? (unsigned)backward_blocks(need) : (unsigned)std::min<int64_t>(need, 1 << 20);
#define GO(T, VEC, IT)                                                                                                        \
  do {                                                                                                                        \
    if (bwd) {                                                                                                                \
      if (c.interleaved) KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, true, true>), dim3(blocks), dim3(256), 0, st, g);           \
      else KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, false, true>), dim3(blocks), dim3(256), 0, st, g);                        \
    } else {                                                                                                                  \
      if (c.interleaved) KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, true, false>), dim3(blocks), dim3(256), 0, st, g);          \
      else KLAUNCH((qk_norm_rope_kernel<T, VEC, IT, false, false>), dim3(blocks), dim3(256), 0, st, g);                       \
    }                                                                                                                         \
  } while (0)
  if (bf) {
    if (vec) GO(bf16_t, 8, 1); else GO(bf16_t, 1, 2);
  } else {
    if (vec) GO(float, 4, 1); else GO(float, 1, 2);
  }
#undef GO
}

}  // namespace

void qk_norm_rope_fwd(hipStream_t st, const ast_qk_cfg& c, const ast_heads& q, const ast_heads& k, const float* gq,
                      const float* gk, const ast_heads& yq, const ast_heads& yk) {
  if (c.tokens <= 0) return;
  const ast_heads x[2] = {q, k}, y[2] = {yq, yk};
  launch(st, c, nullptr, x, gq, gk, y, nullptr);
}

size_t qk_norm_rope_bwd_ws_bytes(int64_t tokens, int head_dim) {
  return (size_t)backward_blocks(tokens) * 2 * head_dim * sizeof(float);
}

void qk_norm_rope_bwd(hipStream_t st, const ast_qk_cfg& c, const ast_heads& dyq, const ast_heads& dyk, const ast_heads& q,
                      const ast_heads& k, const float* gq, const float* gk, const ast_heads& dq, const ast_heads& dk,
                      float* dgq, float* dgk, bool accumulate, void* ws) {
  const ast_heads dy[2] = {dyq, dyk}, x[2] = {q, k}, y[2] = {dq, dk};
  float* part = static_cast<float*>(ws);
  int blocks = 0;
  if (c.tokens > 0) {
    launch(st, c, dy, x, gq, gk, y, part);
    int tb = 1;
    const int most = std::min(16, c.rotary ? QK_TRIG / (c.rotary / 2) : 16);
    while (2 * tb <= most && (int64_t)tb * 2 * 1024 <= c.tokens) tb *= 2;
    blocks = backward_blocks((c.tokens + tb - 1) / tb);
  }
  KLAUNCH(qk_gain_sum_kernel, dim3((unsigned)((2 * c.head_dim + 15) / 16)), dim3(256), 0, st, part, blocks, c.head_dim, dgq, dgk,
          (int)accumulate);
}

}  // namespace ast
