// Weight and bias gradient of a dense layer whose input was kept in 8 bits:
//   dW[n][c] = sum_t dy[t][n] * x'[t][c],   db[n] = sum_t dy[t][n]
// on the bf16 matrix cores (a restored value is exact in bf16, so its product with dy is exact and only the fp32 sum rounds).
// The contraction index is the row of both operands: the tiles lie in LDS as [row][channel] and the operands are read with the
// transposing LDS read (four rows of 16 channels -> lane i gets the four rows of channel i).  Kept values are restored on
// their way into LDS: every one of them once per block.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

constexpr int SW_BN = 128, SW_BC = 128, SW_BK = 32;  // outputs, inputs, rows of a block's step

typedef short sw_short4 __attribute__((ext_vector_type(4)));
typedef short sw_short8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) sw_short4 sw_lds_short4;

struct SwArgs {
  const bf16_t* dy;
  const uint8_t* q;
  const uint8_t* sc;
  float* out;       // dW, or partials [splits][N][C]
  float* bias_out;  // db, or partials [splits][N]; NULL: not wanted
  int64_t rows, rows_per_split;
  int N, C, pitch, tiles_n, tiles_c;
  int add;          // out and bias_out are added to (one split only)
};

// [row][128 channels] bf16 tile, 16-byte chunks swizzled so that the four rows of a transposed read lie in different banks
__device__ __forceinline__ int sw_off(int row, int chunk) { return row * 256 + ((chunk ^ ((row & 3) << 2)) << 4); }

__device__ __forceinline__ bf16x8 sw_frag(const unsigned char* tile, int off) {
  const sw_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sw_lds_short4*)(tile + off));
  const sw_short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sw_lds_short4*)(tile + off + 4 * 256));
  const sw_short8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

__global__ __launch_bounds__(256) void stash8_wgrad_kernel(const SwArgs g) {
  __shared__ __attribute__((aligned(16))) unsigned char sa[SW_BK * 256], sb[SW_BK * 256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  int bid = blockIdx.x;
  const int tc = bid % g.tiles_c; bid /= g.tiles_c;
  const int tn = bid % g.tiles_n;
  const int split = bid / g.tiles_n;
  const int n0 = tn * SW_BN, c0 = tc * SW_BC;
  const int64_t r_begin = split * g.rows_per_split, r_end = min(r_begin + g.rows_per_split, g.rows);

  floatx16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const bool bias = g.bias_out && tc == 0;
  float bsum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bsum[e] = 0.f;

  // this thread copies chunk `ch` (8 channels) of rows r0 and r0 + 16
  const int ch = tid & 15, r0 = tid >> 4;
  const int n = n0 + ch * 8, c = c0 + ch * 8;
  const int j16 = lane & 15, blk = lane >> 4;
  const int krow = 8 * (blk >> 1) + (j16 >> 2);
  int ao[2], bo[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ca = wm * 64 + i * 32 + 16 * (blk & 1) + 4 * (j16 & 3), cb = wn * 64 + i * 32 + 16 * (blk & 1) + 4 * (j16 & 3);
    ao[i] = sw_off(krow, ca >> 3) + (ca & 7) * 2;
    bo[i] = sw_off(krow, cb >> 3) + (cb & 7) * 2;
  }

  for (int64_t r = r_begin; r < r_end; r += SW_BK) {
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int rr = r0 + 16 * p;
      const int64_t row = r + rr;
      float v[8], w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = w[e] = 0.f;
      if (row < r_end) {
        if (n + 8 <= g.N) load8(g.dy + row * g.N + n, v);
        else if (n < g.N) load8_part(g.dy + row * g.N + n, g.N - n, v);
        if (c < g.pitch) {
          const uint2 q = *reinterpret_cast<const uint2*>(g.q + row * g.pitch + c);
          const float s = __uint_as_float((uint32_t)g.sc[row * (g.pitch / kStash8Block) + c / kStash8Block] << 23);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = (float)(int)(int8_t)(q.x >> (8 * e)) * s;
            w[4 + e] = (float)(int)(int8_t)(q.y >> (8 * e)) * s;
          }
        }
      }
      if (bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bsum[e] += v[e];
      }
      *reinterpret_cast<uint4*>(sa + sw_off(rr, ch)) = make_uint4(f2bf_pk(v[0], v[1]), f2bf_pk(v[2], v[3]), f2bf_pk(v[4], v[5]), f2bf_pk(v[6], v[7]));
      *reinterpret_cast<uint4*>(sb + sw_off(rr, ch)) = make_uint4(f2bf_pk(w[0], w[1]), f2bf_pk(w[2], w[3]), f2bf_pk(w[4], w[5]), f2bf_pk(w[6], w[7]));
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = sw_frag(sa, ao[i] + ks * 16 * 256);
        fb[i] = sw_frag(sb, bo[i] + ks * 16 * 256);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
  }

  if (bias) {  // 16 groups of rows, added in order
    float* const sum = reinterpret_cast<float*>(sa);  // [16][128]
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[r0 * 128 + ch * 8 + e] = bsum[e];
    __syncthreads();
    if (tid < SW_BN && n0 + tid < g.N) {
      float t = 0.f;
      for (int k = 0; k < 16; ++k) t += sum[k * 128 + tid];
      float* out = g.bias_out + (int64_t)split * g.N + n0 + tid;
      *out = (g.add ? *out : 0.f) + t;
    }
  }
  // accumulator register r of lane l: row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32
  float* out = g.out + (int64_t)split * g.N * g.C;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int cc = c0 + wn * 64 + j * 32 + (lane & 31);
      if (cc >= g.C) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int nn = n0 + wm * 64 + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
        if (nn >= g.N) continue;
        float* p = out + (int64_t)nn * g.C + cc;
        *p = (g.add ? *p : 0.f) + acc[i][j][r];
      }
    }
}

// out (+)= sum over the splits, in their order, in 64 bits; the same for the bias
__global__ __launch_bounds__(256) void stash8_wgrad_sum_kernel(const float* __restrict__ part, int64_t n, float* out,
                                                               const float* __restrict__ bias_part, int nb, float* bias_out,
                                                               int splits, int add) {
  const int64_t total = n + (bias_out ? nb : 0);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const bool b = i >= n;
    const float* p = b ? bias_part + (i - n) : part + i;
    const int64_t stride = b ? nb : n;
    double s = 0;
    for (int k = 0; k < splits; ++k) s += p[k * stride];
    float* o = b ? bias_out + (i - n) : out + i;
    *o = (add ? *o : 0.f) + (float)s;
  }
}

// shares of the rows: enough blocks for the chip, none of fewer than 256 rows
int wgrad_splits(int64_t rows, int64_t in, int64_t out) {
  const int64_t tiles = ((out + SW_BN - 1) / SW_BN) * ((in + SW_BC - 1) / SW_BC);
  return (int)std::max<int64_t>(1, std::min<int64_t>({(512 + tiles - 1) / tiles, (rows + 255) / 256, 64}));
}

}  // namespace

size_t linear_wgrad_stash8_ws_bytes(int64_t rows, int64_t in, int64_t out) {
  const int s = wgrad_splits(rows, in, out);
  return s > 1 ? (size_t)s * (size_t)(out * in + out) * sizeof(float) : 0;
}

void linear_wgrad_stash8(hipStream_t st, const void* dy, const void* stash, int64_t rows, int64_t in, int64_t out, float* dw,
                         float* db, bool accumulate, void* ws) {
  const int splits = wgrad_splits(rows, in, out);
  SwArgs g = {};
  g.dy = static_cast<const bf16_t*>(dy);
  g.q = static_cast<const uint8_t*>(stash);
  g.sc = stash8_scales(stash, rows, in);
  g.rows = rows;
  g.rows_per_split = ((rows + splits - 1) / splits + SW_BK - 1) / SW_BK * SW_BK;
  g.N = (int)out;
  g.C = (int)in;
  g.pitch = (int)stash8_pitch(in);
  g.tiles_n = (int)((out + SW_BN - 1) / SW_BN);
  g.tiles_c = (int)((in + SW_BC - 1) / SW_BC);
  float* part = static_cast<float*>(ws);
  float* bias_part = part + (size_t)splits * out * in;
  g.out = splits > 1 ? part : dw;
  g.bias_out = !db ? nullptr : splits > 1 ? bias_part : db;
  g.add = splits == 1 && accumulate;
  KLAUNCH(stash8_wgrad_kernel, dim3((unsigned)(g.tiles_n * g.tiles_c * splits)), dim3(256), 0, st, g);
  if (splits > 1) {
    const int64_t n = out * in;
    KLAUNCH(stash8_wgrad_sum_kernel, dim3((unsigned)std::min<int64_t>((n + out + 255) / 256, 1 << 16)), dim3(256), 0, st, part, n, dw,
            bias_part, (int)out, db, splits, (int)accumulate);
  }
}

}  // namespace ast
