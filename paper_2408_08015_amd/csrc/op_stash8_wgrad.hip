// Weight and bias gradient of a dense layer whose input was kept in 8 bits:
//   dW[n][c] = sum_t dy[t][n] * x'[t][c],   db[n] = sum_t dy[t][n]
// on the bf16 matrix cores (a restored value is exact in bf16, so its product with dy is exact and only the fp32 sum rounds).
// The contraction index is the row of both operands: the tiles lie in LDS as [row][channel] and the operands are read with the
// transposing LDS read (four rows of 16 channels -> lane i gets the four rows of channel i).
//
// A block computes a tile of 32 TM WM outputs x 32 TN WN inputs over a range of rows, 64 at a time, with two LDS stages.  The
// next stage is filled while this one is multiplied, a quarter (16 rows) behind each of its four 16-row steps: 16 bytes of dy
// and 8 kept values a thread, requested one stage earlier and restored on the way into LDS, each once per block (a conversion, a
// multiplication, half a byte permutation).  The operands of a step are read while the step in front of it is multiplied.
//
// 16384 rows, 4096 -> 4096: 470 to 490 us, 1120 to 1170 TFLOP/s; the matrix cores are busy 63 % of the cycles, at a clock that they
// pull down (a library's product of the same shape in bf16 takes 460 to 540).  4096 rows, 2048 -> 512: 22 us in four shares and 5.6 for
// their sum; a step of 64 rows takes 0.75 us where its matrix instructions are 0.25: one wavefront to a vector unit waits for its
// own LDS reads, conversions and products in turn (two groups of wavefronts in a block, each with half of the rows, were
// no faster, nor were loads two or three stages ahead).  What a short launch runs once counts too: with the epilogue as branches
// instead of stores to offsets behind the buffer, 64 rows took 13 us instead of 5.8.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

constexpr int SW_BK = 64;  // rows of a stage
constexpr unsigned SW_OOB = 0x80000000u;  // an offset behind every buffer: zeros, and no memory access

typedef short sw_short4 __attribute__((ext_vector_type(4)));
typedef short sw_short8 __attribute__((ext_vector_type(8)));
typedef unsigned int sw_u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int sw_u32x4 __attribute__((ext_vector_type(4)));
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

__device__ __forceinline__ __amdgpu_buffer_rsrc_t sw_rsrc(const void* p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

// [row][CH channels] bf16 tile, 16-byte chunks swizzled so that the four rows of a transposed read lie in different banks
template <int CH>
__device__ __forceinline__ int sw_off(int row, int chunk) { return row * (CH * 2) + ((chunk ^ ((row & 3) << 2)) << 4); }

template <int CH>
__device__ __forceinline__ bf16x8 sw_frag(const unsigned char* tile, int off) {
  const sw_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sw_lds_short4*)(tile + off));
  const sw_short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sw_lds_short4*)(tile + off + 4 * CH * 2));
  const sw_short8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

// four kept values (the bytes of w) restored: bf16 pairs (exact, so the upper halves of the fp32 values)
__device__ __forceinline__ void sw_restore4(uint32_t w, float s, uint32_t& lo, uint32_t& hi) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)(int)(int8_t)(w >> (8 * i)) * s;
  lo = __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x07060302u);
  hi = __builtin_amdgcn_perm(__float_as_uint(v[3]), __float_as_uint(v[2]), 0x07060302u);
}

// EVEN: rows of dy start at 16-byte addresses
template <int WM, int WN, int TM, int TN, bool EVEN>
__device__ __forceinline__ void stash8_wgrad_body(const SwArgs& g, int bid) {  // bid: block of this product
  constexpr int BN = 32 * TM * WM, BC = 32 * TN * WN, NT = 64 * WM * WN;
  static_assert(16 * BN / 8 == NT && 16 * BC / 8 == NT, "a thread fills one chunk of each operand per quarter");
  constexpr int A_BYTES = SW_BK * BN * 2, STAGE = A_BYTES + SW_BK * BC * 2;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / WN, wn = wave % WN;
  const int tc = bid % g.tiles_c; bid /= g.tiles_c;
  const int tn = bid % g.tiles_n;
  const int split = bid / g.tiles_n;
  const int n0 = tn * BN, c0 = tc * BC;
  const int64_t r_begin = split * g.rows_per_split, r_end = min(r_begin + g.rows_per_split, g.rows);
  const int nk = (int)((r_end - r_begin + SW_BK - 1) / SW_BK);

  floatx16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const bool bias = g.bias_out && tc == 0;
  float bsum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bsum[e] = 0.f;

  // ---- what this thread copies: one chunk of eight channels of each operand, of row `trow` of every quarter
  const int chunk = tid % (BN / 8), trow = tid / (BN / 8);
  const int n = n0 + chunk * 8, c = c0 + chunk * 8;
  const int sp = g.pitch / kStash8Block;
  unsigned a_voff[4], q_voff[4], s_voff[4];
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    a_voff[h] = n < g.N ? (unsigned)((16 * h + trow) * g.N + n) * 2u : SW_OOB;
    q_voff[h] = c < g.pitch ? (unsigned)((16 * h + trow) * g.pitch + c) : SW_OOB;
    s_voff[h] = c < g.pitch ? (unsigned)((16 * h + trow) * sp + c / kStash8Block) : SW_OOB;
  }
  // A last chunk that would reach behind its row is read from `over` values further in front, and shifted when it is used.
  const int over = !EVEN && g.N >= 8 && n < g.N ? max(n + 8 - g.N, 0) : 0;
  const bool ragged = !EVEN && g.N >= 8 && n0 + BN > g.N;
  uint32_t ra[4][4], rq[4][2], rs[4];
  // Rows behind the range come back as zeros (the buffers end with it).  Kept values behind a row's are the next row's: they belong
  // to inputs that do not exist, and are never written.
  struct Stage { const bf16_t* dy; __amdgpu_buffer_rsrc_t a, q, s; unsigned left; };
  auto stage_of = [&](int kt) __attribute__((always_inline)) {
    const int64_t r = r_begin + (int64_t)kt * SW_BK;
    const unsigned left = (unsigned)max((int64_t)0, min((int64_t)SW_BK, r_end - r));
    return Stage{g.dy + r * g.N, sw_rsrc(g.dy + r * g.N, left * (unsigned)g.N * 2u), sw_rsrc(g.q + r * g.pitch, left * (unsigned)g.pitch),
                 sw_rsrc(g.sc + r * sp, left * (unsigned)sp), left};
  };
  auto request = [&](const Stage& t, int h) __attribute__((always_inline)) {
    if (EVEN) {
      const sw_u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(t.a, a_voff[h], 0, 0);
      ra[h][0] = v.x; ra[h][1] = v.y; ra[h][2] = v.z; ra[h][3] = v.w;
    } else {
      ra[h][0] = ra[h][1] = ra[h][2] = ra[h][3] = 0;
      if (n < g.N && (unsigned)(16 * h + trow) < t.left) {
        const bf16_t* src = t.dy + (unsigned)((16 * h + trow) * g.N + n);
        if (g.N >= 8) {
          const Raw16 v = *reinterpret_cast<const Raw16*>(src - over);
#pragma unroll
          for (int e = 0; e < 4; ++e) ra[h][e] = v.w[e];
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (e < g.N) ra[h][e / 2] |= (uint32_t)src[e] << (16 * (e & 1));
        }
      }
    }
    const sw_u32x2 q = __builtin_amdgcn_raw_buffer_load_b64(t.q, q_voff[h], 0, 0);
    rq[h][0] = q.x; rq[h][1] = q.y;
    rs[h] = __builtin_amdgcn_raw_buffer_load_b8(t.s, s_voff[h], 0, 0);
  };
  const int w_off = sw_off<BN>(trow, chunk), w_off_c = A_BYTES + sw_off<BC>(trow, chunk);
  auto fill = [&](int h, int stage) __attribute__((always_inline)) {
    if (ragged) {
      uint64_t lo = ra[h][0] | (uint64_t)ra[h][1] << 32, hi = ra[h][2] | (uint64_t)ra[h][3] << 32;
      const int by = 16 * (over & 3);
      if (over >= 4) lo = hi, hi = 0;
      lo = by ? lo >> by | hi << (64 - by) : lo;
      hi >>= by;
      ra[h][0] = (uint32_t)lo; ra[h][1] = (uint32_t)(lo >> 32); ra[h][2] = (uint32_t)hi; ra[h][3] = (uint32_t)(hi >> 32);
    }
    if (bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bsum[2 * e] += __uint_as_float(ra[h][e] << 16);
        bsum[2 * e + 1] += __uint_as_float(ra[h][e] & 0xffff0000u);
      }
    }
    *reinterpret_cast<uint4*>(smem + stage + w_off + h * 16 * BN * 2) = make_uint4(ra[h][0], ra[h][1], ra[h][2], ra[h][3]);
    const float s = __uint_as_float(rs[h] << 23);
    uint4 v;
    sw_restore4(rq[h][0], s, v.x, v.y);
    sw_restore4(rq[h][1], s, v.z, v.w);
    *reinterpret_cast<uint4*>(smem + stage + w_off_c + h * 16 * BC * 2) = v;
  };

  // ---- operand fragments: lane l of a transposed read gives the address of four channels of one row
  const int j16 = lane & 15, blk = lane >> 4;
  const int krow = 8 * (blk >> 1) + (j16 >> 2);
  int ao[TM], bo[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int ch = wm * (32 * TM) + i * 32 + 16 * (blk & 1) + 4 * (j16 & 3);
    ao[i] = sw_off<BN>(krow, ch >> 3) + (ch & 7) * 2;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int ch = wn * (32 * TN) + j * 32 + 16 * (blk & 1) + 4 * (j16 & 3);
    bo[j] = A_BYTES + sw_off<BC>(krow, ch >> 3) + (ch & 7) * 2;
  }
  bf16x8 fa[2][TM], fb[2][TN];  // of two steps: the next one's are read while this one's are multiplied
  auto read = [&](int stage, int ks) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[ks & 1][i] = sw_frag<BN>(smem, stage + ao[i] + ks * 16 * BN * 2);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[ks & 1][j] = sw_frag<BC>(smem, stage + bo[j] + ks * 16 * BC * 2);
  };
  // every LDS access of the wavefront has been made; loads from memory stay in flight (__syncthreads() would wait for them)
  // (the empty statements keep the compiler from moving accesses across the wait or the barrier, which it knows of neither)
  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  {
    const Stage t0 = stage_of(0), t1 = stage_of(1);
#pragma unroll
    for (int h = 0; h < 4; ++h) request(t0, h);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      fill(h, 0);
      request(t1, h);
    }
  }
  barrier();
  read(0, 0);
  for (int kt = 0; kt < nk; ++kt) {
    const int cur = (kt & 1) * STAGE, nxt = STAGE - cur;
    const Stage t2 = stage_of(kt + 2);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      if (ks < 3) read(cur, ks + 1);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[ks & 1][i], fb[ks & 1][j], acc[i][j], 0, 0, 0);
      fill(ks, nxt);
      request(t2, ks);
    }
    barrier();
    read(nxt, 0);  // (behind the last stage: zeros that nothing is made of)
  }

  if (bias) {  // 16 groups of rows, added in order
    barrier();
    float* const sum = reinterpret_cast<float*>(smem);  // [16][BN]
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[trow * BN + chunk * 8 + e] = bsum[e];
    __syncthreads();
    if (tid < BN && n0 + tid < g.N) {
      float t = 0.f;
      for (int k = 0; k < 16; ++k) t += sum[k * BN + tid];
      float* out = g.bias_out + (int64_t)split * g.N + n0 + tid;
      *out = (g.add ? *out : 0.f) + t;
    }
  }
  // Accumulator register r of lane l: row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32.  What lies outside the matrix goes to
  // an offset behind the buffer, where a store is dropped.
  const unsigned rows_here = (unsigned)min(BN, g.N - n0);
  float* const tile = g.out + ((int64_t)split * g.N + n0) * g.C;
  const __amdgpu_buffer_rsrc_t ro = sw_rsrc(tile, rows_here * (unsigned)g.C * 4u);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int cc = c0 + wn * (32 * TN) + j * 32 + (lane & 31);
      const unsigned row = wm * (32 * TM) + i * 32 + 4 * (lane >> 5);
      const unsigned at = cc < g.C ? (row * (unsigned)g.C + (unsigned)cc) * 4u : SW_OOB;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const unsigned off = at + (unsigned)(8 * (r >> 2) + (r & 3)) * (unsigned)g.C * 4u;
        float v = acc[i][j][r];
        if (g.add) v += __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ro, off, 0, 0));
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), ro, off, 0, 0);
      }
    }
}

template <int WM, int WN, int TM, int TN, bool EVEN>
__global__ __launch_bounds__(64 * WM * WN, 2) void stash8_wgrad_kernel(const SwArgs g) {
  // neighbouring tiles on one XCD: they share their rows of dy, or the kept values, in its L2
  stash8_wgrad_body<WM, WN, TM, TN, EVEN>(g, (int)xcd_grouped(blockIdx.x, gridDim.x));
}

// Several products in one launch, none in shares: blocks holds (product, block of it).
__global__ __launch_bounds__(256, 2) void stash8_wgrad_group_kernel(const SwArgs* __restrict__ tasks, const uint2* __restrict__ blocks) {
  const uint2 b = blocks[xcd_grouped(blockIdx.x, gridDim.x)];
  const SwArgs g = tasks[__builtin_amdgcn_readfirstlane(b.x)];
  stash8_wgrad_body<2, 2, 2, 2, true>(g, (int)__builtin_amdgcn_readfirstlane(b.y));
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

// Tile and shares of the rows: the cheapest by a model in us of what was measured - 64 rows of a 256 x 256 tile take 1.85, of a
// 128 x 128 tile 0.85 (one block a compute unit), a launch's ends 8 and 6, and shares write and read partials of 4 bytes
// (6 TB/s) and cost a second launch, 5.  2048 -> 512 of 4096 rows in small tiles and 4 shares 28 us, in big ones 42 by the model;
// 4096 -> 4096 of 16384 rows in big tiles 472 us, in small ones 870.  A round pays its rows by the part of a stage, and nearly a
// stage more for its first loads: by whole stages alone the model takes 22 shares instead of 15 for 5465 rows of 1408 -> 128, 22.0
// us instead of 19.4, and the small tiles for 64 rows of 4096 -> 4096, 15.8 instead of 15.5.  Then shares that have no rows are left
// out (4097 rows of 40 -> 300: 32 shares of 192 rows 18.1 us, the 22 that have any 15.7).
struct WgradShape { bool big; int64_t tiles_n, tiles_c; int splits; int64_t rows_per_split; };
WgradShape wgrad_shape(int64_t rows, int64_t in, int64_t out, int most) {
  WgradShape best = {};
  double least = 0;
  for (const bool big : {false, true}) {
    const int b = big ? 256 : 128;
    const int64_t tn = (out + b - 1) / b, tc = (in + b - 1) / b;
    for (const int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (s > most || (s > 1 && rows < (int64_t)s * 128)) break;
      const double steps = (double)((rows + s - 1) / s + SW_BK - 1) / SW_BK, rounds = (double)((tn * tc * s + 255) / 256);
      double us = rounds * steps * (big ? 1.85 : 0.85) + (big ? 8 : 6);
      if (s > 1) us += 5 + (double)s * (double)in * (double)out * 8 / 6e6;
      if (!best.splits || us < least) {
        least = us;
        best = {big, tn, tc, s, 0};
      }
    }
  }
  // whole stages of 64 rows a share, and as many shares as then have any
  best.rows_per_split = std::max<int64_t>(((rows + best.splits - 1) / best.splits + SW_BK - 1) / SW_BK, 1) * SW_BK;
  best.splits = (int)std::max<int64_t>((rows + best.rows_per_split - 1) / best.rows_per_split, 1);
  return best;
}

template <int WM, int WN, int TM, int TN>
void launch(hipStream_t st, const SwArgs& g, unsigned blocks, bool even) {
  constexpr int lds = 2 * SW_BK * 2 * (32 * TM * WM + 32 * TN * WN);
  auto go = [&](auto kernel) {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    KLAUNCH_NAMED("stash8_wgrad_kernel", kernel, dim3(blocks), dim3(64 * WM * WN), lds, st, g);
  };
  if (even) go(stash8_wgrad_kernel<WM, WN, TM, TN, true>);
  else go(stash8_wgrad_kernel<WM, WN, TM, TN, false>);
}

}  // namespace

size_t stash8_group_task_bytes() { return sizeof(SwArgs); }

int stash8_group_blocks(int64_t in, int64_t out) { return (int)(((out + 127) / 128) * ((in + 127) / 128)); }

void stash8_group_task(void* task, const void* dy, const void* stash, int64_t rows, int64_t in, int64_t out, float* dw, float* db) {
  SwArgs g = {};
  g.dy = static_cast<const bf16_t*>(dy);
  g.q = static_cast<const uint8_t*>(stash);
  g.sc = stash8_scales(stash, rows, in);
  g.out = dw;
  g.bias_out = db;
  g.rows = rows;
  g.rows_per_split = (rows + SW_BK - 1) / SW_BK * SW_BK;
  g.N = (int)out;
  g.C = (int)in;
  g.pitch = (int)stash8_pitch(in);
  g.tiles_n = (int)((out + 127) / 128);
  g.tiles_c = (int)((in + 127) / 128);
  g.add = 1;
  *static_cast<SwArgs*>(task) = g;
}

void linear_wgrad_stash8_group(hipStream_t st, const void* tasks_dev, const void* blocks_dev, int blocks) {
  constexpr int lds = 2 * SW_BK * 2 * (128 + 128);
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(stash8_wgrad_group_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  KLAUNCH(stash8_wgrad_group_kernel, dim3((unsigned)blocks), dim3(256), lds, st, static_cast<const SwArgs*>(tasks_dev),
          static_cast<const uint2*>(blocks_dev));
}

size_t linear_wgrad_stash8_ws_bytes(int64_t rows, int64_t in, int64_t out, int most) {
  const int s = wgrad_shape(rows, in, out, most).splits;
  return s > 1 ? (size_t)s * (size_t)(out * in + out) * sizeof(float) : 0;
}

void linear_wgrad_stash8(hipStream_t st, const void* dy, const void* stash, int64_t rows, int64_t in, int64_t out, float* dw,
                         float* db, bool accumulate, void* ws, int most) {
  const WgradShape s = wgrad_shape(rows, in, out, most);
  const int splits = s.splits;
  SwArgs g = {};
  g.dy = static_cast<const bf16_t*>(dy);
  g.q = static_cast<const uint8_t*>(stash);
  g.sc = stash8_scales(stash, rows, in);
  g.rows = rows;
  g.rows_per_split = s.rows_per_split;
  g.N = (int)out;
  g.C = (int)in;
  g.pitch = (int)stash8_pitch(in);
  g.tiles_n = (int)s.tiles_n;
  g.tiles_c = (int)s.tiles_c;
  float* part = static_cast<float*>(ws);
  float* bias_part = part + (size_t)splits * out * in;
  g.out = splits > 1 ? part : dw;
  g.bias_out = !db ? nullptr : splits > 1 ? bias_part : db;
  g.add = splits == 1 && accumulate;
  const bool even = out % 8 == 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0;
  const unsigned blocks = (unsigned)(g.tiles_n * g.tiles_c * splits);
  if (s.big) launch<4, 2, 2, 4>(st, g, blocks, even);
  else launch<2, 2, 2, 2>(st, g, blocks, even);
  if (splits > 1) {
    const int64_t n = out * in;
    KLAUNCH(stash8_wgrad_sum_kernel, dim3((unsigned)std::min<int64_t>((n + out + 255) / 256, 1 << 16)), dim3(256), 0, st, part, n, dw,
            bias_part, (int)out, db, splits, (int)accumulate);
  }
}

}  // namespace ast

// The choice of wgrad_shape, for tests: the tile's edge, shares of the rows.
extern "C" void ast_stash8_wgrad_choice(int64_t rows, int64_t in, int64_t out, int choice[2]) {
  const ast::WgradShape s = ast::wgrad_shape(rows, in, out, INT_MAX);
  choice[0] = s.big ? 256 : 128;
  choice[1] = s.splits;
}
