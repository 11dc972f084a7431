// Token embedding: y[t] = scale * W[ids[t]] and its gradient dW[v] = scale * sum of dy[t] over the tokens t of id v.
//
// Both move bytes and compute next to nothing.  The gradient orders the tokens by id first (stably, ids outside the table
// last), so that the tokens of a row lie next to each other and are added in their order: no atomics on values, equal calls
// give equal bits.  A wavefront takes a fixed number of sorted tokens, so an id that fills half of the micro-batch costs no
// more than many different ones; what crosses the shares is joined by a second launch.
// Measured: lookup of 65521 rows of 1024 bf16 values 46 us (3.6 TB/s of what has to move), of 1021 56 to 61; gradient of 4096
// tokens of 512 into 32768 rows 21 us (67 MB of zeros alone take 10), of 65536 of 1024 into 131072 rows 183 us (537 MB of zeros 78
// to 95, the sums 76).
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"
#include "prof.h"

namespace ast {

namespace {

// Forward: bound by its bytes, so the output is taken as one run of values, eight of a thread at 16-byte addresses whatever the
// row length, U times a thread with all ids, then all rows requested before the first is used.  A group of eight that goes on
// in the next row takes the last eight values of its row and the first eight of the next one.  (width >= 8)
template <typename TW, typename TY, int U, bool EVEN>  // EVEN: rows of the table start at 16-byte addresses
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const int32_t* __restrict__ ids, int64_t tokens,
                                                            const TW* __restrict__ table, uint32_t rows, int width,
                                                            float inv_width, float scale, TY* __restrict__ y) {
  constexpr int SPAN = 256 * 8 * U;  // values of a block
  const int64_t total = tokens * width;
  for (int64_t base = (int64_t)blockIdx.x * SPAN; base < total; base += (int64_t)gridDim.x * SPAN) {
    // (base < 2^51: exact, but for the last bit of the quotient)
    int64_t t0 = (int64_t)((double)base / (double)width);
    int64_t in_row = base - t0 * width;
    if (in_row < 0) --t0, in_row += width;
    if (in_row >= width) ++t0, in_row -= width;
    int c[U], over[U];  // place in the row, and values that lie in the next one
    uint32_t k0[U], k1[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int off = (int)in_row + (u * 256 + (int)threadIdx.x) * 8;  // (< 2^21)
      int q = (int)((float)off * inv_width), r = off - q * width;
      if (r < 0) --q, r += width;
      if (r >= width) ++q, r -= width;
      over[u] = max(r + 8 - width, 0);
      c[u] = r - over[u];
      k0[u] = (uint32_t)ids[min(t0 + q, tokens - 1)];
      k1[u] = (uint32_t)ids[min(t0 + q + 1, tokens - 1)];
    }
    Eight<TW, EVEN> a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      a[u].load(table + (size_t)(k0[u] < rows ? k0[u] : 0) * width + c[u]);
      b[u] = a[u];
      if (over[u]) b[u].load(table + (size_t)(k1[u] < rows ? k1[u] : 0) * width);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      constexpr int W = Eight<TW, EVEN>::W;
      uint32_t w[W];
      a[u].words(w);
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = k0[u] < rows ? w[i] : 0;
      if (__any(over[u])) {
        uint32_t x[W];
        b[u].words(x);
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = k1[u] < rows ? x[i] : 0;
        funnel<W>(w, x, (uint32_t)over[u] * (uint32_t)sizeof(TW));
      }
      float v[8];
      eight_values<TW>(w, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= scale;
      const int64_t f = base + (u * 256 + (int)threadIdx.x) * 8;
      if (f + 8 <= total) store8(y + f, v);
      else if (f < total) store8_part(y + f, (int)(total - f), v);
    }
  }
}

// ... and rows of fewer than eight values: one value a thread
template <typename TW, typename TY>
__global__ __launch_bounds__(256) void embedding_fwd_narrow_kernel(const int32_t* __restrict__ ids, int64_t tokens,
                                                                   const TW* __restrict__ table, uint32_t rows, int width,
                                                                   float scale, TY* __restrict__ y) {
  const int64_t total = tokens * width;
  for (int64_t f = (int64_t)blockIdx.x * 256 + threadIdx.x; f < total; f += (int64_t)gridDim.x * 256) {
    const int64_t t = f / width;
    const uint32_t k = (uint32_t)ids[t];
    store1(y + f, k < rows ? load1(table + (size_t)k * width + (f - t * width)) * scale : 0.f);
  }
}

// ids outside the table sort behind every row
__device__ __forceinline__ uint32_t sort_key(int32_t id, uint32_t rows) { return min((uint32_t)id, rows); }

// The gradient of a large table is mostly zeros, and writing them takes longer than the sort: they are written by blocks of
// their own beside the blocks of the sort's launches, a share with each.
struct ZeroShare {
  float* p;         // 16-byte aligned
  size_t n4;        // groups of four
  float* edge[2];   // what is left in front of and behind the aligned part: single values
  int edges[2];
};

__device__ __forceinline__ void zero_share(const ZeroShare& z, unsigned block, unsigned blocks) {
  float4* const p = reinterpret_cast<float4*>(z.p);
  for (size_t i = (size_t)block * blockDim.x + threadIdx.x; i < z.n4; i += (size_t)blocks * blockDim.x)
    p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (block == 0)
    for (int e = 0; e < 2; ++e)
      if ((int)threadIdx.x < z.edges[e]) z.edge[e][threadIdx.x] = 0.f;
}

// Order of few tokens: the place of a token is the number of tokens in front of it, counted.  A block places 64 tokens; each
// of its 16 wavefronts counts over its share of all tokens, 64 of them in a register of the wavefront, handed out one by one
// to all lanes (three vector instructions a comparison, and no memory access among them).
constexpr int RANK_WAVES = 16;
__global__ __launch_bounds__(64 * RANK_WAVES) void embedding_rank_kernel(const int32_t* __restrict__ ids, int tokens,
                                                                         uint32_t rows, uint32_t* __restrict__ key,
                                                                         uint32_t* __restrict__ order, unsigned sort_blocks,
                                                                         ZeroShare z) {
  if (blockIdx.x >= sort_blocks) {
    zero_share(z, blockIdx.x - sort_blocks, gridDim.x - sort_blocks);
    return;
  }
  __shared__ uint32_t part[RANK_WAVES][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * 64, t = t0 + lane;
  // shares of whole groups of 64, so that one of them is exactly the block's own tokens
  const int groups = (tokens + 63) / 64, per = (groups + RANK_WAVES - 1) / RANK_WAVES;
  const int g0 = wave * per, g1 = min(g0 + per, groups);
  // (behind the last token: a key that is in front of no token)
  auto load = [&](int g) { const int u = g * 64 + lane; return g < g1 && u < tokens ? sort_key(ids[u], rows) : 0xffffffffu; };
  uint32_t cur = load(g0), next = load(g0 + 1);
  const uint32_t mine = t < tokens ? sort_key(ids[t], rows) : 0;
  uint32_t rank = 0;
  for (int g = g0; g < g1; ++g) {
    const uint32_t after = load(g + 2);
    if (g * 64 == t0) {
#pragma unroll
      for (int i = 0; i < 64; ++i) rank += (uint32_t)__builtin_amdgcn_readlane(cur, i) < mine + (i < lane ? 1u : 0u);
    } else {
      const uint32_t limit = mine + (g * 64 < t0 ? 1 : 0);  // an equal id in front counts
#pragma unroll
      for (int i = 0; i < 64; ++i) rank += (uint32_t)__builtin_amdgcn_readlane(cur, i) < limit;
    }
    cur = next;
    next = after;
  }
  part[wave][lane] = rank;
  __syncthreads();
  if (wave == 0 && t < tokens) {
    rank = 0;
#pragma unroll
    for (int w = 0; w < RANK_WAVES; ++w) rank += part[w][lane];
    key[rank] = mine;
    order[rank] = (uint32_t)t;
  }
}

// Order of many tokens: passes over digits of up to nine bits, from the lowest, each stable.  A tile of tokens is one block's;
// a pass counts the digits of every tile and then places the tiles' tokens.
constexpr int RADIX_BITS = 9, RADIX_BINS = 1 << RADIX_BITS;
constexpr int RADIX_STEP = 2048;  // tokens of a tile at a time: 8 of a thread
constexpr int RADIX_TILES = 256;  // at most

struct RadixArgs {
  const int32_t* ids;                          // first pass
  const uint32_t *key_in, *order_in;           // later ones
  uint32_t *key, *order;
  uint32_t* count;                             // [tiles][bins]
  int64_t tokens, tile;
  uint32_t rows;
  int shift, bits;
  unsigned tiles;
};

__device__ __forceinline__ uint32_t radix_key(const RadixArgs& a, int64_t i) {
  return a.ids ? sort_key(a.ids[i], a.rows) : a.key_in[i];
}

__global__ __launch_bounds__(256) void embedding_count_kernel(const RadixArgs a, ZeroShare z) {
  if (blockIdx.x >= a.tiles) {
    zero_share(z, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    return;
  }
  __shared__ uint32_t bin[RADIX_BINS];
  const int bins = 1 << a.bits;
  for (int b = threadIdx.x; b < bins; b += 256) bin[b] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * a.tile, hi = min(lo + a.tile, a.tokens);
  for (int64_t i = lo + threadIdx.x; i < hi; i += 256) atomicAdd(&bin[(radix_key(a, i) >> a.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 256) a.count[(size_t)blockIdx.x * bins + b] = bin[b];
}

// LDS accesses of the wavefront's lanes in front of it are made before those behind it (no instruction: the hardware keeps a
// wavefront's LDS accesses in order, the compiler only what one lane can see)
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(256) void embedding_place_kernel(const RadixArgs a, ZeroShare z) {
  if (blockIdx.x >= a.tiles) {
    zero_share(z, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    return;
  }
  __shared__ uint32_t next[RADIX_BINS];          // where the next token of a digit goes
  __shared__ uint32_t seen[4][RADIX_BINS];       // tokens of a digit that each wavefront holds of this step
  __shared__ uint32_t wsum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bins = 1 << a.bits;
  {  // first place of a digit in this tile: all smaller digits, and this digit in the tiles in front
    uint32_t before[2] = {0, 0}, all[2] = {0, 0};
    if (2 * tid < bins) {
      const uint2* const c = reinterpret_cast<const uint2*>(a.count) + tid;  // (two digits, of one tile after the other)
#pragma unroll 16
      for (unsigned t = 0; t < a.tiles; ++t) {
        const uint2 v = c[(size_t)t * (bins / 2)];
        before[0] += t < blockIdx.x ? v.x : 0;
        before[1] += t < blockIdx.x ? v.y : 0;
        all[0] += v.x;
        all[1] += v.y;
      }
    }
    uint32_t sum = all[0] + all[1];  // inclusive prefix over the threads
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    if (lane == 63) wsum[wave] = sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) sum += wsum[w];
    const uint32_t start = sum - all[0] - all[1];
    if (2 * tid < bins) next[2 * tid] = start + before[0];
    if (2 * tid + 1 < bins) next[2 * tid + 1] = start + all[0] + before[1];
  }
  const int64_t lo = blockIdx.x * a.tile, hi = min(lo + a.tile, a.tokens);
  for (int64_t s = lo; s < hi; s += RADIX_STEP) {
    __syncthreads();
    for (int b = tid; b < 4 * RADIX_BINS; b += 256) (&seen[0][0])[b] = 0;
    __syncthreads();
    // a wavefront holds 512 consecutive tokens, 64 at a time; tokens of equal digit are numbered in their order
    uint32_t k[8], o[8], at[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int64_t i = s + wave * 512 + r * 64 + lane;
      const bool on = i < hi;
      k[r] = on ? radix_key(a, i) : 0;
      o[r] = on ? (a.ids ? (uint32_t)i : a.order_in[i]) : 0;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const bool on = s + wave * 512 + r * 64 + lane < hi;
      const uint32_t d = (k[r] >> a.shift) & (bins - 1);
      uint64_t same = __ballot(on);
      for (int b = 0; b < a.bits; ++b) {
        const uint64_t bit = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? bit : ~bit;
      }
      const uint64_t below = same & ((1ull << lane) - 1);
      at[r] = on ? seen[wave][d] + (uint32_t)__popcll(below) : 0;
      wave_order();
      if (on && below == 0) seen[wave][d] = at[r] + (uint32_t)__popcll(same);  // one lane a digit, behind every lane's read
      wave_order();
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if (s + wave * 512 + r * 64 + lane >= hi) continue;
      const uint32_t d = (k[r] >> a.shift) & (bins - 1);
      uint32_t p = next[d] + at[r];
      for (int w = 0; w < wave; ++w) p += seen[w][d];
      a.key[p] = k[r];
      a.order[p] = o[r];
    }
    __syncthreads();
    for (int b = tid; b < bins; b += 256) next[b] += seen[0][b] + seen[1][b] + seen[2][b] + seen[3][b];
  }
}

// Sums over the sorted tokens.  A wavefront takes `chunk` of them and 512 columns, eight a lane, and adds up runs of equal
// ids; a run that lies inside the chunk is a row's gradient, one that crosses its border leaves a partial: part[c][0] where it
// began in front of the chunk, part[c][1] where it begins in it.
struct SumArgs {
  const uint32_t *key, *order;
  int64_t tokens;
  uint32_t rows;
  int width, chunk, accumulate;
  float scale;
  float* dtable;
  float* part;  // [chunks][2][width]
};

constexpr int SUM_COLS = 512;

// How the columns are read and written: eight at 16-byte addresses; eight at any address, where the last lane of a row takes its
// last eight and so some of its neighbour's (what is written comes out the same from both; what is added to is written by its
// own lane alone); or what there is, of rows of fewer than eight and of those whose last SUM_COLS columns are fewer than eight.
enum : int { COLS_EVEN = 0, COLS_ANY = 1, COLS_NARROW = 2 };
template <int COLS>
__device__ __forceinline__ int first_col(int width, int lane) {
  const int c = blockIdx.x * SUM_COLS + lane * 8;
  return COLS == COLS_ANY && c < width ? min(c, width - 8) : c;
}
template <int COLS>
__device__ __forceinline__ void put8(float* p, int n, const float (&v)[8]) {
  if (COLS == COLS_NARROW) store8_part(p, n, v);
  else store8(p, v);
}
template <int COLS>
__device__ __forceinline__ void put_row(const SumArgs& g, uint32_t k, int c, const float (&v)[8]) {
  float* p = g.dtable + (size_t)k * g.width + c;
  float f[8];
  if (g.accumulate) {
    if (COLS == COLS_NARROW) load8_part(p, g.width - c, f);
    else load8(p, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = fmaf(v[i], g.scale, f[i]);
    const int over = blockIdx.x * SUM_COLS + (threadIdx.x & 63) * 8 - c;  // leading ones that are the neighbour's
    if (COLS == COLS_ANY && over > 0) {
#pragma unroll
      for (int i = 1; i < 8; ++i)
        if (i >= over) p[i] = f[i];
      return;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i] * g.scale;
  }
  put8<COLS>(p, g.width - c, f);
}

template <typename T, int COLS>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const SumArgs g, const T* __restrict__ dy) {
  constexpr int B = COLS == COLS_EVEN ? 8 : 4;  // tokens whose rows are requested at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t chunk_id = (int64_t)blockIdx.y * 4 + wave;
  const int64_t lo = chunk_id * g.chunk, hi = min(lo + g.chunk, g.tokens);
  if (lo >= hi) return;
  const int c = first_col<COLS>(g.width, lane);
  const bool live = c < g.width;
  if (g.key[lo] >= g.rows) return;  // behind the last row: padding
  const bool began = lo > 0 && g.key[lo - 1] == g.key[lo];
  const uint32_t next = hi < g.tokens ? g.key[hi] : 0xffffffffu;
  float acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  uint32_t cur = g.key[lo];
  bool first = true;
  auto flush = [&](bool last) __attribute__((always_inline)) {
    if (cur >= g.rows) return;
    const bool open = first && began;
    if (open || (last && next == cur)) {
      if (live) put8<COLS>(g.part + ((size_t)chunk_id * 2 + (open ? 0 : 1)) * g.width + c, g.width - c, acc);
    } else if (live) {
      put_row<COLS>(g, cur, c, acc);
    }
  };
  for (int64_t i = lo; i < hi; i += B) {
    Eight<T, COLS == COLS_EVEN> raw[B];
    float part[COLS == COLS_NARROW ? B : 1][8];
    uint32_t k[B];
    const int m = (int)min((int64_t)B, hi - i);
#pragma unroll
    for (int r = 0; r < B; ++r) {  // (behind the end: the last row once more)
      const int64_t at = i + min(r, m - 1);
      k[r] = g.key[at];
      const T* src = dy + (size_t)g.order[at] * g.width + (live ? c : 0);
      if (COLS == COLS_NARROW) load8_part(src, live ? g.width - c : 0, part[COLS == COLS_NARROW ? r : 0]);
      else raw[r].load(src);
    }
#pragma unroll
    for (int r = 0; r < B; ++r) {
      if (r >= m) break;
      if (k[r] != cur) {
        flush(false);
        first = false;
        cur = k[r];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      }
      float v[8];
      if (COLS != COLS_NARROW) raw[r].values(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += COLS == COLS_NARROW ? part[COLS == COLS_NARROW ? r : 0][e] : v[e];
    }
  }
  flush(true);
}

// Runs that cross chunks: the block of the chunk in which one begins adds up its partials, each wavefront every eighth, in 64
// bits, and the wavefronts' sums in their order.
template <int COLS>
__global__ __launch_bounds__(512, 6) void embedding_join_kernel(const SumArgs g) {
  __shared__ double sh[8][SUM_COLS];
  const int64_t c0 = blockIdx.y;
  const int64_t lo = c0 * g.chunk, hi = lo + g.chunk;  // (the last chunk has no block)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t chunks = (g.tokens + g.chunk - 1) / g.chunk;
  const uint32_t k = g.key[hi - 1], behind = g.key[hi], first = g.key[lo], before = lo > 0 ? g.key[lo - 1] : 0xffffffffu;
  // does the run go on in a chunk (its first key)?  Every wavefront looks at 64 chunks at a time
  auto goes_on = [&](int64_t j) { return j < chunks && g.key[j * g.chunk] == k; };
  uint64_t on = __ballot(goes_on(c0 + 1 + lane));
  if (k >= g.rows || behind != k) return;     // nothing goes on behind this chunk
  if (first == k && before == k) return;      // it began in front of it
  int64_t last = c0 + (~on ? __builtin_ctzll(~on) : 64);
  if (!~on) {  // a long one: 64 steps of 64 chunks, then the chunks of the last step
    for (;;) {
      on = __ballot(goes_on(last + 64 * (lane + 1)));
      if (~on) break;
      last += 64 * 64;
    }
    last += 64 * __builtin_ctzll(~on);
    on = __ballot(goes_on(last + 1 + lane));
    last += ~on ? __builtin_ctzll(~on) : 64;
  }
  const int c = first_col<COLS>(g.width, lane), n = g.width - c;
  double v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0;
  if (n > 0)
    for (int64_t j0 = c0 + wave; j0 <= last; j0 += 16) {  // two at a time
      float f[2][8];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int64_t j = min(j0 + 8 * q, last);
        const float* p = g.part + ((size_t)j * 2 + (j == c0 ? 1 : 0)) * g.width + c;
        if (COLS == COLS_NARROW) load8_part(p, n, f[q]);
        else load8(p, f[q]);
      }
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += j0 + 8 * q <= last ? f[q][i] : 0.f;
    }
#pragma unroll
  for (int i = 0; i < 8; ++i) sh[wave][i * 64 + lane] = v[i];
  __syncthreads();
  if (wave == 0 && n > 0) {
    float f[8];
    for (int w = 1; w < 8; ++w)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += sh[w][i * 64 + lane];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
    put_row<COLS>(g, k, c, f);
  }
}

// Groups of eight values of a thread: four where that leaves the chip full; 0: rows of fewer than eight, a value a thread.
int fwd_groups(int64_t tokens, int64_t width) { return width < 8 ? 0 : tokens * width >= 8 * 256 * 4 * 1024 ? 4 : 1; }

}  // namespace

void embedding_fwd(hipStream_t st, const int32_t* ids, int64_t tokens, const void* table, bool table_bf16, int64_t rows,
                   int64_t width, float scale, void* y, bool y_bf16) {
  if (tokens <= 0) return;
  const int64_t total = tokens * width;
  const unsigned most = 1 << 20;
#define NARROW(TW, TY)                                                                                                       \
  KLAUNCH((embedding_fwd_narrow_kernel<TW, TY>), dim3((unsigned)std::min<int64_t>((total + 255) / 256, most)), dim3(256), 0, st, ids, \
          tokens, static_cast<const TW*>(table), (uint32_t)rows, (int)width, scale, static_cast<TY*>(y))
#define LAUNCH(TW, TY, U, EVEN)                                                                                              \
  KLAUNCH((embedding_fwd_kernel<TW, TY, U, EVEN>), dim3((unsigned)std::min<int64_t>((total + 2048 * U - 1) / (2048 * U), most)), \
          dim3(256), 0, st, ids, tokens, static_cast<const TW*>(table), (uint32_t)rows, (int)width, 1.f / (float)width, scale,  \
          static_cast<TY*>(y))
  const int groups = fwd_groups(tokens, width);
  const bool even = width * (table_bf16 ? 2 : 4) % 16 == 0 && reinterpret_cast<uintptr_t>(table) % 16 == 0;
#define PICK(TW, TY)                            \
  do {                                          \
    if (!groups) NARROW(TW, TY);                \
    else if (groups == 4 && even) LAUNCH(TW, TY, 4, true);  \
    else if (groups == 4) LAUNCH(TW, TY, 4, false);         \
    else LAUNCH(TW, TY, 1, false);              \
  } while (0)
  if (table_bf16) {
    if (y_bf16) PICK(bf16_t, bf16_t); else PICK(bf16_t, float);
  } else {
    if (y_bf16) PICK(float, bf16_t); else PICK(float, float);
  }
#undef PICK
#undef LAUNCH
#undef NARROW
}

namespace {

// Tokens that are placed by counting (it grows with their square, the passes hardly; the whole gradient, added to, us, counting /
// passes: 32768 rows of 512, 8192 tokens 28.7 / 38.5, 12288 38.8 / 45.2, 16384 48.7 / 50.3; 2000 rows of 64, 8192 23.8 / 31.4,
// 12288 32.0 / 35.3, 16384 37.2 / 35.1; written, rows of 64, 16384 44 / 42, 32768 122 / 42).
constexpr int64_t RANK_MOST = 16384;

// Tokens of a wavefront: the chip filled, and no more than 8192 partials.  (65536 tokens of 1024: chunks of 32 187 us, of 16 192, of
// 8 207, each before the shares of a row were put side by side; 4096 tokens of 512: of 8 21.4, of 4 21.9.)
int chunk_of(int64_t tokens) {
  int c = 8;
  while (c < 32 && tokens / c >= 2048) c *= 2;
  while ((tokens + c - 1) / c > 8192) c *= 2;
  return c;
}
int64_t chunks_of(int64_t tokens) { return (tokens + chunk_of(tokens) - 1) / chunk_of(tokens); }
size_t align16(size_t v) { return (v + 15) / 16 * 16; }

int radix_passes(int64_t rows, int* bits) {  // digits of equal size for the keys 0 .. rows
  int b = 1;
  while (((int64_t)1 << b) <= rows) ++b;
  const int passes = (b + RADIX_BITS - 1) / RADIX_BITS;
  *bits = (b + passes - 1) / passes;
  return passes;
}
int64_t radix_tile(int64_t tokens) {
  const int64_t per = (tokens + RADIX_TILES - 1) / RADIX_TILES;
  return (per + RADIX_STEP - 1) / RADIX_STEP * RADIX_STEP;
}

}  // namespace

// key and order, for the radix passes twice, the digit counts; then the partials
size_t embedding_bwd_ws_bytes(int64_t tokens, int64_t, int64_t width) {
  if (tokens <= 0) return 0;
  const size_t lists = align16((size_t)tokens * 4) * (tokens > RANK_MOST ? 4 : 2);
  const size_t counts = tokens > RANK_MOST ? (size_t)RADIX_TILES * RADIX_BINS * 4 : 0;
  return lists + counts + align16((size_t)chunks_of(tokens) * 2 * width * 4);
}

void embedding_bwd(hipStream_t st, const int32_t* ids, int64_t tokens, const void* dy, bool dy_bf16, int64_t rows,
                   int64_t width, float scale, bool accumulate, float* dtable, void* ws) {
  char* at = static_cast<char*>(ws);
  auto take = [&](size_t bytes) { char* p = at; at += align16(bytes); return p; };
  const bool radix = tokens > RANK_MOST;
  int bits = 0;
  const int passes = radix ? radix_passes(rows, &bits) : 0;
  const int shares = tokens <= 0 ? 1 : radix ? 2 * passes : 1;

  // zeros: a 16-byte aligned middle in equal shares, the edges with the first
  const size_t n = accumulate ? 0 : (size_t)rows * width;
  const size_t head = std::min<size_t>((16 - (reinterpret_cast<uintptr_t>(dtable) & 15)) / 4 % 4, n);
  const size_t n4 = (n - head) / 4;
  auto share = [&](int i) {
    ZeroShare z = {};
    const size_t lo = n4 * i / shares, hi = n4 * (i + 1) / shares;
    z.p = dtable + head + 4 * lo;
    z.n4 = hi - lo;
    if (i == 0) {
      z.edge[0] = dtable;
      z.edges[0] = (int)head;
      z.edge[1] = dtable + head + 4 * n4;
      z.edges[1] = (int)(n - head - 4 * n4);
    }
    return z;
  };
  auto zero_blocks = [&](const ZeroShare& z, unsigned threads) {
    if (!z.n4 && !z.edges[0] && !z.edges[1]) return 0u;
    return (unsigned)std::min<size_t>(z.n4 / (4 * threads) + 1, 4096);
  };

  if (tokens <= 0) {
    const ZeroShare z = share(0);
    const unsigned zb = zero_blocks(z, 64 * RANK_WAVES);
    if (zb) KLAUNCH(embedding_rank_kernel, dim3(zb), dim3(64 * RANK_WAVES), 0, st, ids, 0, 0u, nullptr, nullptr, 0u, z);
    return;
  }
  uint32_t* key = reinterpret_cast<uint32_t*>(take((size_t)tokens * 4));
  uint32_t* order = reinterpret_cast<uint32_t*>(take((size_t)tokens * 4));
  if (!radix) {
    const ZeroShare z = share(0);
    const unsigned sort = (unsigned)((tokens + 63) / 64);
    KLAUNCH(embedding_rank_kernel, dim3(sort + zero_blocks(z, 64 * RANK_WAVES)), dim3(64 * RANK_WAVES), 0, st, ids, (int)tokens,
            (uint32_t)rows, key, order, sort, z);
  } else {
    RadixArgs a = {};
    uint32_t* key2 = reinterpret_cast<uint32_t*>(take((size_t)tokens * 4));
    uint32_t* order2 = reinterpret_cast<uint32_t*>(take((size_t)tokens * 4));
    a.count = reinterpret_cast<uint32_t*>(take((size_t)RADIX_TILES * RADIX_BINS * 4));
    a.tokens = tokens;
    a.tile = radix_tile(tokens);
    a.tiles = (unsigned)((tokens + a.tile - 1) / a.tile);
    a.rows = (uint32_t)rows;
    a.bits = bits;
    uint32_t *ka = key2, *oa = order2;
    for (int p = 0; p < passes; ++p) {
      a.ids = p == 0 ? ids : nullptr;
      a.key_in = key;
      a.order_in = order;
      a.key = ka;
      a.order = oa;
      a.shift = p * bits;
      const ZeroShare z0 = share(2 * p), z1 = share(2 * p + 1);
      KLAUNCH(embedding_count_kernel, dim3(a.tiles + zero_blocks(z0, 256)), dim3(256), 0, st, a, z0);
      KLAUNCH(embedding_place_kernel, dim3(a.tiles + zero_blocks(z1, 256)), dim3(256), 0, st, a, z1);
      std::swap(ka, key);
      std::swap(oa, order);
    }
  }
  SumArgs g = {};
  g.key = key;
  g.order = order;
  g.tokens = tokens;
  g.rows = (uint32_t)rows;
  g.width = (int)width;
  g.chunk = chunk_of(tokens);
  g.accumulate = accumulate;
  g.scale = scale;
  g.dtable = dtable;
  const int64_t chunks = chunks_of(tokens);
  g.part = reinterpret_cast<float*>(take((size_t)chunks * 2 * width * 4));
  const unsigned cols_blocks = (unsigned)((width + SUM_COLS - 1) / SUM_COLS);
  // (The shares of a row's columns in neighbouring blocks, so that its memory is read at one time: 65536 tokens of 1024 183 us; a share
  // of all rows after another 187.  chunks_of() stays far below the 65535 blocks of this direction.)
  const dim3 grid(cols_blocks, (unsigned)((chunks + 3) / 4));
  const bool even = width % 8 == 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0 && reinterpret_cast<uintptr_t>(dtable) % 16 == 0;
  auto go = [&](auto cols) {
    constexpr int C = decltype(cols)::value;
    if (dy_bf16) KLAUNCH_NAMED("embedding_sum_kernel", (embedding_sum_kernel<bf16_t, C>), grid, dim3(256), 0, st, g, static_cast<const bf16_t*>(dy));
    else KLAUNCH_NAMED("embedding_sum_kernel", (embedding_sum_kernel<float, C>), grid, dim3(256), 0, st, g, static_cast<const float*>(dy));
    if (chunks > 1) KLAUNCH_NAMED("embedding_join_kernel", (embedding_join_kernel<C>), dim3(cols_blocks, (unsigned)(chunks - 1)), dim3(512), 0, st, g);
  };
  if (even) go(std::integral_constant<int, COLS_EVEN>());
  else if (width >= 8 && (width % SUM_COLS == 0 || width % SUM_COLS >= 8)) go(std::integral_constant<int, COLS_ANY>());
  else go(std::integral_constant<int, COLS_NARROW>());
}

}  // namespace ast

// The choice of the lookup's kernel, for tests: groups of eight values of a thread (0: a value a thread).
extern "C" int ast_embedding_fwd_choice(int64_t tokens, int64_t width) { return ast::fwd_groups(tokens, width); }
