// Selection of key blocks for block-sparse reads of the retained shards: channel
// bounds of every block of keys, the score that a block's bounds allow, and the
// topk blocks of each shard.
#include <algorithm>
#include <type_traits>

#include "tiles.hpp"

namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Bounds: bounds[shard][kvh][b][0 | 1][i] = min | max over the block's keys of
// channel i.  The values are keys' own, so nothing is rounded; a NaN key gives
// NaN.  One thread per 16-byte column of a block, U rows in flight; bound by
// reading K once.
__global__ __launch_bounds__(256) void key_bounds_kernel(const uint16_t* __restrict__ K, int64_t S,
                                                         int Hkv, int d, int block, int blocks,
                                                         uint16_t* __restrict__ bounds,
                                                         int64_t total) {
  constexpr int U = 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const int cols = Hkv * d / 8;
  const int c = (int)(i % cols);
  const int64_t sb = i / cols;
  const int b = (int)(sb % blocks);
  const int64_t shard = sb / blocks;
  const int64_t row0 = (int64_t)b * block;
  const int rows = (int)min((int64_t)block, S - row0);
  const bf16x8* src = reinterpret_cast<const bf16x8*>(K) + (shard * S + row0) * cols + c;
  f32x8 lo = __builtin_convertvector(src[0], f32x8), hi = lo;
  for (int r = 0; r < rows; r += U) {
    bf16x8 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = src[(int64_t)min(r + u, rows - 1) * cols];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const f32x8 y = __builtin_convertvector(x[u], f32x8);
      lo = __builtin_elementwise_minimum(lo, y);
      hi = __builtin_elementwise_maximum(hi, y);
    }
  }
  const int kvh = c * 8 / d, dim = c * 8 - kvh * d;
  uint16_t* dst = bounds + ((shard * Hkv + kvh) * blocks + b) * 2 * d + dim;
  *reinterpret_cast<bf16x8*>(dst) = __builtin_convertvector(lo, bf16x8);
  *reinterpret_cast<bf16x8*>(dst + d) = __builtin_convertvector(hi, bf16x8);
}

// ---------------------------------------------------------------------------
// Scores: score[shard][t][kvh][b] = max over the heads of the group of
// sum_i max(q_i lo_i, q_i hi_i) = sum_i max(q_i, 0) hi_i + min(q_i, 0) lo_i, in
// fp64 (the products are exact) and rounded once to fp32.  A score that is not a
// number, and that of a block with any bound that is not finite, ranks above all: +inf.

// Magnitudes as their bits: without their signs bf16 rank as integers, what is not finite
// from kInfinite on.
constexpr int kInfinite = 0x7f80;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
struct Magnitudes {
  int most = 0, least = 0xffff;  // of those that are not 0
  template <typename T, int N>
  __device__ __forceinline__ void add(const T (&x)[N]) {
    u16x2 top = {0, 0}, low = {0xffff, 0xffff};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) / 4)));
      const words w = __builtin_bit_cast(words, x[i]) & 0x7fff7fffu;
#pragma unroll
      for (int k = 0; k < (int)(sizeof(T) / 4); ++k) {
        const u16x2 y = __builtin_bit_cast(u16x2, (uint32_t)w[k]);
        top = __builtin_elementwise_max(top, y);
        low = __builtin_elementwise_min(low, y - (u16x2){1, 1});  // (a 0 is passed over)
      }
    }
    most = max(most, max((int)top[0], (int)top[1]));
    least = min(least, min((int)low[0], (int)low[1]));
  }
  // over the lanes r, r + 16, r + 32, r + 48
  __device__ __forceinline__ void join_rows() {
#pragma unroll
    for (int lanes = 16; lanes < 64; lanes <<= 1) {
      most = max(most, __shfl_xor(most, lanes, 64));
      least = min(least, __shfl_xor(least, lanes, 64));
    }
  }
  __device__ __forceinline__ double size() const { return (double)__int_as_float(most << 16); }
  // the exponent of a unit that all of them are multiples of
  __device__ __forceinline__ int unit() const { return max((least + 1) >> 7, 1) - 134; }
};

// The score's sum of D products is that of sixteen parts of consecutive channels, added
// two by two: as sixteen lanes form it for the selection, or one lane here.
template <int D>
__device__ __forceinline__ double sum_in_order(const uint16_t* q, const uint16_t* b) {
  double half[4];  // sums of 1, 2, 4 and 8 parts that wait for as many more
#pragma unroll 1
  for (int part = 0;; ++part) {
    double s = 0.;
    for (int i = part * (D / 16); i < (part + 1) * (D / 16); ++i) {
      const float y = __uint_as_float((uint32_t)q[i] << 16);
      const float x = __uint_as_float((uint32_t)b[y < 0.f ? i : D + i] << 16);
      s = __builtin_fma((double)y, (double)x, s);
    }
    bool ends = true;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!ends) continue;
      ends = (part >> k) & 1;
      if (ends) s = half[k] + s;
      else half[k] = s;
    }
    if (ends) return s;
  }
}
// Whether a sum s of the same products in another order gives the same fp32.  In any
// order it is off by at most D 2^-52 of sum_i |q_i b_i|, which D times the largest factors
// bound: either no fp32 ends within twice that of s, or all sums are multiples of the
// factors' units that fp64 holds exactly (as nearly all of random values are, 6 to 22 %
// of which end at the border between two fp32).
template <int D>
__device__ __forceinline__ bool any_order(double s, const Magnitudes& q, const Magnitudes& b) {
  const double size = D * (q.size() * b.size());
  const double off = size * (D * 0x1p-51);
  return (float)(s - off) == (float)(s + off) || s - s != 0. ||
         size <= __builtin_ldexp(1., 53 + q.unit() + b.unit());
}

// Where the caller wants the scores: a wave takes 16 blocks as the rows of 16x16x4
// fp64 matrix products and walks over tiles of 16 (token, head) columns.  Lane (r,
// g) holds channels g D/4 .. of its block, so that it loads whole 16-byte pieces;
// the channels of a product are then D/4 apart, the same for both operands.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void block_scores_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ bounds, int Tq, int Hq, int Hkv,
    int blocks, int tiles, int tiles_per_wg, float* __restrict__ scores) {
  constexpr int N = D / 4;  // channels per lane
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int group = Hq / Hkv;
  const int64_t shard = blockIdx.y / Hkv;
  const int kvh = (int)(blockIdx.y - shard * Hkv);
  const int b0 = (blockIdx.x * 4 + wave) * 16;
  if (b0 >= blocks) return;
  bf16x8 lo[N / 8], hi[N / 8];
  {
    const uint16_t* p =
        bounds + ((int64_t)blockIdx.y * blocks + min(b0 + r, blocks - 1)) * 2 * D + g * N;
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      lo[i] = reinterpret_cast<const bf16x8*>(p)[i];
      hi[i] = reinterpret_cast<const bf16x8*>(p + D)[i];
    }
  }
  // the bounds of row r, then of the rows whose products a lane gets, 4v + g
  Magnitudes mine, block[4];
  mine.add(lo);
  mine.add(hi);
  mine.join_rows();
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    block[v].most = __shfl(mine.most, 4 * v + g, 64);
    block[v].least = __shfl(mine.least, 4 * v + g, 64);
  }
  // columns: 16 / group tokens of `group` heads, or 16 heads of one token at a time
  const int tokens = max(16 / group, 1);
  const int passes = (group + 15) / 16;
  const int first = blockIdx.z * tiles_per_wg, last = min(first + tiles_per_wg, tiles);
  for (int tile = first; tile < last; ++tile) {
    float best[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) best[v] = -INFINITY;
    const int tl = group >= 16 ? 0 : r / group;
    const int t = tile * tokens + tl;
    for (int pass = 0; pass < passes; ++pass) {
      const int h = group >= 16 ? pass * 16 + r : r - tl * group;
      const bool live = tl < tokens && t < Tq && h < group;
      bf16x8 x[N / 8];
      const bf16x8* p = reinterpret_cast<const bf16x8*>(
          q + (live ? ((int64_t)t * Hq + kvh * group + h) * D : 0) + g * N);
#pragma unroll
      for (int i = 0; i < N / 8; ++i) x[i] = p[i];
      f64x4 up = {0., 0., 0., 0.}, down = up;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float qi = (float)x[i / 8][i % 8];
        up = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)hi[i / 8][i % 8],
                                                  (double)(qi < 0.f ? 0.f : qi), up, 0, 0, 0);
        down = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)lo[i / 8][i % 8],
                                                    (double)(qi < 0.f ? qi : 0.f), down, 0, 0, 0);
      }
      Magnitudes head;
      head.add(x);
      head.join_rows();
      double sum[4];
      int open = 0;  // sums to be formed in order
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        sum[v] = up[v] + down[v];
        if (live && !any_order<D>(sum[v], head, block[v])) open |= 1 << v;
      }
      if (open != 0)
#pragma unroll 1
        for (int v = 0; v < 4; ++v) {
          if (!((open >> v) & 1)) continue;
          const int64_t b = (int64_t)blockIdx.y * blocks + min(b0 + 4 * v + g, blocks - 1);
          const double x = sum_in_order<D>(q + ((int64_t)t * Hq + kvh * group + h) * D,
                                           bounds + b * 2 * D);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[k] = k == v ? x : sum[k];
        }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float s = (float)sum[v];
        s = s != s || block[v].most >= kInfinite ? INFINITY : s;
        best[v] = fmaxf(best[v], live ? s : -INFINITY);
      }
    }
    // the largest of each token's columns; register v holds block 4v + g
    const int width = min(group, 16);
    const int base = lane - r + tl * width;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      float s = best[v];
      for (int j = 0; j < width; ++j) s = fmaxf(s, __shfl(best[v], min(base + j, 63), 64));
      const int b = b0 + 4 * v + g;
      if (r == tl * width && tl < tokens && t < Tq && b < blocks)
        scores[((shard * Tq + t) * Hkv + kvh) * (int64_t)blocks + b] = s;
    }
  }
}

// ---------------------------------------------------------------------------
// Near scores, for the selection alone: the same sums by bf16 matrix products
// (16x16x32, exact products, fp32 sums).  The fp64 products bound the exact form (64
// tokens, 4096 blocks of 8 KV heads: 123 us with the pick); the selection needs them
// only for the few blocks whose near scores lie within their errors of the last one
// that it keeps.
//
// Error.  A sum of n = 2 D products in any order, each addition off by at most
// 2^-23 of the running size, is off by n 2^-23 times the size sum_i |q_i| m_i <=
// |q| |m| of the block, with m_i the larger magnitude of lo_i and hi_i and |.| the
// Euclidean norm (at random values a quarter above the sum itself).  The fiftieth on
// top covers the norms' rounding and that of the exact score to fp32.  Where |q| |m|
// leaves the fp32 range all blocks are scored exactly; kNearLeast covers products
// that vanish in it.
template <int D>
constexpr float kNearError = 2 * D * 0x1p-23f * 1.02f;
constexpr float kNearLeast = 0x1p-90f;

// Rows of 16-byte chunks in LDS, the chunks of a row permuted by it, so that the
// same chunk of eight rows lies in different banks: CPR chunks a row.
template <int CPR>
__device__ __forceinline__ int chunk_at(int row, int chunk) {
  return row * CPR + (chunk ^ (CPR == 8 ? (row >> 1) & 7 : row & 7));
}

// Reductions over lanes without LDS: exchanges within a row of 16, then of rows.
template <int CTRL>
__device__ __forceinline__ int dpp(int x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)dpp<CTRL>((int)x); }
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(dpp<CTRL>(__float_as_int(x)));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const u32x2 u = __builtin_bit_cast(u32x2, x);
  return __builtin_bit_cast(double, u32x2{dpp<CTRL>(u[0]), dpp<CTRL>(u[1])});
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;
// op over the 16 lanes of a row; every lane has the result.
template <typename T, typename OP>
__device__ __forceinline__ T over_row(T x, OP op) {
  x = op(x, dpp<kSwap1>(x));
  x = op(x, dpp<kSwap2>(x));
  x = op(x, dpp<kMirror8>(x));
  return op(x, dpp<kMirror16>(x));
}
template <typename OP>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, OP op) {
  x = over_row(x, op);
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return op(b[0], b[1]);
}
struct Least {
  __device__ uint32_t operator()(uint32_t x, uint32_t y) const { return min(x, y); }
};
struct Most {
  template <typename T>
  __device__ T operator()(T x, T y) const { return max(x, y); }
};
// The largest of a row's values, none of them negative or NaN.
__device__ __forceinline__ float max_of_row_floats(float x) {
  return __int_as_float(over_row(__float_as_int(x), Most{}));
}
// The sum of the four lanes r, r + 16, r + 32, r + 48.
__device__ __forceinline__ float sum_of_rows(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
// A sum of squares that fp32 holds well enough for a norm; others are formed in fp64,
// in which no square of a bf16 leaves the range.
__device__ __forceinline__ bool in_range(float x) { return x > 0x1p-80f && x < 0x1p126f; }
__device__ __forceinline__ float norm_of(double x) {
  const float y = (float)__builtin_sqrt(x);
  return y == y ? y : INFINITY;
}
struct Sum {
  template <typename T>
  __device__ T operator()(T x, T y) const { return x + y; }
};
// The sum of the lanes below.
__device__ __forceinline__ int scan_below(int x) {
  int y = x;
  y += __builtin_amdgcn_update_dpp(0, y, 0x111, 0xf, 0xf, false);  // 1, 2, 4, 8 to the right
  y += __builtin_amdgcn_update_dpp(0, y, 0x112, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x114, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x118, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x142, 0xa, 0xf, false);  // row ends to the next row
  y += __builtin_amdgcn_update_dpp(0, y, 0x143, 0xc, 0xf, false);  // lane 31's to the upper half
  return y - x;
}
// The largest of `width` neighbouring lanes of a row of 16 (base: the first one) for
// each of N values, where they are a power of two by exchanges within the row.
template <int N>
__device__ __forceinline__ void max_of_columns(int (&x)[N], int width, int base) {
  if ((width & (width - 1)) == 0) {
    if (width >= 2)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = max(x[i], dpp<kSwap1>(x[i]));
    if (width >= 4)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = max(x[i], dpp<kSwap2>(x[i]));
    if (width >= 8)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = max(x[i], dpp<kMirror8>(x[i]));
    if (width >= 16)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = max(x[i], dpp<kMirror16>(x[i]));
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int y = x[i];
    for (int j = 0; j < width; ++j) y = max(y, __shfl(x[i], min(base + j, 63), 64));
    x[i] = y;
  }
}

// Lane (r, g): channels 32 s + 8 g .. of row r of 16 staged block rows (lo, then hi).
template <int D>
struct BoundsTile {
  bf16x8 lo[D / 32], hi[D / 32];
  __device__ __forceinline__ void read(const u32x4* rows, int r, int g) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      lo[s] = __builtin_bit_cast(bf16x8, rows[chunk_at<D / 4>(r, 4 * s + g)]);
      hi[s] = __builtin_bit_cast(bf16x8, rows[chunk_at<D / 4>(r, D / 8 + 4 * s + g)]);
    }
  }
  // The largest |m| of the 16 blocks.  (Without the sign bits magnitudes rank as
  // integers, what is not a number last.)
  __device__ __forceinline__ float norm() const {
    bf16x8 big[D / 32];
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const auto bits = [](bf16x8 x) {
        return __builtin_bit_cast(s16x8, __builtin_bit_cast(u32x4, x) & 0x7fff7fffu);
      };
      big[s] = __builtin_bit_cast(bf16x8, __builtin_elementwise_max(bits(lo[s]), bits(hi[s])));
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = __builtin_fmaf((float)big[s][i], (float)big[s][i], sum);
    }
    sum = sum_of_rows(sum);
    if (__any(!in_range(sum))) {
      double wide = 0.;
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double x = (double)(float)big[s][i];
          wide += x * x;
        }
      wide += __shfl_xor(wide, 16, 64);
      wide += __shfl_xor(wide, 32, 64);
      return max_of_row_floats(norm_of(wide));
    }
    return max_of_row_floats(__builtin_sqrtf(sum));
  }
};
// 16 block rows b0 .. of 4 D bytes each, whole rows by neighbouring lanes; a row past
// the last is loaded as the last.
template <int D>
__device__ __forceinline__ void stage_bounds(const uint16_t* bounds, int b0, int blocks, int lane,
                                             u32x4* rows) {
  constexpr int CPR = D / 4, U = 16 * CPR / 64;
  u32x4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * 64 + lane;
    x[u] = reinterpret_cast<const u32x4*>(
        bounds)[(int64_t)min(b0 + i / CPR, blocks - 1) * CPR + i % CPR];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * 64 + lane;
    rows[chunk_at<CPR>(i / CPR, i % CPR)] = x[u];
  }
}
// Column r of 16 staged rows of q, channels 32 s + 8 g ..
template <int D>
__device__ __forceinline__ void read_columns(const u32x4* rows, int r, int g,
                                             bf16x8 (&x)[D / 32]) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s)
    x[s] = __builtin_bit_cast(bf16x8, rows[chunk_at<D / 8>(r, 4 * s + g)]);
}

// |q| of one head, by a wave: two channels (one at D = 64) to a lane.
template <int D>
__device__ __forceinline__ float head_norm(const uint16_t* q, int lane) {
  float y[D / 64], x = 0.f;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    y[i] = __uint_as_float((uint32_t)q[lane * (D / 64) + i] << 16);
    x += y[i] * y[i];
  }
  x = sum_of_rows(over_row(x, Sum{}));
  if (in_range(x)) return __builtin_sqrtf(x);
  double wide = 0.;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) wide += (double)y[i] * (double)y[i];
  wide = over_row(wide, Sum{});
  wide += __shfl_xor(wide, 16, 64);
  wide += __shfl_xor(wide, 32, 64);
  return norm_of(wide);
}

// As 16-bit integers the larger of a bf16 and 0 is its positive part, the smaller its
// negative part.
template <typename T>
__device__ __forceinline__ T positive(T x) {
  return __builtin_bit_cast(
      T, __builtin_elementwise_max(__builtin_bit_cast(s16x8, x), (s16x8){}));
}
template <typename T>
__device__ __forceinline__ T negative(T x) {
  return __builtin_bit_cast(
      T, __builtin_elementwise_min(__builtin_bit_cast(s16x8, x), (s16x8){}));
}
// Near scores of 16 blocks (rows 4g + v) and the parts of 16 columns of q (lane (r, g):
// channels 32 s + 8 g .. of column r).
template <int D>
__device__ __forceinline__ f32x4 near_scores(const BoundsTile<D>& b, const bf16x8 (&pos)[D / 32],
                                             const bf16x8 (&neg)[D / 32]) {
  f32x4 up = {0.f, 0.f, 0.f, 0.f}, down = up;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    up = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.hi[s], pos[s], up, 0, 0, 0);
    down = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.lo[s], neg[s], down, 0, 0, 0);
  }
  return up + down;
}

// Scores as integers of the same order (their own inverse), which take one
// instruction to compare across lanes; -0 ranks below 0.
__device__ __forceinline__ int ordered(int x) { return x ^ ((x >> 31) & 0x7fffffff); }
constexpr int kLeast = (int)0x80000000;
__device__ __forceinline__ float ordered_float(int x) { return __int_as_float(ordered(x)); }

// near[row][b] for every row (shard, t, kvh), and norms[shard][kvh][b / 16], the
// largest |m| of 16 blocks.  A workgroup holds 64 blocks and walks over eight units of 16
// columns: 16 / group tokens, or 16 heads of one token of a larger group, whose units
// follow one another.  Bound by instructions: q is split into its parts once, where it
// is staged, not by each wave (64 tokens over 4096 blocks of 8 KV heads, 15.5 -> 15.0 us;
// 4 or 16 units per workgroup 17 and 18 us).
// (The blocks pass through the same LDS first, so that four workgroups fit a compute
// unit: that call is then one round of them.)
constexpr int kUnits = 4;    // staged at a time
constexpr int kUnitsWg = 8;  // of a workgroup
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4)))
void block_near_kernel(const uint16_t* __restrict__ q, const uint16_t* __restrict__ bounds, int Tq,
                       int Hq, int Hkv, int blocks, int units, int units_per_wg,
                       float* __restrict__ near, float* __restrict__ norms) {
  constexpr int CQ = D / 8;
  constexpr int PER = 256 / (16 * CQ), U = kUnits / PER;  // a thread's units: every PER-th, U
  __shared__ u32x4 s_rows[kUnits][2][16 * CQ];  // q's positive and negative parts
  static_assert(kUnits * 2 * CQ == 4 * (D / 4), "the blocks take as much");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int group = Hq / Hkv;
  const int64_t shard = blockIdx.y / Hkv;
  const int kvh = (int)(blockIdx.y - shard * Hkv);
  const int row_tile = blockIdx.x * 4 + wave, row_tiles = (blocks + 15) / 16;
  const int b0 = row_tile * 16;
  const int tokens = max(16 / group, 1);
  const int passes = (group + 15) / 16;
  const int width = min(group, 16);
  const int tl = group >= 16 ? 0 : r / group;
  const int base = lane - r + tl * width;
  const int first = blockIdx.z * units_per_wg, last = min(first + units_per_wg, units);
  // one chunk of U units from u0 on, all loads in flight
  const int c = threadIdx.x / CQ % 16, chunk = threadIdx.x % CQ;
  const int cl = group >= 16 ? 0 : c / group;
  const int unit0 = wave / (4 / PER);
  u32x4 staged[U];
  auto fetch = [&](int u0) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = u0 + i * PER + unit0;
      const int t = (passes == 1 ? u : u / passes) * tokens + cl;
      const int h = group >= 16 ? (passes == 1 ? 0 : u % passes) * 16 + c : c - cl * group;
      staged[i] = u32x4{0u, 0u, 0u, 0u};
      if (u < last && cl < tokens && t < Tq && h < group)
        staged[i] =
            reinterpret_cast<const u32x4*>(q)[((int64_t)t * Hq + kvh * group + h) * CQ + chunk];
    }
  };
  fetch(first);
  BoundsTile<D> b;
  {
    u32x4* const mine = &s_rows[0][0][0] + wave * 16 * (D / 4);
    stage_bounds<D>(bounds + (int64_t)blockIdx.y * blocks * 2 * D, b0, blocks, lane, mine);
    b.read(mine, r, g);  // (the wave's own rows)
  }
  if (blockIdx.z == 0) {
    const float norm = b.norm();
    if (lane == 0 && b0 < blocks) norms[(int64_t)blockIdx.y * row_tiles + row_tile] = norm;
  }
  int top[4];  // of the 4 blocks of a lane
  for (int u0 = first; u0 < last; u0 += kUnits) {
    __syncthreads();  // the rows before have been read
    const int n = min(kUnits, last - u0);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      s_rows[i * PER + unit0][0][chunk_at<CQ>(c, chunk)] = positive(staged[i]);
      s_rows[i * PER + unit0][1][chunk_at<CQ>(c, chunk)] = negative(staged[i]);
    }
    __syncthreads();
    if (u0 + kUnits < last) fetch(u0 + kUnits);
    for (int u = 0; u < n; ++u) {
      const int t = (passes == 1 ? u0 + u : (u0 + u) / passes) * tokens + tl;
      const int pass = passes == 1 ? 0 : (u0 + u) % passes;
      bf16x8 pos[D / 32], neg[D / 32];
      read_columns<D>(s_rows[u][0], r, g, pos);
      read_columns<D>(s_rows[u][1], r, g, neg);
      const f32x4 score = near_scores<D>(b, pos, neg);
      int now[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) now[v] = ordered(__float_as_int(score[v]));
      if (passes == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = now[i];
      } else {  // columns past the group's heads, staged as zeros, score nothing
        const bool live = pass * 16 + r < group;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          top[i] = max(pass == 0 ? kLeast : top[i], live ? now[i] : kLeast);
        if (pass + 1 < passes) continue;
      }
      int all[4] = {top[0], top[1], top[2], top[3]};
      max_of_columns(all, width, base);
      if (r != tl * width || tl >= tokens || t >= Tq || b0 >= blocks) continue;
      const int64_t row = (shard * Tq + t) * Hkv + kvh;
      float* const dst = near + row * blocks + b0 + 4 * g;
      if ((blocks & 3) == 0 && b0 + 16 <= blocks) {
        *reinterpret_cast<f32x4*>(dst) = f32x4{ordered_float(all[0]), ordered_float(all[1]),
                                               ordered_float(all[2]), ordered_float(all[3])};
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (b0 + 4 * g + v < blocks) dst[v] = ordered_float(all[v]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The topk largest of a row of scores, in index order; of equal scores the lower
// index.  W waves hold the row as rising integers in registers, R values per lane,
// and look for a value that topk of them reach: one wave bisects, counting with
// ballots; several narrow the range by histograms of 256 bins in LDS (4096 values:
// two to three rounds, where a bisection takes a barrier for each of about twelve).
//
// NEAR: the row holds near scores off by at most E.  With a the topk-th largest of
// them and b the next, a - b > 2 E settles the selection.  Otherwise a block above
// a + 2 E is kept, one below a - 2 E is not (at most topk - 1 exact scores lie above
// a + E, and at least topk reach a - E), and those between are scored exactly, 16
// lanes to a block, and take part in a second selection with their exact scores.
//
// FUSED: eight waves form the row's near scores first, 16 blocks at a time, and
// hand them over through LDS.
__device__ __forceinline__ uint32_t rising(float s) {
  const uint32_t u = __float_as_uint(s == 0.f ? 0.f : s);  // -0 ranks as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unrising(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kKept = 0xffffffffu;  // above every score's key; 0 is below

enum PickMode : int { PICK_EXACT, PICK_NEAR, PICK_FUSED };
constexpr int kFusedWaves = 8;
constexpr int kFusedHeads = 64;    // heads per KV head that a fused row stages
constexpr int kFusedBlocks = 512;  // and its blocks at most

template <int D>
struct FusedLds {
  u32x4 bounds[kFusedWaves][16 * (D / 4)];
  u32x4 q[kFusedHeads * (D / 8)];
  uint32_t row[kFusedBlocks];
  float norm[kFusedWaves], head_norm[kFusedWaves];
};

// Near scores of a row into s_row; the largest |m| of the wave's blocks is returned.
template <int D>
__device__ __forceinline__ float fused_scores(const uint16_t* qt, const uint16_t* bt, int group,
                                              int blocks, float* s_row, FusedLds<D>& l) {
  constexpr int CQ = D / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  float most = 0.f;
  stage_bounds<D>(bt, wave * 16, blocks, lane, l.bounds[wave]);
  for (int i = threadIdx.x; i < (group + 15) / 16 * 16 * CQ; i += 64 * kFusedWaves) {
    const int c = i / CQ;
    u32x4 x = {0u, 0u, 0u, 0u};
    if (c < group) x = reinterpret_cast<const u32x4*>(qt)[i];
    l.q[(c & ~15) * CQ + chunk_at<CQ>(c & 15, i % CQ)] = x;
  }
  __syncthreads();
  for (int b0 = wave * 16; b0 < blocks; b0 += kFusedWaves * 16) {
    BoundsTile<D> b;
    b.read(l.bounds[wave], r, g);
    most = fmaxf(most, b.norm());
    int top[4] = {kLeast, kLeast, kLeast, kLeast};
    for (int h0 = 0; h0 < group; h0 += 16) {
      const bool live = h0 + r < group;
      bf16x8 x[D / 32], pos[D / 32], neg[D / 32];
      read_columns<D>(l.q + h0 * CQ, r, g, x);
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        pos[s] = positive(x[s]);
        neg[s] = negative(x[s]);
      }
      const f32x4 score = near_scores<D>(b, pos, neg);
#pragma unroll
      for (int v = 0; v < 4; ++v)
        top[v] = max(top[v], live ? ordered(__float_as_int(score[v])) : kLeast);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float x = ordered_float(over_row(top[v], Most{}));
      if (r == 0 && b0 + 4 * g + v < blocks) s_row[b0 + 4 * g + v] = x;
    }
    if (b0 + kFusedWaves * 16 < blocks)
      stage_bounds<D>(bt, b0 + kFusedWaves * 16, blocks, lane, l.bounds[wave]);
  }
  return most;
}

template <int D, int W, int R, int MODE>
__global__ __launch_bounds__(MODE == PICK_FUSED ? 64 * kFusedWaves : 64 * W)
void block_pick_kernel(const uint16_t* __restrict__ q, const uint16_t* __restrict__ bounds,
                       const float* __restrict__ scores, const float* __restrict__ norms, int Tq,
                       int Hq, int Hkv, int blocks, int topk, int32_t* __restrict__ sel) {
  extern __shared__ uint32_t s_dynamic[];  // NEAR: [blocks]
  uint32_t* s_row = s_dynamic;
  __shared__ int s_gt[W], s_eq[W];
  __shared__ u32x4 s_ends[W];
  __shared__ int s_bin[W > 1 ? 256 : 1], s_found[3];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x;
  const int kvh = (int)(row % Hkv);
  const int64_t st = row / Hkv;
  const int t = (int)(st % Tq);
  const int group = Hq / Hkv;
  const uint16_t* const qt = q + ((int64_t)t * Hq + kvh * group) * D;
  const uint16_t* const bt = bounds + ((st / Tq) * Hkv + kvh) * blocks * 2 * D;
  const uint64_t below = (1ull << lane) - 1;

  float most = 0.f, heads = 0.f;
  __shared__ std::conditional_t<MODE == PICK_FUSED, FusedLds<D>, int> s_fused;
  if constexpr (MODE == PICK_FUSED) {
    static_assert(W == 1, "one wave selects");
    s_row = s_fused.row;
    float mine = 0.f;  // each wave's heads
    for (int h = wave; h < group; h += kFusedWaves)
      mine = fmaxf(mine, head_norm<D>(qt + h * D, lane));
    if (lane == 0) s_fused.head_norm[wave] = mine;
    mine = fused_scores<D>(qt, bt, group, blocks, reinterpret_cast<float*>(s_row), s_fused);
    if (lane == 0) s_fused.norm[wave] = mine;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < kFusedWaves; ++w) {
      most = fmaxf(most, s_fused.norm[w]);
      heads = fmaxf(heads, s_fused.head_norm[w]);
    }
  } else if constexpr (MODE == PICK_NEAR) {
    const int n = (blocks + 15) / 16;
    const float* const p = norms + ((st / Tq) * Hkv + kvh) * n;
    for (int i = tid; i < n; i += 64 * W) most = fmaxf(most, p[i]);
  }
  // the selecting waves meet; one alone only keeps its LDS accesses in order
  auto sync = [&]() {
    if constexpr (W > 1) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  };

  const int i0 = wave * (64 * R) + lane;
  uint32_t key[R];  // 0 past the row's end
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = min(i0 + 64 * i, blocks - 1);
    if constexpr (MODE == PICK_FUSED) key[i] = s_row[at];
    else key[i] = __float_as_uint(scores[row * blocks + at]);
  }
  // the largest |q| of the group's heads: a wave takes every W-th
  if constexpr (MODE == PICK_NEAR)
    for (int h = wave; h < group; h += W) heads = fmaxf(heads, head_norm<D>(qt + h * D, lane));
#pragma unroll
  for (int i = 0; i < R; ++i) key[i] = i0 + 64 * i < blocks ? rising(__uint_as_float(key[i])) : 0u;
  // The smallest lo, the largest of each other value.
  auto spread = [&](uint32_t lo, uint32_t hi, float x = 0.f, float y = 0.f) {
    u32x4 all = {over_wave(lo, Least{}), over_wave(hi, Most{}), 0u, 0u};
    if (W > 1) {  // (x and y are not negative: they rank as their bits)
      all[2] = over_wave(__float_as_uint(x), Most{});
      all[3] = over_wave(__float_as_uint(y), Most{});
      __syncthreads();
      if (lane == 0) s_ends[wave] = all;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const u32x4 other = s_ends[w];
        all[0] = min(all[0], other[0]);
#pragma unroll
        for (int k = 1; k < 4; ++k) all[k] = max(all[k], other[k]);
      }
    } else if (MODE == PICK_NEAR) {
      all[2] = over_wave(__float_as_uint(x), Most{});
      all[3] = over_wave(__float_as_uint(y), Most{});
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) all[k] = __builtin_amdgcn_readfirstlane(all[k]);
    return all;
  };
  // A value that `reach` >= topk keys reach, and fewer than topk a larger one where
  // reach > topk.  `kept` keys are kKept, those that are 0 take no part.
  uint32_t cut = 0;
  int reach = 0;
  auto find_cut = [&](int kept) {
    uint32_t lo = kKept, hi = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      // (as the last of all numbers a 0 is passed over, kKept as the first)
      lo = min(lo, key[i] - 1);
      hi = max(hi, key[i] + 1);
    }
    const u32x4 ends = spread(lo, hi, heads, most);
    lo = ends[0] + 1;
    hi = ends[1] - 1;
    if constexpr (MODE == PICK_NEAR) {
      heads = __uint_as_float(ends[2]);
      most = __uint_as_float(ends[3]);
    }
    if constexpr (W == 1) {
      reach = 0;
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        int n = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] >= mid));
        if (n >= topk) {
          lo = mid;
          reach = n;
        } else {
          hi = mid - 1;
        }
        if (n == topk) break;
      }
      if (reach == 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) reach += __popcll(__ballot(key[i] >= lo));
      }
      cut = lo;
    } else {
      int above = kept;  // keys above hi
      while (true) {
        const uint32_t span = hi - lo;
        const int shift = span > 255u ? 24 - __builtin_clz(span) : 0;  // span >> shift <= 255
        for (int i = tid; i < 256; i += 64 * W) s_bin[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (key[i] - lo <= span) atomicAdd(&s_bin[(key[i] - lo) >> shift], 1);
        __syncthreads();
        if (wave == 0) {  // four bins per lane, from the highest; counted from the top
          int c[4], sum = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            c[k] = s_bin[255 - 4 * lane - k];
            sum += c[k];
          }
          int before = above + scan_below(sum);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (before < topk && before + c[k] >= topk) {
              s_found[0] = 255 - 4 * lane - k;
              s_found[1] = before + c[k];
              s_found[2] = before;
            }
            before += c[k];
          }
        }
        __syncthreads();
        const uint32_t bin = __builtin_amdgcn_readfirstlane(s_found[0]);
        reach = __builtin_amdgcn_readfirstlane(s_found[1]);
        above = __builtin_amdgcn_readfirstlane(s_found[2]);
        lo += bin << shift;
        // (a distance from lo: below the keys of infinities lo + 2^shift passes 32 bits)
        hi = lo + min(hi - lo, (1u << shift) - 1);
        cut = lo;
        if (reach == topk || shift == 0) break;
      }
    }
  };
  find_cut(0);

  if constexpr (MODE != PICK_EXACT) {
    // the smallest key that reaches the cut, the largest that does not
    uint32_t a = kKept, b = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (key[i] >= cut) a = min(a, key[i]);
      else b = max(b, key[i]);
    }
    const u32x4 ends = spread(a, b);
    const bool zeros = (heads == 0.f && most < INFINITY) || (most == 0.f && heads < INFINITY);
    // (all scores of zeros are 0)
    // (no number where one of the norms is 0 and the other infinite)
    const float off = heads * most * kNearError<D>;
    const float E = zeros ? 0.f : off < INFINITY ? fmaxf(off, kNearLeast) : INFINITY;
    const float fa = unrising(ends[0]);
    const bool settled = topk == blocks ||
                         (reach == topk && fa - unrising(ends[1]) > 2 * E) || zeros;
    if (!settled) {
      // an infinite E leaves all open
      const bool none = !(E < INFINITY);
      const uint32_t above = none ? kKept - 1 : rising(fa + 2 * E);
      const uint32_t under = none ? 1u : rising(fa - 2 * E);
      uint32_t open = 0;  // bit i: key i is to be scored
      int n = 0, kept = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const bool in = key[i] > above, may = !in && key[i] >= under;
        key[i] = in ? kKept : 0u;
        if (may) open |= 1u << i;
        n += __popcll(__ballot(may));
        kept += __popcll(__ballot(in));
      }
      // their indices, listed after those of the waves before
      int at = 0, all = n;
      if (W > 1) {
        if (lane == 0) {
          s_gt[wave] = n;
          s_eq[wave] = kept;
        }
        __syncthreads();
        all = kept = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          at += w < wave ? s_gt[w] : 0;
          all += s_gt[w];
          kept += s_eq[w];
        }
        all = __builtin_amdgcn_readfirstlane(all);
        kept = __builtin_amdgcn_readfirstlane(kept);
      }
      const int mine = at;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const uint64_t vote = __ballot((open >> i) & 1);
        if ((open >> i) & 1) s_row[at + __popcll(vote & below)] = i0 + 64 * i;
        at += __popcll(vote);
      }
      sync();
      constexpr int N = D / 16;  // channels per lane
      typedef __bf16 bf16xN __attribute__((ext_vector_type(N)));
      typedef double f64xN __attribute__((ext_vector_type(N)));
      const int sub = tid & 15;
      for (int c = tid >> 4; c < all; c += 4 * W) {
        // channels sub N .. of the block and of each head: a fused row that took one
        // round has its blocks, and always its heads, in LDS
        const int b = (int)s_row[c];
        bf16xN lo16, hi16;
        constexpr int PER = 8 / N;  // lanes to a 16-byte chunk
        const bool staged = MODE == PICK_FUSED && blocks <= kFusedWaves * 16;
        if constexpr (MODE == PICK_FUSED) {
          if (staged) {
            const u32x4* const rows = s_fused.bounds[b >> 4];
            lo16 = reinterpret_cast<const bf16xN*>(
                rows + chunk_at<D / 4>(b & 15, sub / PER))[sub % PER];
            hi16 = reinterpret_cast<const bf16xN*>(
                rows + chunk_at<D / 4>(b & 15, D / 8 + sub / PER))[sub % PER];
          }
        }
        if (!staged) {
          const bf16xN* const p = reinterpret_cast<const bf16xN*>(bt + (int64_t)b * 2 * D) + sub;
          lo16 = p[0];
          hi16 = p[16];
        }
        const auto lo = __builtin_convertvector(lo16, f64xN);
        const auto hi = __builtin_convertvector(hi16, f64xN);
        Magnitudes m;
        m.add({lo16, hi16});
        float best = over_row(m.most, Most{}) >= kInfinite ? INFINITY : -INFINITY;
        constexpr int HU = 4;  // heads at a time
        for (int h0 = 0; h0 < group; h0 += HU) {
          bf16xN y[HU];
#pragma unroll
          for (int u = 0; u < HU; ++u) {
            const int h = min(h0 + u, group - 1);
            if constexpr (MODE == PICK_FUSED)
              y[u] = reinterpret_cast<const bf16xN*>(
                  s_fused.q + (h & ~15) * (D / 8) + chunk_at<D / 8>(h & 15, sub / PER))[sub % PER];
            else
              y[u] = *reinterpret_cast<const bf16xN*>(qt + h * D + sub * N);
          }
#pragma unroll
          for (int u = 0; u < HU; ++u) {
            const auto z = __builtin_convertvector(y[u], f64xN);
            double x = 0.;
#pragma unroll
            for (int i = 0; i < N; ++i) {
              x = __builtin_fma(z[i] < 0. ? 0. : z[i], hi[i], x);
              x = __builtin_fma(z[i] < 0. ? z[i] : 0., lo[i], x);
            }
            const float s = (float)over_row(x, Sum{});
            best = fmaxf(best, s != s ? INFINITY : s);
          }
        }
        if (sub == 0) s_row[c] = rising(best);
      }
      sync();
      at = mine;
      if (all <= 64) {
        // few: every wave ranks them, one to a lane (they are listed by index, so of
        // equal ones the earlier is the better)
        const uint32_t own = lane < all ? s_row[lane] : 0u;
        int better = 0;
        for (int k = 0; k < all; ++k) {
          const uint32_t x = __builtin_amdgcn_readlane(own, k);
          better += x > own || (x == own && k < lane);
        }
        const uint64_t taken = __ballot(lane < all && better < topk - kept);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const uint64_t vote = __ballot((open >> i) & 1);
          if ((open >> i) & 1) key[i] = (taken >> (at + __popcll(vote & below))) & 1 ? kKept : 0u;
          at += __popcll(vote);
        }
        cut = kKept;
        reach = topk;
      } else {
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const uint64_t vote = __ballot((open >> i) & 1);
          if ((open >> i) & 1) key[i] = s_row[at + __popcll(vote & below)];
          at += __popcll(vote);
        }
        find_cut(kept);
      }
    }
  }

  // All that reach the cut, or all above it and of those equal to it the first ones
  // that still fit.
  const bool every = reach == topk;
  int gt = 0, eq = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    gt += __popcll(__ballot(every ? key[i] >= cut : key[i] > cut));
    eq += __popcll(__ballot(!every && key[i] == cut));
  }
  int gt0 = 0, eq0 = 0, gts = gt;  // before this wave; in all
  if (W > 1) {
    __syncthreads();
    if (lane == 0) {
      s_gt[wave] = gt;
      s_eq[wave] = eq;
    }
    __syncthreads();
    gts = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      gt0 += w < wave ? s_gt[w] : 0;
      eq0 += w < wave ? s_eq[w] : 0;
      gts += s_gt[w];
    }
  }
  const int room = topk - gts;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const bool over = every ? key[i] >= cut : key[i] > cut;
    const bool level = !every && key[i] == cut;
    const uint64_t vg = __ballot(over), ve = __ballot(level);
    const int e = eq0 + __popcll(ve & below);
    const int at = gt0 + __popcll(vg & below) + min(e, room);
    if (over || (level && e < room)) sel[row * topk + at] = i0 + 64 * i;
    gt0 += __popcll(vg);
    eq0 += __popcll(ve);
  }
}

}  // namespace

int launch_key_bounds(const uint16_t* K, int n_shards, int64_t S, int Hkv, int d, int block,
                      uint16_t* bounds, hipStream_t stream) {
  const int64_t blocks = (S + block - 1) / block;
  const int64_t total = n_shards * blocks * (Hkv * d / 8);
  const int64_t nwg = (total + 255) / 256;
  if (!grid_fits(nwg, 256)) return PULSAR_EUNSUPPORTED;
  hipLaunchKernelGGL(key_bounds_kernel, dim3((unsigned)nwg), dim3(256), 0, stream, K, S, Hkv, d,
                     block, (int)blocks, bounds, total);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

int launch_block_scores(const uint16_t* q, const uint16_t* bounds, int n_shards, int Tq, int Hq,
                        int Hkv, int d, int blocks, float* scores, hipStream_t stream) {
  const int group = Hq / Hkv, tokens = std::max(16 / group, 1);
  const int tiles = (Tq + tokens - 1) / tokens;
  const unsigned x = (blocks + 63) / 64, y = n_shards * Hkv;
  const int per = 8;
  const dim3 grid(x, y, (tiles + per - 1) / per);
  const auto kern = d == 128 ? block_scores_kernel<128> : block_scores_kernel<64>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, q, bounds, Tq, Hq, Hkv, blocks, tiles, per,
                     scores);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

int launch_block_near(const uint16_t* q, const uint16_t* bounds, int n_shards, int Tq, int Hq,
                      int Hkv, int d, int blocks, float* near, float* norms, hipStream_t stream) {
  const int group = Hq / Hkv, tokens = std::max(16 / group, 1), passes = (group + 15) / 16;
  const int64_t units = (int64_t)((Tq + tokens - 1) / tokens) * passes;
  // a token's passes stay in one workgroup
  const int per = std::max(kUnitsWg / passes, 1) * passes;
  const int64_t z = (units + per - 1) / per;
  const dim3 grid((blocks + 63) / 64, n_shards * Hkv, (unsigned)z);
  const auto kern = d == 128 ? block_near_kernel<128> : block_near_kernel<64>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, q, bounds, Tq, Hq, Hkv, blocks, (int)units,
                     per, near, norms);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

namespace {
template <int D, int MODE>
int pick(const PickLaunch& a, hipStream_t stream) {
  const auto go = [&](auto kern, int waves) {
    const size_t lds = MODE == PICK_NEAR ? (size_t)a.blocks * 4 : 0;
    if (lds > 32768) {
      if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize,
                              (int)lds) != hipSuccess)
        return (int)PULSAR_EHIP;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.n_shards * a.Tq * a.Hkv)),
                       dim3(64 * waves), lds, stream, a.q, a.bounds, a.scores, a.norms, a.Tq, a.Hq,
                       a.Hkv, a.blocks, a.topk, a.sel);
    return (int)(hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP);
  };
  if constexpr (MODE == PICK_FUSED) {
    return a.blocks <= 128 ? go(block_pick_kernel<D, 1, 2, MODE>, kFusedWaves)
                           : go(block_pick_kernel<D, 1, 8, MODE>, kFusedWaves);
  } else {
    if (a.blocks <= 256) return go(block_pick_kernel<D, 1, 4, MODE>, 1);
    if (a.blocks <= 1024) return go(block_pick_kernel<D, 4, 4, MODE>, 4);
    if (a.blocks <= 4096) return go(block_pick_kernel<D, 8, 8, MODE>, 8);
    if (a.blocks <= 16384) return go(block_pick_kernel<D, 16, 16, MODE>, 16);
    return go(block_pick_kernel<D, 16, 32, MODE>, 16);
  }
}
}  // namespace

int launch_block_pick(const PickLaunch& a, hipStream_t stream) {
  if (a.scores == nullptr)
    return a.d == 128 ? pick<128, PICK_FUSED>(a, stream) : pick<64, PICK_FUSED>(a, stream);
  if (a.norms == nullptr)
    return a.d == 128 ? pick<128, PICK_EXACT>(a, stream) : pick<64, PICK_EXACT>(a, stream);
  return a.d == 128 ? pick<128, PICK_NEAR>(a, stream) : pick<64, PICK_NEAR>(a, stream);
}

// A workgroup per row forms the scores itself where that is one launch of little
// work: few blocks, and few tokens that would each read them again.
bool select_fused(int Tq, int blocks, int group) {
  return blocks <= kFusedBlocks && Tq <= 8 && group <= kFusedHeads;
}
