// Selection of key blocks for block-sparse reads of the retained shards: channel
// bounds of every block of keys, the score that a block's bounds allow, and the
// topk blocks of each shard.
#include <algorithm>

#include "common.hpp"

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
// fp64 (the products are exact, so that equal sums come out equal whatever the
// kernel's order) and rounded once to fp32.  A score that is not a number, as
// from a bound that is not finite, ranks above all: +inf.
//
// A wave takes 16 blocks as the rows of 16x16x4 fp64 matrix products and walks
// over tiles of 16 (token, head) columns.  Lane (r, g) holds channels
// g D/4 .. of its block, so that it loads whole 16-byte pieces; the channels of a
// product are then D/4 apart, the same for both operands.
template <int D>
__global__ __launch_bounds__(256) void block_scores_kernel(
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
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float s = (float)(up[v] + down[v]);
        s = s != s ? INFINITY : s;
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
// The topk largest of a row of scores, in index order; of equal scores the lower
// index.  W waves hold the row as rising integers in registers, R values per lane,
// and bisect the value of the smallest one kept, counting with ballots.
__device__ __forceinline__ uint32_t rising(float s) {
  const uint32_t u = __float_as_uint(s == 0.f ? 0.f : s);  // -0 ranks as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int W, int R>
__global__ __launch_bounds__(64 * W) void block_topk_kernel(const float* __restrict__ scores,
                                                            int blocks, int topk,
                                                            int32_t* __restrict__ sel) {
  __shared__ int s_n[2][W];
  __shared__ int s_gt[W], s_eq[W];
  __shared__ uint32_t s_lo[W], s_hi[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  const float* src = scores + row * blocks;
  const int i0 = wave * (64 * R) + lane;
  uint32_t key[R];  // 0 past the row's end, below every score
  uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = i0 + 64 * i;
    key[i] = at < blocks ? rising(src[at]) : 0u;
    lo = min(lo, at < blocks ? key[i] : 0xffffffffu);
    hi = max(hi, key[i]);
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, x, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, x, 64));
  }
  if (W > 1) {
    if (lane == 0) {
      s_lo[wave] = lo;
      s_hi[wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = min(lo, s_lo[w]);
      hi = max(hi, s_hi[w]);
    }
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  // the largest value that at least topk scores reach
  for (int it = 0; lo < hi; ++it) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) n += __popcll(__ballot(key[i] >= mid));
    if (W > 1) {
      if (lane == 0) s_n[it & 1][wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) n += s_n[it & 1][w];
      n = __builtin_amdgcn_readfirstlane(n);
    }
    if (n >= topk) lo = mid;
    else hi = mid - 1;
    if (n == topk) break;
  }
  // all above it, and of those equal to it the first ones that still fit
  int gt = 0, eq = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    gt += __popcll(__ballot(key[i] > lo));
    eq += __popcll(__ballot(key[i] == lo));
  }
  int gt0 = 0, eq0 = 0, gts = gt;  // before this wave; in all
  if (W > 1) {
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
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const uint64_t vg = __ballot(key[i] > lo), ve = __ballot(key[i] == lo);
    const int e = eq0 + __popcll(ve & below);
    const int at = gt0 + __popcll(vg & below) + min(e, room);
    if (key[i] > lo || (key[i] == lo && e < room)) sel[row * topk + at] = i0 + 64 * i;
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
  if (nwg > 0x7fffffff) return PULSAR_EUNSUPPORTED;
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

int launch_block_topk(const float* scores, int64_t rows, int blocks, int topk, int32_t* sel,
                      hipStream_t stream) {
  const auto go = [&](auto kern, int waves) {
    hipLaunchKernelGGL(kern, dim3((unsigned)rows), dim3(64 * waves), 0, stream, scores, blocks,
                       topk, sel);
    return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
  };
  if (blocks <= 256) return go(block_topk_kernel<1, 4>, 1);
  if (blocks <= 1024) return go(block_topk_kernel<4, 4>, 4);
  if (blocks <= 4096) return go(block_topk_kernel<16, 4>, 16);
  if (blocks <= 16384) return go(block_topk_kernel<16, 16>, 16);
  return go(block_topk_kernel<16, 32>, 16);
}
