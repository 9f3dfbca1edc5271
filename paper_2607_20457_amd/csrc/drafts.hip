// Drafted tokens in Phase 2: the visibility of a tree of drafts, the merge that
// adds each token's own branch to its partials, and the move of the rows that are
// kept to the front of a generation shard.
#include "common.hpp"

// ---------------------------------------------------------------------------
// Visibility of a tree: row t's bits are t and its ancestors.  parent[t] < t, so a
// walk from t meets falling indices and fills the row's words from the last to the
// first.  One thread per token, the parents in LDS: a step of the walk is one LDS
// read, and a draft's depth is a few steps.
__global__ __launch_bounds__(256) void tree_mask_kernel(const int32_t* __restrict__ parent, int T,
                                                        uint32_t* __restrict__ mask,
                                                        int32_t* __restrict__ depth) {
  extern __shared__ int s_parent[];
  const int last = min(T, (int)(blockIdx.x + 1) * 256);
  for (int i = threadIdx.x; i < last; i += 256) s_parent[i] = parent[i];
  __syncthreads();
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= T) return;
  const int words = (T + 31) / 32;
  uint32_t* const row = mask + (int64_t)t * words;
  int cur = t, deep = -1;
  bool none = false;  // the walk met something that is no parent
  for (int w = words - 1; w >= 0; --w) {
    uint32_t bits = 0;
    while (cur >= 32 * w) {
      bits |= 1u << (cur & 31);
      ++deep;
      const int up = s_parent[cur];
      none |= up >= cur || up < -1;
      cur = none ? -1 : up;
    }
    row[w] = bits;
  }
  if (none)
    for (int w = 0; w < words; ++w) row[w] = 0;
  if (depth) depth[t] = none ? -1 : deep;
}

int launch_tree_mask(const int32_t* parent, int T, uint32_t* mask, int32_t* depth,
                     hipStream_t stream) {
  if (T == 0) return PULSAR_OK;
  hipLaunchKernelGGL(tree_mask_kernel, dim3((T + 255) / 256), dim3(256), (size_t)T * 4, stream,
                     parent, T, mask, depth);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

// ---------------------------------------------------------------------------
// The online-softmax merge of a drafted token's partials, with its own branch
// folded in: a visible draft j is a part of one key, whose log-sum-exp is the
// score q . k_j * scale and whose output is v_j.  A branch is a few rows that
// differ from token to token, so a matrix tile over all drafts would compute
// mostly masked scores and would read rows that a token must not see; here each
// token reads its own rows only.
//
// One workgroup per (token, head).  DL lanes hold four values each of one part's
// or row's head_dim; the PG groups of DL lanes fold parts pg, pg + PG, ... and the
// branch's rows pg, pg + PG, ..., then the groups are folded across lanes and,
// through LDS, across wavefronts.  The drafts are listed THREADS at a time by
// ballots over the token's mask bits.
template <int D, int THREADS, typename OUT>
__global__ __launch_bounds__(THREADS) void tree_merge_kernel(
    const float* __restrict__ o_parts, const float* __restrict__ lse_parts, int H, int Tq, int Hq,
    TreeRows tree, OUT* __restrict__ o, float* __restrict__ lse) {
  constexpr int DL = D / 4;
  constexpr int PG = THREADS / DL;
  constexpr int W = THREADS / 64;
  constexpr int CH = 4;
  __shared__ int s_list[THREADS];
  __shared__ int s_cnt[W];
  __shared__ float s_m[W], s_s[W];
  __shared__ f32x4 s_a[W][DL];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int dv = tid % DL, pg = tid / DL;
  const int64_t row = blockIdx.x;
  const int h = (int)(row % Hq), t = (int)(row / Hq);
  const int kvh = h / (Hq / tree.Hkv);
  const int words = (Tq + 31) / 32;
  const uint32_t* const bits = tree.mask + (int64_t)t * words;

  // The first loads go out together: the mask, the first parts; then, once the mask is
  // there, the group's first row.
  uint32_t word = tid < Tq ? bits[tid >> 5] : 0u;
  const f32x4 q = __builtin_convertvector(
      reinterpret_cast<const bf16x4*>(tree.q + row * D)[dv], f32x4);
  const float* lp = lse_parts + (int64_t)h * Tq + t;
  const f32x4* op = reinterpret_cast<const f32x4*>(o_parts) + row * DL + dv;
  const int64_t ostride = (int64_t)Tq * Hq * DL, lstride = (int64_t)Tq * Hq;
  float l[CH];
  f32x4 v[CH];
  auto load_parts = [&](int p0) {
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      const int p = min(p0 + u * PG, H - 1);  // a part past the last weighs zero
      l[u] = lp[p * lstride];
      v[u] = op[p * ostride];
    }
  };
  if (H > 0) load_parts(pg);

  const int64_t stride = (int64_t)tree.Hkv * D;
  const uint16_t* const Kh = tree.Kd + (int64_t)kvh * D;
  const uint16_t* const Vh = tree.Vd + (int64_t)kvh * D;
  bf16x4 k4 = {}, v4 = {};
  auto load_row = [&](int i) {
    const int64_t off = s_list[i] * stride;
    k4 = reinterpret_cast<const bf16x4*>(Kh + off)[dv];
    v4 = reinterpret_cast<const bf16x4*>(Vh + off)[dv];
  };
  // The drafts from j0 on that the token sees, listed; their number.
  auto list_rows = [&](int j0) {
    const int j = j0 + tid;
    const bool sees = (word >> (j & 31)) & 1u;
    const uint64_t vote = __ballot(sees && j < Tq);
    if (lane == 0) s_cnt[wave] = __popcll(vote);
    __syncthreads();
    int at = 0, n = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      at += w < wave ? s_cnt[w] : 0;
      n += s_cnt[w];
    }
    if ((vote >> lane) & 1) s_list[at + __popcll(vote & ((1ull << lane) - 1))] = j;
    __syncthreads();
    return n;
  };
  int n = list_rows(0);
  if (pg < n) load_row(pg);

  float m = -INFINITY, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = pg; p0 < H; p0 += CH * PG) {
    if (p0 != pg) load_parts(p0);
    float nm = m;
#pragma unroll
    for (int u = 0; u < CH; ++u)
      if (p0 + u * PG < H) nm = fmaxf(nm, l[u]);
    const float use = nm == -INFINITY ? 0.f : nm;  // no key yet: weights 0
    const float alpha = __expf(m - use);
    sum *= alpha;
    acc *= alpha;
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      const bool part = p0 + u * PG < H;
      const float w = part ? __expf(l[u] - use) : 0.f;
      sum += w;
      acc += w * (part ? v[u] : f32x4{0.f, 0.f, 0.f, 0.f});  // (zero would not heed an infinity)
    }
    m = nm;
  }

  for (int j0 = 0; j0 < Tq; j0 += THREADS) {
    if (j0 > 0) {
      __syncthreads();  // the list of the drafts before has been read
      word = j0 + tid < Tq ? bits[(j0 + tid) >> 5] : 0u;
      n = list_rows(j0);
      if (pg < n) load_row(pg);
    }
    for (int i = pg; i < n; i += PG) {
      const f32x4 k = __builtin_convertvector(k4, f32x4), x = __builtin_convertvector(v4, f32x4);
      if (i + PG < n) load_row(i + PG);
      float s = (q[0] * k[0] + q[1] * k[1]) + (q[2] * k[2] + q[3] * k[3]);
#pragma unroll
      for (int lanes = 1; lanes < DL; lanes <<= 1) s += __shfl_xor(s, lanes, 64);
      s *= tree.scale;
      const float nm = fmaxf(m, s);
      const float use = nm == -INFINITY ? 0.f : nm;
      const float alpha = __expf(m - use), w = __expf(s - use);
      sum = sum * alpha + w;
      acc = acc * alpha + w * x;
      m = nm;
    }
  }

#pragma unroll
  for (int off = DL; off < 64; off <<= 1) {
    const float m2 = __shfl_xor(m, off, 64);
    const float nm = fmaxf(m, m2);
    const float use = nm == -INFINITY ? 0.f : nm;
    const float w1 = __expf(m - use), w2 = __expf(m2 - use);
    sum = sum * w1 + __shfl_xor(sum, off, 64) * w2;
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = acc[k] * w1 + __shfl_xor(acc[k], off, 64) * w2;
    m = nm;
  }
  if (lane == 0) {
    s_m[wave] = m;
    s_s[wave] = sum;
  }
  if (lane < DL) s_a[wave][lane] = acc;
  __syncthreads();
  if (tid >= DL) return;
  m = s_m[0];
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, s_m[w]);
  const float use = m == -INFINITY ? 0.f : m;
  sum = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float e = __expf(s_m[w] - use);
    sum += s_s[w] * e;
    acc += s_a[w][tid] * e;
  }
  float ell = -INFINITY;
  if (sum != 0.f) {  // (a NaN score leaves a NaN sum)
    ell = m + __logf(sum);
    acc *= 1.f / sum;
  }
  o[row * DL + dv] = __builtin_convertvector(acc, OUT);
  if (lse && dv == 0) lse[(int64_t)h * Tq + t] = ell;
}

int launch_tree_merge(const float* o_parts, const float* lse_parts, int H, int Tq, int Hq, int d,
                      const TreeRows& tree, void* o, int o_bf16, float* lse, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)Tq * Hq));
  const auto go = [&](auto kern, auto* out) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, o_parts, lse_parts, H, Tq, Hq, tree, out,
                       lse);
    return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
  };
  if (o_bf16)
    return d == 128 ? go(tree_merge_kernel<128, 256, bf16x4>, static_cast<bf16x4*>(o))
                    : go(tree_merge_kernel<64, 256, bf16x4>, static_cast<bf16x4*>(o));
  return d == 128 ? go(tree_merge_kernel<128, 256, f32x4>, static_cast<f32x4*>(o))
                  : go(tree_merge_kernel<64, 256, f32x4>, static_cast<f32x4*>(o));
}

// ---------------------------------------------------------------------------
// Rows G + keep[j] of every layer's K and V moved to G + j, in place.  The list
// rises, so keep[j] >= j: a row is overwritten only by a step that has read it or by
// a later one.  The list ends at its first entry that does not rise or lies past the
// cache; every thread finds the same end.
//
// A few rows (the path of a draft): a thread owns one 16-byte column of one layer and
// moves its rows in the list's order, U loads in flight before their stores.
template <int U>
__global__ __launch_bounds__(64) void kv_compact_kernel(u32x4* __restrict__ K, u32x4* __restrict__ V,
                                                        int64_t layer16, int row16, int64_t G,
                                                        int past, const int32_t* __restrict__ keep,
                                                        int n, int64_t columns) {
  const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x;
  if (i >= columns) return;
  const int64_t layer = i / row16;
  u32x4* const x = (blockIdx.y ? V : K) + layer * layer16 + G * row16 + (i - layer * row16);
  int prev = -1;
  for (int j0 = 0; j0 < n; j0 += U) {
    int from[U];
    u32x4 r[U];
    int live = 0;
    bool ended = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      from[u] = keep[min(j0 + u, n - 1)];
      ended |= j0 + u >= n || from[u] <= prev || from[u] >= past;
      if (!ended) {
        ++live;
        prev = from[u];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < live && from[u] != j0 + u) r[u] = x[(int64_t)from[u] * row16];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < live && from[u] != j0 + u) x[(int64_t)(j0 + u) * row16] = r[u];
    if (live < U) return;
  }
}

// Many rows: a workgroup owns `cols` columns of one layer and moves 1024 / cols * U
// rows at a time, all of them read before any is written (a later batch reads only
// rows past those that this one writes).  Bound by the bytes in flight: 1500 of 4000
// rows in 32 layers, 393 MB, take 872 us with one thread per column.
constexpr int kCompactThreads = 1024;
template <int U>
__global__ __launch_bounds__(kCompactThreads) void kv_compact_many_kernel(
    u32x4* K, u32x4* V, int64_t layer16, int row16, int64_t G, int past,
    const int32_t* __restrict__ keep, int n, int cols, int groups) {
  __shared__ int s_end;
  if (threadIdx.x == 0) s_end = n;
  __syncthreads();
  for (int j = threadIdx.x; j < n; j += kCompactThreads) {
    const int k = keep[j];
    if (k < 0 || k >= past || (j > 0 && k <= keep[j - 1])) {
      atomicMin(&s_end, j);
      break;
    }
  }
  __syncthreads();
  const int end = s_end;
  const int64_t layer = blockIdx.x / groups;
  const int col = (int)(blockIdx.x - layer * groups) * cols + threadIdx.x % cols;
  const int slot = threadIdx.x / cols, slots = kCompactThreads / cols;
  const bool mine = col < row16;
  u32x4* const x =
      (blockIdx.y ? V : K) + layer * layer16 + G * row16 + (mine ? col : 0);
  for (int j0 = 0; j0 < end; j0 += slots * U) {
    int from[U];
    u32x4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * slots + slot;
      from[u] = mine && j < end ? keep[j] : -1;
      if (from[u] == j) from[u] = -1;  // in its place already
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = u32x4{0u, 0u, 0u, 0u};
      if (from[u] >= 0) r[u] = x[(int64_t)from[u] * row16];
    }
    // every load has arrived before any thread stores
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+v"(r[u])::"memory");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (from[u] >= 0) x[(int64_t)(j0 + u * slots + slot) * row16] = r[u];
  }
}

int launch_kv_compact(void* K, void* V, int layers, int64_t capacity, int64_t row_bytes, int64_t G,
                      const int32_t* keep, int n, hipStream_t stream) {
  const int row16 = (int)(row_bytes / 16);
  const int past = (int)(capacity - G < 0x7fffffff ? capacity - G : 0x7fffffff);
  if (n <= 32) {
    const int64_t columns = (int64_t)layers * row16;
    hipLaunchKernelGGL(kv_compact_kernel<16>, dim3((unsigned)((columns + 63) / 64), 2), dim3(64),
                       0, stream, (u32x4*)K, (u32x4*)V, capacity * row16, row16, G, past, keep, n,
                       columns);
  } else {
    // columns in powers of two, no more than leave a workgroup per compute unit,
    // whole 256-byte runs at least
    int cols = kCompactThreads;
    while (cols > 16 && (cols >= 2 * row16 ||
                         (int64_t)2 * layers * ((row16 + cols - 1) / cols) < 256))
      cols /= 2;
    const int groups = (row16 + cols - 1) / cols;
    if (!grid_fits((int64_t)layers * groups, kCompactThreads)) return PULSAR_EUNSUPPORTED;
    hipLaunchKernelGGL(kv_compact_many_kernel<4>, dim3((unsigned)(layers * groups), 2),
                       dim3(kCompactThreads), 0, stream, (u32x4*)K, (u32x4*)V, capacity * row16,
                       row16, G, past, keep, n, cols, groups);
  }
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}
