// Phase-2 attention of new tokens over the blocks of the retained shards that were
// selected for each of them (and KV head), and over the generation shard.
//
// Work.  A token's keys are a list of 16-key halves: the halves of its selected
// blocks in the list's order, then those of the generation shard's rows.  Two
// halves are a 32-key step.  A workgroup of four waves takes one part of the steps
// of one (token, KV head, 16 heads of the group): wave w steps w, w + 4, ... of
// it, on its own; then the four states are merged through LDS.  A step of a wave:
//   K   straight into registers as the A operand of S^T = K Q^T (16x16x32): tile
//       h holds half h, row r its key r, so that the scores of a lane are keys
//       4g .. 4g+3 of both halves, which is how PV takes them in;
//   V   into the wave's LDS double buffer by loads that write LDS directly, read
//       transposed as the A operand of O^T += V^T P^T;
//   softmax  online, log2 domain; the reference is raised, O and the sums
//       rescaled, when a step's maximum exceeds it by more than 2^8.  P enters PV
//       rounded to bf16 (2^-9 of each weight), O is divided by the sum of those
//       rounded weights, the log-sum-exp uses the fp32 sum.
// The next step's K and V are in flight while a step is multiplied.
//
// Where the halves lie is worked out for 32 steps at a time, one half per lane:
// the row, the rows that may be loaded and the rows that the token sees.  A row
// that it does not see is loaded as a copy of one that it does, so that nothing
// a masked row holds can reach the output; a step without any such row is left out.
//
// Heads fill the 16 columns of a tile only where 16 heads share a KV head, but the
// rows read from memory or L2 bound the kernel, not the matrix work.
#include <algorithm>
#include <type_traits>

#include "tiles.hpp"

namespace {

constexpr int SP_WAVES = 4;
constexpr int SP_KEYS = 32;       // keys per step
constexpr float SP_SLACK = 8.0f;  // log2 slack before the reference is raised

struct SparseArgs {
  const uint16_t *q, *K, *V, *Kg, *Vg;
  const int32_t* sel;
  const uint32_t* mask;
  int Tq, Hq, Hkv, group, col_tiles;
  int topk, entries;     // listed blocks per shard; of all shards
  int half_log2;         // log2 of a block's halves
  int blocks;            // blocks per shard
  int gen_rows;          // G + Tq, or 0 without a generation shard
  int64_t S, G;
  int sparse_steps;      // steps of the listed blocks; the generation shard's follow
  int parts, part_steps;
  float scale_log2;
  void* O;               // parts > 1: float [parts, Tq, Hq, D]; else the output
  float* lse;            // [parts, Hq, Tq]; nullable for the output
};

template <int D>
struct SpLds {
  static constexpr int STAGE = SP_KEYS * D * 2;              // a V step
  static constexpr int LOOP = SP_WAVES * 2 * STAGE;
  static constexpr int PITCH = D + 4;                        // floats of a state's column
  static constexpr int MERGE = SP_WAVES * 16 * (PITCH + 3) * 4;
  static constexpr int BYTES = LOOP > MERGE ? LOOP : MERGE;
};

__device__ __forceinline__ int64_t lane_value64(uint32_t lo, uint32_t hi, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, lane) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane(lo, lane));
}

template <int D, typename OUT>
__global__ __launch_bounds__(64 * SP_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2)))
void sparse_attn_kernel(SparseArgs a) {
  using L = SpLds<D>;
  constexpr int CPR = D / 8;               // 16-byte chunks per row
  constexpr int DS = D / 32;               // k-steps of S
  constexpr int DT = D / 16;               // 16-row tiles of O^T
  constexpr int V_SEGS = L::STAGE / 1024;  // 1 KiB segments: one 16-byte load per lane each
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  // workgroup -> (KV head, token, heads, part), the KV head fastest: with eight of
  // them each XCD reads one head's keys
  int64_t wg = blockIdx.x;
  const int kvh = (int)(wg % a.Hkv);
  wg /= a.Hkv;
  const int t = (int)(wg % a.Tq);
  wg /= a.Tq;
  const int tile = (int)(wg % a.col_tiles);
  const int part = (int)(wg / a.col_tiles);
  const int gen_end =
      a.gen_rows == 0 ? 0 : a.mask ? a.gen_rows : (int)(a.G + t + 1);  // rows it may see
  const int total = a.sparse_steps + (gen_end + SP_KEYS - 1) / SP_KEYS;
  const int step0 = part * a.part_steps, step1 = min(step0 + a.part_steps, total);
  const int nsteps = max(0, (step1 - step0 - wave + SP_WAVES - 1) / SP_WAVES);
  const float c2 = a.scale_log2;
  const uint32_t row_bytes = (uint32_t)(a.Hkv * D * 2);
  const uint32_t head_off = (uint32_t)(kvh * D * 2);

  // ---- Q fragments (B operand): column r = head tile * 16 + r of the group ------
  const int col = tile * 16 + r;
  const int head = kvh * a.group + col;
  const bool live = col < a.group;
  bf16x8 qf[DS];
  {
    const bf16x8* src = reinterpret_cast<const bf16x8*>(
                            a.q + ((int64_t)t * a.Hq + (live ? head : 0)) * D) + g;
#pragma unroll
    for (int s = 0; s < DS; ++s) qf[s] = live ? src[4 * s] : bf16x8{};
  }

  // ---- where the halves lie: lane 2i + h, half h of the wave's step base + i -----
  // row: of K (or Kg); info: the rows it sees (16 bits), the last row that may be
  // loaded (4 bits), whether it is the generation shard's; seen: rows to copy from
  uint32_t tab_lo = 0, tab_hi = 0, tab_info = 0;
  auto fill = [&](int base) {
    const int st = step0 + wave + SP_WAVES * (base + (lane >> 1));
    int64_t row = 0;
    int rows = 0;  // loadable rows from `row` on
    uint32_t sees = 0;
    const bool gen = st >= a.sparse_steps;
    if (st < step1 && !gen) {
      const int e = st * 2 + (lane & 1);
      const int entry = e >> a.half_log2;
      if (entry < a.entries) {
        const int shard = entry / a.topk;
        const int b = a.sel[(((int64_t)shard * a.Tq + t) * a.Hkv + kvh) * a.topk +
                            (entry - shard * a.topk)];
        const int64_t at =
            ((int64_t)b << (a.half_log2 + 4)) + ((e & ((1 << a.half_log2) - 1)) << 4);
        if (b >= 0 && b < a.blocks && at < a.S) {
          row = shard * a.S + at;
          rows = (int)min((int64_t)16, a.S - at);
          sees = (1u << rows) - 1;
        }
      }
    } else if (st < step1) {
      const int at = (st - a.sparse_steps) * SP_KEYS + (lane & 1) * 16;
      rows = max(0, min(16, gen_end - at));
      if (rows > 0) {
        row = at;
        sees = (1u << rows) - 1;
        if (a.mask != nullptr && at + rows > a.G) {
          // drafts at - G .. are visible by the token's bits
          const int words = (a.Tq + 31) / 32;
          const uint32_t* bits = a.mask + (int64_t)t * words;
          const int from = (int)(at - a.G);
          uint64_t w;
          if (from < 0) {
            w = ((uint64_t)bits[0] << -from) | ((1u << -from) - 1);
          } else {
            const int i = from >> 5;
            w = (bits[i] | (i + 1 < words ? (uint64_t)bits[i + 1] << 32 : 0)) >> (from & 31);
          }
          sees &= (uint32_t)w;
        }
      }
    }
    // a half of which nothing is seen is loaded as its neighbour
    const uint32_t lo = (uint32_t)row, hi = (uint32_t)((uint64_t)row >> 32);
    const uint32_t n_lo = __shfl_xor((int)lo, 1, 64), n_hi = __shfl_xor((int)hi, 1, 64);
    const uint32_t n_sees = __shfl_xor((int)sees, 1, 64);
    tab_lo = sees ? lo : n_lo;
    tab_hi = sees ? hi : n_hi;
    tab_info = sees | (sees ? sees : n_sees) << 16;
  };
  struct Half {
    uint32_t sees, load;  // rows that count; rows to load from
    int64_t row;
  };
  auto half = [&](int j, int h) {
    const int at = 2 * (j & 31) + h;
    const uint32_t info = __builtin_amdgcn_readlane(tab_info, at);
    return Half{info & 0xffffu, info >> 16, lane_value64(tab_lo, tab_hi, at)};
  };

  // ---- loads of one step --------------------------------------------------------
  auto rsrc_of = [&](const uint16_t* base, int64_t row) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base + row * a.Hkv * D),
                                             (short)0, (int)(16 * row_bytes), kBufferFlags);
  };
  lds_u8* const wave_lds = (lds_u8*)smem + wave * 2 * L::STAGE;
  // row i of a half, or the first one that is seen
  auto seen_row = [](uint32_t load, int i) {
    return (load >> i) & 1 ? i : __builtin_ctz(load | 0x10000u) & 15;
  };
  auto issue = [&](int j, bf16x8 (&kf)[2][DS], int stage) {
    const uint32_t st = __builtin_amdgcn_readfirstlane(
        (uint32_t)(uintptr_t)(wave_lds + stage * L::STAGE));
    const bool gen = step0 + wave + SP_WAVES * j >= a.sparse_steps;
    const uint16_t* const kb = gen ? a.Kg : a.K;
    const uint16_t* const vb = gen ? a.Vg : a.V;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Half x = half(j, h);
      const __amdgpu_buffer_rsrc_t kr = rsrc_of(kb, x.row);
      const uint32_t off = seen_row(x.load, r) * row_bytes + head_off + 16u * g;
#pragma unroll
      for (int s = 0; s < DS; ++s) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b128(kr, off + 64u * s, 0, 0);
        kf[h][s] = __builtin_bit_cast(bf16x8, v);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Half x = half(j, h);
      const __amdgpu_buffer_rsrc_t vr = rsrc_of(vb, x.row);
#pragma unroll
      for (int i = 0; i < V_SEGS / 2; ++i) {
        const int slot = i * 64 + lane;  // chunk slot within the half
        const int row = slot / CPR;
        const int chunk = (slot % CPR) ^ v_swizzle<D>(row);
        lds_dma16(vr, seen_row(x.load, row) * row_bytes + head_off + chunk * 16u,
                  st + (h * (V_SEGS / 2) + i) * 1024);
      }
    }
  };
  // V^T rows e*16 .. of the step: lane (r, g) of a transposing read addresses row
  // 4g + r/4 of a half at head_dim 16e + 4 (r%4) and receives head_dim 16e + r of
  // keys 4g .. 4g+3 of it
  uint32_t v_at[DT];
  {
    const int row = 4 * g + (r >> 2), q4 = r & 3;
#pragma unroll
    for (int e = 0; e < DT; ++e)
      v_at[e] = row * (2 * D) + 16 * ((2 * e + (q4 >> 1)) ^ v_swizzle<D>(row)) + 8 * (q4 & 1);
  }
  auto v_frag = [&](const lds_u8* sV, int e) -> bf16x8 {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(sV + v_at[e]));
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(sV + v_at[e] + 16 * (2 * D)));
    return __builtin_bit_cast(bf16x8,
                              (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
  };

  f32x4 acc[DT];
#pragma unroll
  for (int e = 0; e < DT; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f, lr_run = 0.f;

  bf16x8 kbuf[2][2][DS];
  if (nsteps > 0) {
    fill(0);
    issue(0, kbuf[0], 0);
  }
  // one step; KB = j % 2, a compile-time index into the register buffers
  auto step = [&](int j, auto kb_tag) {
    constexpr int KB = decltype(kb_tag)::value;
    const uint32_t sees[2] = {half(j, 0).sees, half(j, 1).sees};
    f32x4 S[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      S[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < DS; ++s)
        S[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kbuf[KB][h][s], qf[s], S[h], 0, 0, 0);
    }
    const bool more = j + 1 < nsteps;
    if (more) {
      if (((j + 1) & 31) == 0) fill(j + 1);
      issue(j + 1, kbuf[KB ^ 1], KB ^ 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if ((sees[0] & sees[1]) != 0xffffu) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (!((sees[h] >> (4 * g + v)) & 1)) S[h][v] = -INFINITY;
    }
    float mx = S[0][0];
#pragma unroll
    for (int v = 1; v < 8; ++v) mx = fmaxf(mx, S[v >> 2][v & 3]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c2;
    if (__any(mx > m_run + SP_SLACK)) {
      const float m_new = mx > m_run + SP_SLACK ? mx : m_run;
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
      for (int e = 0; e < DT; ++e) acc[e] *= alpha;
      l_run *= alpha;
      lr_run *= alpha;
      m_run = m_new;
    }
    // a column that has seen no key takes its weights against 0: they come out 0
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    bf16x8 P;
    {
      f32x8 p;
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[v >> 2][v & 3], c2, -m_use));
        l_run += p[v];
      }
      P = __builtin_convertvector(p, bf16x8);
#pragma unroll
      for (int v = 0; v < 8; v += 2)
        lr_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{P[v], P[v + 1]}, kOnes2, lr_run, false);
    }
    // V(j) is in LDS once only the loads issued after it are outstanding
    __builtin_amdgcn_sched_barrier(0);
    if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * DS + V_SEGS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if ((sees[0] | sees[1]) != 0) {
      const lds_u8* sV = wave_lds + KB * L::STAGE;
#pragma unroll
      for (int e = 0; e < DT; ++e)
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(sV, e), P, acc[e], 0, 0, 0);
    }
  };
  for (int j = 0; j < nsteps; j += 2) {
    step(j, std::integral_constant<int, 0>{});
    if (j + 1 < nsteps) step(j + 1, std::integral_constant<int, 1>{});
  }

  // ---- the four waves' states, merged through LDS ---------------------------------
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  lr_run += __shfl_xor(lr_run, 16, 64);
  lr_run += __shfl_xor(lr_run, 32, 64);
  __syncthreads();  // every wave is done with its stages
  float* const states = reinterpret_cast<float*>(smem);
  float* const sums = states + SP_WAVES * 16 * L::PITCH;
  {
    float* const mine = states + (wave * 16 + r) * L::PITCH;
#pragma unroll
    for (int e = 0; e < DT; ++e) *reinterpret_cast<f32x4*>(mine + 16 * e + 4 * g) = acc[e];
    if (g == 0) {
      sums[(wave * 16 + r) * 3] = m_run;
      sums[(wave * 16 + r) * 3 + 1] = l_run;
      sums[(wave * 16 + r) * 3 + 2] = lr_run;
    }
  }
  __syncthreads();
  // thread -> (column, four consecutive values), a row of D / 4 threads at a time
  constexpr int DL = D / 4;
  const int dv = threadIdx.x % DL;
  for (int c = threadIdx.x / DL; c < min(16, a.group - tile * 16); c += 64 * SP_WAVES / DL) {
    float m = -INFINITY, l = 0.f, lr = 0.f;
#pragma unroll
    for (int w = 0; w < SP_WAVES; ++w) m = fmaxf(m, sums[(w * 16 + c) * 3]);
    const float use = m == -INFINITY ? 0.f : m;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < SP_WAVES; ++w) {
      const float* x = sums + (w * 16 + c) * 3;
      const float e = __builtin_amdgcn_exp2f(x[0] - use);
      l += e * x[1];
      lr += e * x[2];
      o += e * *reinterpret_cast<const f32x4*>(states + (w * 16 + c) * L::PITCH + 4 * dv);
    }
    o *= lr != 0.f ? 1.f / lr : 0.f;  // (a NaN score leaves a NaN sum)
    const int hd = kvh * a.group + tile * 16 + c;
    const int64_t at = ((int64_t)part * a.Tq + t) * a.Hq + hd;
    static_cast<OUT*>(a.O)[at * DL + dv] = __builtin_convertvector(o, OUT);
    if (dv == 0 && a.lse != nullptr)
      a.lse[((int64_t)part * a.Hq + hd) * a.Tq + t] =
          l != 0.f ? (m + __log2f(l)) * 0.69314718055994531f : -INFINITY;
  }
}

}  // namespace

// Parts per (token, KV head): enough workgroups for two on each compute unit, at
// least one step for each wave of a workgroup.
constexpr int kSparseTarget = 512;

int sparse_parts(int Tq, int Hq, int Hkv, int64_t keys, int64_t gen_rows) {
  const int64_t steps = (keys + SP_KEYS - 1) / SP_KEYS + (gen_rows + SP_KEYS - 1) / SP_KEYS;
  const int64_t wgs = (int64_t)Tq * Hkv;
  const int64_t most = (steps + SP_WAVES - 1) / SP_WAVES;
  return (int)std::max<int64_t>(1, std::min(kSparseTarget / wgs, most));
}

// Rows of partials (tokens times parts) of any call of up to Tq tokens.
int64_t sparse_part_rows_most(int Tq, int Hkv) {
  return std::max<int64_t>(0, std::min<int64_t>((int64_t)Tq * kSparseTarget, kSparseTarget / Hkv));
}

int launch_sparse(const SparseLaunch& x, int parts, void* o, int o_bf16, float* lse,
                  hipStream_t stream) {
  SparseArgs a{};
  a.q = x.q;
  a.K = x.K;
  a.V = x.V;
  a.Kg = x.Kg;
  a.Vg = x.Vg;
  a.sel = x.sel;
  a.mask = x.mask;
  a.Tq = x.Tq;
  a.Hq = x.Hq;
  a.Hkv = x.Hkv;
  a.group = x.Hq / x.Hkv;
  a.col_tiles = (a.group + 15) / 16;
  a.topk = x.topk;
  a.entries = x.S > 0 ? x.n_shards * x.topk : 0;
  a.half_log2 = __builtin_ctz(x.block) - 4;
  a.blocks = (int)((x.S + x.block - 1) / x.block);
  a.gen_rows = x.Kg != nullptr ? (int)(x.G + x.Tq) : 0;
  a.S = x.S;
  a.G = x.G;
  a.sparse_steps = (int)(((int64_t)a.entries * x.block + SP_KEYS - 1) / SP_KEYS);
  const int steps = a.sparse_steps + (a.gen_rows + SP_KEYS - 1) / SP_KEYS;
  a.parts = parts;
  a.part_steps = std::max(1, (steps + parts - 1) / parts);
  a.scale_log2 = x.scale * 1.4426950408889634f;
  a.O = o;
  a.lse = lse;
  const int64_t nwg = (int64_t)a.Hkv * a.Tq * a.col_tiles * parts;
  if (nwg > 0x7fffffff) return PULSAR_EUNSUPPORTED;
  const auto go = [&](auto kern, int lds) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds) !=
        hipSuccess)
      return (int)PULSAR_EHIP;
    hipLaunchKernelGGL(kern, dim3((unsigned)nwg), dim3(64 * SP_WAVES), lds, stream, a);
    return (int)(hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP);
  };
  if (o_bf16)
    return x.d == 128 ? go(sparse_attn_kernel<128, bf16x4>, SpLds<128>::BYTES)
                      : go(sparse_attn_kernel<64, bf16x4>, SpLds<64>::BYTES);
  return x.d == 128 ? go(sparse_attn_kernel<128, f32x4>, SpLds<128>::BYTES)
                    : go(sparse_attn_kernel<64, f32x4>, SpLds<64>::BYTES);
}
