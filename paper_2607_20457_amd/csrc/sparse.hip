// Phase-2 attention of new tokens over the blocks of the retained shards that were
// selected for each of them (and KV head), and over the generation shard.
//
// Work.  A token's keys are a list of 16-key halves: the halves of its selected
// blocks in the list's order, then those of the generation shard's rows.  Two
// halves are a 32-key step.  A workgroup of four waves takes one part of the steps
// of one (token, KV head, 16 heads of the group): wave w steps w, w + 4, ... of
// it, on its own; then the four states are merged through LDS.  A step of a wave:
//   K, V  into the wave's LDS stage by loads that write LDS directly, whole rows
//       by neighbouring lanes (K straight into registers, where neighbouring lanes
//       hold different rows, kept the L1 cache busy with 64 accesses a load
//       instead of 16: 128 tokens over 4096 keys each 149 us);
//   S^T = K Q^T (16x16x32): tile h holds half h, row r its key r, so that the
//       scores of a lane are keys 4g .. 4g+3 of both halves, which is how PV takes
//       them in; then O^T += V^T P^T with V read transposed;
//   softmax  online, log2 domain; the reference is raised, O and the sums
//       rescaled, when a step's maximum exceeds it by more than 2^8.  P enters PV
//       rounded to bf16 (2^-8 of each weight at most), O is divided by the sum of
//       those rounded weights, the log-sum-exp uses the fp32 sum.
// The next step's K is sent for once the scores have consumed this one's, its V
// once PV has: each has the time of a step to arrive, with one stage per wave, and
// two waves per SIMD (four at d 64) hide each other's waits.
//
// Where the halves lie is worked out for 32 steps at a time, one half per lane:
// the row, the rows that may be loaded and the rows that the token sees.  A row
// that it does not see is loaded as a copy of one that it does, so that nothing
// a masked row holds can reach the output; a step without any such row is left out.
//
// Heads fill the 16 columns of a tile only where 16 heads share a KV head, but the
// rows read from memory or L2 bound the kernel, not the matrix work.
#include <algorithm>

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
  static constexpr int STAGE = SP_KEYS * D * 2;              // a K or V step
  static constexpr int LOOP = SP_WAVES * 2 * STAGE;
  static constexpr int PITCH = D + 4;                        // floats of a state's column
  static constexpr int MERGE = SP_WAVES * 16 * (PITCH + 3) * 4;
  static constexpr int BYTES = LOOP > MERGE ? LOOP : MERGE;
  static_assert(BYTES <= 65536, "two workgroups per compute unit");
};

template <int D, typename OUT>
__global__ __launch_bounds__(64 * SP_WAVES)
__attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 4, D == 128 ? 2 : 4)))
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
  // Byte offset of the half's first row in K (or Kg), and its rows: those that the
  // token sees (bits 0-15) and those to load (bits 16-31).  A half of which nothing
  // is seen is loaded as its neighbour.
  uint32_t tab_lo = 0, tab_hi = 0, tab_rows = 0;
  auto fill = [&](int base) {
    const int st = step0 + wave + SP_WAVES * (base + (lane >> 1));
    int64_t row = 0;
    uint32_t sees = 0;
    if (st < step1 && st < a.sparse_steps) {
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
          sees = (1u << (int)min((int64_t)16, a.S - at)) - 1;
        }
      }
    } else if (st < step1) {
      const int at = (st - a.sparse_steps) * SP_KEYS + (lane & 1) * 16;
      const int rows = min(16, gen_end - at);
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
    const uint64_t off = (uint64_t)row * row_bytes;
    const uint32_t lo = (uint32_t)off, hi = (uint32_t)(off >> 32);
    const uint32_t n_lo = __shfl_xor((int)lo, 1, 64), n_hi = __shfl_xor((int)hi, 1, 64);
    const uint32_t n_sees = __shfl_xor((int)sees, 1, 64);
    tab_lo = sees ? lo : n_lo;
    tab_hi = sees ? hi : n_hi;
    tab_rows = sees | (sees ? sees : n_sees) << 16;
  };
  struct Half {
    uint32_t sees, load;
    int64_t off;
  };
  auto half = [&](int j, int h) {
    const int at = 2 * (j & 31) + h;
    const uint32_t rows = __builtin_amdgcn_readlane(tab_rows, at);
    return Half{rows & 0xffffu, rows >> 16,
                (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(tab_hi, at) << 32 |
                          (uint32_t)__builtin_amdgcn_readlane(tab_lo, at))};
  };

  // ---- loads of one step --------------------------------------------------------
  // Lane l of segment i fills the 16-byte chunk position (64 i + l) % CPR of row
  // (64 i + l) / CPR of a half with the chunk that its swizzle puts there: for K,
  // so that 16 rows' chunks of one column lie in different banks; for V, so that
  // the 32 bytes that a transposing read takes of each of 8 rows do.
  auto k_swizzle = [](int row) { return CPR == 16 ? row & 15 : (row >> 1) & 7; };
  auto v_swizzle8 = [](int row) { return CPR == 16 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
  constexpr int H_SEGS = L::STAGE / 2048;  // 1 KiB segments of a half
  constexpr int SEG_ROWS = 64 / CPR;
  const int seg_row = lane / CPR;
  uint32_t k_off[H_SEGS], v_off[H_SEGS];  // byte offsets of a lane from segment row 0
#pragma unroll
  for (int i = 0; i < H_SEGS; ++i) {
    const int row = i * SEG_ROWS + seg_row, at = lane % CPR;
    k_off[i] = head_off + seg_row * row_bytes + (uint32_t)(at ^ k_swizzle(row)) * 16u;
    v_off[i] = head_off + seg_row * row_bytes + (uint32_t)(at ^ v_swizzle8(row)) * 16u;
  }
  lds_u8* const k_lds = (lds_u8*)smem + wave * 2 * L::STAGE;
  lds_u8* const v_lds = k_lds + L::STAGE;
  struct Step {
    Half half[2];
    bool gen;
  };
  auto step_at = [&](int j) {
    return Step{{half(j, 0), half(j, 1)}, step0 + wave + SP_WAVES * j >= a.sparse_steps};
  };
  // A row that is not to be loaded is loaded as the first one that is.
  auto issue = [&](const Step& x, const uint16_t* base, lds_u8* lds,
                   const uint32_t (&off)[H_SEGS]) {
    const uint32_t st = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
    const bool whole = (x.half[0].load & x.half[1].load) == 0xffffu;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
          reinterpret_cast<uint8_t*>(const_cast<uint16_t*>(base)) + x.half[h].off, (short)0,
          (int)(16 * row_bytes), kBufferFlags);
      if (whole) {
#pragma unroll
        for (int i = 0; i < H_SEGS; ++i)
          lds_dma16(rsrc, off[i], i * SEG_ROWS * row_bytes, st + (h * H_SEGS + i) * 1024);
      } else {
        const uint32_t load = x.half[h].load;
        const int first = __builtin_ctz(load | 0x10000u) & 15;
#pragma unroll
        for (int i = 0; i < H_SEGS; ++i) {
          const int row = i * SEG_ROWS + seg_row;
          const int from = (load >> row) & 1 ? row : first;
          lds_dma16(rsrc, off[i] + (from - seg_row) * row_bytes, st + (h * H_SEGS + i) * 1024);
        }
      }
    }
  };
  uint32_t k_at[DS];  // chunk 4s + g of row r of a half
#pragma unroll
  for (int s = 0; s < DS; ++s) k_at[s] = (r * CPR + ((4 * s + g) ^ k_swizzle(r))) * 16;
  // V^T rows e*16 .. of the step: lane (r, g) of a transposing read addresses row
  // 4g + r/4 of a half at head_dim 16e + 4 (r%4) and receives head_dim 16e + r of
  // keys 4g .. 4g+3 of it
  uint32_t v_at[DT];
  {
    const int row = 4 * g + (r >> 2), q4 = r & 3;
#pragma unroll
    for (int e = 0; e < DT; ++e)
      v_at[e] = row * (2 * D) + 16 * ((2 * e + (q4 >> 1)) ^ v_swizzle8(row)) + 8 * (q4 & 1);
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

  Step next{};
  if (nsteps > 0) {
    fill(0);
    next = step_at(0);
    issue(next, next.gen ? a.Kg : a.K, k_lds, k_off);
    issue(next, next.gen ? a.Vg : a.V, v_lds, v_off);
  }
  for (int j = 0; j < nsteps; ++j) {
    const uint32_t sees[2] = {next.half[0].sees, next.half[1].sees};
    const bool more = j + 1 < nsteps;
    // K(j) is in LDS once only V(j)'s loads are outstanding
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(V_SEGS) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    f32x4 S[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      S[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < DS; ++s)
        S[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            *reinterpret_cast<const lds_bf16x8*>(k_lds + h * (L::STAGE / 2) + k_at[s]), qf[s],
            S[h], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) {
      if (((j + 1) & 31) == 0) fill(j + 1);
      next = step_at(j + 1);
      issue(next, next.gen ? a.Kg : a.K, k_lds, k_off);
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
    mx = max_of_rows(mx) * c2;
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
    // V(j) is in LDS once only K(j + 1)'s loads are outstanding
    __builtin_amdgcn_sched_barrier(0);
    if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(V_SEGS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if ((sees[0] | sees[1]) != 0) {
#pragma unroll
      for (int e = 0; e < DT; ++e)
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_frag(v_lds, e), P, acc[e], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) issue(next, next.gen ? a.Vg : a.V, v_lds, v_off);
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

// Parts per (token, KV head): enough workgroups for all that the chip holds at
// once (two on each compute unit, four at d 64), at least one step for each wave of
// a workgroup.
static int sparse_target(int d) { return d == 64 ? 1024 : 512; }

int sparse_parts(int Tq, int Hkv, int d, int64_t keys, int64_t gen_rows) {
  const int64_t steps = (keys + SP_KEYS - 1) / SP_KEYS + (gen_rows + SP_KEYS - 1) / SP_KEYS;
  const int64_t most = (steps + SP_WAVES - 1) / SP_WAVES;
  return (int)std::max<int64_t>(1, std::min(sparse_target(d) / ((int64_t)Tq * Hkv), most));
}

// Rows of partials (tokens times parts) of any call of up to Tq tokens.
int64_t sparse_part_rows_most(int Tq, int Hkv, int d) {
  return Tq > 0 ? sparse_target(d) / Hkv : 0;
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
  const auto go = [&](auto kern, size_t lds) {
    hipLaunchKernelGGL(kern, dim3((unsigned)nwg), dim3(64 * SP_WAVES), lds, stream, a);
    return (int)(hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP);
  };
  if (o_bf16)
    return x.d == 128 ? go(sparse_attn_kernel<128, bf16x4>, SpLds<128>::BYTES)
                      : go(sparse_attn_kernel<64, bf16x4>, SpLds<64>::BYTES);
  return x.d == 128 ? go(sparse_attn_kernel<128, f32x4>, SpLds<128>::BYTES)
                    : go(sparse_attn_kernel<64, f32x4>, SpLds<64>::BYTES);
}
