// Phase-2 attention of new tokens over shards held in 8 bits and over the generation
// shard, which is bf16.
//
// Work.  A tile is 16 CG columns of one KV head: column n is head n % group of the
// tile's token n / group (or, of a larger group, 16 CG of one token's heads).  Its
// keys are steps of KEYS rows of a shard, or of KEYS / 2 rows of the generation shard: KEYS
// * D bytes of K and of V either way.  A workgroup takes one part of a tile's steps, wave w
// of NW the steps w, w + NW, ... of it on its own; then the waves' states are merged through
// LDS, and the parts by the log-sum-exp merge.  A step of a wave:
//   K, V  into the wave's LDS stage by loads that write LDS directly: a head's rows
//       are contiguous, so a step is KEYS * D consecutive bytes;
//   S^T = K Q^T (16x16x32), K's codes widened to bf16, which holds them exactly, as
//       they are read: lane (r, g) takes channels D/4 * g .. of row r, so that 16 bytes
//       are two operands; the queries lie in the same order.  Then O^T += V^T P^T, V read
//       transposed in 8 bits and widened;
//   softmax  online, log2 domain.  A step's weights are formed against the reference as it
//       is; only where their sums show a score more than 2^8 above it is the step's maximum
//       looked for, the reference raised and the step weighed again (a maximum in every step
//       made 64 tokens over 16 x 8192 keys 4 % slower, in int8 6 %).  A score is
//       (q . code) * (scale * ks log2 e), one product of the block; the weight that enters PV
//       is exp2(score - reference + log2 vs): V's scale is in it before it is rounded to bf16
//       (2^-8 of each at most), and sums of weights are taken times 1 / vs.  (A scale below
//       2^-32 is multiplied to the rounded weights after their sums: exactly, if it is a power
//       of two.)  O is divided by the sum of the rounded weights, the log-sum-exp uses the fp32
//       sum.
// The next step's K is sent for once the scores have consumed this one's, its V once PV
// has.
//
// What bounds it.  One token: HBM.  16 x 8192 keys of 8 heads of 128 (268 MB of codes) take
// 41 to 44 us and the merge 4: 6.3 TB/s, where a read alone reaches 6.5.  Many tokens: the
// issue of instructions, one kind after another.  64 tokens over the same keys take 180 to 188
// us with the merge (0.73 to 0.76 PFLOP/s).  A step of 64 keys and 32 columns has 64 matrix
// instructions, and beside them 128 that widen codes and five for each of a lane's 32 scores, one
// of them an exponential of four times the others' length.  Counted over the call, of a SIMD's
// cycles matrix instructions take 31 %, vector ones 47 %, scalar ones 13 %; a vector one runs
// beside 29 % of the matrix cycles only.  int8 codes take three instructions to widen a pair, not
// one: vector ones take 58 % of the cycles and matrix ones 23 (236 us).  Tried there and no
// faster: three waves to a SIMD, key and value stages shared by two or four waves, 64 columns a
// wave with one wave to a SIMD (a third slower).  e4m3 codes in the matrix unit as they are, q in
// two e4m3 parts, leave the scores less than fp32's precision: a log-sum-exp was 5e-3 off.
//
// What must not be seen.  Rows from a shard's live length on are not loaded (a copy of
// the step's last live row is) and score -inf; their scales are not read.  Of the new
// tokens' own rows, which only some columns see, unseen ones score -inf; where V holds a
// NaN or an infinity among them, the product is taken key by key, each key's only into the
// columns that see it.
#include <algorithm>
#include <type_traits>

#include "tiles.hpp"

namespace {

constexpr float QA_SLACK = 8.0f;      // log2 slack before the reference is raised
constexpr float QA_OVER = 4 * 0x1p8f; // a lane's four weights of 2^QA_SLACK
constexpr float QA_LEAST = 0x1p-100f; // a smaller scale counts as this
constexpr float QA_SMALL = 0x1p-32f;  // scales of V that weights get after their sums
constexpr float QA_BIG = 0x1p64f;     // above it scales of V have weights with QA_ROOM
constexpr float QA_MOST = 0x1p124f;   // larger ones make their block no number
// Values near the largest number leave fp32 in a sum of theirs, though not in their average,
// which O is.  Steps with such values keep their weights at 2^-QA_ROOM or less, the reference
// that far above the scores: 2^32 of them, more than a call has keys, sum to half a value.
// (Not so in all steps: products of small values would fall below 2^-126.)
constexpr float QA_ROOM = 33.0f;

struct QuantAttnArgs {
  const uint16_t* q;
  const uint8_t *K, *V;    // [n_shards, Hkv, S, D]
  const float *ks, *vs;    // [n_shards, Hkv, blocks]
  const int32_t* rows;     // [n_shards] live rows, or NULL: S
  const uint16_t *Kg, *Vg; // bf16 [G + Tq, Hkv, D], or NULL
  const uint32_t* mask;    // [Tq, ceil(Tq / 32)], or NULL for index-causal
  int Tq, Hq, Hkv, group;
  int tile_tokens, token_tiles, col_tiles, slices;
  int n_shards, S, blocks, block_log2;
  int gen_rows;            // G + Tq, or 0
  int G;
  int shard_steps;         // of a shard of S rows
  int parts;
  float scale_log2;
  int o_bf16;
  void* O;                 // parts > 1: float [parts, Tq, Hq, D]; else the output
  float* lse;              // [parts, Hq, Tq]; nullable for the output
};

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

template <int D, int NW, int KEYS>
struct QaLds {
  static constexpr int STAGE = KEYS * D;     // a K or V step
  static constexpr int LOOP = NW * 2 * STAGE;
  static constexpr int PITCH = D + 4;        // floats of a state's column
  static constexpr int MERGE = NW * 16 * (PITCH + 3) * 4;
  static constexpr int REUSED = LOOP > MERGE ? LOOP : MERGE;
  // with lengths: the steps before each shard
  static constexpr int STEPS = (kMaxQuantShards + 1) * 4 + NW * 4;
};

// lds_dma16, its scalars possibly fresh from a vector instruction (a lane read, or a spilled
// register taken back): five wait states lie between those and a load, which the compiler
// does not count before asm.
template <bool ONCE = false>  // (of what nobody reads again: kept out of the way in the caches)
__device__ __forceinline__ void lds_load16(__amdgpu_buffer_rsrc_t rsrc, uint32_t voffset,
                                           uint32_t soffset, uint32_t lds_base) {
  if constexpr (ONCE)
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen nt lds"
                 :
                 : "v"(voffset), "s"(rsrc), "s"(soffset), "{m0}"(lds_base)
                 : "memory");
  else
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                 :
                 : "v"(voffset), "s"(rsrc), "s"(soffset), "{m0}"(lds_base)
                 : "memory");
}

// Eight codes (two dwords) as bf16, exactly.
template <int FORMAT>
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
  if constexpr (FORMAT == PULSAR_KV_E4M3) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  } else {
    f32x8 y;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      y[b] = (float)((int)(lo << (24 - 8 * b)) >> 24);
      y[4 + b] = (float)((int)(hi << (24 - 8 * b)) >> 24);
    }
    return __builtin_convertvector(y, bf16x8);
  }
}

template <int D, int FORMAT, int NW, int KEYS, int CG>
__global__ __launch_bounds__(64 * NW)
__attribute__((amdgpu_waves_per_eu(CG == 1 || D == 64 ? 4 : 2, CG == 1 || D == 64 ? 4 : 2)))
void quant_attn_kernel(QuantAttnArgs a) {
  using L = QaLds<D, NW, KEYS>;
  constexpr int HALVES = KEYS / 16;       // of a step, 16 rows each
  constexpr int GEN = KEYS / 2;           // rows of the generation shard per step
  constexpr int AT_A_TIME = 64 / HALVES;  // steps that a table of one entry per lane holds
  constexpr int COLS = 16 * CG;           // of a tile
  constexpr int CPR = D / 16;             // 16-byte chunks of a row of codes
  constexpr int GCPR = D / 8;             // of a bf16 row
  constexpr int DS = D / 32;              // k-steps of S
  constexpr int DT = D / 16;              // 16-row tiles of O^T
  constexpr int SEGS = L::STAGE / 1024;   // 1 KiB segments: one 16-byte load per lane each
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  // Workgroup -> tile of a (KV head, part): all tiles of one head's part, which read the
  // same keys, go to one XCD, one after another (few such parts: to `slices` of them).
  // (all of them fit 32 bits, as the workgroups of a launch do)
  const uint32_t tiles = a.token_tiles * a.col_tiles, deep = (tiles + a.slices - 1) / a.slices;
  const uint32_t wg = blockIdx.x >> 3;
  const uint32_t row = wg / deep, unit = row * 8 + (blockIdx.x & 7);
  const uint32_t pair = unit / a.slices;
  const int tile = (int)((wg - row * deep) * a.slices + (unit - pair * a.slices));
  if (pair >= (uint32_t)a.Hkv * a.parts || tile >= (int)tiles) return;
  const int part = (int)(pair / a.Hkv), kvh = (int)(pair - part * a.Hkv);
  const int t0 = tile % a.token_tiles * a.tile_tokens;
  const int heads0 = tile / a.token_tiles * COLS;
  const int tokens = min(a.tile_tokens, a.Tq - t0);
  const int cols = a.col_tiles > 1 ? min(COLS, a.group - heads0) : tokens * a.group;
  const float c2 = a.scale_log2;

  // ---- the tile's steps: those of the shards' live rows, then the generation shard's --
  int* const before = reinterpret_cast<int*>(smem + L::REUSED);  // [n_shards + 1]
  int list_steps = a.n_shards * a.shard_steps;
  auto live_rows = [&](int shard) { return min(max(a.rows[shard], 0), a.S); };
  if (a.rows != nullptr) {
    int* const sums = before + kMaxQuantShards + 1;
    int total = 0;
    for (int i0 = 0; i0 < a.n_shards; i0 += 64 * NW) {
      const int i = i0 + tid;
      const int steps = i < a.n_shards ? (live_rows(i) + KEYS - 1) / KEYS : 0;
      const int excl = wave_excl_scan(steps);
      if (lane == 63) sums[wave] = excl + steps;
      __syncthreads();
      int at = total + excl;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        at += w < wave ? sums[w] : 0;
        total += sums[w];
      }
      if (i < a.n_shards) before[i] = at;
      __syncthreads();
    }
    list_steps = __builtin_amdgcn_readfirstlane(total);
  }
  const int gen_end = a.gen_rows == 0 ? 0 : a.mask != nullptr ? a.gen_rows : a.G + t0 + tokens;
  const int total = list_steps + (gen_end + GEN - 1) / GEN;
  // (the first `more` parts take one step more than the others)
  const int per_part = total / a.parts, more = total - per_part * a.parts;
  const int step0 = __builtin_amdgcn_readfirstlane(part * per_part + min(part, more));
  const int step1 = __builtin_amdgcn_readfirstlane(step0 + per_part + (part < more ? 1 : 0));
  // Wave w takes the steps w, w + NW, ... of them, its last ones of the generation shard.
  auto of_wave = [&](int steps) { return max(0, (steps - wave + NW - 1) / NW); };
  const int nsteps = of_wave(step1 - step0);
  const int code_steps = of_wave(min(step1, list_steps) - step0);

  // The rows at .. at + GEN - 1 of the generation shard that token `token` sees.
  auto gen_sees = [&](int at, int token) -> uint32_t {
    const int end = a.mask != nullptr ? a.gen_rows : a.G + token + 1;
    const int rows = end - at;
    if (rows <= 0) return 0u;
    uint32_t sees = rows >= 32 ? 0xffffffffu : (1u << rows) - 1;
    if (a.mask != nullptr && at + GEN > a.G) {
      // drafts at - G .. are visible by the token's bits
      const int words = (a.Tq + 31) / 32;
      const uint32_t* bits = a.mask + (int64_t)token * words;
      const int from = at - a.G;
      uint64_t w;
      if (from < 0) {
        w = ((uint64_t)bits[0] << -from) | ((1u << -from) - 1);
      } else {
        const int i = from >> 5;
        w = (bits[i] | (i + 1 < words ? (uint64_t)bits[i + 1] << 32 : 0)) >> (from & 31);
      }
      sees &= (uint32_t)w;
    }
    return sees;
  };

  // ---- where the steps lie: lane HALVES i + h, half h of the wave's step base + i --
  struct Place {
    uint64_t off;  // of the step's first row in K (or Kg), in bytes
    int rows;      // of the step
    int64_t scale; // where the half's scales are, or -1
  };
  auto place = [&](int base) {
    const int st = step0 + wave + NW * (base + lane / HALVES);
    Place x{0, 0, -1};
    if (st < step1 && st < list_steps) {
      int shard, first, end = a.S;
      if (a.rows == nullptr) {
        shard = st / a.shard_steps;
        first = st - shard * a.shard_steps;
      } else {
        // the last shard with no more than st steps before it
        int lo = 0, hi = a.n_shards;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (before[mid] <= st) lo = mid;
          else hi = mid;
        }
        shard = lo;
        first = st - before[lo];
        end = live_rows(shard);
      }
      const int row = first * KEYS;
      const int64_t plane = (int64_t)shard * a.Hkv + kvh;
      // (one at least, also of a shard that somebody shortens meanwhile: in its capacity still)
      x.rows = max(1, min(KEYS, end - row));
      x.off = (uint64_t)(plane * a.S + row) * D;
      x.scale = plane * a.blocks + ((row + min(16 * (lane % HALVES), x.rows - 1)) >> a.block_log2);
    } else if (st < step1) {
      const int row = (st - list_steps) * GEN;
      x.rows = min(GEN, gen_end - row);
      x.off = ((uint64_t)row * a.Hkv + kvh) * (2 * D);
    }
    return x;
  };
  // What is needed to send for a step ...
  uint32_t tab_lo = 0, tab_hi = 0;
  int tab_send = 0;
  auto fill_send = [&](const Place& x) {
    tab_lo = (uint32_t)x.off;
    tab_hi = (uint32_t)(x.off >> 32);
    tab_send = x.rows;
  };
  // ... and to multiply it: its rows and what the half's scales come to, the factor of its
  // scores, log2 vs and 1 / vs.  A vs below QA_SMALL counts as 1 there, and weights are
  // multiplied by it after their sums: with vs in it, 2^-100 in a block of zeros, a weight below
  // 2^-26 would be 0 and its key missing from the sums.
  int tab_rows = 0;
  float tab_ck = c2, tab_lv = 0.f, tab_iv = 1.f, tab_vs = 1.f;
  // halves whose vs is no number or above QA_MOST, above QA_BIG, and below QA_SMALL
  uint64_t nan_v = 0, big_v = 0, small_v = 0;
  auto fill_use = [&](const Place& x) {
    tab_rows = x.rows;
    tab_ck = c2;
    tab_lv = 0.f;
    tab_iv = 1.f;
    tab_vs = 1.f;
    bool bad = false, big = false, small = false;
    if (x.scale >= 0) {
      float k = a.ks[x.scale], v = a.vs[x.scale];
      k = k < QA_LEAST ? QA_LEAST : k;
      v = v < QA_LEAST ? QA_LEAST : v;
      bad = !(v <= QA_MOST);
      // (a factor of zero would make -inf a NaN)
      k *= c2;
      tab_ck = k < 0x1p-126f ? 0x1p-126f : k;
      big = v > QA_BIG;
      small = v < QA_SMALL;
      tab_lv = bad || small ? 0.f : __log2f(v);
      tab_iv = bad || small ? 1.f : 1.f / v;
      tab_vs = small ? v : 1.f;
    }
    nan_v = __ballot(bad);
    big_v = __ballot(big);
    small_v = __ballot(small);
  };
  auto lane_f = [&](float x, int at) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), at));
  };

  // ---- loads of one step ------------------------------------------------------------
  // Lane l of segment i fills the 16-byte chunk position (64 i + l) % CPR of row
  // (64 i + l) / CPR with the chunk that its swizzle puts there: for K, so that 16 rows'
  // chunks of one column lie in different banks; for V, so that the 16 bytes that a
  // transposing read takes of each of 16 rows do.
  auto k_swizzle = [](int row) { return CPR == 8 ? (row >> 1) & 7 : (row >> 2) & 3; };
  auto v_swizzle = [](int row) {
    return CPR == 8 ? ((row >> 1) & 3) | ((row >> 2) & 4) : ((row >> 2) & 1) | ((row >> 3) & 2);
  };
  auto gk_swizzle = [](int row) { return GCPR == 16 ? row & 15 : (row >> 1) & 7; };
  auto gv_swizzle = [](int row) { return GCPR == 16 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
  lds_u8* const k_lds = (lds_u8*)smem + wave * 2 * L::STAGE;
  lds_u8* const v_lds = k_lds + L::STAGE;
  const uint32_t gen_row = (uint32_t)(a.Hkv * D * 2);
  // byte offsets of a lane from a whole step's segment 0
  const uint32_t k_off = (lane / CPR) * D + ((lane % CPR) ^ k_swizzle(lane / CPR)) * 16;
  const uint32_t v_off = (lane / CPR) * D + ((lane % CPR) ^ v_swizzle(lane / CPR)) * 16;
  // K (or V) of the wave's step j into its stage.
  auto send = [&](int j, bool is_v) {
    const int at = HALVES * (j % AT_A_TIME);
    const uint32_t off_lo = (uint32_t)__builtin_amdgcn_readlane((int)tab_lo, at);
    const uint32_t off_hi = (uint32_t)__builtin_amdgcn_readlane((int)tab_hi, at);
    const int rows = __builtin_amdgcn_readlane(tab_send, at);
    const int64_t off = (int64_t)((uint64_t)off_hi << 32 | off_lo);
    const uint32_t st = __builtin_amdgcn_readfirstlane(
        (uint32_t)(uintptr_t)(is_v ? v_lds : k_lds));
    int l = lane;  // (computed anew at each step: kept, the offsets do not fit the registers)
    if (__builtin_amdgcn_readfirstlane(step0 + wave + NW * j < list_steps)) {
      const uint8_t* base = (is_v ? a.V : a.K) + off;
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(base), (short)0, rows * D, kBufferFlags);
      constexpr int kRows = 64 / CPR;
      // a whole step: the swizzles of rows 64 / CPR apart differ in one bit
      auto whole = [&](auto once) {
#pragma unroll
        for (int i = 0; i < SEGS; ++i) {
          const int row = i * kRows;
          const uint32_t flip = 16 * (is_v ? v_swizzle(row & 31) : k_swizzle(row & 15));
          lds_load16<decltype(once)::value>(rsrc, (is_v ? v_off : k_off) ^ flip, i * 1024,
                                            st + i * 1024);
        }
      };
      if (KEYS == 32 && rows == KEYS && tiles == 1) {  // (64 rows: more tiles than one)
        whole(std::true_type{});
      } else if (rows == KEYS) {
        whole(std::false_type{});
      } else {
        asm volatile("" : "+v"(l));
#pragma unroll
        for (int i = 0; i < SEGS; ++i) {
          const int row = i * kRows + l / CPR;
          const int chunk = (l % CPR) ^ (is_v ? v_swizzle(row & 31) : k_swizzle(row & 15));
          lds_load16(rsrc, (uint32_t)(min(row, rows - 1) * D + chunk * 16), 0,
                     st + i * 1024);
        }
      }
    } else {
      const uint8_t* base = reinterpret_cast<const uint8_t*>(is_v ? a.Vg : a.Kg) + off;
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(base), (short)0, (int)((rows - 1) * gen_row + 2 * D), kBufferFlags);
      asm volatile("" : "+v"(l));
#pragma unroll
      for (int i = 0; i < SEGS; ++i) {
        const int row = i * (64 / GCPR) + l / GCPR;
        const int chunk = (l % GCPR) ^ (is_v ? gv_swizzle(row & 15) : gk_swizzle(row & 15));
        lds_load16(rsrc, (uint32_t)min(row, rows - 1) * gen_row + chunk * 16, 0,
                   st + i * 1024);
      }
    }
  };

  // ---- operands out of LDS ------------------------------------------------------------
  // K: channels D/4 * g .. of row r of a half; V^T: keys 16 h + 4 g + v (slot 4 h + v) of a
  // 32-row tile, at head_dim 16 e + r.  A transposing read of 8 bits hands lane i of 16, for
  // slot j, byte i % 8 of the eight that lane 2 j + i / 8 addressed.
  // (In the generation shard's steps their addresses are computed anew from `at`, a lane's number
  // that the compiler does not know to be the same in each step: kept beside those of the steps of
  // codes, they do not fit the registers.)
  auto fresh_lane = [&]() {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };
  auto k_codes = [&](int at, int h, int i) -> u32x4 {  // 16 of them
    const int row = at & 15, chunk = (CPR == 8 ? 2 * (at >> 4) + i : at >> 4) ^ k_swizzle(row);
    return *reinterpret_cast<const lds_u32x4*>(k_lds + row * D + chunk * 16 + 16 * h * D);
  };
  auto k_gen = [&](int at, int h, int s) -> bf16x8 {
    const int row = at & 15, chunk = (DS * (at >> 4) + s) ^ gk_swizzle(row);
    return *reinterpret_cast<const lds_bf16x8*>(k_lds + row * (2 * D) + chunk * 16 +
                                                16 * h * (2 * D));
  };
  auto v_codes = [&](int at, int u, int e) -> bf16x8 {
    const int j = (at >> 1) & 7, row = 16 * (j >> 2) + 4 * (at >> 4) + (j & 3);
    const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (lds_i32x2*)(v_lds + row * D + (e ^ v_swizzle(row)) * 16 + 8 * (at & 1) + 32 * u * D));
    return widen<FORMAT>((uint32_t)x[0], (uint32_t)x[1]);
  };
  auto v_gen = [&](int at, int e) -> bf16x8 {
    const int row = 4 * (at >> 4) + ((at >> 2) & 3), q4 = at & 3;
    const lds_u8* from =
        v_lds + row * (2 * D) + 16 * ((2 * e + (q4 >> 1)) ^ gv_swizzle(row)) + 8 * (q4 & 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)from);
    const s16x4 hi =
        GEN == 32 ? __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 16 * (2 * D)))
                  : s16x4{0, 0, 0, 0};
    return __builtin_bit_cast(bf16x8,
                              (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
  };

  f32x4 acc[CG][DT];
  float m_run[CG], l_run[CG], lr_run[CG];
#pragma unroll
  for (int c = 0; c < CG; ++c) {
#pragma unroll
    for (int e = 0; e < DT; ++e) acc[c][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[c] = -INFINITY;
    l_run[c] = lr_run[c] = 0.f;
  }
  // The reference of every group against mx, the largest of a lane's scores of it: where these
  // are above it by more than `slack`, it is raised to `above` more than they are, O and the sums
  // rescaled.
  bool unset = true;  // columns without a reference (the same in all lanes)
  auto raise = [&](const float* mx, float slack, float above) {
    bool any = false;
#pragma unroll
    for (int c = 0; c < CG; ++c) any |= mx[c] > m_run[c] + slack;
    if (!__any(any)) return;
#pragma unroll
    for (int c = 0; c < CG; ++c) {
      const float top = max_of_rows(mx[c]);
      const float m_new = top > m_run[c] + slack ? top + above : m_run[c];
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[c] - m_new);
#pragma unroll
      for (int e = 0; e < DT; ++e) acc[c][e] *= alpha;
      l_run[c] *= alpha;
      lr_run[c] *= alpha;
      m_run[c] = m_new;
    }
    bool still = false;
#pragma unroll
    for (int c = 0; c < CG; ++c) still |= m_run[c] == -INFINITY;
    unset = __any(still);
  };
  // Weights of two halves of group c as PV takes them in; their sums are added to l and lr.
  auto weigh = [&](int c, const f32x4* S, const float* ck, const float* lv, const float* iv,
                   float& l, float& lr) {
    // a column that has seen no key takes its weights against 0: they come out 0
    const float m_use = m_run[c] == -INFINITY ? 0.f : m_run[c];
    f32x8 p;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        p[4 * h + v] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[h][v], ck[h], lv[h] - m_use));
      const float sum = (p[4 * h] + p[4 * h + 1]) + (p[4 * h + 2] + p[4 * h + 3]);
      l = __builtin_fmaf(sum, iv[h], l);
    }
    const bf16x8 P = __builtin_convertvector(p, bf16x8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{P[4 * h], P[4 * h + 1]}, kOnes2, 0.f,
                                                  false);
      sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{P[4 * h + 2], P[4 * h + 3]}, kOnes2, sum,
                                            false);
      lr = __builtin_fmaf(sum, iv[h], lr);
    }
    return P;
  };
  auto largest = [](f32x4 x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); };

  const Place first = place(0);
  fill_send(first);
  if (nsteps > 0) {
    send(0, false);
    send(0, true);
  }

  // ---- Q fragments (B operand): column 16 c + r, channels D/4 * g + 8 s .. ----
  // (columns past the tile's are its first one again: loads without a branch around each, where
  // the compiler waits for all before; 1 token over 4 x 1021 keys 0.3 us)
  int t[CG];
  bf16x8 qf[CG][DS];
  {
#pragma unroll
    for (int c = 0; c < CG; ++c) {
      const int n = 16 * c + r;
      const bool live = n < cols;
      const int tl = live && a.col_tiles == 1 ? n / a.group : 0;
      t[c] = t0 + tl;
      const int head = kvh * a.group + heads0 + (live ? n - tl * a.group : 0);
      const bf16x8* src =
          reinterpret_cast<const bf16x8*>(a.q + ((int64_t)t[c] * a.Hq + head) * D) + DS * g;
#pragma unroll
      for (int s = 0; s < DS; ++s) qf[c][s] = src[s];
    }
  }
  fill_use(first);
  // (Q is there: else the compiler waits for it in every step, and so for all loads before)
#pragma unroll
  for (int c = 0; c < CG; ++c)
#pragma unroll
    for (int s = 0; s < DS; ++s) asm volatile("" : "+v"(qf[c][s]));

  // A wave has one stage: K of step j + 1 is sent for once the scores have consumed this
  // one's, its V once PV has.
  auto need_k = [&]() {
    // K(j) is in LDS once only V(j)'s loads are outstanding
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(SEGS) : "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto scored = [&](int j) {
    __builtin_amdgcn_sched_barrier(0);
    if (j + 1 < nsteps) {
      if ((j + 1) % AT_A_TIME == 0) fill_send(place(j + 1));
      send(j + 1, false);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // V(j) is in LDS once only K(j + 1)'s loads are outstanding, if these have been sent for
  auto need_v = [&](bool sent) {
    __builtin_amdgcn_sched_barrier(0);
    if (sent) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(SEGS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto done = [&](int j) {
    __builtin_amdgcn_sched_barrier(0);
    if (j + 1 < nsteps) send(j + 1, true);
  };

  // ---- the wave's steps of codes ----------------------------------------------------
  int j = 0;
  for (; j < code_steps; ++j) {
    if (j > 0 && j % AT_A_TIME == 0) fill_use(place(j));
    const int at = HALVES * (j % AT_A_TIME);
    const int rows = __builtin_amdgcn_readlane(tab_rows, at);
    float ck[HALVES], lv[HALVES], iv[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      ck[h] = lane_f(tab_ck, at + h);
      lv[h] = lane_f(tab_lv, at + h);
      iv[h] = lane_f(tab_iv, at + h);
    }
    const uint32_t bad_v = (uint32_t)(nan_v >> at) & ((1u << HALVES) - 1);
    const bool big = (big_v >> at & ((1u << HALVES) - 1)) != 0;
    const bool small = (small_v >> at & ((1u << HALVES) - 1)) != 0;
    need_k();
    // (a wave at its matrix products goes before one at its weights: 64 tokens over 16 x 8192
    // keys 4 % faster, in int8 7 %)
    __builtin_amdgcn_s_setprio(1);
    f32x4 S[CG][HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
#pragma unroll
      for (int c = 0; c < CG; ++c) S[c][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DS / 2; ++i) {
        const u32x4 w = k_codes(lane, h, i);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const bf16x8 k = widen<FORMAT>(w[2 * s], w[2 * s + 1]);
#pragma unroll
          for (int c = 0; c < CG; ++c)
            S[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[c][2 * i + s], S[c][h], 0, 0,
                                                              0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    scored(j);
    if (rows < KEYS) {
#pragma unroll
      for (int c = 0; c < CG; ++c)
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (16 * h + 4 * g + v >= rows) S[c][h][v] = -INFINITY;
    }
    // The weights against the reference as it is; if a lane's sum shows that a score is above
    // it by more than QA_SLACK (or where there is none yet), the step's maximum is looked for,
    // the reference raised and they are formed again.
    bf16x8 P[CG][HALVES / 2];
    float l[CG], lr[CG];
    for (bool raised = unset || big;; raised = true) {
      if (raised) {
        float mx[CG];
#pragma unroll
        for (int c = 0; c < CG; ++c) {
          mx[c] = -INFINITY;
#pragma unroll
          for (int h = 0; h < HALVES; ++h) mx[c] = fmaxf(mx[c], largest(S[c][h]) * ck[h]);
        }
        raise(mx, big ? -QA_ROOM : QA_SLACK, big ? QA_ROOM + QA_SLACK : 0.f);
      }
      bool over = false;
#pragma unroll
      for (int c = 0; c < CG; ++c) {
        l[c] = lr[c] = 0.f;
#pragma unroll
        for (int u = 0; u < HALVES / 2; ++u)
          P[c][u] = weigh(c, S[c] + 2 * u, ck + 2 * u, lv + 2 * u, iv + 2 * u, l[c], lr[c]);
        over |= l[c] > QA_OVER * HALVES;
      }
      if (raised || !__any(over)) break;
    }
#pragma unroll
    for (int c = 0; c < CG; ++c) l_run[c] += l[c], lr_run[c] += lr[c];
    if (small) {
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        const float vs = lane_f(tab_vs, at + h);
#pragma unroll
        for (int c = 0; c < CG; ++c)
#pragma unroll
          for (int v = 4 * (h & 1); v < 4 * (h & 1) + 4; ++v)
            P[c][h / 2][v] = (__bf16)((float)P[c][h / 2][v] * vs);
      }
    }
    need_v(j + 1 < nsteps);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < HALVES / 2; ++u)
#pragma unroll
      for (int e = 0; e < DT; ++e) {
        const bf16x8 v = v_codes(lane, u, e);
#pragma unroll
        for (int c = 0; c < CG; ++c)
          acc[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[c][u], acc[c][e], 0, 0, 0);
      }
    __builtin_amdgcn_s_setprio(0);
    if (bad_v != 0) {
      // values that are not numbers, in blocks that every column sees
#pragma unroll
      for (int c = 0; c < CG; ++c)
#pragma unroll
        for (int e = 0; e < DT; ++e) acc[c][e] = f32x4{} + __builtin_nanf("");
    }
    done(j);
  }

  // ---- those of the generation shard --------------------------------------------------
  for (; j < nsteps; ++j) {
    const int st = step0 + wave + NW * j;
    const int row0 = (st - list_steps) * GEN;
    const int la = fresh_lane();
    need_k();
    f32x4 S[CG][2];
#pragma unroll
    for (int c = 0; c < CG; ++c)
      S[c][0] = f32x4{0.f, 0.f, 0.f, 0.f},
      S[c][1] = f32x4{} + (GEN == 32 ? 0.f : -INFINITY);
#pragma unroll
    for (int h = 0; h < GEN / 16; ++h)
#pragma unroll
      for (int s = 0; s < DS; ++s) {
        const bf16x8 k = k_gen(la, h, s);
#pragma unroll
        for (int c = 0; c < CG; ++c)
          S[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[c][s], S[c][h], 0, 0, 0);
      }
    scored(j);
    const bool some = row0 + GEN > a.G;  // rows that only some columns see
    uint32_t vis[CG];
    float mx[CG];
#pragma unroll
    for (int c = 0; c < CG; ++c) {
      vis[c] = some ? gen_sees(row0, t[c]) : 0xffffffffu;
      if (some) {
#pragma unroll
        for (int h = 0; h < GEN / 16; ++h)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (!((vis[c] >> (16 * h + 4 * g + v)) & 1)) S[c][h][v] = -INFINITY;
      }
      mx[c] = fmaxf(largest(S[c][0]), largest(S[c][1])) * c2;
    }
    raise(mx, QA_SLACK, 0.f);
    bf16x8 P[CG];
    float l[CG], lr[CG];
    auto weigh_all = [&]() {
      const float one[2] = {1.f, 1.f}, zero[2] = {0.f, 0.f}, cc[2] = {c2, c2};
#pragma unroll
      for (int c = 0; c < CG; ++c) {
        l[c] = lr[c] = 0.f;
        P[c] = weigh(c, S[c], cc, zero, one, l[c], lr[c]);
      }
    };
    weigh_all();
    need_v(j + 1 < nsteps);
    // A step whose squares sum to 2^120 or more has values of 2^57 and more, or ones that are not
    // finite: its weights get room, and rows that only some columns see are taken one by one.
    bf16x8 vt[DT];
    float squares = 0.f;
#pragma unroll
    for (int e = 0; e < DT; ++e) {
      vt[e] = v_gen(la, e);
#pragma unroll
      for (int k = 0; k < GEN / 4; k += 2) {
        const bf16x2 x = {vt[e][k], vt[e][k + 1]};
        squares = __builtin_amdgcn_fdot2_f32_bf16(x, x, squares, false);
      }
    }
    const bool huge = __any(!(squares < 0x1p120f));
    if (huge) {
      raise(mx, -QA_ROOM, QA_ROOM + QA_SLACK);
      weigh_all();
    }
    const bool odd = some && huge;  // (of which some may not be finite)
#pragma unroll
    for (int c = 0; c < CG; ++c) l_run[c] += l[c], lr_run[c] += lr[c];
    // all keys at once, or key by key
    for (int k = 0; k < (odd ? GEN : 1); ++k) {
      u32x4 keep;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        // key k sits in slot (k % 4) + 4 (k / 16) of lane group (k % 16) / 4
        const bool here = g == ((k >> 2) & 3) && ((k & 3) + (k >> 4) * 4) >> 1 == x;
        keep[x] = !odd ? 0xffffffffu : here ? (k & 1 ? 0xffff0000u : 0xffffu) : 0u;
      }
#pragma unroll
      for (int e = 0; e < DT; ++e) {
        if (CG > 1) __builtin_amdgcn_sched_barrier(0);
        const bf16x8 v =
            __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, vt[e]) & keep);
#pragma unroll
        for (int c = 0; c < CG; ++c) {
          const f32x4 x =
              __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[c], acc[c][e], 0, 0, 0);
          if (!odd || ((vis[c] >> k) & 1)) acc[c][e] = x;
        }
      }
    }
    done(j);
  }

  // ---- the waves' states, merged through LDS --------------------------------------
  float* const states = reinterpret_cast<float*>(smem);
  float* const sums = states + NW * 16 * L::PITCH;
  constexpr int DL = D / 4;
  const int dv = tid % DL;
#pragma unroll
  for (int c = 0; c < CG; ++c) {
    l_run[c] += __shfl_xor(l_run[c], 16, 64);
    l_run[c] += __shfl_xor(l_run[c], 32, 64);
    lr_run[c] += __shfl_xor(lr_run[c], 16, 64);
    lr_run[c] += __shfl_xor(lr_run[c], 32, 64);
    __syncthreads();  // every wave is done with its stages, or the states before
    {
      float* const mine = states + (wave * 16 + r) * L::PITCH;
#pragma unroll
      for (int e = 0; e < DT; ++e) *reinterpret_cast<f32x4*>(mine + 16 * e + 4 * g) = acc[c][e];
      if (g == 0) {
        sums[(wave * 16 + r) * 3] = m_run[c];
        sums[(wave * 16 + r) * 3 + 1] = l_run[c];
        sums[(wave * 16 + r) * 3 + 2] = lr_run[c];
      }
    }
    __syncthreads();
    // thread -> (column, four consecutive values), a row of D / 4 threads at a time
    for (int x = tid / DL; x < min(16, cols - 16 * c); x += 64 * NW / DL) {
      float m = -INFINITY, l = 0.f, lr = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, sums[(w * 16 + x) * 3]);
      const float use = m == -INFINITY ? 0.f : m;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* y = sums + (w * 16 + x) * 3;
        const float e = __builtin_amdgcn_exp2f(y[0] - use);
        l += e * y[1];
        lr += e * y[2];
        o += e * *reinterpret_cast<const f32x4*>(states + (w * 16 + x) * L::PITCH + 4 * dv);
      }
      o *= lr != 0.f ? 1.f / lr : 0.f;  // (a NaN score leaves a NaN sum)
      const int n = 16 * c + x, nth = a.col_tiles > 1 ? 0 : n / a.group;
      const int hd = kvh * a.group + heads0 + n - nth * a.group;
      const int64_t at = ((int64_t)part * a.Tq + t0 + nth) * a.Hq + hd;
      if (a.o_bf16)
        static_cast<bf16x4*>(a.O)[at * DL + dv] = __builtin_convertvector(o, bf16x4);
      else
        static_cast<f32x4*>(a.O)[at * DL + dv] = o;
      if (dv == 0 && a.lse != nullptr) {
        // (l's exponent, which QA_ROOM makes large, goes to m: no bits of its logarithm)
        const float log2_l = __log2f(__builtin_amdgcn_frexp_mantf(l));
        a.lse[((int64_t)part * a.Hq + hd) * a.Tq + t0 + nth] =
            l != 0.f ? ((m + (float)__builtin_amdgcn_frexp_expf(l)) + log2_l) *
                           0.69314718055994531f
                     : -INFINITY;
      }
    }
  }
}

template <int D, int FORMAT, int NW, int KEYS, int CG>
int launch_one(const QuantAttnArgs& a, hipStream_t stream) {
  using L = QaLds<D, NW, KEYS>;
  const size_t lds = L::REUSED + (a.rows != nullptr ? L::STEPS : 0);
  const int64_t tiles = (int64_t)a.token_tiles * a.col_tiles;
  const int64_t nwg = ((int64_t)a.Hkv * a.parts * a.slices + 7) / 8 * 8 *
                      ((tiles + a.slices - 1) / a.slices);
  if (!grid_fits(nwg, 64 * NW)) return PULSAR_EUNSUPPORTED;
  const auto kern = quant_attn_kernel<D, FORMAT, NW, KEYS, CG>;
  if (lds > 65536 &&
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize,
                          (int)lds) != hipSuccess)
    return PULSAR_EHIP;
  hipLaunchKernelGGL(kern, dim3((unsigned)nwg), dim3(64 * NW), lds, stream, a);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

template <int D, int FORMAT>
int launch_tile(const QuantAttnArgs& a, const QuantPlan& p, hipStream_t stream) {
  if constexpr (D == 128) {
    if (p.keys == 64) return launch_one<D, FORMAT, 4, 64, 2>(a, stream);
    if (p.columns == 48) return launch_one<D, FORMAT, 8, 32, 3>(a, stream);
  }
  if (p.columns == 32) return launch_one<D, FORMAT, 8, 32, 2>(a, stream);
  return launch_one<D, FORMAT, 8, 32, 1>(a, stream);
}

// Workgroups that give each compute unit one, and two, as many as it holds.
constexpr int QA_ONE_EACH = 256, QA_AT_ONCE = 512;

}  // namespace

// Four shapes of tiles.  Each code is widened and read once for all columns of a tile, so wide
// tiles do less, but narrow ones wait less: 16 columns have four waves to a SIMD, the others
// two (of d 128).  Us in replayed graphs, with the merge and 100 rows of the generation shard;
// 32 / 8 heads of 128 in e4m3 where nothing else is said.
//   16 columns, steps of 32 rows, eight waves: up to 13 steps of a wave with all compute units
//   at work (12 where the others are of 32 columns and d is 128).  16 columns / 32 in steps of 32
//   rows: 8 tokens over 32768 keys 21.0 / 23.1, 40960 24.8 / 25.2, 49152 27.9 / 27.5, 65536 33.8
//   / 32.1; of d 64, 16 / 16 heads, 24 tokens over 8192 13.2 / 14.0, 16384 16.6 / 16.5, 32768
//   21.5 / 21.6.  16 columns / 48: 12 tokens over 32768 25.4 / 27.3, 49152 34.6 / 31.5, 24 tokens
//   over 8192 18.3 / 22.7, 16384 25.0 / 25.0 (32 columns 22.7), 24576 31.1 / 28.3.
//   48 columns, as above (d 128), where that is a third fewer tiles than of 32.  48 / the best of
//   32: 12 tokens over 49152 keys 31.5 / 31.5, 131072 55 / 62, 24 tokens 72 / 84, 36 tokens 105 /
//   128; but 64 (6 tiles against 8) 188 / 180.
//   32 columns, as above (d 128): one tile, bound by its keys (8 tokens over 131072 51 against
//   57 of the next shape), or up to 28 steps of a wave.  Steps of 32 / of 64 rows, 64 tokens over
//   8192 keys 26.6 / 29.0, 16384 36.1 / 36.7, 24576 46.4 / 46.4, 32768 57.6 / 57.7, 49152 79.9 /
//   78.4, 131072 189 / 180.  (int8, which the rule does not ask for: 16384 41.5 / 43.9, 32768
//   68.9 / 72.0, 131072 234 / 236.)
//   32 columns, steps of 64 rows, four waves: the rest of d 128.  Of d 64, whose 32 columns
//   leave room for four waves to a SIMD: steps of 32 rows and eight waves (64 rows, when they were
//   built for d 64, took 64 tokens of 32 / 8 heads over 131072 keys 7 % longer, in int8 6 %).
// Parts: as many as give each compute unit one workgroup.  Two for the last two shapes, but for
// one tile of d 64 (one / two: 16 / 16 heads, 24 tokens over 131072 keys 50.1 / 52.3; of two tiles,
// 64 tokens over 16384 20.7 / 21.6, 65536 48.5 / 43.2, and 32 / 8 heads, 64 tokens over 16384 29.8
// / 28.8, 131072 160 / 130).  Two too for 16 columns where waves would have ten steps or more and
// tiles share their keys (12 tokens over 16384 17.4 / 18.6, 32768 25.4 / 24.2; 1 token over 16384
// 13.1 / 14.2, 131072 47.9 / 48.3; 16 / 16 of 64, 1 token over 4084 9.8 / 10.3, 131072 48.8 /
// 49.2).
// But one part up to five steps of a wave: parts need the merge's launch and a workspace, 4 us
// of the host's time, for which calls from the host wait and replayed ones do not.  A replayed
// graph / calls from the host, several parts and one: 1 token over 480 keys 9.1 / 15.4 and 9.5 /
// 11.3, 1000 9.6 / 15.5 and 11.9 / 11.8, 1500 9.8 / 15.4 and 14.1 / 14.0; 16 / 16 of 64, 24 tokens
// over 1000 keys 8.9 / 15.4 and 9.9 / 11.3.
QuantPlan quant_plan(int n_shards, int Tq, int64_t S, int Hq, int Hkv, int d, int64_t gen_rows) {
  QuantPlan p{};
  const int group = Hq / Hkv;
  const int64_t gen = (gen_rows + 31) / 32;  // (whole 32 rows, for few sizes to ask for)
  auto tiles = [&](int columns) {
    const int tokens = std::max(1, columns / group);
    return (int64_t)((Tq + tokens - 1) / tokens) * ((group + columns - 1) / columns);
  };
  auto steps = [&](int keys) { return n_shards * ((S + keys - 1) / keys) + gen * (64 / keys); };
  auto take = [&](int columns, int keys, int at_once) {
    const int waves = keys == 32 ? 8 : 4;
    const int64_t own = tiles(columns), fill = at_once / std::max<int64_t>(own * Hkv, 1);
    p.columns = columns;
    p.keys = keys;
    p.tokens = std::max(1, columns / group);
    p.parts = parts_at_once(std::min(fill, (steps(keys) + waves - 1) / waves), Hkv, own,
                            at_once / 8);
    return p;
  };
  const int64_t of32 = tiles(32);
  const bool of48 = d == 128 && 3 * tiles(48) <= 2 * of32;
  const int64_t at_once = 8 * QA_ONE_EACH;  // waves
  if ((int64_t)Tq * group > 16 &&
      tiles(16) * Hkv * steps(32) >= (d == 64 || of48 ? 13 : 12) * at_once) {
    if (of48) return take(48, 32, QA_ONE_EACH);
    if (d == 128 && (of32 == 1 || of32 * Hkv * steps(32) <= 28 * at_once))
      return take(32, 32, QA_ONE_EACH);
    if (d == 64) return take(32, 32, of32 == 1 ? QA_ONE_EACH : QA_AT_ONCE);
    return take(32, 64, QA_AT_ONCE);
  }
  take(16, 32, QA_ONE_EACH);
  if (steps(32) <= 5 * 8) p.parts = 1;
  else if (steps(32) >= 10 * 8 * (int64_t)p.parts && tiles(16) > 1)
    take(16, 32, QA_AT_ONCE);
  return p;
}

// Rows of partials (tokens times parts) of any call of up to Tq tokens: parts are QA_AT_ONCE /
// (tiles * Hkv) at most, of tiles that hold 32 columns at most, or half as many of 48.
int64_t quant_part_rows_most(int Tq, int Hq, int Hkv) {
  if (Tq <= 0) return 0;
  const int64_t tokens = std::min(std::max(32 / (Hq / Hkv), 1), Tq);
  return (int64_t)QA_AT_ONCE / Hkv * tokens;
}

int launch_quant_attn(const QuantAttnLaunch& x, const QuantPlan& p, void* o, int o_bf16,
                      float* lse, hipStream_t stream) {
  QuantAttnArgs a{};
  a.q = x.q;
  a.K = x.K;
  a.V = x.V;
  a.ks = x.ks;
  a.vs = x.vs;
  a.rows = x.n_shards > 0 ? x.rows : nullptr;
  a.Kg = x.Kg;
  a.Vg = x.Vg;
  a.mask = x.mask;
  a.Tq = x.Tq;
  a.Hq = x.Hq;
  a.Hkv = x.Hkv;
  a.group = x.Hq / x.Hkv;
  const int most = p.columns;
  a.tile_tokens = p.tokens;
  a.token_tiles = (x.Tq + p.tokens - 1) / p.tokens;
  a.col_tiles = (a.group + most - 1) / most;
  a.slices = tile_slices((int64_t)x.Hkv * p.parts, (int64_t)a.token_tiles * a.col_tiles);
  a.n_shards = x.n_shards;
  a.S = (int)x.S;
  a.block_log2 = __builtin_ctz(x.block);
  a.blocks = (int)((x.S + x.block - 1) >> a.block_log2);
  a.gen_rows = x.Kg != nullptr ? (int)(x.G + x.Tq) : 0;
  a.G = (int)x.G;
  a.shard_steps = (int)((x.S + p.keys - 1) / p.keys);
  a.parts = p.parts;
  a.scale_log2 = x.scale * 1.4426950408889634f;
  a.O = o;
  a.o_bf16 = o_bf16;
  a.lse = lse;
  const bool e4m3 = x.format == PULSAR_KV_E4M3;
  if (x.d == 128)
    return e4m3 ? launch_tile<128, PULSAR_KV_E4M3>(a, p, stream)
                : launch_tile<128, PULSAR_KV_INT8>(a, p, stream);
  return e4m3 ? launch_tile<64, PULSAR_KV_E4M3>(a, p, stream)
              : launch_tile<64, PULSAR_KV_INT8>(a, p, stream);
}
