// Phase-2 attention of few new tokens by 16-row tiles of (token, head) rows: over
// the blocks of the retained shards that were selected for each token (and KV head)
// and over the generation shard; or over all keys, for the partials of drafts.
//
// Work.  A tile is the columns of one pass over keys: one token's heads (16 of them
// at a time), or as many tokens as fit.  Its keys are a list of 16-key halves, two of
// them a 32-key step:
//   LISTED  one token: its listed blocks in the list's order, then the generation
//           shard's rows;
//   UNION   several tokens, in one or two groups of 16 columns: the blocks that any of
//           them lists, each with the tokens that list it, found in LDS; then the
//           generation shard's rows.  Where neighbouring tokens list the same blocks
//           these are read and multiplied once, and else no column does more than it
//           would alone;
//   DENSE   all rows of the shards, then the appended rows.
// A workgroup takes one part of the steps of one tile: wave w of NW the steps w,
// w + NW, ... of it, on its own; then the waves' states are merged through LDS.  A
// step of a wave:
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
// What must not be seen.  A row that no column sees is replaced by a copy of one of its
// half, or of the other half, that some column does.  A step without any such row (LISTED:
// of entries that are no block; of unseen drafts) is loaded from some row of the tensor and
// scored as others are, all -inf, and PV is left out: it takes the time of a step, and the
// plan counts it as one (a token with 16 x 4 entries of 64 keys 10.2 us, all of them -1
// 10.1).  Of the rows that only some columns see, weights of zero keep the others clear of
// them unless they hold a NaN or an infinity: a pass that ends with a NaN is repeated key by
// key, each key's product taken over only into the columns that see it.
#include <algorithm>
#include <type_traits>

#include "tiles.hpp"

namespace {

constexpr int SP_KEYS = 32;       // keys per step
constexpr float SP_SLACK = 8.0f;  // log2 slack before the reference is raised
// A union's list in LDS, in entries, and its map, a byte per block: as much as leaves
// room for all the workgroups that the registers do.
constexpr int sp_list(int d) { return d == 64 ? 1792 : 3584; }
constexpr int sp_map(int d) { return d == 64 ? 32768 : 65536; }

enum SparseMode : int { SP_LISTED, SP_UNION, SP_DENSE };

struct SparseArgs {
  const uint16_t *q, *K, *V, *Kg, *Vg;
  const int32_t* sel;
  const uint32_t* mask;
  int Tq, Hq, Hkv, group;
  int tile_tokens;       // tokens per tile
  int token_tiles;       // tiles over the tokens
  int col_tiles;         // tiles over a token's heads (1 where a tile holds them all)
  int slices;            // XCDs over which the tiles of a head's part are spread
  int n_shards, topk, entries;  // listed blocks per shard; of all shards
  int half_log2;         // log2 of a block's halves
  int blocks;            // blocks per shard
  int gen_rows;          // G + Tq (DENSE: G), or 0 without a generation shard
  int64_t S, G;          // (DENSE: S is of all shards)
  int list_steps;        // LISTED, DENSE: steps of the shards; the generation shard's follow
  int parts, part_steps; // (UNION: counted per tile)
  float scale_log2;
  int o_bf16;
  void* O;               // parts > 1, DENSE: float [parts, Tq, Hq, D]; else the output
  float* lse;            // [parts, Hq, Tq]; nullable for the output
};

typedef __attribute__((address_space(4))) SparseArgs ConstArgs;

template <int D, int NW, int MODE>
struct SpLds {
  static constexpr int STAGE = SP_KEYS * D * 2;              // a K or V step
  static constexpr int LOOP = NW * 2 * STAGE;
  static constexpr int PITCH = D + 4;                        // floats of a state's column
  static constexpr int MERGE = NW * 16 * (PITCH + 3) * 4;
  static constexpr int REUSED = LOOP > MERGE ? LOOP : MERGE;
  // UNION: the list, and the sums of its waves
  static constexpr int LIST = sp_list(D);
  static constexpr int BYTES = REUSED + (MODE == SP_UNION ? LIST * 4 + 64 : 0);
  static_assert(MODE != SP_UNION || REUSED >= sp_map(D), "the map passes through the stages");
};

template <int D, int NW, int MODE, int CG>
__global__ __launch_bounds__(64 * NW)
__attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 4, D == 128 ? 2 : 4)))
void sparse_attn_kernel(SparseArgs a) {
  using L = SpLds<D, NW, MODE>;
  constexpr int CPR = D / 8;               // 16-byte chunks per row
  constexpr int DS = D / 32;               // k-steps of S
  constexpr int DT = D / 16;               // 16-row tiles of O^T
  constexpr int V_SEGS = L::STAGE / 1024;  // 1 KiB segments: one 16-byte load per lane each
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];

  // the arguments as they lie in memory, for what few steps need
  // (kept in registers with the rest they do not fit)
  auto reread = [&]() {
    auto p = (const ConstArgs*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
  };
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  // Workgroup -> (token tile, heads) of a (KV head, part).  Workgroups go to the eight
  // XCDs in turn, each with an L2 of its own: all tiles of one head's part, which read
  // the same keys (or blocks that they share), go to one of them, one after another;
  // where there are few such parts, to `slices` of them.
  const int tiles = a.token_tiles * a.col_tiles, deep = (tiles + a.slices - 1) / a.slices;
  int64_t wg = blockIdx.x >> 3;
  const int in = (int)(wg % deep);
  wg = wg / deep * 8 + (blockIdx.x & 7);
  const int tile = in * a.slices + (int)(wg % a.slices);
  wg /= a.slices;
  if (wg >= (int64_t)a.Hkv * a.parts || tile >= tiles) return;
  const int kvh = (int)(wg % a.Hkv), part = (int)(wg / a.Hkv);
  const int t0 = tile % a.token_tiles * a.tile_tokens;
  const int heads0 = tile / a.token_tiles * 16;
  const int tokens = min(a.tile_tokens, a.Tq - t0);  // of this tile
  const int per = CG > 1 ? 16 / a.group : a.tile_tokens;  // of 16 columns
  const float c2 = a.scale_log2;
  const uint32_t row_bytes = (uint32_t)(a.Hkv * D * 2);
  const uint32_t head_off = (uint32_t)(kvh * D * 2);

  // ---- Q fragments (B operand): column r of group c = token tl of the tile, head ----
  int tl[CG], t[CG];
  bf16x8 qf[CG][DS];
#pragma unroll
  for (int c = 0; c < CG; ++c) {
    const int nth = a.tile_tokens == 1 ? 0 : r / a.group;
    tl[c] = c * per + nth;
    const int col = heads0 + r - nth * a.group;  // head of the group
    const bool live = nth < per && tl[c] < tokens && col < a.group;
    t[c] = t0 + (live ? tl[c] : 0);
    const int head = kvh * a.group + (live ? col : 0);
    const bf16x8* src =
        reinterpret_cast<const bf16x8*>(a.q + ((int64_t)t[c] * a.Hq + head) * D) + g;
#pragma unroll
    for (int s = 0; s < DS; ++s) qf[c][s] = live ? src[4 * s] : bf16x8{};
  }

  // ---- the union of the tile's lists --------------------------------------------
  // A byte per block of all shards, bit i set where token i lists it, through the
  // stages' LDS; then its non-zero bytes in order, block << 8 | byte.  A token that
  // lists a block twice has its tile processed token by token (`doubled`).
  uint32_t* const list = reinterpret_cast<uint32_t*>(smem + L::REUSED);
  int listed = 0;
  bool doubled = false;
  if constexpr (MODE == SP_UNION) {
    int* const s_sum = reinterpret_cast<int*>(list + L::LIST);
    uint32_t* const map = reinterpret_cast<uint32_t*>(smem);
    const int quads = (a.n_shards * a.blocks + 15) / 16;  // 16 blocks each
    for (int i = tid; i < quads; i += 64 * NW)
      reinterpret_cast<u32x4*>(map)[i] = u32x4{0u, 0u, 0u, 0u};
    if (tid == 0) s_sum[NW] = 0;
    __syncthreads();
    const int per_token = a.entries;
    for (int i = tid; i < tokens * per_token; i += 64 * NW) {
      const int token = i / per_token, e = i - token * per_token;
      const int shard = e / a.topk;
      const int b = a.sel[(((int64_t)shard * a.Tq + t0 + token) * a.Hkv + kvh) * a.topk +
                          (e - shard * a.topk)];
      if (b < 0 || b >= a.blocks) continue;
      const int at = shard * a.blocks + b;
      const uint32_t bit = 1u << (8 * (at & 3) + token);
      if (atomicOr(&map[at >> 2], bit) & bit) s_sum[NW] = 1;
    }
    __syncthreads();
    doubled = __builtin_amdgcn_readfirstlane(s_sum[NW]) != 0;
    for (int i0 = 0; i0 < quads; i0 += 64 * NW) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (i0 + tid < quads) w = reinterpret_cast<const u32x4*>(map)[i0 + tid];
      int n = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) n += ((w[k / 4] >> (8 * (k % 4))) & 0xffu) != 0;
      int at = wave_excl_scan(n);
      if (lane == 63) s_sum[wave] = at + n;
      __syncthreads();
      int sum = 0;
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        at += k < wave ? s_sum[k] : 0;
        sum += s_sum[k];
      }
      at += listed;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const uint32_t who = (w[k / 4] >> (8 * (k % 4))) & 0xffu;
        if (who) list[at++] = (16 * (i0 + tid) + k) << 8 | who;
      }
      listed += sum;
      __syncthreads();
    }
    listed = __builtin_amdgcn_readfirstlane(listed);
  }

  // ---- the tile's steps -----------------------------------------------------------
  // (`one`: the token whose list is read where a tile is processed token by token)
  const uint32_t tile_bits = (1u << tokens) - 1;
  const int gen_end = a.gen_rows == 0                ? 0
                      : MODE == SP_DENSE || a.mask ? a.gen_rows
                                                     : (int)(a.G + t0 + tokens);
  int list_steps, step0, step1, nsteps, one = 0;
  auto plan = [&]() {
    const int halves = MODE == SP_UNION ? (doubled ? a.entries : listed) << a.half_log2 : 0;
    list_steps = MODE == SP_UNION ? (halves + 1) / 2 : a.list_steps;
    // the generation shard's rows once, with the first token's list
    const int gen_steps = MODE == SP_UNION && one > 0 ? 0 : (gen_end + SP_KEYS - 1) / SP_KEYS;
    const int total = list_steps + gen_steps;
    const int per = MODE == SP_UNION ? (total + a.parts - 1) / a.parts : a.part_steps;
    step0 = part * per;
    step1 = min(step0 + per, total);
    nsteps = max(0, (step1 - step0 - wave + NW - 1) / NW);
  };
  // The rows at .. at + 15 of the generation shard that token `token` sees.
  auto gen_sees = [&](int at, int token) -> uint32_t {
    const ConstArgs& a = *reread();
    const int end = MODE == SP_DENSE || a.mask ? a.gen_rows : (int)(a.G + token + 1);
    const int rows = min(16, end - at);
    if (rows <= 0) return 0u;
    uint32_t sees = (1u << rows) - 1;
    if (MODE != SP_DENSE && a.mask != nullptr && at + rows > a.G) {
      // drafts at - G .. are visible by the token's bits
      const int words = (a.Tq + 31) / 32;
      const uint32_t* bits = a.mask + (int64_t)token * words;
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
    return sees;
  };

  // ---- where the halves lie: lane 2i + h, half h of the wave's step base + i -----
  // Byte offset of the half's first row in K (or Kg), and its rows: those that some
  // column sees (bits 0-15) and those to load (bits 16-31); UNION: the tokens that
  // see a listed half, and kEvery where both are seen whole, by the same ones.  A half
  // of which nothing is seen is loaded as its neighbour.
  constexpr uint32_t kEvery = 1u << 16;
  uint32_t tab_lo = 0, tab_hi = 0, tab_rows = 0, tab_tokens = 0;
  auto fill = [&](int base) {
    const ConstArgs& a = *reread();
    const int st = step0 + wave + NW * (base + (lane >> 1));
    int64_t row = 0;
    uint32_t sees = 0, who = tile_bits;
    if (st < step1 && st < list_steps) {
      const int e = st * 2 + (lane & 1);
      if constexpr (MODE == SP_DENSE) {
        const int64_t at = (int64_t)e * 16;
        if (at < a.S) {
          row = at;
          sees = (1u << (int)min((int64_t)16, a.S - at)) - 1;
        }
      } else {
        const int entry = e >> a.half_log2;
        int shard = 0, b = -1;
        if (MODE == SP_UNION && !doubled) {
          if (entry < listed) {
            const uint32_t x = list[entry];
            who = x & 0xffu;
            shard = (int)(x >> 8) / a.blocks;
            b = (int)(x >> 8) - shard * a.blocks;
          }
        } else if (entry < a.entries) {
          shard = entry / a.topk;
          b = a.sel[(((int64_t)shard * a.Tq + t0 + one) * a.Hkv + kvh) * a.topk +
                    (entry - shard * a.topk)];
          who = 1u << one;
        }
        const int64_t at =
            ((int64_t)b << (a.half_log2 + 4)) + ((e & ((1 << a.half_log2) - 1)) << 4);
        if (b >= 0 && b < a.blocks && at < a.S) {
          row = shard * a.S + at;
          sees = (1u << (int)min((int64_t)16, a.S - at)) - 1;
        }
      }
    } else if (st < step1) {
      const int at = (st - list_steps) * SP_KEYS + (lane & 1) * 16;
      row = at < gen_end ? at : 0;
      if constexpr (MODE == SP_UNION) {
        for (int i = 0; i < tokens; ++i) sees |= gen_sees(at, t0 + i);
      } else {
        sees = gen_sees(at, t0);
      }
    }
    const uint64_t off = (uint64_t)row * row_bytes;
    const uint32_t lo = (uint32_t)off, hi = (uint32_t)(off >> 32);
    const uint32_t n_lo = __shfl_xor((int)lo, 1, 64), n_hi = __shfl_xor((int)hi, 1, 64);
    const uint32_t n_sees = __shfl_xor((int)sees, 1, 64);
    tab_lo = sees ? lo : n_lo;
    tab_hi = sees ? hi : n_hi;
    tab_rows = sees | (sees ? sees : n_sees) << 16;
    // (a half that is not seen at all is seen by nobody: as its neighbour)
    const uint32_t n_who = MODE == SP_UNION ? __shfl_xor((int)who, 1, 64) : 0u;
    const uint32_t own = sees ? who : n_who, other = n_sees ? n_who : who;
    tab_tokens = lane & 1 ? other | own << 8 : own | other << 8;
    if (MODE == SP_UNION && st < list_steps && sees == 0xffffu && n_sees == 0xffffu && own == other)
      tab_tokens |= kEvery;
  };
  struct Half {
    uint32_t rows;  // seen, and << 16 to load
    int64_t off;
  };
  auto half = [&](int j, int h) {
    const int at = 2 * (j & 31) + h;
    return Half{(uint32_t)__builtin_amdgcn_readlane(tab_rows, at),
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
    int st;
    uint32_t tokens;
  };
  auto step_at = [&](int j) {
    return Step{{half(j, 0), half(j, 1)}, step0 + wave + NW * j,
                MODE == SP_UNION
                    ? (uint32_t)__builtin_amdgcn_readlane(tab_tokens, 2 * (j & 31)) : 0u};
  };
  auto is_gen = [&](const Step& x) { return x.st >= list_steps; };
  // A row that is not to be loaded is loaded as the first one that is.
  auto issue = [&](const Step& x, const uint16_t* base, lds_u8* lds,
                   const uint32_t (&off)[H_SEGS]) {
    const uint32_t st = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
    __amdgpu_buffer_rsrc_t rsrc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      rsrc[h] = __builtin_amdgcn_make_buffer_rsrc(
          reinterpret_cast<uint8_t*>(const_cast<uint16_t*>(base)) + x.half[h].off, (short)0,
          (int)(16 * row_bytes), kBufferFlags);
    if ((x.half[0].rows & x.half[1].rows) >> 16 == 0xffffu) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < H_SEGS; ++i)
          lds_dma16(rsrc[h], off[i], i * SEG_ROWS * row_bytes, st + (h * H_SEGS + i) * 1024);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t load = x.half[h].rows >> 16;
        const int first = __builtin_ctz(load | 0x10000u) & 15;
#pragma unroll
        for (int i = 0; i < H_SEGS; ++i) {
          const int row = i * SEG_ROWS + seg_row;
          const int from = (load >> row) & 1 ? row : first;
          lds_dma16(rsrc[h], off[i] + (from - seg_row) * row_bytes, st + (h * H_SEGS + i) * 1024);
        }
      }
    }
  };
  const lds_u8* k_at[DS];  // chunk 4s + g of row r of a half
#pragma unroll
  for (int s = 0; s < DS; ++s) k_at[s] = k_lds + (r * CPR + ((4 * s + g) ^ k_swizzle(r))) * 16;
  // V^T rows e*16 .. of the step: lane (r, g) of a transposing read addresses row
  // 4g + r/4 of a half at head_dim 16e + 4 (r%4) and receives head_dim 16e + r of
  // keys 4g .. 4g+3 of it
  const lds_u8* v_at[DT];
  {
    const int row = 4 * g + (r >> 2), q4 = r & 3;
#pragma unroll
    for (int e = 0; e < DT; ++e)
      v_at[e] = v_lds + row * (2 * D) + 16 * ((2 * e + (q4 >> 1)) ^ v_swizzle8(row)) + 8 * (q4 & 1);
  }
  auto v_frag = [&](int e) -> bf16x8 {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)v_at[e]);
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v_at[e] + 16 * (2 * D)));
    return __builtin_bit_cast(bf16x8,
                              (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
  };

  f32x4 acc[CG][DT];
  float m_run[CG], l_run[CG], lr_run[CG];
  auto clear = [&]() {
#pragma unroll
    for (int c = 0; c < CG; ++c) {
#pragma unroll
      for (int e = 0; e < DT; ++e) acc[c][e] = f32x4{0.f, 0.f, 0.f, 0.f};
      m_run[c] = -INFINITY;
      l_run[c] = lr_run[c] = 0.f;
    }
  };
  // The wave's steps of the present plan; `guard`: key by key (see above).
  auto run = [&](auto guard_tag) {
    constexpr bool guard = decltype(guard_tag)::value;
    Step next{};
    if (nsteps > 0) {
      fill(0);
      next = step_at(0);
      issue(next, is_gen(next) ? a.Kg : a.K, k_lds, k_off);
      issue(next, is_gen(next) ? a.Vg : a.V, v_lds, v_off);
    }
    for (int j = 0; j < nsteps; ++j) {
      // the keys of the step that some column sees, and the tokens that list it
      const uint32_t seen = (next.half[0].rows & 0xffffu) | next.half[1].rows << 16;
      const int st = next.st;
      const uint32_t who = next.tokens;
      const bool more = j + 1 < nsteps;
      // K(j) is in LDS once only V(j)'s loads are outstanding
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(V_SEGS) : "memory");
      __builtin_amdgcn_sched_barrier(0);
      f32x4 S[CG][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < CG; ++c) S[c][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < DS; ++s) {
          const bf16x8 k =
              *reinterpret_cast<const lds_bf16x8*>(k_at[s] + h * (L::STAGE / 2));
#pragma unroll
          for (int c = 0; c < CG; ++c)
            S[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[c][s], S[c][h], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (more) {
        if (((j + 1) & 31) == 0) fill(j + 1);
        next = step_at(j + 1);
        issue(next, is_gen(next) ? a.Kg : a.K, k_lds, k_off);
      }
      __builtin_amdgcn_sched_barrier(0);
      // UNION: a column sees all of the step's keys or none (`every`), else some of them
      uint32_t vis[CG];
      const bool every = MODE == SP_UNION && !guard && (who & kEvery) != 0;
#pragma unroll
      for (int c = 0; c < CG; ++c) vis[c] = seen;
      if (!every && (MODE == SP_UNION || seen != 0xffffffffu)) {
#pragma unroll
        for (int c = 0; c < CG; ++c) {
          if constexpr (MODE == SP_UNION) {
            const int at = (st - list_steps) * SP_KEYS;
            if (st < list_steps)
              vis[c] &= ((who >> tl[c]) & 1 ? 0xffffu : 0u) |
                        ((who >> (8 + tl[c])) & 1 ? 0xffff0000u : 0u);
            else if (a.mask != nullptr || at + SP_KEYS > a.G)
              vis[c] = gen_sees(at, t[c]) | gen_sees(at + 16, t[c]) << 16;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int v = 0; v < 4; ++v)
              if (!((vis[c] >> (16 * h + 4 * g + v)) & 1)) S[c][h][v] = -INFINITY;
        }
      }
      bf16x8 P[CG];
#pragma unroll
      for (int c = 0; c < CG; ++c) {
        // (16 columns whose tokens see nothing of the step weigh nothing)
        if (CG > 1 && (((who | who >> 8) & 0xffu) >> (c * per) & ((1u << per) - 1)) == 0) {
          P[c] = bf16x8{};
          continue;
        }
        const bool mine = !every || ((who >> tl[c]) & 1);
        float mx = S[c][0][0];
#pragma unroll
        for (int v = 1; v < 8; ++v) mx = fmaxf(mx, S[c][v >> 2][v & 3]);
        mx = max_of_rows(mx) * c2;
        if (MODE == SP_UNION) mx = mine ? mx : -INFINITY;
        if (__any(mx > m_run[c] + SP_SLACK)) {
          const float m_new = mx > m_run[c] + SP_SLACK ? mx : m_run[c];
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[c] - m_new);
#pragma unroll
          for (int e = 0; e < DT; ++e) acc[c][e] *= alpha;
          l_run[c] *= alpha;
          lr_run[c] *= alpha;
          m_run[c] = m_new;
        }
        // a column that has seen no key takes its weights against 0: they come out 0
        float m_use = m_run[c] == -INFINITY ? 0.f : m_run[c];
        // (against infinity the weights of a step that it does not see come out 0, or not
        // a number, which the pass's end finds)
        if (MODE == SP_UNION) m_use = mine ? m_use : INFINITY;
        f32x8 p;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[c][v >> 2][v & 3], c2, -m_use));
          l_run[c] += p[v];
        }
        P[c] = __builtin_convertvector(p, bf16x8);
#pragma unroll
        for (int v = 0; v < 8; v += 2)
          lr_run[c] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{P[c][v], P[c][v + 1]}, kOnes2,
                                                      lr_run[c], false);
      }
      // V(j) is in LDS once only K(j + 1)'s loads are outstanding
      __builtin_amdgcn_sched_barrier(0);
      if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(V_SEGS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if (seen != 0) {
        if constexpr (MODE == SP_UNION && guard) {
          for (int k = 0; k < SP_KEYS; ++k) {
            // key k sits in slots of lane group (k % 16) / 4
            const int slot = (k & 3) + (k >> 4) * 4;
            u32x4 keep = {0u, 0u, 0u, 0u};
            if (g == ((k >> 2) & 3)) {
#pragma unroll
              for (int x = 0; x < 4; ++x)
                keep[x] = slot >> 1 == x ? (slot & 1 ? 0xffff0000u : 0xffffu) : 0u;
            }
#pragma unroll
            for (int e = 0; e < DT; ++e) {
              const bf16x8 v = __builtin_bit_cast(
                  bf16x8, __builtin_bit_cast(u32x4, v_frag(e)) & keep);
#pragma unroll
              for (int c = 0; c < CG; ++c) {
                const f32x4 x =
                    __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[c], acc[c][e], 0, 0, 0);
                if ((vis[c] >> k) & 1) acc[c][e] = x;
              }
            }
          }
        } else if (MODE == SP_UNION || seen == 0xffffffffu) {
#pragma unroll
          for (int e = 0; e < DT; ++e) {
            const bf16x8 v = v_frag(e);
#pragma unroll
            for (int c = 0; c < CG; ++c)
              acc[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[c], acc[c][e], 0, 0, 0);
          }
        } else {
          // zeros in place of the copies, whose weights of zero an infinity would not heed
          u32x4 keep;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t two = seen >> (16 * (x >> 1) + 4 * g + 2 * (x & 1));
            keep[x] = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
          }
#pragma unroll
          for (int e = 0; e < DT; ++e) {
            const bf16x8 v = __builtin_bit_cast(
                bf16x8, __builtin_bit_cast(u32x4, v_frag(e)) & keep);
            acc[0][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[0], acc[0][e], 0, 0, 0);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (more) issue(next, is_gen(next) ? a.Vg : a.V, v_lds, v_off);
    }
  };
  if constexpr (MODE == SP_UNION) {
    __syncthreads();  // the map has been read: the stages are free
    const int turns = doubled ? tokens : 1;
    auto pass = [&](auto guard) {
      clear();
      for (one = 0; one < turns; ++one) {
        plan();
        run(guard);
      }
      bool bad = false;
#pragma unroll
      for (int c = 0; c < CG; ++c)
#pragma unroll
        for (int e = 0; e < DT; ++e)
#pragma unroll
          for (int v = 0; v < 4; ++v) bad |= acc[c][e][v] != acc[c][e][v];
      return __builtin_amdgcn_readfirstlane(__any(bad)) != 0;
    };
    if (pass(std::false_type{})) pass(std::true_type{});
  } else {
    clear();
    plan();
    run(std::false_type{});
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
    const int cols = a.tile_tokens == 1 ? min(16, a.group - heads0)
                                        : min(per, tokens - c * per) * a.group;
    for (int x = tid / DL; x < cols; x += 64 * NW / DL) {
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
      const int nth = a.tile_tokens == 1 ? 0 : x / a.group;
      const int hd = kvh * a.group + heads0 + x - nth * a.group;
      const int64_t at = ((int64_t)part * a.Tq + t0 + c * per + nth) * a.Hq + hd;
      if (a.o_bf16)
        static_cast<bf16x4*>(a.O)[at * DL + dv] = __builtin_convertvector(o, bf16x4);
      else
        static_cast<f32x4*>(a.O)[at * DL + dv] = o;
      if (dv == 0 && a.lse != nullptr)
        a.lse[((int64_t)part * a.Hq + hd) * a.Tq + t0 + c * per + nth] =
            l != 0.f ? (m + __log2f(l)) * 0.69314718055994531f : -INFINITY;
    }
  }
}

template <int D, int NW, int MODE, int CG = 1>
int launch_tiles(const SparseArgs& a, hipStream_t stream) {
  constexpr size_t lds = SpLds<D, NW, MODE>::BYTES;
  const int64_t tiles = (int64_t)a.token_tiles * a.col_tiles;
  const int64_t nwg = ((int64_t)a.Hkv * a.parts * a.slices + 7) / 8 * 8 *
                      ((tiles + a.slices - 1) / a.slices);
  if (!grid_fits(nwg, 64 * NW)) return PULSAR_EUNSUPPORTED;
  const auto kern = sparse_attn_kernel<D, NW, MODE, CG>;
  if (lds > 65536 &&
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize,
                          (int)lds) != hipSuccess)
    return PULSAR_EHIP;
  hipLaunchKernelGGL(kern, dim3((unsigned)nwg), dim3(64 * NW), lds, stream, a);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

// Workgroups of four waves that the chip holds at once: two on each compute unit,
// four at d 64.
int tiles_at_once(int d) { return d == 64 ? 1024 : 512; }

int64_t steps_of(int64_t keys) { return (keys + SP_KEYS - 1) / SP_KEYS; }

// XCDs over which the `tiles` of each of `units` (KV head, part) pairs are spread: few
// pairs that are no multiple of eight, so that all XCDs are at work.
int tile_slices(int64_t units, int64_t tiles) {
  int slices = 1;
  if (units < 32)
    while (units * slices % 8 != 0 && slices * 2 <= tiles) slices *= 2;
  return slices;
}
// The most parts, up to `parts`, whose workgroups an XCD holds at once.
int parts_at_once(int64_t parts, int Hkv, int64_t tiles, int64_t held) {
  while (parts > 1) {
    const int slices = tile_slices(Hkv * parts, tiles);
    if ((Hkv * parts * slices + 7) / 8 * ((tiles + slices - 1) / slices) <= held) break;
    --parts;
  }
  return (int)std::max<int64_t>(parts, 1);
}

}  // namespace

// Tokens whose lists one tile reads together, where their own tiles are more than a
// workgroup for each compute unit and the rows that they read one by one enough to pay
// for finding the union: as many as fit 16 columns, or two groups of 16 at d 128 (at d
// 64 these do not fit the registers of four waves), a block's byte and the union's map
// and list.  Tokens that draw a quarter of the same blocks each, us, one by one / 16
// columns / 32: 32 heads of 128 over 8, 256 tiles 558 MB 27.6 / 31.7 / 34.6, 288 of 326 MB
// 25.7 / 22.4 / 25.3, 512 of 587 MB 27.5 / 27.0 / 29.0, 512 of 1074 MB 44.9 / 41.0 / 40.3,
// 640 of 1342 MB 75 / 48 / 44, 1024 of 2.2 GB 84 / 65 / 58; 16 over 2, 512 tiles 638 MB
// 28.6 / 30.7 / 33.6, 400 of 839 MB 43.1 / 42.0 / 44.4; 16 of 64 over 16, 384 tiles 223 MB
// 17.9 / 18.9, 640 of 372 MB 24.0 / 20.7; 4 over 2, 512 of 319 MB 17.4 / 19.8.
// What they share the host does not see.  With the same lists: 264 tiles of 554 MB 42.8 /
// 19.9 / 23.0, 512 of 1074 MB 44.7 / 22.6 / 25.2, 1024 of 2.1 GB 84 / 31 / 31.  With lists
// that share nothing, whose blocks each tile reads for one column in eight: 264 of 554 MB
// 100 / 88 / 98, 512 of 1074 MB 123 / 136 / 148, 640 of 1342 MB 170 / 162 / 175, 1024 of 2.1
// GB 250 / 191 / 238; 16 over 2, 400 of 839 MB 48 / 59 / 77; 16 of 64 over 16, 640 of 336 MB
// 55 / 59, 1280 of 671 MB 96 / 108.
static int tile_tokens_most(int group, int d) {
  return std::min(16 / group * (d == 128 ? 2 : 1), 8);
}
static int union_tokens(int Tq, int Hkv, int group, int d, int64_t blocks, int64_t entries,
                        int64_t steps) {
  const int64_t mb = (int64_t)Tq * Hkv * steps * (SP_KEYS * d * 4) / 1000000;
  if (blocks > sp_map(d) || (int64_t)Tq * Hkv <= 256 || mb < (group <= 4 ? 320 : 800)) return 1;
  for (const int most : {mb < 1200 ? 1 : tile_tokens_most(group, d), std::min(16 / group, 8)}) {
    const int fit = std::min(most, Tq);
    if (fit > 1 && std::min(entries * fit, blocks) <= sp_list(d)) return fit;
  }
  return 1;
}

SparsePlan sparse_plan(int n_shards, int Tq, int64_t S, int Hq, int Hkv, int d, int block, int topk,
                       int64_t gen_rows) {
  SparsePlan p{};
  const int group = Hq / Hkv;
  const int64_t entries = S > 0 ? (int64_t)n_shards * topk : 0;
  const int64_t steps = steps_of(entries * block) + steps_of(gen_rows);
  p.tokens = union_tokens(Tq, Hkv, group, d, S > 0 ? n_shards * ((S + block - 1) / block) : 0,
                          entries, steps);
  const int64_t own = (int64_t)((Tq + p.tokens - 1) / p.tokens) * ((group + 15) / 16);
  const int64_t tiles = own * Hkv;
  const int64_t fill = tiles_at_once(d) / tiles, most = (steps + 3) / 4;
  p.waves = 4;
  p.parts = parts_at_once(std::min(fill, most), Hkv, own, tiles_at_once(d) / 8);
  if (p.tokens > 1 || p.parts == 1) return p;
  // Eight waves: for few steps in one part, so without a merge (4 x 8 blocks of 16 keys
  // and 46 rows, 18 steps: 7.2 us against 7.7 in five parts and a launch less); where the
  // workgroups fill the chip in fewer parts, as many as are one on each compute unit
  // (four waves / eight, us: 64 tiles of 67 steps 13.0 / 12.4, 128 of 68 15.4 / 14.5, 256
  // of 69 20.0 / 16.6, 176 of 130 30 / 26; at d 64 128 of 131 18.6 / 16.0, 384 of 71 18.8 /
  // 17.4).  But not for long lists in one part that leaves a third of the places idle, one
  // on each compute unit or, for more tiles than these, two at d 64: d 128, 168 tiles of
  // 60 / 100 / 260 steps 15.6 / 15.0, 21.5 / 22.4, 43 / 48, against 176 18.3 / 14.9, 25.1 /
  // 22.5, 58 / 48; d 64, 144 of 260 29 / 34, 336 40 / 46, against 400 48 / 46.  Nor, at d 64,
  // for long lists of more than 32 tokens, which read each other's blocks from cache, where
  // the four waves' twice as many help: 192 tiles of 260 steps that share a quarter, 96
  // tokens 28.6 / 33.9, 48 31 / 34, against 24 33 / 34, 12 45 / 37, and 256 of 32 tokens 38 /
  // 34.  (The same lists, 24 tokens, 26 / 31, lists of their own 45 / 37.)
  const int64_t places = tiles <= 256 ? 256 : 512;
  if (steps <= (d == 64 ? 40 : 32)) {
    p.waves = 8;
    p.parts = 1;
  } else if (fill < most) {
    const int parts = parts_at_once(std::min(256 / tiles, (steps + 7) / 8), Hkv, own, 32);
    if (parts == 1 && steps > 80 && 3 * tiles < 2 * places) return p;
    if (d == 64 && parts == 1 && tiles <= 256 && steps > 160 && Tq > 32) return p;
    p.waves = 8;
    p.parts = parts;
  }
  return p;
}

// Rows of partials (tokens times parts) of any call of up to Tq tokens.
int64_t sparse_part_rows_most(int Tq, int Hq, int Hkv, int d) {
  if (Tq <= 0) return 0;
  // of tiles of several tokens: all of a tile's tokens have its parts
  return (int64_t)tiles_at_once(d) / Hkv * std::min(std::max(tile_tokens_most(Hq / Hkv, d), 1), Tq);
}

namespace {
SparseArgs tile_args(const SparseLaunch& x, int tokens, int parts) {
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
  a.tile_tokens = tokens;
  a.token_tiles = (x.Tq + tokens - 1) / tokens;
  a.col_tiles = (a.group + 15) / 16;
  a.n_shards = x.n_shards;
  a.G = x.G;
  a.parts = parts;
  a.slices = tile_slices((int64_t)x.Hkv * parts, (int64_t)a.token_tiles * a.col_tiles);
  a.scale_log2 = x.scale * 1.4426950408889634f;
  return a;
}
}  // namespace

int launch_sparse(const SparseLaunch& x, const SparsePlan& p, void* o, int o_bf16, float* lse,
                  hipStream_t stream) {
  SparseArgs a = tile_args(x, p.tokens, p.parts);
  a.topk = x.topk;
  a.entries = x.S > 0 ? x.n_shards * x.topk : 0;
  a.half_log2 = __builtin_ctz(x.block) - 4;
  a.blocks = (int)((x.S + x.block - 1) / x.block);
  if (a.entries == 0) a.n_shards = 0;
  a.gen_rows = x.Kg != nullptr ? (int)(x.G + x.Tq) : 0;
  a.S = x.S;
  a.list_steps = (int)steps_of((int64_t)a.entries * x.block);
  const int64_t steps = a.list_steps + steps_of(a.gen_rows);
  a.part_steps = (int)std::max<int64_t>(1, (steps + p.parts - 1) / p.parts);
  a.O = o;
  a.o_bf16 = o_bf16;
  a.lse = lse;
  if (p.tokens > std::max(16 / a.group, 1)) return launch_tiles<128, 4, SP_UNION, 2>(a, stream);
  if (p.tokens > 1)
    return x.d == 128 ? launch_tiles<128, 4, SP_UNION>(a, stream)
                      : launch_tiles<64, 4, SP_UNION>(a, stream);
  if (p.waves == 8)
    return x.d == 128 ? launch_tiles<128, 8, SP_LISTED>(a, stream)
                      : launch_tiles<64, 8, SP_LISTED>(a, stream);
  return x.d == 128 ? launch_tiles<128, 4, SP_LISTED>(a, stream)
                    : launch_tiles<64, 4, SP_LISTED>(a, stream);
}

// Partials of all tokens over all rows of the shards and the first G appended rows.
bool dense_tiles_apply(int Hq, int Hkv) { return Hq / Hkv <= 16; }
static SparsePlan dense_plan(int64_t keys, int Tq, int64_t G, int Hq, int Hkv, int d) {
  SparsePlan p{};
  p.tokens = 16 / (Hq / Hkv);
  const int64_t own = (Tq + p.tokens - 1) / p.tokens, tiles = own * Hkv;
  const int64_t steps = steps_of(keys) + steps_of(G);
  p.waves = 4;
  p.parts = parts_at_once(std::min(tiles_at_once(d) / tiles, (steps + 3) / 4), Hkv, own,
                          tiles_at_once(d) / 8);
  // Eight waves where that is a workgroup for 112 compute units at least and, unless the
  // steps end before the parts do, in long ranges for four fifths of them.  With the merge,
  // four waves / eight, us: 32 / 8 heads of 128 over 4 x 1021 keys, 8 tiles (128 workgroups)
  // 11.9 / 11.1, 64 (256) 18.7 / 17.1; 8 / 2 heads over 4 x 1021, 6 tiles (96) 10.8 / 11.0; 96
  // tiles (192) of 32 / 8 over 2048 keys 19.7 / 18.5, 4 x 1021 22.8 / 22.7, 8192 30.9 / 33.5,
  // 80 (240) over 8192 27.1 / 27.0; 16 / 8 of 64, 96 over 4 x 1021 19.6 / 18.7.  Over 145 shapes
  // the choice is 0.1 % slower than the better one of both on average, and 4 % at most.
  if (tiles <= 256) {
    const int parts = parts_at_once(std::min(256 / tiles, (steps + 7) / 8), Hkv, own, 32);
    const int64_t nwg = tiles * parts;
    if (nwg >= 112 && (nwg >= 205 || steps <= std::max(160, 8 * parts))) {
      p.waves = 8;
      p.parts = parts;
    }
  }
  return p;
}
int dense_parts(int n_shards, int Tq, int64_t S, int64_t G, int Hq, int Hkv, int d) {
  return dense_plan(n_shards * S, Tq, G, Hq, Hkv, d).parts;
}
// Rows of partials of any call of up to Tq tokens: a part of every token, or the
// chip's workgroups' tiles.
int64_t dense_part_rows_most(int Tq, int Hq, int Hkv, int d) {
  const int tokens = 16 / (Hq / Hkv);
  return std::max<int64_t>(Tq, (int64_t)tiles_at_once(d) / Hkv * std::min(tokens, Tq));
}
int launch_dense(const SparseLaunch& x, int parts, float* o, float* lse, hipStream_t stream) {
  SparseArgs a = tile_args(x, 16 / (x.Hq / x.Hkv), parts);
  a.S = x.n_shards * x.S;
  a.gen_rows = (int)x.G;
  a.list_steps = (int)steps_of(a.S);
  const int64_t steps = a.list_steps + steps_of(x.G);
  a.part_steps = (int)std::max<int64_t>(1, (steps + parts - 1) / parts);
  a.O = o;
  a.lse = lse;
  if (dense_plan(a.S, x.Tq, x.G, x.Hq, x.Hkv, x.d).waves == 8)
    return x.d == 128 ? launch_tiles<128, 8, SP_DENSE>(a, stream)
                      : launch_tiles<64, 8, SP_DENSE>(a, stream);
  return x.d == 128 ? launch_tiles<128, 4, SP_DENSE>(a, stream)
                    : launch_tiles<64, 4, SP_DENSE>(a, stream);
}
