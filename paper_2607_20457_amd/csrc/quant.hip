// A cache held in 8 bits: rows quantised as they are written, and read back.
//
// Codes are e4m3 or int8, [n][head][row][d], so that a head's rows lie one after
// another and a reader of one head streams them; a scale for each block of rows and
// head, [n][head][block], fp32.  The scale is 2^e with the least e >= -100 for which
// the block's largest magnitude is at most 448 * 2^e (e4m3) or 127 * 2^e (int8), and a
// code the nearest to x / 2^e, ties to even: one rounding, since bf16 divides by a power
// of two exactly; and code * 2^e is a bf16 number, so that reading back rounds nothing.
// (A scale of amax / 448 costs e4m3 as much precision on average, two roundings more;
// for int8 amax / 127 would have steps smaller by 2^(1/2) on average.)
#include <type_traits>

#include "common.hpp"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int QZ_WAVES = 4;
constexpr int QZ_ROWS = 64;  // rows of a wave

struct QuantizeArgs {
  const uint16_t* X[2];  // K and V: bf16, rows of Hkv * D at these strides (in elements)
  int64_t shard_stride, row_stride;
  uint8_t* codes[2];     // [n, Hkv, capacity, D]
  float* scales[2];      // [n, Hkv, blocks]
  int Hkv;
  int64_t rows, first, capacity, blocks;
  int block_log2;
  uint32_t row_groups;   // workgroups over the rows of a shard
  uint32_t head_groups;  // and over its heads
  int waves_log2;        // log2 of a block's waves
  int once;              // more rows than the caches hold
};

// The largest 16-bit magnitude of both halves of x, over all lanes.
__device__ __forceinline__ uint32_t wave_max_bits(u16x2 x) {
  uint32_t m = x[0] > x[1] ? x[0] : x[1];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)m, off, 64);
    m = y > m ? y : m;
  }
  return m;
}

// Eight bf16 values as codes.  s = 2^e.
template <int FORMAT>
__device__ __forceinline__ u32x2 encode(u32x4 w, float s, float inv) {
  u32x2 out;
  if constexpr (FORMAT == PULSAR_KV_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t lo = w[2 * i], hi = w[2 * i + 1];
      s16x2 c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, lo), s, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, hi), s, true);
      out[i] = __builtin_bit_cast(uint32_t, c);
    }
  } else {
    // x / s + 1.5 * 2^23, rounded once, holds the code in its low byte
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16;
      t[i] = __float_as_uint(__builtin_fmaf(__uint_as_float(bits), inv, 12582912.f));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t lo = __builtin_amdgcn_perm(t[4 * i + 1], t[4 * i], 0x0c0c0400u);
      const uint32_t hi = __builtin_amdgcn_perm(t[4 * i + 3], t[4 * i + 2], 0x0c0c0400u);
      out[i] = lo | hi << 16;
    }
  }
  return out;
}

// Bound by HBM.  Workgroup: 64 rows of four heads, or of fewer heads where a block has
// more rows.  A wave holds its 64 rows of one head in registers, so that each value is
// read once; blocks of more rows exchange their magnitudes through LDS.  Four heads side
// by side are 1 KiB of a row of the source.  K and V of 16 x 8192 rows of 8 heads of 128
// (805 MB): 141 us, 134 with stores that pass the caches by, 124 (6.5 TB/s) where from 256
// MB on the loads do so too; below, where the rows may lie in the last-level cache, those
// loads lose (5 x 3001 rows of 16 heads of 64, 61 MB of K and V: 16.3 / 18.4).
template <int D, int FORMAT>
__global__ __launch_bounds__(64 * QZ_WAVES) void quantize_kernel(QuantizeArgs a) {
  constexpr int CPR = D / 8;          // 16-byte chunks per row
  constexpr int SEG = 64 / CPR;       // rows of a load
  constexpr int LOADS = QZ_ROWS / SEG;
  __shared__ uint32_t s_max[QZ_WAVES];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int which = blockIdx.x & 1;
  const uint32_t wg = blockIdx.x >> 1, groups = wg / a.head_groups;
  const int hg = (int)(wg - groups * a.head_groups);
  const int64_t shard = groups / a.row_groups, rg = groups - (uint32_t)shard * a.row_groups;
  const int per_head = 1 << a.waves_log2;
  const int head = hg * (QZ_WAVES >> a.waves_log2) + (wave >> a.waves_log2);
  const int64_t row0 = (rg * per_head + (wave & (per_head - 1))) * QZ_ROWS;
  const bool live = head < a.Hkv;
  const int at = lane % CPR;

  u32x4 w[LOADS];
  const uint16_t* const x = a.X[which] + shard * a.shard_stride + (int64_t)head * D + 8 * at;
  auto load = [&](auto once) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int64_t row = row0 + i * SEG + lane / CPR;
      const u32x4* const from = reinterpret_cast<const u32x4*>(x + row * a.row_stride);
      w[i] = u32x4{0u, 0u, 0u, 0u};
      if (live && row < a.rows) {
        if constexpr (decltype(once)::value) w[i] = __builtin_nontemporal_load(from);
        else w[i] = *from;
      }
    }
  };
  if (a.once) load(std::true_type{});
  else load(std::false_type{});
  const int64_t plane = shard * a.Hkv + head;
  uint8_t* const out = a.codes[which] + (plane * a.capacity + a.first + row0) * D + 8 * at;
  float* const scales =
      a.scales[which] + plane * a.blocks + ((a.first + row0) >> a.block_log2);
  // one block of rows of the wave: loads I0 .. I1, block nth of them
  auto finish = [&](auto from, auto to, uint32_t top, int nth, bool writes) {
    constexpr int I0 = decltype(from)::value, I1 = decltype(to)::value;
    const int exponent = (int)(top >> 7), fraction = (int)(top & 127);
    const bool bad = exponent == 255;  // a NaN or an infinity
    constexpr int kMost = FORMAT == PULSAR_KV_E4M3 ? 8 : 6;       // 448 = 1.75 * 2^8, 127 =
    constexpr int kFraction = FORMAT == PULSAR_KV_E4M3 ? 96 : 126;  // (1 + 126 / 128) * 2^6
    int e = exponent - 127 - kMost + (fraction > kFraction);
    e = e < -100 ? -100 : e;
    const float s = __uint_as_float((uint32_t)(e + 127) << 23);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    // the largest scale's codes stop where code * s is still finite: at 240 and 63
    constexpr int kLast = FORMAT == PULSAR_KV_E4M3 ? 120 : 122;
    constexpr uint32_t kCut = FORMAT == PULSAR_KV_E4M3 ? 0x7f70u : 0x7f7cu;
#pragma unroll
    for (int i = I0; i < I1; ++i) {
      u32x4 y = w[i];
      if (e == kLast) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const u16x2 m = __builtin_elementwise_min(
              __builtin_bit_cast(u16x2, y[k] & 0x7fff7fffu), u16x2{kCut, kCut});
          y[k] = (y[k] & 0x80008000u) | __builtin_bit_cast(uint32_t, m);
        }
      }
      u32x2 c = encode<FORMAT>(y, s, inv);
      if (bad) c = u32x2{0u, 0u};
      if (live && row0 + i * SEG + lane / CPR < a.rows)
        __builtin_nontemporal_store(c,
                                    reinterpret_cast<u32x2*>(out + (i * SEG + lane / CPR) * D));
    }
    if (writes && live && lane == 0) scales[nth] = bad ? __uint_as_float(0x7fc00000u) : s;
  };
  auto magnitude = [&](auto from, auto to) {
    constexpr int I0 = decltype(from)::value, I1 = decltype(to)::value;
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = I0; i < I1; ++i) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i][k] & 0x7fff7fffu));
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_max_bits(m));
  };
  // blocks of 16, 32 or 64 rows: block B of the wave, and those after it
  auto blocks_from = [&](auto self, auto per_tag, auto nth_tag) -> void {
    constexpr int PER = decltype(per_tag)::value, B = decltype(nth_tag)::value;
    if constexpr (B * PER < LOADS) {
      const std::integral_constant<int, B * PER> from{};
      const std::integral_constant<int, (B + 1) * PER> to{};
      finish(from, to, magnitude(from, to), B, row0 + B * PER * SEG < a.rows);
      self(self, per_tag, std::integral_constant<int, B + 1>{});
    }
  };
  const std::integral_constant<int, 0> zero{};
  const std::integral_constant<int, LOADS> all{};
  if (a.waves_log2 > 0) {
    const uint32_t mine = magnitude(zero, all);
    if (lane == 0) s_max[wave] = mine;
    __syncthreads();
    uint32_t top = 0;
    for (int k = 0; k < per_head; ++k) top = max(top, s_max[(wave & ~(per_head - 1)) + k]);
    top = __builtin_amdgcn_readfirstlane(top);
    finish(zero, all, top, 0, (wave & (per_head - 1)) == 0 && row0 < a.rows);
  } else if (a.block_log2 == 6) {
    blocks_from(blocks_from, std::integral_constant<int, 64 / SEG>{}, zero);
  } else if (a.block_log2 == 5) {
    blocks_from(blocks_from, std::integral_constant<int, 32 / SEG>{}, zero);
  } else {
    blocks_from(blocks_from, std::integral_constant<int, 16 / SEG>{}, zero);
  }
}

struct DequantizeArgs {
  const uint8_t* codes[2];  // [n, Hkv, capacity, D]
  const float* scales[2];   // [n, Hkv, blocks]
  uint16_t* X[2];           // bf16 [n, rows, Hkv, D]
  int Hkv;
  int64_t rows, first, capacity, blocks;
  int block_log2;
  uint32_t row_groups, head_groups;
};

// The quantiser's shape the other way: a wave reads 64 rows of one head, four heads side
// by side write 1 KiB of a row.  A lane takes 8 codes, 16 bytes of output.  16 x 8192 rows
// of 8 heads of 128 (805 MB): 149 us, 5.4 TB/s (a copy: 5.0); with stores that pass the
// caches by, 4 x 1021 rows 6.4 us against 8.5, 32768 rows 35.5 against 40.8.
template <int D, int FORMAT>
__global__ __launch_bounds__(64 * QZ_WAVES, 4) void dequantize_kernel(DequantizeArgs a) {
  constexpr int CPR = D / 8;
  constexpr int SEG = 64 / CPR;
  constexpr int LOADS = QZ_ROWS / SEG;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int which = blockIdx.x & 1;
  const uint32_t wg = blockIdx.x >> 1, groups = wg / a.head_groups;
  const int head = (int)(wg - groups * a.head_groups) * QZ_WAVES + wave;
  const int64_t shard = groups / a.row_groups;
  const int64_t row0 = (int64_t)(groups - (uint32_t)shard * a.row_groups) * QZ_ROWS;
  if (head >= a.Hkv) return;
  const int at = lane % CPR;
  const int64_t plane = shard * a.Hkv + head;
  const uint8_t* const in = a.codes[which] + (plane * a.capacity + a.first + row0) * D + 8 * at;
  const float* const scales = a.scales[which] + plane * a.blocks;
  uint16_t* const out =
      a.X[which] + ((shard * a.rows + row0) * a.Hkv + head) * D + 8 * at;
  u32x2 c[LOADS];
  float s[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = i * SEG + lane / CPR;
    c[i] = u32x2{0u, 0u};
    s[i] = 0.f;
    if (row0 + r < a.rows) {
      c[i] = *reinterpret_cast<const u32x2*>(in + r * D);
      s[i] = scales[(a.first + row0 + r) >> a.block_log2];
    }
  }
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = i * SEG + lane / CPR;
    f32x8 y;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if constexpr (FORMAT == PULSAR_KV_E4M3) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i][k], false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i][k], true);
        y[4 * k] = lo[0], y[4 * k + 1] = lo[1], y[4 * k + 2] = hi[0], y[4 * k + 3] = hi[1];
      } else {
#pragma unroll
        for (int b = 0; b < 4; ++b) y[4 * k + b] = (float)((int)(c[i][k] << (24 - 8 * b)) >> 24);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] *= s[i];
    if (row0 + r < a.rows)
      __builtin_nontemporal_store(
          __builtin_bit_cast(u32x4, __builtin_convertvector(y, bf16x8)),
          reinterpret_cast<u32x4*>(out + (int64_t)r * a.Hkv * D));
  }
}

}  // namespace

int launch_quantize(const KvQuantLaunch& x, hipStream_t stream) {
  QuantizeArgs a{};
  for (int i = 0; i < 2; ++i) {
    a.X[i] = x.X[i];
    a.codes[i] = x.codes[i];
    a.scales[i] = x.scales[i];
  }
  a.shard_stride = x.shard_stride;
  a.row_stride = x.row_stride;
  a.Hkv = x.Hkv;
  a.rows = x.rows;
  a.first = x.first;
  a.capacity = x.capacity;
  a.block_log2 = __builtin_ctz(x.block);
  a.blocks = (x.capacity + x.block - 1) >> a.block_log2;
  a.waves_log2 = a.block_log2 > 6 ? a.block_log2 - 6 : 0;
  const int heads = QZ_WAVES >> a.waves_log2, rows = QZ_ROWS << a.waves_log2;
  a.head_groups = (x.Hkv + heads - 1) / heads;
  a.row_groups = (uint32_t)((x.rows + rows - 1) / rows);
  a.once = (int64_t)x.n * x.rows * x.Hkv * x.d * 4 >= 256 << 20;
  const int64_t nwg = 2 * (int64_t)x.n * a.row_groups * a.head_groups;
  if (!grid_fits(nwg, 64 * QZ_WAVES)) return PULSAR_EUNSUPPORTED;
  const bool e4m3 = x.format == PULSAR_KV_E4M3;
  const auto kern = x.d == 128 ? (e4m3 ? quantize_kernel<128, PULSAR_KV_E4M3>
                                       : quantize_kernel<128, PULSAR_KV_INT8>)
                               : (e4m3 ? quantize_kernel<64, PULSAR_KV_E4M3>
                                       : quantize_kernel<64, PULSAR_KV_INT8>);
  hipLaunchKernelGGL(kern, dim3((unsigned)nwg), dim3(64 * QZ_WAVES), 0, stream, a);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}

int launch_dequantize(const KvQuantLaunch& x, uint16_t* const (&out)[2], hipStream_t stream) {
  DequantizeArgs a{};
  for (int i = 0; i < 2; ++i) {
    a.X[i] = out[i];
    a.codes[i] = x.codes[i];
    a.scales[i] = x.scales[i];
  }
  a.Hkv = x.Hkv;
  a.rows = x.rows;
  a.first = x.first;
  a.capacity = x.capacity;
  a.block_log2 = __builtin_ctz(x.block);
  a.blocks = (x.capacity + x.block - 1) >> a.block_log2;
  a.head_groups = (x.Hkv + QZ_WAVES - 1) / QZ_WAVES;
  a.row_groups = (uint32_t)((x.rows + QZ_ROWS - 1) / QZ_ROWS);
  const int64_t nwg = 2 * (int64_t)x.n * a.row_groups * a.head_groups;
  if (!grid_fits(nwg, 64 * QZ_WAVES)) return PULSAR_EUNSUPPORTED;
  const bool e4m3 = x.format == PULSAR_KV_E4M3;
  const auto kern = x.d == 128 ? (e4m3 ? dequantize_kernel<128, PULSAR_KV_E4M3>
                                       : dequantize_kernel<128, PULSAR_KV_INT8>)
                               : (e4m3 ? dequantize_kernel<64, PULSAR_KV_E4M3>
                                       : dequantize_kernel<64, PULSAR_KV_INT8>);
  hipLaunchKernelGGL(kern, dim3((unsigned)nwg), dim3(64 * QZ_WAVES), 0, stream, a);
  return hipGetLastError() == hipSuccess ? PULSAR_OK : PULSAR_EHIP;
}
