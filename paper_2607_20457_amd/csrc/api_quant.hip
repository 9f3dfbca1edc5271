// C ABI entry points of a cache held in 8 bits: host-side validation, then kernel
// launches.
#include <math.h>

#include <initializer_list>

#include "common.hpp"

namespace {

constexpr int64_t kMaxInt = 0x7fffffff;

bool quant_block(int block) { return block >= 16 && block <= 256 && (block & (block - 1)) == 0; }
bool quant_format(int format) { return format == PULSAR_KV_E4M3 || format == PULSAR_KV_INT8; }

// What both directions refuse of a cache and of its rows.
int check_rows(int n, int64_t rows, int Hkv, int d, int block, int format, int64_t first,
               int64_t capacity) {
  if (n < 0 || rows < 0 || Hkv < 1 || d < 1 || block < 1 || first < 0 || capacity < 0 ||
      !quant_format(format))
    return PULSAR_EINVAL;
  if (first > capacity || rows > capacity - first) return PULSAR_EINVAL;
  if ((d != 64 && d != 128) || !quant_block(block)) return PULSAR_EUNSUPPORTED;
  if (capacity > kMaxInt || (int64_t)Hkv * d >= 1 << 23 ||
      (__int128)n * capacity * Hkv * d >= (__int128)1 << 48)
    return PULSAR_EUNSUPPORTED;
  return PULSAR_OK;
}

// Memory [from, to), and whether two pieces of it have any in common.
struct Span {
  __int128 from, to;
};
bool meet(const Span& a, const Span& b) { return a.from < b.to && b.from < a.to; }
Span span(const void* p, __int128 bytes) {
  const __int128 at = (__int128) reinterpret_cast<uintptr_t>(p);
  return Span{at, at + bytes};
}
// bf16 rows of `width` values at these strides.
Span rows_span(const void* p, int n, int64_t rows, int64_t width, int64_t shard_stride,
               int64_t row_stride) {
  Span s = span(p, (__int128)width * 2);
  for (const __int128 far : {(__int128)(n - 1) * shard_stride * 2,
                             (__int128)(rows - 1) * row_stride * 2})
    (far < 0 ? s.from : s.to) += far;
  return s;
}

KvQuantLaunch cache_of(const void* k_codes, const void* v_codes, const float* k_scales,
                       const float* v_scales, int n, int64_t rows, int Hkv, int d, int block,
                       int format, int64_t first, int64_t capacity) {
  KvQuantLaunch a{};
  a.codes[0] = static_cast<uint8_t*>(const_cast<void*>(k_codes));
  a.codes[1] = static_cast<uint8_t*>(const_cast<void*>(v_codes));
  a.scales[0] = const_cast<float*>(k_scales);
  a.scales[1] = const_cast<float*>(v_scales);
  a.n = n;
  a.Hkv = Hkv;
  a.d = d;
  a.block = block;
  a.format = format;
  a.rows = rows;
  a.first = first;
  a.capacity = capacity;
  return a;
}

}  // namespace

extern "C" {

int pulsar_kv_quantize(const void* K, const void* V, int64_t shard_stride, int64_t row_stride,
                       int n, int64_t rows, int Hkv, int d, int block, int format, int64_t first,
                       int64_t capacity, void* k_codes, void* v_codes, float* k_scales,
                       float* v_scales, void* stream) {
  const int st = check_rows(n, rows, Hkv, d, block, format, first, capacity);
  if (st != PULSAR_OK) return st;
  if (first % block != 0) return PULSAR_EINVAL;
  if (n == 0 || rows == 0) return PULSAR_OK;
  if (K == nullptr || V == nullptr || k_codes == nullptr || v_codes == nullptr ||
      k_scales == nullptr || v_scales == nullptr)
    return PULSAR_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(k_codes) || !aligned16(v_codes) ||
      shard_stride % 8 != 0 || row_stride % 8 != 0)
    return PULSAR_EINVAL;
  const __int128 codes = (__int128)n * Hkv * capacity * d;
  const __int128 scales = (__int128)n * Hkv * ((capacity + block - 1) / block) * 4;
  const Span all[6] = {span(k_codes, codes),
                       span(v_codes, codes),
                       span(k_scales, scales),
                       span(v_scales, scales),
                       rows_span(K, n, rows, (int64_t)Hkv * d, shard_stride, row_stride),
                       rows_span(V, n, rows, (int64_t)Hkv * d, shard_stride, row_stride)};
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 6; ++j)
      if (meet(all[i], all[j])) return PULSAR_EINVAL;
  KvQuantLaunch a = cache_of(k_codes, v_codes, k_scales, v_scales, n, rows, Hkv, d, block, format,
                             first, capacity);
  a.X[0] = static_cast<const uint16_t*>(K);
  a.X[1] = static_cast<const uint16_t*>(V);
  a.shard_stride = shard_stride;
  a.row_stride = row_stride;
  return launch_quantize(a, (hipStream_t)stream);
}

int pulsar_kv_dequantize(const void* k_codes, const void* v_codes, const float* k_scales,
                         const float* v_scales, int n, int64_t capacity, int Hkv, int d, int block,
                         int format, int64_t first, int64_t rows, void* K, void* V, void* stream) {
  const int st = check_rows(n, rows, Hkv, d, block, format, first, capacity);
  if (st != PULSAR_OK) return st;
  if (n == 0 || rows == 0) return PULSAR_OK;
  if (K == nullptr || V == nullptr || k_codes == nullptr || v_codes == nullptr ||
      k_scales == nullptr || v_scales == nullptr)
    return PULSAR_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(k_codes) || !aligned16(v_codes))
    return PULSAR_EINVAL;
  const KvQuantLaunch a = cache_of(k_codes, v_codes, k_scales, v_scales, n, rows, Hkv, d, block,
                                   format, first, capacity);
  uint16_t* const out[2] = {static_cast<uint16_t*>(K), static_cast<uint16_t*>(V)};
  return launch_dequantize(a, out, (hipStream_t)stream);
}

size_t pulsar_phase2_quant_workspace_bytes(int Tq, int Hq, int Hkv, int d) {
  if (Tq < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1) return 0;
  return (size_t)quant_part_rows_most(Tq, Hq, Hkv) * Hq * (d + 1) * 4;
}

size_t pulsar_phase2_quant_call_bytes(int n_shards, int Tq, int64_t S, int64_t gen_rows, int Hq,
                                      int Hkv, int d) {
  if (n_shards < 0 || Tq < 1 || S < 0 || S > kMaxInt || gen_rows < 0 || Hq < 1 || Hkv < 1 ||
      Hq % Hkv != 0 || (d != 64 && d != 128))
    return 0;
  const int parts = quant_plan(n_shards, Tq, S, Hq, Hkv, d, gen_rows).parts;
  return parts == 1 ? 0 : (size_t)parts * Tq * Hq * (d + 1) * 4;
}

int pulsar_phase2_quant(const void* q, const void* k_codes, const void* v_codes,
                        const float* k_scales, const float* v_scales, int n_shards, int Tq,
                        int64_t S, int block, int format, const int32_t* rows, const void* Kg,
                        const void* Vg, int64_t G, const uint32_t* mask, int Hq, int Hkv, int d,
                        float softmax_scale, void* o, int o_dtype, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (n_shards < 0 || Tq < 0 || S < 0 || G < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1 ||
      block < 1 || !quant_format(format))
    return PULSAR_EINVAL;
  if (!(softmax_scale > 0.f) || !isfinite(softmax_scale)) return PULSAR_EINVAL;
  if (o_dtype != PULSAR_OUT_F32 && o_dtype != PULSAR_OUT_BF16) return PULSAR_EINVAL;
  if ((Kg == nullptr) != (Vg == nullptr) || (Kg == nullptr && (G > 0 || mask != nullptr)))
    return PULSAR_EINVAL;
  if ((d != 64 && d != 128) || !quant_block(block)) return PULSAR_EUNSUPPORTED;
  if (S > kMaxInt || Tq >= PULSAR_MAX_ROWS || G >= PULSAR_MAX_ROWS || G + Tq >= PULSAR_MAX_ROWS ||
      (int64_t)Hkv * d * 2 >= 1 << 24 || (int64_t)n_shards * S > kMaxInt ||
      (int64_t)n_shards * ((S + 31) / 32) >= 1 << 30)
    return PULSAR_EUNSUPPORTED;
  const bool keys = n_shards > 0 && S > 0;
  if (keys && rows != nullptr && n_shards > kMaxQuantShards) return PULSAR_EUNSUPPORTED;
  if (Tq == 0) return PULSAR_OK;
  if (q == nullptr || o == nullptr || !aligned16(q) || !aligned16(o)) return PULSAR_EINVAL;
  if (keys && (k_codes == nullptr || v_codes == nullptr || k_scales == nullptr ||
               v_scales == nullptr || !aligned16(k_codes) || !aligned16(v_codes)))
    return PULSAR_EINVAL;
  if (Kg != nullptr && (!aligned16(Kg) || !aligned16(Vg))) return PULSAR_EINVAL;

  QuantAttnLaunch a{};
  a.q = static_cast<const uint16_t*>(q);
  a.K = static_cast<const uint8_t*>(k_codes);
  a.V = static_cast<const uint8_t*>(v_codes);
  a.ks = k_scales;
  a.vs = v_scales;
  a.rows = rows;
  a.Kg = static_cast<const uint16_t*>(Kg);
  a.Vg = static_cast<const uint16_t*>(Vg);
  a.mask = mask;
  a.n_shards = keys ? n_shards : 0;
  a.Tq = Tq;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.block = block;
  a.format = format;
  a.S = keys ? S : 0;
  a.G = G;
  a.scale = softmax_scale;
  const QuantPlan plan =
      quant_plan(a.n_shards, Tq, a.S, Hq, Hkv, d, Kg != nullptr ? G + Tq : 0);
  const int parts = plan.parts;
  const bool bf16 = o_dtype == PULSAR_OUT_BF16;
  if (parts == 1) return launch_quant_attn(a, plan, o, bf16, lse, (hipStream_t)stream);

  const int64_t orows = (int64_t)parts * Tq * Hq;
  if (workspace == nullptr || !aligned16(workspace) ||
      workspace_bytes < (size_t)orows * (d + 1) * 4)
    return PULSAR_EWORKSPACE;
  float* po = static_cast<float*>(workspace);
  float* pl = po + orows * d;
  const int st = launch_quant_attn(a, plan, po, false, pl, (hipStream_t)stream);
  if (st != PULSAR_OK) return st;
  return bf16 ? launch_lse_merge_bf16(po, pl, parts, Tq, Hq, d, o, lse, (hipStream_t)stream)
              : launch_lse_merge(po, pl, parts, 1, Tq, Hq, d, (int64_t)Tq * Hq * d,
                                 (int64_t)Hq * Tq, static_cast<float*>(o), lse,
                                 (hipStream_t)stream);
}

}  // extern "C"
