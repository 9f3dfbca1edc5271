// C ABI entry points of block-sparse Phase 2 and of drafted tokens: host-side
// validation, then kernel launches.  (pulsar_phase2_tree shares the plans of
// pulsar_phase2_query and stands with it.)
#include <math.h>

#include <algorithm>

#include "common.hpp"

namespace {

constexpr int64_t kMaxInt = 0x7fffffff;
constexpr int kMaxTree = 16384;  // drafts whose parents fit a workgroup's LDS

bool block_supported(int block) {
  return block >= 16 && block <= 256 && (block & (block - 1)) == 0;
}

}  // namespace

extern "C" {

int pulsar_tree_mask(const int32_t* parent, int T, uint32_t* mask, int32_t* depth, void* stream) {
  if (T < 0) return PULSAR_EINVAL;
  if (T > kMaxTree) return PULSAR_EUNSUPPORTED;
  if (T == 0) return PULSAR_OK;
  if (parent == nullptr || mask == nullptr) return PULSAR_EINVAL;
  return launch_tree_mask(parent, T, mask, depth, (hipStream_t)stream);
}

int pulsar_kv_compact(void* K, void* V, int layers, int64_t capacity, int Hkv, int d, int64_t G,
                      const int32_t* keep, int n, void* stream) {
  if (layers < 0 || capacity < 0 || Hkv < 1 || d < 1 || G < 0 || G > capacity || n < 0)
    return PULSAR_EINVAL;
  if (n > capacity - G) return PULSAR_EINVAL;
  if ((int64_t)Hkv * d % 8 != 0) return PULSAR_EUNSUPPORTED;
  if ((int64_t)layers * Hkv * d / 8 > kMaxInt || (int64_t)Hkv * d * 2 > kMaxInt)
    return PULSAR_EUNSUPPORTED;
  if (layers == 0 || n == 0) return PULSAR_OK;
  if (K == nullptr || V == nullptr || keep == nullptr) return PULSAR_EINVAL;
  if (!aligned16(K) || !aligned16(V)) return PULSAR_EINVAL;
  return launch_kv_compact(K, V, layers, capacity, (int64_t)Hkv * d * 2, G, keep, n,
                           (hipStream_t)stream);
}

int pulsar_key_bounds(const void* K, int n_shards, int64_t S, int Hkv, int d, int block,
                      void* bounds, void* stream) {
  if (n_shards < 0 || S < 0 || Hkv < 1 || d < 1 || block < 1) return PULSAR_EINVAL;
  if ((d != 64 && d != 128) || !block_supported(block)) return PULSAR_EUNSUPPORTED;
  if (S > kMaxInt || (int64_t)Hkv * d > kMaxInt) return PULSAR_EUNSUPPORTED;
  if (n_shards == 0 || S == 0) return PULSAR_OK;
  if (K == nullptr || bounds == nullptr || !aligned16(K) || !aligned16(bounds))
    return PULSAR_EINVAL;
  return launch_key_bounds(static_cast<const uint16_t*>(K), n_shards, S, Hkv, d, block,
                           static_cast<uint16_t*>(bounds), (hipStream_t)stream);
}

size_t pulsar_block_select_workspace_bytes(int n_shards, int Tq, int blocks, int Hq, int Hkv) {
  if (n_shards < 0 || Tq < 0 || blocks < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return 0;
  if (select_fused(Tq, blocks, Hq / Hkv)) return 0;
  return (size_t)n_shards * Hkv * ((size_t)Tq * blocks + (blocks + 15) / 16) * 4;
}

int pulsar_block_select(const void* q, const void* bounds, int n_shards, int Tq, int blocks, int Hq,
                        int Hkv, int d, int topk, int32_t* sel, float* scores, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (n_shards < 0 || Tq < 0 || blocks < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1)
    return PULSAR_EINVAL;
  if (topk < 0 || topk > blocks) return PULSAR_EINVAL;
  if (d != 64 && d != 128) return PULSAR_EUNSUPPORTED;
  if (blocks > kMaxSelectBlocks || Tq >= PULSAR_MAX_ROWS) return PULSAR_EUNSUPPORTED;
  const int64_t rows = (int64_t)n_shards * Tq * Hkv;
  if (!grid_fits(rows, blocks > 4096 ? 1024 : 512) || (int64_t)n_shards * Hkv > 65535 ||
      Tq > (Hq / Hkv > 16 ? 65535 : 65535 * 8))
    return PULSAR_EUNSUPPORTED;
  if (rows == 0 || blocks == 0 || (topk == 0 && scores == nullptr)) return PULSAR_OK;
  if (q == nullptr || bounds == nullptr || (topk > 0 && sel == nullptr)) return PULSAR_EINVAL;
  if (!aligned16(q) || !aligned16(bounds)) return PULSAR_EINVAL;
  PickLaunch a{};
  a.q = static_cast<const uint16_t*>(q);
  a.bounds = static_cast<const uint16_t*>(bounds);
  a.n_shards = n_shards;
  a.Tq = Tq;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.blocks = blocks;
  a.topk = topk;
  a.sel = sel;
  if (scores != nullptr) {
    const int st = launch_block_scores(a.q, a.bounds, n_shards, Tq, Hq, Hkv, d, blocks, scores,
                                       (hipStream_t)stream);
    if (st != PULSAR_OK || topk == 0) return st;
    a.scores = scores;
  } else if (!select_fused(Tq, blocks, Hq / Hkv)) {
    if (workspace == nullptr || !aligned16(workspace) ||
        workspace_bytes < pulsar_block_select_workspace_bytes(n_shards, Tq, blocks, Hq, Hkv))
      return PULSAR_EWORKSPACE;
    float* const near = static_cast<float*>(workspace);
    float* const norms = near + rows * blocks;
    const int st = launch_block_near(a.q, a.bounds, n_shards, Tq, Hq, Hkv, d, blocks, near, norms,
                                     (hipStream_t)stream);
    if (st != PULSAR_OK) return st;
    a.scores = near;
    a.norms = norms;
  }
  return launch_block_pick(a, (hipStream_t)stream);
}

size_t pulsar_phase2_sparse_workspace_bytes(int Tq, int Hq, int Hkv, int d) {
  if (Tq < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1) return 0;
  return (size_t)sparse_part_rows_most(Tq, Hq, Hkv, d) * Hq * (d + 1) * 4;
}

size_t pulsar_phase2_sparse_call_bytes(int n_shards, int Tq, int64_t S, int block, int topk,
                                       int64_t gen_rows, int Hq, int Hkv, int d) {
  if (n_shards < 0 || Tq < 1 || S < 0 || topk < 0 || gen_rows < 0 || Hq < 1 || Hkv < 1 ||
      Hq % Hkv != 0 || (d != 64 && d != 128) || !block_supported(block))
    return 0;
  const int parts = sparse_plan(n_shards, Tq, S, Hq, Hkv, d, block, topk, gen_rows).parts;
  return parts == 1 ? 0 : (size_t)parts * Tq * Hq * (d + 1) * 4;
}

int pulsar_phase2_sparse(const void* q, const void* K, const void* V, const int32_t* sel,
                         int n_shards, int Tq, int64_t S, int block, int topk, const void* Kg,
                         const void* Vg, int64_t G, const uint32_t* mask, int Hq, int Hkv, int d,
                         float softmax_scale, void* o, int o_dtype, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (n_shards < 0 || Tq < 0 || S < 0 || G < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1 ||
      block < 1 || topk < 0)
    return PULSAR_EINVAL;
  if (!(softmax_scale > 0.f) || !isfinite(softmax_scale)) return PULSAR_EINVAL;
  if (o_dtype != PULSAR_OUT_F32 && o_dtype != PULSAR_OUT_BF16) return PULSAR_EINVAL;
  if ((Kg == nullptr) != (Vg == nullptr) || (Kg == nullptr && (G > 0 || mask != nullptr)))
    return PULSAR_EINVAL;
  if ((d != 64 && d != 128) || !block_supported(block)) return PULSAR_EUNSUPPORTED;
  if (S > kMaxInt || Tq >= PULSAR_MAX_ROWS || G + Tq >= PULSAR_MAX_ROWS ||
      (int64_t)Hkv * d * 2 >= 1 << 24)
    return PULSAR_EUNSUPPORTED;
  const int64_t keys = S > 0 ? (int64_t)n_shards * topk * block : 0;
  if (keys >= 1 << 30) return PULSAR_EUNSUPPORTED;
  if (Tq == 0) return PULSAR_OK;
  if (q == nullptr || o == nullptr || !aligned16(q) || !aligned16(o)) return PULSAR_EINVAL;
  if (keys > 0 && (K == nullptr || V == nullptr || sel == nullptr || !aligned16(K) ||
                   !aligned16(V)))
    return PULSAR_EINVAL;
  if (Kg != nullptr && (!aligned16(Kg) || !aligned16(Vg))) return PULSAR_EINVAL;

  const int64_t gen_rows = Kg != nullptr ? G + Tq : 0;
  const SparsePlan plan = sparse_plan(n_shards, Tq, S, Hq, Hkv, d, block, topk, gen_rows);
  const int parts = plan.parts;
  SparseLaunch a{};
  a.q = static_cast<const uint16_t*>(q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.sel = sel;
  a.Kg = static_cast<const uint16_t*>(Kg);
  a.Vg = static_cast<const uint16_t*>(Vg);
  a.mask = mask;
  a.n_shards = n_shards;
  a.Tq = Tq;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.topk = topk;
  a.block = block;
  a.S = S;
  a.G = G;
  a.scale = softmax_scale;
  const bool bf16 = o_dtype == PULSAR_OUT_BF16;
  if (parts == 1) return launch_sparse(a, plan, o, bf16, lse, (hipStream_t)stream);

  const int64_t orows = (int64_t)parts * Tq * Hq;
  if (workspace == nullptr || !aligned16(workspace) ||
      workspace_bytes < (size_t)orows * (d + 1) * 4)
    return PULSAR_EWORKSPACE;
  float* po = static_cast<float*>(workspace);
  float* pl = po + orows * d;
  const int st = launch_sparse(a, plan, po, false, pl, (hipStream_t)stream);
  if (st != PULSAR_OK) return st;
  return bf16 ? launch_lse_merge_bf16(po, pl, parts, Tq, Hq, d, o, lse, (hipStream_t)stream)
              : launch_lse_merge(po, pl, parts, 1, Tq, Hq, d, (int64_t)Tq * Hq * d,
                                 (int64_t)Hq * Tq, static_cast<float*>(o), lse,
                                 (hipStream_t)stream);
}

}  // extern "C"
