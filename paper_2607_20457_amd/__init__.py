"""Pulsar Attention Phase-1 / Phase-2 hot path for MI355X (gfx950).

The computation lives in ``libpulsar.so`` (HIP kernels behind the C ABI of
``include/pulsar.h``); ``api`` is its thin torch-facing binding and
``workload`` draws the seeded synthetic inputs.
"""
from .api import (OUT_BF16, OUT_F32, POS_CONTIGUOUS, POS_NONE, POS_SPARSE,  # noqa: F401
                  PREFIX_ANCHOR, PREFIX_EVEN, PREFIX_SUMMARY, SCORE_BM25,
                  SCORE_ENTROPY, SCORE_MAXIDF, SCORE_TFIDF, block_select,
                  block_select_workspace_bytes, chunk_summaries, chunk_workspace_bytes, key_bounds,
                  kv_compact_, kv_dequantize, kv_quantize, kv_quantize_, lse_merge,
                  maxidf_summaries, maxidf_workspace_bytes, phase1_attn, phase1_gather, phase1_len,
                  phase1_positions, phase2_partial, phase2_quant, phase2_quant_workspace_bytes,
                  phase2_query, phase2_query_noalloc, phase2_sparse, phase2_sparse_workspace_bytes,
                  phase2_tree, phase2_tree_workspace_bytes, phase2_workspace_bytes, rope_, tree_mask)
