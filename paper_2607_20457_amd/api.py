"""Python binding of the C ABI: argument marshalling only.

Every function takes and returns torch tensors on a HIP device; torch is
used to allocate the output buffers and to name the current stream.  All
computation happens in the HIP kernels behind ``libpulsar.so``.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch

from . import _lib

PREFIX_SUMMARY = 0
PREFIX_ANCHOR = 1
PREFIX_EVEN = 2
OUT_F32 = 0
OUT_BF16 = 1
POS_SPARSE = 0
POS_CONTIGUOUS = 1
POS_NONE = 2
SCORE_MAXIDF = 0
SCORE_TFIDF = 1
SCORE_BM25 = 2
SCORE_ENTROPY = 3


def _stream():
    # the current stream's handle without the Stream object around it (0.2
    # against 2.9 us, of calls whose kernels take 10)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, dtype, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def maxidf_workspace_bytes(batch: int, L: int, num_blocks: int, chunk: int, vocab: int) -> int:
    return int(_lib.lib().pulsar_maxidf_workspace_bytes(batch, L, num_blocks, chunk, vocab))


def maxidf_summaries(ids: torch.Tensor, num_blocks: int, chunk: int, topk: int, vocab: int,
                     return_mindf: bool = False, return_idf: bool = False, workspace="auto"):
    """Top-k Max-IDF chunks per block.  ids int32 [batch, L] ->
    sel int32 [batch, num_blocks, topk] (+ mindf [batch, N, C], idf [batch, V]).
    workspace: "auto" allocates the split path's workspace when the shapes
    use one, None runs one workgroup per sequence, or a device buffer."""
    if ids.dim() == 1:
        ids = ids[None]
    _need(ids, torch.int32, "ids")
    batch, L = ids.shape
    C = (L // num_blocks) // chunk if num_blocks > 0 and chunk > 0 else 0
    sel = ids.new_empty((batch, num_blocks, topk), dtype=torch.int32)
    mindf = ids.new_empty((batch, num_blocks, C), dtype=torch.int32) if return_mindf else None
    idf = ids.new_empty((batch, vocab), dtype=torch.float32) if return_idf else None
    if isinstance(workspace, str):
        need = maxidf_workspace_bytes(batch, L, num_blocks, chunk, vocab) if num_blocks > 0 else 0
        workspace = ids.new_empty(need, dtype=torch.uint8) if need else None
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.lib().pulsar_maxidf_summaries(_ptr(ids), batch, L, num_blocks, chunk, topk, vocab,
                                            _ptr(sel), _ptr(mindf), _ptr(idf), _ptr(workspace),
                                            ws_bytes, _stream())
    _lib.check(st, "pulsar_maxidf_summaries")
    out = [sel]
    if return_mindf:
        out.append(mindf)
    if return_idf:
        out.append(idf)
    return out[0] if len(out) == 1 else tuple(out)


def chunk_workspace_bytes(batch: int, L: int, num_blocks: int, chunk: int, vocab: int,
                          scorer: int) -> int:
    return int(_lib.lib().pulsar_chunk_workspace_bytes(batch, L, num_blocks, chunk, vocab, scorer))


def chunk_summaries(ids: torch.Tensor, num_blocks: int, chunk: int, topk: int, vocab: int,
                    scorer: int, return_scores: bool = False, workspace="auto"):
    """Top-k chunks per block under a scorer (SCORE_*).  ids int32 [batch, L]
    -> sel int32 [batch, num_blocks, topk] (+ fp32 scores [batch, N, C]).
    workspace: "auto" allocates the split path's workspace when the shapes
    use one, None runs one workgroup per sequence, or a device buffer."""
    if ids.dim() == 1:
        ids = ids[None]
    _need(ids, torch.int32, "ids")
    batch, L = ids.shape
    C = (L // num_blocks) // chunk if num_blocks > 0 and chunk > 0 else 0
    sel = ids.new_empty((batch, num_blocks, topk), dtype=torch.int32)
    scores = ids.new_empty((batch, num_blocks, C), dtype=torch.float32) \
        if return_scores else None
    if isinstance(workspace, str):
        need = chunk_workspace_bytes(batch, L, num_blocks, chunk, vocab, scorer) \
            if num_blocks > 0 else 0
        workspace = ids.new_empty(need, dtype=torch.uint8) if need else None
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.lib().pulsar_chunk_summaries(_ptr(ids), batch, L, num_blocks, chunk, topk, vocab,
                                           scorer, _ptr(sel), _ptr(scores), _ptr(workspace),
                                           ws_bytes, _stream())
    _lib.check(st, "pulsar_chunk_summaries")
    return (sel, scores) if return_scores else sel


def phase1_len(L: int, num_blocks: int, block_idx: int, sink: int, chunk: int, topk: int,
               prefix_mode: int = PREFIX_SUMMARY) -> int:
    n = _lib.lib().pulsar_phase1_len(L, num_blocks, block_idx, sink, chunk, topk, prefix_mode)
    if n < 0:
        _lib.check(int(n), "pulsar_phase1_len")
    return int(n)


def phase1_positions(sel, batch: int, L: int, num_blocks: int, block_idx: int, sink: int,
                     chunk: int, topk: int, prefix_mode: int = PREFIX_SUMMARY,
                     device=None) -> torch.Tensor:
    """Row -> global position map of Input_i, int32 [batch, n_i]."""
    n = phase1_len(L, num_blocks, block_idx, sink, chunk, topk, prefix_mode)
    if sel is not None:
        _need(sel, torch.int32, "sel")
        device = sel.device
    pos = torch.empty((batch, n), dtype=torch.int32, device=device or "cuda")
    st = _lib.lib().pulsar_phase1_positions(_ptr(sel), batch, L, num_blocks, block_idx, sink,
                                            chunk, topk, prefix_mode, _ptr(pos), _stream())
    _lib.check(st, "pulsar_phase1_positions")
    return pos


def _freq_table(inv_freq, d):
    if inv_freq is None:
        return None
    vals = [float(v) for v in (inv_freq.tolist() if hasattr(inv_freq, "tolist") else inv_freq)]
    if len(vals) != d // 2:
        raise ValueError("inv_freq must hold d/2 values")
    return (ctypes.c_float * len(vals))(*vals)


def phase1_gather(X, num_blocks: int, block_idx: int, sink: int, chunk: int, topk: int,
                  sel=None, prefix_mode: int = PREFIX_SUMMARY, pos_mode: int = POS_SPARSE,
                  inv_freq=None, base: float = 500000.0):
    """Block i's assembled input from X bf16 [b, L, H, d], each row rotated
    by its global position (POS_SPARSE), its row index (POS_CONTIGUOUS) or not
    at all (POS_NONE) -> bf16 [b, n_i, H, d]."""
    _need(X, torch.bfloat16, "X")
    if sel is not None:
        _need(sel, torch.int32, "sel")
    b, L, H, d = X.shape
    n = phase1_len(L, num_blocks, block_idx, sink, chunk, topk, prefix_mode)
    out = X.new_empty((b, n, H, d), dtype=torch.bfloat16)
    table = _freq_table(inv_freq, d)
    st = _lib.lib().pulsar_phase1_gather(_ptr(X), b, L, H, d, num_blocks, block_idx, sink, chunk,
                                         topk, _ptr(sel), prefix_mode, pos_mode,
                                         None if table is None else
                                         ctypes.cast(table, ctypes.c_void_p),
                                         float(base), _ptr(out), _stream())
    _lib.check(st, "pulsar_phase1_gather")
    return out


def phase1_attn(Q, K, V, num_blocks: int, block_idx: int, sink: int, chunk: int, topk: int,
                sel=None, prefix_mode: int = PREFIX_SUMMARY, softmax_scale: float | None = None,
                o_dtype: int = OUT_F32, return_lse: bool = True, keep_kv: bool = False,
                out=None):
    """Phase-1 causal attention over Input_i.  Q bf16 [b, L, Hq, d], K/V bf16
    [b, L, Hkv, d] -> O [b, n_i, Hq, d] (+ lse [b, Hq, n_i], K_keep, V_keep)."""
    for t, name in ((Q, "Q"), (K, "K"), (V, "V")):
        _need(t, torch.bfloat16, name)
    if sel is not None:
        _need(sel, torch.int32, "sel")
    b, L, Hq, d = Q.shape
    Hkv = K.shape[2]
    if K.shape != (b, L, Hkv, d) or V.shape != K.shape:
        raise ValueError("K and V must be [batch, L, Hkv, d] matching Q")
    n = phase1_len(L, num_blocks, block_idx, sink, chunk, topk, prefix_mode)
    scale = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    if out is not None:
        O = out
        _need(O, torch.bfloat16 if o_dtype == OUT_BF16 else torch.float32, "out")
        if O.shape != (b, n, Hq, d):
            raise ValueError("out has the wrong shape")
    else:
        O = Q.new_empty((b, n, Hq, d),
                        dtype=torch.bfloat16 if o_dtype == OUT_BF16 else torch.float32)
    lse = Q.new_empty((b, Hq, n), dtype=torch.float32) if return_lse else None
    Lb = L // num_blocks
    Kk = Q.new_empty((b, Lb, Hkv, d), dtype=torch.bfloat16) if keep_kv else None
    Vk = Q.new_empty((b, Lb, Hkv, d), dtype=torch.bfloat16) if keep_kv else None
    st = _lib.lib().pulsar_phase1_attn(_ptr(Q), _ptr(K), _ptr(V), b, L, Hq, Hkv, d, num_blocks,
                                       block_idx, sink, chunk, topk, _ptr(sel), prefix_mode,
                                       scale, _ptr(O), o_dtype, _ptr(lse), _ptr(Kk), _ptr(Vk),
                                       _stream())
    _lib.check(st, "pulsar_phase1_attn")
    res = [O]
    if return_lse:
        res.append(lse)
    if keep_kv:
        res += [Kk, Vk]
    return res[0] if len(res) == 1 else tuple(res)


def phase2_workspace_bytes(n_shards: int, Tq: int, S: int, Hq: int, Hkv: int, d: int) -> int:
    return int(_lib.lib().pulsar_phase2_workspace_bytes(n_shards, Tq, S, Hq, Hkv, d))


def phase2_partial(q, K, V, softmax_scale: float | None = None, workspace=None):
    """Per-shard partials.  q bf16 [Tq, Hq, d]; K/V bf16 [n_shards, S, Hkv, d]
    -> (o_parts f32 [n_shards, Tq, Hq, d], lse_parts f32 [n_shards, Hq, Tq])."""
    _need(q, torch.bfloat16, "q")
    _need(K, torch.bfloat16, "K")
    _need(V, torch.bfloat16, "V")
    Tq, Hq, d = q.shape
    H, S, Hkv, dk = K.shape
    if dk != d or V.shape != K.shape:
        raise ValueError("K/V must be [n_shards, S, Hkv, d]")
    scale = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    o = q.new_empty((H, Tq, Hq, d), dtype=torch.float32)
    lse = q.new_empty((H, Hq, Tq), dtype=torch.float32)
    need = phase2_workspace_bytes(H, Tq, S, Hq, Hkv, d)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = q.new_empty(need, dtype=torch.uint8)
    st = _lib.lib().pulsar_phase2_partial(_ptr(q), _ptr(K), _ptr(V), H, Tq, S, Hq, Hkv, d, scale,
                                          _ptr(o), _ptr(lse), _ptr(workspace),
                                          need, _stream())
    _lib.check(st, "pulsar_phase2_partial")
    return o, lse


def lse_merge(o_parts, lse_parts):
    """Merge H partials: o_parts f32 [H, Tq, Hq, d], lse_parts f32 [H, Hq, Tq]
    -> (o [Tq, Hq, d], lse [Hq, Tq])."""
    _need(o_parts, torch.float32, "o_parts")
    _need(lse_parts, torch.float32, "lse_parts")
    H, Tq, Hq, d = o_parts.shape
    if lse_parts.shape != (H, Hq, Tq):
        raise ValueError("lse_parts must be [H, Hq, Tq]")
    o = o_parts.new_empty((Tq, Hq, d), dtype=torch.float32)
    lse = o_parts.new_empty((Hq, Tq), dtype=torch.float32)
    st = _lib.lib().pulsar_lse_merge(_ptr(o_parts), _ptr(lse_parts), H, Tq, Hq, d, _ptr(o),
                                     _ptr(lse), _stream())
    _lib.check(st, "pulsar_lse_merge")
    return o, lse


def rope_(x, pos=None, pos_offset: int = 0, inv_freq=None, base: float = 500000.0):
    """Rotate x bf16 [batch, n, H, d] (or [n, H, d]) in place by the rows'
    positions: pos int32 [batch, n] (None: row index) plus pos_offset.
    inv_freq: the d/2 frequencies (a host sequence of floats), or None for
    base^(-2i/d).  Returns x."""
    _need(x, torch.bfloat16, "x")
    xv = x[None] if x.dim() == 3 else x
    batch, n, H, d = xv.shape
    if pos is not None:
        _need(pos, torch.int32, "pos")
        if pos.numel() != batch * n:
            raise ValueError("pos must hold one position per row")
    table = _freq_table(inv_freq, d)
    st = _lib.lib().pulsar_rope(_ptr(xv), batch, n, H, d, _ptr(pos), int(pos_offset),
                                None if table is None else ctypes.cast(table, ctypes.c_void_p),
                                float(base), _stream())
    _lib.check(st, "pulsar_rope")
    return x


def phase2_query(q, Kg, Vg, G: int, K=None, V=None, softmax_scale: float | None = None,
                 workspace=None):
    """Attention of Tq new tokens: q bf16 [Tq, Hq, d] over the retained
    shards K/V bf16 [n_shards, S, Hkv, d] (or None) and the generation shard's
    appended rows Kg/Vg bf16 [G + Tq, Hkv, d] up to each token itself
    -> (o f32 [Tq, Hq, d], lse f32 [Hq, Tq])."""
    _need(q, torch.bfloat16, "q")
    _need(Kg, torch.bfloat16, "Kg")
    _need(Vg, torch.bfloat16, "Vg")
    Tq, Hq, d = q.shape
    Hkv = Kg.shape[1]
    if Kg.shape != (G + Tq, Hkv, d) or Vg.shape != Kg.shape:
        raise ValueError("Kg/Vg must be [G + Tq, Hkv, d]")
    n_shards, S = 0, 0
    if K is not None:
        _need(K, torch.bfloat16, "K")
        _need(V, torch.bfloat16, "V")
        n_shards, S = K.shape[0], K.shape[1]
        if K.shape != (n_shards, S, Hkv, d) or V.shape != K.shape:
            raise ValueError("K/V must be [n_shards, S, Hkv, d]")
    scale = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    o = q.new_empty((Tq, Hq, d), dtype=torch.float32)
    lse = q.new_empty((Hq, Tq), dtype=torch.float32)
    need = _lib.lib().pulsar_phase2_query_workspace_bytes(n_shards, Tq, S, G, Hq, Hkv, d)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = q.new_empty(max(need, 16), dtype=torch.uint8)
    st = _lib.lib().pulsar_phase2_query(_ptr(q), _ptr(Kg), _ptr(Vg), G, _ptr(K), _ptr(V), n_shards,
                                        Tq, S, Hq, Hkv, d, scale, _ptr(o), _ptr(lse),
                                        _ptr(workspace), need, _stream())
    _lib.check(st, "pulsar_phase2_query")
    return o, lse


def phase2_query_noalloc(q, Kg, Vg, G: int, K=None, V=None, softmax_scale: float | None = None):
    """``phase2_query`` through the entry point that allocates nothing: the
    partials live in the library's static per-device scratch.  The outputs
    are allocated here by torch, as for every binding."""
    _need(q, torch.bfloat16, "q")
    _need(Kg, torch.bfloat16, "Kg")
    _need(Vg, torch.bfloat16, "Vg")
    Tq, Hq, d = q.shape
    Hkv = Kg.shape[1]
    if Kg.shape != (G + Tq, Hkv, d) or Vg.shape != Kg.shape:
        raise ValueError("Kg/Vg must be [G + Tq, Hkv, d]")
    n_shards, S = 0, 0
    if K is not None:
        _need(K, torch.bfloat16, "K")
        _need(V, torch.bfloat16, "V")
        n_shards, S = K.shape[0], K.shape[1]
        if K.shape != (n_shards, S, Hkv, d) or V.shape != K.shape:
            raise ValueError("K/V must be [n_shards, S, Hkv, d]")
    scale = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    o = q.new_empty((Tq, Hq, d), dtype=torch.float32)
    lse = q.new_empty((Hq, Tq), dtype=torch.float32)
    st = _lib.lib().pulsar_phase2_query_noalloc(_ptr(q), _ptr(Kg), _ptr(Vg), G, _ptr(K), _ptr(V),
                                                n_shards, Tq, S, Hq, Hkv, d, scale, _ptr(o),
                                                _ptr(lse), _stream())
    _lib.check(st, "pulsar_phase2_query_noalloc")
    return o, lse


_BF16 = torch.bfloat16


def _check(dev, dtype, named):
    """Every (tensor, name) is a contiguous tensor of dtype on device dev, the
    current one, whose current stream the call uses."""
    for t, name in named:
        if t.get_device() != dev or t.dtype is not dtype or not t.is_contiguous():
            _need(t, dtype, name)
            raise ValueError(f"{name} must be on the current device")


def _int32(x, name):
    """The C entry points take x as an int: a larger one would wrap around."""
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} out of range")


def _raw_stream(dev):
    return torch._C._cuda_getCurrentRawStream(dev)


def _generation_shape(Kg, Vg, G, Tq, Hkv, d):
    if G < 0 or Kg.shape != (G + Tq, Hkv, d) or Vg.shape != Kg.shape:
        raise ValueError("Kg/Vg must be [G + Tq, Hkv, d]")


def _mask_shape(mask, Tq):
    if mask.shape != (Tq, (Tq + 31) // 32):
        raise ValueError("mask must be [Tq, ceil(Tq / 32)]")


def _out(q, o_dtype):
    if o_dtype == OUT_BF16:
        return torch.empty_like(q)
    if o_dtype != OUT_F32:
        raise ValueError("o_dtype must be OUT_F32 or OUT_BF16")
    return torch.empty_like(q, dtype=torch.float32)


def _scratch(workspace, need, dev, like):
    """The caller's workspace where it is large enough, else a new one, and its
    address (None where none is needed)."""
    if workspace is not None and workspace.numel() * workspace.element_size() >= need:
        _check(dev, workspace.dtype, ((workspace, "workspace"),))
        return workspace, workspace.data_ptr()
    if not need:
        return None, None
    workspace = like.new_empty(need, dtype=torch.uint8)
    return workspace, workspace.data_ptr()


def tree_mask(parent):
    """Visibility of a tree of drafted tokens.  parent int32 [T]: the earlier
    draft that each follows, -1 for the last token before them (any other value:
    no token) -> (mask int32 [T, ceil(T / 32)], each token's bits set for itself
    and its ancestors; depth int32 [T], its number of ancestors, -1 for none)."""
    dev = torch.cuda.current_device() if parent.is_cuda else None
    _check(dev, torch.int32, ((parent, "parent"),))
    if parent.dim() != 1:
        raise ValueError("parent must be [T]")
    T = parent.shape[0]
    mask = parent.new_empty((T, (T + 31) // 32))
    depth = torch.empty_like(parent)
    st = _lib.lib().pulsar_tree_mask(parent.data_ptr(), T, mask.data_ptr(), depth.data_ptr(),
                                     _raw_stream(dev))
    _lib.check(st, "pulsar_tree_mask")
    return mask, depth


@functools.lru_cache(maxsize=4096)
def phase2_tree_workspace_bytes(n_shards: int, Tq: int, S: int, G: int, Hq: int, Hkv: int,
                                d: int) -> int:
    return int(_lib.lib().pulsar_phase2_tree_workspace_bytes(n_shards, Tq, S, G, Hq, Hkv, d))


def phase2_tree(q, Kg, Vg, G: int, mask, K=None, V=None, softmax_scale: float | None = None,
                o_dtype: int = OUT_F32, workspace=None):
    """Attention of a tree of Tq drafted tokens: q bf16 [Tq, Hq, d] over the
    retained shards K/V bf16 [n_shards, S, Hkv, d] (or None), the G earlier rows
    of the generation shard Kg/Vg bf16 [G + Tq, Hkv, d], and those of the drafts'
    own rows that mask int32 [Tq, ceil(Tq / 32)] (``tree_mask``) sets for each
    -> (o [Tq, Hq, d] per o_dtype, lse f32 [Hq, Tq])."""
    dev = torch.cuda.current_device() if q.is_cuda else None
    _check(dev, _BF16, ((q, "q"), (Kg, "Kg"), (Vg, "Vg")))
    _check(dev, torch.int32, ((mask, "mask"),))
    Tq, Hq, d = q.shape
    Hkv = Kg.shape[1]
    _generation_shape(Kg, Vg, G, Tq, Hkv, d)
    _mask_shape(mask, Tq)
    n_shards, S, k_ptr, v_ptr = 0, 0, None, None
    if (K is None) != (V is None):
        raise ValueError("K and V go together")
    if K is not None:
        _check(dev, _BF16, ((K, "K"), (V, "V")))
        n_shards, S = K.shape[:2]
        if K.shape != (n_shards, S, Hkv, d) or V.shape != K.shape:
            raise ValueError("K/V must be [n_shards, S, Hkv, d]")
        k_ptr, v_ptr = K.data_ptr(), V.data_ptr()
    o = _out(q, o_dtype)
    lse = q.new_empty((Hq, Tq), dtype=torch.float32)
    need = phase2_tree_workspace_bytes(n_shards, Tq, S, G, Hq, Hkv, d)
    workspace, ws_ptr = _scratch(workspace, need, dev, q)
    st = _lib.lib().pulsar_phase2_tree(
        q.data_ptr(), Kg.data_ptr(), Vg.data_ptr(), G, mask.data_ptr(), k_ptr, v_ptr, n_shards, Tq,
        S, Hq, Hkv, d, 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale,
        o.data_ptr(), o_dtype, lse.data_ptr(), ws_ptr, need, _raw_stream(dev))
    _lib.check(st, "pulsar_phase2_tree")
    return o, lse


def kv_compact_(K, V, G: int, keep):
    """Rows G + keep[j] of every layer of K/V bf16 [layers, capacity, Hkv, d]
    moved to row G + j, in place.  keep int32 [n], rising; it ends at the first
    entry that is negative, does not rise or lies past the cache.  Returns K, V."""
    dev = torch.cuda.current_device() if K.is_cuda else None
    _check(dev, _BF16, ((K, "K"), (V, "V")))
    _check(dev, torch.int32, ((keep, "keep"),))
    if K.dim() != 4 or V.shape != K.shape or keep.dim() != 1:
        raise ValueError("K/V must be [layers, capacity, Hkv, d], keep [n]")
    if abs(K.data_ptr() - V.data_ptr()) < 2 * K.numel():
        raise ValueError("K and V must not share memory")
    layers, capacity, Hkv, d = K.shape
    st = _lib.lib().pulsar_kv_compact(K.data_ptr(), V.data_ptr(), layers, capacity, Hkv, d, G,
                                      keep.data_ptr(), keep.shape[0], _raw_stream(dev))
    _lib.check(st, "pulsar_kv_compact")
    return K, V


def key_bounds(K, block: int):
    """Channel minima and maxima of every block of `block` keys (16, 32, 64, 128
    or 256).  K bf16 [n_shards, S, Hkv, d] -> bounds bf16 [n_shards, Hkv,
    ceil(S / block), 2, d]."""
    dev = torch.cuda.current_device() if K.is_cuda else None
    _check(dev, _BF16, ((K, "K"),))
    n_shards, S, Hkv, d = K.shape
    _int32(block, "block")
    bounds = K.new_empty((n_shards, Hkv, -(-S // block) if block > 0 else 0, 2, d))
    st = _lib.lib().pulsar_key_bounds(K.data_ptr(), n_shards, S, Hkv, d, block, bounds.data_ptr(),
                                      _raw_stream(dev))
    _lib.check(st, "pulsar_key_bounds")
    return bounds


@functools.lru_cache(maxsize=4096)
def block_select_workspace_bytes(n_shards: int, Tq: int, blocks: int, Hq: int, Hkv: int) -> int:
    return int(_lib.lib().pulsar_block_select_workspace_bytes(n_shards, Tq, blocks, Hq, Hkv))


def block_select(q, bounds, topk: int, return_scores: bool = False, workspace=None):
    """The topk blocks of each shard for every token and KV head, by the largest
    q . k that their bounds allow.  q bf16 [Tq, Hq, d], bounds as ``key_bounds``
    returns them -> sel int32 [n_shards, Tq, Hkv, topk], ascending (+ the scores
    f32 [n_shards, Tq, Hkv, blocks])."""
    dev = torch.cuda.current_device() if q.is_cuda else None
    _check(dev, _BF16, ((q, "q"), (bounds, "bounds")))
    Tq, Hq, d = q.shape
    n_shards, Hkv, blocks, two, db = bounds.shape
    if two != 2 or db != d:
        raise ValueError("bounds must be [n_shards, Hkv, blocks, 2, d]")
    _int32(topk, "topk")
    sel = q.new_empty((n_shards, Tq, Hkv, max(topk, 0)), dtype=torch.int32)
    scores, ws_ptr, need = None, None, 0
    if return_scores:
        scores = q.new_empty((n_shards, Tq, Hkv, blocks), dtype=torch.float32)
    else:
        need = block_select_workspace_bytes(n_shards, Tq, blocks, Hq, Hkv)
        workspace, ws_ptr = _scratch(workspace, need, dev, q)
    st = _lib.lib().pulsar_block_select(q.data_ptr(), bounds.data_ptr(), n_shards, Tq, blocks, Hq,
                                        Hkv, d, topk, sel.data_ptr(), _ptr(scores), ws_ptr, need,
                                        _raw_stream(dev))
    _lib.check(st, "pulsar_block_select")
    return (sel, scores) if return_scores else sel


@functools.lru_cache(maxsize=4096)
def phase2_sparse_workspace_bytes(Tq: int, Hq: int, Hkv: int, d: int) -> int:
    return int(_lib.lib().pulsar_phase2_sparse_workspace_bytes(Tq, Hq, Hkv, d))


@functools.lru_cache(maxsize=4096)
def _sparse_call_bytes(n_shards, Tq, S, block, topk, gen_rows, Hq, Hkv, d):
    return int(_lib.lib().pulsar_phase2_sparse_call_bytes(n_shards, Tq, S, block, topk, gen_rows,
                                                          Hq, Hkv, d))


def phase2_sparse(q, K, V, sel, block: int, Kg=None, Vg=None, G: int = 0, mask=None,
                  softmax_scale: float | None = None, o_dtype: int = OUT_F32, workspace=None):
    """Attention of Tq new tokens over their selected blocks of the retained
    shards and over the generation shard: q bf16 [Tq, Hq, d], K/V bf16 [n_shards,
    S, Hkv, d], sel int32 [n_shards, Tq, Hkv, topk] (``block_select``; an entry
    that is no block of the shard lists none), Kg/Vg bf16 [G + Tq, Hkv, d] (None:
    the shards alone) up to each token itself, or by a tree's mask
    -> (o [Tq, Hq, d] per o_dtype, lse f32 [Hq, Tq])."""
    dev = torch.cuda.current_device() if q.is_cuda else None
    _check(dev, _BF16, ((q, "q"), (K, "K"), (V, "V")))
    _check(dev, torch.int32, ((sel, "sel"),))
    Tq, Hq, d = q.shape
    n_shards, S, Hkv, dk = K.shape
    _int32(block, "block")
    if dk != d or V.shape != K.shape:
        raise ValueError("K/V must be [n_shards, S, Hkv, d]")
    if sel.dim() != 4 or sel.shape[:3] != (n_shards, Tq, Hkv):
        raise ValueError("sel must be [n_shards, Tq, Hkv, topk]")
    kg_ptr = vg_ptr = mask_ptr = None
    if Kg is not None or Vg is not None:
        if Kg is None or Vg is None:
            raise ValueError("Kg and Vg go together")
        _check(dev, _BF16, ((Kg, "Kg"), (Vg, "Vg")))
        _generation_shape(Kg, Vg, G, Tq, Hkv, d)
        kg_ptr, vg_ptr = Kg.data_ptr(), Vg.data_ptr()
    if mask is not None:
        _check(dev, torch.int32, ((mask, "mask"),))
        _mask_shape(mask, Tq)
        mask_ptr = mask.data_ptr()
    o = _out(q, o_dtype)
    lse = q.new_empty((Hq, Tq), dtype=torch.float32)
    # (the plan takes the appended rows 32 at a time: few sizes to remember)
    gen_rows = (G + Tq + 31 & ~31) if kg_ptr else 0
    need = _sparse_call_bytes(n_shards, Tq, S, block, sel.shape[3], gen_rows, Hq, Hkv, d)
    workspace, ws_ptr = _scratch(workspace, need, dev, q)
    st = _lib.lib().pulsar_phase2_sparse(
        q.data_ptr(), K.data_ptr(), V.data_ptr(), sel.data_ptr(), n_shards, Tq, S, block,
        sel.shape[3], kg_ptr, vg_ptr, G, mask_ptr, Hq, Hkv, d,
        1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale, o.data_ptr(), o_dtype,
        lse.data_ptr(), ws_ptr, need, _raw_stream(dev))
    _lib.check(st, "pulsar_phase2_sparse")
    return o, lse


_FORMATS = {torch.float8_e4m3fn: 0, torch.int8: 1}


def _cache_of(Kc, Vc, k_scale, v_scale, block, dev):
    """The shape [n, Hkv, capacity, d] of a cache in 8 bits, and its format."""
    _int32(block, "block")
    dtype, shape = Kc.dtype, Kc.shape
    if dtype not in _FORMATS:
        raise ValueError(f"codes must be torch.float8_e4m3fn or torch.int8, got {dtype}")
    _check(dev, dtype, ((Kc, "Kc"), (Vc, "Vc")))
    _check(dev, torch.float32, ((k_scale, "k_scale"), (v_scale, "v_scale")))
    if len(shape) != 4 or Vc.shape != shape:
        raise ValueError("Kc/Vc must be [n, Hkv, capacity, d]")
    scales = (shape[0], shape[1], -(-shape[2] // block) if block > 0 else 0)
    if k_scale.shape != scales or v_scale.shape != scales:
        raise ValueError("k_scale/v_scale must be [n, Hkv, ceil(capacity / block)]")
    return shape, _FORMATS[dtype]


def _row_strides(K, V):
    """Elements from shard to shard and from row to row of K and V [n, rows, Hkv, d]."""
    n, rows, Hkv, d = K.shape
    a = K.stride()
    if a != V.stride() or a[3] != 1 or a[2] != d:
        # (a dimension of one has any stride)
        sizes = (n, rows, Hkv, d)
        if K.numel() and any(
                size > 1 and (x != y or i == 3 and x != 1 or i == 2 and x != d)
                for i, (size, x, y) in enumerate(zip(sizes, a, V.stride()))):
            raise ValueError("K and V must have the same strides, each row [Hkv, d] contiguous")
    return a[0] if n > 1 else 0, a[1] if rows > 1 else 0


def kv_quantize_(K, V, Kc, Vc, k_scale, v_scale, block: int, first: int = 0):
    """Rows [first, first + rows) of a cache in 8 bits written from K/V bf16 [n, rows,
    Hkv, d] (the rows of any longer tensors: strides of a multiple of 8 elements), whole
    blocks of them: first is a multiple of block (16, 32, 64, 128 or 256), the last block may
    be short.  Kc/Vc float8_e4m3fn or int8 [n, Hkv, capacity, d], k_scale/v_scale f32 [n, Hkv,
    ceil(capacity / block)]: a code stands for code * scale, the scale a power of two for each
    block and head, NaN (and codes 0) where the block holds a NaN or an infinity.  None of
    the cache's tensors shares memory with another, or with K and V.
    Returns the cache: Kc, Vc, k_scale, v_scale."""
    dev = torch.cuda.current_device() if K.is_cuda else None
    for t, name in ((K, "K"), (V, "V")):
        if t.get_device() != dev or t.dtype is not _BF16:
            if t.is_cuda and t.dtype is _BF16:
                raise ValueError(f"{name} must be on the current device")
            raise ValueError(f"{name} must be a device tensor of {_BF16}")
    (n, Hkv, capacity, d), form = _cache_of(Kc, Vc, k_scale, v_scale, block, dev)
    shape = K.shape
    if len(shape) != 4 or V.shape != shape or shape != (n, shape[1], Hkv, d):
        raise ValueError("K/V must be [n, rows, Hkv, d]")
    rows = shape[1]
    if not 0 <= first <= capacity - rows:
        raise ValueError("first and the rows must lie within the cache")
    shard_stride, row_stride = _row_strides(K, V)
    st = _lib.lib().pulsar_kv_quantize(K.data_ptr(), V.data_ptr(), shard_stride, row_stride, n,
                                       rows, Hkv, d, block, form, first, capacity, Kc.data_ptr(),
                                       Vc.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                       _raw_stream(dev))
    _lib.check(st, "pulsar_kv_quantize")
    return Kc, Vc, k_scale, v_scale


def kv_quantize(K, V, block: int = 64, dtype=torch.float8_e4m3fn, capacity: int | None = None):
    """K/V bf16 [n, rows, Hkv, d] as a new cache in 8 bits (``kv_quantize_``), with room for
    `capacity` rows (None: rows); what lies behind the rows is undefined
    -> Kc, Vc, k_scale, v_scale."""
    if dtype not in _FORMATS:
        raise ValueError("dtype must be torch.float8_e4m3fn or torch.int8")
    if K.dim() != 4:
        raise ValueError("K/V must be [n, rows, Hkv, d]")
    n, rows, Hkv, d = K.shape
    _int32(block, "block")
    capacity = rows if capacity is None else capacity
    if block < 1 or capacity < rows:
        raise ValueError("block must be positive, capacity at least the rows")
    Kc = K.new_empty((n, Hkv, capacity, d), dtype=dtype)
    k_scale = K.new_empty((n, Hkv, -(-capacity // block)), dtype=torch.float32)
    return kv_quantize_(K, V, Kc, torch.empty_like(Kc), k_scale, torch.empty_like(k_scale), block)


def kv_dequantize(Kc, Vc, k_scale, v_scale, block: int, first: int = 0, rows: int | None = None):
    """Rows [first, first + rows) (None: all from first on) of a cache in 8 bits
    -> K, V bf16 [n, rows, Hkv, d]."""
    dev = torch.cuda.current_device() if Kc.is_cuda else None
    (n, Hkv, capacity, d), form = _cache_of(Kc, Vc, k_scale, v_scale, block, dev)
    rows = capacity - first if rows is None else rows
    if first < 0 or rows < 0 or first + rows > capacity:
        raise ValueError("first and rows must lie within the cache")
    K = Kc.new_empty((n, rows, Hkv, d), dtype=_BF16)
    V = torch.empty_like(K)
    st = _lib.lib().pulsar_kv_dequantize(Kc.data_ptr(), Vc.data_ptr(), k_scale.data_ptr(),
                                         v_scale.data_ptr(), n, capacity, Hkv, d, block, form,
                                         first, rows, K.data_ptr(), V.data_ptr(),
                                         _raw_stream(dev))
    _lib.check(st, "pulsar_kv_dequantize")
    return K, V


@functools.lru_cache(maxsize=4096)
def phase2_quant_workspace_bytes(Tq: int, Hq: int, Hkv: int, d: int) -> int:
    return int(_lib.lib().pulsar_phase2_quant_workspace_bytes(Tq, Hq, Hkv, d))


@functools.lru_cache(maxsize=4096)
def _quant_call_bytes(n_shards, Tq, S, gen_rows, Hq, Hkv, d):
    return int(_lib.lib().pulsar_phase2_quant_call_bytes(n_shards, Tq, S, gen_rows, Hq, Hkv, d))


def phase2_quant(q, Kc, Vc, k_scale, v_scale, block: int, rows=None, Kg=None, Vg=None, G: int = 0,
                 mask=None, softmax_scale: float | None = None, o_dtype: int = OUT_F32,
                 workspace=None):
    """Attention of Tq new tokens over shards held in 8 bits (``kv_quantize``) and over the
    generation shard: q bf16 [Tq, Hq, d], Kc/Vc [n_shards, Hkv, S, d], rows int32 [n_shards]
    the shards' live rows (None: all S), Kg/Vg bf16 [G + Tq, Hkv, d] (None: the shards alone)
    up to each token itself, or by a tree's mask -> (o [Tq, Hq, d] per o_dtype, lse f32
    [Hq, Tq])."""
    dev = torch.cuda.current_device() if q.is_cuda else None
    _check(dev, _BF16, ((q, "q"),))
    (n_shards, Hkv, S, dk), form = _cache_of(Kc, Vc, k_scale, v_scale, block, dev)
    Tq, Hq, d = q.shape
    if dk != d:
        raise ValueError("Kc/Vc must be [n_shards, Hkv, S, d]")
    rows_ptr = kg_ptr = vg_ptr = mask_ptr = None
    if rows is not None:
        _check(dev, torch.int32, ((rows, "rows"),))
        if rows.shape != (n_shards,):
            raise ValueError("rows must be [n_shards]")
        rows_ptr = rows.data_ptr()
    if Kg is not None or Vg is not None:
        if Kg is None or Vg is None:
            raise ValueError("Kg and Vg go together")
        _check(dev, _BF16, ((Kg, "Kg"), (Vg, "Vg")))
        _generation_shape(Kg, Vg, G, Tq, Hkv, d)
        kg_ptr, vg_ptr = Kg.data_ptr(), Vg.data_ptr()
    elif G != 0 or mask is not None:
        raise ValueError("G and mask belong to Kg and Vg")
    if mask is not None:
        _check(dev, torch.int32, ((mask, "mask"),))
        _mask_shape(mask, Tq)
        mask_ptr = mask.data_ptr()
    o = _out(q, o_dtype)
    lse = q.new_empty((Hq, Tq), dtype=torch.float32)
    # (the plan takes the appended rows 32 at a time: few sizes to remember)
    gen_rows = (G + Tq + 31 & ~31) if kg_ptr else 0
    need = _quant_call_bytes(n_shards, Tq, S, gen_rows, Hq, Hkv, d)
    workspace, ws_ptr = _scratch(workspace, need, dev, q)
    st = _lib.lib().pulsar_phase2_quant(
        q.data_ptr(), Kc.data_ptr(), Vc.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
        n_shards, Tq, S, block, form, rows_ptr, kg_ptr, vg_ptr, G, mask_ptr, Hq, Hkv, d,
        1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale, o.data_ptr(), o_dtype,
        lse.data_ptr(), ws_ptr, need, _raw_stream(dev))
    _lib.check(st, "pulsar_phase2_quant")
    return o, lse
