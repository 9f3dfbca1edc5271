"""Drafted tokens and block-sparse reads in Phase 2 (oracle).

TEST INFRASTRUCTURE ONLY -- see ``oracle/__init__.py``.

All arithmetic is fp64 on inputs that are already bf16-rounded.

* A tree of drafts: ``parent[t]`` in [-1, t) is the draft that t follows (-1: the
  last token before the drafts); any other value, or a parent that is none, makes
  t no token.  A token sees itself and its ancestors among the drafts.
* Attention with key multiplicities: softmax over the keys that a token sees, a key
  that is listed c times weighing c times.  No key at all gives o = 0, lse = -inf.
* Block bounds: the smallest and largest value of every channel over a block's keys.
* Block score: max over the heads of a KV head's group of
  sum_i max(q_i lo_i, q_i hi_i), in sixteen parts of consecutive channels that are
  added two by two, and rounded once to fp32; what is not a number is +inf.
* Selection: the topk blocks by score, then by the lower index, in index order.
* Compaction: row G + keep[j] to row G + j while the list rises within the cache.
"""
from __future__ import annotations

import numpy as np


def tree_visible(parent):
    """(sees bool [T, T], depth int [T]) of a tree of drafts."""
    parent = [int(p) for p in parent]
    T = len(parent)
    sees, depth = np.zeros((T, T), dtype=bool), np.full(T, -1)
    for t, p in enumerate(parent):
        if p == -1:
            depth[t] = 0
        elif 0 <= p < t and depth[p] >= 0:
            sees[t] = sees[p]
            depth[t] = depth[p] + 1
        else:
            continue
        sees[t, t] = True
    return sees, depth


def mask_words(sees):
    """uint32 [T, ceil(T / 32)]: bit j % 32 of word j // 32 is sees[t, j]."""
    T = sees.shape[0]
    words = np.zeros((T, (T + 31) // 32), dtype=np.uint64)
    for t in range(T):
        for j in range(T):
            if sees[t, j]:
                words[t, j // 32] |= np.uint64(1 << (j % 32))
    return words.astype(np.uint32)


def counted_attention(q, K, V, counts, scale):
    """q [Tq, Hq, d] over K, V [n, Hkv, d], key c of KV head g counting
    counts[t, g, c] times for token t.  -> (o [Tq, Hq, d], lse [Hq, Tq],
    weighted |v| [Tq, Hq, d], the largest sum_i |q_i k_i| scale of a counted key)."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    Tq, Hq, d = q.shape
    n, Hkv = K.shape[:2]
    counts = np.broadcast_to(np.asarray(counts, dtype=np.float64), (Tq, Hkv, n))
    o, size = np.zeros((Tq, Hq, d)), np.zeros((Tq, Hq, d))
    lse, most = np.full((Hq, Tq), -np.inf), 0.0
    for t in range(Tq):
        for h in range(Hq):
            g = h // (Hq // Hkv)
            keys = np.flatnonzero(counts[t, g])
            if keys.size == 0:
                continue
            c, k, v = counts[t, g, keys], K[keys, g], V[keys, g]
            s = (k @ q[t, h]) * scale
            most = max(most, float((np.abs(k) @ np.abs(q[t, h])).max()) * scale)
            m = s.max()
            p = c * np.exp(s - m)
            den = p.sum()
            o[t, h], size[t, h] = (p @ v) / den, (p @ np.abs(v)) / den
            lse[h, t] = m + np.log(den)
    return o, lse, size, most


def key_bounds(K, block):
    """K [n_shards, S, Hkv, d] -> [n_shards, Hkv, ceil(S / block), 2, d]."""
    n, S, Hkv, d = K.shape
    out = np.zeros((n, Hkv, -(-S // block), 2, d))
    for b in range(out.shape[2]):
        rows = K[:, b * block:(b + 1) * block]
        out[:, :, b, 0], out[:, :, b, 1] = rows.min(axis=1), rows.max(axis=1)
    return out


def _sum_of_parts(x):
    """x [..., d] summed in the order of a block score."""
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (-x.shape[-1] % 16,))], axis=-1)
    x = x.reshape(x.shape[:-1] + (16, x.shape[-1] // 16))
    x = np.add.accumulate(x, axis=-1)[..., -1]
    while x.shape[-1] > 1:
        x = x[..., ::2] + x[..., 1::2]
    return x[..., 0]


def block_scores(q, bounds):
    """q [Tq, Hq, d], bounds [n, Hkv, blocks, 2, d] -> float32 [n, Tq, Hkv, blocks]."""
    q, bounds = np.asarray(q, dtype=np.float64), np.asarray(bounds, dtype=np.float64)
    n, Hkv, blocks, _, d = bounds.shape
    Tq, Hq, _ = q.shape
    group = Hq // Hkv
    out = np.empty((n, Tq, Hkv, blocks), dtype=np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(Tq):
            for g in range(Hkv):
                x = q[t, g * group:(g + 1) * group, None, None, :]
                s = np.maximum(x * bounds[:, g, :, 0], x * bounds[:, g, :, 1])
                s = _sum_of_parts(s).astype(np.float32)
                bad = ~np.isfinite(bounds[:, g]).all(axis=(2, 3))
                s = np.where(np.isnan(s) | bad, np.float32(np.inf), s)
                out[:, t, g] = s.max(axis=0)
    return out


def block_select(scores, topk):
    """int32 [n, Tq, Hkv, topk]: the best blocks in index order."""
    order = np.argsort(-scores, axis=-1, kind="stable")[..., :topk]
    return np.sort(order, axis=-1).astype(np.int32)


def sparse_counts(sel, blocks, block, S):
    """[Tq, Hkv, n_shards * S]: how often sel [n_shards, Tq, Hkv, topk] lists each
    retained key; an entry outside [0, blocks) lists none."""
    n, Tq, Hkv, _ = sel.shape
    out = np.zeros((Tq, Hkv, n, S))
    for h, t, g in np.ndindex(n, Tq, Hkv):
        for b in sel[h, t, g]:
            if 0 <= b < blocks:
                out[t, g, h, b * block:(b + 1) * block] += 1
    return out.reshape(Tq, Hkv, n * S)


def kv_compact(x, G, keep):
    """x [layers, capacity, ...] with rows G + keep[j] moved to G + j."""
    y = np.array(x)
    prev = -1
    for j, k in enumerate(int(v) for v in keep):
        if k <= prev or k >= x.shape[1] - G:
            break
        y[:, G + j] = x[:, G + k]
        prev = k
    return y
