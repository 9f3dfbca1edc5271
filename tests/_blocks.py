"""Helpers of the tests of drafted tokens and block-sparse reads."""
import numpy as np
import torch

from oracle import blocks as ob
from paper_2607_20457_amd import workload
from tests._helpers import f64, to_dev_bf16


def normal(seed, shape, scale=1.0):
    return workload.bf16_normal(seed, shape, scale=scale)


def host(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()


def dev_i32(x) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x)).astype(np.int64)).to(
        torch.int32).cuda()


def dev_mask(sees) -> torch.Tensor:
    words = ob.mask_words(np.asarray(sees, dtype=bool))
    return torch.from_numpy(words.view(np.int32).copy()).cuda()


def check(o, lse, ref, keys, what, bf16_out=False):
    """(o, lse) against oracle.blocks.counted_attention.

    A score is a sum of d exact products in fp32: off by at most e = (d + 4) 2^-24
    sum |q_i k_i| scale (any order; the scale and the base change round it twice
    more), so a weight by a factor exp(2 e).  exp2, the sums over `keys` keys and
    the merge of parts add at most (keys + 64) 2^-23.  Every weight is rounded to
    bf16 once (2^-8 of it) and O divided by the sum of the rounded ones, which
    moves o by at most 2 * 2^-8 of the weighted |v|.  A bf16 output is rounded
    once more, by 2^-8 of it."""
    o_ref, lse_ref, size, most = ref
    d = o_ref.shape[-1]
    e = (d + 4) * 2.0 ** -24 * most
    sums = (keys + 64) * 2.0 ** -23
    o, lse = host(o), host(lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(lse_ref)), f"{what}: rows without keys"
    seen = ~np.isneginf(lse_ref)
    off = np.abs(lse[seen] - lse_ref[seen])
    bound = 2 * e + sums + 2.0 ** -22 * np.abs(lse_ref[seen])
    assert np.all(off <= bound), f"{what}: LSE off by {off.max()}, bound {bound.max()}"
    bound = (2.0 ** -7 + 4 * e + 2 * sums) * size
    if bf16_out:
        bound = bound + 2.0 ** -8 * (np.abs(o_ref) + bound)
    off = np.abs(o - o_ref)
    assert np.all(off <= bound), f"{what}: O off by {off.max()} at {np.argmax(off - bound)}"


def tree_reference(q, kg, vg, G, sees, k, v, scale):
    """The oracle's phase2_tree; k and v [n_shards, S, Hkv, d] or None."""
    Hkv, d = kg.shape[1:]
    shards = f64(k).reshape(-1, Hkv, d) if k is not None else np.zeros((0, Hkv, d))
    vals = f64(v).reshape(-1, Hkv, d) if v is not None else np.zeros((0, Hkv, d))
    Tq = q.shape[0]
    n = shards.shape[0]
    counts = np.ones((Tq, 1, n + G + Tq))
    counts[:, 0, n + G:] = sees
    return ob.counted_attention(f64(q), np.concatenate([shards, f64(kg)]),
                                np.concatenate([vals, f64(vg)]), counts, scale), n + G + Tq


def sparse_reference(q, k, v, sel, block, kg, vg, G, sees, scale):
    """The oracle's phase2_sparse; kg and vg may be None, sees None is causal."""
    n, S, Hkv, d = k.shape
    Tq = q.shape[0]
    counts = ob.sparse_counts(np.asarray(sel), -(-S // block), block, S)
    K, V = f64(k).reshape(-1, Hkv, d), f64(v).reshape(-1, Hkv, d)
    if kg is not None:
        gen = np.ones((Tq, Hkv, G + Tq))
        gen[:, :, G:] = (np.tri(Tq) if sees is None else sees)[:, None, :]
        counts = np.concatenate([counts, gen], axis=2)
        K, V = np.concatenate([K, f64(kg)]), np.concatenate([V, f64(vg)])
    return ob.counted_attention(f64(q), K, V, counts, scale), K.shape[0]


def random_tree(seed, T, dead=()):
    rng = np.random.default_rng(seed)
    parent = np.array([rng.integers(-1, t) if t else -1 for t in range(T)])
    for t in dead:
        parent[t] = t + 5
    return parent


__all__ = ["normal", "host", "dev_i32", "dev_mask", "check", "tree_reference",
           "sparse_reference", "random_tree", "f64", "to_dev_bf16"]
