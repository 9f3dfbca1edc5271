"""Pins of oracle.blocks: hand-worked trees and lists, brute-force bounds, and
attention against oracle.attention (CPU)."""
import itertools
import math

import numpy as np
import pytest

from oracle import attention as oatt
from oracle import blocks as ob


def test_tree_by_hand():
    #   -1 -> 0 -> 2 -> 3,  -1 -> 1 -> 4; 5 is no token, nor 6, which follows it
    sees, depth = ob.tree_visible([-1, -1, 0, 2, 1, 9, 5])
    want = np.zeros((7, 7), bool)
    for t, branch in enumerate([[0], [1], [0, 2], [0, 2, 3], [1, 4], [], []]):
        want[t, branch] = True
    assert np.array_equal(sees, want)
    assert depth.tolist() == [0, 0, 1, 2, 1, -1, -1]
    assert ob.mask_words(sees)[:, 0].tolist() == [1, 2, 5, 13, 18, 0, 0]


def test_mask_words_past_32():
    sees = np.zeros((40, 40), bool)
    sees[39, [0, 31, 32, 39]] = True
    assert ob.mask_words(sees)[39].tolist() == [1 | 1 << 31, 1 | 1 << 7]


def test_chain_is_the_query_step():
    rng = np.random.default_rng(1)
    Tq, G, Hq, Hkv, d = 4, 3, 4, 2, 8
    q, kg, vg = (rng.standard_normal(s) for s in ((Tq, Hq, d), (G + Tq, Hkv, d), (G + Tq, Hkv, d)))
    K, V = rng.standard_normal((2, 5, Hkv, d)), rng.standard_normal((2, 5, Hkv, d))
    sees, _ = ob.tree_visible(np.arange(Tq) - 1)
    counts = np.ones((Tq, 1, 10 + G + Tq))
    counts[:, 0, 10 + G:] = sees
    o, lse, size, _ = ob.counted_attention(q, np.concatenate([K.reshape(10, Hkv, d), kg]),
                                           np.concatenate([V.reshape(10, Hkv, d), vg]), counts, 0.3)
    want = oatt.query_attention(q, K, V, kg, vg, G, 0.3)
    assert np.allclose(o, want[0], atol=1e-13) and np.allclose(lse, want[1], atol=1e-13)
    assert (size >= np.abs(o) - 1e-13).all()


def test_counts_are_copies_of_keys():
    rng = np.random.default_rng(2)
    q, K, V = rng.standard_normal((1, 2, 4)), rng.standard_normal((3, 1, 4)), \
        rng.standard_normal((3, 1, 4))
    o, lse, _, _ = ob.counted_attention(q, K, V, np.array([2, 0, 1]), 0.5)
    want = oatt.dense_attention(q, K[[0, 0, 2]], V[[0, 0, 2]], 0.5)
    assert np.allclose(o, want[0]) and np.allclose(lse, want[1])
    o, lse, _, _ = ob.counted_attention(q, K, V, np.zeros(3), 0.5)
    assert (o == 0).all() and np.isneginf(lse).all()


def test_score_bounds_every_key_and_is_reached():
    # the score is the largest q . k over all corners of the box
    rng = np.random.default_rng(3)
    K = rng.standard_normal((1, 6, 1, 3))
    q = rng.standard_normal((2, 2, 3))
    b = ob.key_bounds(K, 4)
    assert b.shape == (1, 1, 2, 2, 3)
    assert np.array_equal(b[0, 0, 1, 0], K[0, 4:, 0].min(axis=0))
    s = ob.block_scores(q, b)
    for t, blk in itertools.product(range(2), range(2)):
        corners = itertools.product(*zip(b[0, 0, blk, 0], b[0, 0, blk, 1]))
        best = max(float(np.dot(q[t, h], c)) for c in corners for h in range(2))
        assert s[0, t, 0, blk] == np.float32(best) or math.isclose(s[0, t, 0, blk], best, rel_tol=1e-7)
        assert s[0, t, 0, blk] >= (K[0, 4 * blk:4 * blk + 4, 0] @ q[t].T).max() - 1e-6


@pytest.mark.parametrize("scores,topk,want", [
    ([1, 5, 5, 2, 5], 2, [1, 2]), ([3, 3, 3], 1, [0]), ([-1, -3, -2], 2, [0, 2]),
    ([0, np.inf, 4, np.inf], 3, [1, 2, 3])])
def test_selection_by_hand(scores, topk, want):
    got = ob.block_select(np.array(scores, dtype=np.float32)[None, None, None], topk)
    assert got[0, 0, 0].tolist() == want


def test_sparse_counts_by_hand():
    sel = np.array([1, -1, 2, 1, 7]).reshape(1, 1, 1, 5)
    got = ob.sparse_counts(sel, 3, 4, 10)
    assert got[0, 0].tolist() == [0, 0, 0, 0, 2, 2, 2, 2, 1, 1]


def test_compact_by_hand():
    x = np.arange(8)[None, :, None]
    assert ob.kv_compact(x, 2, [1, 3, -1, 4])[0, :, 0].tolist() == [0, 1, 3, 5, 4, 5, 6, 7]
    assert ob.kv_compact(x, 2, [0, 5, 6])[0, :, 0].tolist() == [0, 1, 2, 7, 4, 5, 6, 7]
    assert ob.kv_compact(x, 2, [2, 2])[0, :, 0].tolist() == [0, 1, 4, 3, 4, 5, 6, 7]
