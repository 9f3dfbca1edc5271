"""block_select and phase2_sparse where their dispatch, their lists and their
values have edges, against oracle.blocks."""
import numpy as np
import pytest
import torch

import paper_2607_20457_amd as P
from oracle import blocks as ob
from tests import test_gpu_blocks as lists
from tests._blocks import dev_mask, f64, host, normal, to_dev_bf16

pytestmark = pytest.mark.gpu


def _both_selections(q, bounds, topk, what):
    """The selection with scores and the one without, which has to be the same."""
    print(f"block_select: {what} {tuple(bounds.shape)} Tq={q.shape[0]} topk={topk}", flush=True)
    sel, scores = P.block_select(to_dev_bf16(q), bounds.cuda(), topk, return_scores=True)
    assert torch.equal(sel, P.block_select(to_dev_bf16(q), bounds.cuda(), topk)), what
    return sel.cpu().numpy(), scores.cpu().numpy()


def _single_key_bounds(seed, blocks, d):
    """Blocks of one key each, so that scores have either sign."""
    x = f64(normal(seed, (1, 1, blocks, 1, d)))
    return torch.from_numpy(np.repeat(x, 2, axis=3)).to(torch.bfloat16)


@pytest.mark.parametrize("blocks,Hq,d,Tq", [(90, 4, 64, 2), (200, 4, 128, 9), (250, 24, 64, 12)])
def test_one_bound_alone_that_is_not_finite(blocks, Hq, d, Tq):
    # a lower bound of +inf or an upper one of -inf beside a finite one: +inf as well
    b = _single_key_bounds(210, blocks, d)
    b[0, 0, 7, 0, 3], b[0, 0, 50, 1, 60], b[0, 0, 80, 0, 21], b[0, 0, 81, 1, 20] = (
        np.inf, -np.inf, -np.inf, np.nan)
    q = normal(211, (Tq, Hq, d))
    want = ob.block_scores(f64(q), host(b))
    for topk in (2, 4, 9):
        sel, scores = _both_selections(q, b, topk, "one bound")
        assert np.array_equal(scores, want)
        assert np.array_equal(sel, ob.block_select(want, topk)), topk


@pytest.mark.parametrize("blocks", [300, 700, 1500, 5000, 17000])
def test_more_infinite_scores_than_are_selected(blocks):
    # of several blocks that rank as +inf, beside scores below 0, the first ones
    b = _single_key_bounds(200, blocks, 64)
    bad = np.sort(np.random.default_rng(blocks).permutation(blocks)[:6])
    for i, at in enumerate(bad):
        b[0, 0, at, i % 2, 5 * i] = (np.inf, -np.inf, np.nan)[i % 3]
    q = normal(201, (9, 4, 64))
    want = ob.block_scores(f64(q), host(b))
    assert (want.min(axis=3) < 0).all()
    for topk in (1, 2, 5, 6, 20):
        sel, scores = _both_selections(q, b, topk, "infinite scores")
        assert np.array_equal(scores, want)
        assert np.array_equal(sel, ob.block_select(want, topk)), topk


@pytest.mark.parametrize("blocks,Tq", [(90, 8), (240, 9), (700, 64), (5000, 12)])
@pytest.mark.parametrize("Hq,d", [(4, 128), (24, 64)])
def test_large_channels_that_cancel(blocks, Tq, Hq, d):
    # two channels whose products cancel at 2^44, 2^20 and not at all beside those of N(0, 1):
    # the sums of fp64 depend on their order, the scores and the selection do not
    q, k = f64(normal(220, (Tq, Hq, d))), f64(normal(221, (1, 1, blocks, 1, d)))
    a, b = 5, d - 9
    for size in (22, 10):
        x, y = q.copy(), k.copy()
        x[..., a] = x[..., b] = 2.0 ** size * (1 + np.arange(Tq)[:, None] % 7 / 8)
        y[..., a] = 2.0 ** size * (1 + np.arange(blocks)[None, None, :, None] % 5 / 8)
        y[..., b] = -y[..., a]
        y = torch.from_numpy(np.repeat(y, 2, axis=3)).to(torch.bfloat16)
        words = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
        want = ob.block_scores(f64(words), host(y))
        for topk in (3, blocks // 3):
            sel, scores = _both_selections(words, y, topk, f"cancelling at 2^{2 * size}")
            assert np.array_equal(scores, want)
            assert np.array_equal(sel, ob.block_select(want, topk)), topk


def test_shards_of_drafts_go_together():
    q, kg, k = (to_dev_bf16(normal(230 + i, s)) for i, s in enumerate(
        ((2, 8, 64), (6, 4, 64), (1, 40, 4, 64))))
    mask = dev_mask(np.eye(2, dtype=bool))
    for kw in (dict(K=k), dict(V=k)):
        with pytest.raises(ValueError):
            P.phase2_tree(q, kg, kg, 4, mask, **kw)


# heads and lists whose tokens fill two groups of 16 columns from 1200 MB of listed keys on
TWO_GROUPS = [shape[:8] + (1300,) for shape in lists.TOGETHER
              if shape[2] == 128 and shape[0] // shape[1] > 2 and shape[8] == 800]


@pytest.mark.parametrize("Hq,Hkv,d,Tq,ns,S,block,topk,mb", TWO_GROUPS)
def test_two_groups_of_tokens_read_together(Hq, Hkv, d, Tq, ns, S, block, topk, mb):
    lists.test_tokens_read_together(Hq, Hkv, d, Tq, ns, S, block, topk, mb)


# (the one before the last block is to be token 3's alone: not among the first topk - 1)
@pytest.mark.parametrize("Hq,Hkv,d,Tq,ns,S,block,topk,mb",
                         [x for x in TWO_GROUPS if -(-x[5] // x[6]) - 2 >= x[7] - 1])
def test_two_groups_of_tokens_keep_their_rows(Hq, Hkv, d, Tq, ns, S, block, topk, mb):
    lists.test_tokens_read_together_keep_their_rows(Hq, Hkv, d, Tq, ns, S, block, topk, mb)
