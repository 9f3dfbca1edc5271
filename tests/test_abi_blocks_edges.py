"""Limits of the entry points of drafted tokens and block-sparse reads, on the host
before any GPU call (runs without a GPU; with one, calls that are not refused are left
out, since they would be launched)."""
import pytest
import torch

from tests.test_abi_blocks import BIG, EUNSUP, FAKE, caller

GPU = torch.cuda.is_available()


def test_tree_rows_that_a_tile_cannot_address():
    # the 16 rows of a tile are addressed with 32 bits
    names = ("q Kg Vg G mask K V n_shards Tq S Hq Hkv d scale o o_dtype lse ws wsb stream")
    call = caller("pulsar_phase2_tree", names, q=FAKE, Kg=FAKE, Vg=FAKE, G=1, mask=FAKE,
                  n_shards=0, Tq=1, S=0, scale=0.1, o=FAKE, o_dtype=0, ws=FAKE, wsb=BIG)
    for heads, d in ((1 << 20, 128), (1 << 21, 64)):
        assert call(Hq=heads, Hkv=heads, d=d) == EUNSUP
        if not GPU:
            assert call(Hq=heads - 1, Hkv=heads - 1, d=d) != EUNSUP


def test_key_bounds_of_the_widest_rows():
    # a row's channels are counted in 32 bits
    call = caller("pulsar_key_bounds", "K n_shards S Hkv d block bounds stream", K=FAKE,
                  n_shards=1, S=1, block=16, bounds=FAKE)
    for heads, d in ((1 << 24, 128), (1 << 25, 64)):
        assert call(Hkv=heads, d=d) == EUNSUP
        if not GPU:
            assert call(Hkv=heads - 1, d=d) != EUNSUP


@pytest.mark.skipif(GPU, reason="the calls would be launched")
@pytest.mark.parametrize("Hkv", [1, 3, 8, 33, 41, 65, 1000])
def test_sparse_launches_below_their_limit(Hkv):
    # as many tokens as the documented limit leaves, whatever the KV heads: blocks too many
    # for tokens to be read together, and lists of one step and of many
    names = ("q K V sel n_shards Tq S block topk Kg Vg G mask Hq Hkv d scale o o_dtype lse ws wsb "
             "stream")
    call = caller("pulsar_phase2_sparse", names, q=FAKE, K=FAKE, V=FAKE, sel=FAKE, n_shards=1,
                  S=16 * 70000, block=16, G=0, Hkv=Hkv, scale=0.1, o=FAKE, o_dtype=0, ws=FAKE, wsb=BIG)
    for d in (64, 128):
        for group, tiles in ((1, 1), (4, 1), (40, 3)):
            for topk in (1, 2000):
                Tq = ((1 << 23) - 1) // (Hkv * tiles)
                assert call(Hq=Hkv * group, d=d, Tq=Tq, topk=topk) != EUNSUP, (d, group, topk)
                assert call(Hq=Hkv * group, d=d, Tq=Tq * 5, topk=topk) == EUNSUP
