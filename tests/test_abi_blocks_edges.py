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
