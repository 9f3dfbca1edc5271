"""Refusals of the entry points of drafted tokens and block-sparse reads, on the
host before any GPU call (runs without a GPU)."""
import math

import pytest
import torch

import paper_2607_20457_amd as P
from paper_2607_20457_amd import _lib

EINVAL, EUNSUP, EWS = -1, -2, -4
FAKE = 1 << 20  # a non-NULL, 16-byte aligned address that is never dereferenced
BIG = 1 << 40


def caller(name, names, **ok):
    fn = getattr(_lib.lib(), name)
    names = names.split()

    def call(**kw):
        args = {**ok, **kw}
        assert set(args) <= set(names), args
        return fn(*(args.get(n) for n in names))
    return call


def test_tree_mask():
    call = caller("pulsar_tree_mask", "parent T mask depth stream", parent=FAKE, T=8, mask=FAKE)
    assert call(T=-1) == EINVAL
    assert call(parent=None) == EINVAL
    assert call(mask=None) == EINVAL
    assert call(T=16385) == EUNSUP
    assert call(T=0, parent=None, mask=None) == 0


def test_phase2_tree():
    names = ("q Kg Vg G mask K V n_shards Tq S Hq Hkv d scale o o_dtype lse ws wsb stream")
    call = caller("pulsar_phase2_tree", names, q=FAKE, Kg=FAKE, Vg=FAKE, G=10, mask=FAKE, K=FAKE,
                  V=FAKE, n_shards=2, Tq=5, S=100, Hq=32, Hkv=8, d=128, scale=0.1, o=FAKE,
                  o_dtype=0, ws=FAKE, wsb=BIG)
    for kw in (dict(n_shards=-1), dict(Tq=-1), dict(S=-1), dict(G=-1), dict(Hq=0), dict(Hkv=0),
               dict(Hq=12), dict(d=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
               dict(scale=math.inf), dict(q=None), dict(Kg=None), dict(Vg=None), dict(mask=None),
               dict(K=None), dict(V=None), dict(o=None), dict(o_dtype=2), dict(o_dtype=-1),
               dict(q=FAKE + 2), dict(Kg=FAKE + 8), dict(K=FAKE + 8), dict(V=FAKE + 4),
               dict(o=FAKE + 4)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(d=96), dict(Hq=24), dict(G=1 << 24), dict(S=1 << 20, Hkv=8),
               dict(Tq=1 << 19, Kg=FAKE, G=0)):
        assert call(**kw) == EUNSUP, kw
    need = P.phase2_tree_workspace_bytes(2, 5, 100, 10, 32, 8, 128)
    assert need > 0
    assert call(ws=None) == EWS and call(ws=FAKE + 8) == EWS and call(wsb=0) == EWS
    assert call(Tq=0) == 0


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (4, 1, 64), (16, 16, 64), (64, 1, 64)])
def test_phase2_tree_workspace_serves_every_smaller_step(Hq, Hkv, d):
    # (without a GPU a call that finds its workspace large enough fails at the launch)
    names = ("q Kg Vg G mask K V n_shards Tq S Hq Hkv d scale o o_dtype lse ws wsb stream")
    call = caller("pulsar_phase2_tree", names, q=FAKE, Kg=FAKE, Vg=FAKE, mask=FAKE, K=FAKE,
                  V=FAKE, Hq=Hq, Hkv=Hkv, d=d, scale=0.1, o=FAKE, o_dtype=0, ws=FAKE)
    if torch.cuda.is_available():
        pytest.skip("the calls would be launched")
    sizes = (1, 7, 16, 33, 130), (1, 3, 20), (1, 100, 700, 5000), (0, 1, 300, 5000)
    for Tq, n, S, G in ((130, 20, 5000, 5000), (33, 3, 700, 300), (16, 1, 5000, 300)):
        size = P.phase2_tree_workspace_bytes(n, Tq, S, G, Hq, Hkv, d)
        for t in sizes[0]:
            for h in sizes[1]:
                for s in sizes[2]:
                    for g in sizes[3]:
                        if t <= Tq and h <= n and s <= S and g <= G:
                            got = call(Tq=t, n_shards=h, S=s, G=g, wsb=size)
                            assert got != EWS, (Tq, n, S, G, t, h, s, g)


def test_kv_compact():
    names = "K V layers capacity Hkv d G keep n stream"
    call = caller("pulsar_kv_compact", names, K=FAKE, V=2 * FAKE, layers=2, capacity=100, Hkv=8,
                  d=128, G=10, keep=FAKE, n=5)
    for kw in (dict(layers=-1), dict(capacity=-1), dict(Hkv=0), dict(d=0), dict(G=-1),
               dict(G=101), dict(n=-1), dict(n=91), dict(K=None), dict(V=None), dict(keep=None),
               dict(K=FAKE + 8), dict(V=FAKE + 2)):
        assert call(**kw) == EINVAL, kw
    assert call(Hkv=3, d=4) == EUNSUP
    assert call(layers=0, K=None, V=None) == 0 and call(n=0, keep=None) == 0


def test_key_bounds():
    call = caller("pulsar_key_bounds", "K n_shards S Hkv d block bounds stream", K=FAKE,
                  n_shards=2, S=100, Hkv=8, d=128, block=32, bounds=FAKE)
    for kw in (dict(n_shards=-1), dict(S=-1), dict(Hkv=0), dict(d=0), dict(block=0),
               dict(K=None), dict(bounds=None), dict(K=FAKE + 8), dict(bounds=FAKE + 8)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(d=32), dict(block=8), dict(block=48), dict(block=512), dict(S=1 << 31)):
        assert call(**kw) == EUNSUP, kw
    assert call(S=0, K=None, bounds=None) == 0 and call(n_shards=0) == 0


def test_block_select():
    names = "q bounds n_shards Tq blocks Hq Hkv d topk sel scores ws wsb stream"
    call = caller("pulsar_block_select", names, q=FAKE, bounds=FAKE, n_shards=2, Tq=3, blocks=50,
                  Hq=32, Hkv=8, d=128, topk=4, sel=FAKE, ws=FAKE, wsb=BIG)
    for kw in (dict(n_shards=-1), dict(Tq=-1), dict(blocks=-1), dict(Hq=0), dict(Hq=31),
               dict(d=0), dict(topk=-1), dict(topk=51), dict(q=None), dict(bounds=None),
               dict(sel=None), dict(q=FAKE + 8), dict(bounds=FAKE + 8)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(d=96), dict(blocks=32769), dict(n_shards=8192), dict(Tq=600000),
               dict(Tq=65536, Hkv=1), dict(n_shards=8, Tq=1 << 17),
               dict(n_shards=8, Tq=1 << 16, blocks=4097)):
        assert call(**kw) == EUNSUP, kw
    need = P.block_select_workspace_bytes(2, 3, 600, 32, 8)
    assert need > 0
    for kw in (dict(ws=None), dict(wsb=need - 1), dict(ws=FAKE + 8)):
        assert call(blocks=600, **kw) == EWS, kw
    for kw in (dict(n_shards=0), dict(Tq=0), dict(blocks=0, topk=0), dict(topk=0, sel=None)):
        assert call(**kw, ws=None) == 0, kw


def test_phase2_sparse():
    names = ("q K V sel n_shards Tq S block topk Kg Vg G mask Hq Hkv d scale o o_dtype lse ws wsb "
             "stream")
    call = caller("pulsar_phase2_sparse", names, q=FAKE, K=FAKE, V=FAKE, sel=FAKE, n_shards=2,
                  Tq=3, S=500, block=32, topk=4, Kg=FAKE, Vg=FAKE, G=10, Hq=32, Hkv=8, d=128,
                  scale=0.1, o=FAKE, o_dtype=0, ws=FAKE, wsb=BIG)
    for kw in (dict(n_shards=-1), dict(Tq=-1), dict(S=-1), dict(G=-1), dict(Hq=0), dict(Hq=31),
               dict(d=0), dict(block=0), dict(topk=-1), dict(scale=0.0), dict(scale=math.nan),
               dict(o_dtype=2), dict(q=None), dict(K=None), dict(V=None), dict(sel=None),
               dict(o=None), dict(Kg=None), dict(Vg=None), dict(Kg=None, Vg=None),
               dict(Kg=None, Vg=None, G=0, mask=FAKE), dict(q=FAKE + 8), dict(K=FAKE + 8),
               dict(V=FAKE + 8), dict(Kg=FAKE + 8), dict(o=FAKE + 8)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(d=96), dict(block=24), dict(block=8), dict(S=1 << 31), dict(G=1 << 24),
               dict(topk=1 << 25), dict(Hkv=1 << 17, Hq=1 << 17), dict(Tq=1 << 23, Hq=128),
               dict(Tq=1 << 23, Hkv=1, Hq=32)):
        assert call(**kw) == EUNSUP, kw
    assert P.phase2_sparse_workspace_bytes(3, 32, 8, 128) > 0
    for kw in (dict(ws=None), dict(wsb=16), dict(ws=FAKE + 8)):
        assert call(topk=60, **kw) == EWS, kw
    assert call(Tq=0) == 0


def test_phase2_sparse_workspace_serves_fewer_tokens():
    if torch.cuda.is_available():
        pytest.skip("the calls would be launched")
    names = ("q K V sel n_shards Tq S block topk Kg Vg G mask Hq Hkv d scale o o_dtype lse ws wsb "
             "stream")
    for Hq, Hkv in ((32, 8), (4, 1), (16, 16), (64, 1)):
        call = caller("pulsar_phase2_sparse", names, q=FAKE, K=FAKE, V=FAKE, sel=FAKE, block=32,
                      Kg=FAKE, Vg=FAKE, Hq=Hq, Hkv=Hkv, d=128, scale=0.1, o=FAKE, o_dtype=0,
                      ws=FAKE)
        for most in (1, 5, 64, 1000):
            size = P.phase2_sparse_workspace_bytes(most, Hq, Hkv, 128)
            for Tq in (1, 2, 3, 5, 17, 64, 300, 1000):
                for n, topk, G in ((1, 1, 0), (1, 300, 0), (16, 64, 5000)):
                    if Tq <= most:
                        assert call(Tq=Tq, n_shards=n, S=99999, topk=topk, G=G, wsb=size) != EWS


def test_phase2_sparse_call_bytes():
    # what a call takes: never more than the size for all calls, and neither less
    lib = _lib.lib()
    names = ("q K V sel n_shards Tq S block topk Kg Vg G mask Hq Hkv d scale o o_dtype lse ws wsb "
             "stream")
    for Hq, Hkv, d in ((32, 8, 128), (4, 1, 64), (16, 16, 64), (64, 1, 128), (28, 4, 128)):
        call = caller("pulsar_phase2_sparse", names, q=FAKE, K=FAKE, V=FAKE, sel=FAKE, block=32,
                      S=99999, Hq=Hq, Hkv=Hkv, d=d, scale=0.1, o=FAKE, o_dtype=0, ws=FAKE)
        for Tq in (1, 2, 5, 64, 1000):
            for n, topk, G in ((0, 0, 0), (1, 1, 0), (1, 300, 31), (16, 64, 5000), (2, 9, 100000)):
                for gen in (0, G + Tq):
                    size = lib.pulsar_phase2_sparse_call_bytes(n, Tq, 99999, 32, topk, gen, Hq, Hkv,
                                                               d)
                    assert size <= P.phase2_sparse_workspace_bytes(Tq, Hq, Hkv, d)
                    if gen:
                        assert size == lib.pulsar_phase2_sparse_call_bytes(
                            n, Tq, 99999, 32, topk, gen + 31 & ~31, Hq, Hkv, d)
                    kv = dict(Kg=FAKE, Vg=FAKE, G=G) if gen else dict(G=0)
                    if size:
                        assert call(n_shards=n, Tq=Tq, topk=topk, wsb=size - 1, **kv) == EWS
                    if not torch.cuda.is_available():
                        assert call(n_shards=n, Tq=Tq, topk=topk, wsb=size, **kv) != EWS
    for bad in ((-1, 1, 1, 32, 1, 0, 8, 8, 64), (1, 0, 1, 32, 1, 0, 8, 8, 64),
                (1, 1, -1, 32, 1, 0, 8, 8, 64), (1, 1, 1, 24, 1, 0, 8, 8, 64),
                (1, 1, 1, 32, -1, 0, 8, 8, 64), (1, 1, 1, 32, 1, -1, 8, 8, 64),
                (1, 1, 1, 32, 1, 0, 8, 3, 64), (1, 1, 1, 32, 1, 0, 8, 0, 64),
                (1, 1, 1, 32, 1, 0, 8, 8, 96)):
        assert lib.pulsar_phase2_sparse_call_bytes(*bad) == 0


def test_binding_refuses_host_tensors():
    t = torch.zeros((1, 32, 1, 64), dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    for fn in (lambda: P.key_bounds(t, 16), lambda: P.tree_mask(i),
               lambda: P.kv_compact_(t, t.clone(), 0, i),
               lambda: P.block_select(t[0], t, 1), lambda: P.phase2_sparse(t[0], t, t, i, 16),
               lambda: P.phase2_tree(t[0], t[0], t[0], 0, i)):
        with pytest.raises(ValueError):
            fn()
