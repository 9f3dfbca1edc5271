"""Refusals of the entry points of a cache held in 8 bits, on the host before any GPU
call (runs without a GPU)."""
import math

import pytest
import torch

import paper_2607_20457_amd as P
from paper_2607_20457_amd import _lib
from tests.test_abi_blocks import BIG, EINVAL, EUNSUP, EWS, FAKE, caller

EHIP = -3  # (without a GPU: what a call that is not refused ends with)
QUANTIZE = ("K V shard_stride row_stride n rows Hkv d block format first capacity kc vc ks vs "
            "stream")
DEQUANTIZE = "kc vc ks vs n capacity Hkv d block format first rows K V stream"
ATTN = ("q kc vc ks vs n_shards Tq S block format rows Kg Vg G mask Hq Hkv d scale o o_dtype lse "
        "ws wsb stream")


# apart from each other: rows of K and V, codes of 2 x 8 x 200 x 64, scales of 2 x 8 x 7
KC, VC, KS, VS = 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE


def quantizer(**kw):
    ok = dict(K=FAKE, V=FAKE, shard_stride=800, row_stride=512, n=2, rows=50, Hkv=8, d=64,
              block=32, format=0, first=64, capacity=200, kc=KC, vc=VC, ks=KS, vs=VS)
    return caller("pulsar_kv_quantize", QUANTIZE, **{**ok, **kw})


def attention(**kw):
    ok = dict(q=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, n_shards=2, Tq=3, S=500, block=32,
              format=0, Kg=FAKE, Vg=FAKE, G=10, Hq=32, Hkv=8, d=128, scale=0.1, o=FAKE, o_dtype=0,
              ws=FAKE, wsb=BIG)
    return caller("pulsar_phase2_quant", ATTN, **{**ok, **kw})


def test_kv_quantize():
    call = quantizer()
    for kw in (dict(n=-1), dict(rows=-1), dict(Hkv=0), dict(d=0), dict(block=0), dict(format=2),
               dict(format=-1), dict(first=-32), dict(capacity=-1), dict(first=224),
               dict(rows=137), dict(rows=1 << 62), dict(first=1 << 62), dict(first=48),
               dict(K=None), dict(V=None), dict(kc=None), dict(vc=None), dict(ks=None),
               dict(vs=None), dict(K=FAKE + 8), dict(V=FAKE + 2), dict(kc=FAKE + 8),
               dict(vc=FAKE + 1), dict(shard_stride=801), dict(row_stride=516)):
        assert call(**kw) == EINVAL, kw
    # memory in common
    rows = ((800 + 49 * 512) + 8 * 64) * 2
    codes, scales = 2 * 8 * 200 * 64, 2 * 8 * 7 * 4
    for kw in (dict(vc=KC), dict(vs=KS), dict(kc=FAKE), dict(vc=KC + codes - 16), dict(ks=KC),
               dict(ks=KC + codes - 4), dict(vs=KS - scales + 4), dict(kc=FAKE + rows - 16),
               dict(V=KC + codes - 16), dict(K=VC - rows + 16),
               dict(K=VC + codes + 800 * 2 - 16, shard_stride=-800),
               dict(V=VS + 49 * 512 * 2, row_stride=-512), dict(K=FAKE, shard_stride=1 << 61)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(vc=KC + codes), dict(vs=KS + scales), dict(kc=FAKE + rows),
               dict(K=VC + codes + 800 * 2, shard_stride=-800), dict(V=FAKE + 16)):
        if not torch.cuda.is_available():
            assert call(**kw) == EHIP, kw
    for kw in (dict(d=96), dict(block=8, first=0), dict(block=48, first=48),
               dict(block=512, first=0), dict(capacity=1 << 31), dict(Hkv=1 << 17),
               dict(n=1 << 22, capacity=1 << 20, Hkv=1),
               dict(n=1 << 24, kc=1 << 50, vc=1 << 51, ks=1 << 52, vs=1 << 53, K=1 << 54, V=1 << 54)):
        assert call(**kw) == EUNSUP, kw
    assert call(n=0, K=None, V=None) == 0 and call(rows=0, K=None, kc=None) == 0
    assert call(capacity=0, first=0, rows=0) == 0


def test_kv_dequantize():
    call = caller("pulsar_kv_dequantize", DEQUANTIZE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, n=2,
                  capacity=200, Hkv=8, d=64, block=32, format=1, first=3, rows=50, K=FAKE, V=FAKE)
    for kw in (dict(n=-1), dict(rows=-1), dict(Hkv=0), dict(d=0), dict(block=0), dict(format=2),
               dict(first=-1), dict(capacity=-1), dict(first=201), dict(rows=198),
               dict(rows=1 << 62), dict(K=None), dict(V=None), dict(kc=None), dict(vc=None),
               dict(ks=None), dict(vs=None), dict(K=FAKE + 8), dict(V=FAKE + 2),
               dict(kc=FAKE + 8), dict(vc=FAKE + 1)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(d=96), dict(block=8), dict(block=48), dict(block=512),
               dict(capacity=1 << 31), dict(Hkv=1 << 17), dict(n=1 << 30),
               dict(n=(1 << 31) - 1, capacity=(1 << 31) - 64, rows=(1 << 31) - 100, Hkv=1 << 16),
               dict(n=1 << 22, capacity=1 << 20, Hkv=1)):
        assert call(**kw) == EUNSUP, kw
    assert call(n=0, K=None) == 0 and call(rows=0, K=None, kc=None) == 0


def test_phase2_quant():
    call = attention()
    for kw in (dict(n_shards=-1), dict(Tq=-1), dict(S=-1), dict(G=-1), dict(Hq=0), dict(Hkv=0),
               dict(Hq=31), dict(d=0), dict(block=0), dict(format=2), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(o_dtype=2),
               dict(q=None), dict(kc=None), dict(vc=None), dict(ks=None), dict(vs=None),
               dict(o=None), dict(Kg=None), dict(Vg=None), dict(Kg=None, Vg=None),
               dict(Kg=None, Vg=None, G=0, mask=FAKE), dict(q=FAKE + 8), dict(kc=FAKE + 8),
               dict(vc=FAKE + 8), dict(Kg=FAKE + 8), dict(Vg=FAKE + 2), dict(o=FAKE + 8)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(d=96), dict(block=24), dict(block=8), dict(S=1 << 31), dict(G=1 << 24),
               dict(G=1 << 62), dict(n_shards=1 << 20, S=1 << 11), dict(n_shards=1 << 30, S=1),
               dict(n_shards=1025, rows=FAKE),
               dict(Hkv=1 << 17, Hq=1 << 17), dict(Tq=1 << 23, Hq=128),
               dict(Tq=1 << 23, Hkv=1, Hq=128)):
        assert call(**kw) == EUNSUP, kw
    size = P.phase2_quant_workspace_bytes(3, 32, 8, 128)
    assert size > 0
    for kw in (dict(ws=None), dict(wsb=16), dict(ws=FAKE + 8)):
        assert call(S=50000, **kw) == EWS, kw
    assert call(Tq=0) == 0


LAYERS = [(32, 8, 128), (4, 1, 64), (16, 16, 64), (64, 1, 64), (28, 4, 128), (200, 2, 64)]


@pytest.mark.parametrize("Hq,Hkv,d", LAYERS)
def test_workspace_serves_fewer_tokens(Hq, Hkv, d):
    if torch.cuda.is_available():
        pytest.skip("the calls would be launched")
    call = attention(Hq=Hq, Hkv=Hkv, d=d)
    for most in (1, 5, 64, 1000):
        size = P.phase2_quant_workspace_bytes(most, Hq, Hkv, d)
        for Tq in (1, 2, 3, 4, 5, 8, 9, 17, 33, 64, 65, 300, 1000):
            for n, S, G in ((0, 0, 0), (1, 1, 0), (1, 300, 0), (16, 64, 5000), (7, 99999, 31)):
                if Tq <= most:
                    assert call(Tq=Tq, n_shards=n, S=S, G=G, wsb=size) != EWS, (Tq, most, n, S)


@pytest.mark.parametrize("Hq,Hkv,d", LAYERS)
def test_call_bytes(Hq, Hkv, d):
    # what a call takes: never more than the size for all calls, and neither less
    fn = _lib.lib().pulsar_phase2_quant_call_bytes
    call = attention(Hq=Hq, Hkv=Hkv, d=d)
    for Tq in (1, 2, 5, 64, 1000):
        for n, S, G in ((0, 0, 0), (1, 1, 0), (1, 300, 31), (16, 64, 5000), (2, 99999, 100000)):
            for gen in (0, G + Tq):
                size = fn(n, Tq, S, gen, Hq, Hkv, d)
                assert size <= P.phase2_quant_workspace_bytes(Tq, Hq, Hkv, d)
                if gen:
                    assert size == fn(n, Tq, S, gen + 31 & ~31, Hq, Hkv, d)
                kv = dict(G=G) if gen else dict(Kg=None, Vg=None, G=0)
                if size:
                    assert call(n_shards=n, Tq=Tq, S=S, wsb=size - 1, **kv) == EWS
                if not torch.cuda.is_available():
                    assert call(n_shards=n, Tq=Tq, S=S, wsb=size, **kv) != EWS
    for bad in ((-1, 1, 1, 0, 8, 8, 64), (1, 0, 1, 0, 8, 8, 64), (1, 1, -1, 0, 8, 8, 64),
                (1, 1, 1 << 31, 0, 8, 8, 64), (1, 1, 1, -1, 8, 8, 64), (1, 1, 1, 0, 8, 3, 64),
                (1, 1, 1, 0, 8, 0, 64), (1, 1, 1, 0, 8, 8, 96)):
        assert fn(*bad) == 0
    for bad in ((-1, 8, 8, 64), (1, 0, 8, 64), (1, 8, 0, 64), (1, 8, 3, 64), (1, 8, 8, 0)):
        assert P.phase2_quant_workspace_bytes(*bad) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    t = torch.zeros((1, 32, 1, 64), dtype=torch.bfloat16)
    c = torch.zeros((1, 1, 32, 64), dtype=torch.int8)
    s = torch.zeros((1, 1, 2))
    for fn in (lambda: P.kv_quantize(t, t, 16), lambda: P.kv_quantize_(t, t, c, c, s, s, 16),
               lambda: P.kv_dequantize(c, c, s, s, 16),
               lambda: P.phase2_quant(t[0], c, c, s, s, 16),
               lambda: P.kv_quantize(t, t, 16, torch.uint8),
               lambda: P.kv_quantize(t, t, 16, capacity=31), lambda: P.kv_quantize(t, t, 0),
               lambda: P.kv_quantize(t[0], t[0], 16), lambda: P.kv_quantize(t, t, (1 << 32) + 16)):
        with pytest.raises(ValueError):
            fn()
