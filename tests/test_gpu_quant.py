"""A cache held in 8 bits on the GPU: kv_quantize, kv_dequantize and phase2_quant against
oracle.quant and oracle.blocks (tolerances: tests._blocks.check)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_20457_amd as P
from tests._blocks import dev_i32, dev_mask, random_tree
from oracle import blocks as ob
from tests._quant import (DTYPES, check, codes_of, dev_cache, dev_codes, f64, host, normal, oq,
                          long_reference, reference, softmax_scale, spread, to_dev_bf16)

pytestmark = pytest.mark.gpu

FMTS = ["e4m3", "int8"]


# ---- quantising -------------------------------------------------------------------


def _same_cache(cache, k, v, block, fmt, what, rows=None):
    for name, codes, scale, x in (("K", cache[0], cache[2], k), ("V", cache[1], cache[3], v)):
        want, s = oq.quantize(f64(x), block, fmt)
        got = codes_of(codes)[:, :, :rows], host(scale)[:, :, :s.shape[2]]
        assert np.array_equal(got[1], s, equal_nan=True), f"{what}: scales of {name}"
        assert np.array_equal(got[0], want), f"{what}: codes of {name}"


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n,rows,Hkv,d,block", [
    (1, 1, 1, 64, 16),            # one row
    (1, 64, 1, 128, 64),
    (2, 65, 3, 64, 64),           # a row in a block of its own, heads that fill no workgroup
    (3, 200, 8, 128, 16),
    (2, 129, 5, 128, 32),
    (2, 300, 2, 128, 128),        # blocks of two waves
    (2, 700, 3, 64, 256),         # and of four
    (1, 257, 1, 128, 256),
    (5, 1021, 4, 64, 128),
])
def test_quantize(n, rows, Hkv, d, block, fmt):
    k, v = (spread(s, (n, rows, Hkv, d)) for s in (1, 2))
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block, DTYPES[fmt])
    assert cache[0].shape == (n, Hkv, rows, d) and cache[0].dtype == DTYPES[fmt]
    _same_cache(cache, k, v, block, fmt, f"{n}x{rows}x{Hkv}x{d} block {block}")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("block", [16, 64, 256])
def test_quantize_every_magnitude(fmt, block):
    # every finite bf16 number, of like size in a block: zeros, subnormals, the largest
    bits = np.arange(0x7f80, dtype=np.uint16)
    bits = np.stack([bits, bits | 0x8000], axis=1).reshape(-1)
    rows = -(-bits.size // 64)
    k = np.zeros((1, rows, 1, 64), dtype=np.uint16)
    k.reshape(-1)[:bits.size] = bits
    v = k[:, ::-1].copy()
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block, DTYPES[fmt])
    _same_cache(cache, k, v, block, fmt, f"{fmt} block {block}")
    back = P.kv_dequantize(*cache, block)
    assert all(bool(torch.isfinite(x).all()) for x in back)


@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_ties(fmt):
    # values half way between two codes of a block whose scale is 1
    top = 448 if fmt == "e4m3" else 127
    table = oq.e4m3_values() if fmt == "e4m3" else np.arange(128.0)
    mid = (table[1:] + table[:-1]) / 2
    x = np.concatenate([[top], mid, -mid])
    x = np.resize(x, 16 * 64).reshape(1, 16, 1, 64)
    k = torch.from_numpy(x).to(torch.bfloat16)
    assert np.array_equal(k.double().numpy(), x)
    bits = k.view(torch.int16).numpy().view(np.uint16)
    cache = P.kv_quantize(k.cuda(), -k.cuda(), 16, DTYPES[fmt])
    _same_cache(cache, bits, bits ^ 0x8000, 16, fmt, "ties")
    assert (cache[2] == 1).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("block", [16, 128])
def test_quantize_what_is_not_finite(fmt, block):
    n, rows, Hkv, d = 2, 300, 5, 64
    k, v = (spread(s, (n, rows, Hkv, d)) for s in (3, 4))
    for i, bits in enumerate((0x7fc0, 0xff80, 0x7f80, 0xffff, 0x7f81)):
        k[i % n, 37 * (i + 1), i, 5 * i] = bits
        v[1 - i % n, 299 - 70 * i, 4 - i, 63] = bits
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block, DTYPES[fmt])
    _same_cache(cache, k, v, block, fmt, f"{fmt} block {block}")
    K, _ = P.kv_dequantize(*cache, block)
    want = np.isnan(oq.values(*oq.quantize(f64(k), block, fmt), block))
    assert np.array_equal(torch.isnan(K).cpu().numpy(), want) and want.any()


@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_into_a_cache(fmt):
    # rows of a longer generation shard, strided, into the middle of a cache; what is not
    # written stays as it was
    layers, Hkv, d, block, capacity = 3, 4, 128, 32, 250
    first, rows = 96, 70
    k, v = (spread(s, (layers, 200, Hkv, d)) for s in (5, 6))
    K, V = to_dev_bf16(k), to_dev_bf16(v)
    codes = [torch.full((layers, Hkv, capacity, d), 0x5a, dtype=torch.uint8, device="cuda")
             for _ in range(2)]
    scales = [torch.full((layers, Hkv, 8), -7.0, device="cuda") for _ in range(2)]
    cache = [c.view(DTYPES[fmt]) for c in codes] + scales
    out = P.kv_quantize_(K[:, 41:41 + rows], V[:, 41:41 + rows], *cache, block, first)
    assert all(a is b for a, b in zip(out, cache))
    for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
        want, ws = oq.quantize(f64(x[:, 41:41 + rows]), block, fmt)
        assert np.array_equal(codes_of(c.view(DTYPES[fmt]))[:, :, first:first + rows], want)
        assert np.array_equal(host(s)[:, :, 3:6], ws)
        assert (c[:, :, :first] == 0x5a).all() and (c[:, :, first + rows:] == 0x5a).all()
        assert (s[:, :, :3] == -7).all() and (s[:, :, 6:] == -7).all()
    # the last block, which was short, again from its first row with one row more
    P.kv_quantize_(K[:, 105:112], V[:, 105:112], *cache, block, 160)
    want, ws = oq.quantize(f64(k[:, 105:112]), block, fmt)
    assert np.array_equal(codes_of(cache[0])[:, :, 160:167], want)
    assert np.array_equal(host(scales[0])[:, :, 5:6], ws) and (scales[0][:, :, 6:] == -7).all()


def test_quantize_strided_sources():
    # K and V inside one fused projection, rows and shards far apart; and a broadcast shard
    n, rows, Hkv, d = 2, 50, 2, 64
    x = spread(7, (n, rows, 3 * Hkv, d))
    X = to_dev_bf16(x)
    cache = P.kv_quantize(X[:, :, Hkv:2 * Hkv], X[:, :, 2 * Hkv:], 16)
    _same_cache(cache, x[:, :, Hkv:2 * Hkv], x[:, :, 2 * Hkv:], 16, "e4m3", "fused")
    every = X[:, ::3, :Hkv]
    cache = P.kv_quantize(every, every, 16)
    _same_cache(cache, x[:, ::3, :Hkv], x[:, ::3, :Hkv], 16, "e4m3", "every third row")
    same = X[:1, :, :Hkv].expand(4, rows, Hkv, d)
    cache = P.kv_quantize(same, same, 16)
    _same_cache(cache, *(np.repeat(x[:1, :, :Hkv], 4, axis=0),) * 2, 16, "e4m3", "expanded")


def test_quantize_refusals():
    bf = dict(dtype=torch.bfloat16, device="cuda")
    K, V = torch.zeros(2, 40, 4, 64, **bf), torch.zeros(2, 40, 4, 64, **bf)
    cache = P.kv_quantize(K, V, 16, capacity=64)
    Kc, Vc, ks, vs = cache
    wrong = [
        lambda: P.kv_quantize_(K.float(), V, *cache, 16), lambda: P.kv_quantize_(K, V.cpu(), *cache, 16),
        lambda: P.kv_quantize_(K, V[:, :39], *cache, 16), lambda: P.kv_quantize_(K[:1], V[:1], *cache, 16),
        lambda: P.kv_quantize_(K, V.transpose(1, 2).contiguous().transpose(1, 2), *cache, 16),
        lambda: P.kv_quantize_(K, V, *cache, 32), lambda: P.kv_quantize_(K, V, *cache, 16, 25),
        lambda: P.kv_quantize_(K, V, *cache, 16, 32), lambda: P.kv_quantize_(K, V, *cache, 16, 1 << 64),
        lambda: P.kv_quantize_(K, V, *cache, 16, -16),
        lambda: P.kv_quantize_(K, V, Kc, Vc.view(torch.int8), ks, vs, 16),
        lambda: P.kv_quantize_(K, V, Kc.view(torch.uint8), Vc.view(torch.uint8), ks, vs, 16),
        lambda: P.kv_quantize_(K, V, Kc, Vc, ks.double(), vs.double(), 16),
        lambda: P.kv_quantize_(K, V, Kc, Vc, ks[:, :, :3], vs[:, :, :3], 16),
        lambda: P.kv_quantize_(K[..., ::2], V[..., ::2], *cache, 16),
        lambda: P.kv_quantize(K, V, 16, torch.float8_e5m2), lambda: P.kv_quantize(K, V, 16, capacity=39),
        lambda: P.kv_dequantize(*cache, 16, 60, 5), lambda: P.kv_dequantize(*cache, 16, -1),
        lambda: P.kv_dequantize(*cache, 16, 65), lambda: P.kv_dequantize(*cache, 16, 0, -1),
        lambda: P.kv_dequantize(Kc[:, :, ::2], Vc[:, :, ::2], ks, vs, 32),
        lambda: P.kv_dequantize(Kc.cpu(), Vc, ks, vs, 16),
    ]
    for i, fn in enumerate(wrong):
        with pytest.raises(ValueError):
            fn()
            pytest.fail(f"call {i} was not refused")
    # a source that begins inside the cache, and rows whose strides are no multiple of 8
    raw = torch.zeros(2 * 4 * 64 * 64 * 3, dtype=torch.uint8, device="cuda")
    inside = raw.view(torch.bfloat16)[4096:4096 + 2 * 40 * 256].view(2, 40, 4, 64)
    outer = raw[:32768].view(torch.int8).view(2, 4, 64, 64), torch.zeros_like(Kc).view(torch.int8)
    odd = torch.zeros(2, 40, 260, **bf)[:, :, :256].unflatten(2, (4, 64))
    small = torch.zeros(1, 16, 1, 32, **bf)
    for fn in (lambda: P.kv_quantize_(inside, inside, *outer, ks, vs, 16),
               lambda: P.kv_quantize_(K, V, Kc, Kc, ks, vs, 16),
               lambda: P.kv_quantize_(K, V, Kc, Vc, ks, ks, 16),
               lambda: P.kv_quantize_(odd, odd, *cache, 16), lambda: P.kv_quantize_(K, V, *cache, 16, 8),
               lambda: P.kv_quantize(K, V, 24), lambda: P.kv_quantize(small, small, 16)):
        with pytest.raises(RuntimeError):
            fn()


# ---- reading back -------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n,cap,Hkv,d,block,first,rows", [
    (1, 1, 1, 64, 16, 0, 1), (2, 130, 5, 128, 16, 0, 130), (2, 130, 5, 128, 64, 33, 71),
    (3, 700, 2, 64, 256, 255, 300), (1, 100, 9, 64, 32, 100, 0), (4, 65, 1, 128, 128, 64, 1),
])
def test_dequantize(n, cap, Hkv, d, block, first, rows, fmt):
    # any scales, also ones that are no power of two: the product in fp32, rounded once
    rng = np.random.default_rng(11)
    raw = rng.integers(0, 256, (2, n, Hkv, cap, d)).astype(np.uint8)
    codes = [torch.from_numpy(x).cuda().view(DTYPES[fmt]) for x in raw]
    scales = [torch.from_numpy(np.exp(rng.uniform(-40, 40, (n, Hkv, -(-cap // block)))
                                      ).astype(np.float32)).cuda() for _ in range(2)]
    got = P.kv_dequantize(*codes, *scales, block, first, rows)
    for x, c, s in zip(got, codes, scales):
        want = c.cpu().float() * torch.repeat_interleave(s.cpu(), block, 2)[:, :, :cap, None]
        want = want[:, :, first:first + rows].transpose(1, 2).to(torch.bfloat16)
        assert x.shape == (n, rows, Hkv, d)
        assert torch.equal(torch.isnan(x).cpu(), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(x.cpu()), torch.nan_to_num(want))


@pytest.mark.parametrize("fmt", FMTS)
def test_read_back_again(fmt):
    # what a cache stands for is bf16, and quantises to itself
    k, v = (spread(s, (2, 333, 3, 64)) for s in (12, 13))
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), 64, DTYPES[fmt])
    back = P.kv_dequantize(*cache, 64)
    for x, bits in zip(back, (k, v)):
        assert np.array_equal(host(x), oq.values(*oq.quantize(f64(bits), 64, fmt), 64))
    again = P.kv_dequantize(*P.kv_quantize(*back, 64, DTYPES[fmt]), 64)
    assert all(torch.equal(a, b) for a, b in zip(back, again))


# ---- attention ------------------------------------------------------------------------


def _attn(Hq, Hkv, d, Tq, G, n, S, block, fmt, seed, sees=None, rows=None, gen=True,
          bf16_out=False, q_scale=1.0, what="", long=False):
    print(f"phase2_quant parity: {what} Hq={Hq} Hkv={Hkv} d={d} Tq={Tq} G={G} {n}x{S} "
          f"block={block} {fmt}", flush=True)
    q = normal(seed, (Tq, Hq, d), q_scale)
    k, v = (spread(seed + i, (n, S, Hkv, d)) for i in (1, 2))
    kg, vg = (normal(seed + i, (G + Tq, Hkv, d)) for i in (3, 4)) if gen else (None, None)
    if long:  # (the oracle quantises block by block)
        cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block, DTYPES[fmt])
    else:
        cache, (K, V) = dev_cache(k, v, block, fmt)
    o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block,
                            None if rows is None else dev_i32(rows),
                            *((to_dev_bf16(kg), to_dev_bf16(vg), G) if gen else ()),
                            mask=None if sees is None else dev_mask(sees),
                            o_dtype=P.OUT_BF16 if bf16_out else P.OUT_F32)
    rest = rows, kg, vg, G, sees, softmax_scale(d)
    ref, keys = long_reference(q, cache, block, *rest) if long else reference(q, K, V, *rest)
    check(o, lse, ref, max(keys, 1), what, bf16_out)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("Hq,Hkv,d,Tq,G,n,S,block", [
    (32, 8, 128, 1, 0, 1, 1, 16),        # one retained key and the token's own
    (32, 8, 128, 1, 45, 4, 251, 64),
    (4, 1, 64, 1, 31, 1, 33, 32),
    (4, 1, 64, 5, 100, 3, 64, 128),      # a block longer than its shard
    (16, 16, 64, 24, 70, 2, 130, 32),    # one head per KV head
    (8, 2, 128, 17, 33, 2, 190, 16),
    (32, 8, 128, 64, 5, 1, 320, 256),    # many rows
    (6, 2, 64, 7, 3, 2, 100, 64),        # three heads per KV head
    (28, 4, 128, 3, 9, 2, 77, 16),       # seven
    (32, 1, 64, 2, 9, 1, 140, 64),       # 32: more than a tile's columns
    (70, 1, 128, 1, 0, 1, 65, 16),       # 70
    (40, 2, 64, 3, 2, 2, 90, 32),        # 20
    (8, 8, 128, 1, 0, 1, 700, 64),
    (8, 8, 64, 100, 0, 1, 63, 64),       # a long question, mostly among its own rows
    (4, 4, 128, 33, 31, 0, 0, 64),       # no shard at all
])
def test_attention(Hq, Hkv, d, Tq, G, n, S, block, fmt):
    _attn(Hq, Hkv, d, Tq, G, n, S, block, fmt, 100 + Tq, bf16_out=Tq % 2 == 0, what="parity")


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_of_the_shards_alone(fmt):
    _attn(32, 8, 128, 2, 0, 3, 100, 32, fmt, 120, gen=False, what="no generation shard")
    _attn(8, 8, 64, 40, 0, 1, 400, 16, fmt, 121, gen=False, what="no generation shard")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("Hq,Hkv,d,Tq", [(8, 2, 128, 1), (16, 16, 64, 3), (8, 1, 64, 20)])
def test_attention_over_many_steps(Hq, Hkv, d, Tq, fmt):
    # more steps than a wave's table holds at a time
    _attn(Hq, Hkv, d, Tq, 400, 2, 9000 // Tq + 3000 // Tq, 64, fmt, 130, what="long")
    _attn(Hq, Hkv, d, Tq, 9000 // Tq, 1, 70, 64, fmt, 131, what="long generation")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("Hq,Hkv,d,Tq,n,S", [
    (64, 64, 128, 1, 1, 3500),    # 16 columns: three steps of every wave, most of them whole
    (128, 128, 128, 1, 1, 17600), # more steps than a wave's table holds at a time
    (128, 64, 128, 20, 1, 4700),  # 48 columns, 40 of them in use
    (64, 8, 128, 6, 3, 12500),    # 48, whole ones
    (64, 64, 128, 192, 1, 8700),  # four tiles of 48, more than the table
    (64, 64, 128, 30, 1, 7100),   # 32 columns in steps of 32 rows
    (16, 16, 128, 64, 1, 14000),  # two tiles of 32
    (16, 16, 128, 256, 1, 17600), # 32 columns in steps of 64 rows, more than the table
    (64, 64, 64, 128, 1, 8700),   # 32 columns of heads of 64
    (32, 32, 64, 256, 1, 17000),  # more than the table
    (60, 4, 64, 20, 2, 8300),     # 15 heads per KV head
])
def test_attention_of_full_waves(Hq, Hkv, d, Tq, n, S, fmt):
    _attn(Hq, Hkv, d, Tq, 70, n, S, 64, fmt, 135, what="full waves", long=True)
    # a tree of drafts over shards that are filled to different lengths
    rng = np.random.default_rng(136)
    sees, _ = ob.tree_visible(random_tree(Tq, Tq))
    rows = np.r_[S - rng.integers(0, 500, n - 1), S - 77]
    _attn(Hq, Hkv, d, Tq, 13, n, S, 16, fmt, 137, sees=sees, rows=rows, bf16_out=True,
          what="full waves, a tree, lengths", long=True)


@pytest.mark.parametrize("lengths", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,Tq,n,S", [
    (32, 8, 128, 1, 4, 1021), (16, 16, 64, 24, 5, 3001), (32, 8, 128, 12, 4, 8192),
    (32, 8, 128, 12, 16, 8192), (64, 8, 128, 6, 3, 12500), (32, 8, 128, 8, 7, 9999),
    (16, 16, 128, 64, 1, 14000), (64, 64, 64, 128, 1, 8700), (20, 1, 64, 3, 2, 77),
    (16, 16, 128, 256, 1, 17600),
])
def test_every_row_counts_once(Hq, Hkv, d, Tq, n, S, lengths):
    # Equal weights and a code in every row of V: a row that a plan drops, doubles or replaces
    # shows as a whole 1 in a channel.  Scores are 0, weights and their sums whole numbers, so
    # that only the log-sum-exps of the parts (log2 of at most 2^18, off by an ulp of it and
    # of its product: 2^-18), the weights that merge them and a division are rounded.
    G, rng = 45, np.random.default_rng(160)
    rows = rng.integers(0, S + 1, n) if lengths else np.full(n, S)
    rows[-1] = S - 13 * lengths
    q = torch.zeros((Tq, Hq, d), dtype=torch.bfloat16, device="cuda")
    k, kg = (torch.ones(x, dtype=torch.bfloat16, device="cuda")
             for x in ((n, S, Hkv, d), (G + Tq, Hkv, d)))
    nth = np.arange(n * S).reshape(n, S)
    live = np.arange(S) < rows[:, None]
    for code in (lambda i: i % d, lambda i: i // d % d):
        vs, vg = (torch.nn.functional.one_hot(torch.from_numpy(code(i)).cuda(), d)
                  .to(torch.bfloat16).unsqueeze(-2).expand(*i.shape, Hkv, d).contiguous()
                  for i in (nth, n * S + np.arange(G + Tq)))
        o, lse = P.phase2_quant(q, *P.kv_quantize(k, vs, 64), 64,
                                dev_i32(rows) if lengths else None, kg, vg, G)
        counts = np.bincount(code(nth)[live], minlength=d).astype(float)
        for i in range(G):
            counts[code(n * S + i)] += 1
        for t in range(Tq):
            counts[code(n * S + G + t)] += 1
            total = counts.sum()
            assert np.abs(host(o[t]) * total - counts).max() <= 2.0 ** -16 * counts.max(), t
            assert np.abs(host(lse[:, t]) - math.log(total)).max() <= 2.0 ** -17, t


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("block", [16, 64, 256])
def test_attention_over_live_rows(block, fmt):
    # lengths of zero, one, past the shard and negative; behind them codes and scales of
    # anything, NaN included
    Hq, Hkv, d, Tq, G, n, S = 8, 2, 128, 3, 20, 9, 300
    rows = np.array([0, 1, 300, 17, -5, 299, 400, 64, 2**31 - 1])
    q = normal(140, (Tq, Hq, d))
    k, v = (spread(s, (n, S, Hkv, d)) for s in (141, 142))
    kg, vg = (normal(s, (G + Tq, Hkv, d)) for s in (143, 144))
    cache, vals = dev_cache(k, v, block, fmt)
    for i, live in enumerate(np.clip(rows, 0, S)):
        for c, s in ((cache[0], cache[2]), (cache[1], cache[3])):
            c.view(torch.uint8)[i, :, live:] = 0x7f
            s[i, :, -(-live // block):] = math.nan
    for what, r in (("some", rows), ("none", np.zeros(n)), ("all but the first", np.r_[0, [S] * 8])):
        if what == "all but the first":
            cache, vals = dev_cache(k, v, block, fmt)
        o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block, dev_i32(r), to_dev_bf16(kg),
                                to_dev_bf16(vg), G)
        ref, keys = reference(q, *vals, r, kg, vg, G, None, softmax_scale(d))
        check(o, lse, ref, keys, what)
        o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block, dev_i32(r))
        ref, keys = reference(q, *vals, r, None, None, 0, None, softmax_scale(d))
        check(o, lse, ref, max(keys, 1), f"{what}, shards alone")


def test_attention_over_many_shards_with_lengths():
    rng = np.random.default_rng(150)
    for n, S in ((1024, 33), (300, 130), (257, 64)):
        rows = rng.integers(0, S + 1, n) * rng.integers(0, 2, n)
        _attn(4, 1, 64, 2, 10, n, S, 32, "int8", 151, rows=rows, what=f"{n} shards")
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    c = torch.zeros((1025, 1, 16, 64), dtype=torch.int8, device="cuda")
    s = torch.ones((1025, 1, 1), device="cuda")
    with pytest.raises(RuntimeError):
        P.phase2_quant(q, c, c, s, s, 16, dev_i32(np.zeros(1025)))
    o, lse = P.phase2_quant(q, c, c, s, s, 16)
    assert (o == 0).all() and torch.allclose(lse, torch.full_like(lse, math.log(1025 * 16)))


@pytest.mark.parametrize("Hq,Hkv,d,Tq,G", [(32, 8, 128, 12, 45), (4, 4, 64, 40, 20),
                                           (8, 1, 64, 70, 0), (2, 2, 128, 33, 31)])
def test_attention_of_trees(Hq, Hkv, d, Tq, G):
    sees, _ = ob.tree_visible(random_tree(Tq, Tq, dead=(Tq // 2,)))
    _attn(Hq, Hkv, d, Tq, G, 2, 100, 32, "e4m3", 160, sees=sees, what="tree")
    rng = np.random.default_rng(161)
    sees = rng.random((Tq, Tq)) < 0.4
    sees[1] = False
    _attn(Hq, Hkv, d, Tq, G, 2, 100, 64, "int8", 162, sees=sees, bf16_out=True, what="any mask")
    # rows that see nothing at all
    _attn(Hq, Hkv, d, Tq, 0, 1, 64, 64, "int8", 163, sees=sees, rows=[0], what="empty rows")


@pytest.mark.parametrize("Tq,G", [(12, 45), (40, 0), (5, 64)])
def test_unseen_rows_that_are_not_finite(Tq, G):
    # the drafts that nobody sees, or only some, hold NaN and infinities
    Hq, Hkv, d, n, S, block = 8, 2, 64, 1, 40, 16
    q, kg, vg = normal(170, (Tq, Hq, d)), *(normal(s, (G + Tq, Hkv, d)) for s in (171, 172))
    k, v = (spread(s, (n, S, Hkv, d)) for s in (173, 174))
    sees = np.tri(Tq, dtype=bool)
    sees[:, 2] = False
    clean = kg.copy(), vg.copy()
    for row, bits in ((2, 0x7fc0), (Tq - 1, 0x7f80), (Tq - 2, 0xff80)):
        kg[G + row], vg[G + row] = bits, bits
    cache, vals = dev_cache(k, v, block, "e4m3")
    args = (to_dev_bf16(q), *cache, block, None, to_dev_bf16(kg), to_dev_bf16(vg), G)
    for mask in (dev_mask(sees), None):
        o, lse = P.phase2_quant(*args, mask=mask)
        see = sees if mask is not None else np.tri(Tq, dtype=bool)
        bad = see[:, [2, Tq - 1, Tq - 2]].any(axis=1)
        ref, keys = reference(q, *vals, None, *clean, G, see, softmax_scale(d))
        good = np.flatnonzero(~bad)
        assert good.size >= 2
        check(o[torch.from_numpy(good).cuda()], lse[:, torch.from_numpy(good).cuda()],
              (ref[0][good], ref[1][:, good], ref[2][good], ref[3]), keys, f"mask {mask is not None}")
        assert np.isnan(host(o)[bad]).all()


def test_blocks_that_are_not_numbers():
    Hq, Hkv, d, Tq, G, n, S, block = 8, 2, 128, 3, 4, 2, 200, 32
    q, kg, vg = normal(180, (Tq, Hq, d)), *(normal(s, (G + Tq, Hkv, d)) for s in (181, 182))
    k, v = (spread(s, (n, S, Hkv, d)) for s in (183, 184))
    v[1, 150, 1, 7] = 0x7f80
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block)
    vals = [oq.values(*oq.quantize(f64(x), block, "e4m3"), block) for x in (k, v)]
    gen = to_dev_bf16(kg), to_dev_bf16(vg), G
    o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block, None, *gen)
    clean = np.nan_to_num(vals[1])
    ref, keys = reference(q, vals[0], clean, None, kg, vg, G, None, softmax_scale(d))
    # a NaN in V leaves the log-sum-exp and the other KV head's outputs as they are
    assert np.isnan(host(o)[:, 4:]).all()
    check(o[:, :4], lse[:4], (ref[0][:, :4], ref[1][:4], ref[2][:, :4], ref[3]), keys, "V, o")
    check(torch.zeros_like(o), lse, (np.zeros_like(ref[0]), ref[1], ref[2], ref[3]), keys, "V, lse")
    k[0, 10, 0, 0] = 0x7fc0
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block)
    o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block, None, *gen)
    assert np.isnan(host(o)).all() and np.isnan(host(lse)[:4]).all()
    check(torch.zeros_like(o), lse[4:], (np.zeros_like(ref[0]), ref[1][4:], ref[2], ref[3]), keys,
          "the other head's lse")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("block", [16, 128])
def test_attention_with_any_scales(block, fmt):
    # scales that are no powers of two, of very different sizes, zero and subnormal ones
    Hq, Hkv, d, Tq, n, S = 8, 2, 64, 5, 2, 333
    rng = np.random.default_rng(190)
    q = normal(191, (Tq, Hq, d))
    blocks = -(-S // block)
    codes = [rng.integers(-100, 101, (n, Hkv, S, d)) if fmt == "int8" else
             oq.nearest(rng.standard_normal((n, Hkv, S, d)) * 60, fmt) for _ in range(2)]
    ks = np.exp(rng.uniform(-9, -4, (n, Hkv, blocks))).astype(np.float32)
    vs = np.exp(rng.uniform(-40, 5, (n, Hkv, blocks))).astype(np.float32)
    ks[0, 0, 0], vs[0, 1, 1], vs[1, 0, 0] = 0.0, 0.0, 1e-40
    o, lse = P.phase2_quant(to_dev_bf16(q), *(dev_codes(c, fmt) for c in codes),
                            torch.from_numpy(ks).cuda(), torch.from_numpy(vs).cuda(), block)
    # (a scale below 2^-100 counts as 2^-100: at most 448 * 2^-100 off, far below the bounds)
    vals = [oq.values(c, s.astype(np.float64), block) for c, s in zip(codes, (ks, vs))]
    ref, keys = reference(q, *vals, None, None, None, 0, None, softmax_scale(d))
    # log2 of a scale is 58 at most and rounded to 2^-23 of it, once more in the exponent
    # (2^-18 in all); 1 / vs and the sums' products by it are each rounded once
    o_ref, lse_ref, size, most = ref
    extra = 2.0 ** -17
    check(o, lse, (o_ref, lse_ref, size + 1e-25, most + extra * 2.0 ** 24 / (d + 4)), keys, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("Hkv,d,Tq,S", [(32, 64, 1, 4096), (32, 128, 24, 1 << 14)])
def test_values_near_the_largest(Hkv, d, Tq, S, fmt):
    # Keys whose weights are 2^7.5 times those of the keys that a wave sees before them (32 or
    # 64 rows each wave of four or eight) and whose values, 2^127 in one channel, times such a
    # weight leave fp32: the log-sum-exp and the other channels stay what they are.
    high = (np.arange(S) // 256 % 2 == 1)
    q, k, v = (np.zeros(x) for x in ((Tq, Hkv, d), (1, S, Hkv, d), (1, S, Hkv, d)))
    q[..., 0] = 1.0
    k[0, high, :, 0] = 1.0
    v[0, high, :, 3] = 2.0 ** 127
    v[0, ~high, :, 5] = 1.0
    q, k, v = (torch.from_numpy(x).to(torch.bfloat16).cuda() for x in (q, k, v))
    o, lse = P.phase2_quant(q, *P.kv_quantize(k, v, 32, DTYPES[fmt]), 32,
                            softmax_scale=7.5 * math.log(2.0))
    total = S / 2 * (1 + 2 ** 7.5)
    # (scores are exact but for the scale and the base change; sums as in tests._blocks.check)
    off = 7.5 * 2.0 ** -22 + (S + 64) * 2.0 ** -23
    assert np.abs(host(lse) - math.log(total)).max() <= off
    o = host(o)
    assert np.abs(o[..., 5] - S / 2 / total).max() <= (2.0 ** -7 + 2 * off) * S / 2 / total
    assert (np.delete(o, [3, 5], axis=-1) == 0).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_scales_of_v_out_of_range(fmt):
    c = _small(310)
    (Kc, Vc, ks, vs), vals = dev_cache(c["k"], c["v"], c["block"], fmt)
    vs[0, 0, 0], vs[1, 0, 1] = math.inf, 2.0 ** 125
    o, lse = P.phase2_quant(to_dev_bf16(c["q"]), Kc, Vc, ks, vs, c["block"], None,
                            to_dev_bf16(c["kg"]), to_dev_bf16(c["vg"]), c["G"])
    ref, keys = reference(c["q"], *vals, None, c["kg"], c["vg"], c["G"], None,
                          softmax_scale(c["d"]))
    half = c["q"].shape[1] // c["k"].shape[2]
    assert np.isnan(host(o)[:, :half]).all()
    check(o[:, half:], lse[half:], (ref[0][:, half:], ref[1][half:], ref[2][:, half:], ref[3]),
          keys, "the other heads")
    zero = np.zeros_like(ref[0])
    check(torch.zeros_like(o), lse, (zero, ref[1], zero, ref[3]), keys, "lse")


@pytest.mark.parametrize("q_scale", [1e-3, 30.0])
def test_attention_of_flat_and_peaked_scores(q_scale):
    _attn(8, 2, 128, 3, 50, 2, 500, 64, "e4m3", 200, q_scale=q_scale, what=f"q times {q_scale}")
    _attn(8, 8, 64, 20, 50, 2, 500, 64, "int8", 201, q_scale=q_scale, what=f"q times {q_scale}")


@pytest.mark.parametrize("rise", [0.4, 2.0, 5.5, 5.6, 8.3, 9.5, 40.0, 95.0, -5.6, -40.0])
@pytest.mark.parametrize("Hq,Hkv,d,Tq,S", [(8, 2, 64, 2, 2500), (4, 1, 128, 12, 1100),
                                           (64, 64, 128, 30, 7100)])
def test_scores_that_rise(Hq, Hkv, d, Tq, S, rise):
    # The score of a wave's next step is `rise` nats (0.4 to 95: weights of 2^0.6 to 2^137)
    # above the one before, of a few of its keys or of all of them
    rng = np.random.default_rng(220)
    q = normal(221, (Tq, Hq, d), 0.01)
    k, v = f64(normal(222, (1, S, Hkv, d), 0.01)), normal(223, (1, S, Hkv, d))
    q[..., 0] = 0x3f80
    some = rng.random(S) < (0.2 if Tq == 2 else 1.0)
    k[0, :, :, 0] = np.where(some, np.arange(S) // 256, 0)[:, None]
    k = torch.from_numpy(k).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    q[1:, :, 0] = 0x3f00  # (half as steep for the other tokens)
    if rise < 0:
        q[..., 0] |= 0x8000
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), 32, torch.int8)
    o, lse = P.phase2_quant(to_dev_bf16(q), *cache, 32, softmax_scale=abs(rise))
    ref, keys = long_reference(q, cache, 32, None, None, None, 0, None, abs(rise))
    check(o, lse, ref, keys, f"rising by {rise}")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_queries_with_outliers(d, fmt):
    # channels of one query that differ by up to 2^30, columns that differ by up to 2^60 and
    # one that is zero; the keys' large channels are small where the queries' are large
    Hq, Hkv, Tq, n, S, block = 8, 2, 5, 2, 300, 32
    rng = np.random.default_rng(205)
    size = 2.0 ** rng.integers(-30, 1, (Tq, Hq, d))
    size *= 2.0 ** -(np.arange(Tq * Hq).reshape(Tq, Hq, 1) % 60)
    x = f64(normal(206, (Tq, Hq, d))) * size
    x[2, 3] = 0
    q = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    k, v = (spread(s, (n, S, Hkv, d)) for s in (207, 208))
    k[:, :, :, ::7] = 0
    cache, vals = dev_cache(k, v, block, fmt)
    for scale in (1.0, 2.0 ** 20):
        o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block, softmax_scale=scale)
        ref, keys = reference(q, *vals, None, None, None, 0, None, scale)
        check(o, lse, ref, keys, f"outliers, scale {scale}")


@pytest.mark.parametrize("fmt", FMTS)
def test_queries_that_are_not_finite(fmt):
    Hq, Hkv, d, Tq, S, block = 8, 2, 64, 3, 200, 32
    q = normal(209, (Tq, Hq, d))
    good = f64(q).copy()
    q[0, 1, 5], q[1, 6, 63], q[2, 0, 0] = 0x7fc0, 0x7f80, 0xff80
    k, v = (spread(s, (1, S, Hkv, d)) for s in (215, 216))
    cache, vals = dev_cache(k, v, block, fmt)
    o, lse = P.phase2_quant(to_dev_bf16(q), *cache, block)
    bad = np.zeros((Tq, Hq), dtype=bool)
    bad[0, 1] = bad[1, 6] = bad[2, 0] = True
    assert np.isnan(host(o)[bad]).all() and np.isnan(host(lse).T[bad]).all()
    assert np.isfinite(host(o)[~bad]).all() and np.isfinite(host(lse).T[~bad]).all()
    ref, keys = ob.counted_attention(good, vals[0][0], vals[1][0], np.ones((Tq, 1, S)),
                                     softmax_scale(d)), S
    keep = torch.from_numpy(~bad).cuda()
    check(torch.where(keep[..., None], o, 0), torch.where(keep.t(), lse, 0),
          (np.where(bad[..., None], 0, ref[0]), np.where(bad.T, 0, ref[1]), ref[2], ref[3]), keys,
          "the other columns")


def test_attention_scale_and_refusals():
    q = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    kg = torch.zeros((5, 2, 64), dtype=torch.bfloat16, device="cuda")
    c = torch.zeros((3, 2, 40, 64), dtype=torch.int8, device="cuda")
    s = torch.ones((3, 2, 3), device="cuda")
    mask = dev_mask(np.tri(2))
    rows = dev_i32([1, 2, 3])
    P.phase2_quant(q, c, c, s, s, 16, rows, kg, kg, 3, mask)
    wrong = [
        lambda: P.phase2_quant(q.float(), c, c, s, s, 16), lambda: P.phase2_quant(q, c, c, s, s, 32),
        lambda: P.phase2_quant(q, c, c[:2], s, s, 16), lambda: P.phase2_quant(q, c, c, s, s[:2], 16),
        lambda: P.phase2_quant(q, c, c.view(torch.uint8), s, s, 16),
        lambda: P.phase2_quant(q[..., :32].contiguous(), c, c, s, s, 16),
        lambda: P.phase2_quant(q, c, c, s, s, 16, rows[:2]), lambda: P.phase2_quant(q, c, c, s, s, 16, rows.long()),
        lambda: P.phase2_quant(q, c, c, s, s, 16, rows.cpu()),
        lambda: P.phase2_quant(q, c, c, s, s, 16, None, kg), lambda: P.phase2_quant(q, c, c, s, s, 16, None, kg, kg, 2),
        lambda: P.phase2_quant(q, c, c, s, s, 16, None, kg, kg, 3, mask[:, :0]),
        lambda: P.phase2_quant(q, c, c, s, s, 16, mask=mask), lambda: P.phase2_quant(q, c, c, s, s, 16, G=1 << 64),
        lambda: P.phase2_quant(q, c, c, s, s, (1 << 32) + 16), lambda: P.phase2_quant(q, c, c, s, s, 16, o_dtype=5),
        lambda: P.phase2_quant(q, c.float(), c.float(), s, s, 16),
    ]
    for i, fn in enumerate(wrong):
        with pytest.raises(ValueError):
            fn()
            pytest.fail(f"call {i} was not refused")
    for fn in (lambda: P.phase2_quant(q[:, :7].contiguous(), c, c, s, s, 16),
               lambda: P.phase2_quant(q, c, c, s, s, 16, softmax_scale=0.0),
               lambda: P.phase2_quant(q, c, c, s, s, 16, softmax_scale=math.nan)):
        with pytest.raises(RuntimeError):
            fn()
    # no tokens, no shards, no keys
    o, lse = P.phase2_quant(q[:0], c, c, s, s, 16)
    assert o.shape == (0, 8, 64) and lse.shape == (8, 0)
    o, lse = P.phase2_quant(q, c[:0], c[:0], s[:0], s[:0], 16)
    assert (o == 0).all() and torch.isneginf(lse).all()
    o, lse = P.phase2_quant(q, c, c, s, s, 16, dev_i32([0, 0, 0]))
    assert (o == 0).all() and torch.isneginf(lse).all()


# ---- a run of them, streams, graphs, workspaces, far offsets -----------------------


def test_a_generation_with_closing_blocks():
    # after the prefill the shards are quantised; each step attends to them and to the
    # generation shard, whose closed blocks move into a growing shard of the cache
    Hq, Hkv, d, block, S = 8, 2, 64, 16, 100
    k, v = (spread(s, (1, S, Hkv, d)) for s in (210, 211))
    cache = P.kv_quantize(to_dev_bf16(k), to_dev_bf16(v), block, torch.int8)
    grown = P.kv_quantize(to_dev_bf16(k[:, :0]), to_dev_bf16(v[:, :0]), block, torch.int8, 64)
    live = torch.zeros(1, dtype=torch.int32, device="cuda")
    gk, gv = (normal(s, (60, Hkv, d)) for s in (212, 213))
    Kg, Vg = to_dev_bf16(gk), to_dev_bf16(gv)
    vals = [oq.values(*oq.quantize(f64(x), block, "int8"), block) for x in (k, v)]
    moved = 0
    for step in range(50):
        q = normal(220 + step, (1, Hq, d))
        x = to_dev_bf16(q)
        a = P.phase2_quant(x, *cache, block, None, o_dtype=P.OUT_F32)
        b = P.phase2_quant(x, *grown, block, live, Kg[moved:step + 1], Vg[moved:step + 1],
                           step - moved)
        o, lse = P.lse_merge(torch.stack([a[0], b[0]]), torch.stack([a[1], b[1]]))
        closed = [oq.values(*oq.quantize(f64(y[None, :moved]), block, "int8"), block)
                  for y in (gk, gv)]
        K, V = (np.concatenate([x, y], axis=1) for x, y in zip(vals, closed))
        ref, keys = reference(q, K, V, None, gk[moved:step + 1], gv[moved:step + 1], step - moved,
                              None, softmax_scale(d))
        check(o, lse, ref, keys, f"step {step}")
        if step + 1 - moved == block:
            P.kv_quantize_(Kg[None, moved:step + 1], Vg[None, moved:step + 1], *grown, block, moved)
            moved += block
            live.fill_(moved)


def _small(seed, Tq=2, G=20, rows=None):
    Hq, Hkv, d, n, S, block = 8, 2, 64, 3, 260, 32
    q, kg, vg = normal(seed, (Tq, Hq, d)), *(normal(seed + i, (G + Tq, Hkv, d)) for i in (1, 2))
    k, v = (spread(seed + i, (n, S, Hkv, d)) for i in (3, 4))
    return dict(q=q, k=k, v=v, kg=kg, vg=vg, G=G, block=block, S=S, n=n, d=d)


def test_captured_write_and_step_replayed():
    # one graph: rows written into the cache, then attention over its live rows, whose
    # number grows on the device between the replays
    c = _small(240)
    K, V = to_dev_bf16(c["k"]), to_dev_bf16(c["v"])
    cache = P.kv_quantize(K, V, c["block"])
    q, kg, vg = (to_dev_bf16(c[x]) for x in ("q", "kg", "vg"))
    rows = dev_i32([64, 64, 64])
    src = K[:, :32].clone(), V[:, :32].clone()
    ws = torch.zeros(P.phase2_quant_workspace_bytes(2, 8, 2, 64), dtype=torch.uint8, device="cuda")

    def step():
        P.kv_quantize_(*src, *cache, c["block"], 32)
        return P.phase2_quant(q, *cache, c["block"], rows, kg, vg, c["G"], workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        new = [spread(250 + 2 * i + j, (3, 32, 2, 64)) for j in range(2)]
        live = np.array([64, 64, 64]) + [i, 50 * i, -20 * i]
        for s, x in zip(src, new):
            s.copy_(to_dev_bf16(x))
        rows.copy_(dev_i32(live))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        ws.fill_(0xff)
        k, v = c["k"].copy(), c["v"].copy()
        k[:, 32:64], v[:, 32:64] = new
        vals = [oq.values(*oq.quantize(f64(x), 32, "e4m3"), 32) for x in (k, v)]
        ref, keys = reference(c["q"], *vals, live, c["kg"], c["vg"], c["G"], None,
                              softmax_scale(c["d"]))
        check(*got, ref, keys, f"replay {i}")
        eager = step()
        assert all(torch.equal(a, b) for a, b in zip(eager, got)), i


def test_two_graphs_share_a_workspace():
    cases = [_small(260), _small(270, Tq=5, G=3)]
    ws = torch.zeros(P.phase2_quant_workspace_bytes(5, 8, 2, 64), dtype=torch.uint8, device="cuda")
    graphs, refs = [], []
    for c in cases:
        cache, vals = dev_cache(c["k"], c["v"], c["block"], "int8")
        args = (to_dev_bf16(c["q"]), *cache, c["block"], None, to_dev_bf16(c["kg"]),
                to_dev_bf16(c["vg"]), c["G"])
        P.phase2_quant(*args, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = P.phase2_quant(*args, workspace=ws)
        graphs.append((g, out, args))
        refs.append(reference(c["q"], *vals, None, c["kg"], c["vg"], c["G"], None,
                              softmax_scale(64)))
    for turn in range(3):
        for (g, out, _), (ref, keys) in zip(graphs, refs):
            for x in out:
                x.fill_(math.nan)
            g.replay()
            torch.cuda.synchronize()
            check(*out, ref, keys, f"turn {turn}")


def test_other_streams():
    c = _small(280)
    cache, vals = dev_cache(c["k"], c["v"], c["block"], "e4m3")
    args = (to_dev_bf16(c["q"]), *cache, c["block"], None, to_dev_bf16(c["kg"]),
            to_dev_bf16(c["vg"]), c["G"])
    ref, keys = reference(c["q"], *vals, None, c["kg"], c["vg"], c["G"], None, softmax_scale(64))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            made = P.kv_quantize(to_dev_bf16(c["k"]), to_dev_bf16(c["v"]), c["block"])
            outs.append((P.phase2_quant(*args), P.phase2_quant(args[0], *made, *args[5:])))
    torch.cuda.synchronize()
    for pair in outs:
        for o, lse in pair:
            check(o, lse, ref, keys, "on another stream")


def test_past_two_gib():
    # the second shard of a cache lies behind the 32-bit offsets of its codes
    Hq, Hkv, d, Tq, S, block = 4, 1, 128, 2, (1 << 24) + 80, 64
    q, few = normal(290, (Tq, Hq, d)), 150
    k, v = (spread(s, (1, few, Hkv, d)) for s in (291, 292))
    shape = (2, Hkv, S, d)
    codes = [torch.zeros(shape, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    scales = [torch.ones((2, Hkv, -(-S // block)), device="cuda") for _ in range(2)]
    # the first rows of both shards, and the last whole blocks of the second
    first = S // block * block - 128
    P.kv_quantize_(*(torch.zeros((2, few, Hkv, d), dtype=torch.bfloat16, device="cuda")
                     for _ in range(2)), *codes, *scales, block)
    part = [x[1:] for x in codes], [x[1:] for x in scales]
    P.kv_quantize_(to_dev_bf16(k), to_dev_bf16(v), *part[0], *part[1], block)
    P.kv_quantize_(to_dev_bf16(k[:, :128]), to_dev_bf16(v[:, :128]), *part[0], *part[1], block,
                   first)
    vals = [oq.values(*oq.quantize(f64(x), block, "e4m3"), block) for x in (k, v)]
    back = P.kv_dequantize(*codes, *scales, block, first + 3, 100)
    for x, want in zip(back, vals):
        assert (x[0] == 0).all() and np.array_equal(host(x[1]), want[0, 3:103])
    o, lse = P.phase2_quant(to_dev_bf16(q), *codes, *scales, block, dev_i32([0, few]))
    ref, keys = reference(q, *vals, None, None, None, 0, None, softmax_scale(d))
    check(o, lse, ref, keys, "second shard")


@pytest.mark.parametrize("Tq", [1, 12])
def test_results_repeat(Tq):
    c = _small(300, Tq=Tq)
    cache, _ = dev_cache(c["k"], c["v"], c["block"], "int8")
    args = (to_dev_bf16(c["q"]), *cache, c["block"], None, to_dev_bf16(c["kg"]),
            to_dev_bf16(c["vg"]), c["G"])
    first = P.phase2_quant(*args)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, P.phase2_quant(*args)))
