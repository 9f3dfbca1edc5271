"""phase2_quant at its edges, in every shape of tile: scales, values and scores of extreme
size, what is not finite, and what must not be seen."""
import math

import numpy as np
import pytest
import torch

import paper_2607_20457_amd as P
from tests import _blocks
from tests._blocks import dev_i32, dev_mask, host
from tests._plan import SHAPES, plan
from tests._quant import DTYPES, check, long_reference, softmax_scale

pytestmark = pytest.mark.gpu


# ---- keys whose values are tiny ---------------------------------------------------


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("ordinary", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,Tq,S,shape", [
    (64, 64, 64, 1, 131072, (16, 32)), (64, 64, 128, 1, 65536, (16, 32)),
    (64, 64, 128, 40, 65536, (48, 32)), (64, 64, 128, 30, 65536, (32, 32)),
    (64, 64, 128, 64, 65536, (32, 64)), (64, 64, 64, 64, 65536, (32, 32)),
])
def test_low_scores_in_blocks_of_the_least_scale(Hq, Hkv, d, Tq, S, shape, ordinary, fmt):
    # The first key of each wave's first step has the score 0, all others 2^-26.5 of its weight
    # and the scale 2^-100 that blocks of zeros have: together they are a share `tail` of the
    # sum.  (The first keys' blocks have the scale 1 and values 0, or are as the others.)
    p = plan(1, Tq, S, Hq, Hkv, d)
    assert (p.columns, p.keys) == shape
    steps, low = S // p.keys, 2.0 ** -26.5
    first = np.concatenate([i * steps // p.parts + np.arange(p.waves)
                            for i in range(p.parts)]) * p.keys
    assert steps % p.parts == 0
    codes = [torch.zeros((1, Hkv, S, d), dtype=torch.int8, device="cuda") for _ in range(2)]
    codes[0][..., 0] = -1
    codes[1] += 1
    ks, vs = (torch.full((1, Hkv, S // 16), x, device="cuda") for x in (1.0, 2.0 ** -100))
    at = torch.from_numpy(first).cuda()
    codes[0][:, :, at, 0] = 0
    if ordinary:
        rows = (at[:, None] + torch.arange(16, device="cuda")).view(-1)
        codes[1][:, :, rows] = 0
        vs[:, :, at // 16] = 1
    if fmt == "e4m3":
        codes = [x.to(torch.float8_e4m3fn) for x in codes]
    q = torch.zeros((Tq, Hq, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    o, lse = P.phase2_quant(q, *codes, ks, vs, 16, softmax_scale=26.5 * math.log(2))
    tail = (S / first.size - 1) * low
    # Sums are exact but in the lanes of the first keys, a quarter of all: they add 2^-23.5
    # (two halves of a step) or 2^-22.5 (four) at a time to 1, whose steps are 2^-23: off by
    # half of it at most.  Beside it the log-sum-exp is rounded, to 2^-21 of log2 32 and
    # of log 32, in each wave and in the merge.
    want = math.log(first.size) + math.log1p(tail)
    assert np.abs(host(lse) - want).max() <= tail / 8 + 2.0 ** -20
    if ordinary:
        # (weights of a value 2^-100 come to 2^-126 of it, the least normal number)
        assert float(o.abs().max()) <= 2.0 ** -100
    else:
        # low weights times 2^-100 are lost or not
        assert np.abs(host(o) * 2.0 ** 100 - 1).max() <= 2.0 ** -8 + tail


# ---- every shape of tile ------------------------------------------------------------


def _bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _normal(gen, shape, size=1.0):
    return (size * torch.randn(shape, generator=gen, device="cuda")).to(torch.bfloat16)


class Case:
    """Sizes that take one shape of tile, its inputs on the device, and a cache of 32-row
    blocks."""

    def __init__(self, shape, fmt, seed, G=70):
        (self.Hq, self.Hkv, self.d, self.Tq, self.n, self.S), want = SHAPES[shape]
        p = plan(self.n, self.Tq, self.S, self.Hq, self.Hkv, self.d, G + self.Tq)
        assert (p.columns, p.keys) == want
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rows = (self.n, self.S, self.Hkv, self.d)
        self.group, self.G, self.fmt, self.block = self.Hq // self.Hkv, G, fmt, 32
        self.q = _normal(gen, (self.Tq, self.Hq, self.d))
        self.k, self.v = _normal(gen, rows), _normal(gen, rows)
        self.kg, self.vg = (_normal(gen, (G + self.Tq, self.Hkv, self.d)) for _ in range(2))
        self.scale = softmax_scale(self.d)
        print(f"phase2_quant edges: {shape} {fmt} seed {seed} {self.n}x{self.S}", flush=True)

    def quantize(self):
        self.cache = P.kv_quantize(self.k, self.v, self.block, DTYPES[self.fmt])

    def call(self, rows=None, mask=None, **kw):
        return P.phase2_quant(self.q, *self.cache, self.block,
                              None if rows is None else dev_i32(rows), self.kg, self.vg, self.G,
                              mask, softmax_scale=self.scale, **kw)

    def reference(self, rows=None, sees=None, cache=None, **kw):
        x = {**dict(q=self.q, kg=self.kg, vg=self.vg), **kw}
        return long_reference(_bits(x["q"]), cache or self.cache, self.block, rows,
                              _bits(x["kg"]), _bits(x["vg"]), self.G, sees, self.scale)


def _compare(out, ref, keys, bad_o, bad_lse, what, bf16_out=False):
    """`check`, but for what has to be NaN: outputs bad_o [Tq, Hq] and sums bad_lse [Hq, Tq]."""
    o, lse = out
    assert np.array_equal(np.isnan(host(o)), np.broadcast_to(bad_o[..., None], o.shape)), what
    assert np.array_equal(np.isnan(host(lse)), bad_lse), what
    o = torch.where(torch.from_numpy(bad_o).cuda()[..., None], 0, o)
    lse = torch.where(torch.from_numpy(bad_lse).cuda(), 0, lse)
    check(o, lse, (np.where(bad_o[..., None], 0, ref[0]), np.where(bad_lse, 0, ref[1]), ref[2],
                   ref[3]), keys, what, bf16_out)


ALL = pytest.mark.parametrize("shape", list(SHAPES))
FMTS = pytest.mark.parametrize("fmt", ["e4m3", "int8"])


@FMTS
@ALL
@pytest.mark.parametrize("where", ["codes", "generation", "both"])
def test_average_of_values_near_the_largest(shape, fmt, where):
    # The largest bf16 number in some channels of every second block, of all kinds of scores: a
    # few of them leave fp32 in a sum, none in the average.  Other channels, and other blocks,
    # are ordinary.
    c = Case(shape, fmt, 400)
    top = torch.finfo(torch.bfloat16).max
    second = (torch.arange(c.S, device="cuda") // 64 % 2 == 1).nonzero().view(-1)
    if where != "generation":
        c.v[:, second[:, None], :, 3] = top
        c.v[:, second[:, None], 0, 5] = -top
    if where != "codes":
        c.vg[..., 3] = top
        c.vg[::2, :, 7] = -top
    c.quantize()
    for bf16_out in (False, True):
        o, lse = c.call(o_dtype=P.OUT_BF16 if bf16_out else P.OUT_F32)
        assert torch.isfinite(o).all()
        # (the bound goes by the weighted |v| of each channel, so ordinary ones count as such)
        check(o, lse, *c.reference(), where, bf16_out)
    # all keys alike and all values the largest: their average is one of them
    c.q.zero_()
    c.v.fill_(top)
    c.vg.fill_(top)
    c.quantize()
    o, lse = c.call()
    check(o, lse, *c.reference(), "all of them")


@FMTS
@ALL
def test_scales_of_every_kind(shape, fmt):
    # head 0: blocks of V whose scale is none (NaN, infinity, past the largest); the last head:
    # K's too; in all of them scales of V from 2^-90 to 2^110, and blocks of zeros
    c = Case(shape, fmt, 410)
    rng = np.random.default_rng(411)
    blocks = -(-c.S // c.block)
    size = 2.0 ** rng.integers(-90, 111, (c.n, blocks, c.Hkv))
    size[:, ::2] = rng.integers(0, 2, size[:, ::2].shape)
    size = torch.from_numpy(size.repeat(c.block, axis=1)[:, :c.S, :, None]).cuda()
    c.v = (c.v.double() * size).to(torch.bfloat16)
    c.quantize()
    ref, keys = c.reference()
    none = np.zeros((c.Tq, c.Hq), dtype=bool)
    _compare(c.call(), ref, keys, none, none.T, "scales of any size")
    bad = none.copy()
    bad[:, :c.group] = True
    vs = c.cache[3]
    at = blocks // 3
    for x in (math.nan, math.inf, 2.0 ** 125):
        was = vs[0, 0, at].clone()
        vs[0, 0, at] = x
        _compare(c.call(), ref, keys, bad, none.T, f"a scale of {x}")
        vs[0, 0, at] = was
    last = none.copy()
    last[:, -c.group:] = True
    c.cache[2][-1, -1, -1] = math.nan
    _compare(c.call(), ref, keys, last, last.T, "a scale of K that is none")


@FMTS
@ALL
def test_nothing_behind_live_rows_is_seen(shape, fmt):
    # lengths that end inside steps and blocks, of zero and one; codes and scales of anything
    # behind them
    c = Case(shape, fmt, 420, G=7)
    c.quantize()
    for most in (c.S - 5, c.S // 2 + 17, 33, 1, 0):
        rows = np.minimum(c.S - 5, most + 100 * np.arange(c.n))
        ref, keys = c.reference(rows)
        was = [x.clone() for x in c.cache]
        for i, live in enumerate(rows):
            for x, s in ((c.cache[0], c.cache[2]), (c.cache[1], c.cache[3])):
                x.view(torch.uint8)[i, :, live:] = 0x7f
                s[i, :, -(-live // c.block):] = math.nan
        check(*c.call(rows), ref, keys, f"{most} rows")
        c.cache = was


@FMTS
@ALL
def test_unseen_generation_rows_that_are_not_finite(shape, fmt):
    # drafts that hold NaN and infinities reach only those that see them, by a mask and by
    # order; G ends inside a step of 16 or 32 rows
    c = Case(shape, fmt, 430, G=21)
    c.quantize()
    Tq = c.Tq
    sees = np.tri(Tq, dtype=bool)
    odd = {1: math.nan, Tq // 2 + 1: -math.inf, Tq - 1: math.inf}
    for row in odd:
        sees[row + 1:, row] = False
    clean = c.kg.clone(), c.vg.clone()
    for row, x in odd.items():
        c.kg[c.G + row, :, ::5] = x
        c.vg[c.G + row] = x
    for see, mask in ((sees, dev_mask(sees)), (np.tri(Tq, dtype=bool), None)):
        bad = np.repeat(see[:, list(odd)].any(axis=1)[:, None], c.Hq, axis=1)
        assert bad.any() and not bad.all()
        ref, keys = c.reference(None, see, kg=clean[0], vg=clean[1])
        _compare(c.call(None, mask), ref, keys, bad, bad.T, f"mask {mask is not None}")


@FMTS
@ALL
def test_queries_that_are_not_finite_in_every_tile(shape, fmt):
    c = Case(shape, fmt, 440)
    c.quantize()
    bad = np.zeros((c.Tq, c.Hq), dtype=bool)
    ref, keys = c.reference()
    for t, h, ch, x in ((0, c.Hq - 1, 5, math.nan), (c.Tq - 1, 0, c.d - 1, math.inf),
                        (c.Tq // 2, c.Hq // 2, 0, -math.inf)):
        c.q[t, h, ch] = x
        bad[t, h] = True
    _compare(c.call(), ref, keys, bad, bad.T, "queries")


@ALL
@pytest.mark.parametrize("rise", [0.4, 5.6, 8.3, 40.0, 95.0, -5.6, -40.0])
def test_scores_that_rise_in_every_tile(shape, rise):
    # The score of a wave's next step (256 rows on, in all shapes) is `rise` nats above the one
    # before, for the first token twice as steeply
    c = Case(shape, "int8", 450)
    c.q *= 0.01
    c.k *= 0.01
    c.q[..., 0] = math.copysign(0.5, rise)
    c.q[0, :, 0] = math.copysign(1.0, rise)
    some = torch.rand((1, c.S, 1), generator=torch.Generator("cuda").manual_seed(451),
                      device="cuda") < 0.3
    c.k[..., 0] = torch.where(some, torch.arange(c.S, device="cuda")[None, :, None] // 256, 0)
    c.scale = abs(rise)
    c.quantize()
    check(*c.call(), *c.reference(), f"rising by {rise}")


@FMTS
def test_the_last_shard_of_a_cache_grows(fmt):
    # retained shards and one that takes the generation shard's closed blocks, in one cache
    Hq, Hkv, d, n, S, block = 8, 2, 128, 4, 100, 16
    gen = torch.Generator(device="cuda").manual_seed(460)
    k, v, more_k, more_v = (_normal(gen, (m, S, Hkv, d)) for m in (n, n, 1, 1))
    cache = P.kv_quantize(*(torch.cat([x, torch.zeros_like(x[:1])]) for x in (k, v)), block,
                          DTYPES[fmt])
    last = [x[-1:] for x in cache]
    rows = dev_i32([S] * n + [0])
    q = _normal(gen, (1, Hq, d))
    for step in range(0, 2 * block + 3):
        moved = step // block * block
        if step == moved > 0:
            new = slice(moved - block, moved)
            P.kv_quantize_(more_k[:, new], more_v[:, new], *last, block, moved - block)
            rows[-1] = moved
        kg, vg = more_k[0, moved:step + 1], more_v[0, moved:step + 1]
        o, lse = P.phase2_quant(q, *cache, block, rows, kg, vg, step - moved)
        check(o, lse, *long_reference(_bits(q), cache, block, [S] * n + [moved], _bits(kg),
                                      _bits(vg), step - moved, None, softmax_scale(d)),
              f"step {step}")


@FMTS
@ALL
@pytest.mark.parametrize("size", [-60, -105])
def test_values_that_are_all_tiny(shape, fmt, size):
    # The codes' and the generation rows'.  Scores within 2^12 of each other leave weights of
    # 2^-20 and more against any reference that trails by 2^8: products of 2^-125 and more, so
    # that nothing but the weights' rounding is off (tests._blocks.check).
    c = Case(shape, fmt, 470)
    c.v *= 2.0 ** size
    c.vg *= 2.0 ** size
    c.quantize()
    ref, keys = c.reference()
    _blocks.check(*c.call(), ref, keys, "tiny values")
