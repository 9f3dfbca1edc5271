"""Phase 2 of drafts and of selected blocks, row by row: every kernel and plan that the
sizes choose counts each row of K and V as often as it is seen.

Row codes: all queries are 0, so that all scores are and every weight is 1 exactly, in
bf16 as well; row r holds a 1 in one channel of V and zeros elsewhere.  An output times
the number of keys is then the number of rows of each channel, and a row that is
dropped, doubled or taken from its neighbour moves it by a whole 1 or more.  Rounding
moves it less: sums of ones are exact (equal weights other than 1 would put keys 2^-24
of them off); the logarithms of partials (up to 10) and the exponentials that the merge
takes of their differences are off by 2.5e-6, numerator and denominator; the merge's sums
over up to 256 parts by 256 2^-24 and the division by two roundings: 2^-14 in all covers
these, and `_check_codes` asserts that the whole is below a quarter of one row's share.
"""
import math

import numpy as np
import pytest
import torch

import paper_2607_20457_amd as P
from oracle import blocks as ob
from tests._blocks import check, dev_i32, dev_mask, random_tree

pytestmark = pytest.mark.gpu

BF = {"dtype": torch.bfloat16, "device": "cuda"}


def _codes(rows, Hkv, d, first=0):
    """int64 [rows, Hkv]: the channel in which each row holds its 1."""
    r = torch.arange(first, first + rows, device="cuda")
    return (r[:, None] * 17 + torch.arange(Hkv, device="cuda") * 5 + r[:, None] // d) % d


def _coded(codes, d):
    return torch.zeros(codes.shape + (d,), **BF).scatter_(-1, codes[..., None], 1.0)


def _check_codes(o, lse, counts, codes, Hq, d, what):
    """counts float64 [Tq, Hkv, n], how often each key is seen; codes [n, Hkv]."""
    Tq, Hkv, n = counts.shape
    total = counts.sum(-1)                                     # [Tq, Hkv]
    want = torch.zeros((Tq, Hkv, d), dtype=torch.float64, device="cuda")
    want.scatter_add_(2, codes.T[None].expand(Tq, Hkv, n).contiguous(), counts)
    most = float(total.max())
    off = 2.0 ** -14 + most * 2.0 ** -24
    assert off * float(want.max()) < 0.25, f"{what}: the bound hides a row"
    got = o.double().view(Tq, Hkv, Hq // Hkv, d) * total[:, :, None, None]
    bad = (got - want[:, :, None]).abs() > off * want[:, :, None]
    assert not bad.any(), f"{what}: rows miscounted, first at {bad.nonzero()[0].tolist()}"
    lse = lse.double().T.reshape(Tq, Hkv, Hq // Hkv)
    ref = total.log()[:, :, None].expand_as(lse)
    assert torch.equal(torch.isneginf(lse), torch.isneginf(ref)), what
    seen = ~torch.isneginf(ref)
    bound = (most + 64) * 2.0 ** -23 + 2.0 ** -22 * ref[seen].abs()
    assert ((lse[seen] - ref[seen]).abs() <= bound).all(), f"{what}: lse"


def _gen_counts(Tq, Hkv, G, sees):
    gen = np.ones((Tq, G + Tq))
    gen[:, G:] = np.tri(Tq) if sees is None else sees
    return torch.from_numpy(gen).cuda()[:, None].expand(Tq, Hkv, G + Tq)


def _sparse(Hq, Hkv, d, Tq, G, ns, S, block, sel, what, sees=None, gen=True):
    topk = sel.shape[3]
    print(f"phase2_sparse rows: {what} Hq={Hq} Hkv={Hkv} d={d} Tq={Tq} G={G} {ns}x{S} "
          f"block={block} topk={topk}", flush=True)
    codes = _codes(ns * S, Hkv, d)
    V = _coded(codes, d).view(ns, S, Hkv, d)
    counts = torch.zeros((Tq, Hkv, ns * S), dtype=torch.float64, device="cuda")
    blocks = -(-S // block)
    listed = dev_i32(sel).long().permute(1, 2, 0, 3)           # [Tq, Hkv, ns, topk]
    at = (listed[..., None] * block + torch.arange(block, device="cuda"))
    ok = ((listed >= 0) & (listed < blocks))[..., None] & (at < S)
    at = torch.where(ok, at, 0) + torch.arange(ns, device="cuda")[:, None, None] * S
    counts.scatter_add_(2, at.reshape(Tq, Hkv, -1), ok.double().reshape(Tq, Hkv, -1))
    kg = vg = None
    if gen:
        gcodes = _codes(G + Tq, Hkv, d, ns * S)
        kg, vg = torch.zeros((G + Tq, Hkv, d), **BF), _coded(gcodes, d)
        codes = torch.cat([codes, gcodes])
        counts = torch.cat([counts, _gen_counts(Tq, Hkv, G, sees)], dim=2)
    o, lse = P.phase2_sparse(torch.zeros((Tq, Hq, d), **BF), torch.ones_like(V), V, dev_i32(sel),
                             block, kg, vg, G, None if sees is None else dev_mask(sees))
    _check_codes(o, lse, counts, codes, Hq, d, what)


def _lists(rng, ns, Tq, Hkv, blocks, topk):
    u = rng.random((ns, Tq, Hkv, blocks))
    return np.argsort(u, axis=3)[..., :topk]


LISTED = [  # Hq, Hkv, d, Tq, G, ns, S, block, topk
    (32, 8, 128, 1, 45, 4, 1021, 16, 8),     # eight waves, one part
    (32, 8, 128, 2, 45, 3, 4099, 16, 30),    # four waves in as many parts as pay
    (32, 8, 128, 2, 45, 3, 4099, 16, 100),   # eight waves in sixteen parts
    (32, 8, 128, 12, 30, 2, 1333, 16, 60),   # eight waves in two parts
    (8, 2, 128, 50, 30, 1, 2777, 32, 70),    # eight waves, two parts
    (32, 8, 128, 66, 7, 1, 700, 32, 5),      # four waves, one part each
    (16, 16, 64, 1, 33, 5, 501, 32, 4),      # the same at d 64
    (16, 16, 64, 2, 33, 5, 3001, 32, 9),
    (16, 16, 64, 5, 33, 5, 3001, 32, 30),
    (16, 16, 64, 16, 300, 5, 1301, 32, 12),  # eight waves, one part
    (4, 2, 64, 120, 20, 3, 2222, 16, 90),
    (16, 16, 64, 66, 20, 2, 300, 16, 6),
    (24, 1, 64, 9, 5, 1, 1500, 16, 60),      # two column tiles
    (40, 1, 128, 3, 5, 2, 2000, 64, 20),     # three
]


@pytest.mark.parametrize("Hq,Hkv,d,Tq,G,ns,S,block,topk", LISTED)
def test_rows_of_lists(Hq, Hkv, d, Tq, G, ns, S, block, topk):
    rng = np.random.default_rng(Tq + S)
    blocks = -(-S // block)
    sel = _lists(rng, ns, Tq, Hkv, blocks, topk)
    sel[:, 0, :, 0] = blocks - 1  # the ragged end is among them (twice, it may be)
    _sparse(Hq, Hkv, d, Tq, G, ns, S, block, sel, "lists")
    sees, _ = ob.tree_visible(random_tree(S, Tq, dead=(Tq - 1,)))
    _sparse(Hq, Hkv, d, Tq, G, ns, S, block, sel, "lists and a tree", sees=sees)
    sel[rng.random(sel.shape) < 0.2] = -1
    _sparse(Hq, Hkv, d, Tq, 0, ns, S, block, sel, "gaps, shards alone", gen=False)


TOGETHER = [  # Hq, Hkv, d, Tq, ns, S, block, topk: from 320 MB of listed keys, or 800
    (32, 8, 128, 131, 2, 3001, 32, 42),    # two groups of 16 columns
    (12, 4, 128, 266, 1, 5555, 64, 44),    # eight tokens of three heads
    (32, 8, 128, 67, 2, 3001, 32, 38),     # one group
    (8, 8, 128, 67, 2, 3001, 32, 38),      # eight tokens in eight columns
    (16, 2, 128, 258, 1, 5100, 64, 60),    # eight heads, two groups
    (16, 16, 64, 67, 3, 2003, 16, 60),     # d 64
    (4, 2, 64, 259, 2, 4003, 128, 19),
]


@pytest.mark.parametrize("Hq,Hkv,d,Tq,ns,S,block,topk", TOGETHER)
def test_rows_of_tokens_read_together(Hq, Hkv, d, Tq, ns, S, block, topk):
    rng = np.random.default_rng(Tq + S)
    blocks, G = -(-S // block), 37
    own = _lists(rng, ns, Tq, Hkv, blocks, topk)               # of each token
    same = np.broadcast_to(own[:, :1], own.shape).copy()       # of all
    same[..., 0] = blocks - 1
    some = same.copy()                                         # half their own
    some[..., topk // 2:] = own[..., topk // 2:]
    _sparse(Hq, Hkv, d, Tq, G, ns, S, block, own, "lists of their own")
    _sparse(Hq, Hkv, d, Tq, G, ns, S, block, some, "half shared, some twice")
    _sparse(Hq, Hkv, d, Tq, 0, ns, S, block, same, "shared, shards alone", gen=False)
    sees, _ = ob.tree_visible(random_tree(S, Tq, dead=(Tq - 1,)))
    _sparse(Hq, Hkv, d, Tq, G, ns, S, block, np.sort(own, axis=3), "a tree", sees=sees)


TREES = [  # Hq, Hkv, d, Tq, G, ns, S
    (32, 8, 128, 1, 9, 4, 1021),      # 16-row tiles: one token
    (32, 8, 128, 12, 45, 4, 1021),    # three tiles, eight waves
    (32, 8, 128, 64, 45, 4, 1021),
    (8, 2, 128, 48, 33, 8, 2049),
    (32, 8, 128, 4, 700, 2, 4000),    # one tile over many keys, four waves
    (16, 16, 64, 16, 5, 3, 1999),     # d 64
    (12, 1, 128, 5, 300, 3, 999),     # 12 heads: one token a tile
    (16, 16, 64, 20, 45, 3, 5001),    # decode kernel
    (16, 16, 64, 40, 10, 3, 4101),    # packed kernel, appended rows in ranges of their own
    (16, 16, 64, 40, 300, 20, 621),   # packed kernel, appended rows join
    (16, 4, 64, 100, 300, 2, 3001),   # attention kernel, appended rows in 16-row tiles
    (16, 4, 64, 100, 5000, 1, 501),   # attention kernel for both
    (16, 8, 64, 200, 3000, 1, 501),   # appended rows in the decode kernel
    (32, 8, 128, 20, 64, 3, 6001),    # d 128
    (32, 8, 128, 70, 777, 6, 2049),   # attention kernel, appended rows in 16-row tiles
    (32, 8, 128, 7, 700, 0, 0),       # appended rows alone
]


@pytest.mark.parametrize("Hq,Hkv,d,Tq,G,ns,S", TREES)
def test_rows_of_drafts(Hq, Hkv, d, Tq, G, ns, S):
    print(f"phase2_tree rows: Hq={Hq} Hkv={Hkv} d={d} Tq={Tq} G={G} {ns}x{S}", flush=True)
    codes = _codes(ns * S + G + Tq, Hkv, d)
    sees, _ = ob.tree_visible(random_tree(S + G, Tq, dead=(Tq - 1,) if Tq > 1 else ()))
    vg = _coded(codes[ns * S:], d)
    V = _coded(codes[:ns * S], d).view(ns, S, Hkv, d) if ns else None
    o, lse = P.phase2_tree(torch.zeros((Tq, Hq, d), **BF), torch.ones_like(vg), vg, G,
                           dev_mask(sees), None if V is None else torch.ones_like(V), V)
    counts = torch.ones((Tq, Hkv, ns * S), dtype=torch.float64, device="cuda")
    counts = torch.cat([counts, _gen_counts(Tq, Hkv, G, sees)], dim=2)
    _check_codes(o, lse, counts, codes, Hq, d, "drafts")


def _device_reference(q, K, V, sel, block, scale):
    """oracle.blocks.counted_attention of listed blocks, in float64 on the device."""
    Tq, Hq, d = q.shape
    ns, S, Hkv, _ = K.shape
    group = Hq // Hkv
    o, size = (torch.zeros((Tq, Hq, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((Hq, Tq), -math.inf, dtype=torch.float64, device="cuda")
    most = 0.0
    for t in range(Tq):
        for g in range(Hkv):
            at = sel[:, t, g].long()[..., None] * block + torch.arange(block, device="cuda")
            at = (at + torch.arange(ns, device="cuda")[:, None, None] * S)[at < S]
            k, v = (x.view(ns * S, Hkv, d)[at, g].double() for x in (K, V))
            qt = q[t, g * group:(g + 1) * group].double()
            s = (qt @ k.T) * scale
            most = max(most, float((qt.abs() @ k.abs().T).max()) * scale)
            lse[g * group:(g + 1) * group, t] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            o[t, g * group:(g + 1) * group] = p @ v
            size[t, g * group:(g + 1) * group] = p @ v.abs()
    return o.cpu().numpy(), lse.cpu().numpy(), size.cpu().numpy(), most


@pytest.mark.parametrize("Hq,Hkv,d,Tq,ns,blocks,topk,what", [
    # more than 256 tokens and 320 MB: read together up to the union's map and list in LDS
    (2, 1, 128, 257, 1, 65536, 160, "a full map"),
    (2, 1, 128, 257, 1, 65537, 160, "a block too many for the map"),
    (2, 1, 128, 257, 2, 32769, 80, "two too many, of two shards"),
    (2, 1, 128, 260, 1, 5000, 448, "a full list"),
    (2, 1, 128, 260, 1, 5000, 449, "too long a list"),
    (2, 1, 128, 260, 1, 3584, 1000, "a list of every block"),
    (4, 1, 64, 600, 1, 32768, 448, "d 64: a full map and list"),
    (4, 1, 64, 600, 1, 32769, 448, "d 64: too many blocks"),
    (4, 1, 64, 600, 1, 6000, 449, "d 64: too long a list"),
])
def test_limits_of_tokens_read_together(Hq, Hkv, d, Tq, ns, blocks, topk, what):
    block = 16
    S = blocks * block - 3
    print(f"limits: {what} Hq={Hq} Hkv={Hkv} d={d} Tq={Tq} {ns}x{S} topk={topk}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(blocks + topk)
    q, K, V = (torch.randn(s, generator=gen, **BF) for s in
               ((Tq, Hq, d), (ns, S, Hkv, d), (ns, S, Hkv, d)))
    # tokens of a tile that share nothing: as many blocks as their lists can hold
    u = torch.rand((ns, Tq, Hkv, blocks), generator=gen, device="cuda")
    if topk * 8 <= blocks:
        u += (torch.arange(blocks, device="cuda") % 8
              == torch.arange(Tq, device="cuda")[:, None, None] % 8)
    sel = torch.topk(u, topk, dim=3).indices.sort(dim=3).values.to(torch.int32)
    sel[:, (blocks - 1) % 8, :, -1] = blocks - 1  # the ragged one
    o, lse = P.phase2_sparse(q, K, V, sel, block)
    check(o, lse, _device_reference(q, K, V, sel, block, 1 / math.sqrt(d)), ns * topk * block, what)
    again = P.phase2_sparse(q, K, V, sel, block)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("Hq,Hkv,d,Tq,ns,blocks,topk", [
    (32, 8, 128, 12, 2, 90, 60),   # eight waves in several parts
    (8, 2, 128, 50, 1, 150, 130),
    (32, 8, 128, 15, 1, 300, 150),
    (16, 16, 64, 5, 4, 100, 25),   # d 64
    (4, 2, 64, 60, 3, 140, 90),
])
def test_eight_waves_in_several_parts(Hq, Hkv, d, Tq, ns, blocks, topk):
    block = 16
    S = blocks * block - 5
    need = P.api._lib.lib().pulsar_phase2_sparse_call_bytes(ns, Tq, S, block, topk, 0, Hq, Hkv, d)
    assert need > Tq * Hq * (d + 1) * 4  # several parts
    gen = torch.Generator(device="cuda").manual_seed(blocks + topk)
    q, K, V = (torch.randn(s, generator=gen, **BF) for s in
               ((Tq, Hq, d), (ns, S, Hkv, d), (ns, S, Hkv, d)))
    u = torch.rand((ns, Tq, Hkv, blocks), generator=gen, device="cuda")
    sel = torch.topk(u, topk, dim=3).indices.to(torch.int32)
    o, lse = P.phase2_sparse(q, K, V, sel, block)
    ref = _device_reference(q, K, V, sel, block, 1 / math.sqrt(d))
    check(o, lse, ref, ns * topk * block, "eight waves")


@pytest.mark.parametrize("Hq,Hkv,d,Tq,ns,S,block,topk", [
    (32, 8, 128, 100, 2, 1600, 32, 48),   # two groups of 16 columns: eight tokens of four heads
    (12, 4, 128, 203, 1, 3301, 64, 50),   # eight of three heads
    (16, 2, 128, 301, 1, 5100, 64, 66),   # four of eight heads
    (20, 4, 128, 202, 1, 4800, 64, 50),   # six of five heads, four in the last
])
def test_two_groups_of_columns(Hq, Hkv, d, Tq, ns, S, block, topk):
    # scores and values of any size, lists that share half, against 64 bits
    gen = torch.Generator(device="cuda").manual_seed(Tq + S)
    q, K, V = (torch.randn(s, generator=gen, **BF) for s in
               ((Tq, Hq, d), (ns, S, Hkv, d), (ns, S, Hkv, d)))
    assert Tq * Hkv * ns * topk * block * d * 4 >= 1200000000  # from here on two groups
    u = torch.rand((ns, Tq, Hkv, -(-S // block)), generator=gen, device="cuda")
    u += torch.rand((ns, 1, Hkv, -(-S // block)), generator=gen, device="cuda")
    sel = torch.topk(u, topk, dim=3).indices.to(torch.int32)
    for x in (q, q * 4):
        o, lse = P.phase2_sparse(x, K, V, sel, block, o_dtype=P.OUT_BF16)
        ref = _device_reference(x, K, V, sel, block, 1 / math.sqrt(d))
        check(o, lse, ref, ns * topk * block, "two groups", bf16_out=True)
