"""Drafted tokens on the GPU: tree_mask, phase2_tree and kv_compact_ against
oracle.blocks (tolerances: tests._blocks.check)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_20457_amd as P
from oracle import blocks as ob
from tests._blocks import (check, dev_i32, dev_mask, host, normal, random_tree, to_dev_bf16,
                           tree_reference)

pytestmark = pytest.mark.gpu


def _check_mask(parent, what):
    mask, depth = P.tree_mask(dev_i32(parent))
    sees, deep = ob.tree_visible(parent)
    words = mask.cpu().numpy().view(np.uint32)
    assert np.array_equal(words, ob.mask_words(sees)), what
    assert np.array_equal(depth.cpu().numpy(), deep), what


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 100, 257, 600])
def test_tree_mask(T):
    _check_mask(random_tree(T, T), f"random tree of {T}")
    _check_mask(np.arange(T) - 1, f"chain of {T}")
    _check_mask(np.full(T, -1), f"{T} single tokens")


def test_tree_mask_of_what_is_no_tree():
    # parents at or after the token, below -1, far outside: no token, nor any after it
    _check_mask(np.array([-1, 1, 0, 2, -2, 4, 7, 2**31 - 1, -2**31, 3, 9, 10]), "bad parents")
    _check_mask(random_tree(5, 80, dead=(0, 40, 79)), "padded tree")
    mask, depth = P.tree_mask(dev_i32(np.zeros(0)))
    assert mask.shape == (0, 0) and depth.shape == (0,)


def test_tree_mask_of_the_largest_tree():
    T = 16384
    parent = random_tree(3, T)
    mask, depth = P.tree_mask(dev_i32(parent))
    deep = np.zeros(T, dtype=np.int64)
    for t in range(T):
        deep[t] = 0 if parent[t] < 0 else deep[parent[t]] + 1
    assert np.array_equal(depth.cpu().numpy(), deep)
    words = mask.cpu().numpy().view(np.uint32)
    for t in (0, 31, 32, 5000, T - 1):
        seen, j = set(), t
        while j >= 0:
            seen.add(j)
            j = parent[j]
        bits = np.unpackbits(words[t].view(np.uint8), bitorder="little")
        assert set(np.flatnonzero(bits)) == seen


def _tree(Hq, Hkv, d, Tq, G, ns, S, seed, sees=None, bf16_out=False, what="", q_scale=1.0):
    print(f"phase2_tree parity: {what} Hq={Hq} Hkv={Hkv} d={d} Tq={Tq} G={G} {ns}x{S}", flush=True)
    scale = 1.0 / math.sqrt(d)
    q = normal(seed, (Tq, Hq, d), q_scale)
    kg, vg = (normal(seed + i, (G + Tq, Hkv, d)) for i in (1, 2))
    k, v = ((normal(seed + i, (ns, S, Hkv, d)) for i in (3, 4)) if ns else (None, None))
    if sees is None:
        sees, _ = ob.tree_visible(random_tree(seed, Tq))
    o, lse = P.phase2_tree(to_dev_bf16(q), to_dev_bf16(kg), to_dev_bf16(vg), G, dev_mask(sees),
                           to_dev_bf16(k) if ns else None, to_dev_bf16(v) if ns else None,
                           o_dtype=P.OUT_BF16 if bf16_out else P.OUT_F32)
    ref, keys = tree_reference(q, kg, vg, G, sees, k, v, scale)
    check(o, lse, ref, keys, what, bf16_out)


@pytest.mark.parametrize("Hq,Hkv,d,Tq,G,ns,S", [
    (32, 8, 128, 1, 0, 0, 0),        # one draft, nothing before it: no partial at all
    (32, 8, 128, 1, 0, 2, 100),      # one draft over shards alone
    (32, 8, 128, 8, 45, 4, 251),     # 32 packed rows: the decode kernel
    (8, 8, 128, 32, 1, 0, 0),        # one head per KV head, one appended row
    (32, 8, 128, 7, 700, 0, 0),      # appended rows alone, in ranges
    (4, 1, 64, 5, 31, 1, 33),        # one KV head
    (32, 1, 64, 1, 9, 1, 40),        # 32 heads per KV head
    (32, 8, 128, 12, 0, 3, 129),     # packed kernel, no appended rows
    (32, 8, 128, 20, 300, 32, 40),   # packed kernel, a full chip: appended rows join
    (32, 8, 128, 32, 900, 1, 500),   # packed kernel, ranges of their own
    (32, 8, 128, 32, 40, 0, 0),      # packed kernel, appended rows alone
    (16, 16, 64, 50, 7, 2, 127),     # d 64, two tiles
    (16, 4, 64, 44, 10, 2, 640),     # d 64, six tiles
    (32, 8, 128, 33, 0, 2, 300),     # attention kernel, no appended rows
    (32, 8, 128, 64, 70, 2, 513),    # attention kernel, appended rows in the decode kernel
    (8, 8, 64, 200, 33, 1, 90),      # more drafts than a word and a packed launch hold
    (16, 8, 64, 300, 5, 1, 64),      # 600 rows per KV head: appended rows in the attention kernel
    (32, 8, 128, 40, 4200, 1, 256),  # a long generation shard
    (64, 1, 64, 3, 10, 1, 100),      # 64 heads per KV head
    (4, 1, 128, 300, 0, 0, 0),       # drafts alone, more than a list of 256
])
def test_tree_shapes(Hq, Hkv, d, Tq, G, ns, S):
    _tree(Hq, Hkv, d, Tq, G, ns, S, 2000 + Hq + Tq + G, bf16_out=Tq % 2 == 0, what="shapes")


@pytest.mark.parametrize("Hq,Hkv,d,Tq,G,ns,S", [
    # more bytes than 16-row tiles read again: the query step's kernels
    (16, 16, 64, 20, 45, 3, 6000),   # decode kernel
    (16, 16, 64, 40, 10, 3, 4100),   # packed kernel, appended rows in ranges of their own
    (16, 16, 64, 40, 300, 20, 620),  # packed kernel, a full chip: appended rows join
    (16, 16, 64, 40, 12000, 0, 0),   # packed kernel, appended rows alone
    (16, 4, 64, 100, 300, 2, 3000),  # attention kernel, appended rows in 16-row tiles
    (16, 4, 64, 100, 6000, 1, 500),  # attention kernel for both
    (16, 8, 64, 200, 3000, 1, 500),  # attention kernel, appended rows in the decode kernel
    (32, 8, 128, 20, 64, 4, 6000),   # d 128
])
def test_tree_shapes_of_the_query_step(Hq, Hkv, d, Tq, G, ns, S):
    _tree(Hq, Hkv, d, Tq, G, ns, S, 2100 + Hq + Tq + G, bf16_out=Tq % 40 == 0, what="query step")


def test_tree_rows_without_any_key():
    # rows whose mask is empty: over nothing they give 0 and -inf, over shards the shards
    Tq = 40
    sees, _ = ob.tree_visible(random_tree(11, Tq, dead=(0, 17, 39)))
    assert not sees[17].any()
    _tree(8, 2, 128, Tq, 0, 0, 0, 2100, sees=sees, what="empty rows")
    _tree(8, 2, 128, Tq, 0, 1, 50, 2101, sees=sees, what="empty rows over a shard")
    _tree(8, 2, 64, 3, 0, 0, 0, 2102, sees=np.zeros((3, 3), bool), what="all rows empty")


def test_tree_any_visibility():
    # no tree: a token may see later drafts, and not its own row
    rng = np.random.default_rng(12)
    for Tq in (9, 70):
        _tree(8, 2, 128, Tq, 20, 1, 60, 2110 + Tq, sees=rng.random((Tq, Tq)) < 0.4, what="random")


def test_tree_of_a_chain_is_a_query_step():
    Tq, G, Hq, Hkv, d = 20, 33, 32, 8, 128
    q, kg, vg = (to_dev_bf16(normal(s, sh)) for s, sh in (
        (1, (Tq, Hq, d)), (2, (G + Tq, Hkv, d)), (3, (G + Tq, Hkv, d))))
    k, v = (to_dev_bf16(normal(s, (2, 300, Hkv, d))) for s in (4, 5))
    mask, _ = P.tree_mask(dev_i32(np.arange(Tq) - 1))
    o, lse = P.phase2_tree(q, kg, vg, G, mask, k, v)
    o2, lse2 = P.phase2_query(q, kg, vg, G, k, v)
    assert np.allclose(host(lse), host(lse2), atol=1e-4)
    assert np.abs(host(o) - host(o2)).max() <= 2.0 ** -6


def test_tree_peaked():
    _tree(32, 8, 128, 16, 9, 2, 400, 2200, q_scale=8.0, what="peaked")


@pytest.mark.parametrize("Tq", [6, 20, 70])
def test_unseen_drafts_may_hold_anything(Tq):
    # NaN and infinities in the rows of drafts that a token does not see, and of the
    # rows behind the last, leave its output as it is
    G, Hq, Hkv, d = 21, 16, 4, 128
    q = normal(31, (Tq, Hq, d))
    kg, vg = (normal(s, (G + Tq, Hkv, d)) for s in (32, 33))
    k, v = (normal(s, (1, 100, Hkv, d)) for s in (34, 35))
    sees, _ = ob.tree_visible(random_tree(36, Tq))
    bad = np.arange(Tq) % 3 == 1
    sees = sees & ~bad[None, :]
    ref = P.phase2_tree(*map(to_dev_bf16, (q, kg, vg)), G, dev_mask(sees),
                        *map(to_dev_bf16, (k, v)))
    for word in (0x7FC0, 0x7F80, 0xFF80):  # NaN, inf, -inf
        kb, vb = kg.copy(), vg.copy()
        kb[G:][bad], vb[G:][bad] = word, word
        got = P.phase2_tree(*map(to_dev_bf16, (q, kb, vb)), G, dev_mask(sees),
                            *map(to_dev_bf16, (k, v)))
        for a, b in zip(got, ref):
            assert torch.equal(a, b)


def test_nan_in_a_seen_draft_shows():
    Tq, Hq, Hkv, d = 3, 4, 1, 64
    q, kg, vg = (normal(s, sh) for s, sh in ((41, (Tq, Hq, d)), (42, (Tq, Hkv, d)),
                                             (43, (Tq, Hkv, d))))
    kg[0, 0, 0] = 0x7FC0
    o, lse = P.phase2_tree(*map(to_dev_bf16, (q, kg, vg)), 0, dev_mask(np.eye(3, dtype=bool)))
    assert torch.isnan(o[0]).all() and torch.isnan(lse[:, 0]).all()
    assert torch.isfinite(o[1:]).all() and torch.isfinite(lse[:, 1:]).all()


def test_tree_captured_and_replayed():
    # mask and attention of two steps in one graph, replayed with eager calls between
    Tq, G, Hq, Hkv, d = 24, 40, 32, 8, 128
    q, kg, vg = (to_dev_bf16(normal(s, sh)) for s, sh in (
        (51, (Tq, Hq, d)), (52, (G + Tq, Hkv, d)), (53, (G + Tq, Hkv, d))))
    k, v = (to_dev_bf16(normal(s, (4, 200, Hkv, d))) for s in (54, 55))
    parent = dev_i32(random_tree(56, Tq))

    def both():
        mask, _ = P.tree_mask(parent)
        return P.phase2_tree(q, kg, vg, G, mask, k, v) + P.phase2_tree(
            q[:5].contiguous(), kg[:G + 5], vg[:G + 5], G, mask[:5].contiguous(), k, v)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for i in range(3):
        parent.copy_(dev_i32(random_tree(60 + i, Tq)))
        q.mul_(-1)
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i


def test_tree_workspace_sized_once():
    # a loop sizes its workspace for its largest step; every smaller one finds room
    H, S, Hq, Hkv, d, G = 3, 700, 32, 8, 128, 1200
    size = P.phase2_tree_workspace_bytes(H, 40, S, G, Hq, Hkv, d)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    k, v = (to_dev_bf16(normal(s, (H, S, Hkv, d))) for s in (71, 72))
    kg, vg = (to_dev_bf16(normal(s, (G + 40, Hkv, d))) for s in (73, 74))
    for Tq in (1, 3, 8, 9, 20, 32, 33, 40):
        q = to_dev_bf16(normal(75, (Tq, Hq, d)))
        mask, _ = P.tree_mask(dev_i32(random_tree(Tq, Tq)))
        for g0 in (0, 31, 257, 1100, 1200):
            for h, s in ((1, 64), (2, 700), (3, 512), (3, 700)):
                kc, vc = k[:h, :s].contiguous(), v[:h, :s].contiguous()
                args = (q, kg[:g0 + Tq], vg[:g0 + Tq], g0, mask, kc, vc)
                o = torch.empty((Tq, Hq, d), device="cuda")
                lse = torch.empty((Hq, Tq), device="cuda")
                ptr = torch.Tensor.data_ptr
                assert P.api._lib.lib().pulsar_phase2_tree(
                    ptr(q), ptr(kg), ptr(vg), g0, ptr(mask), ptr(kc), ptr(vc), h, Tq, s, Hq, Hkv,
                    d, 1 / math.sqrt(d), ptr(o), 0, ptr(lse), ptr(ws), size,
                    P.api._stream()) == 0, (Tq, g0, h, s)
                ref = P.phase2_tree(*args)
                assert torch.equal(o, ref[0]) and torch.equal(lse, ref[1]), (Tq, g0, h, s)


def test_tree_over_more_than_four_gib():
    # shards of 2 GB each in one launch: rows whose byte offsets pass 32 bits
    ns, Hq, Hkv, d, S, G = 3, 32, 8, 128, 1000000, 2
    q = normal(76, (1, Hq, d))
    q[:, :, 0] = 0x4100  # 8
    ks, vs = normal(77, (6, Hkv, d)), normal(78, (6, Hkv, d))
    ks[:, :, 0] = 0
    kg, vg = (normal(s, (G + 1, Hkv, d)) for s in (79, 80))
    kg[:, :, 0] = 0
    K = torch.zeros((ns, S, Hkv, d), dtype=torch.bfloat16, device="cuda")
    V = torch.ones_like(K)
    K[..., 0] = -256.0  # scores below -180: weights of 0 beside those of the six
    at = [(0, 0), (0, S - 1), (1, 0), (1, 77777), (2, 400001), (2, S - 1)]
    for i, (h, r) in enumerate(at):
        K[h, r], V[h, r] = to_dev_bf16(ks[i]), to_dev_bf16(vs[i])
    o, lse = P.phase2_tree(to_dev_bf16(q), to_dev_bf16(kg), to_dev_bf16(vg), G,
                           dev_mask(np.ones((1, 1), bool)), K, V)
    ref, keys = tree_reference(q, kg, vg, G, np.ones((1, 1), bool), ks[None], vs[None],
                               1 / math.sqrt(d))
    check(o, lse, ref, keys, "4 GiB")


def test_refusals_of_device_tensors():
    bf = {"dtype": torch.bfloat16, "device": "cuda"}
    q, kg, k = torch.zeros(2, 8, 64, **bf), torch.zeros(6, 4, 64, **bf), torch.zeros(1, 40, 4, 64, **bf)
    mask, sel = dev_i32([[1], [3]]), dev_i32(np.zeros((1, 2, 4, 1)))
    bounds = P.key_bounds(k, 16)
    keep = dev_i32([0, 1])
    wrong = [
        lambda: P.tree_mask(mask), lambda: P.tree_mask(keep.long()), lambda: P.tree_mask(keep.cpu()),
        lambda: P.tree_mask(dev_i32(range(8))[::2]),
        lambda: P.phase2_tree(q.float(), kg, kg, 4, mask), lambda: P.phase2_tree(q, kg, kg, 3, mask),
        lambda: P.phase2_tree(q, kg, kg[:5], 4, mask), lambda: P.phase2_tree(q, kg, kg, 4, mask[:1]),
        lambda: P.phase2_tree(q, kg, kg, 4, mask.cpu()),
        lambda: P.phase2_tree(q, kg, kg, 4, mask, k, k[:, :9]),
        lambda: P.phase2_tree(q, kg, kg, 4, mask, k[:, ::2], k[:, ::2]),
        lambda: P.phase2_tree(q, kg, kg, 4, mask, o_dtype=7),
        lambda: P.phase2_tree(q, kg.cpu(), kg, 4, mask),
        lambda: P.phase2_tree(q.transpose(0, 1).contiguous().transpose(0, 1), kg, kg, 4, mask),
        lambda: P.kv_compact_(k, k, 0, keep), lambda: P.kv_compact_(k, k.clone()[:, :9], 0, keep),
        lambda: P.kv_compact_(torch.zeros(3, 9, 1, 8, **bf)[:2], torch.zeros(2, 9, 1, 8), 0, keep),
        lambda: P.kv_compact_(k, k.clone(), 0, keep[None]),
        lambda: P.key_bounds(k.float(), 16), lambda: P.key_bounds(k, (1 << 32) + 16),
        lambda: P.key_bounds(k, 16 - (1 << 32)),
        lambda: P.block_select(q, bounds[..., :32].contiguous(), 1),
        lambda: P.block_select(q, bounds, (1 << 32) + 1),
        lambda: P.block_select(q, bounds, 2 - (1 << 32)), lambda: P.block_select(q, bounds.cpu(), 1),
        lambda: P.phase2_sparse(q, k, k[:, :9].contiguous(), sel, 16),
        lambda: P.phase2_sparse(q, k, k, sel[:, :1].contiguous(), 16),
        lambda: P.phase2_sparse(q, k, k, sel.long(), 16), lambda: P.phase2_sparse(q, k, k, sel, 16, kg),
        lambda: P.phase2_sparse(q, k, k, sel, 16, kg, kg, 3),
        lambda: P.phase2_sparse(q, k, k, sel, 16, kg, kg, 4, mask[:, :0]),
        lambda: P.phase2_sparse(q, k, k, sel, (1 << 32) + 16),
    ]
    for i, fn in enumerate(wrong):
        with pytest.raises(ValueError):
            fn()
            pytest.fail(f"call {i} was not refused")
    both = torch.zeros(2, 1, 40, 4, 64, **bf)
    shared = both.view(-1)[:both.numel() // 2 + 8 * 4 * 64]
    with pytest.raises(ValueError):  # the second half begins inside the first
        P.kv_compact_(shared[:40 * 256].view(1, 40, 4, 64),
                      shared[8 * 256:].view(1, 40, 4, 64), 0, keep)
    for fn in (lambda: P.key_bounds(k, 24), lambda: P.key_bounds(k, 0),
               lambda: P.block_select(q, bounds, 4), lambda: P.block_select(q, bounds, -1),
               lambda: P.phase2_sparse(q, k, k, sel, 24), lambda: P.kv_compact_(k, k.clone(), 39, keep),
               lambda: P.kv_compact_(k, k.clone(), -1, keep),
               lambda: P.phase2_sparse(q, k, k, sel, 16, softmax_scale=0.0),
               lambda: P.phase2_sparse(q, k, k, sel, 16, mask=mask)):
        with pytest.raises(RuntimeError):
            fn()


def _compact(layers, capacity, Hkv, d, G, keep, what):
    shape = (layers, capacity, Hkv, d)
    k, v = normal(81, shape), normal(82, shape)
    K, V = to_dev_bf16(k), to_dev_bf16(v)
    out = P.kv_compact_(K, V, G, dev_i32(keep))
    assert out[0] is K and out[1] is V
    for got, x in ((K, k), (V, v)):
        want = ob.kv_compact(x, G, keep)
        assert np.array_equal(got.view(torch.int16).cpu().numpy().view(np.uint16), want), what


@pytest.mark.parametrize("layers,capacity,Hkv,d,G,keep", [
    (1, 1, 1, 64, 0, [0]),
    (3, 40, 8, 128, 10, [0, 2, 5, 11]),
    (2, 40, 8, 128, 10, [29]),                       # the last row
    (2, 70, 1, 64, 3, list(range(67))),              # all in place
    (2, 70, 3, 8, 3, list(range(1, 67))),            # every row moves by one, odd rows
    (2, 900, 2, 64, 7, list(range(0, 800, 2))),      # many, overlapping
    (2, 40, 2, 64, 10, []),
    (2, 40, 2, 64, 10, [-1, 3, 4]),                  # nothing accepted
    (2, 40, 2, 64, 10, [2, 4, -1, 9]),               # a list filled up with -1
    (2, 40, 2, 64, 10, [2, 4, 4, 9]),                # the same row twice ends it
    (2, 40, 2, 64, 10, [2, 8, 5, 9]),                # a row that falls ends it
    (2, 40, 2, 64, 10, [2, 29, 30, 31]),             # past the cache
    (2, 60, 2, 64, 10, list(range(3, 19)) + [-1] + list(range(30, 40))),  # ends after 16
])
def test_compact(layers, capacity, Hkv, d, G, keep):
    _compact(layers, capacity, Hkv, d, G, keep, f"{keep[:20]}")


def test_compact_random_lists():
    rng = np.random.default_rng(83)
    for n in (5, 16, 17, 32, 33, 100, 333):
        keep = np.sort(rng.choice(500, size=n, replace=False))
        _compact(3, 600, 4, 64, 100, keep, f"{n} of 500")
        for bad in (0, n // 2, n - 1):  # where the list ends
            cut = keep.copy()
            cut[bad] = -1
            _compact(1, 600, 3, 8, 100, cut, f"{n} of 500, -1 at {bad}")
    # many batches of rows, few columns; rows that stay; columns beyond a power of two
    _compact(1, 4100, 1, 64, 50, np.sort(rng.choice(4000, size=3000, replace=False)), "3000")
    _compact(2, 2000, 5, 72, 9, np.r_[0:700, 701:1900], "the first 700 stay")
    _compact(1, 1500, 1, 8, 0, np.arange(1, 1500), "all by one")
    _compact(130, 60, 9, 64, 2, np.arange(3, 58), "many layers")


@pytest.mark.parametrize("n", [7, 200])
def test_compact_captured_and_replayed(n):
    # the list changes on the device between the replays, its length with it
    layers, capacity, Hkv, d, G = 3, 400, 2, 64, 50
    k, v = (normal(s, (layers, capacity, Hkv, d)) for s in (84, 85))
    K, V = to_dev_bf16(k), to_dev_bf16(v)
    keep = dev_i32(np.full(n, -1))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        P.kv_compact_(K, V, G, keep)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.kv_compact_(K, V, G, keep)
    rng = np.random.default_rng(n)
    for i in range(4):
        rows = np.full(n, -1)
        m = (n, n // 2, 0, n)[i]
        rows[:m] = np.sort(rng.choice(capacity - G, size=m, replace=False))
        keep.copy_(dev_i32(rows))
        graph.replay()
        torch.cuda.synchronize()
        k, v = (ob.kv_compact(x, G, rows) for x in (k, v))
        for got, x in ((K, k), (V, v)):
            assert np.array_equal(got.view(torch.int16).cpu().numpy().view(np.uint16), x), i


def test_compact_past_two_gib():
    # a layer behind the 32-bit offsets of the cache
    layers, capacity, Hkv, d, G = 3, 530000, 8, 128, 500000
    K = torch.zeros((layers, capacity, Hkv, d), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    rows = torch.arange(capacity - G, device="cuda", dtype=torch.float32)
    K[:, G:] = (rows % 251)[None, :, None, None].to(torch.bfloat16)
    V[:, G:] = (rows % 241)[None, :, None, None].to(torch.bfloat16)
    keep = [5, 100, 101, 29999]
    P.kv_compact_(K, V, G, dev_i32(keep))
    for x, m in ((K, 251), (V, 241)):
        for j, r in enumerate(keep):
            assert (x[:, G + j] == r % m).all()
        assert (x[:, G + len(keep)] == len(keep) % m).all() and (x[:, G - 1] == 0).all()
