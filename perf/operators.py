"""Performance cases of Phase 2 with drafted tokens and with block-sparse reads
of the retained shards, through the package's public entry points.

Each case is one call, or the short sequence of calls that a program makes
together, on inputs that the program already holds on the GPU:

  kind "bounds"   ``key_bounds``: the smallest and largest value of every key
                  channel in each block of a retained shard.
  kind "select"   ``block_select``: the blocks of each shard whose bounds allow
                  the largest score, for every token and KV head.
  kind "sparse"   ``phase2_sparse``: attention of new tokens over their selected
                  blocks and the generation shard.
  kind "step"     ``block_select`` and ``phase2_sparse``, as a generation step
                  of a layer makes them.
  kind "tree"     ``tree_mask`` and ``phase2_tree``: attention of a tree of
                  drafted tokens over the shards, the generation shard and each
                  token's own branch.
  kind "compact"  ``kv_compact_``: the rows that are kept moved to the front,
                  in K and V of every layer.

``run`` gives each kind in its plain form (elementary torch operations) or,
where ``own`` is set, as the framework's calls.  ``listed()`` and ``draw(rng)``
give the cases, ``prepare`` the inputs, ``work`` the bytes and operations that
the path cannot do without, and ``exact`` the outputs in 64 bits.
"""
import math

import torch

own = False


def listed():
    return [
        # Bounds of a 4K context in shards of an odd length, once per layer after
        # its prefill: the smallest call.
        dict(name="bounds_4k", kind="bounds", shards=4, S=1021, block=32, Hkv=8, d=128),
        # Bounds of a 128K context's retained keys: streams all of them.
        dict(name="bounds_128k", kind="bounds", shards=16, S=8192, block=64, Hkv=8, d=128),
        # A generation step's selection from 16 shards of 8192 keys, four blocks
        # of each.
        dict(name="select_1_128k", kind="select", Tq=1, shards=16, S=8192, block=64, topk=4,
             Hq=32, Hkv=8, d=128),
        # Selection for a 64-token question from one long shard in small blocks.
        dict(name="select_64_128k", kind="select", Tq=64, shards=1, S=131072, block=32, topk=128,
             Hq=32, Hkv=8, d=128),
        # A generation step over a 4K context, small blocks of shards of an odd
        # length: the smallest attention, where latency and launches count.
        dict(name="sparse_1_4k", kind="sparse", Tq=1, G=45, shards=4, S=1021, block=16, topk=8,
             Hq=32, Hkv=8, d=128),
        # A short question in a layer with one query head per KV head, sizes that
        # divide into no tile.
        dict(name="sparse_24_mha_ragged", kind="sparse", Tq=24, G=300, shards=5, S=3001, block=32,
             topk=12, Hq=16, Hkv=16, d=64),
        # A long question over a 128K context, 4096 keys for each token.
        dict(name="sparse_128_128k", kind="sparse", Tq=128, G=0, shards=1, S=131072, block=64,
             topk=64, Hq=32, Hkv=8, d=128),
        # A generation step of a layer over a 128K context: selection, then
        # attention, of 4096 of its keys.
        dict(name="step_1_128k", kind="step", Tq=1, G=100, shards=16, S=8192, block=64, topk=4,
             Hq=32, Hkv=8, d=128),
        # Verification of 12 drafted tokens over a 4K context.
        dict(name="tree_12_4k", kind="tree", Tq=12, G=45, shards=4, S=1021, Hq=32, Hkv=8, d=128),
        # Verification of a large tree over a 128K context: reads every key.
        dict(name="tree_64_128k", kind="tree", Tq=64, G=700, shards=16, S=8192, Hq=32, Hkv=8,
             d=128),
        # The accepted path of a draft moved to the front in every layer: a few
        # rows, once per verification.
        dict(name="compact_draft", kind="compact", layers=32, G=1000, rows=64, keep=6, Hkv=8,
             d=128),
        # A long generation shard thinned to the rows that are kept.
        dict(name="compact_long", kind="compact", layers=32, G=64, rows=4000, keep=1500, Hkv=8,
             d=128),
    ]


# Layer shapes (query heads, KV heads, head dimension) that the draws use.
LAYERS = [(32, 8, 128), (32, 8, 128), (4, 1, 64), (16, 16, 64), (8, 2, 128), (16, 8, 64)]
# Keys that a drawn sparse case reads at most, over its tokens and KV heads, in
# channels: the largest listed one's.
MOST_READ = 128 * 8 * 4096 * 128


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["bounds", "select", "select", "sparse", "sparse", "sparse", "step", "step",
                       "tree", "tree", "tree", "compact"])
    Hq, Hkv, d = rng.choice(LAYERS)
    if kind == "compact":
        rows = _log_int(rng, 4, 4000)
        return dict(kind=kind, layers=rng.randint(1, 32), G=_log_int(rng, 1, 2000), rows=rows,
                    keep=_log_int(rng, 1, max(1, rows // 2)), Hkv=Hkv, d=d)
    shards = rng.choice([1, 1, 4, 5, 8, 16])
    S = _log_int(rng, 512, 131072 // shards)
    if kind == "tree":
        return dict(kind=kind, Tq=_log_int(rng, 2, 64), G=_log_int(rng, 1, 2000), shards=shards,
                    S=S, Hq=Hq, Hkv=Hkv, d=d)
    block = rng.choice([16, 32, 64, 64, 128])
    if kind == "bounds":
        return dict(kind=kind, shards=shards, S=S, block=block, Hkv=Hkv, d=d)
    blocks = -(-S // block)
    topk = _log_int(rng, 1, max(1, min(blocks // 2, 8192 // (block * shards))))
    most = 128
    if kind != "select":
        most = max(1, min(most, MOST_READ // (Hkv * d * shards * topk * block)))
    case = dict(kind=kind, Tq=_log_int(rng, 1, most), shards=shards, S=S, block=block, topk=topk,
                Hq=Hq, Hkv=Hkv, d=d)
    if kind == "select":
        case["Tq"] = _log_int(rng, 1, max(1, min(64, (64 * 32 * 4096) // (Hq * shards * blocks))))
    else:
        case["G"] = _log_int(rng, 1, 1000)
    return case


# ---- inputs ---------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape):
    """bf16 N(0, 1), as the activations of a normalised layer."""
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _pool(case):
    """Blocks of a shard and KV head that any token of the case selects."""
    return min(-(-case["S"] // case["block"]), 4 * case["topk"])


def _selection(case, gen):
    """int32 [shards, Tq, Hkv, topk]: ascending blocks of every shard.  The
    tokens of a question draw theirs from the same few blocks of a KV head."""
    n, Tq, Hkv, blocks = case["shards"], case["Tq"], case["Hkv"], -(-case["S"] // case["block"])
    u = torch.rand((n, 1, Hkv, blocks), generator=gen, device="cuda")
    pool = torch.topk(u, _pool(case), dim=3).indices.expand(n, Tq, Hkv, -1)
    u = torch.rand((n, Tq, Hkv, _pool(case)), generator=gen, device="cuda")
    pick = torch.topk(u, case["topk"], dim=3).indices
    return torch.sort(torch.gather(pool, 3, pick), dim=3).values.to(torch.int32).contiguous()


def _min_max(K, block):
    """bf16 [shards, Hkv, blocks, 2, d]: each block's channel minima and maxima."""
    n, S, Hkv, d = K.shape
    blocks = -(-S // block)
    # the last block is filled up with copies of the shard's last key
    at = torch.arange(blocks * block, device="cuda").clamp_(max=S - 1)
    x = K.float()[:, at].view(n, blocks, block, Hkv, d)
    both = torch.stack([x.amin(2), x.amax(2)], dim=3)      # [n, blocks, Hkv, 2, d]
    return both.transpose(1, 2).contiguous().to(torch.bfloat16)


def _parents(case, gen):
    """int32 [Tq]: a random recursive tree, several tokens after the last row."""
    t = torch.arange(case["Tq"], device="cuda")
    u = torch.rand(case["Tq"], generator=gen, device="cuda", dtype=torch.float64)
    return (torch.floor(u * (t + 1)) - 1).to(torch.int32)


def prepare(case, seed):
    kind, gen = case["kind"], _gen(seed)
    Hkv, d = case["Hkv"], case["d"]
    if kind == "compact":
        shape = (case["layers"], case["G"] + case["rows"], Hkv, d)
        K, V = _normal(gen, shape), _normal(gen, shape)
        u = torch.rand(case["rows"], generator=gen, device="cuda")
        keep = torch.sort(torch.topk(u, case["keep"]).indices).values.to(torch.int32)
        return dict(case=case, K=K, V=V, keep=keep)
    K = _normal(gen, (case["shards"], case["S"], Hkv, d))
    if kind == "bounds":
        return dict(case=case, K=K)
    st = dict(case=case, q=_normal(gen, (case["Tq"], case["Hq"], d)), K=K)
    if kind in ("select", "step"):
        st["bounds"] = _min_max(K, case["block"])
    if kind == "select":
        del st["K"]
        return st
    st["V"] = _normal(gen, K.shape)
    rows = (case["G"] + case["Tq"], Hkv, d)
    st["Kg"], st["Vg"] = _normal(gen, rows), _normal(gen, rows)
    if kind == "sparse":
        st["sel"] = _selection(case, gen)
    if kind == "tree":
        st["parent"] = _parents(case, gen)
    return st


# ---- the plain forms --------------------------------------------------------


def _softmax(s, V):
    """Weights exp(s - max) over the last axis of s, then their product with V
    (one more axis) and the log-sum-exp; a row without keys gives 0 and -inf."""
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    z = p.sum(-1, keepdim=True)
    o = (p @ V) / torch.where(z == 0, 1.0, z)
    return o, (m + torch.log(z)).squeeze(-1)


def _plain_mask(parent):
    """The bits of each token's branch, 32 to a word, and its depth."""
    T = parent.numel()
    p = parent.long()
    t = torch.arange(T, device="cuda")
    reach = ((p[:, None] == t[None, :]) | (t[:, None] == t[None, :])).float()
    for _ in range(max(1, T - 1).bit_length()):
        reach = ((reach @ reach) > 0).float()
    words = (T + 31) // 32
    bits = torch.zeros((T, words * 32), dtype=torch.int64, device="cuda")
    bits[:, :T] = reach.long()
    word = (bits.view(T, words, 32) << torch.arange(32, device="cuda")).sum(2)
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
    return word, reach.sum(1).to(torch.int32) - 1, reach > 0


def _plain_tree(q, Kg, Vg, G, sees, K, V):
    Tq, Hq, d = q.shape
    Hkv = Kg.shape[1]
    group = Hq // Hkv
    Kc = torch.cat([K.flatten(0, 1), Kg]).float().permute(1, 2, 0)      # [Hkv, d, n]
    Vc = torch.cat([V.flatten(0, 1), Vg]).float().transpose(0, 1)      # [Hkv, n, d]
    x = q.float().view(Tq, Hkv, group, d).transpose(0, 1).reshape(Hkv, Tq * group, d)
    s = (x @ Kc.contiguous()) / math.sqrt(d)
    n = s.shape[2]
    s = s.view(Hkv, Tq, group, n)
    s[..., n - Tq:].masked_fill_(~sees[None, :, None, :], -math.inf)
    o, lse = _softmax(s.view(Hkv, Tq * group, n), Vc.contiguous())
    o = o.view(Hkv, Tq, group, d).transpose(0, 1).reshape(Tq, Hq, d)
    return o.to(torch.bfloat16), lse.view(Hkv, Tq, group).transpose(1, 2).reshape(Hq, Tq)


def _plain_select(q, bounds, topk):
    n, Hkv, blocks, _, d = bounds.shape
    Tq, Hq, _ = q.shape
    lo, hi = bounds[..., 0, :].double(), bounds[..., 1, :].double()
    x = q.double().view(Tq, Hkv, Hq // Hkv, d).transpose(0, 1).reshape(Hkv, -1, d)
    s = x.clamp(min=0) @ hi.transpose(2, 3) + x.clamp(max=0) @ lo.transpose(2, 3)
    s = s.float().view(n, Hkv, Tq, Hq // Hkv, blocks).amax(3)
    best = torch.sort(s, dim=3, descending=True, stable=True).indices[..., :topk]
    return torch.sort(best, dim=3).values.transpose(1, 2).to(torch.int32).contiguous()


def _plain_sparse(q, K, V, sel, block, Kg, Vg, G):
    n, S, Hkv, d = K.shape
    Tq, Hq, _ = q.shape
    group, topk = Hq // Hkv, sel.shape[3]
    row = sel.long()[..., None] * block + torch.arange(block, device="cuda")
    inside = (row < S) & (sel >= 0)[..., None]
    at = row.clamp(0, S - 1) + torch.arange(n, device="cuda").view(n, 1, 1, 1, 1) * S
    head = torch.arange(Hkv, device="cuda").view(1, 1, Hkv, 1, 1)
    keys = n * topk * block

    def of_token(x):  # [n, Tq, Hkv, topk, block, ...] -> [Tq, Hkv, keys, ...]
        return x.permute(1, 2, 0, 3, 4, *range(5, x.dim())).reshape(Tq, Hkv, keys, *x.shape[5:])

    Ks = of_token(K.flatten(0, 1)[at, head]).float()
    Vs = of_token(V.flatten(0, 1)[at, head]).float()
    x = q.float().view(Tq, Hkv, group, d)
    s = x @ Ks.transpose(2, 3)
    s.masked_fill_(~of_token(inside)[:, :, None, :], -math.inf)
    g = x @ Kg.float().permute(1, 2, 0).contiguous()                    # [Tq, Hkv, group, G + Tq]
    t = torch.arange(Tq, device="cuda")[:, None]
    after = torch.arange(G + Tq, device="cuda")[None, :] > G + t
    g.masked_fill_(after[:, None, None, :], -math.inf)
    s = torch.cat([s, g], dim=3) / math.sqrt(d)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    o = (p[..., :keys] @ Vs + p[..., keys:] @ Vg.float().transpose(0, 1).contiguous()) / z
    lse = (m + torch.log(z)).view(Tq, Hq).t().contiguous()
    return o.reshape(Tq, Hq, d).to(torch.bfloat16), lse


# ---- one pass -------------------------------------------------------------


def run(state):
    c = state["case"]
    kind = c["kind"]
    if own:
        import paper_2607_20457_amd as P
        if kind == "bounds":
            return P.key_bounds(state["K"], c["block"])
        if kind == "select":
            return P.block_select(state["q"], state["bounds"], c["topk"])
        if kind == "sparse":
            return P.phase2_sparse(state["q"], state["K"], state["V"], state["sel"], c["block"],
                                   state["Kg"], state["Vg"], c["G"], o_dtype=P.OUT_BF16)
        if kind == "step":
            sel = P.block_select(state["q"], state["bounds"], c["topk"])
            return (sel,) + tuple(P.phase2_sparse(state["q"], state["K"], state["V"], sel,
                                                  c["block"], state["Kg"], state["Vg"], c["G"],
                                                  o_dtype=P.OUT_BF16))
        if kind == "tree":
            mask, depth = P.tree_mask(state["parent"])
            return (mask, depth) + tuple(P.phase2_tree(state["q"], state["Kg"], state["Vg"], c["G"],
                                                       mask, state["K"], state["V"],
                                                       o_dtype=P.OUT_BF16))
        return P.kv_compact_(state["K"], state["V"], c["G"], state["keep"])
    if kind == "bounds":
        return _min_max(state["K"], c["block"])
    if kind == "select":
        return _plain_select(state["q"], state["bounds"], c["topk"])
    if kind in ("sparse", "step"):
        sel = state["sel"] if kind == "sparse" else \
            _plain_select(state["q"], state["bounds"], c["topk"])
        out = _plain_sparse(state["q"], state["K"], state["V"], sel, c["block"], state["Kg"],
                            state["Vg"], c["G"])
        return out if kind == "sparse" else (sel,) + out
    if kind == "tree":
        mask, depth, sees = _plain_mask(state["parent"])
        return (mask, depth) + _plain_tree(state["q"], state["Kg"], state["Vg"], c["G"], sees,
                                           state["K"], state["V"])
    rows = c["G"] + state["keep"].long()
    for x in (state["K"], state["V"]):
        x[:, c["G"]:c["G"] + c["keep"]] = x[:, rows]
    return state["K"], state["V"]


# ---- what a pass cannot do without -----------------------------------------


def work(case):
    kind, Hkv, d = case["kind"], case["Hkv"], case["d"]
    row = Hkv * d * 2
    if kind == "compact":
        # K and V rows read and written
        return dict(bytes=2 * 2 * case["layers"] * case["keep"] * row, flops=0)
    n, S = case["shards"], case["S"]
    if kind == "bounds":
        blocks = n * -(-S // case["block"])
        return dict(bytes=n * S * row + blocks * 2 * row, flops=2 * n * S * Hkv * d)
    Tq, Hq = case["Tq"], case["Hq"]
    nbytes, flops = Tq * Hq * d * 2, 0
    if kind in ("select", "step"):
        blocks = n * -(-S // case["block"])
        nbytes += blocks * 2 * row + 4 * n * Tq * Hkv * case["topk"]
        flops += 4 * d * Hq * Tq * blocks
    if kind == "select":
        return dict(bytes=nbytes, flops=flops)
    nbytes += Tq * Hq * (2 * d + 4) + 2 * (case["G"] + Tq) * row
    pairs = Tq * case["G"] + Tq * (Tq + 1) // 2
    if kind == "tree":
        words = (Tq + 31) // 32
        nbytes += 2 * n * S * row + Tq * (8 + 4 * words)
        # the drafts' own branches are a few tokens each, counted as one
        pairs = Tq * (n * S + case["G"] + 1)
    else:
        if kind == "sparse":
            nbytes += 4 * n * Tq * Hkv * case["topk"]
        # blocks that at least one token selects, each read once
        pool = _pool(case) if kind == "sparse" else -(-S // case["block"])
        used = pool * (1 - (1 - case["topk"] / pool) ** Tq)
        nbytes += int(2 * n * used * case["block"] * row)
        pairs += Tq * n * case["topk"] * case["block"]
    return dict(bytes=nbytes, flops=flops + 4 * d * Hq * pairs)


# ---- the same outputs in 64 bits ------------------------------------------


def _weighted(q, K, V, counts):
    """q [T, Hq, d] over K, V [n, Hkv, d] in fp64, key c of KV head g counting
    counts(g)[t, c] times for token t -> (o [T, Hq, d], lse [Hq, T])."""
    T, Hq, d = q.shape
    group = Hq // K.shape[1]
    o = torch.empty((T, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((Hq, T), dtype=torch.float64, device="cuda")
    for g in range(K.shape[1]):
        Kt, Vg = K[:, g].double().t().contiguous(), V[:, g].double().contiguous()
        lc = torch.log(counts(g))
        for h in range(g * group, (g + 1) * group):
            s = (q[:, h].double() / math.sqrt(d)) @ Kt + lc
            ell = torch.logsumexp(s, 1)
            o[:, h] = torch.exp_(s - ell[:, None]) @ Vg
            lse[h] = ell
    return o, lse


def _best_blocks(q, bounds, topk):
    """int [shards, Tq, Hkv, topk]: the blocks with the largest value that some
    key within their bounds could score, from the products themselves."""
    n, Hkv, blocks, _, d = bounds.shape
    Tq, group = q.shape[0], q.shape[1] // Hkv
    sel = torch.empty((n, Tq, Hkv, topk), dtype=torch.int64, device="cuda")
    index = torch.arange(blocks, device="cuda").expand(n, blocks)
    for g in range(Hkv):
        lo, hi = bounds[:, g, None, :, 0].double(), bounds[:, g, None, :, 1].double()
        for t in range(Tq):
            x = q[t, g * group:(g + 1) * group].double()[None, :, None, :]
            s = torch.maximum(x * lo, x * hi).sum(-1).amax(1).float()
            # a stable order by falling score: the lower index first among equals
            order = torch.argsort(-s, dim=1, stable=True)
            rank = torch.empty_like(order).scatter_(1, order, index)
            sel[:, t, g] = torch.nonzero(rank < topk)[:, 1].view(n, topk)
    return sel


def exact(case, seed):
    kind = case["kind"]
    if kind == "select":
        return None
    st = prepare(case, seed)
    if kind == "compact":
        out = []
        for x in (st["K"], st["V"]):
            y = x.double()
            y[:, case["G"]:case["G"] + case["keep"]] = x.double()[:, case["G"] + st["keep"].long()]
            out.append(y)
        return tuple(out)
    n, S = case["shards"], case["S"]
    if kind == "bounds":
        parts = torch.split(st["K"].double(), case["block"], dim=1)
        return torch.stack([torch.stack([x.amin(1), x.amax(1)], 2) for x in parts], 2)
    Tq, G = case["Tq"], case["G"]
    Kc = torch.cat([st["K"].flatten(0, 1), st["Kg"]])
    Vc = torch.cat([st["V"].flatten(0, 1), st["Vg"]])
    total = n * S + G + Tq
    t = torch.arange(Tq, device="cuda")
    if kind == "tree":
        sees = torch.ones((Tq, total), dtype=torch.float64, device="cuda")
        own_rows = torch.zeros((Tq, Tq), dtype=torch.float64)
        parent = st["parent"].tolist()
        for i in range(Tq):
            j = i
            while j >= 0:
                own_rows[i, j] = 1
                j = parent[j]
        sees[:, n * S + G:] = own_rows.cuda()
        return (None, None) + _weighted(st["q"], Kc, Vc, lambda g: sees)
    if kind == "step":
        sel = _best_blocks(st["q"], st["bounds"], case["topk"])
    else:
        sel = st["sel"]

    def counts(g):
        w = torch.zeros((Tq, total), dtype=torch.float64, device="cuda")
        for h in range(n):
            per = torch.zeros((Tq, -(-S // case["block"])), dtype=torch.float64, device="cuda")
            chosen = sel[h, :, g].long()
            per.scatter_add_(1, chosen, torch.ones_like(chosen, dtype=torch.float64))
            w[:, h * S:(h + 1) * S] = torch.repeat_interleave(per, case["block"], dim=1)[:, :S]
        w[:, n * S:] = (torch.arange(G + Tq, device="cuda")[None, :] <= G + t[:, None]).double()
        return w

    out = _weighted(st["q"], Kc, Vc, counts)
    return out if kind == "sparse" else (None,) + out
