"""Performance cases of a cache held in 8 bits: rows quantised as they are
written, read back, and attended to in Phase 2, through the package's public
entry points.

A cache is codes [n, Hkv, capacity, d] of K and of V, in e4m3 or int8, with an
fp32 scale for each block of tokens and head, [n, Hkv, ceil(capacity / block)].
A scale is the least power of two with which the block's largest magnitude is no
more than the largest code (448 or 127), a code the nearest one, ties to even.

Each case is one call, or the short sequence of calls that a program makes
together, on inputs that the program already holds on the GPU:

  kind "write"   ``kv_quantize_``: rows of every layer written into caches that
                 the program keeps.
  kind "trip"    ``kv_quantize`` and ``kv_dequantize``: a cache written, and read
                 back as a bf16 tensor.
  kind "read"    ``kv_dequantize``.
  kind "attn"    ``phase2_quant``: attention of new tokens over quantised shards
                 and the generation shard.
  kind "tree"    the same of a tree of drafted tokens.
  kind "step"    ``kv_quantize_`` and ``phase2_quant``: the generation shard's
                 oldest rows moved into the quantised shard, then a step.

``run`` gives each kind in its plain form (elementary torch operations) or,
where ``own`` is set, as the framework's calls.  ``listed()`` and ``draw(rng)``
give the cases, ``prepare`` the inputs, ``work`` the bytes and operations that
the path cannot do without, and ``exact`` the outputs in 64 bits.
"""
import math

import torch

own = False

FORMATS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def listed():
    return [
        # The generation shard's oldest block moved into the quantised caches of
        # all layers, once every 64 tokens: the smallest write.
        dict(name="write_block", kind="write", n=32, rows=64, first=128, capacity=192, block=64,
             Hkv=8, d=128, fmt="e4m3"),
        # A 128K context's retained shards, once per layer after its prefill.
        dict(name="write_128k", kind="write", n=16, rows=8192, first=0, capacity=8192, block=64,
             Hkv=8, d=128, fmt="e4m3"),
        # Shards of an odd length in a layer of small heads, written and read back.
        dict(name="trip_ragged", kind="trip", n=5, rows=3001, block=32, Hkv=16, d=64, fmt="int8"),
        # A 4K context in shards of an odd length, read back: the smallest call.
        dict(name="read_4k", kind="read", n=4, rows=1021, block=16, Hkv=8, d=128, fmt="e4m3"),
        # A 128K context read back, for a reader that takes bf16 alone.
        dict(name="read_128k", kind="read", n=16, rows=8192, block=128, Hkv=8, d=128, fmt="int8"),
        # A generation step over a 4K context: the smallest attention, where
        # latency and launches count.
        dict(name="attn_1_4k", kind="attn", Tq=1, G=45, n=4, S=1021, live=0, block=16, Hq=32,
             Hkv=8, d=128, fmt="e4m3"),
        # A generation step of a layer over a 128K context: streams every code.
        dict(name="attn_1_128k", kind="attn", Tq=1, G=100, n=16, S=8192, live=0, block=64, Hq=32,
             Hkv=8, d=128, fmt="e4m3"),
        # The same in int8, over shards that are filled to different lengths.
        dict(name="attn_1_live_int8", kind="attn", Tq=1, G=100, n=16, S=8192, live=1, block=64,
             Hq=32, Hkv=8, d=128, fmt="int8"),
        # A short question in a layer with one query head per KV head, sizes that
        # divide into no tile.
        dict(name="attn_24_mha_ragged", kind="attn", Tq=24, G=300, n=5, S=3001, live=0, block=32,
             Hq=16, Hkv=16, d=64, fmt="int8"),
        # A 64-token question over a 128K context: bound by the matrix units.
        dict(name="attn_64_128k", kind="attn", Tq=64, G=0, n=16, S=8192, live=0, block=128, Hq=32,
             Hkv=8, d=128, fmt="e4m3"),
        # Verification of 12 drafted tokens over a 32K context.
        dict(name="tree_12_32k", kind="tree", Tq=12, G=45, n=4, S=8192, live=0, block=64, Hq=32,
             Hkv=8, d=128, fmt="e4m3"),
        # A long generation: 64 rows into the quantised shard, and the next step.
        dict(name="step_1_32k", kind="step", Tq=1, G=40, n=1, S=32768, live=1, block=64, rows=64,
             Hq=32, Hkv=8, d=128, fmt="e4m3"),
    ]


# Layer shapes (query heads, KV heads, head dimension) that the draws use.
LAYERS = [(32, 8, 128), (32, 8, 128), (4, 1, 64), (16, 16, 64), (8, 2, 128), (16, 8, 64)]
# Pairs of query rows and keys, in channels, that a drawn attention has at most: the
# largest listed one's.
MOST_PAIRS = 64 * 32 * 131072 * 128


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "write", "trip", "read", "attn", "attn", "attn", "attn", "tree",
                       "tree", "step"])
    Hq, Hkv, d = rng.choice(LAYERS)
    fmt = rng.choice(["e4m3", "int8"])
    block = rng.choice([16, 32, 64, 64, 128, 256])
    case = dict(kind=kind, block=block, Hkv=Hkv, d=d, fmt=fmt)
    n = rng.choice([1, 1, 4, 5, 8, 16])
    if kind == "write":
        n = rng.choice([n, 32])
        blocks = rng.choice([0, 0, 1, 3])
        rows = _log_int(rng, 1, 131072 // n)
        case.update(n=n, rows=rows, first=blocks * block,
                    capacity=blocks * block + rows + rng.choice([0, 0, 17]), fmt="e4m3")
    elif kind in ("trip", "read"):
        case.update(n=n, rows=_log_int(rng, 1, 131072 // n))
    else:
        S = _log_int(rng, 64, 131072 // n)
        case.update(n=n, S=S, G=_log_int(rng, 1, 2000), live=rng.choice([0, 0, 1]), Hq=Hq)
        case["Tq"] = _log_int(rng, 1, min(256, max(1, MOST_PAIRS // (Hq * d * n * S))))
        if kind == "step":
            case.update(n=1, live=1, rows=block, fmt="e4m3", S=max(S, 2 * block))
    return case


# ---- inputs ---------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(gen, shape):
    """bf16 rows [n, rows, heads, d] whose channels differ in size, as keys' and values' do."""
    spread = torch.exp(0.7 * torch.randn((1, 1) + shape[2:], generator=gen, device="cuda"))
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(torch.bfloat16)


def _blocks_of(x, block):
    """f32 [n, heads, blocks, block, d] of rows [n, rows, heads, d], filled up with zeros."""
    n, rows, heads, d = x.shape
    blocks = -(-rows // block)
    y = torch.zeros((n, heads, blocks * block, d), device="cuda")
    y[:, :, :rows] = x.transpose(1, 2)
    return y.view(n, heads, blocks, block, d)


def _quantised(x, block, fmt):
    """Codes [n, heads, rows, d] and scales [n, heads, blocks] of rows [n, rows, heads, d]."""
    n, rows, heads, d = x.shape
    y = _blocks_of(x, block)
    most = 448.0 if fmt == "e4m3" else 127.0
    e = torch.frexp(y.abs().amax((3, 4)) / most)
    # amax / most = m 2^e with m in [1/2, 1): one half is 2^(e-1) itself
    exp = torch.where(e.mantissa == 0.5, e.exponent - 1, e.exponent).clamp(min=-100)
    s = ((exp.to(torch.int32) + 127) << 23).view(torch.float32)  # 2^exp, from its bits
    y = (y / s[..., None, None]).view(n, heads, -1, d)[:, :, :rows]
    if fmt == "int8":
        y = torch.round(y)
    return y.to(FORMATS[fmt]), s


def _values(codes, s, block):
    """f32 [n, heads, rows, d] that the codes stand for."""
    return codes.float() * torch.repeat_interleave(s, block, dim=2)[:, :, :codes.shape[2], None]


def _parents(case, gen):
    """int32 [Tq]: a random recursive tree, several tokens after the last row."""
    t = torch.arange(case["Tq"], device="cuda")
    u = torch.rand(case["Tq"], generator=gen, device="cuda", dtype=torch.float64)
    return (torch.floor(u * (t + 1)) - 1).to(torch.int32)


def _reach(parent):
    """bool [T, T]: whether token t follows draft j, or is it."""
    T = parent.numel()
    t = torch.arange(T, device="cuda")
    reach = ((parent.long()[:, None] == t[None, :]) | (t[:, None] == t[None, :])).float()
    for _ in range(max(1, T - 1).bit_length()):
        reach = ((reach @ reach) > 0).float()
    return reach > 0


def _words(sees):
    """int32 [T, ceil(T / 32)]: the bits of each row, 32 to a word."""
    T = sees.shape[0]
    words = (T + 31) // 32
    bits = torch.zeros((T, words * 32), dtype=torch.int64, device="cuda")
    bits[:, :T] = sees.long()
    word = (bits.view(T, words, 32) << torch.arange(32, device="cuda")).sum(2)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)


def prepare(case, seed):
    kind, gen = case["kind"], _gen(seed)
    n, Hkv, d, block, fmt = (case[k] for k in ("n", "Hkv", "d", "block", "fmt"))
    st = dict(case=case)
    if kind == "write":
        # rows inside a longer generation shard of every layer; caches that hold others
        more = _rows(gen, (n, case["rows"] + 100, Hkv, d)), _rows(gen, (n, case["rows"] + 100, Hkv, d))
        st["K"], st["V"] = (x[:, 36:36 + case["rows"]] for x in more)
        old = (n, case["capacity"], Hkv, d)
        st["Kc"], st["ks"] = _quantised(_rows(gen, old), block, fmt)
        st["Vc"], st["vs"] = _quantised(_rows(gen, old), block, fmt)
        return st
    rows = case["rows"] if kind in ("trip", "read") else case["S"]
    K, V = _rows(gen, (n, rows, Hkv, d)), _rows(gen, (n, rows, Hkv, d))
    if kind == "trip":
        return dict(st, K=K, V=V)
    st["Kc"], st["ks"] = _quantised(K, block, fmt)
    st["Vc"], st["vs"] = _quantised(V, block, fmt)
    if kind == "read":
        return st
    S, Tq = case["S"], case["Tq"]
    st["q"] = torch.randn((Tq, case["Hq"], d), generator=gen, device="cuda", dtype=torch.bfloat16)
    st["live"] = None
    if case["live"]:
        # from a quarter of the shard's length on
        st["live"] = torch.randint((S + 3) // 4, S + 1, (n,), generator=gen, device="cuda",
                                   dtype=torch.int32)
    if kind == "step":
        # the rows that are moved are the last whole block of those that are live then
        st["first"] = (S // case["rows"] - 1) * case["rows"]
        st["live"] = torch.full((1,), st["first"] + case["rows"], dtype=torch.int32, device="cuda")
        st["K"], st["V"] = (_rows(gen, (1, case["rows"], Hkv, d)) for _ in range(2))
    new = (1, case["G"] + Tq, Hkv, d)
    st["Kg"], st["Vg"] = _rows(gen, new)[0], _rows(gen, new)[0]
    if kind == "tree":
        st["sees"] = _reach(_parents(case, gen))
        st["mask"] = _words(st["sees"])
    return st


# ---- the plain forms --------------------------------------------------------


def _plain_write(K, V, Kc, Vc, ks, vs, block, first, fmt):
    for x, codes, s in ((K, Kc, ks), (V, Vc, vs)):
        c, t = _quantised(x, block, fmt)
        codes[:, :, first:first + c.shape[2]] = c
        s[:, :, first // block:first // block + t.shape[2]] = t


def _plain_read(Kc, Vc, ks, vs, block):
    return tuple(_values(c, s, block).transpose(1, 2).to(torch.bfloat16).contiguous()
                 for c, s in ((Kc, ks), (Vc, vs)))


def _plain_attn(q, Kc, Vc, ks, vs, block, live, Kg, Vg, G, sees):
    n, Hkv, S, d = Kc.shape
    Tq, Hq, _ = q.shape
    group = Hq // Hkv

    def all_rows(codes, s, more):
        x = _values(codes, s, block).transpose(0, 1).reshape(Hkv, n * S, d)
        return torch.cat([x, more.float().transpose(0, 1)], dim=1)

    K, V = all_rows(Kc, ks, Kg), all_rows(Vc, vs, Vg)
    x = q.float().view(Tq, Hkv, group, d).transpose(0, 1).reshape(Hkv, Tq * group, d)
    s = (x @ K.transpose(1, 2).contiguous()) / math.sqrt(d)
    s = s.view(Hkv, Tq, group, n * S + G + Tq)
    if live is not None:
        dead = torch.arange(S, device="cuda")[None, :] >= live[:, None]
        s[..., :n * S].masked_fill_(dead.view(-1), -math.inf)
    if sees is None:
        t = torch.arange(Tq, device="cuda")
        sees = t[None, :] <= t[:, None]
    s[..., n * S + G:].masked_fill_(~sees[None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    o = (p.view(Hkv, Tq * group, -1) @ V).view(Hkv, Tq, group, d) / z
    lse = (m + torch.log(z)).squeeze(-1).transpose(1, 2).reshape(Hq, Tq)
    return o.transpose(0, 1).reshape(Tq, Hq, d).to(torch.bfloat16), lse


# ---- one pass -------------------------------------------------------------


def run(state):
    c = state["case"]
    kind, block, fmt = c["kind"], c["block"], c["fmt"]
    cache = tuple(state.get(k) for k in ("Kc", "Vc", "ks", "vs"))
    if own:
        import paper_2607_20457_amd as P
        if kind == "write":
            return P.kv_quantize_(state["K"], state["V"], *cache, block, c["first"])
        if kind == "trip":
            made = P.kv_quantize(state["K"], state["V"], block, FORMATS[fmt])
            return P.kv_dequantize(*made, block) + made[2:]
        if kind == "read":
            return P.kv_dequantize(*cache, block)
        if kind == "step":
            P.kv_quantize_(state["K"], state["V"], *cache, block, state["first"])
        out = P.phase2_quant(state["q"], *cache, block, state["live"], state["Kg"], state["Vg"],
                             c["G"], mask=state.get("mask"), o_dtype=P.OUT_BF16)
        return cache + tuple(out) if kind == "step" else out
    if kind == "write":
        _plain_write(state["K"], state["V"], *cache, block, c["first"], fmt)
        return cache
    if kind == "trip":
        (Kc, ks), (Vc, vs) = (_quantised(state[k], block, fmt) for k in ("K", "V"))
        return _plain_read(Kc, Vc, ks, vs, block) + (ks, vs)
    if kind == "read":
        return _plain_read(*cache, block)
    if kind == "step":
        _plain_write(state["K"], state["V"], *cache, block, state["first"], fmt)
    out = _plain_attn(state["q"], *cache, block, state["live"], state["Kg"], state["Vg"], c["G"],
                      state.get("sees"))
    return cache + out if kind == "step" else out


# ---- what a pass cannot do without -----------------------------------------


def work(case):
    kind, n, Hkv, d, block = (case[k] for k in ("kind", "n", "Hkv", "d", "block"))
    wide, flops = Hkv * d, 0
    nbytes = 0
    if kind in ("write", "trip", "read", "step"):
        rows = n * case["rows"]
        scales = n * -(-case["rows"] // block) * Hkv * 4
        # K and V: bf16 rows on one side, codes and scales on the other
        nbytes = 2 * (rows * wide * 3 + scales)
        if kind == "trip":
            nbytes = 2 * (rows * wide * 6 + 2 * scales)
        if kind != "read":
            flops = 4 * rows * wide
    if kind in ("attn", "tree", "step"):
        Tq, Hq, G = case["Tq"], case["Hq"], case["G"]
        keys = n * case["S"]
        if kind == "step":
            keys = case["S"] // case["rows"] * case["rows"]
        elif case["live"]:
            keys = keys * 5 // 8
        nbytes += 2 * (keys * wide + keys // block * Hkv * 4 + (G + Tq) * wide * 2)
        nbytes += Tq * Hq * (4 * d + 4)
        # a draft's own branch is a few tokens, counted as one
        pairs = Tq * (keys + G) + (Tq if kind == "tree" else Tq * (Tq + 1) // 2)
        flops += 4 * d * Hq * pairs
    return dict(bytes=nbytes, flops=flops)


# ---- the same outputs in 64 bits ------------------------------------------


def _two_to(e):
    """2^e in 64 bits, exactly, of whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x, block, fmt):
    """f64 codes [n, heads, rows, d] and scales [n, heads, blocks] of bf16 rows
    [n, rows, heads, d], block by block."""
    most = 448.0 if fmt == "e4m3" else 127.0
    codes, scales = [], []
    for part in torch.split(x.double().transpose(1, 2), block, dim=2):
        top = part.abs().amax((2, 3))
        e = torch.ceil(torch.log2(top / most)).clamp(min=-100)
        # the logarithm may be off by a rounding where the quotient is a power of two
        e = torch.where(_two_to(e) * most < top, e + 1, e)
        e = torch.where(_two_to(e - 1) * most >= top, e - 1, e).clamp(min=-100)
        s = _two_to(e)
        y = part / s[:, :, None, None]
        if fmt == "e4m3":
            # eight steps to a binade from 2^-6 on, and the same steps below it
            size = torch.maximum(y.abs(), torch.full_like(y, 2.0 ** -6))
            step = _two_to(torch.frexp(size).exponent - 4)
            y = torch.round(y / step) * step
        else:
            y = torch.round(y)
        codes.append(y)
        scales.append(s)
    return torch.cat(codes, dim=2), torch.stack(scales, dim=2)


def _exact_write(st, first, block, fmt):
    out = []
    for x, codes, s in ((st["K"], st["Kc"], st["ks"]), (st["V"], st["Vc"], st["vs"])):
        c, t = _exact_codes(x, block, fmt)
        all_c, all_s = codes.double(), s.double()
        all_c[:, :, first:first + c.shape[2]] = c
        at = first // block
        all_s[:, :, at:at + t.shape[2]] = t
        out.append((all_c, all_s))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _exact_values(codes, s, block):
    parts = torch.split(codes.double(), block, dim=2)
    return torch.cat([p * s[:, :, i, None, None].double() for i, p in enumerate(parts)], dim=2)


def exact(case, seed):
    kind, block, fmt = case["kind"], case["block"], case["fmt"]
    st = prepare(case, seed)
    if kind == "write":
        return _exact_write(st, case["first"], block, fmt)
    if kind == "trip":
        made = [_exact_codes(st[k], block, fmt) for k in ("K", "V")]
        vals = [_exact_values(c, s, block).transpose(1, 2).contiguous() for c, s in made]
        return tuple(vals) + tuple(s for _, s in made)
    if kind == "read":
        return tuple(_exact_values(st[c], st[s], block).transpose(1, 2).contiguous()
                     for c, s in (("Kc", "ks"), ("Vc", "vs")))
    cache = tuple(st[k] for k in ("Kc", "Vc", "ks", "vs"))
    if kind == "step":
        cache = _exact_write(st, st["first"], block, fmt)
    Kc, Vc, ks, vs = cache
    n, Hkv, S, d = Kc.shape
    Tq, Hq, G = case["Tq"], case["Hq"], case["G"]
    group = Hq // Hkv
    weight = torch.ones((Tq, n * S + G + Tq), dtype=torch.float64, device="cuda")
    if st["live"] is not None:
        for i, most in enumerate(st["live"].tolist()):
            weight[:, i * S + most:(i + 1) * S] = 0
    weight[:, n * S + G:] = st["sees"].double() if kind == "tree" else \
        torch.ones((Tq, Tq), dtype=torch.float64, device="cuda").tril()
    o = torch.empty((Tq, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((Hq, Tq), dtype=torch.float64, device="cuda")
    for g in range(Hkv):
        K, V = (torch.cat([_exact_values(c[:, g:g + 1], s[:, g:g + 1], block).reshape(n * S, d),
                           more[:, g].double()])
                for c, s, more in ((Kc, ks, st["Kg"]), (Vc, vs, st["Vg"])))
        for h in range(g * group, (g + 1) * group):
            x = (st["q"][:, h].double() @ K.t().contiguous()) / math.sqrt(d) + torch.log(weight)
            lse[h] = torch.logsumexp(x, 1)
            o[:, h] = torch.exp(x - lse[h][:, None]) @ V
    return (cache if kind == "step" else ()) + (o, lse)
