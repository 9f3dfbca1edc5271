"""Helpers of the tests of a cache held in 8 bits."""
import math

import numpy as np
import torch

from oracle import blocks as ob
from oracle import quant as oq
from tests import _blocks
from tests._blocks import host, normal
from tests._helpers import f64, to_dev_bf16

DTYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def spread(seed, shape):
    """bf16 bits [n, rows, H, d] of normal values whose channels and blocks differ in size."""
    rng = np.random.default_rng(seed)
    x = f64(normal(seed, shape)) * np.exp(rng.standard_normal((1, 1) + tuple(shape[2:])))
    x *= 2.0 ** rng.integers(-3, 4, (shape[0], -(-shape[1] // 16), shape[2], 1)
                             ).repeat(16, axis=1)[:, :shape[1]]
    return torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def codes_of(t):
    """The values of a tensor of codes, as the format has them."""
    return t.cpu().double().numpy()


def dev_codes(codes, fmt):
    """Codes (values) on the device."""
    return torch.from_numpy(np.asarray(codes, dtype=np.float32)).to(DTYPES[fmt]).cuda()


def dev_cache(k, v, block, fmt):
    """The cache of bf16 bits k and v [n, rows, H, d], made by the oracle:
    (Kc, Vc, k_scale, v_scale) and the values of K and V that it stands for."""
    made = [oq.quantize(f64(x), block, fmt) for x in (k, v)]
    vals = [oq.values(c, s, block) for c, s in made]
    codes = [dev_codes(c, fmt) for c, _ in made]
    scales = [torch.from_numpy(s).float().cuda() for _, s in made]
    return (*codes, *scales), vals


def _seen(q, K, V, rows, kg, vg, G, sees):
    """The keys and values that are live, one after another, and how often each token sees
    them [Tq, 1, keys]."""
    n, S, Hkv, d = K.shape
    Tq = q.shape[0]
    live = np.full(n, S) if rows is None else np.clip(np.asarray(rows), 0, S).astype(int)
    Ks = [K[i, :live[i]] for i in range(n)]
    Vs = [V[i, :live[i]] for i in range(n)]
    counts = np.ones((Tq, 1, int(live.sum())))
    if kg is not None:
        gen = np.ones((Tq, 1, G + Tq))
        gen[:, 0, G:] = np.tri(Tq) if sees is None else sees
        counts = np.concatenate([counts, gen], axis=2)
        Ks.append(f64(kg))
        Vs.append(f64(vg))
    K, V = (np.concatenate(x) if x else np.zeros((0, Hkv, d)) for x in (Ks, Vs))
    return K, V, counts


def reference(q, K, V, rows, kg, vg, G, sees, scale):
    """The oracle's phase2_quant: q bf16 bits, K and V [n, S, Hkv, d] the values of the codes,
    rows the live ones of each shard (None: all), kg and vg bf16 bits or None, sees None is
    causal -> what tests._blocks.check takes, and the number of keys."""
    K, V, counts = _seen(q, K, V, rows, kg, vg, G, sees)
    return ob.counted_attention(f64(q), K, V, counts, scale), counts.shape[2]


def long_reference(q, cache, block, rows, kg, vg, G, sees, scale):
    """`reference` of a cache on the device by matrix products in fp64 there, a KV head at a
    time, for long shards."""
    Kc, Vc, ks, vs = cache
    n, Hkv, S, d = Kc.shape
    Tq, Hq = q.shape[:2]
    group = Hq // Hkv
    live = np.full(n, S) if rows is None else np.clip(np.asarray(rows), 0, S).astype(int)
    x = torch.from_numpy(f64(q)).cuda()
    dead = torch.zeros((Tq, int(live.sum()) + (0 if kg is None else G + Tq)), dtype=torch.bool,
                       device="cuda")
    if kg is not None:
        see = np.tri(Tq) if sees is None else np.asarray(sees)
        dead[:, dead.shape[1] - Tq:] = torch.from_numpy(see == 0).cuda()
    dead = torch.repeat_interleave(dead, group, dim=0)
    o, size = (torch.zeros((Tq, Hq, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse, most = torch.zeros((Hq, Tq), dtype=torch.float64, device="cuda"), 0.0
    for g in range(Hkv):
        both = []
        for codes, scales, more in ((Kc, ks, kg), (Vc, vs, vg)):
            s = torch.repeat_interleave(scales[:, g].double(), block, dim=1)[:, :S, None]
            v = codes[:, g].double() * s
            v = [v[i, :live[i]] for i in range(n)]
            if more is not None:
                v.append(torch.from_numpy(f64(more[:, g])).cuda())
            both.append(torch.cat(v))
        k, v = both[0].t().contiguous(), both[1]
        y = x[:, g * group:(g + 1) * group].reshape(Tq * group, d)
        s = ((y @ k) * scale).masked_fill_(dead, -np.inf)
        most = max(most, float((y.abs() @ k.abs()).masked_fill_(dead, 0).max()) * scale)
        ell = torch.logsumexp(s, dim=1)
        p = torch.exp_(s - ell[:, None])
        for out, w in ((o, v), (size, v.abs())):
            out[:, g * group:(g + 1) * group] = (p @ w).view(Tq, group, d)
        lse[g * group:(g + 1) * group] = ell.view(Tq, group).t()
    return (o.cpu().numpy(), lse.cpu().numpy(), size.cpu().numpy(), most), dead.shape[1]


def check(o, lse, ref, keys, what, bf16_out=False):
    """tests._blocks.check, and what weights below fp32's smallest normal number, 2^-126,
    lose.  Codes may be exactly 0 where the weight is, so that such keys are all that an
    output is made of.  A weight is taken against a reference no larger than the row's
    largest score, so the largest weight is 1 or more and divides the sum; one that is lost,
    alone or times its V scale, takes at most 2^-126 of a code of 448 with it (of a bf16
    value, 2^-126 of at most 448 too in these tests), in a wave's sum, in the merge of the
    waves and in that of the parts: less than 4 * 448 * 2^-126 a key."""
    lost = keys * 4 * 448 * 2.0 ** -126
    o_ref, lse_ref, size, most = ref
    _blocks.check(o, lse, (o_ref, lse_ref, size + 2.0 ** 7 * lost, most), keys, what, bf16_out)


def softmax_scale(d):
    return 1.0 / math.sqrt(d)


__all__ = ["DTYPES", "spread", "codes_of", "dev_codes", "dev_cache", "reference", "long_reference", "check", "host",
           "normal", "f64", "to_dev_bf16", "softmax_scale", "oq"]
