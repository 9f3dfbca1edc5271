"""phase2_quant at its edges, in every shape of tile: scales, values and scores of extreme
size, what is not finite, and what must not be seen."""
import math

import numpy as np
import pytest
import torch

import paper_2607_20457_amd as P
from tests._blocks import host
from tests._plan import plan

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
