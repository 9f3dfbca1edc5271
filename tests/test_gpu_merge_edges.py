"""lse_merge of partial outputs near the largest numbers: an average of them is no larger than
they are, whatever their sum."""
import pytest
import torch

import paper_2607_20457_amd as P

pytestmark = pytest.mark.gpu


def _parts(seed, H, Tq, Hq, d):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    o = torch.rand((H, Tq, Hq, d), generator=gen, device="cuda") + 0.9
    lse = 3 * torch.randn((H, Hq, Tq), generator=gen, device="cuda")
    return o, lse


# few parts and many outputs (a thread for each output), and a workgroup for each row
SIZES = [(2, 3, 4, 64), (3, 1, 2, 128), (7, 5, 8, 128), (9, 600, 16, 128), (9, 1, 8, 64),
         (33, 4, 32, 128), (70, 2, 8, 64), (129, 1, 32, 128), (513, 1, 2, 64), (65, 1, 4, 260),
         (33, 1, 4, 4)]


@pytest.mark.parametrize("H,Tq,Hq,d", SIZES)
def test_merge_near_the_largest(H, Tq, Hq, d):
    o, lse = _parts(1, H, Tq, Hq, d)
    o[:, :, 0, 1::3] *= -1
    o[:, :, -1, ::2] *= 2.0 ** -30     # (channels of ordinary size beside large ones)
    small, ell = P.lse_merge(o, lse)
    # 1.9 * 2^126: two of them leave fp32.  Powers of two change no rounding.
    for e in (40, 92, 110, 126):
        big, same = P.lse_merge(o * 2.0 ** e, lse)
        assert torch.isfinite(big).all(), e
        assert torch.equal(big, small * 2.0 ** e) and torch.equal(same, ell), e


@pytest.mark.parametrize("H,Tq,Hq,d", SIZES)
def test_merge_near_the_largest_beside_what_is_missing(H, Tq, Hq, d):
    # parts that saw nothing, whatever they hold, and a part that is no number
    o, lse = _parts(2, H, Tq, Hq, d)
    lse[0, :, 0] = -torch.inf
    small, ell = P.lse_merge(o, lse)
    o *= 2.0 ** 126
    for x in (torch.nan, torch.inf, 3e38):
        o[0, 0] = x
        big, same = P.lse_merge(o, lse)
        assert torch.equal(big, small * 2.0 ** 126) and torch.equal(same, ell), x
    o[-1, -1, 0, 2] = -torch.inf
    big, same = P.lse_merge(o, lse)
    assert torch.equal(same, ell) and torch.isneginf(big[-1, 0, 2])
    o[-1, -1, 0, 2] = torch.nan
    big, same = P.lse_merge(o, lse)
    assert torch.equal(same, ell) and torch.isnan(big[-1, 0, 2])
    big[-1, 0, 2] = 0
    small[-1, 0, 2] = 0
    assert torch.equal(big, small * 2.0 ** 126)


@pytest.mark.parametrize("H,Tq,Hq,d", SIZES)
def test_merge_of_parts_that_are_all_no_number(H, Tq, Hq, d):
    # (not a row that saw no key: a merge of its result would leave it out)
    o, lse = _parts(3, H, Tq, Hq, d)
    small, ell = P.lse_merge(o, lse)
    lse[:, 0, 0] = torch.nan
    lse[:, Hq - 1, Tq - 1] = -torch.inf
    o[:, 0, 0] = torch.nan
    for some in (False, True):
        if some:  # one part that saw no key, or a key
            lse[0, 0, 0] = -torch.inf
        got, sums = P.lse_merge(o, lse)
        assert torch.isnan(got[0, 0]).all() and torch.isnan(sums[0, 0]), some
        assert (got[-1, -1] == 0).all() and torch.isneginf(sums[-1, -1])
        got[0, 0], sums[0, 0], got[-1, -1], sums[-1, -1] = (
            small[0, 0], ell[0, 0], small[-1, -1], ell[-1, -1])
        assert torch.equal(got, small) and torch.equal(sums, ell)
