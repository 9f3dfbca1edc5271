"""Pins of the oracle of a cache held in 8 bits (runs without a GPU)."""
import numpy as np
import pytest
import torch

from oracle import quant as oq


def test_e4m3_values_are_the_formats():
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oq.e4m3_values(), want)
    assert want[-1] == 448 and want[1] == 2.0 ** -9


def test_nearest_e4m3_is_the_rounding_of_a_cast():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(20000) * 100, rng.standard_normal(20000) * 0.01,
                        # ties between neighbouring codes, and values next to them
                        (oq.e4m3_values()[1:] + oq.e4m3_values()[:-1]) / 2])
    x = np.clip(x.astype(np.float32), -448, 448)
    x = np.concatenate([x, -x, np.nextafter(x, np.float32(0))])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oq.nearest(x.astype(np.float64), "e4m3"), want)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scale_is_the_least_power_of_two(fmt):
    most = oq.MOST[fmt]
    assert oq.scale_exponent(0.0, fmt) == -100
    assert oq.scale_exponent(most * 2.0 ** -100, fmt) == -100
    for e in (-99, -3, 0, 7, 60):
        assert oq.scale_exponent(most * 2.0 ** e, fmt) == e
        assert oq.scale_exponent(np.nextafter(most * 2.0 ** e, np.inf), fmt) == e + 1


@pytest.mark.parametrize("fmt,step", [("e4m3", None), ("int8", 1.0)])
def test_values_are_within_half_a_step(fmt, step):
    rng = np.random.default_rng(2)
    X = rng.standard_normal((2, 37, 3, 8)) * np.exp(rng.standard_normal((1, 1, 3, 8)))
    codes, scales = oq.quantize(X, 16, fmt)
    back = oq.values(codes, scales, 16)
    s = np.swapaxes(np.repeat(scales, 16, axis=2)[:, :, :37, None], 1, 2)
    # e4m3: eight steps to a binade from 2^-6 on, the same steps below it
    size = np.maximum(np.abs(X / s), 2.0 ** -6)
    half = 0.5 * step if step else 0.5 * 2.0 ** (np.floor(np.log2(size)) - 3)
    assert np.all(np.abs(back - X) <= half * s)
    # quantising what was read back changes nothing
    again, scales2 = oq.quantize(back, 16, fmt)
    assert np.array_equal(oq.values(again, scales2, 16), back)


def test_blocks_that_are_not_finite():
    X = np.ones((1, 40, 2, 4))
    X[0, 17, 1, 2], X[0, 39, 0, 0] = np.nan, -np.inf
    codes, scales = oq.quantize(X, 16, "e4m3")
    assert np.isnan(scales[0]).tolist() == [[False, False, True], [False, True, False]]
    assert (codes[0, 1, 16:32] == 0).all() and (codes[0, 0, 32:] == 0).all()
    assert np.isnan(oq.values(codes, scales, 16)[0, 16:32, 1]).all()
