"""Pins of the fp64 definitions behind the 8-bit codes, the norm and the gradient limit: hand-worked values, an independent
conversion, finite differences."""
import numpy as np
import pytest
import torch

from oracle import codes as oc


def test_values_of_bytes():
    v = oc.code_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6
    assert v[0x38] == 1.0 and v[0x3C] == 1.5 and v[0x7E] == 448.0 and v[0xFE] == -448.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF])
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, t, equal_nan=True)


def test_nearest_codes_against_an_independent_conversion_and_on_ties():
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.standard_normal(20000) * 30, rng.standard_normal(20000) * 0.01, [448.0, -448.0, 0.0]])
    v = np.clip(v.astype(np.float32).astype(np.float64), -448, 448)
    mags = oc.code_values()[:0x7F]
    ties = (mags[:-1] + mags[1:]) / 2
    v = np.concatenate([v, ties, -ties])
    want = torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = oc.nearest_codes(v)
    assert np.array_equal(oc.code_values()[got], oc.code_values()[want])
    assert oc.nearest_codes(np.array([17.0]))[0] == oc.nearest_codes(np.array([16.0]))[0]          # 16, 18: even fraction
    assert oc.nearest_codes(np.array([19.0]))[0] == oc.nearest_codes(np.array([20.0]))[0]
    assert list(oc.nearest_codes(np.array([np.inf, -np.inf, np.nan]))) == [0x7F] * 3


@pytest.mark.parametrize("a,e", [(448.0, 0), (448.1, 1), (224.0, -1), (224.1, 0), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, 0),
                                 (2.0 ** -140, -127), (448.0 * 2.0 ** -127, -127), (2.0 ** 127, 119), (1.99 * 2.0 ** 127, 120)])
def test_exponents(a, e):
    assert oc.exponent(a) == e


def test_norm_gradients_against_differences():
    rng = np.random.default_rng(2)
    u, dy, gain = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7)
    eps, h = 1e-3, 1e-6
    _, inv = oc.rms_norm(u, gain, eps)
    du, dg = oc.rms_norm_backward(dy, u, gain, inv)
    risk = lambda a, b: float((oc.rms_norm(a, b, eps)[0] * dy).sum())  # noqa: E731
    for i in range(3):
        for j in range(7):
            d = np.zeros_like(u)
            d[i, j] = h
            assert abs((risk(u + d, gain) - risk(u - d, gain)) / (2 * h) - du[i, j]) < 1e-8
    for j in range(7):
        d = np.zeros(7)
        d[j] = h
        assert abs((risk(u, gain + d) - risk(u, gain - d)) / (2 * h) - dg[j]) < 1e-8


def test_limit():
    g = [np.array([3.0]), np.array([[4.0]])]
    assert oc.limit(g, 5.0) == (5.0, 1.0) and oc.limit(g, 1.0) == (5.0, 0.2) and oc.limit([np.zeros(3)], 0.0) == (0.0, 1.0)
