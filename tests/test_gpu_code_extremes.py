"""Products of codes at both ends of the scales, 2^-127 and 2^120, far apart in a row, and with NaN codes, on the units of both result types.
Bounds as in test_gpu_scaled_products.py."""
import numpy as np
import pytest
import torch

from codes_common import STEP, assert_within, f64, upload_codes
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb
from test_gpu_scaled_products import _coded, _dropped, _weights

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
NUMBERS = np.array([b for b in range(256) if b & 0x7F != 0x7F], dtype=np.uint8)
LARGEST = 0x78                       # 256: what finite numbers above 1.94 2^127 become under the scale 2^120
ENDS = [-127, -126, -125, -124, -123, -118, 118, 119, 120]


def _under(e):
    """Codes that a scale of 2^e can have: at 2^120 what fp32 numbers become."""
    return NUMBERS[(NUMBERS & 0x7F) <= LARGEST] if e == 120 else NUMBERS


def _row(width, code, e):
    """One row whose first column is `code`, zeros behind it, one scale for all."""
    c = np.zeros((1, width), np.uint8)
    c[0, 0] = code
    return c, np.full((1, -(-width // 128)), e, np.int64)


def _taken(values):
    """What the products with fp32 results and the weight gradients take numbers for: as fp32 does, 2^128 for an infinity. What that takes part in
    is not finite: infinite, or NaN where a zero lies opposite, be it one of those behind the last row or column."""
    return np.where(np.abs(values) >= 2.0 ** 128, np.copysign(np.inf, values), values)


def _assert_equal_or_both_not_finite(got, want):
    finite = np.isfinite(want)
    assert np.array_equal(got[finite], want[finite]) and not np.isfinite(got[~finite]).any()


# Operands of the bf16 units below 2^-126 are multiples of 2^-133: numbers under scales from 2^-124 on (codes are multiples of 2^-9) are such, smaller
# ones off by half of that. Their products with a power of two are multiples of 2^-149 and are kept.
@pytest.mark.parametrize("e", ENDS)
@pytest.mark.parametrize("back", [0, 1])
def test_every_code_at_the_ends_of_the_scales(e, back):
    """All codes against a single power of two, 1 or one that brings the product into the middle of fp32's range."""
    codes = _under(e)
    other = min(max(-e, -110), 110) if back else 0
    one = _row(1, 0x38, other)
    value = oc.values(codes[None, :], np.full((1, -(-len(codes) // 128)), e, np.int64))[0]
    want = _taken(value) * 2.0 ** other
    lower = 2.0 ** -134 * 2.0 ** other if e < -124 else 0.0
    dh = torch.empty((len(codes), 1), device="cuda")
    y8 = upload_codes(codes[None, :], np.full((1, -(-len(codes) // 128)), e, np.int64), len(codes))
    vb.scaled_bwd_weight(*y8, *upload_codes(*one, 1), dh)
    c = torch.empty((len(codes), 1), device="cuda")
    vb.scaled_transform(*upload_codes(codes[:, None], np.full((len(codes), 1), e, np.int64), 1), *upload_codes(*one, 1), 1, c)
    turned = torch.empty((1, len(codes)), device="cuda")
    blocks = np.full((-(-len(codes) // 128), 1), e, np.int64)
    vb.scaled_transform(*upload_codes(*one, 1), *upload_codes(codes[:, None], blocks, 1), 1, turned)
    finite = np.isfinite(want)
    assert finite.all() == (e < 120)
    for got in (f64(dh)[:, 0], f64(c)[:, 0], f64(turned)[0]):
        assert_within(got[finite], want[finite], lower, e)
        assert not np.isfinite(got[~finite]).any()


@pytest.mark.parametrize("e", [119, 120])
@pytest.mark.parametrize("n_in", [100, 512, 700, 2048])
@pytest.mark.parametrize("dtype", TYPES)
def test_the_largest_numbers_and_zeros_opposite(dtype, e, n_in):
    """448 2^119 and 240 2^120 are numbers everywhere; 256 2^120 is one in products with bf16 results, and in the others no finite one."""
    largest = LARGEST if e == 120 else 0x7E
    xc, xe = _row(n_in, largest, e)
    x = np.repeat(xc, 4, axis=0)
    x[1, 0], x[2, 0], x[3, 0] = 0, largest | 0x80, 0x77
    xe = np.repeat(xe, 4, axis=0)
    wc = np.zeros((5, n_in), np.uint8)                                 # rows of weights are outputs
    wc[1, 0], wc[2, 0], wc[3, 1] = 0x38, 0xB0, 0x7E
    we = np.full((1, -(-n_in // 128)), -40, np.int64)
    X, W = oc.values(x, xe), oc.values(wc, np.repeat(we, 5, axis=0))
    if dtype == torch.float32:
        X = _taken(X)
    c = torch.empty((4, 5), dtype=dtype, device="cuda")
    vb.scaled_transform(*upload_codes(x, xe, n_in), *upload_codes(wc, we, n_in), n_in, c)
    with np.errstate(invalid="ignore"):
        _assert_equal_or_both_not_finite(f64(c), X @ W.T)
    if dtype == torch.bfloat16:
        return
    d, de = np.array([[0x38, 0], [0x7E, 0x30], [0, 0], [0x38, 0]], np.uint8), np.full((4, 1), -20, np.int64)
    dh = torch.empty((n_in, 2), device="cuda")
    vb.scaled_bwd_weight(*upload_codes(x, xe, n_in), *upload_codes(d, de, 2), dh)
    with np.errstate(invalid="ignore"):
        _assert_equal_or_both_not_finite(f64(dh), X.T @ oc.values(d, de))


@pytest.mark.parametrize("n", [1, 700, 9000])
@pytest.mark.parametrize("n_in,n_out", [(40, 3), (300, 100), (256, 256), (140, 513)])
def test_rows_behind_the_last_add_nothing_to_gradients(n, n_in, n_out):
    """The largest numbers in the last row, opposite errors of zero."""
    yc, ye = _coded(n, n_in, 51)
    yc[-1], ye[-1] = 0x7E, 119
    dc, de = _coded(n, n_out, 52)
    dc[-1], de[-1] = 0, 0
    y, d = oc.values(yc, ye), oc.values(dc, de)
    dh = torch.empty((n_in, n_out), device="cuda")
    vb.scaled_bwd_weight(*upload_codes(yc, ye, n_in), *upload_codes(dc, de, n_out), dh)
    assert_within(f64(dh), y.T @ d, n * 2.0 ** -24 * (np.abs(y[:-1].T) @ np.abs(d[:-1])) + 1e-38, "dh")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,n_in,n_out", [(20, 384, 20), (20, 1200, 70), (9000, 384, 64), (9000, 1200, 520), (8200, 768, 2048)])
def test_scales_far_apart_in_a_row(dtype, n, n_in, n_out):
    """Blocks of a row 2^120 apart, and the weights' against them."""
    rng = np.random.default_rng(7)
    period = 20
    v, h = rng.standard_normal((period, n_in)), rng.standard_normal((n_in, n_out))
    third = n_in // 384 * 128
    v[:, :third] *= 2.0 ** 60
    v[:, -third:] *= 2.0 ** -60
    h[:third] *= 2.0 ** -60
    h[-third:] *= 2.0 ** 60
    codes, exps = oc.quantize_rows(v)
    hc, he = oc.quantize_weights(h)
    x, w = oc.values(codes, exps), oc.weight_values(hc, he)
    at = np.arange(n) % period
    c = torch.empty((n, n_out), dtype=dtype, device="cuda")
    vb.scaled_transform(*upload_codes(codes[at], exps[at], n_in), *upload_codes(hc.T, he.T, n_in), n_in, c)
    sums = n_in * 2.0 ** -24 * (np.abs(x) @ np.abs(w)) + _dropped(dtype, x, w)
    assert_within(f64(c), (x @ w)[at], (sums + STEP[dtype] * (np.abs(x @ w) + sums))[at], "c")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", [vb.ACT_IDENTITY, vb.ACT_RELU])
@pytest.mark.parametrize("n,n_in,n_out", [(40, 200, 70), (40, 1000, 70), (5003, 1000, 300), (8200, 768, 2048)])
def test_nan_codes_reach_their_row_or_their_output(dtype, act, n, n_in, n_out):
    codes, exps = _coded(40, n_in, 8)
    at = np.arange(n) % 40
    codes, exps = codes[at], exps[at]
    codes[7, 150] = codes[n - 1, n_in - 1] = oc.NAN_CODE
    h = np.random.default_rng(9).standard_normal((n_in, n_out))
    h[3, 5] = np.nan
    hc, he = oc.quantize_weights(h)
    c = torch.empty((n, n_out), dtype=dtype, device="cuda")
    vb.scaled_transform(*upload_codes(codes, exps, n_in), *upload_codes(hc.T, he.T, n_in), n_in, c, act=act)
    bad = torch.isnan(c).cpu().numpy()
    assert bad[7].all() and bad[n - 1].all() and bad[:, 5].all()
    bad[[7, n - 1]] = False
    bad[:, 5] = False
    assert not bad.any()
