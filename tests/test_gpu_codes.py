"""Rows and weights as 8-bit codes, through the C ABI: bit for bit the fp64 definition, which on fp32 and bf16 inputs is exact."""
import numpy as np
import pytest
import torch

from codes_common import assert_codes, code_buffers, f64, strided
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


def _rows(n, w, dtype, seed):
    """Rows of very different size, blocks of zeros, limits of the type, codes' ties."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, w)) * np.exp(rng.standard_normal((n, 1)) * 8)
    x[rng.random((n, w)) < 0.1] = 0.0
    if n > 3:
        x[1] = 0.0
        x[2, : w // 2] = rng.integers(-40, 40, w // 2)               # ties of the codes
        x[3] = rng.standard_normal(w) * 2.0 ** -138                    # below the smallest normal number
    return torch.from_numpy(x).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,w", [(1, 1), (1, 128), (5, 47), (7, 129), (33, 256), (300, 100), (19, 511), (4, 513), (3, 2047), (2, 16384)])
def test_rows(dtype, n, w):
    x = _rows(n, w, dtype, n * 10007 + w)
    codes, scales = code_buffers(n, w)
    vb.quantize_rows(x, codes, scales)
    assert_codes(codes, scales, *oc.quantize_rows(f64(x)), w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,w", [(64, 47), (31, 256), (9, 333)])
def test_gated_rows_in_wider_memory(dtype, n, w):
    x, g = _rows(n, w, dtype, 5), _rows(n, w, dtype, 6)
    g[0, 0] = float("nan")                                            # not above zero
    g[-1] = 0.0                                                       # a row that nothing passes
    xs, _ = strided(x, 5, 1)
    gs, _ = strided(g, 2, 3)
    codes, scales = code_buffers(n, w)
    vb.quantize_rows(xs, codes, scales, gate=gs)
    assert_codes(codes, scales, *oc.quantize_rows(np.where(f64(g) > 0, f64(x), 0.0)), w)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_stays_where_it_is(dtype):
    x = _rows(6, 300, dtype, 8)
    x[0, 5], x[0, 200], x[4, 299] = float("inf"), float("nan"), float("-inf")
    x[5, :128] = float("nan")                                         # a block without a finite number
    codes, scales = code_buffers(6, 300)
    vb.quantize_rows(x, codes, scales)
    assert_codes(codes, scales, *oc.quantize_rows(f64(x)), 300)


def test_largest_and_smallest_numbers():
    top = torch.finfo(torch.float32).max
    x = torch.zeros(4, 128)
    x[0, :3] = torch.tensor([top, -top / 2, top / 1000])
    x[1, :3] = torch.tensor([2.0 ** -149, -2.0 ** -140, 2.0 ** -126])
    x[2, :3] = torch.tensor([448.0 * 2.0 ** -127, 2.0 ** -136, 2.0 ** -137])
    x[3, :2] = torch.tensor([448.0, np.nextafter(np.float32(448.0), np.float32(1e9)).item()])
    codes, scales = code_buffers(4, 128)
    vb.quantize_rows(x.cuda(), codes, scales)
    assert_codes(codes, scales, *oc.quantize_rows(f64(x)), 128)


@pytest.mark.parametrize("n_in,n_out", [(1, 1), (128, 128), (100, 47), (257, 129), (512, 40), (16, 600), (300, 1030)])
@pytest.mark.parametrize("both", ["turned", "codes", "both"])
def test_weights(n_in, n_out, both):
    rng = np.random.default_rng(n_in + n_out)
    h = rng.standard_normal((n_in, n_out)).astype(np.float32)
    h[:, 0] *= 1000.0
    if n_in > 1:
        h[-1, -1] = np.inf
    ht, _ = strided(torch.from_numpy(h).cuda(), 1, 1)
    turned, turned_scales = code_buffers(n_out, n_in, -(-n_out // 128)) if both != "codes" else (None, None)
    codes, scales = code_buffers(n_in, n_out, -(-n_in // 128)) if both != "turned" else (None, None)
    vb.quantize_weights(ht, turned, turned_scales, codes, scales)
    want, exps = oc.quantize_weights(h.astype(np.float64))
    if codes is not None:
        assert_codes(codes, scales, want, exps, n_out)
    if turned is not None:
        assert_codes(turned, turned_scales, want.T, exps.T, n_in)


def test_rows_without_rows():
    codes, scales = code_buffers(0, 64)
    vb.quantize_rows(torch.empty((0, 64), device="cuda"), codes, scales)
