"""1 / rms is rounded once: with elements whose squares' sums are exact (small integers, widths of a power of two) it is the number of fp32
next to the fp64 value, the fp32 output is off by two roundings more, and codes are within half a step of a code of that."""
import numpy as np
import pytest
import torch

from codes_common import assert_within, code_buffers, f64
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb

pytestmark = pytest.mark.gpu

# Half a step, 2^-24 relative to a power of two, and what the Newton step's terms of second order leave, below 2^-40; two products more.
ONCE = 2.0 ** -24 * (1 + 2.0 ** -16)
THRICE = 3 * ONCE


def _integers(n, w, dtype, seed):
    x = torch.randint(-15, 16, (n, w), generator=torch.Generator().manual_seed(seed)).to(dtype)
    x[:, 0] = torch.arange(n) % 15 + 1                                # no row of zeros
    return x.cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,w", [(4000, 4), (4000, 64), (2000, 256), (2000, 512), (700, 2048), (300, 8192)])
def test_the_root_is_rounded_once(dtype, n, w):
    x = _integers(n, w, dtype, w)
    gain = (torch.rand(w, generator=torch.Generator().manual_seed(1)) + 0.5).cuda()
    inv, y = torch.empty(n, device="cuda"), torch.empty_like(x)
    codes, scales = code_buffers(n, w)
    vb.rms_norm_fwd(x, gain, 0.0, y=y, codes=codes, scales=scales, inv_rms=inv)
    want, want_inv = oc.rms_norm(f64(x), f64(gain), 0.0)
    assert_within(f64(inv), want_inv, ONCE * want_inv, "inv_rms")
    if dtype == torch.float32:
        assert_within(f64(y), want, THRICE * np.abs(want), "y")
    c, e = codes.cpu().numpy()[:, :w], scales.cpu().numpy().astype(np.int64)[:, :-(-w // 128)] - 127
    s = np.repeat(2.0 ** e, 128, axis=1)[:, :w]
    off = np.abs(oc.values(c, e) - want)
    # half a step of a code: 2^-4 of its power of two, or 2^-10 of the scale
    half = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 1e-30) / s)) - 4), 2.0 ** -10) * s
    assert (off <= half + THRICE * np.abs(want)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("w,eps", [(47, 1e-5), (300, 1e-5), (777, 0.0), (1000, 1e-5), (3000, 1e-5)])
def test_roots_of_any_rows(dtype, w, eps):
    """A lane adds at most 32 squares in fp32, k of them before the k-th rounding: 16.5 roundings of its own sum at most; the root halves them. The
    lanes' sums, the mean and eps are added in fp64 and the root is rounded once. The mean over rows is far less: a lane's roundings are 0.43 2^-24 of
    where they occur and independent, (1 + 4 + .. + 64) / 64 = 3.2 of them by squares for 8 elements (32: 10.7), a sixth of that or less over the lanes
    of 47 columns (a sixty-fourth for 2,048): below 0.2 2^-24 for the root."""
    x = (torch.randn(3000, w, generator=torch.Generator().manual_seed(w)) * 2.0).to(dtype).cuda()
    inv = torch.empty(3000, device="cuda")
    vb.rms_norm_fwd(x, None, eps, inv_rms=inv)
    _, want = oc.rms_norm(f64(x), 1.0, float(np.float32(eps)))
    rel = f64(inv) / want - 1.0
    assert np.abs(rel).max() <= 16.5 / 2 * 2.0 ** -24 + ONCE
    once = want.astype(np.float32).astype(np.float64) / want - 1.0
    assert np.sqrt((rel ** 2).mean()) <= np.sqrt((once ** 2).mean() + (0.2 * 2.0 ** -24) ** 2)


def test_gains_that_are_not_finite():
    x = torch.tensor([[1.0, 2.0, 0.0, -4.0], [3.0, 3.0, 3.0, 3.0]], device="cuda")
    gain = torch.tensor([float("inf"), float("-inf"), float("inf"), float("nan")], device="cuda")
    y = torch.empty_like(x)
    vb.rms_norm_fwd(x, gain, 0.0, y=y)
    got = f64(y)
    assert got[0, 0] == np.inf and got[0, 1] == -np.inf and np.isnan(got[0, 2]) and np.isnan(got[:, 3]).all()
    assert got[1, 0] == np.inf and got[1, 1] == -np.inf and got[1, 2] == np.inf
