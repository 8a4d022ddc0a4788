"""The norm of rows whose squares come to the ends of fp32, as the header states it."""
import numpy as np
import pytest
import torch

from codes_common import assert_within, f64
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb

pytestmark = pytest.mark.gpu

INV = 48 * 2.0 ** -24           # test_gpu_rms_norm.py derives it


@pytest.mark.parametrize("w", [1, 47, 512, 3000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_and_large_rows_without_eps(dtype, w):
    """Squares between 2^-126 and 2^127 / w keep all bits; below 2^-149 they are none, beyond 2^128 infinite."""
    kept, gone, beyond = [2.0 ** -62, 2.0 ** -40, 2.0 ** 50], [2.0 ** -76, 2.0 ** -120], [2.0 ** 65, 2.0 ** 120]
    g = torch.Generator().manual_seed(w)
    x = (torch.rand(len(kept + gone + beyond), w, generator=g) * 0.49 + 1.0) * torch.tensor(kept + gone + beyond)[:, None]
    x = x.to(dtype).cuda()
    y, inv = torch.empty_like(x), torch.empty(x.shape[0], device="cuda")
    vb.rms_norm_fwd(x, None, 0.0, y=y, inv_rms=inv)
    want, want_inv = oc.rms_norm(f64(x), 1.0, 0.0)
    n, m = len(kept), len(gone)
    assert_within(f64(inv)[:n], want_inv[:n], INV * want_inv[:n], "inv_rms")
    assert_within(f64(y)[:n], want[:n], (INV + 3 * 2.0 ** -24 + (2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8)) * np.abs(want[:n]), "y")
    assert torch.isinf(inv[n:n + m]).all() and torch.isinf(y[n:n + m]).all()
    assert (inv[n + m:] == 0).all() and (y[n + m:] == 0).all()


def test_small_rows_beside_eps():
    """With eps as it is used the squares that vanish would not count."""
    x = (torch.randn(6, 300, generator=torch.Generator().manual_seed(1)) * torch.tensor([1e-3, 1e-6, 1e-12, 1e-19, 1e-25, 1e-38])[:, None]).cuda()
    y, inv = torch.empty_like(x), torch.empty(6, device="cuda")
    vb.rms_norm_fwd(x, None, 1e-5, y=y, inv_rms=inv)
    want, want_inv = oc.rms_norm(f64(x), 1.0, float(np.float32(1e-5)))
    assert_within(f64(inv), want_inv, INV * want_inv, "inv_rms")
    assert_within(f64(y), want, (INV + 4 * 2.0 ** -24) * np.abs(want) + 1e-38, "y")
