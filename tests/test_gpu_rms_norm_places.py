"""Rows of the norm's inputs and outputs side by side in one matrix, and behind one another: what is not an overlap is served, and what lies
around is left alone."""
import pytest
import torch

from codes_common import assert_within, code_buffers, f64
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,w", [(1, 100), (7, 47), (300, 256), (40, 2500)])
def test_columns_of_one_matrix(dtype, n, w):
    g = torch.Generator().manual_seed(n)
    wide = torch.randn(n, 5 * w, generator=g).to(dtype).cuda()
    x, r, total, y, dx = (wide[:, k * w:(k + 1) * w] for k in range(5))
    gain, inv = torch.rand(w, generator=g).cuda(), torch.empty(n, device="cuda")
    apart = [t.clone() for t in (x, r)]
    want_total, want_y, want_dx, want_inv = torch.empty_like(apart[0]), torch.empty_like(apart[0]), torch.empty_like(apart[0]), torch.empty_like(inv)
    vb.rms_norm_fwd(*apart[:1], gain, EPS, residual=apart[1], total=want_total, y=want_y, inv_rms=want_inv)
    vb.rms_norm_bwd(want_y, want_total, gain, want_inv, want_dx)
    vb.rms_norm_fwd(x, gain, EPS, residual=r, total=total, y=y, inv_rms=inv)
    vb.rms_norm_bwd(y, total, gain, inv, dx)
    for got, want in zip((x, r, total, y, dx, inv), (*apart, want_total, want_y, want_dx, want_inv)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("n,w", [(1, 100), (6, 64)])
def test_rows_behind_one_another_and_over_one_another(n, w):
    flat = torch.randn(3 * n * w, generator=torch.Generator().manual_seed(1)).cuda()
    x, y = flat[:n * w].view(n, w), flat[n * w:2 * n * w].view(n, w)
    codes, scales = code_buffers(n, w)
    vb.rms_norm_fwd(x, None, EPS, y=y, codes=codes, scales=scales)
    want, _ = oc.rms_norm(f64(x), 1.0, EPS)
    assert_within(f64(y), want, 52 * 2.0 ** -24 * abs(want), "y")         # (test_gpu_rms_norm.py derives it)
    keep = flat.clone()
    shifted = flat[1:n * w + 1].view(n, w)
    for call in (lambda: vb.rms_norm_fwd(x, None, EPS, y=shifted), lambda: vb.rms_norm_fwd(shifted, None, EPS, total=x),
                 lambda: vb.rms_norm_bwd(x, y, None, torch.ones(n, device="cuda"), shifted)):
        with pytest.raises(vb.VarcoError) as e:
            call()
        assert e.value.code == vb.ERR_INVALID_ARG
    assert torch.equal(flat, keep)
