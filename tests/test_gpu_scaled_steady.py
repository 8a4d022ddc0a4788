"""Short reductions over so many rows that every workgroup goes through its ring of buffers and beyond, where it waits by a count of
the copies and stores that may still be under way. Every result is compared with fp64; bounds as in test_gpu_scaled_products.py."""
import numpy as np
import pytest
import torch

from codes_common import STEP, f64, upload_codes
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb
from test_gpu_scaled_products import _coded, _dropped_few, _weights

pytestmark = pytest.mark.gpu

PERIOD = 211


def _ring(dtype, n, n_in, n_out):
    """(buffers, steps of a workgroup) that the launch for these sizes has: sizes of the ring and of the grid in kernels_scaled.hip."""
    half = dtype == torch.bfloat16
    kb = -(-n_in // 128)
    wn = 1 if n_out <= 64 else 2 if n_out <= 128 else 4
    r, ni = 2 if wn == 4 else 1, 2 if not half and kb > 2 else 4
    rows = 16 * r * (4 // wn)
    size = kb * rows * 128 + 1024
    depth = 3 if size > 24 * 1024 else 4
    resident = max(1, min(3 if kb <= 2 and half else 2, 160 * 1024 // (depth * size)))
    columns, steps = -(-n_out // (16 * ni * wn)), -(-n // rows)
    groups = min(steps, max(8, 256 * resident // columns // 8 * 8))
    return depth, steps // groups


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,n_in,n_out", [
    (169343, 256, 256), (60001, 512, 512), (130003, 512, 47), (130003, 512, 64), (170003, 384, 64), (110003, 384, 128), (65003, 384, 320),
    (110003, 512, 128), (310003, 128, 64), (310003, 100, 47), (310003, 200, 64), (160003, 128, 128), (160003, 200, 100), (170003, 128, 256)])
@pytest.mark.parametrize("gap,act", [(0, vb.ACT_RELU), (3, vb.ACT_IDENTITY)])
def test_steps_beyond_the_ring(dtype, n, n_in, n_out, gap, act):
    """Rows repeat with a period that no step's count of rows divides, so that a buffer read too early holds other rows. gap 0: rows of
    whole cache lines where n_out allows it."""
    depth, steps = _ring(dtype, n, n_in, n_out)
    assert steps >= depth + 2, (depth, steps)
    codes, exps = _coded(PERIOD, n_in, n)
    w, turned, _ = _weights(n_in, n_out, n_out)
    x = oc.values(codes, exps)
    want, size = x @ w, np.abs(x) @ np.abs(w)
    if act == vb.ACT_RELU:
        want = np.maximum(want, 0.0)
    sums = n_in * 2.0 ** -24 * size + _dropped_few(dtype, x, w)
    bound = torch.from_numpy(sums + STEP[dtype] * (np.abs(want) + sums) + 1e-38).cuda()
    want = torch.from_numpy(want).cuda()
    at = torch.arange(n, device="cuda") % PERIOD
    x8, s8 = (t[at].contiguous() for t in upload_codes(codes, exps, n_in))
    flat = torch.full((n, n_out + gap), float("nan"), dtype=dtype, device="cuda")
    c = flat[:, :n_out]
    vb.scaled_transform(x8, s8, *turned, n_in, c, act=act)
    first = c[:PERIOD].clone()
    for r0 in range(0, n, 1 << 16):
        rows = at[r0:r0 + (1 << 16)]
        got = c[r0:r0 + (1 << 16)]
        assert bool(((got.double() - want[rows]).abs() <= bound[rows]).all()), r0
        assert torch.equal(got, first[rows]), r0                       # one order of sums: equal rows give equal bits
    assert bool(torch.isnan(flat[:, n_out:]).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,n_in,n_out", [(169343, 256, 256), (60001, 512, 512), (130003, 512, 47)])
def test_added_to_beyond_the_ring(dtype, n, n_in, n_out):
    """The form that also loads what c holds."""
    depth, steps = _ring(dtype, n, n_in, n_out)
    assert steps >= depth + 2, (depth, steps)
    codes, exps = _coded(PERIOD, n_in, n)
    w, turned, _ = _weights(n_in, n_out, n_out)
    x = oc.values(codes, exps)
    start = torch.randn(PERIOD, n_out, generator=torch.Generator().manual_seed(1)).to(dtype)
    want, size = f64(start) + x @ w, np.abs(f64(start)) + np.abs(x) @ np.abs(w)
    sums = (n_in + 1) * 2.0 ** -24 * size + _dropped_few(dtype, x, w)
    bound = torch.from_numpy(sums + STEP[dtype] * (np.abs(want) + sums) + 1e-38).cuda()
    want = torch.from_numpy(want).cuda()
    at = torch.arange(n, device="cuda") % PERIOD
    x8, s8 = (t[at].contiguous() for t in upload_codes(codes, exps, n_in))
    c = start.cuda()[at].contiguous()
    vb.scaled_transform(x8, s8, *turned, n_in, c, accumulate=True)
    for r0 in range(0, n, 1 << 16):
        rows = at[r0:r0 + (1 << 16)]
        assert bool(((c[r0:r0 + (1 << 16)].double() - want[rows]).abs() <= bound[rows]).all()), r0
