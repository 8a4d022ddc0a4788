"""Codes, products, norms and limited gradients at the largest widths and counts that fit a test: many outputs, many rows of few columns, tensors of more
than 2^31 elements. Bounds as in the files of each call; sums over more rows than a test can add in fp64 by torch's fp64 product."""
import numpy as np
import pytest
import torch

from codes_common import STEP, assert_within, code_buffers, f64, upload_codes
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb
from test_gpu_scaled_products import _coded, _dropped_few

pytestmark = pytest.mark.gpu

WIDEST = vb.MAX_CODE_WIDTH


def _weights_with_few_different_columns(n_in, n_out, period, seed):
    """Values [n_in, period] and device buffers of n_out outputs that repeat them."""
    rng = np.random.default_rng(seed)
    codes, exps = oc.quantize_rows(rng.standard_normal((period, n_in)))
    exps[:] = exps.max(axis=0)                                         # (a scale for 128 outputs)
    at = np.arange(n_out) % period
    return oc.values(codes, exps), at, upload_codes(codes[at], np.repeat(exps[:1], -(-n_out // 128), axis=0), n_in)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,n_in,n_out", [(3, WIDEST, WIDEST), (300, 700, WIDEST), (700, 128, WIDEST), (2100, 512, WIDEST - 1), (5000, 640, 16001), (300, WIDEST, 300)])
def test_many_outputs(dtype, n, n_in, n_out):
    period = 37
    codes, exps = _coded(min(n, 53), n_in, n)
    rows = np.arange(n) % len(codes)
    w, at, w8 = _weights_with_few_different_columns(n_in, n_out, period, n_out)
    x = oc.values(codes, exps)
    want, size = x @ w.T, np.abs(x) @ np.abs(w.T)
    sums = n_in * 2.0 ** -24 * size + _dropped_few(dtype, x, w.T)
    bound = sums + STEP[dtype] * (np.abs(want) + sums) + 1e-38
    c = torch.full((n, n_out), float("nan"), dtype=dtype, device="cuda")
    vb.scaled_transform(*upload_codes(codes[rows], exps[rows], n_in), *w8, n_in, c)
    want, bound = (torch.from_numpy(t[rows][:, at]).cuda() for t in (want, bound))
    assert bool(((c.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("n,n_in,n_out", [(40, WIDEST, WIDEST), (3000, WIDEST, 70), (3000, 50, WIDEST), (70_001, WIDEST, 16), (1, WIDEST, 1000)])
def test_gradients_of_wide_weights(n, n_in, n_out):
    yc, ye = _coded(min(n, 61), n_in, 1)
    dc, de = _coded(min(n, 61), n_out, 2)
    rows = np.arange(n) % len(yc)
    count = np.bincount(rows, minlength=len(yc))[:, None]
    y, d = (torch.from_numpy(t).cuda() for t in (oc.values(yc, ye), oc.values(dc, de) * count))
    (y8, ys), (d8, ds) = upload_codes(yc, ye, n_in), upload_codes(dc, de, n_out)
    at = torch.from_numpy(rows).cuda()
    dh = torch.full((n_in, n_out), float("nan"), device="cuda")
    vb.scaled_bwd_weight(y8[at].contiguous(), ys[at].contiguous(), d8[at].contiguous(), ds[at].contiguous(), dh)
    for i in range(0, n_in, 2048):
        part = y[:, i:i + 2048].t().contiguous()
        want, size = torch.mm(part, d), torch.mm(part.abs(), d.abs())
        assert bool(((dh[i:i + 2048].double() - want).abs() <= n * 2.0 ** -24 * size + 1e-38).all())


@pytest.mark.parametrize("n_in,n_out", [(WIDEST, 300), (300, WIDEST), (5000, 5000)])
def test_codes_of_wide_weights(n_in, n_out):
    g = torch.Generator().manual_seed(3)
    small = torch.randn(256, 256, generator=g)
    i, j = torch.arange(n_in) % 256, torch.arange(n_out) % 256
    h = small[i][:, j].contiguous()
    turned, codes = code_buffers(n_out, n_in, -(-n_out // 128)), code_buffers(n_in, n_out, -(-n_in // 128))
    vb.quantize_weights(h.cuda(), *turned, *codes)
    want, _ = oc.quantize_weights(f64(small))
    full_exps = np.array([[oc.exponent(float(h[128 * a:128 * a + 128, 128 * b:128 * b + 128].abs().max())) for b in range(-(-n_out // 128))]
                          for a in range(-(-n_in // 128))])
    got = codes[1].cpu().numpy().astype(np.int64)[:, :full_exps.shape[1]] - 127
    assert np.array_equal(got, full_exps)
    assert np.array_equal(turned[1].cpu().numpy().astype(np.int64)[:, :full_exps.shape[0]] - 127, full_exps.T)
    # whole blocks have the small matrix's scales; what the others hold are codes of the same numbers under a smaller one
    whole_i, whole_j = n_in // 128 * 128, n_out // 128 * 128
    table = oc.code_values()
    want = table[want][i[:whole_i].numpy()][:, j[:whole_j].numpy()]
    assert np.array_equal(table[codes[0].cpu().numpy()[:whole_i, :whole_j]], want)
    assert np.array_equal(codes[0].cpu().numpy()[:, :n_out], turned[0].cpu().numpy()[:, :n_in].T)
    assert (codes[0].cpu().numpy()[:, n_out:] == 0).all() and (turned[0].cpu().numpy()[:, n_in:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("w", [1, 8, 20])
def test_tens_of_millions_of_narrow_rows(dtype, w):
    """Norm, codes, products and gradients over 20 million rows, of which a period repeats."""
    n, period = 20_000_003, 499
    base = torch.randn(period, w, generator=torch.Generator().manual_seed(w)).to(dtype).cuda()
    at = torch.arange(n, device="cuda") % period
    x, gain = base[at].contiguous(), torch.rand(w, device="cuda") + 0.5

    def passes(x):
        rows = x.shape[0]
        y, inv = torch.empty_like(x), torch.empty(rows, device="cuda")
        codes, scales = code_buffers(rows, w)
        vb.rms_norm_fwd(x, gain, 1e-5, y=y, codes=codes, scales=scales, inv_rms=inv)
        dx, dgain = torch.empty_like(x), torch.empty(w, device="cuda")
        vb.rms_norm_bwd(y, x, gain, inv, dx, dgain)
        z = torch.empty((rows, 5), dtype=dtype, device="cuda")
        vb.scaled_transform(codes, scales, *w8, w, z)
        return y, inv, codes, scales, dx, z, dgain

    w8 = _weights_with_few_different_columns(w, 5, 5, 1)[2]
    many, few = passes(x), passes(base)
    for a, b in zip(many[:-1], few[:-1]):
        for r0 in range(0, n, 1 << 22):
            assert torch.equal(a[r0:r0 + (1 << 22)], b[at[r0:r0 + (1 << 22)]])
    count = np.bincount(np.arange(n) % period, minlength=period)[:, None]
    V, D = f64(base) * f64(few[1])[:, None], f64(few[0])
    # a lane adds at most 20 million / (1,024 workgroups x 64 rows) + 1 rows in fp32, a workgroup 64 lanes, the rest in fp64
    assert_within(f64(many[-1]), (D * V * count).sum(axis=0), (n // 65536 + 70) * 2.0 ** -24 * (np.abs(D * V) * count).sum(axis=0), "dgain")
    dh = torch.empty((w, w), device="cuda")
    vb.scaled_bwd_weight(many[2], many[3], many[2], many[3], dh)
    c, e = few[2].cpu().numpy()[:, :w], few[3].cpu().numpy().astype(np.int64)[:, :1] - 127
    v = oc.values(c, e)
    # 512 slabs: a slab's rows in fp32, then 512 sums
    assert_within(f64(dh), v.T @ (v * count), (n // 256 + 600) * 2.0 ** -24 * (np.abs(v).T @ (np.abs(v) * count)), "dh")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_tensor_of_more_than_two_to_the_31_elements(dtype):
    n = (1 << 31) + 5
    big = torch.zeros(n, dtype=dtype, device="cuda")
    big[0], big[1 << 30], big[n - 1] = 3.0, 4.0, 12.0
    small, out = torch.full((1,), 84.0, dtype=dtype, device="cuda"), torch.empty(2, device="cuda")
    vb.clip_gradients([big, small], 17.0, out)
    assert float(out[0]) == 85.0 and abs(float(out[1]) - 0.2) < 2.0 ** -26
    f = np.float64(0.2)
    got = f64(torch.stack([big[0], big[1 << 30], big[n - 1], small[0]]))
    assert_within(got, f * np.array([3.0, 4.0, 12.0, 84.0]), (STEP[dtype] + 2.0 ** -23) * f * np.array([3.0, 4.0, 12.0, 84.0]), "clipped")
    big[0] = big[1 << 30] = big[n - 1] = 0
    assert not bool(big.any())


@pytest.mark.parametrize("n_in,n_out", [(1, 1), (1, 40), (300, 47)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_gradients_over_no_rows_of_buffers_that_are_there(n_in, n_out, accumulate):
    """Through the C ABI, whose callers keep their buffers when a batch is empty: before, inside and behind the gradient's memory."""
    memory = torch.ones(1 << 16, device="cuda")
    at = memory.data_ptr() + (1 << 17)
    dh = memory[1 << 15:(1 << 15) + n_in * n_out]
    for codes in (memory.data_ptr(), at, at + (1 << 16)):
        dh.fill_(1.0)
        code = vb.lib().varco_scaled_bwd_weight(0, n_in, n_out, codes, codes, codes, codes, at, n_out, accumulate, None, 0,
                                                torch.cuda.current_stream().cuda_stream)
        assert code == vb.OK and bool((dh == accumulate).all())
    assert bool((memory[:1 << 15] == 1).all()) and bool((memory[(1 << 15) + n_in * n_out:] == 1).all())
