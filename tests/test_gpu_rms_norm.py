"""Root-mean-square norm and its backward pass, through the C ABI, against fp64 on the same stored inputs.

Bounds. A lane adds at most 32 squares one after the other, lanes join in at most 9 more additions; with the mean, the addition of eps, the root and the
division 1 / rms is off by at most 48 2^-24 of itself (half of the sum's error: the root halves it). An output adds two products and the rounding to its type."""
import numpy as np
import pytest
import torch

from codes_common import STEP, assert_within, code_buffers, f64, strided
from oracle import codes as oc
from paper_2406_17611_amd import binding as vb

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
F = 2.0 ** -24
INV = 48 * F
EPS = 1e-5


def _rows(n, w, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, w, generator=g) * torch.exp(torch.randn(n, 1, generator=g) * 2)
    if n > 2:
        x[1] = 0.0
    return x.to(dtype).cuda()


WIDTHS = [1, 5, 16, 33, 47, 64, 100, 128, 129, 256, 300, 512, 513, 1000, 1024, 2048, 2049, 4096, 4100, 9001, 16384]


def _check_codes(codes, scales, y, w):
    """The codes stand for numbers within half a step of y (2^-4 of it, or 2^-10 of the scale), the scale fits the block's largest."""
    c, e = codes.cpu().numpy(), scales.cpu().numpy().astype(np.int64) - 127
    nb = -(-w // 128)
    assert (c[:, w:] == 0).all() and (e[:, nb:] == 0).all()
    exps = e[:, :nb]
    got = oc.values(c[:, :w], exps)
    s = np.repeat(2.0 ** exps, 128, axis=1)[:, :w]
    off = INV + 4 * F
    assert_within(got, y, (2.0 ** -4 + off) * np.abs(y) + 2.0 ** -10 * s, "codes")
    for b in range(nb):
        a = np.abs(y[:, 128 * b:128 * (b + 1)]).max(axis=1)
        fits = (a * (1 - off) <= 448.0 * 2.0 ** exps[:, b]) & (a * (1 + off) >= 224.0 * 2.0 ** exps[:, b])
        assert (fits | ((a == 0) & (exps[:, b] == 0))).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("w", WIDTHS)
def test_forward(dtype, w):
    n = 37 if w < 4000 else 5
    x, r = _rows(n, w, dtype, w), _rows(n, w, dtype, w + 1)
    gain = torch.randn(w, generator=torch.Generator().manual_seed(w)).cuda()
    total, y = torch.empty_like(x), torch.empty_like(x)
    inv = torch.empty(n, device="cuda")
    codes, scales = code_buffers(n, w)
    vb.rms_norm_fwd(x, gain, EPS, residual=r, total=total, y=y, codes=codes, scales=scales, inv_rms=inv)
    assert torch.equal(total, (x.float() + r.float()).to(dtype))
    want, want_inv = oc.rms_norm(f64(total), f64(gain), EPS)
    assert_within(f64(inv), want_inv, INV * want_inv, "inv_rms")
    assert_within(f64(y), want, (INV + 3 * F + STEP[dtype]) * np.abs(want) + 1e-38, "y")
    _check_codes(codes, scales, want, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,w", [(1, 256), (3, 47), (1000, 75), (70, 512)])
def test_outputs_one_by_one_without_residual_or_gain(dtype, n, w):
    x = _rows(n, w, dtype, 3)
    xs, _ = strided(x, 5, 1)
    want, want_inv = oc.rms_norm(f64(x), 1.0, EPS)
    y, flat = strided(torch.zeros_like(x), 3, 2)
    vb.rms_norm_fwd(xs, None, EPS, y=y)
    assert_within(f64(y), want, (INV + 3 * F + STEP[dtype]) * np.abs(want) + 1e-38, "y")
    assert torch.isnan(flat[2:].view(n, w + 3)[:, w:]).all() and torch.isnan(flat[:2]).all()
    inv = torch.empty(n, device="cuda")
    vb.rms_norm_fwd(xs, None, EPS, inv_rms=inv)
    assert_within(f64(inv), want_inv, INV * want_inv, "inv_rms")
    codes, scales = code_buffers(n, w)
    vb.rms_norm_fwd(xs, None, EPS, codes=codes, scales=scales)
    _check_codes(codes, scales, want, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("w", [48, 256, 3000])
def test_in_place(dtype, w):
    x, r = _rows(9, w, dtype, 4), _rows(9, w, dtype, 5)
    gain = torch.rand(w, device="cuda") + 0.5
    total, y = torch.empty_like(x), torch.empty_like(x)
    vb.rms_norm_fwd(x, gain, EPS, residual=r, total=total, y=y)
    x2, r2 = x.clone(), r.clone()
    vb.rms_norm_fwd(x2, gain, EPS, residual=r2, total=r2, y=x2)
    assert torch.equal(r2, total) and torch.equal(x2, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_stays_in_its_row(dtype):
    x = _rows(8, 300, dtype, 6)
    x[2, 10], x[5, 299] = float("inf"), float("nan")
    y, inv = torch.empty_like(x), torch.empty(8, device="cuda")
    codes, scales = code_buffers(8, 300)
    vb.rms_norm_fwd(x, None, EPS, y=y, codes=codes, scales=scales, inv_rms=inv)
    others = [0, 1, 3, 4, 6, 7]
    want, _ = oc.rms_norm(f64(x)[others], 1.0, EPS)
    assert_within(f64(y)[others], want, (INV + 3 * F + STEP[dtype]) * np.abs(want) + 1e-38, "y")
    _check_codes(codes[others], scales[others], want, 300)
    y, table = f64(y), oc.code_values()
    assert np.isnan(y[2, 10]) and (np.delete(y[2], 10) == 0).all() and np.isnan(y[5]).all()
    values = table[codes.cpu().numpy()[:, :300]]
    assert np.isnan(values[2, 10]) and (np.delete(values[2], 10) == 0).all() and np.isnan(values[5]).all()


# Backward: 48 + 2 roundings in 1 / rms (as it is given: none) aside, a row's sum of w products adds 41 roundings of its sizes as above.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("w", WIDTHS)
@pytest.mark.parametrize("more", [False, True])
def test_backward(dtype, w, more):
    n = 75 if w < 4000 else 5
    u, dy, du = _rows(n, w, dtype, w), _rows(n, w, dtype, w + 1), _rows(n, w, dtype, w + 2)
    gain = torch.randn(w, generator=torch.Generator().manual_seed(w)).cuda()
    inv = torch.from_numpy(oc.rms_norm(f64(u), 1.0, EPS)[1].astype(np.float32)).cuda()
    start = torch.randn(w, generator=torch.Generator().manual_seed(w + 3)).cuda()
    dx, dgain = torch.empty_like(u), start.clone()
    vb.rms_norm_bwd(dy, u, gain, inv, dx, dgain, dtotal=du if more else None, accumulate=more)
    U, D, G, S = f64(u), f64(dy), f64(gain), f64(inv)
    want, want_g = oc.rms_norm_backward(D, U, G, S)
    V = np.abs(U * S[:, None])
    H = np.abs(D * G)
    size = S[:, None] * (H + V * (H * V).mean(axis=1, keepdims=True))
    size_g = (np.abs(D) * V).sum(axis=0)
    if more:
        want, size = want + f64(du), size + np.abs(f64(du))
        want_g, size_g = want_g + f64(start), size_g + np.abs(f64(start))
    assert_within(f64(dx), want, 52 * F * size + STEP[dtype] * (np.abs(want) + 52 * F * size) + 1e-38, "dx")
    assert_within(f64(dgain), want_g, (n + 4) * F * size_g + 1e-38, "dgain")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,w", [(0, 64), (1, 64), (20000, 40), (5000, 256), (3000, 1000)])
def test_gain_gradient_over_many_rows(dtype, n, w):
    u, dy = _rows(n, w, dtype, 7), _rows(n, w, dtype, 8)
    inv = torch.rand(n, generator=torch.Generator().manual_seed(9)).cuda()
    out = [torch.empty(w, device="cuda") for _ in range(2)]
    dx = torch.empty_like(u)
    vb.rms_norm_bwd(dy, u, None, inv, None, out[0])                    # the gain's gradient alone
    vb.rms_norm_bwd(dy, u, None, inv, dx, out[1])
    assert torch.equal(out[0], out[1])                                 # one order of sums
    V = f64(u) * f64(inv)[:, None]
    assert_within(f64(out[0]), (f64(dy) * V).sum(axis=0), (n + 4) * F * (np.abs(f64(dy)) * np.abs(V)).sum(axis=0), "dgain")
    again = torch.empty_like(u)
    vb.rms_norm_bwd(dy, u, None, inv, again)                           # the rows' gradient alone
    assert torch.equal(dx, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("into", ["dy", "u", "dtotal"])
@pytest.mark.parametrize("w", [100, 512, 5000])
def test_backward_in_place(dtype, into, w):
    t = dict(dy=_rows(11, w, dtype, 10), u=_rows(11, w, dtype, 11), dtotal=_rows(11, w, dtype, 12))
    gain, inv = torch.rand(w, device="cuda"), torch.rand(11, device="cuda")
    want, dgain = torch.empty_like(t["u"]), torch.empty(w, device="cuda")
    vb.rms_norm_bwd(t["dy"], t["u"], gain, inv, want, dgain, dtotal=t["dtotal"])
    again = torch.empty_like(dgain)
    vb.rms_norm_bwd(t["dy"], t["u"], gain, inv, t[into], again, dtotal=t["dtotal"])
    assert torch.equal(t[into], want) and torch.equal(again, dgain)


def test_gradients_against_differences():
    """The kernel's gradients against differences of the kernel's own fp32 forward pass, summed in fp64: a step of 2^-7 leaves 2^-24 2^7
    of rounding and 2^-14 of curvature."""
    g = torch.Generator().manual_seed(13)
    u, dy, gain = torch.randn(2, 24, generator=g).cuda(), torch.randn(2, 24, generator=g).cuda(), torch.rand(24, generator=g).cuda() + 0.5
    inv, y = torch.empty(2, device="cuda"), torch.empty_like(u)
    vb.rms_norm_fwd(u, gain, 0.1, inv_rms=inv)
    dx, dgain = torch.empty_like(u), torch.empty_like(gain)
    vb.rms_norm_bwd(dy, u, gain, inv, dx, dgain)

    def risk(a, b):
        vb.rms_norm_fwd(a, b, 0.1, y=y)
        return float((y.double() * dy.double()).sum())

    h = 2.0 ** -7
    for at in [(0, 0), (0, 23), (1, 7)]:
        d = torch.zeros_like(u)
        d[at] = h
        assert abs((risk(u + d, gain) - risk(u - d, gain)) / (2 * h) - float(dx[at])) < 2e-3
    for j in (0, 11, 23):
        d = torch.zeros_like(gain)
        d[j] = h
        assert abs((risk(u, gain + d) - risk(u, gain - d)) / (2 * h) - float(dgain[j])) < 2e-3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("w", [48, 75, 512, 1000, 4100])
def test_more_rows_than_a_launch_takes_at_once(dtype, w):
    """Rows that repeat with a period give results that repeat, forward and backward; codes too."""
    period, n = 191, 150_001 if w < 1000 else 40_001
    at = torch.arange(n, device="cuda") % period
    base = [_rows(period, w, dtype, w + k) for k in range(3)]
    x, r, dy = (t[at].contiguous() for t in base)
    gain = torch.rand(w, device="cuda") + 0.5

    def passes(x, r, dy):
        total, y, inv = torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[0], device="cuda")
        codes, scales = code_buffers(x.shape[0], w)
        vb.rms_norm_fwd(x, gain, EPS, residual=r, total=total, y=y, codes=codes, scales=scales, inv_rms=inv)
        dx = torch.empty_like(x)
        vb.rms_norm_bwd(dy, total, gain, inv, dx, None, dtotal=y)
        again, again_scales = code_buffers(x.shape[0], w)
        vb.quantize_rows(x, again, again_scales, gate=r)
        return total, y, inv, codes, scales, dx, again, again_scales

    for many, few in zip(passes(x, r, dy), passes(*base)):
        assert torch.equal(many, few[at])


def test_rows_beyond_32_bits_of_bytes():
    n, w = 2_200_001, 1000
    x = torch.zeros((n, w), device="cuda")
    x[-3:] = torch.randn(3, w, generator=torch.Generator().manual_seed(5)).cuda()
    codes, scales = code_buffers(n, w)
    y = torch.empty_like(x)
    vb.rms_norm_fwd(x, None, EPS, y=y, codes=codes, scales=scales)
    want, _ = oc.rms_norm(f64(x[-3:]), 1.0, EPS)
    assert_within(f64(y[-3:]), want, (INV + 4 * F) * np.abs(want), "y")
    _check_codes(codes[-3:], scales[-3:], want, w)
    assert bool((y[:-3] == 0).all()) and bool((codes[:-3] == 0).all())
