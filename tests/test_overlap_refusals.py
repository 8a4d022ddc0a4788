"""Outputs that overlap what is read, other than the documented use in place: refused on the host before anything is launched, so no device is
needed and the pointers are never followed."""
import pytest

from paper_2406_17611_amd import binding as vb
from test_scaled_refusals import refused

X = 1 << 20
N, W, LD = 5, 100, 300              # rows of x: 400 of every 1,200 bytes
FAR = [X + (k << 20) for k in range(1, 9)]


def _fwd(x=X, ldx=LD, r=None, ldr=0, total=None, ldt=0, y=None, ldy=0, codes=None, scales=None, n=N):
    return [vb.F32, n, W, x, ldx, r, ldr, None, 1e-5, total, ldt, y, ldy, codes, scales, None, None]


def _bwd(dx, lddx, dy=X, u=FAR[0], dtotal=FAR[1], n=N):
    return [vb.F32, n, W, dy, LD, u, LD, None, FAR[2], dtotal, LD, dx, lddx, None, 0, None, 0, None]


SHIFTS = [
    (4, LD), (-4, LD), (396, LD), (-396, LD),                 # rows that begin inside the other's
    (LD * 4 + 4, LD), (-LD * 4 - 4, LD),                      # a row further on or back
    (LD * 4, LD), (-LD * 4, LD), (LD * 16, LD),               # the other's rows, but not at their place
    (804, LD), (-804, LD),                                    # a row's end in the next one
    (0, LD + 1), (0, W), (400, W),                            # rows of another distance
]


@pytest.mark.parametrize("by,ld", SHIFTS)
def test_rows_that_overlap_others(by, ld):
    for into in ("total", "y"):
        at = {into: X + by, ("ldt" if into == "total" else "ldy"): ld}
        refused("varco_rms_norm_fwd", _fwd(**at), vb.ERR_INVALID_ARG, "overlap")
        refused("varco_rms_norm_fwd", _fwd(x=FAR[0], r=X, ldr=LD, **at), vb.ERR_INVALID_ARG, "overlap")
    refused("varco_rms_norm_fwd", _fwd(x=FAR[0], total=X, ldt=LD, y=X + by, ldy=ld), vb.ERR_INVALID_ARG, "overlap" if by else "same memory")
    refused("varco_rms_norm_bwd", _bwd(X + by, ld), vb.ERR_INVALID_ARG, "overlap")
    refused("varco_rms_norm_bwd", _bwd(X + by, ld, dy=FAR[0], u=X), vb.ERR_INVALID_ARG, "overlap")
    refused("varco_rms_norm_bwd", _bwd(X + by, ld, dy=FAR[0], u=FAR[1], dtotal=X), vb.ERR_INVALID_ARG, "overlap")


@pytest.mark.parametrize("at", [X, X - 400, X + 384, X + 1200, X + 4 * 1200 + 384])
def test_codes_over_rows_that_are_read(at):
    codes, scales = at // 16 * 16, FAR[3]
    refused("varco_rms_norm_fwd", _fwd(codes=codes, scales=scales), vb.ERR_INVALID_ARG, "overlap")
    refused("varco_rms_norm_fwd", _fwd(codes=scales, scales=X + 1200), vb.ERR_INVALID_ARG, "overlap")
    refused("varco_quantize_rows", [vb.F32, N, W, X, LD, None, 0, codes, scales, None], vb.ERR_INVALID_ARG, "overlap")
    refused("varco_quantize_rows", [vb.F32, N, W, FAR[0], LD, X, LD, codes, scales, None], vb.ERR_INVALID_ARG, "overlap")


@pytest.mark.parametrize("operand", range(4))
def test_results_of_products_over_their_operands(operand):
    c = FAR[4]
    at = [FAR[0], FAR[1], FAR[2], FAR[3]]
    at[operand] = c + 4 * LD * 4 + 384                         # the last row of c
    refused("varco_scaled_transform", [vb.F32, N, 100, W, *at, c, LD, 0, 0, None], vb.ERR_INVALID_ARG, "overlap")
    refused("varco_scaled_bwd_weight", [N, 5, W, *at, c, LD, 0, None, 0, None], vb.ERR_INVALID_ARG, "overlap")


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("at", [X, X + 1200 * 4 + 384])
def test_codes_of_weights_over_the_weights_or_each_other(which, at):
    out = [FAR[0], FAR[1], FAR[2], FAR[3]]
    out[which] = at
    refused("varco_quantize_weights", [N, W, X, LD, *out, None], vb.ERR_INVALID_ARG, "overlap")
    out[which] = out[which - 1]
    refused("varco_quantize_weights", [N, W, X, LD, *out, None], vb.ERR_INVALID_ARG, "overlap")
