"""Inputs and comparisons shared by the tests of 8-bit codes, their products, the norm and the gradient limit. Expected values come from
oracle/codes.py in fp64 on the same stored inputs."""
import numpy as np
import torch

from oracle import codes as oc
from paper_2406_17611_amd import binding as vb

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # half a step, relative to the value


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def code_buffers(rows, width, scale_rows=None):
    """Buffers full of what a call has to overwrite."""
    c = torch.full((rows, vb.code_ld(width)), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((rows if scale_rows is None else scale_rows, vb.scale_ld(width)), 0x5A, dtype=torch.uint8, device="cuda")
    return c, s


def strided(t, gap=3, lead=1):
    """The same matrix in memory with `gap` elements behind each row and `lead` in front of the first."""
    n, w = t.shape
    flat = torch.full((lead + n * (w + gap),), float("nan"), dtype=t.dtype, device=t.device)
    view = flat[lead:].view(n, w + gap)[:, :w]
    view.copy_(t)
    return view, flat


def upload_codes(codes, exps, width):
    """Device buffers of numpy codes and exponents, padded as the library pads them."""
    c = np.zeros((codes.shape[0], vb.code_ld(width)), dtype=np.uint8)
    c[:, :width] = codes
    s = np.full((exps.shape[0], vb.scale_ld(width)), 127, dtype=np.uint8)
    s[:, :exps.shape[1]] = exps + 127
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


def assert_codes(codes, scales, want_codes, want_exps, width):
    """Bit for bit (a zero's sign and a NaN's apart), padding included."""
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    nb = want_exps.shape[1]
    assert np.array_equal(s[:, :nb].astype(np.int64) - 127, want_exps)
    assert (s[:, nb:] == 127).all() and (c[:, width:] == 0).all()
    table = oc.code_values()
    assert np.array_equal(table[c[:, :width]], table[want_codes], equal_nan=True)


def assert_within(got, want, bound, what):
    """|got - want| <= bound, element by element."""
    got, want, bound = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64), np.asarray(bound, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= bound)
    if bad.any():
        at = np.argwhere(np.broadcast_to(bad, got.shape))[0]
        i = tuple(at)
        raise AssertionError(f"{what}: {int(bad.sum())} elements off, first at {i}: {got[i]!r} for {want[i]!r}, "
                             f"allowed {np.broadcast_to(bound, got.shape)[i]!r}")
