"""What the calls of codes, norms, products and limited steps refuse, and the sizes of their workspaces: all decided on the host,
before anything is launched, so no device is needed. The pointers are never followed."""
import ctypes as C

import pytest
import torch

from paper_2406_17611_amd import binding as vb
from paper_2406_17611_amd.runner import KTapNetwork

P, ODD = 0x10000, 0x10001            # addresses, aligned and not
NAN, INF = float("nan"), float("inf")


def refused(name, args, code, text):
    got = getattr(vb.lib(), name)(*args)
    said = vb.lib().varco_last_error(None).decode()
    assert got == code, (name, got, said)
    assert said.startswith(name + ": ") and text in said, said


def changed(args, **at):
    """args with those at the positions of `at` (a0=..., a1=...) replaced."""
    out = list(args)
    for k, v in at.items():
        out[int(k[1:])] = v
    return out


ROWS = [vb.F32, 5, 100, P, 100, None, 0, P, P, None]


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=7), vb.ERR_UNSUPPORTED, "dtype"), (dict(a1=-1), vb.ERR_SHAPE, "row count"), (dict(a1=2 ** 31), vb.ERR_SHAPE, "row count"),
    (dict(a2=0), vb.ERR_SHAPE, "width"), (dict(a2=16385, a4=16385), vb.ERR_SHAPE, "width"), (dict(a3=None), vb.ERR_INVALID_ARG, "null"),
    (dict(a3=P + 2), vb.ERR_INVALID_ARG, "address"), (dict(a0=vb.BF16, a3=ODD), vb.ERR_INVALID_ARG, "address"),
    (dict(a4=99), vb.ERR_SHAPE, "leading"), (dict(a5=P, a6=99), vb.ERR_SHAPE, "leading"), (dict(a7=None), vb.ERR_INVALID_ARG, "codes"),
    (dict(a8=None), vb.ERR_INVALID_ARG, "codes"), (dict(a7=P + 8), vb.ERR_INVALID_ARG, "multiple of 16"), (dict(a8=P + 2), vb.ERR_INVALID_ARG, "multiple of 16")])
def test_quantize_rows(change, code, text):
    refused("varco_quantize_rows", changed(ROWS, **change), code, text)


WEIGHTS = [100, 40, P, 40, P, P, P, P, None]


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=0), vb.ERR_SHAPE, "width"), (dict(a1=16385, a3=16385), vb.ERR_SHAPE, "width"), (dict(a2=None), vb.ERR_INVALID_ARG, "null"),
    (dict(a3=39), vb.ERR_SHAPE, "leading"), (dict(a5=None), vb.ERR_INVALID_ARG, "codes"), (dict(a6=None), vb.ERR_INVALID_ARG, "codes"),
    (dict(a4=None, a5=None, a6=None, a7=None), vb.ERR_INVALID_ARG, "codes")])
def test_quantize_weights(change, code, text):
    refused("varco_quantize_weights", changed(WEIGHTS, **change), code, text)


PRODUCT = [vb.BF16, 5, 100, 40, P, P, P, P, P, 40, 0, vb.ACT_RELU, None]


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=-1), vb.ERR_UNSUPPORTED, "dtype"), (dict(a1=-5), vb.ERR_SHAPE, "row count"), (dict(a2=0), vb.ERR_SHAPE, "width"),
    (dict(a3=0), vb.ERR_SHAPE, "width"), (dict(a4=None), vb.ERR_INVALID_ARG, "codes"), (dict(a6=P + 1), vb.ERR_INVALID_ARG, "multiple of 16"),
    (dict(a8=None), vb.ERR_INVALID_ARG, "null"), (dict(a9=39), vb.ERR_SHAPE, "leading"), (dict(a11=5), vb.ERR_INVALID_ARG, "activation")])
def test_scaled_transform(change, code, text):
    refused("varco_scaled_transform", changed(PRODUCT, **change), code, text)


GRADIENT = [5000, 100, 40, P, P, P, P, P, 40, 0, P, 1 << 30, None]


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=-5), vb.ERR_SHAPE, "row count"), (dict(a1=0), vb.ERR_SHAPE, "width"), (dict(a2=20000, a8=20000), vb.ERR_SHAPE, "width"),
    (dict(a3=None), vb.ERR_INVALID_ARG, "codes"), (dict(a6=None), vb.ERR_INVALID_ARG, "codes"), (dict(a7=None), vb.ERR_INVALID_ARG, "null"),
    (dict(a8=39), vb.ERR_SHAPE, "leading"), (dict(a11=0), vb.ERR_STATE, "workspace"), (dict(a10=None), vb.ERR_STATE, "workspace"),
    (dict(a10=P + 16), vb.ERR_INVALID_ARG, "256-byte")])
def test_scaled_bwd_weight(change, code, text):
    refused("varco_scaled_bwd_weight", changed(GRADIENT, **change), code, text)


FORWARD = [vb.F32, 5, 100, P, 100, P, 100, P, 1e-5, P, 100, 2 * P, 100, P, P, P, None]


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=9), vb.ERR_UNSUPPORTED, "dtype"), (dict(a1=-1), vb.ERR_SHAPE, "row count"), (dict(a2=0), vb.ERR_SHAPE, "width"),
    (dict(a3=None), vb.ERR_INVALID_ARG, "null"), (dict(a4=50), vb.ERR_SHAPE, "leading"), (dict(a6=50), vb.ERR_SHAPE, "leading"),
    (dict(a7=P + 2), vb.ERR_INVALID_ARG, "address"), (dict(a8=-1.0), vb.ERR_INVALID_ARG, "eps"), (dict(a8=NAN), vb.ERR_INVALID_ARG, "eps"),
    (dict(a8=INF), vb.ERR_INVALID_ARG, "eps"), (dict(a10=99), vb.ERR_SHAPE, "leading"), (dict(a12=99), vb.ERR_SHAPE, "leading"),
    (dict(a13=None), vb.ERR_INVALID_ARG, "codes"), (dict(a9=2 * P), vb.ERR_INVALID_ARG, "same memory"),
    (dict(a9=None, a11=None, a13=None, a14=None, a15=None), vb.ERR_INVALID_ARG, "no output")])
def test_rms_norm_fwd(change, code, text):
    refused("varco_rms_norm_fwd", changed(FORWARD, **change), code, text)


BACKWARD = [vb.F32, 5000, 100, P, 100, P, 100, P, P, P, 100, P, 100, P, 0, P, 1 << 30, None]


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=9), vb.ERR_UNSUPPORTED, "dtype"), (dict(a1=-1), vb.ERR_SHAPE, "row count"), (dict(a2=0), vb.ERR_SHAPE, "width"),
    (dict(a3=None), vb.ERR_INVALID_ARG, "null"), (dict(a5=None), vb.ERR_INVALID_ARG, "null"), (dict(a8=None), vb.ERR_INVALID_ARG, "null"),
    (dict(a4=99), vb.ERR_SHAPE, "leading"), (dict(a10=99), vb.ERR_SHAPE, "leading"), (dict(a12=99), vb.ERR_SHAPE, "leading"),
    (dict(a11=None, a13=None), vb.ERR_INVALID_ARG, "no output"), (dict(a16=64), vb.ERR_STATE, "workspace"), (dict(a15=P + 64), vb.ERR_INVALID_ARG, "256-byte")])
def test_rms_norm_bwd(change, code, text):
    refused("varco_rms_norm_bwd", changed(BACKWARD, **change), code, text)


def _list(*a):
    return (C.c_void_p * len(a))(*a)


def _sizes(*n):
    return (C.c_int64 * len(n))(*n)


TWO, N = _list(P, P + 400), _sizes(100, 50)


@pytest.mark.parametrize("change,code,text", [
    (dict(a0=3), vb.ERR_UNSUPPORTED, "dtype"), (dict(a1=-1), vb.ERR_SHAPE, "negative"), (dict(a2=None), vb.ERR_INVALID_ARG, "null array"),
    (dict(a2=_list(P, None)), vb.ERR_INVALID_ARG, "null or at no"), (dict(a2=_list(P, P + 2)), vb.ERR_INVALID_ARG, "null or at no"),
    (dict(a1=2 ** 20 + 1), vb.ERR_SHAPE, "2^20"), (dict(a3=None), vb.ERR_INVALID_ARG, "null array"), (dict(a3=_sizes(1, -1)), vb.ERR_SHAPE, "element count"),
    (dict(a3=_sizes(1, 2 ** 43)), vb.ERR_SHAPE, "element count"), (dict(a3=_sizes(2 ** 42, 2 ** 42)), vb.ERR_SHAPE, "2^42"),
    (dict(a4=-1.0), vb.ERR_INVALID_ARG, "max_norm"), (dict(a4=NAN), vb.ERR_INVALID_ARG, "max_norm"), (dict(a5=None), vb.ERR_INVALID_ARG, "out"),
    (dict(a7=0), vb.ERR_STATE, "workspace"), (dict(a6=None), vb.ERR_STATE, "workspace"), (dict(a6=P + 8), vb.ERR_INVALID_ARG, "256-byte")])
def test_gradient_norm_and_what_is_limited_by_it(change, code, text):
    norm = [vb.F32, 2, TWO, N, 1.0, P, P, 1 << 20, None]
    refused("varco_gradient_norm", changed(norm, **change), code, text)
    at = {f"a{int(k[1:]) + (int(k[1:]) > 2)}": v for k, v in change.items()}
    refused("varco_clip_gradients", changed(norm[:3] + [TWO] + norm[3:], **at), code, text)
    if "a0" not in change:
        at = {f"a{i if i < 3 else i if i == 3 else i + 1}": v for i, v in ((int(k[1:]), v) for k, v in change.items())}
        at = {("a0" if k == "a1" else k): v for k, v in at.items()}
        step = [2, TWO, TWO, N, 0.1, 1.0, P, P, 1 << 20, None]
        refused("varco_sgd_step_clipped", changed(step, **at), code, text)
    if "a2" in change:
        refused("varco_clip_gradients", [vb.F32, 2, TWO, change["a2"], N, 1.0, P, P, 1 << 20, None], code, text)
        refused("varco_sgd_step_clipped", [2, change["a2"], TWO, N, 0.1, 1.0, P, P, 1 << 20, None], code, text)


def test_calls_without_rows_or_columns_do_nothing():
    L = vb.lib()
    assert L.varco_quantize_rows(vb.F32, 0, 8, None, 0, None, 0, None, None, None) == vb.OK
    assert L.varco_scaled_transform(vb.F32, 0, 8, 8, None, None, None, None, None, 0, 0, 0, None) == vb.OK
    assert L.varco_rms_norm_fwd(vb.F32, 0, 8, None, 0, None, 0, None, 0.0, None, 0, None, 0, None, None, None, None) == vb.OK
    assert L.varco_rms_norm_bwd(vb.F32, 0, 8, None, 0, None, 0, None, None, None, 0, None, 0, None, 0, None, 0, None) == vb.OK


@pytest.mark.parametrize("n", [0, 1, 31, 255, 256, 257, 5000, 169343, 2449029, 2 ** 31 - 1])
@pytest.mark.parametrize("w", [1, 47, 128, 256, 513, 2048, 16384])
def test_workspaces_have_bounds(n, w):
    assert 0 <= vb.rms_norm_workspace(vb.F32, n, w) <= 1024 * 16384 * 4
    for other in (1, 100, 512, 16384):
        size = vb.scaled_weight_workspace(n, w, other)
        assert 0 <= size <= 128 << 20 or size == 0
    assert vb.rms_norm_workspace(vb.BF16, min(n, 1), w) == 0 and vb.scaled_weight_workspace(min(n, 1), w, w) == 0


@pytest.mark.parametrize("sizes", [[], [0], [1], [0, 0, 5], [7] * 1000, [2 ** 40], [2 ** 31, 1, 2 ** 33]])
def test_norm_workspace(sizes):
    class Listed:
        def __init__(self, n):
            self.sizes = (C.c_int64 * len(n))(*n)
            self.n = len(n)

        def __len__(self):
            return self.n
    need = vb.gradient_norm_workspace(Listed(sizes))
    assert need % 8 == 0 and (need > 0) == (sum(sizes) > 0) and need <= 8 * 1024 * (1 + len(sizes) // 128)


@pytest.mark.parametrize("name,args", [("varco_rms_norm_workspace", [vb.F32, 5, 5, None]), ("varco_scaled_weight_workspace", [5, 5, 5, None]),
                                       ("varco_gradient_norm_workspace", [0, None, None])])
def test_workspace_queries_refuse_no_output(name, args):
    refused(name, args, vb.ERR_INVALID_ARG, "null output")


def test_streams_of_another_device_are_refused(monkeypatch):
    class Stream:
        cuda_stream, device_index = 64, 1
    vb._load_torch()
    monkeypatch.setattr(vb, "_device", lambda: 0)
    with pytest.raises(vb.VarcoError) as e:
        vb._on_device(Stream())
    assert e.value.code == vb.ERR_INVALID_ARG
    Stream.device_index = 0
    assert vb._on_device(Stream(), None) == Stream.cuda_stream
    with pytest.raises(vb.VarcoError):
        vb._on_device(Stream(), torch.zeros(1))


@pytest.mark.parametrize("workspace", [torch.zeros(1, dtype=torch.uint8).expand(4096), torch.zeros(8192, dtype=torch.uint8)[::2]])
def test_scratch_memory_in_pieces_is_refused(workspace):
    with pytest.raises(vb.VarcoError) as e:
        vb._scratch(0, workspace, "cpu", None)
    assert e.value.code == vb.ERR_SHAPE


def test_layers_of_taps_refuse_a_limited_step():
    """Their weights are not the matrices that the runner's step updates."""
    with pytest.raises(ValueError):
        KTapNetwork.sgd(object.__new__(KTapNetwork), 0.1, max_norm=1.0)
