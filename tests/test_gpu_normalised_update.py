"""The update that a limited step makes to weights and gain, as the last part of a training step of normalised layers: compared with
the fp64 step's by itself, relative to its own size (beside the weights it is small)."""
import numpy as np
import pytest
import torch

from codes_common import f64
from test_gpu_normalised_layers import LIMIT, LR, Block, _reference

pytestmark = pytest.mark.gpu


# tol: norm-wise bound of a gradient (test_gpu_normalised_layers.py derives it), which holds for the norm of all of them as well. The update
# is lr f dw: (1 + tol)^2 / (1 - tol) - 1 < 3.3 tol, and the weight is rounded once, 2^-24 of it. lr is a number of fp32: 2^-24 of the update.
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2.0 ** -10), (torch.bfloat16, 2.0 ** -5)])
@pytest.mark.parametrize("n,width,hidden,classes", [(700, 100, 256, 47), (333, 256, 130, 8), (1, 64, 32, 5)])
def test_the_update_is_the_limited_step(dtype, tol, n, width, hidden, classes):
    b = Block(n, width, hidden, classes, dtype, n)
    before = [f64(w) for w in b.weights + [b.gain]]
    norm, f, *gradients = [np.array(g) for g in (*_reference(b)[5], *_reference(b)[6:9])]
    assert norm > LIMIT and abs(norm * f - LIMIT) < 1e-9               # the limit is what counts here
    b.step()
    for i, (w, old, g) in enumerate(zip(b.weights + [b.gain], before, gradients)):
        update = -LR * f * g
        size = np.linalg.norm(update)
        allowed = 3.3 * tol * size + 2.0 ** -24 * (np.linalg.norm(old) + 2 * size)
        assert allowed < size / 4, (i, allowed, size)                  # no step at all, or one the other way, would fail
        off = np.linalg.norm(f64(w) - old - update)
        assert off <= allowed, (i, off, allowed, size)
