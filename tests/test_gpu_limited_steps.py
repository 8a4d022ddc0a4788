"""What the runner's limited steps leave to their caller."""
import pytest
import torch

from test_gpu_normalised_layers import _network

pytestmark = pytest.mark.gpu


def test_norm_and_factor_lie_in_a_buffer_of_the_network():
    """Made with the network, as its other buffers are: a step on another stream finds no memory that earlier work of the current stream still
    uses. The same tensor after every step, by its public name."""
    net = _network()
    at = net.gradient_norm.data_ptr()
    assert net.gradient_norm.shape == (2,) and net.gradient_norm.dtype == torch.float32
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.train_step(0, (2, 1), 0.1, stream=side, max_norm=0.5)
    torch.cuda.synchronize()
    first = net.gradient_norm.clone()
    assert bool(torch.isfinite(first).all()) and float(first[0]) > 0 and abs(float(first[1]) - min(1.0, 0.5 / float(first[0]))) < 1e-6
    returned = net.sgd(0.0, max_norm=0.25)
    assert returned is net.gradient_norm and returned.data_ptr() == at
    assert float(returned[0]) == float(first[0]) and abs(float(returned[1]) - min(1.0, 0.25 / float(first[0]))) < 1e-6
