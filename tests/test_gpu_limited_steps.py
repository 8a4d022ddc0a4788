"""What the runner's limited steps leave to their caller."""
import pytest
import torch

from paper_2406_17611_amd.runner import PartitionedNetwork
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

def test_a_subclass_with_a_step_of_its_own_still_trains():
    class Network(PartitionedNetwork):
        steps = 0

        def sgd(self, lr, stream=None):
            Network.steps += 1
            return super().sgd(lr, stream)

    a, b = _network(), _network()
    b.__class__ = Network
    for step in range(2):
        a.train_step(step, (2, 1), 0.3)
        b.train_step(step, (2, 1), 0.3)
    assert Network.steps == 2
    for x, y in zip(a.h1 + a.h0, b.h1 + b.h0):
        assert torch.equal(x, y)
