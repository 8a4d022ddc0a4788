"""Lists of tensors that are updated together: which pairs of lists the limited steps refuse. Decided on the host from addresses and sizes alone,
so stand-ins for device tensors do."""
import pytest
import torch

from paper_2406_17611_amd import binding as vb


class Memory:
    """What a list asks of a device tensor."""
    is_cuda = True

    def __init__(self, address, n, dtype=torch.float32):
        self.address, self.n, self.dtype = address, n, dtype

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.n

    def element_size(self):
        return 4 if self.dtype == torch.float32 else 2

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0


BASE = 1 << 20


def _tensors(*at, n=100):
    """Tensors of n elements that start so many elements behind BASE."""
    return [Memory(BASE + 4 * a, n) for a in at]


@pytest.fixture(autouse=True)
def _on_the_current_device(monkeypatch):
    vb._load_torch()
    monkeypatch.setattr(vb, "_device", lambda: 0)
    monkeypatch.setattr(vb, "_handle", lambda device: 0)


GRADS = (0, 100, 200, 1000)
OVERLAPPING = [
    (0, 100, 200, 1001),        # one that is shifted by an element
    (0, 100, 200, 901),         # by all but one
    (0, 200, 100, 1000),        # the same memory in another order
    (100, 200, 300, 1000),      # each the next one
    (5000, 150, 6000, 7000),    # over two of them
    (5000, 6000, 7000, 50),
]


@pytest.mark.parametrize("at", OVERLAPPING)
@pytest.mark.parametrize("made", [False, True])
def test_lists_that_overlap_are_refused(at, made):
    grads, others = _tensors(*GRADS), _tensors(*at)
    if made:
        grads, others = vb.TensorList(grads), vb.TensorList(others)
    out = Memory(64, 2)
    for _ in range(2):
        for call in (lambda: vb.clip_gradients(grads, 1.0, out, into=others), lambda: vb.sgd_step_clipped(others, grads, 0.1, 1.0, out)):
            with pytest.raises(vb.VarcoError) as e:
                call()
            assert e.value.code == vb.ERR_INVALID_ARG and "overlap" in str(e.value)


def test_weights_that_are_their_own_gradients_are_refused():
    """In place is a form of clipping only, also where it has been one with the same lists before."""
    out = Memory(64, 2)
    same, a, b = vb.TensorList(_tensors(*GRADS)), vb.TensorList(_tensors(*GRADS)), vb.TensorList(_tensors(*GRADS))
    vb._check_apart(a, b, True)
    for w, dw in ((same, same), (a, b), (_tensors(*GRADS), _tensors(*GRADS))):
        with pytest.raises(vb.VarcoError) as e:
            vb.sgd_step_clipped(w, dw, 0.1, 1.0, out)
        assert e.value.code == vb.ERR_INVALID_ARG and "overlap" in str(e.value)


@pytest.mark.parametrize("at", [GRADS, (300, 400, 500, 1100), (1100, 800, 700, 600), (0, 5000, 200, 300)])
def test_lists_beside_each_other_or_in_place_are_taken(at):
    for _ in range(2):
        vb._check_apart(vb.TensorList(_tensors(*at)), vb.TensorList(_tensors(*GRADS)), True)


def test_tensors_without_elements_overlap_nothing():
    a = vb.TensorList([Memory(BASE, 10), Memory(BASE + 4, 0), Memory(BASE + 400, 10)])
    b = vb.TensorList([Memory(BASE + 40, 10), Memory(0, 0), Memory(BASE + 440, 10)])
    vb._check_apart(a, b, False)


def test_a_verdict_holds_for_its_pair_only():
    grads, apart, shifted = (vb.TensorList(_tensors(*at)) for at in (GRADS, (2000, 2100, 2200, 2300), (1, 2100, 2200, 2300)))
    vb._check_apart(apart, grads, False)
    vb._check_apart(apart, grads, False)
    for pair in ((apart, apart), (apart, shifted), (shifted, grads)):
        with pytest.raises(vb.VarcoError):
            vb._check_apart(*pair, False)
    vb._check_apart(apart, grads, False)


def test_a_tensor_with_other_memory_is_taken_where_it_is_now():
    """As after t.data = ..., t.set_(...), t.resize_(...): a list never goes on with an address that a tensor no longer has."""
    tensors = _tensors(*GRADS)
    made = vb.TensorList(tensors)
    assert vb._listed(made) is made and list(made.pointers) == [t.address for t in tensors]
    tensors[2].address = BASE - 4096
    assert vb._listed(made) is made and list(made.pointers) == [t.address for t in tensors]
    tensors[1].n = 40
    assert list(vb._listed(made).sizes) == [100, 40, 100, 100]
    need = made.need
    tensors[3].n = 1 << 24
    assert vb._listed(made).need == vb.gradient_norm_workspace(made) > need


def test_other_memory_is_checked_as_a_new_list_is():
    grads, weights = _tensors(*GRADS), _tensors(2000, 2100, 2200, 2300)
    g, w = vb.TensorList(grads), vb.TensorList(weights)
    vb._check_apart(w, g, False)
    out = Memory(64, 2)
    for t, address in ((grads[0], BASE + 4 * 2050), (weights[3], BASE + 4 * 150)):
        keep, t.address = t.address, address
        for _ in range(2):
            with pytest.raises(vb.VarcoError) as e:
                vb.sgd_step_clipped(w, g, 0.1, 1.0, out)
            assert "overlap" in str(e.value)
        t.address = keep
        vb._check_apart(vb._listed(w), vb._listed(g), False)
    grads[0].address = BASE + 4 * 50                                  # over its neighbour
    for _ in range(2):
        with pytest.raises(vb.VarcoError):
            vb.gradient_norm(g, 1.0, out)
    grads[0].address = BASE
    grads[0].n = 99
    with pytest.raises(vb.VarcoError) as e:
        vb.sgd_step_clipped(w, g, 0.1, 1.0, out)
    assert e.value.code == vb.ERR_SHAPE
