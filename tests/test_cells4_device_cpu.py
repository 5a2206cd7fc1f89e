"""A matrix in 4 bits whose memory is on another device than the current one is refused
by every call that it is given to, whatever the other tensors are."""
import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import _MX4


def here():
    return _MX4(3, 40, None, None)


def elsewhere():
    m = _MX4(3, 40, None, None)
    m.device = 1
    return m


CALLS = {
    "quantise": lambda m: octnca.octree_nca_mx4_quantise(torch.zeros(3, 40), m),
    "dequantise": lambda m: octnca.octree_nca_mx4_dequantise(m, torch.zeros(3, 40)),
    "product, rows": lambda m: octnca.octree_nca_mx4_product(m, here(), torch.zeros(3, 3)),
    "product, weights": lambda m: octnca.octree_nca_mx4_product(here(), m, torch.zeros(3, 3)),
    "linear, rows": lambda m: octnca.octree_nca_mx4_linear(torch.zeros(3, 40), m, here(),
                                                           torch.zeros(3, 3)),
    "linear, weights": lambda m: octnca.octree_nca_mx4_linear(torch.zeros(3, 40), here(), m,
                                                              torch.zeros(3, 3)),
    "backward, rows": lambda m: octnca.octree_nca_mx4_backward(torch.zeros(3, 3), m, here()),
    "backward, weights": lambda m: octnca.octree_nca_mx4_backward(torch.zeros(3, 3), here(), m),
}


@pytest.mark.parametrize("call", CALLS)
def test_a_matrix_on_another_device(library_path, monkeypatch, call):
    # the other tensors pass for ones on the current device
    monkeypatch.setattr(octnca, "_current_device", lambda: 0)
    monkeypatch.setattr(octnca, "_on_device", lambda t, name: None)
    monkeypatch.setattr(octnca, "_stream", lambda stream: 0)
    with pytest.raises(octnca.OctreeNCAError, match="cuda:1, the current device is 0"):
        CALLS[call](elsewhere())
    with pytest.raises(octnca.OctreeNCAError, match="invalid"):
        CALLS[call](here())          # gets to the library, which has no memory to work on


def test_a_struct_remembers_its_device(monkeypatch):
    class Codes:
        def __init__(self, shape):
            self.shape, self.dtype = shape, torch.uint8

        def get_device(self):
            return 1
    monkeypatch.setattr(octnca, "_current_device", lambda: 1)
    monkeypatch.setattr(octnca, "_ptr", lambda t, dtype, name: 0x1000)
    m = octnca.MX4Buffers(3, 40, *(Codes(s) for s in octnca.mx4_shapes(3, 40))).struct()
    assert m.device == 1


@pytest.mark.parametrize("call", CALLS)
def test_host_tensors_without_asking_for_a_device(library_path, monkeypatch, call):
    monkeypatch.setattr(octnca, "_current_device", None)
    with pytest.raises(octnca.OctreeNCAError, match="must be a device"):
        CALLS[call](here())
