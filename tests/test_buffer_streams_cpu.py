"""Which streams an object's own memory is kept for, with stand-ins for streams and
tensors: torch does not hand out memory that a recorded stream may still read."""
import pytest
import torch

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import runtime

MAKER = 0x10     # handle of the stream that everything is made on


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.waits = handle, 0

    def wait_event(self, event):
        self.waits += 1


class Event:
    def record(self):
        pass


class Memory:
    """A tensor, as far as its memory goes."""

    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


class Machine:
    """The current stream, and the streams behind handles."""

    def __init__(self):
        self.streams, self.current = {}, MAKER

    def stream(self, handle):
        return self.streams.setdefault(handle, Stream(handle))


@pytest.fixture
def machine(monkeypatch):
    m = Machine()
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", m.stream)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: m.stream(m.current))
    monkeypatch.setattr(octnca, "_current_device", lambda: 0)
    monkeypatch.setattr(octnca, "_current_handle", lambda device: m.current)
    return m


def matrix():
    x = runtime.MX4Matrix.__new__(runtime.MX4Matrix)
    x.struct, x.memory = octnca._MX4(3, 4, None, None), Memory()
    x._own = runtime._Buffers(x.memory)
    return x


@pytest.fixture
def layer(machine, monkeypatch):
    calls = []
    monkeypatch.setattr(runtime, "octree_nca_mx4_product", lambda *a: calls.append(a[-1]))
    monkeypatch.setattr(runtime, "octree_nca_mx4_backward", lambda *a: calls.append(a[-1]))
    x = runtime.CellLayer.__new__(runtime.CellLayer)
    x.w, x.kept, x.bias, x.calls, x.memory = matrix(), matrix(), None, calls, Memory()
    x.last, x.workspace, x.grad_weight, x.grad_bias = x.kept, 1, None, None
    x._own = runtime._Buffers(x.memory)
    return x


def call(layer, machine, way, kind, m, handle):
    """One call of the layer with the matrix m on a stream: given, or the current one."""
    machine.current = handle if kind == "current" else MAKER
    stream = {"object": machine.stream(handle), "handle": handle, "current": None}[kind]
    if way == "forward":
        layer.forward(m, None, stream=stream)
    else:
        layer.backward(None, kept=m, stream=stream)
    machine.current = MAKER


@pytest.mark.parametrize("way", ["forward", "backward"])
@pytest.mark.parametrize("kind", ["object", "current"])
def test_a_matrix_given_to_a_layer_is_kept_for_its_stream(machine, layer, way, kind):
    m = matrix()
    for _ in range(2):
        call(layer, machine, way, kind, m, 0x20)
    assert m.memory.recorded == [0x20] and layer.memory.recorded == [0x20]
    assert machine.stream(0x20).waits == 2       # for the layer's fills, for the matrix's
    assert layer.calls == [0x20, 0x20]
    call(layer, machine, way, kind, m, 0x30)
    assert m.memory.recorded == [0x20, 0x30]


@pytest.mark.parametrize("way", ["forward", "backward"])
def test_a_handle_does_not_stand_for_its_stream(machine, layer, way):
    """After a call with a bare handle (waited for, not recorded), one with the stream
    records it."""
    m = matrix()
    for _ in range(2):
        call(layer, machine, way, "handle", m, 0x20)
    assert m.memory.recorded == [] and machine.stream(0x20).waits == 2
    call(layer, machine, way, "object", m, 0x20)
    assert m.memory.recorded == [0x20] and layer.memory.recorded == [0x20]
    assert machine.stream(0x20).waits == 2


def test_the_making_stream_needs_neither(machine, layer):
    m = matrix()
    call(layer, machine, "forward", "current", m, MAKER)
    call(layer, machine, "forward", "object", m, MAKER)
    assert m.memory.recorded == [] and machine.stream(MAKER).waits == 0
