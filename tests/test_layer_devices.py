"""Calls of the operators around a mixing layer run on their tensors' GPU, whichever is the
current one: a default stream's handle (0) stands for the current device's.  Two GPUs
are stood in for by tensors that say where they are, so these run without any."""
import contextlib

import pytest
import torch

from paper_2509_25223_amd import layer


class OnGPU:
    """What the calls look at of a contiguous tensor on GPU `index`."""
    device = torch.device("cuda:1")

    def __init__(self, *shape, dtype=torch.float32, index=1):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def element_size(self):
        return 4


class Stream:
    def __init__(self, index, handle=0):
        self.device_index, self.cuda_stream = index, handle


@pytest.fixture
def gpus(monkeypatch):
    """Two GPUs, 0 current; the C functions note the device that they are called on."""
    state = dict(current=0, calls=[])

    @contextlib.contextmanager
    def device(index):
        before, state["current"] = state["current"], index
        try:
            yield
        finally:
            state["current"] = before

    class Library:
        def __getattr__(self, name):
            if name.endswith("workspace_size"):
                return lambda *args: 64
            return lambda *args: state["calls"].append((name, state["current"], args[-1])) or state.get("status", 0)

    monkeypatch.setattr(layer, "torch", torch)
    monkeypatch.setattr(layer, "_bound", Library())
    monkeypatch.setattr(layer, "_stream_of", lambda index: 0)
    monkeypatch.setattr(layer, "_current", lambda: state["current"], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(layer, "_new", lambda like, shape, dtype, stream: OnGPU(*(shape if isinstance(shape, tuple) else [shape]),
                                                                                dtype=dtype))
    return state


def calls(stream=None):
    x, w, b = OnGPU(2, 3, 8), OnGPU(8, 4), OnGPU(2, 3, 5)
    A, row, heads = OnGPU(8, 5), OnGPU(8), OnGPU(2, 3, 2, 4)
    half, s = OnGPU(4), dict(stream=stream)
    return {"rla_conv_forward": lambda: layer.rla_conv_forward(x, w, **s),
            "rla_conv_backward": lambda: layer.rla_conv_backward(x, w, x, **s),
            "rla_conv_decode": lambda: layer.rla_conv_decode(x, w, **s),
            "rla_ssm_forward": lambda: layer.rla_ssm_forward(x, x, A, b, b, **s),
            "rla_ssm_backward": lambda: layer.rla_ssm_backward(x, x, A, b, b, x, **s),
            "rla_ssm_decode": lambda: layer.rla_ssm_decode(x, x, A, b, b, **s),
            "rla_addnorm_forward": lambda: layer.rla_addnorm_forward(x, row, **s),
            "rla_addnorm_backward": lambda: layer.rla_addnorm_backward(x, x, row, **s),
            "rla_gatenorm_forward": lambda: layer.rla_gatenorm_forward(heads, heads, half, **s),
            "rla_gatenorm_backward": lambda: layer.rla_gatenorm_backward(heads, heads, heads, half, **s)}


NAMES = list(calls())


@pytest.mark.parametrize("name", NAMES)
def test_current_stream(gpus, name):
    calls()[name]()
    assert gpus["calls"] == [(name, 1, 0)] and gpus["current"] == 0
    gpus["current"] = 1   # the tensors' own is the current one
    calls()[name]()
    assert gpus["calls"][1:] == [(name, 1, 0)] and gpus["current"] == 1


@pytest.mark.parametrize("name", NAMES)
def test_given_stream(gpus, name):
    calls(Stream(1, 77))[name]()
    assert gpus["calls"] == [(name, 1, 77)] and gpus["current"] == 0


@pytest.mark.parametrize("name", NAMES)
def test_stream_of_another_device(gpus, name):
    with pytest.raises(ValueError, match="stream"):
        calls(Stream(0))[name]()
    assert gpus["calls"] == [] and gpus["current"] == 0


def test_status_on_another_device(gpus):
    """A refusal there comes back, and the current device with it."""
    gpus["status"] = 2
    with pytest.raises(layer.RLAError):
        calls()["rla_ssm_decode"]()
    assert gpus["current"] == 0
