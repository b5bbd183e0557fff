"""The mixing operators' calls run on their tensors' GPU, whichever is the current one, and
refuse tensors that are on none.  Two GPUs are stood in for by tensors that say where
they are, so these run without any."""
import contextlib

import pytest
import torch

import paper_2509_25223_amd as rla
from tests.test_layer_devices import OnGPU, Stream

B, T, H, D = 2, 3, 2, 64


@pytest.fixture
def gpus(monkeypatch):
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
            return lambda *args: state["calls"].append((name, state["current"], args[-1])) or 0

    monkeypatch.setattr(rla, "load_library", lambda: Library())
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: state["current"])
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state["current"])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index)
    return state


def calls(stream=None, index=1):
    f32 = torch.float32
    x = [OnGPU(B, T, H, D, index=index) for _ in range(3)] + [OnGPU(B, T, H, index=index) for _ in range(4)]
    state, ws = OnGPU(B, H, D, D, index=index), OnGPU(64, index=index)
    for t in x + [state, ws]:
        t.device = torch.device("cuda", index) if index >= 0 else torch.device("cpu")
    s = dict(stream=stream)
    grads = {"d" + n: t for n, t in zip(("q", "k", "v", "alpha_s", "beta", "alpha_r", "gamma"), x)}
    return {"rdn_forward": lambda: rla.rdn_forward(*x, out=x[2], workspace=ws, return_states=False, **s),
            "rla_forward": lambda: rla.rla_forward(*x, out=x[2], workspace=ws, return_states=False, **s),
            "rdn_forward_noalloc": lambda: rla.rdn_forward_noalloc(*x, out=x[2], S_final=state, R_final=state, **s),
            "rdn_backward": lambda: rla.rdn_backward(*x, x[2], grads=grads, workspace=ws, **s),
            "rla_backward": lambda: rla.rla_backward(*x, x[2], grads=grads, workspace=ws, **s),
            "rdn_decode": lambda: rla.rdn_decode(*x, S_out=state, R_out=state, out=x[2], out_dtype=f32, **s),
            "rla_decode": lambda: rla.rla_decode(*x, S_out=state, R_out=state, out=x[2], out_dtype=f32, **s)}


NAMES = list(calls())


def handle(x):
    return getattr(x, "value", x)


@pytest.mark.parametrize("name", NAMES)
def test_current_stream(gpus, name):
    for current in (0, 1):
        gpus["current"] = current
        calls()[name]()
        got, where, stream = gpus["calls"].pop()
        assert (got, where, handle(stream)) == (name, 1, 101) and gpus["current"] == current


@pytest.mark.parametrize("name", NAMES)
def test_given_stream(gpus, name):
    calls(Stream(1, 77))[name]()
    got, where, stream = gpus["calls"].pop()
    assert (got, where, handle(stream)) == (name, 1, 77) and gpus["current"] == 0
    with pytest.raises(ValueError, match="stream"):
        calls(Stream(0, 77))[name]()
    assert not gpus["calls"]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_on_no_gpu(gpus, name):
    with pytest.raises(ValueError, match="GPU"):
        calls(index=-1)[name]()
    assert not gpus["calls"]
