"""Calls of the operators at a model's ends and of the gated linear recurrence run on their
tensors' GPU, whichever is the current one, and name the arguments that are missing.  GPUs
are stood in for by tensors that say where they are, so these run without any."""
import pytest
import torch

import paper_2509_25223_amd as rla
from paper_2509_25223_amd import layer, model
from tests.test_layer_devices import OnGPU, Stream, gpus  # noqa: F401


@pytest.fixture
def two(gpus, monkeypatch):  # noqa: F811
    monkeypatch.setattr(model, "torch", torch)
    monkeypatch.setattr(model, "_bound", layer._bound)
    monkeypatch.setattr(model, "_new", layer._new)
    return gpus


ids, row = OnGPU(2, 3, dtype=torch.int64), OnGPU(2, 3)
table, x, A = OnGPU(9, 8), OnGPU(2, 3, 8), OnGPU(8)
CALLS = {
    "rla_embed_forward": dict(ids=ids, table=table),
    "rla_embed_backward": dict(ids=ids, dout=x, vocab=9),
    "rla_logprob_forward": dict(logits=x),
    "rla_logprob_backward": dict(logits=x, lse=row),
    "rla_glr_forward": dict(x=x, r=x, A=A),
    "rla_glr_backward": dict(x=x, r=x, A=A, dO=x),
    "rla_glr_decode": dict(x=x, r=x, A=A),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_current_stream(two, name):
    getattr(rla, name)(**CALLS[name])
    assert two["calls"] == [(name, 1, 0)] and two["current"] == 0
    two["current"] = 1   # the tensors' own is the current one
    getattr(rla, name)(**CALLS[name])
    assert two["calls"][1:] == [(name, 1, 0)] and two["current"] == 1


@pytest.mark.parametrize("name", list(CALLS))
def test_given_stream(two, name):
    getattr(rla, name)(**CALLS[name], stream=Stream(1, 77))
    assert two["calls"] == [(name, 1, 77)] and two["current"] == 0
    with pytest.raises(ValueError, match="stream"):
        getattr(rla, name)(**CALLS[name], stream=Stream(0))
    assert len(two["calls"]) == 1 and two["current"] == 0


@pytest.mark.parametrize("name", list(CALLS))
def test_status(two, name):
    two["status"] = 2
    with pytest.raises(rla.RLAError):
        getattr(rla, name)(**CALLS[name])
    assert two["current"] == 0


@pytest.mark.parametrize("name,missing", [(n, m) for n, args in CALLS.items() for m in args])
def test_missing(two, name, missing):
    with pytest.raises(ValueError, match=missing):
        getattr(rla, name)(**dict(CALLS[name], **{missing: None}))
    assert not two["calls"]


@pytest.mark.parametrize("name,args,match", [
    ("rla_embed_forward", dict(ids=OnGPU(4, dtype=torch.int32, index=0)), "table"),
    ("rla_embed_backward", dict(dout=OnGPU(2, 3, 8, index=0)), "dout"),
    ("rla_logprob_forward", dict(targets=OnGPU(2, 3, dtype=torch.int64, index=0)), "targets"),
    ("rla_logprob_backward", dict(lse=OnGPU(2, 3, index=0)), "lse"),
    ("rla_glr_decode", dict(r=OnGPU(2, 3, 8, index=0)), "r must")])
def test_tensors_apart(two, name, args, match):
    with pytest.raises(ValueError, match=match):
        getattr(rla, name)(**dict(CALLS[name], **args))
    assert not two["calls"]


def test_single_tokens_of_packed_rows(two):
    with pytest.raises(ValueError, match="B, T, D"):
        rla.rla_glr_decode(OnGPU(3, 8), OnGPU(3, 8), A)
