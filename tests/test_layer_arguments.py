"""Required arguments that are missing are named, by every call (no GPU needed)."""
import os

import pytest
import torch

import paper_2509_25223_amd as rla
from tests.test_layer_devices import OnGPU


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(rla.LIB_PATH):
        from paper_2509_25223_amd import build
        build.build()


x, w, b, A, row, half = OnGPU(2, 3, 8), OnGPU(8, 4), OnGPU(2, 3, 5), OnGPU(8, 5), OnGPU(8), OnGPU(4)
heads = OnGPU(2, 3, 2, 4)
CALLS = {
    "conv_forward": (rla.rla_conv_forward, dict(x=x, weight=w)),
    "conv_backward": (rla.rla_conv_backward, dict(x=x, weight=w, dy=x)),
    "conv_decode": (rla.rla_conv_decode, dict(x=x, weight=w)),
    "ssm_forward": (rla.rla_ssm_forward, dict(u=x, delta=x, A=A, B=b, C=b)),
    "ssm_backward": (rla.rla_ssm_backward, dict(u=x, delta=x, A=A, B=b, C=b, dO=x)),
    "ssm_decode": (rla.rla_ssm_decode, dict(u=x, delta=x, A=A, B=b, C=b)),
    "addnorm_forward": (rla.rla_addnorm_forward, dict(x=x, weight=row)),
    "addnorm_backward": (rla.rla_addnorm_backward, dict(dn=x, residual_out=x, weight=row)),
    "gatenorm_forward": (rla.rla_gatenorm_forward, dict(x=heads, gate=heads, weight=half)),
    "gatenorm_backward": (rla.rla_gatenorm_backward, dict(dO=heads, x=heads, gate=heads, weight=half)),
}


@pytest.mark.parametrize("name,missing", [(n, m) for n, (_, args) in CALLS.items() for m in args])
def test_missing(name, missing):
    call, args = CALLS[name]
    with pytest.raises(ValueError, match=missing):
        call(**dict(args, **{missing: None}))


@pytest.mark.parametrize("name", ["conv_decode", "ssm_decode"])
def test_single_tokens_of_packed_rows(name):
    call, args = CALLS[name]
    first = next(iter(args))
    with pytest.raises(ValueError, match="B, T, D"):
        call(**dict(args, **{first: OnGPU(3, 8)}))
