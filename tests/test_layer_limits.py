"""Sizes beyond what a launch holds (fewer than 2^32 threads) are refused as shapes on the
host, before any HIP call: these run without a GPU."""
import os

import pytest

import paper_2509_25223_amd as rla
from paper_2509_25223_amd import layer

FAKE = 0x7f0000000000
OK, SHAPE, WORKSPACE = 0, 2, 5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rla.LIB_PATH):
        from paper_2509_25223_amd import build
        build.build()
    return layer._lib()


def ssm(**kw):
    f = dict(batch=2, seq_len=1, channels=64, states=16, groups=1, softplus=1, dtype=rla.RLA_BF16)
    f.update(kw)
    return rla.rla_ssm_problem(**f)


# a workgroup holds 64 channels of up to 16 states, 32 of up to 32, 16 of more
@pytest.mark.parametrize("size", [dict(batch=1 << 24), dict(batch=1 << 20, channels=1024), dict(batch=1 << 23, states=17),
                                  dict(batch=1 << 22, states=64), dict(batch=1 << 18, seq_len=8, channels=4096)])
def test_scan(lib, size):
    p = ssm(**size)
    for op in (rla.RLA_SSM_FORWARD, rla.RLA_SSM_BACKWARD):
        assert rla.rla_ssm_workspace_size(p, op) == 0
    for save in (0, 1):
        assert lib.rla_ssm_forward(p, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None, None, FAKE, None, save, FAKE,
                                   1 << 50, None) == SHAPE
    assert lib.rla_ssm_backward(p, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None, None, FAKE, None, FAKE, FAKE, FAKE,
                                FAKE, FAKE, None, None, None, None, 0, FAKE, 1 << 50, None) == SHAPE
    # one sequence less fits: past the shapes, what is missing is the workspace
    p = ssm(**dict(size, batch=size["batch"] - 1))
    assert rla.rla_ssm_workspace_size(p, rla.RLA_SSM_BACKWARD) > 0
    assert lib.rla_ssm_backward(p, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None, None, FAKE, None, FAKE, FAKE, FAKE,
                                FAKE, FAKE, None, None, None, None, 0, None, 0, None) == WORKSPACE


@pytest.mark.parametrize("size", [dict(batch=(1 << 29) - 1), dict(batch=1 << 28, states=32), dict(batch=1 << 27, states=33),
                                  dict(batch=1 << 26, channels=80, states=64)])
def test_scan_of_single_tokens(lib, size):
    assert lib.rla_ssm_decode(ssm(**size), FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, None) == SHAPE
