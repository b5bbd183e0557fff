"""Sizes beyond what a launch holds (fewer than 2^32 threads) are refused as shapes on the
host, before any HIP call: these run without a GPU."""
import os

import pytest

import paper_2509_25223_amd as rla
from paper_2509_25223_amd import layer

FAKE = 0x7f0000000000
NULL, SHAPE, WORKSPACE = 1, 2, 5


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


def conv(**kw):
    f = dict(batch=1, seq_len=1, channels=4096, taps=4, silu=1, dtype=rla.RLA_BF16)
    f.update(kw)
    return rla.rla_conv_problem(**f)


@pytest.mark.parametrize("size", [dict(batch=1 << 17, seq_len=1 << 10), dict(seq_len=1 << 27), dict(seq_len=1 << 26, dtype=rla.RLA_F32),
                                  dict(seq_len=1 << 27, cu_seqlens=FAKE, num_seqs=100)])
def test_convolution(lib, size):
    p = conv(**size)
    assert rla.rla_conv_workspace_size(p, False) == 0
    assert lib.rla_conv_forward(p, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 50, None) == SHAPE
    # a 32nd less fits: past the shapes, what is missing is the workspace or an output
    p = conv(**dict(size, seq_len=size["seq_len"] * 31 // 32))
    want = WORKSPACE if p.cu_seqlens else NULL
    assert lib.rla_conv_forward(p, FAKE, FAKE, None, None, FAKE if p.cu_seqlens else None, None, None, 0, None) == want


@pytest.mark.parametrize("dtype", [rla.RLA_BF16, rla.RLA_F32])
def test_convolution_gradients(lib, dtype):
    for seq_len, want in ((1 << 27, SHAPE), ((1 << 27) - (1 << 14), WORKSPACE)):
        p = conv(seq_len=seq_len, dtype=dtype)
        assert (rla.rla_conv_workspace_size(p, True) == 0) == (want == SHAPE)
        assert lib.rla_conv_backward(p, FAKE, FAKE, None, None, FAKE, None, FAKE, FAKE, None, None, None, 0, None) == want


def test_convolution_of_single_tokens(lib):
    for batch, want in ((1 << 23, SHAPE), ((1 << 23) - 1, NULL)):
        assert lib.rla_conv_decode(conv(batch=batch), FAKE, FAKE, None, FAKE, None, FAKE, None) == want


def test_workspace_of_few_sequences(lib):
    """Few packed sequences are looked up in place: what the call asks for does not grow with
    the tokens, as the map of many sequences does."""
    def size(n, tokens, backward=False):
        return rla.rla_conv_workspace_size(conv(seq_len=tokens, channels=64, cu_seqlens=FAKE, num_seqs=n), backward)

    assert 0 < size(3, 100) == size(3, 1 << 20) == size(1, 1 << 26)
    assert size(200, 1 << 20) > 4 << 20
    dense = rla.rla_conv_workspace_size(conv(seq_len=1 << 20, channels=64), True)
    assert size(3, 1 << 20, True) - size(3, 1 << 20) == dense
    assert lib.rla_conv_forward(conv(seq_len=100, cu_seqlens=FAKE, num_seqs=3), FAKE, FAKE, None, None, FAKE, None, None,
                                0, None) == WORKSPACE
