"""The C entry points around a mixing layer: exported as declared, and every bad
argument refused on the host before any HIP call (so these run without a GPU)."""
import os
import re

import pytest

import paper_2509_25223_amd as rla
from paper_2509_25223_amd import layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000
NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE, VALUE = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rla.LIB_PATH):
        from paper_2509_25223_amd import build
        build.build()
    return layer._lib()


def test_exports(lib):
    text = open(os.path.join(ROOT, "include", "rla_layer.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(rla_[a-z_]+)\s*\(", text))
    assert names == set(rla.LAYER_SYMBOLS)
    assert all(hasattr(lib, n) for n in names)


def conv(**kw):
    f = dict(batch=2, seq_len=10, channels=24, taps=4, silu=1, dtype=rla.RLA_BF16)
    f.update(kw)
    return rla.rla_conv_problem(**f)


def test_conv(lib):
    def fwd(p, x=FAKE, w=FAKE, s=None, y=FAKE, f=None, ws=None, n=0):
        return lib.rla_conv_forward(p, x, w, None, s, y, f, ws, n, None)

    def bwd(p, dy=FAKE, dx=FAKE, dw=FAKE, ws=FAKE, n=1 << 40):
        return lib.rla_conv_backward(p, FAKE, FAKE, None, None, dy, None, dx, dw, None, None, ws, n, None)

    def dec(p, s=FAKE, y=FAKE, o=FAKE):
        return lib.rla_conv_decode(p, FAKE, FAKE, None, s, y, o, None)

    assert fwd(None) == NULL
    for bad, want in [(dict(taps=1), SHAPE), (dict(taps=5), SHAPE), (dict(channels=0), SHAPE), (dict(batch=-1), SHAPE),
                      (dict(seq_len=1 << 40), SHAPE), (dict(dtype=7), DTYPE), (dict(silu=2), VALUE),
                      (dict(x_stride=8), SHAPE), (dict(x_stride=-24), SHAPE), (dict(x_stride=1 << 60), SHAPE),
                      (dict(cu_seqlens=FAKE), SHAPE), (dict(batch=1, cu_seqlens=FAKE, num_seqs=-1), SHAPE)]:
        assert fwd(conv(**bad)) == want, bad
        assert rla.rla_conv_workspace_size(conv(**bad)) == 0
    p = conv()
    assert fwd(p, x=None) == NULL and fwd(p, w=None) == NULL and fwd(p, y=None) == NULL
    assert fwd(p, x=FAKE + 1) == VALUE and fwd(p, f=FAKE + 1) == VALUE
    assert fwd(p, s=FAKE, f=FAKE) == VALUE   # initial and final states overlap
    packed = conv(batch=1, cu_seqlens=FAKE, num_seqs=3)
    need = rla.rla_conv_workspace_size(packed, False)
    assert fwd(packed) == WORKSPACE and fwd(packed, ws=FAKE, n=need - 1) == WORKSPACE
    assert fwd(packed, ws=FAKE + 16, n=need) == VALUE
    assert bwd(p, dy=None) == NULL and bwd(p, dx=None) == NULL and bwd(p, dw=None) == NULL
    assert bwd(p, ws=None) == WORKSPACE and bwd(p, n=8) == WORKSPACE and bwd(p, ws=FAKE + 64) == VALUE
    assert 0 < need < rla.rla_conv_workspace_size(packed, True)
    assert dec(packed) == UNSUPPORTED and dec(p, o=None) == NULL and dec(p, o=FAKE + 8) == VALUE
    assert dec(conv(batch=0)) == 0


def ssm(**kw):
    f = dict(batch=2, seq_len=10, channels=24, states=16, groups=1, softplus=1, dtype=rla.RLA_BF16)
    f.update(kw)
    return rla.rla_ssm_problem(**f)


def test_ssm(lib):
    def fwd(p, u=FAKE, A=FAKE, o=FAKE, h=None, f=None, save=0, ws=FAKE, n=1 << 40):
        return lib.rla_ssm_forward(p, u, FAKE, A, FAKE, FAKE, None, None, None, h, o, f, save, ws, n, None)

    def bwd(p, skip=None, z=None, bias=None, dO=FAKE, dA=FAKE, dskip=None, dz=None, dbias=None, ws=FAKE, n=1 << 40):
        return lib.rla_ssm_backward(p, FAKE, FAKE, FAKE, FAKE, FAKE, skip, z, bias, None, dO, None, FAKE, FAKE, dA,
                                    FAKE, FAKE, dskip, dz, dbias, None, 0, ws, n, None)

    def dec(p, h=FAKE, o=FAKE, out=FAKE):
        return lib.rla_ssm_decode(p, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None, h, o, out, None)

    assert fwd(None) == NULL
    for bad, want in [(dict(states=0), SHAPE), (dict(states=65), SHAPE), (dict(groups=0), SHAPE),
                      (dict(groups=5), SHAPE), (dict(channels=0), SHAPE), (dict(dtype=-1), DTYPE),
                      (dict(softplus=3), VALUE), (dict(b_stride=8), SHAPE), (dict(z_stride=-24), SHAPE),
                      (dict(seq_len=1 << 33), SHAPE), (dict(cu_seqlens=FAKE), SHAPE)]:
        assert fwd(ssm(**bad)) == want, bad
        assert rla.rla_ssm_workspace_size(ssm(**bad), rla.RLA_SSM_BACKWARD) == 0
    p = ssm(seq_len=4000)
    assert rla.rla_ssm_workspace_size(p, 7) == 0
    need = rla.rla_ssm_workspace_size(p, rla.RLA_SSM_FORWARD)
    assert 0 < need < rla.rla_ssm_workspace_size(p, rla.RLA_SSM_BACKWARD)
    assert fwd(p, u=None) == NULL and fwd(p, A=None) == NULL and fwd(p, o=None) == NULL
    assert fwd(p, u=FAKE + 1) == VALUE and fwd(p, A=FAKE + 2) == VALUE
    assert fwd(p, h=FAKE, f=FAKE + 64) == VALUE
    assert fwd(p, ws=None) == WORKSPACE and fwd(p, n=need - 1) == WORKSPACE and fwd(p, save=1, n=need) == WORKSPACE
    assert fwd(p, ws=FAKE + 8) == VALUE
    assert bwd(p, dO=None) == NULL and bwd(p, dA=None) == NULL
    assert bwd(p, skip=FAKE) == NULL and bwd(p, z=FAKE) == NULL and bwd(p, bias=FAKE) == NULL
    assert bwd(p, n=need) == WORKSPACE
    assert dec(ssm(batch=1, cu_seqlens=FAKE, num_seqs=1)) == UNSUPPORTED
    assert dec(p, o=None) == NULL and dec(p, out=None) == NULL and dec(p, out=FAKE + 64) == VALUE
    assert dec(ssm(batch=0)) == 0


def test_norms(lib):
    def add(**kw):
        f = dict(rows=4, width=24, dtype=rla.RLA_BF16, residual_dtype=rla.RLA_F32, eps=1e-6)
        f.update(kw)
        return rla.rla_addnorm_problem(**f)

    def gate(**kw):
        f = dict(tokens=4, heads=2, width=24, dtype=rla.RLA_BF16, x_dtype=rla.RLA_F32, eps=1e-6)
        f.update(kw)
        return rla.rla_gatenorm_problem(**f)

    def afwd(p, x=FAKE, r=None, o=FAKE):
        return lib.rla_addnorm_forward(p, x, r, FAKE, None, FAKE, o, None)

    def abwd(p, dn=FAKE, x=None, scale=None, ds=None, ws=FAKE, n=1 << 40):
        return lib.rla_addnorm_backward(p, dn, None, FAKE, x, FAKE, scale, FAKE, None, FAKE, ds, ws, n, None)

    def gfwd(p, x=FAKE, g=FAKE):
        return lib.rla_gatenorm_forward(p, x, g, FAKE, FAKE, None)

    def gbwd(p, dO=FAKE, ws=FAKE, n=1 << 40):
        return lib.rla_gatenorm_backward(p, dO, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, ws, n, None)

    assert afwd(None) == NULL and gfwd(None) == NULL
    nan = float("nan")
    for bad, want in [(dict(rows=-1), SHAPE), (dict(width=0), SHAPE), (dict(eps=-1.0), VALUE), (dict(eps=nan), VALUE),
                      (dict(dtype=9), DTYPE), (dict(dtype=rla.RLA_F32, residual_dtype=rla.RLA_BF16), DTYPE),
                      (dict(x_stride=3), SHAPE), (dict(rows=1 << 40), SHAPE)]:
        assert afwd(add(**bad)) == want, bad
        assert rla.rla_addnorm_workspace_size(add(**bad)) == 0
    p = add()
    assert afwd(p, x=None) == NULL and afwd(p, o=None) == NULL and afwd(p, x=FAKE + 1) == VALUE
    assert afwd(p, r=FAKE + 4) == VALUE   # a stream that overlaps its output in part
    assert abwd(p, dn=None) == NULL and abwd(p, scale=FAKE) == NULL and abwd(p, scale=FAKE, ds=FAKE) == NULL
    assert abwd(p, ws=None) == WORKSPACE and abwd(p, n=16) == WORKSPACE and abwd(p, ws=FAKE + 4) == VALUE
    assert afwd(add(rows=0)) == 0
    for bad, want in [(dict(tokens=-1), SHAPE), (dict(heads=0), SHAPE), (dict(width=0), SHAPE), (dict(eps=nan), VALUE),
                      (dict(dtype=rla.RLA_F32, x_dtype=rla.RLA_BF16), DTYPE), (dict(gate_first=2), VALUE),
                      (dict(weight_per_head=5), VALUE), (dict(gate_stride=24), SHAPE), (dict(tokens=1 << 31), SHAPE)]:
        assert gfwd(gate(**bad)) == want, bad
        assert rla.rla_gatenorm_workspace_size(gate(**bad)) == 0
    p = gate()
    assert gfwd(p, x=None) == NULL and gfwd(p, g=FAKE + 1) == VALUE and gfwd(p, x=FAKE + 2) == VALUE
    assert gbwd(p, dO=None) == NULL and gbwd(p, ws=None) == WORKSPACE and gbwd(p, n=1) == WORKSPACE
    assert gfwd(gate(tokens=0)) == 0
