"""The C entry points at a model's ends and of the gated linear recurrence: exported as
declared, and every bad argument refused on the host before any HIP call (so
these run without a GPU)."""
import os
import re

import pytest

import paper_2509_25223_amd as rla
from paper_2509_25223_amd import model

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, APART = 0x7f0000000000, 1 << 40
NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE, VALUE = 1, 2, 3, 4, 5, 6
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rla.LIB_PATH):
        from paper_2509_25223_amd import build
        build.build()
    return model._lib()


def at(k):
    """Arrays apart from each other."""
    return FAKE + k * APART


def test_exports(lib):
    text = open(os.path.join(ROOT, "include", "rla_model.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(rla_[a-z_]+)\s*\(", text))
    assert names == set(rla.MODEL_SYMBOLS)
    assert all(hasattr(lib, n) for n in names)


def test_embed(lib):
    def make(**kw):
        return rla.rla_embed_problem(**dict(dict(tokens=10, vocab=50, width=24, index=1, dtype=rla.RLA_BF16,
                                                 table_dtype=rla.RLA_F32, scale=1.0), **kw))

    def fwd(p, ids=at(0), table=at(1), out=at(2)):
        return lib.rla_embed_forward(p, ids, table, out, None)

    def bwd(p, ids=at(0), dout=at(1), base=None, dtable=at(2), ws=at(3), n=1 << 40):
        return lib.rla_embed_backward(p, ids, dout, base, dtable, ws, n, None)

    assert fwd(None) == NULL and bwd(None) == NULL
    for bad, want in [(dict(tokens=-1), SHAPE), (dict(tokens=1 << 31), SHAPE), (dict(vocab=0), SHAPE),
                      (dict(vocab=1 << 31), SHAPE), (dict(width=0), SHAPE), (dict(width=(1 << 20) + 1), SHAPE),
                      (dict(dout_stride=23), SHAPE), (dict(dout_stride=-24), SHAPE), (dict(dout_stride=1 << 61), SHAPE),
                      (dict(index=2), DTYPE), (dict(dtype=2), DTYPE), (dict(table_dtype=-1), DTYPE),
                      (dict(scale=NAN), VALUE), (dict(scale=INF), VALUE)]:
        assert fwd(make(**bad)) == want and bwd(make(**bad)) == want, bad
        assert rla.rla_embed_workspace_size(make(**bad)) == 0
    p = make()
    for name in ("ids", "table", "out"):
        assert fwd(p, **{name: None}) == NULL
    assert fwd(p, ids=at(0) + 4) == VALUE and fwd(p, table=at(1) + 2) == VALUE and fwd(p, out=at(2) + 1) == VALUE
    assert fwd(p, out=at(1) + 64) == VALUE and fwd(p, out=at(0)) == VALUE      # over the table, over the ids
    assert fwd(make(tokens=0), ids=None) == 0
    assert bwd(make(vocab=1 << 22)) == SHAPE                                    # gradients: fewer rows
    assert rla.rla_embed_workspace_size(make(vocab=(1 << 22) - 1)) > 0
    for name in ("ids", "dout", "dtable"):
        assert bwd(p, **{name: None}) == NULL
    assert bwd(p, base=at(2) + 4) == VALUE and bwd(p, dout=at(2)) == VALUE and bwd(p, dtable=at(0)) == VALUE
    assert bwd(p, dtable=at(2) + 2) == VALUE
    need = rla.rla_embed_workspace_size(p)
    assert bwd(p, ws=None) == WORKSPACE and bwd(p, n=need - 1) == WORKSPACE and bwd(p, ws=at(3) + 8) == VALUE
    # the workspace grows with the tokens up to a slice, then not
    sizes = [rla.rla_embed_workspace_size(make(tokens=n)) for n in (1, 1000, 1 << 20, 1 << 22, 1 << 24)]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2]


def test_logprob(lib):
    def make(**kw):
        return rla.rla_logprob_problem(**dict(dict(rows=6, vocab=50, index=1, dtype=rla.RLA_F32, top=0, scale=1.0), **kw))

    def fwd(p, x=at(0), y=at(1), lp=at(2), lse=at(3), H=at(4), tl=None, ti=None, ws=None, n=0):
        return lib.rla_logprob_forward(p, x, y, lp, lse, H, tl, ti, ws, n, None)

    def bwd(p, x=at(0), y=at(1), lse=at(2), H=None, g=at(3), e=None, dx=at(4)):
        return lib.rla_logprob_backward(p, x, y, lse, H, g, e, dx, None)

    assert fwd(None) == NULL and bwd(None) == NULL
    for bad, want in [(dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(vocab=0), SHAPE),
                      (dict(vocab=(1 << 30) + 1), SHAPE), (dict(top=-1), SHAPE), (dict(top=65, vocab=100), SHAPE),
                      (dict(top=51), SHAPE), (dict(logits_stride=49), SHAPE), (dict(logits_stride=1 << 61), SHAPE),
                      (dict(index=-1), DTYPE), (dict(dtype=3), DTYPE), (dict(scale=0.0), VALUE), (dict(scale=-1.0), VALUE),
                      (dict(scale=NAN), VALUE), (dict(scale=INF), VALUE)]:
        assert fwd(make(**bad)) == want and bwd(make(**bad)) == want, bad
        assert rla.rla_logprob_workspace_size(make(**bad)) == 0
    p = make()
    assert fwd(p, x=None) == NULL and fwd(p, y=None) == NULL
    assert fwd(make(top=3), tl=at(5)) == NULL and fwd(make(top=3), ti=at(5)) == NULL
    assert fwd(p, x=at(0) + 2) == VALUE and fwd(p, y=at(1) + 4) == VALUE and fwd(p, lse=at(3) + 2) == VALUE
    assert fwd(p, lse=at(0) + 8) == VALUE                                        # an output over the logits
    assert fwd(make(rows=0), x=None) == 0
    wide = make(vocab=100000, top=8)
    need = rla.rla_logprob_workspace_size(wide)
    assert need > 0
    tops = dict(tl=at(5), ti=at(6))
    assert fwd(wide, **tops) == WORKSPACE and fwd(wide, ws=at(7), n=need - 1, **tops) == WORKSPACE
    assert fwd(wide, ws=at(7) + 4, n=need, **tops) == VALUE
    for name in ("x", "lse", "dx", "y"):
        assert bwd(p, **{name: None}) == NULL
    assert bwd(p, e=at(5)) == NULL                                               # the entropy is missing
    assert bwd(p, dx=at(0) + 4) == VALUE                                         # over the logits, in part
    assert bwd(make(logits_stride=60), dx=at(0)) == VALUE                        # in place, but rows apart
    assert bwd(p, dx=at(2)) == VALUE and bwd(p, dx=at(4) + 2) == VALUE
    assert bwd(make(rows=0), x=None) == 0


def test_glr(lib):
    def make(**kw):
        return rla.rla_glr_problem(**dict(dict(batch=2, seq_len=10, channels=24, normalize=1, dtype=rla.RLA_BF16), **kw))

    def fwd(p, x=FAKE, r=FAKE, A=FAKE, i=None, h=None, o=FAKE, f=None, save=0, ws=FAKE, n=1 << 40):
        return lib.rla_glr_forward(p, x, r, A, i, None, h, o, f, save, ws, n, None)

    def bwd(p, i=None, z=None, h=None, dO=FAKE, dh=None, dx=FAKE, dA=FAKE, di=None, dz=None, dh0=None, ws=FAKE, n=1 << 40):
        return lib.rla_glr_backward(p, FAKE, FAKE, FAKE, i, z, h, dO, dh, dx, FAKE, dA, di, dz, dh0, 0, ws, n, None)

    def dec(p, h=FAKE, o=FAKE, out=FAKE):
        return lib.rla_glr_decode(p, FAKE, FAKE, FAKE, None, None, h, o, out, None)

    assert fwd(None) == NULL
    for bad, want in [(dict(channels=0), SHAPE), (dict(channels=1 << 23), SHAPE), (dict(batch=-1), SHAPE),
                      (dict(seq_len=1 << 33), SHAPE), (dict(dtype=-1), DTYPE), (dict(normalize=2), VALUE),
                      (dict(x_stride=8), SHAPE), (dict(z_stride=-24), SHAPE), (dict(do_stride=1 << 61), SHAPE), (dict(r_stride=1 << 23), SHAPE),
                      (dict(cu_seqlens=FAKE), SHAPE), (dict(batch=1, cu_seqlens=FAKE, num_seqs=-1), SHAPE)]:
        assert fwd(make(**bad)) == want, bad
        assert rla.rla_glr_workspace_size(make(**bad), rla.RLA_GLR_BACKWARD) == 0
    p = make(batch=1, seq_len=4000)
    assert rla.rla_glr_workspace_size(p, 7) == 0
    need = rla.rla_glr_workspace_size(p, rla.RLA_GLR_FORWARD)
    assert 0 < need < rla.rla_glr_workspace_size(p, rla.RLA_GLR_BACKWARD)
    assert fwd(p, x=None) == NULL and fwd(p, r=None) == NULL and fwd(p, A=None) == NULL and fwd(p, o=None) == NULL
    assert fwd(p, x=FAKE + 1) == VALUE and fwd(p, A=FAKE + 2) == VALUE and fwd(p, i=FAKE + 1) == VALUE
    assert fwd(p, h=FAKE, f=FAKE + 64) == VALUE
    assert fwd(p, ws=None) == WORKSPACE and fwd(p, n=need - 1) == WORKSPACE and fwd(p, save=1, n=need) == WORKSPACE
    assert fwd(p, ws=FAKE + 8) == VALUE
    assert bwd(p, dO=None) == NULL and bwd(p, dA=None) == NULL and bwd(p, dx=None) == NULL
    assert bwd(p, i=FAKE) == NULL and bwd(p, z=FAKE) == NULL
    assert bwd(p, dh=FAKE, dh0=FAKE) == VALUE and bwd(p, h=FAKE, dh0=FAKE) == VALUE
    assert bwd(p, n=need) == WORKSPACE
    assert dec(make(batch=1, cu_seqlens=FAKE, num_seqs=1)) == UNSUPPORTED
    assert dec(p, o=None) == NULL and dec(p, out=None) == NULL and dec(p, out=FAKE + 64) == VALUE
    assert dec(make(batch=0)) == 0


def test_sizes_beyond_a_launch(lib):
    """Single tokens of more workgroups than a launch holds are refused as a shape."""
    for batch, want in ((1 << 29, SHAPE), (1 << 26, NULL)):
        p = rla.rla_glr_problem(batch=batch, seq_len=1, channels=64, normalize=1, dtype=rla.RLA_BF16)
        assert lib.rla_glr_decode(p, FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, None) == want


def test_scale_in_base_2(lib):
    """A scale that times log2 e leaves fp32 is refused."""
    for scale, want in ((3e38, VALUE), (2e38, NULL)):
        p = rla.rla_logprob_problem(rows=1, vocab=5, index=1, dtype=rla.RLA_F32, top=0, scale=scale)
        assert lib.rla_logprob_forward(p, None, FAKE, FAKE, None, None, None, None, None, 0, None) == want


def overlaps(call, outputs, inputs):
    """Each output over each input, at its start and its last value, and over each other output: refused.  (All calls
    here are: none reaches the GPU with these addresses.)"""
    for out, el in outputs:
        for other, offset in [(n, o) for n, last in inputs for o in {0, last}] + [(n, 0) for n, _ in outputs if n != out]:
            assert call(**{out: (other, offset)}) == VALUE, (out, other, offset)


def test_glr_overlaps(lib):
    """Outputs of the recurrence over what it reads, or over each other, strided rows and packed offsets among
    them."""
    names = ("x", "r", "A", "i", "z", "h", "dO", "dh", "cu", "o", "f", "dx", "dr", "dA", "di", "dz", "dh0")
    base = {n: at(k) for k, n in enumerate(names)}
    tokens, D, S, N = 10, 24, 40, 3
    last = 2 * ((tokens - 1) * S + D - 1)   # bytes to the last value of strided rows

    def call(which, **over):
        where = dict(base)
        for n, (other, offset) in over.items():
            where[n] = base[other] + offset
        a = where.__getitem__
        p = rla.rla_glr_problem(batch=1, seq_len=tokens, channels=D, num_seqs=N, cu_seqlens=a("cu"), x_stride=S, r_stride=S,
                                i_stride=S, z_stride=S, do_stride=S, normalize=1, dtype=rla.RLA_BF16)
        ws = (FAKE >> 1, 1 << 40)
        if which == "forward":
            return lib.rla_glr_forward(p, a("x"), a("r"), a("A"), a("i"), a("z"), a("h"), a("o"), a("f"), 0, *ws, None)
        return lib.rla_glr_backward(p, a("x"), a("r"), a("A"), a("i"), a("z"), a("h"), a("dO"), a("dh"), a("dx"), a("dr"),
                                    a("dA"), a("di"), a("dz"), a("dh0"), 0, *ws, None)

    read = [("x", last), ("r", last), ("i", last), ("z", last), ("A", 4 * (D - 1)), ("h", 4 * (N * D - 1)), ("cu", 4 * N)]
    overlaps(lambda **o: call("forward", **o), [("o", 2), ("f", 4)], [(n, t & ~3) for n, t in read])
    overlaps(lambda **o: call("backward", **o), [(n, 4) for n in ("dx", "dr", "dA", "di", "dz", "dh0")],
             [(n, t & ~3) for n, t in read + [("dO", last), ("dh", 4 * (N * D - 1))]])
    # from the front: an output that ends in an input's first value
    assert call("forward", o=("x", 4 - 2 * tokens * D)) == VALUE and call("forward", f=("r", 4 - 4 * N * D)) == VALUE


def test_glr_decode_overlaps(lib):
    B, D = 5, 24

    def call(x=at(0), r=at(1), A=at(2), i=at(3), z=at(4), h=at(5), o=at(6), out=at(7), S=D):
        p = rla.rla_glr_problem(batch=B, seq_len=1, channels=D, x_stride=S, r_stride=S, i_stride=S, z_stride=S, normalize=1,
                                dtype=rla.RLA_BF16)
        return lib.rla_glr_decode(p, x, r, A, i, z, h, o, out, None)

    for k in (0, 1, 3, 4):
        assert call(o=at(k) + 2) == VALUE and call(o=at(k), S=40) == VALUE and call(out=at(k)) == VALUE
        assert call(o=at(k) - 2 * B * D + 2) == VALUE
    for o in (2, 5, 7):
        assert call(o=at(o)) == VALUE
    assert call(out=at(2)) == VALUE and call(out=at(5) + 4) == VALUE


def test_logprob_overlaps(lib):
    """Outputs of the log probabilities over the tokens, or over each other."""
    names = ("y", "lp", "lse", "H", "tl", "ti")
    base = {n: at(k + 1) for k, n in enumerate(names)}
    p = rla.rla_logprob_problem(rows=6, vocab=50, index=1, dtype=rla.RLA_F32, top=3, scale=1.0)

    def call(**over):
        where = dict(base)
        for n, (other, offset) in over.items():
            where[n] = base[other] + offset
        a = where.__getitem__
        return lib.rla_logprob_forward(p, at(0), a("y"), a("lp"), a("lse"), a("H"), a("tl"), a("ti"), None, 0, None)

    overlaps(call, [(n, 4) for n in names[1:]], [("y", 8 * 6 - 4)])


def test_workspaces_serve_smaller_calls(lib):
    """A workspace sized for a call is enough for one of fewer tokens or rows, however each is cut up."""
    def grows(sizes):
        return all(a <= b for a, b in zip(sizes, sizes[1:]))

    tokens = sorted({*range(1, 200), *range(8150, 8230), *range(65500, 65570), *range(200, 70000, 333), 1 << 17, 1 << 20, 1 << 22})
    for V, D in ((50001, 770), (32768, 2048), (100, 3)):
        assert grows([rla.rla_embed_workspace_size(rla.rla_embed_problem(tokens=n, vocab=V, width=D, index=1, dtype=0,
                                                                         table_dtype=0, scale=1.0)) for n in tokens])
    for V in (50000, 65536, 131072, 200003):
        for dtype in (rla.RLA_F32, rla.RLA_BF16):
            for top in (0, 8):
                assert grows([rla.rla_logprob_workspace_size(rla.rla_logprob_problem(rows=n, vocab=V, index=1, dtype=dtype, top=top,
                                                                                     scale=1.0)) for n in range(0, 600)])
    for D in (64, 514, 4096, 12800):
        for op in (rla.RLA_GLR_FORWARD, rla.RLA_GLR_BACKWARD):
            def size(**kw):
                return rla.rla_glr_workspace_size(rla.rla_glr_problem(channels=D, normalize=1, dtype=rla.RLA_BF16, **kw), op)

            assert grows([size(batch=1, seq_len=n) for n in tokens])
            assert grows([size(batch=1, seq_len=n, cu_seqlens=FAKE, num_seqs=5) for n in tokens])
            for T in (1, 100, 2048, 4096):
                assert grows([size(batch=b, seq_len=T) for b in range(0, 700)])
