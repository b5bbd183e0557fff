"""Embedding lookup and the table's gradient."""
import pytest
import torch

import paper_2509_25223_amd as rla
from tests import layer_reference as lref
from tests import model_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def tokens(how, n, V, g):
    """Ids of n tokens: all over the vocabulary, few rows over and over, one, with gaps."""
    if how == "text":
        ids = (V * torch.rand(n, generator=g) ** 4).long().clamp(max=V - 1)
    elif how == "spread":
        ids = torch.randint(V, (n,), generator=g)
    elif how == "one":
        ids = torch.full((n,), V // 2)
    elif how == "none":
        ids = torch.full((n,), -1)
    else:   # outside the table, at its ends, and far outside
        ids = torch.randint(-3, V + 3, (n,), generator=g)
        ids[torch.rand(n, generator=g) < 0.1] = 1 << 30
        ids[torch.rand(n, generator=g) < 0.1] = -(1 << 30)
    return ids


@pytest.mark.parametrize("table,out", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("n,V,D,scale", [(1, 1, 1, 1.0), (5, 7, 8, -0.3), (37, 100, 33, 45.25), (300, 1000, 520, 1.0),
                                         (0, 5, 8, 1.0)])
@pytest.mark.parametrize("wide", [False, True])
def test_lookup(device, table, out, n, V, D, scale, wide):
    """The product in fp32, rounded once: the same bits."""
    g = torch.Generator().manual_seed(n)
    ids = tokens("gaps", n, V, g).to(device, torch.int64 if wide else torch.int32)
    t = torch.randn(V, D, generator=g).to(TYPES[table]).to(device)
    got = rla.rla_embed_forward(ids, t, scale=scale, out_dtype=TYPES[out])
    known = (ids >= 0) & (ids < V)
    want = torch.where(known[:, None], torch.tensor(scale, device=device) * t[ids.long().clamp(0, V - 1)].float(), 0.0)
    assert got.dtype == TYPES[out] and torch.equal(got, want.to(TYPES[out]))
    into = torch.full_like(got, float("nan"))
    assert rla.rla_embed_forward(ids, t, scale=scale, out=into) is into and torch.equal(into, got)
    if n:
        a = ref.embed(ids.cpu(), t.cpu().double(), scale)
        lref.check("out", got, a)


def test_lookup_shape(device):
    """[B, T] ids, beyond the caches' size too; a row of infinities and NaN where no token points."""
    t = torch.randn(3000, 2048, device=device)
    t[17] = float("nan")
    ids = torch.randint(18, 3000, (5, 6000), device=device)
    got = rla.rla_embed_forward(ids, t, scale=2.0, out_dtype=torch.bfloat16)
    assert got.shape == (5, 6000, 2048) and torch.equal(got, (2.0 * t[ids]).bfloat16())


def grad(ids, dout, V, scale, base):
    """The gradient in 64 bits, and the bound: a sum of c products each rounded once, in any
    order, then the factor and the base: (c + 3) half steps of the terms' magnitudes."""
    known = (ids >= 0) & (ids < V)
    want = torch.zeros(V, dout.shape[-1], dtype=torch.float64)
    size, count = want.clone(), torch.zeros(V, 1, dtype=torch.float64)
    d = dout.cpu().double()[known]
    want.index_add_(0, ids[known], d * scale)
    size.index_add_(0, ids[known], (d * scale).abs())
    count.index_add_(0, ids[known], torch.ones(len(d), 1, dtype=torch.float64))
    if base is not None:
        want, size = want + base.cpu().double(), size + base.cpu().double().abs()
    return want, (count + 3) * 2.0 ** -24 * size


def check_grad(got, ids, dout, V, scale, base):
    want, allowed = grad(ids.cpu(), dout, V, scale, base)
    off = (got.cpu().double() - want).abs() - allowed
    assert got.shape == want.shape and torch.isfinite(got).all() and off.max().item() <= 0, off.max().item()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("how", ["text", "spread", "one", "none", "gaps"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (7, 3, 5), (16, 40, 64), (33, 100, 130), (257, 50, 24), (1000, 700, 264),
                                   (1025, 5000, 40), (3000, 129, 2056)])
def test_gradient(device, dtype, how, n, V, D):
    g = torch.Generator().manual_seed(n + D)
    ids = tokens(how, n, V, g).to(device)
    dout = torch.randn(n, D, generator=g).to(TYPES[dtype]).to(device)
    for scale, base in ((1.0, None), (-2.5, torch.randn(V, D, generator=g).to(device))):
        got = rla.rla_embed_backward(ids, dout, V, scale=scale, base=base)
        check_grad(got, ids, dout, V, scale, base)
        again = rla.rla_embed_backward(ids.int(), lref.strided(dout, 1), V, scale=scale, base=base)
        assert torch.equal(got, again)
    # in place: the same where tokens point, nothing elsewhere
    own = base.clone()
    poison = torch.ones(V, dtype=torch.bool, device=device)
    poison[ids[(ids >= 0) & (ids < V)]] = False
    own[poison] = float("nan")
    assert rla.rla_embed_backward(ids, dout, V, scale=scale, base=own, dtable=own) is own
    assert torch.equal(own[~poison], got[~poison]) and own[poison].isnan().all()


@pytest.mark.parametrize("n,V,D", [(65536, 300, 8), (70001, 40000, 12), (200000, 7, 4), (20000, 131072, 64),
                                   (40000, (1 << 22) - 1, 1)])
def test_many_tokens(device, n, V, D):
    """Larger tiles, runs over many chunks, all digits of the ids."""
    g = torch.Generator().manual_seed(V)
    ids = torch.where(torch.rand(n, generator=g) < 0.3, V - 1, tokens("text", n, V, g)).to(device)
    dout = torch.randn(n, D, generator=g).to(device)
    check_grad(rla.rla_embed_backward(ids, dout, V), ids, dout, V, 1.0, None)


def test_more_than_a_slice(device):
    """Tokens beyond a slice are added to those before."""
    n, V, D = (1 << 22) + 4097, 1000, 4
    g = torch.Generator().manual_seed(0)
    ids = tokens("spread", n, V, g).to(device)
    dout = torch.randn(n, D, generator=g).to(device)
    base = torch.randn(V, D, generator=g).to(device)
    check_grad(rla.rla_embed_backward(ids, dout, V, base=base), ids, dout, V, 1.0, base)


def test_rows_apart(device):
    """NaN and infinities reach their own id's row only; large tables are written past the caches."""
    V, D, n = 40000, 700, 500
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(V, (n,), generator=g).to(device)
    dout = torch.randn(n, D, generator=g).to(device)
    want = rla.rla_embed_backward(ids, dout, V)
    dout[100], dout[200] = float("nan"), float("inf")
    got = rla.rla_embed_backward(ids, dout, V)
    bad = torch.zeros(V, dtype=torch.bool, device=device)
    bad[ids[[100, 200]]] = True
    assert torch.equal(got[~bad], want[~bad]) and not torch.isfinite(got[bad]).any()
    untouched = torch.ones(V, dtype=torch.bool, device=device)
    untouched[ids] = False
    assert (got[untouched] == 0).all()


def test_differences(device):
    """<dout, out> along a direction of the table: linear, so the gradient's product with it."""
    g = torch.Generator().manual_seed(2)
    ids = tokens("gaps", 400, 60, g).to(device)
    dout, way = torch.randn(400, 48, generator=g).to(device), torch.randn(60, 48, generator=g).to(device)
    got = rla.rla_embed_backward(ids, dout, 60, scale=0.7)
    out = rla.rla_embed_forward(ids, way, scale=0.7)
    parts = got.double() * way.double()
    assert abs((out.double() * dout.double()).sum() - parts.sum()) <= 2.0 ** -20 * parts.abs().sum()


BAD = {
    "ids type": (dict(ids=lambda t: t.float()), TypeError, "ids"),
    "ids layout": (dict(ids=lambda t: t.repeat(2)[::2]), ValueError, "ids"),
    "table": (dict(table=lambda t: t[0]), ValueError, "table"),
    "table type": (dict(table=lambda t: t.double()), TypeError, "table"),
    "table layout": (dict(table=lambda t: t.t().contiguous().t()), ValueError, "table"),
    "table device": (dict(table=lambda t: t.cpu()), ValueError, "table"),
    "out type": (dict(out_dtype=lambda t: torch.float16), TypeError, "out"),
    "out shape": (dict(out=lambda t: torch.empty(9, 8, device="cuda")), ValueError, "out"),
}


@pytest.mark.parametrize("case", list(BAD))
def test_refused(device, case):
    change, error, match = BAD[case]
    args = dict(ids=torch.zeros(10, dtype=torch.int64, device=device), table=torch.zeros(5, 8, device=device), out_dtype=None,
                out=None)
    args.update({n: f(args[n]) for n, f in change.items()})
    with pytest.raises(error, match=match):
        rla.rla_embed_forward(**args)


def test_refused_gradients(device):
    ids, dout = torch.zeros(10, dtype=torch.int64, device=device), torch.zeros(10, 8, device=device)
    f = rla.rla_embed_backward
    with pytest.raises(ValueError, match="dout"):
        f(ids, dout[:9], 5)
    with pytest.raises(ValueError, match="base"):
        f(ids, dout, 5, base=torch.zeros(4, 8, device=device))
    with pytest.raises(TypeError, match="dtable"):
        f(ids, dout, 5, dtable=torch.zeros(5, 8, device=device, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="workspace"):
        f(ids, dout, 5, workspace=torch.empty(16, dtype=torch.uint8, device=device))
    for bad in (dict(vocab=0), dict(vocab=1 << 22), dict(vocab=5, scale=float("nan"))):
        with pytest.raises((rla.RLAError, ValueError)):
            f(ids, torch.zeros(10, 1, device=device), **bad, dtable=None)


def test_numbers_in_tensors(device):
    """A scale given as a tensor counts as what it holds when the call is made."""
    table, ids = torch.randn(10, 8, device=device), torch.arange(10, device=device)
    scale = torch.tensor(0.5)
    assert torch.equal(rla.rla_embed_forward(ids, table, scale), 0.5 * table)
    scale.fill_(2.0)
    assert torch.equal(rla.rla_embed_forward(ids, table, scale), 2 * table)
    assert torch.equal(rla.rla_embed_backward(ids, table, torch.tensor(10), scale), 2 * table)


@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("V", [1, 5, 40000, (1 << 22) - 1])
@pytest.mark.parametrize("n", [1, 31, 33, 64, 65, 129, 2047, 6144, 6145, 8192, 8193])
def test_places(device, n, V, wide):
    """Few tokens, whose places are counted, and the first that are sorted: sums are of whole
    numbers, so that any order gives the same."""
    D = 3 if V > 50000 else 12
    g = torch.Generator(device).manual_seed(n + V)
    ids = torch.randint(-1, V + 1, (n,), device=device, generator=g)
    ids[n // 2:] = torch.where(torch.rand(n - n // 2, device=device, generator=g) < 0.3, ids[n // 2], ids[n // 2:])
    dout = torch.randint(-8, 9, (n, D), device=device, generator=g).float()
    there = (ids >= 0) & (ids < V)
    want = torch.zeros(V, D, dtype=torch.float64, device=device).index_add_(0, ids[there], dout[there].double()).float()
    given = ids if wide else ids.int()
    table = torch.full((V, D), float("nan"), device=device)
    assert torch.equal(rla.rla_embed_backward(given, dout, V, dtable=table), want)
    base = torch.randint(-99, 99, (V, D), device=device, generator=g).float()
    assert torch.equal(rla.rla_embed_backward(given, dout.bfloat16(), V, base=base), want + base)
    assert torch.equal(rla.rla_embed_backward(given, dout, V, scale=2.0, base=base, dtable=base.clone()), 2 * want + base)
    same = base.clone()
    assert torch.equal(rla.rla_embed_backward(given, dout, V, base=same, dtable=same), want + base)
