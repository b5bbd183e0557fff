"""Log probabilities, entropy and alternatives of rows of logits, and their gradient,
against 64 bits."""
import pytest
import torch

import paper_2509_25223_amd as rla
from tests import layer_reference as lref
from tests import model_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = 2.0 ** -24
NEG = float("-inf")

# Bounds.  A row's sum of exponentials has positive terms, each off by a few half steps and by
# |z - max| of them (weighted by the terms at most the entropy, < 12); up to 64 are added one after the
# other, then over lanes, waves and parts, at most 16 more: 128 half steps of log s, and rounding of
# lse itself.  The entropy's terms have one sign and sum to at most the entropy.


def close(name, got, want, allowed):
    got, want = got.detach().cpu().double(), want.detach().cpu()
    assert got.shape == want.shape, name
    same = (got == want) | (got.isnan() & want.isnan())
    off = torch.where(same, torch.zeros_like(got), (got - want).abs() - allowed)
    assert not off.numel() or off.max().item() <= 0, "%s: %.3e over the bound" % (name, off.max().item())


def check_forward(got, want, top, entropy=True):
    lse = want["lse"].abs().nan_to_num(posinf=0.0)
    close("lse", got["lse"], want["lse"], HALF * (128 + 4 * lse))
    lp = want["logprob"].abs().nan_to_num(posinf=0.0)
    close("logprob", got["logprob"], want["logprob"], HALF * (128 + 4 * lp))
    if entropy:
        close("entropy", got["entropy"], want["entropy"], HALF * 256 * (1 + want["entropy"]))
    if top:
        assert torch.equal(got["top_ids"].cpu(), want["top_ids"])
        tl = want["top_logprobs"]
        close("top_logprobs", got["top_logprobs"], tl, HALF * (128 + 4 * tl.abs().nan_to_num(posinf=0.0)))


def rows(n, V, dtype, seed=0, device="cuda", masked=0.0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (spread * torch.randn(n, V, generator=g)).to(TYPES[dtype])
    if masked:
        x[torch.rand(n, V, generator=g) < masked] = NEG
    y = torch.randint(V, (n,), generator=g)
    return x.to(device), y.to(device), g


SIZES = [(1, 1), (3, 2), (5, 63), (4, 64), (2, 100), (3, 511), (2, 513), (5, 1024), (2, 1500), (3, 2049), (2, 4097),
         (1, 8200), (2, 16384), (1, 16385), (2, 40001)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,V", SIZES)
def test_forward(device, dtype, n, V):
    for top, scale, masked in ((0, 1.0, 0.0), (min(V, 1), 0.37, 0.0), (min(V, 7), 1.0, 0.5), (min(V, 64), 2.1, 0.0)):
        x, y, _ = rows(n, V, dtype, seed=V + top, masked=masked)
        want = ref.logprob(x.cpu().double(), y.cpu(), scale, top)
        got = rla.rla_logprob_forward(x, y, scale=scale, entropy=True, top=top)
        check_forward(got, want, top)
        wide = rla.rla_logprob_forward(lref.strided(x, 1), y.int(), scale=scale, entropy=True, top=top)
        assert all(got[k] is None or torch.equal(got[k], wide[k]) for k in got)
        few = rla.rla_logprob_forward(x, y, scale=scale)
        assert torch.equal(few["lse"], got["lse"]) and torch.equal(few["logprob"], got["logprob"])
        assert few["entropy"] is None and few["top_ids"] is None


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,V", [(1500, 300), (1100, 20000), (70, 20000), (9, 131072), (1, 131072)])
def test_many(device, dtype, n, V):
    """Rows in one part or many, few rows and more than the workgroups that fill the card."""
    x, y, _ = rows(n, V, dtype, seed=n)
    got = rla.rla_logprob_forward(x, y, scale=0.8, entropy=True, top=20)
    some = sorted({0, n // 2, n - 1})
    want = ref.logprob(x[some].cpu().double(), y[some].cpu(), 0.8, 20)
    check_forward({k: t[some] for k, t in got.items()}, want, 20)
    z = x.double() * 0.8
    lse = torch.logsumexp(z, -1)
    close("lse", got["lse"], lse.cpu(), HALF * (128 + 4 * lse.abs().cpu()))
    lp = z - lse[:, None]
    close("entropy", got["entropy"], -(lp.exp() * lp).sum(-1).cpu(), HALF * 256 * 13)
    order = torch.sort(x.float(), dim=-1, descending=True, stable=True).indices[:, :20]
    assert torch.equal(got["top_ids"].long(), order)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [40, 700, 5000, 16384, 50001])
@pytest.mark.parametrize("kind", ["equal", "two", "rising", "falling", "one high", "clustered", "zeros", "empty", "one left",
                                  "lowest"])
def test_ties_and_orders(device, dtype, V, kind):
    """Rows in which many values reach any bound on the largest ones."""
    x = torch.zeros(3, V)
    j = torch.arange(V)
    if kind == "equal":
        x += 1.25
    elif kind == "two":
        x[:, ::2] = 3.0
    elif kind == "rising":
        x += (j // 7).float() * 0.5
    elif kind == "falling":
        x -= (j // 3).float() * 0.25
    elif kind == "one high":
        x[1, V - 1], x[2, 0] = 100.0, 100.0
    elif kind == "clustered":
        x[:, V // 2:V // 2 + 300] = 5.0 + (j[:300] % 11).float()[:x[0, V // 2:V // 2 + 300].numel()]
    elif kind == "zeros":
        x[:, 1::2] = -0.0
    elif kind == "empty":
        x += NEG
    elif kind == "one left":
        x += NEG
        x[:, V // 3] = -2.0
    else:
        x += torch.finfo(TYPES[dtype]).min
        x[1, V // 2] = 0.0
    x = x.to(TYPES[dtype]).to(device)
    y = torch.tensor([0, V // 3, V - 1], device=device)
    for top in (1, 5, 33):
        got = rla.rla_logprob_forward(x, y, entropy=True, top=top)
        # (values in fp32 stand as they are: the definition's order and ties)
        check_forward(got, ref.logprob(x.cpu().double(), y.cpu(), 1.0, top), top)


def test_not_finite(device):
    """NaN and +inf stay in their row; tokens outside the vocabulary leave theirs out."""
    x, y, _ = rows(6, 3000, "f32")
    want = rla.rla_logprob_forward(x, y, entropy=True, top=4)
    x[1, 70], x[3, 2999], x[4, 0] = float("nan"), float("inf"), NEG
    y[0], y[5] = -100, 3000
    got = rla.rla_logprob_forward(x, y, entropy=True, top=4)
    for k in ("lse", "entropy"):
        assert got[k][[1, 3]].isnan().all() and torch.equal(got[k][[0, 2, 5]], want[k][[0, 2, 5]])
    assert got["top_logprobs"][[1, 3]].isnan().all() and torch.equal(got["top_ids"][[0, 2, 5]], want["top_ids"][[0, 2, 5]])
    assert (got["logprob"][[0, 5]] == 0).all() and got["logprob"][[1, 3]].isnan().all()
    assert torch.isfinite(got["lse"][4])
    y[4] = 0
    assert rla.rla_logprob_forward(x, y)["logprob"][4] == NEG
    d = rla.rla_logprob_backward(x, got["lse"], y, torch.ones(6, device=device), got["entropy"], torch.ones(6, device=device))
    assert d[[1, 3]].isnan().all() and torch.isfinite(d[[0, 2, 4, 5]]).all()


def gradient(x, y, scale, g, e):
    """64 bits, by autograd over the values that are there."""
    z = x.cpu().double()
    there = z > NEG
    leaf = torch.where(there, z, torch.zeros_like(z)).requires_grad_(True)
    masked = torch.where(there, leaf * scale, torch.full_like(z, -1e30))
    lse = torch.logsumexp(masked, -1, keepdim=True)
    lp = masked - lse
    y = y.cpu()
    known = (y >= 0) & (y < x.shape[1])
    up = lp.new_zeros(())
    if g is not None:
        up = up + (torch.where(known, lp.gather(1, y.clamp(0, x.shape[1] - 1)[:, None])[:, 0], 0.0) * g.cpu().double()).sum()
    H = -(torch.where(there, lp.exp() * lp, 0.0)).sum(-1)
    if e is not None:
        up = up + (H * e.cpu().double()).sum()
    want = torch.autograd.grad(up, leaf)[0] if up.requires_grad else torch.zeros_like(z)
    p, lp, lse, H = lp.exp().detach() * there, lp.detach().abs() * there, lse.detach().abs(), H.detach()[:, None]
    gg = torch.zeros(len(y)) if g is None else g.cpu().abs().double()
    ee = torch.zeros(len(y)) if e is None else e.cpu().abs().double()
    # p is off by the bound of lse and the rounding of its exponent, the bracket by its parts' rounding
    allowed = scale * HALF * (256 + 4 * lse + 4 * lp) * p * (gg[:, None] + ee[:, None] * (lp + H + 1)) * 2
    return want, allowed + HALF * 8 * want.abs() + (2.0 ** -8 * want.abs() if x.dtype == torch.bfloat16 else 0) + 1e-37


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,V", [(1, 1), (5, 3), (4, 64), (7, 100), (3, 1000), (2, 4097), (3, 20001)])
@pytest.mark.parametrize("which", ["g", "e", "ge"])
def test_gradient(device, dtype, n, V, which):
    x, y, gen = rows(n, V, dtype, seed=V, masked=0.3 if V > 64 else 0.0)
    if "g" in which and V > 64:
        x[torch.arange(n), y] = 1.0   # (a token with a probability)
    y[n // 2] = -100
    g = torch.randn(n, generator=gen).to(device) if "g" in which else None
    e = torch.randn(n, generator=gen).to(device) if "e" in which else None
    for scale in (1.0, 0.6):
        f = rla.rla_logprob_forward(x, y, scale=scale, entropy=True)
        how = dict(entropy=f["entropy"], dentropy=e, scale=scale)
        got = rla.rla_logprob_backward(x, f["lse"], y, g, **how)
        want, allowed = gradient(x, y, scale, g, e)
        close("dlogits", got, want, allowed)
        wide = rla.rla_logprob_backward(lref.strided(x, 1), f["lse"], y.int(), g, **how)
        same = x.clone()
        assert rla.rla_logprob_backward(same, f["lse"], y, g, out=same, **how) is same
        assert torch.equal(wide, got) and torch.equal(same, got)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [50, 3000, 20001])
def test_gradient_of_far_rows(device, dtype, V):
    """Rows whose lse is too large for their probabilities' digits: large logits, the type's lowest
    value throughout or but for one."""
    x, y, gen = rows(5, V, dtype, seed=V)
    x[0] += 30000.0
    x[1] -= 5000.0
    x[2] = torch.finfo(TYPES[dtype]).min
    x[3] = torch.finfo(TYPES[dtype]).min
    x[3, V // 2] = 1.0
    g, e = torch.randn(5, generator=gen).to(device), torch.randn(5, generator=gen).to(device)
    f = rla.rla_logprob_forward(x, y, entropy=True)
    got = rla.rla_logprob_backward(x, f["lse"], y, g, f["entropy"], e)
    # the gradient of the rows shifted to a maximum of 0 (in 64 bits, where z - lse loses digits too), and
    # the bound of such rows: nothing is lost to a large lse.  Values 1e4 below have no probability.
    near = (x.double() - x.double().amax(-1, keepdim=True)).clamp(min=-1e4)
    want, allowed = gradient(near, y, 1.0, g, e)
    close("dlogits", got, want, allowed + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0))


def test_gradient_of_empty_rows(device):
    x, y, _ = rows(3, 500, "f32")
    x[1] = NEG
    one = torch.ones(3, device=device)
    f = rla.rla_logprob_forward(x, y, entropy=True)
    d = rla.rla_logprob_backward(x, f["lse"], y, one, f["entropy"], one)
    assert (d[1] == 0).all() and torch.isfinite(d).all() and (d[0] != 0).any()
    none = rla.rla_logprob_backward(x, f["lse"])
    assert (none == 0).all()


def test_large_gradient(device):
    """Written past the caches, rows of a part at the end."""
    n, V = 2100, 32003
    x, y, _ = rows(1, V, "bf16")
    g = torch.Generator(device).manual_seed(3)
    x = (3 * torch.randn(n, V, device=device, generator=g)).bfloat16()
    y = torch.randint(V, (n,), device=device, generator=g)
    up = torch.randn(n, device=device, generator=g)
    f = rla.rla_logprob_forward(x, y)
    got = rla.rla_logprob_backward(x, f["lse"], y, up)
    some = [0, 1000, n - 1]
    want, allowed = gradient(x[some], y[some], 1.0, up[some], None)
    close("dlogits", got[some], want, allowed)
    # every row: probabilities sum to 1, so gradients to 0, but for their rounding to bf16
    total, size = got.double().sum(-1), got.double().abs().sum(-1)
    assert (total.abs() <= 2.0 ** -8 * size).all()


def test_differences(device):
    """Both gradients along a direction against differences of the 64-bit forward."""
    x, y, gen = rows(4, 300, "f32", seed=9)
    g, e = torch.randn(4, generator=gen), torch.randn(4, generator=gen)
    f = rla.rla_logprob_forward(x, y, scale=0.9, entropy=True)
    d = rla.rla_logprob_backward(x, f["lse"], y, g.to(device), f["entropy"], e.to(device), scale=0.9).cpu().double()
    way = torch.randn(4, 300, generator=gen, dtype=torch.float64)

    def loss(t):
        r = ref.logprob(x.cpu().double() + t * way, y.cpu(), 0.9)
        return (r["logprob"] * g + r["entropy"] * e).sum().item()

    h = 1e-5
    want, parts = (loss(h) - loss(-h)) / (2 * h), d * way
    assert abs(parts.sum().item() - want) <= 5e-6 * parts.abs().sum().item()


def test_empty(device):
    x, y = torch.empty(0, 50, device=device), torch.empty(0, dtype=torch.int64, device=device)
    f = rla.rla_logprob_forward(x, y, entropy=True, top=3)
    assert f["top_ids"].shape == (0, 3) and f["lse"].numel() == 0
    assert rla.rla_logprob_backward(x, f["lse"], y, f["lse"]).shape == (0, 50)


BAD = {
    "logits": (dict(logits=lambda t: t.double()), TypeError, "logits"),
    "logits rows": (dict(logits=lambda t: t.t().contiguous().t()), ValueError, "logits"),
    "targets": (dict(targets=lambda t: t[:-1]), ValueError, "targets"),
    "targets type": (dict(targets=lambda t: t.float()), TypeError, "targets"),
    "targets device": (dict(targets=lambda t: t.cpu()), ValueError, "targets"),
    "top": (dict(top=lambda t: 65), ValueError, "top"),
    "more than there are": (dict(top=lambda t: 41, logits=lambda t: t[:, :40]), ValueError, "top"),
    "scale": (dict(scale=lambda t: 0.0), rla.RLAError, ""),
    "lse": (dict(lse=lambda t: torch.empty(3, device="cuda")), ValueError, "lse"),
    "out without targets": (dict(targets=lambda t: None, out=lambda t: torch.empty(4, device="cuda")), ValueError, "targets"),
    "ids type": (dict(top=lambda t: 2, top_ids=lambda t: torch.empty(4, 2, dtype=torch.int64, device="cuda")), TypeError, "top_ids"),
    "ids without top": (dict(top_ids=lambda t: torch.empty(4, 2, dtype=torch.int32, device="cuda")), ValueError, "top"),
}


@pytest.mark.parametrize("case", list(BAD))
def test_refused(device, case):
    x, y, _ = rows(4, 100, "f32")
    change, error, match = BAD[case]
    args = dict(logits=x, targets=y, scale=1.0, top=0, lse=None, out=None, top_ids=None)
    args.update({n: f(args[n]) for n, f in change.items()})
    with pytest.raises(error, match=match):
        rla.rla_logprob_forward(**args)


def test_refused_gradients(device):
    x, y, _ = rows(4, 100, "f32")
    lse = torch.zeros(4, device=device)
    f = rla.rla_logprob_backward
    with pytest.raises(ValueError, match="lse"):
        f(x, None, y, lse)
    with pytest.raises(ValueError, match="targets"):
        f(x, lse, None, lse)
    with pytest.raises(ValueError, match="entropy"):
        f(x, lse, y, lse, dentropy=lse)
    with pytest.raises(ValueError, match="dlogprob"):
        f(x, lse, y, lse[:3])
    wide = lref.strided(x, 1)
    with pytest.raises(ValueError, match="out"):
        f(wide, lse, y, lse, out=wide)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [20000, 131072])
@pytest.mark.parametrize("allowed", [3, 40, 400, 3000])
def test_few_allowed(device, dtype, V, allowed):
    """A stretch of the vocabulary is allowed, the rest -inf: fewer than the alternatives asked
    for, a few lanes' worth, a few waves' worth."""
    g = torch.Generator(device).manual_seed(allowed)
    x = torch.full((6, V), NEG, dtype=TYPES[dtype], device=device)
    first = [0, 7, V // 2, V - allowed, 1024, 8191]
    for r, a in enumerate(first):
        x[r, a:a + allowed] = (3 * torch.randn(allowed, device=device, generator=g)).to(TYPES[dtype])
    y = torch.tensor(first, device=device)
    y[1] = 0
    for top in (1, 20, 64):
        got = rla.rla_logprob_forward(x, y, entropy=True, top=top)
        check_forward(got, ref.logprob(x.cpu().double(), y.cpu(), 1.0, top), top)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [50, 700, 20001, 200003])
def test_far_rows_in_place(device, dtype, V):
    """Rows that are read again are not read where their gradient already stands."""
    x, y, gen = rows(40, V, dtype, seed=V)
    x[::2] += 30000.0
    x[1::4] = torch.finfo(TYPES[dtype]).min
    g, e = torch.randn(40, generator=gen).to(device), torch.randn(40, generator=gen).to(device)
    f = rla.rla_logprob_forward(x, y, entropy=True)
    want = rla.rla_logprob_backward(x, f["lse"], y, g, f["entropy"], e)
    got = rla.rla_logprob_backward(x, f["lse"], y, g, f["entropy"], e, out=x)
    assert got is x and torch.equal(got, want)


def test_numbers_in_tensors(device):
    """A scale and a count given as tensors count as what they hold when the call is made."""
    x, y, _ = rows(4, 100, "f32")
    scale, top = torch.tensor(0.5), torch.tensor(3)
    first = rla.rla_logprob_forward(x, y, scale=scale, top=top)
    scale.fill_(2.0)
    top.fill_(5)
    second = rla.rla_logprob_forward(x, y, scale=scale, top=top)
    for got, s, n in ((first, 0.5, 3), (second, 2.0, 5)):
        check_forward(got, ref.logprob(x.cpu().double(), y.cpu(), s, n), n, entropy=False)


def test_more_long_rows_than_a_launch(device):
    """Rows that a workgroup of 1024 lanes takes each, beyond the lanes of one launch."""
    n, V = (1 << 22) + 3, 12289
    if torch.cuda.mem_get_info()[0] < 2 * n * V + (4 << 30):
        pytest.skip("needs 107 GB")
    x = torch.zeros(n, V, dtype=torch.bfloat16, device=device)
    some = [0, (1 << 21) - 1, 1 << 21, 1 << 22, n - 1]
    near, y, _ = rows(len(some), V, "bf16")
    x[some] = near
    targets = torch.zeros(n, dtype=torch.int32, device=device)
    targets[some] = y.int()
    f = rla.rla_logprob_forward(x, targets)
    check_forward({k: f[k][some] for k in ("lse", "logprob")}, ref.logprob(near.cpu().double(), y.cpu(), 1.0, 0), 0, entropy=False)
    f["lse"][some] = f["lse"][1].item()
    assert (f["lse"] == f["lse"][1]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [50, 3000, 20001, 200003])
@pytest.mark.parametrize("scale", [1.43, 2.0])
def test_gradient_where_lse_overflows(device, dtype, V, scale):
    """Finite logits whose lse, times the scale, leaves fp32: the probabilities are those of the
    differences, as in the forward; rows without any keep their zeros."""
    x, y, gen = rows(6, V, dtype, seed=V)
    least, most = torch.finfo(TYPES[dtype]).min, torch.finfo(TYPES[dtype]).max
    x[0] = least
    x[1] = most
    x[2, 1:], x[2, 0] = most, 0.0
    x[3, 1:], x[3, 0] = NEG, least
    x[4] = NEG
    y[2], y[3] = 0, 0
    g, e = torch.randn(6, generator=gen).to(device), torch.randn(6, generator=gen).to(device)
    f = rla.rla_logprob_forward(x, y, scale=scale, entropy=True)
    assert (f["lse"][[0, 3, 4]] == NEG).all() and (f["lse"][[1, 2]] == -NEG).all()
    # (the rows shifted to a maximum of 0; values 1e4 below have no probability)
    near = (x.double() - x.double().amax(-1, keepdim=True)).clamp(min=-1e4)
    near[4] = NEG
    want, allowed = gradient(near, y, scale, g, e)
    want[4] = 0
    allowed += 2.0 ** -8 * want.abs() if dtype == "bf16" else 0
    close("dlogits", rla.rla_logprob_backward(x, f["lse"], y, g, f["entropy"], e, scale=scale), want, allowed)
    close("in place", rla.rla_logprob_backward(x, f["lse"], y, g, f["entropy"], e, scale=scale, out=x), want, allowed)


def exact_gradient(x, y, scale, g, e):
    """(gradient, bound) in 64 bits from the definition.  Half steps of p: of the exponent's three roundings (its
    factor's two, its own) 3 |log p|, of those of the row's sum 3 H, e^t, 1 / s and products 10, and of the
    terms added one after the other at most 4 pieces of 8, then 6 in a wave and 16 waves: 54.  log p is off by
    as much, H by the half step that it is given with, the bracket by rounding."""
    z = x.cpu().double() * scale
    lp = z - torch.logsumexp(z, -1, keepdim=True)
    p, H = lp.exp(), -(lp.exp() * lp).sum(-1, keepdim=True)
    g, e = g.cpu().double()[:, None], e.cpu().double()[:, None]
    at = (torch.arange(x.shape[1]) == y.cpu()[:, None]).double()
    want = scale * (g * (at - p) - e * p * (lp + H))
    steps = HALF * (64 + 3 * lp.abs() + 3 * H)
    allowed = scale * p * (steps * (g.abs() + e.abs() * (lp + H).abs()) + e.abs() * (steps + HALF * (2 * H + 2 * lp.abs())))
    return want, allowed + 4 * HALF * (want.abs() + scale * g.abs() * at), H[:, 0]


@pytest.mark.parametrize("V,rows_", [(50, 600), (300, 300), (3000, 60), (20003, 40), (30011, 24)])
@pytest.mark.parametrize("spread,scale", [(1.0, 1.0), (6.0, 0.75)])
def test_digits_of_large_lse(device, V, rows_, spread, scale):
    """A gradient's digits do not go with its row's lse: rows at 30 to 255 and below -30, as exact as near 0 (half a
    step of lse is up to 128 half steps of p)."""
    x, y, gen = rows(rows_, V, "f32", seed=V, spread=spread)
    lse = torch.logsumexp(x.cpu().double() * scale, -1)
    to = torch.empty(rows_, dtype=torch.float64).uniform_(34, 250, generator=gen) * torch.where(torch.arange(rows_) % 4 == 3, -1, 1)
    x += ((to - lse) / scale)[:, None].float().to(device)
    g, e = torch.randn(rows_, generator=gen).to(device), torch.randn(rows_, generator=gen).to(device)
    want, allowed, H = exact_gradient(x, y, scale, g, e)
    f = rla.rla_logprob_forward(x, y, scale=scale)
    assert f["lse"].abs().min() > 32 and f["lse"].abs().max() < 256
    got = rla.rla_logprob_backward(x, f["lse"], y, g, H.float().to(device), e, scale=scale)
    close("dlogits", got, want, allowed)


def test_part_of_a_vocabulary(device):
    """The formula's lse stands where it is not the row's own: each half of the columns, with the lse of
    both, gives its part of the gradient."""
    x, y, gen = rows(40, 6000, "f32", seed=3)
    g = torch.randn(40, generator=gen).to(device)
    f = rla.rla_logprob_forward(x, y)
    whole = rla.rla_logprob_backward(x, f["lse"], y, g)
    for a, b in ((0, 2500), (2500, 6000)):
        own = torch.where((y >= a) & (y < b), y - a, -1)
        got = rla.rla_logprob_backward(x[:, a:b], f["lse"], own, torch.where(own < 0, 0.0, g))
        rest = rla.rla_logprob_backward(x[:, a:b], f["lse"], torch.zeros_like(y), torch.where(own < 0, g, 0.0))
        rest[:, 0] -= torch.where(own < 0, g, 0.0)   # (a row whose token lies elsewhere: the probabilities' part)
        want = whole[:, a:b].cpu().double()
        # lse < 16: off by half a step, 2^-21, and 64 more of p's half steps
        close("part", got + rest, want, 2 ** -20 * want.abs() + HALF * 64 * g.cpu().double().abs()[:, None])
