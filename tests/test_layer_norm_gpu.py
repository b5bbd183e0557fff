"""The norms around a block: outputs and gradients against 64 bits."""
import pytest
import torch

import paper_2509_25223_amd as rla
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def addnorm_inputs(device, lead, D, dtype, stream, scale=True, residual=True, wide=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    t, r = TYPES[dtype], TYPES[stream]
    x = dict(x=rnd(*lead, D).to(t), weight=1 + 0.1 * rnd(D), scale=0.3 + rnd(D) if scale else None,
             residual=(2 * rnd(*lead, D)).to(r) if residual else None, dn=rnd(*lead, D).to(t),
             dresidual_out=rnd(*lead, D).to(r))
    x = {n: None if v is None else v.to(device) for n, v in x.items()}
    if wide:
        for n in ("x", "dn"):
            x[n] = ref.strided(x[n], len(lead))
    return x


# widths of a piece, of less, of one and several pieces a lane, of a workgroup, of two passes
@pytest.mark.parametrize("dtype,stream", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("lead,D,scale,residual,wide", [
    ((3,), 1, True, True, False), ((2, 5), 64, True, True, True), ((7,), 515, False, True, True),
    ((1, 1), 2048, True, True, False), ((2, 301), 1000, True, True, True), ((1100,), 24, True, False, False),
    ((33,), 2056, False, False, True), ((5,), 6001, True, True, False), ((3, 2), 16384, True, True, True),
    ((2,), 8203, True, True, False)])
def test_addnorm(device, dtype, stream, lead, D, scale, residual, wide):
    x = addnorm_inputs(device, lead, D, dtype, stream, scale, residual, wide)
    v = {n: ref.wide(x[n]) for n in ("x", "residual", "weight", "scale")}
    n, r = ref.addnorm(v["x"], v["residual"], v["weight"], v["scale"])
    got_n, got_r = rla.rla_addnorm_forward(x["x"], x["weight"], residual=x["residual"], scale=x["scale"],
                                           residual_dtype=TYPES[stream])
    ref.check("n", got_n, n, 4)
    ref.check("residual", got_r, r)
    # the backward's reference starts from the stream as it is stored
    stored = ref.wide(got_r)
    w = ref.wide(x["weight"])
    up = x["dn"].cpu().double()
    back = ref.gradients([ref.rms(stored) * w], [up], {"r": stored, "weight": w})
    dr = x["dresidual_out"].cpu().double() + back["r"]
    g = rla.rla_addnorm_backward(x["dn"], got_r, x["weight"], x=x["x"] if scale else None, scale=x["scale"],
                                 dresidual_out=x["dresidual_out"])
    ref.check("dresidual", g["dresidual"], dr, 16)
    ref.check("dx", g["dx"], dr if v["scale"] is None else dr * v["scale"], 16)
    rows = dr.numel() // D
    ref.check("dweight", g["dweight"], back["weight"], 8 * rows)
    if scale:
        ref.check("dscale", g["dscale"], (dr * v["x"]).reshape(-1, D).sum(0), 8 * rows)
    assert set(g) == {"dx", "dresidual", "dweight"} | ({"dscale"} if scale else set())


def test_addnorm_in_place(device):
    x = addnorm_inputs(device, (40,), 520, "bf16", "f32")
    n, r = rla.rla_addnorm_forward(x["x"], x["weight"], residual=x["residual"], scale=x["scale"])
    g = rla.rla_addnorm_backward(x["dn"], r, x["weight"], x=x["x"], scale=x["scale"], dresidual_out=x["dresidual_out"])
    same = x["residual"].clone()
    n2, r2 = rla.rla_addnorm_forward(x["x"], x["weight"], residual=same, scale=x["scale"], residual_out=same)
    assert r2 is same and torch.equal(n, n2) and torch.equal(r, r2)
    own = {key: torch.empty_like(t) for key, t in g.items()}
    own["dresidual"] = x["dresidual_out"]
    g2 = rla.rla_addnorm_backward(x["dn"], r, x["weight"], x=x["x"], scale=x["scale"],
                                  dresidual_out=x["dresidual_out"], grads=own)
    assert all(torch.equal(g[key], g2[key]) for key in g)
    # without an upstream gradient of the stream: zeros
    zero = torch.zeros_like(r)
    a = rla.rla_addnorm_backward(x["dn"], r, x["weight"])
    b = rla.rla_addnorm_backward(x["dn"], r, x["weight"], dresidual_out=zero)
    assert all(torch.equal(a[key], b[key]) for key in a)


def test_addnorm_rows_apart(device):
    """A row that holds infinities or NaN leaves the others as they are; rows of zeros."""
    x = addnorm_inputs(device, (9,), 100, "f32", "f32")
    n, r = rla.rla_addnorm_forward(x["x"], x["weight"], residual=x["residual"])
    x["x"][4, 7], x["x"][5, 3] = float("inf"), float("nan")
    m, s = rla.rla_addnorm_forward(x["x"], x["weight"], residual=x["residual"])
    keep = [0, 1, 2, 3, 6, 7, 8]
    assert torch.equal(n[keep], m[keep]) and torch.equal(r[keep], s[keep]) and torch.isnan(m[5]).all()
    zero = torch.zeros(2, 100, device=device)
    n, r = rla.rla_addnorm_forward(zero, x["weight"])
    assert (n == 0).all() and (r == 0).all()


def test_norms_empty(device):
    w = torch.ones(64, device=device)
    x = torch.empty(0, 64, device=device)
    n, r = rla.rla_addnorm_forward(x, w)
    g = rla.rla_addnorm_backward(x, r, w)
    assert n.shape == (0, 64) and (g["dweight"] == 0).all()
    y = torch.empty(0, 4, 64, device=device)
    assert rla.rla_gatenorm_forward(y, y, w).shape == (0, 4, 64)
    assert (rla.rla_gatenorm_backward(y, y, y, w)["dweight"] == 0).all()


def gatenorm_inputs(device, lead, H, d, dtype, xtype, per_head=False, wide=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    x = dict(x=rnd(*lead, H, d).to(TYPES[xtype]), gate=rnd(*lead, H, d).to(TYPES[dtype]),
             weight=1 + 0.1 * (rnd(H, d) if per_head else rnd(d)), dO=rnd(*lead, H, d).to(TYPES[dtype]))
    x = {n: v.to(device) for n, v in x.items()}
    if wide:
        for n in ("x", "gate", "dO"):
            x[n] = ref.strided(x[n], len(lead))
    return x


@pytest.mark.parametrize("dtype,xtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("lead,H,d,per_head,wide", [
    ((5,), 1, 1, False, False), ((2, 3), 4, 33, True, True), ((300,), 3, 64, False, True),
    ((2, 40), 16, 128, True, False), ((11,), 5, 80, False, False), ((4,), 2, 256, False, True),
    ((3,), 3, 600, True, False), ((2, 2), 2, 2100, False, True), ((3,), 2, 2051, True, False)])
def test_gatenorm(device, dtype, xtype, first, lead, H, d, per_head, wide):
    x = gatenorm_inputs(device, lead, H, d, dtype, xtype, per_head, wide)
    v = {n: ref.wide(x[n]) for n in ("x", "gate", "weight")}
    o = ref.gatenorm(v["x"], v["gate"], v["weight"], first)
    grads = ref.gradients([o], [x["dO"].cpu().double()], v)
    got = rla.rla_gatenorm_forward(x["x"], x["gate"], x["weight"], gate_first=first)
    g = rla.rla_gatenorm_backward(x["dO"], x["x"], x["gate"], x["weight"], gate_first=first)
    assert got.dtype == x["gate"].dtype and g["dx"].dtype == x["x"].dtype
    ref.check("o", got, o, 4)
    ref.check("dx", g["dx"], grads["x"], 16)
    ref.check("dgate", g["dgate"], grads["gate"], 16)
    rows = o.numel() // d
    ref.check("dweight", g["dweight"], grads["weight"], 8 * rows)


def test_gatenorm_extreme_gates(device):
    """Gates of large magnitude close (to zero) or open, without NaN."""
    x = gatenorm_inputs(device, (3,), 2, 64, "f32", "f32")
    x["gate"][:, 0] = -200.0
    x["gate"][:, 1] = 200.0
    o = rla.rla_gatenorm_forward(x["x"], x["gate"], x["weight"])
    g = rla.rla_gatenorm_backward(x["dO"], x["x"], x["gate"], x["weight"])
    assert (o[:, 0] == 0).all() and torch.isfinite(o).all() and all(torch.isfinite(t).all() for t in g.values())


def test_norm_differences(device):
    """The gradients along a direction against differences of the 64-bit forward."""
    x = addnorm_inputs(device, (6,), 100, "f32", "f32", seed=3)
    _, r = rla.rla_addnorm_forward(x["x"], x["weight"], residual=x["residual"], scale=x["scale"])
    g = rla.rla_addnorm_backward(x["dn"], r, x["weight"], x=x["x"], scale=x["scale"], dresidual_out=x["dresidual_out"])
    y = gatenorm_inputs(device, (6,), 3, 50, "f32", "f32", seed=4)
    for first in (False, True):
        h = rla.rla_gatenorm_backward(y["dO"], y["x"], y["gate"], y["weight"], gate_first=first)
        compare_differences(lambda v: ref.gatenorm(v["x"], v["gate"], v["weight"], first), [y["dO"]], y,
                            ("x", "gate", "weight"), h)
    compare_differences(lambda v: ref.addnorm(v["x"], v["residual"], v["weight"], v["scale"]),
                        [x["dn"], x["dresidual_out"]], x, ("x", "residual", "weight", "scale"), g)


def compare_differences(forward, up, x, names, grads):
    gen = torch.Generator().manual_seed(9)
    base = {n: x[n].cpu().double() for n in names}
    d = {n: torch.randn(base[n].shape, generator=gen, dtype=torch.float64) for n in names}
    up = [u.cpu().double() for u in up]

    def loss(e):
        out = forward({n: base[n] + e * d[n] for n in names})
        out = out if isinstance(out, tuple) else (out,)
        return sum((o * u).sum().item() for o, u in zip(out, up))

    e = 1e-5
    want = (loss(e) - loss(-e)) / (2 * e)
    parts = [grads["d" + n].cpu().double() * d[n] for n in names]
    assert abs(sum(p.sum().item() for p in parts) - want) <= 2e-6 * sum(p.abs().sum().item() for p in parts)


def test_norm_streams(device):
    x = addnorm_inputs(device, (700,), 520, "bf16", "f32")
    y = gatenorm_inputs(device, (300,), 4, 80, "bf16", "f32")
    _, r = rla.rla_addnorm_forward(x["x"], x["weight"], residual=x["residual"], scale=x["scale"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    back = dict(x=x["x"], scale=x["scale"], dresidual_out=x["dresidual_out"])
    for stream in (None, side):
        a = rla.rla_addnorm_backward(x["dn"], r, x["weight"], stream=stream, **back)
        b = rla.rla_gatenorm_backward(y["dO"], y["x"], y["gate"], y["weight"], stream=stream)
        torch.cuda.synchronize()
        if stream is None:
            want = (a, b)
    assert all(torch.equal(want[0][n], a[n]) for n in a) and all(torch.equal(want[1][n], b[n]) for n in b)


def test_norm_refusals(device):
    x = addnorm_inputs(device, (4,), 64, "bf16", "f32")
    f, b = rla.rla_addnorm_forward, rla.rla_addnorm_backward
    for bad, error, match in [
            (dict(weight=x["weight"][:-1].contiguous()), ValueError, "weight"),
            (dict(weight=x["weight"].bfloat16()), TypeError, "weight"),
            (dict(weight=None), ValueError, "weight"), (dict(x=None), ValueError, "x"),
            (dict(scale=x["scale"].double()), TypeError, "scale"),
            (dict(residual=x["residual"][:-1].contiguous()), ValueError, "residual"),
            (dict(residual=x["residual"].half()), TypeError, "residual"),
            (dict(x=x["x"].float(), residual=x["residual"].bfloat16()), rla.RLAError, "addnorm"),
            (dict(eps=-1.0), rla.RLAError, "addnorm"), (dict(eps=float("nan")), rla.RLAError, "addnorm"),
            (dict(x=x["x"].t().contiguous().t()), ValueError, "contiguous"), (dict(x=x["x"].cpu()), ValueError, "x")]:
        args = dict(x=x["x"], weight=x["weight"], residual=x["residual"], scale=x["scale"])
        args.update(bad)
        with pytest.raises(error, match=match):
            f(**args)
    with pytest.raises(ValueError, match="x is required"):
        b(x["dn"], x["residual"], x["weight"], scale=x["scale"])
    with pytest.raises(ValueError, match="dn"):
        b(None, x["residual"], x["weight"])
    with pytest.raises(ValueError, match="unknown"):
        b(x["dn"], x["residual"], x["weight"], grads=dict(dy=x["dn"]))
    y = gatenorm_inputs(device, (4,), 2, 64, "f32", "f32")
    for bad, error, match in [
            (dict(gate=y["gate"][:, :1].contiguous()), ValueError, "gate"), (dict(gate=None), ValueError, "gate"),
            (dict(weight=y["weight"][1:].contiguous()), ValueError, "weight"),
            (dict(x=y["x"].bfloat16()), rla.RLAError, "gatenorm"), (dict(x=y["x"].half()), TypeError, "x")]:
        args = dict(x=y["x"], gate=y["gate"], weight=y["weight"])
        args.update(bad)
        with pytest.raises(error, match=match):
            rla.rla_gatenorm_forward(**args)
    with pytest.raises(ValueError, match="dO"):
        rla.rla_gatenorm_backward(None, y["x"], y["gate"], y["weight"])
