"""The operators around a mixing layer at sizes that take other routes: outputs written
past the caches, wide grids, offsets beyond 32 bits; and in captured graphs."""
import pytest
import torch

import paper_2509_25223_amd as rla
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


def few(D, n, seed=2):
    """Some columns of D, the last among them."""
    g = torch.Generator().manual_seed(seed)
    return torch.cat([torch.randperm(D - 1, generator=g)[:n - 1], torch.tensor([D - 1])])


def wide_cut(t, cols):
    return ref.wide(t[..., cols.to(t.device)])


@pytest.mark.parametrize("D", [8200, 8203])
def test_conv(device, D):
    """More than 96 MiB of outputs, rows of whole pieces and of a part."""
    T, a, W = 6421, 3000, 4
    g = torch.Generator(device).manual_seed(0)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    x, dy = rnd(T, D).bfloat16(), rnd(T, D).bfloat16()
    weight, bias, state = rnd(D, W), rnd(D), rnd(2, W - 1, D).bfloat16()
    cu = torch.tensor([0, a, T], dtype=torch.int32, device=device)
    how = dict(bias=bias, silu=True, state=state, cu_seqlens=cu)
    y, fin = rla.rla_conv_forward(x, weight, **how)
    got = rla.rla_conv_backward(x, weight, dy, **how)
    cols = few(D, 24)
    v = dict(x=wide_cut(x, cols), weight=ref.wide(weight[cols.to(device)]), bias=wide_cut(bias, cols),
             state=wide_cut(state, cols))
    want, wfin = ref.conv(v["x"], v["weight"], v["bias"], True, v["state"], [(0, a), (a, T)])
    back = ref.gradients([want], [wide_cut(dy, cols).detach()], v)
    c = cols.to(device)
    ref.check("y", y[:, c], want, W)
    assert torch.equal(fin[..., c].cpu().double(), wfin.detach())
    ref.check("dx", got["dx"][:, c], back["x"], W)
    ref.check("dstate", got["dstate"][..., c], back["state"], W)
    ref.check("dweight", got["dweight"][c], back["weight"], 8 * T)
    ref.check("dbias", got["dbias"][c], back["bias"], 8 * T)


def test_addnorm(device):
    rows, D = 12600, 2080   # 52 MB of n, 105 MB of the stream
    g = torch.Generator(device).manual_seed(1)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    x, res, dn, dr = rnd(rows, D).bfloat16(), 2 * rnd(rows, D), rnd(rows, D).bfloat16(), rnd(rows, D)
    weight, scale = 1 + 0.1 * rnd(D), 0.3 + rnd(D)
    n, r = rla.rla_addnorm_forward(x, weight, residual=res, scale=scale)
    got = rla.rla_addnorm_backward(dn, r, weight, x=x, scale=scale, dresidual_out=dr)
    want_n, want_r = ref.addnorm(x.double(), res.double(), weight.double(), scale.double())
    ref.check("n", n, want_n.cpu(), 4)
    ref.check("residual", r, want_r.cpu())
    # the gradient's formula: with m = r / rms, (g w - m mean(g w m)) / rms
    r64, gw = r.double(), dn.double() * weight.double()
    inv = 1 / torch.sqrt((r64 * r64).mean(-1, keepdim=True) + ref.EPS)
    m = r64 * inv
    total = dr.double() + inv * (gw - m * (gw * m).mean(-1, keepdim=True))
    ref.check("dresidual", got["dresidual"], total.cpu(), 16)
    ref.check("dx", got["dx"], (total * scale.double()).cpu(), 16)
    ref.check("dweight", got["dweight"], (dn.double() * m).sum(0).cpu(), 8 * rows)
    ref.check("dscale", got["dscale"], (total * x.double()).sum(0).cpu(), 8 * rows)


@pytest.mark.parametrize("first", [False, True])
def test_gatenorm(device, first):
    rows, H, d = 6600, 60, 136   # 108 MB of o, 215 MB of dx
    g = torch.Generator(device).manual_seed(2)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    x, gate, dO = rnd(rows, H, d), rnd(rows, H, d).bfloat16(), rnd(rows, H, d).bfloat16()
    weight = 1 + 0.1 * rnd(d)
    o = rla.rla_gatenorm_forward(x, gate, weight, gate_first=first)
    got = rla.rla_gatenorm_backward(dO, x, gate, weight, gate_first=first)
    some = torch.cat([torch.arange(0, rows, 97), torch.tensor([rows - 1])]).to(device)
    v = dict(x=ref.wide(x[some]), gate=ref.wide(gate[some]), weight=ref.wide(weight))
    want = ref.gatenorm(v["x"], v["gate"], v["weight"], first)
    back = ref.gradients([want], [dO[some].cpu().double()], v)
    ref.check("o", o[some], want, 4)
    ref.check("dx", got["dx"][some], back["x"], 16)
    ref.check("dgate", got["dgate"][some], back["gate"], 16)
    # dweight = sum of dO times the normalised (and, gate last, gated) values
    gd = gate.double()
    act = gd * torch.sigmoid(gd)
    y = x.double() * act if first else x.double()
    hat = ref.rms(y) if first else ref.rms(y) * act
    ref.check("dweight", got["dweight"], (dO.double() * hat).sum((0, 1)).cpu(), 8 * rows * H)


@pytest.mark.parametrize("N", [16, 13, 64])
def test_scan_of_many_sequences(device, N):
    """Single tokens of an odd number of sequences at a time, two of them a lane."""
    B, T, D = 35, 2, 3800 if N < 64 else 960
    g = torch.Generator(device).manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    u, delta, z, Bm, C = (rnd(B, T, *s).bfloat16() for s in ((D,), (D,), (D,), (1, N), (1, N)))
    A, skip, h = -4 * torch.rand(D, N, device=device, generator=g), rnd(D), rnd(B, D, N)
    o, fin = rla.rla_ssm_decode(u, delta, A, Bm, C, D=skip, z=z, h_in=h)
    cols = few(D, 12)
    want, wfin = ref.ssm(*(wide_cut(t, cols).reshape(B * T, -1) for t in (u, delta)), ref.wide(A[cols.to(device)]),
                         *(ref.wide(t).reshape(B * T, 1, N) for t in (Bm, C)), wide_cut(skip, cols),
                         wide_cut(z, cols).reshape(B * T, -1), None, True, ref.wide(h[:, cols.to(device)]),
                         [(b * T, (b + 1) * T) for b in range(B)])
    ref.check("o", o[..., cols.to(device)], want.reshape(B, T, -1), 8 * N)
    ref.check("h", fin[:, cols.to(device)], wfin, 8)
    # as few at a time, and in place
    for b in (0, 17, 34):
        cut = lambda t: t[b:b + 1].contiguous()   # noqa: E731
        one, hone = rla.rla_ssm_decode(cut(u), cut(delta), A, cut(Bm), cut(C), D=skip, z=cut(z), h_in=cut(h))
        assert torch.equal(one[0], o[b]) and torch.equal(hone[0], fin[b])
    same = h.clone()
    o2, out = rla.rla_ssm_decode(u, delta, A, Bm, C, D=skip, z=z, h_in=same, h_out=same)
    assert out is same and torch.equal(o2, o) and torch.equal(same, fin)


def test_rows_far_apart(device):
    """Rows 2^23 values apart: offsets of more than 32 bits give the same results."""
    T, D, N, apart = 600, 72, 16, 1 << 23
    g = torch.Generator(device).manual_seed(4)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    space = torch.empty(T * apart, dtype=torch.bfloat16, device=device)
    flat = {}

    def far(name, width, at):
        flat[name] = rnd(T, width).bfloat16()
        t = space.as_strided((T, width), (apart, 1), at)
        t.copy_(flat[name])
        return t

    x = {n: far(n, D, 1 + 100 * i) for i, n in enumerate(("u", "delta", "z", "dO"))}
    bc = {n: far(n, N, 500 + 20 * i).unflatten(-1, (1, N)) for i, n in enumerate("BC")}
    near = {n: flat[n] for n in x} | {n: flat[n].unflatten(-1, (1, N)) for n in "BC"}
    A, weight, norm = -4 * torch.rand(D, N, device=device, generator=g), rnd(D, 4), 1 + 0.1 * rnd(D)

    def results(v):
        y, fin = rla.rla_conv_forward(v["u"], weight, silu=True)
        conv = rla.rla_conv_backward(v["u"], weight, v["dO"], silu=True)
        o, h = rla.rla_ssm_forward(v["u"], v["delta"], A, v["B"], v["C"], z=v["z"])
        scan = rla.rla_ssm_backward(v["u"], v["delta"], A, v["B"], v["C"], v["dO"], z=v["z"])
        n, r = rla.rla_addnorm_forward(v["u"], norm)
        add = rla.rla_addnorm_backward(v["dO"], r, norm)
        heads = {m: v[m].unflatten(-1, (2, D // 2)) for m in ("u", "z", "dO")}
        half = norm[:D // 2].contiguous()
        q = rla.rla_gatenorm_forward(heads["u"], heads["z"], half)
        gate = rla.rla_gatenorm_backward(heads["dO"], heads["u"], heads["z"], half)
        return [y, fin, o, h, n, r, q] + [t for gr in (conv, scan, add, gate) for _, t in sorted(gr.items())]

    assert all(torch.equal(a, b) for a, b in zip(results(x | bc), results(near)))


def test_captured(device):
    """A graph of forward, gradients and single tokens, replayed on new inputs with
    other work in between: the results of plain calls."""
    T, D, N = 300, 136, 16
    g = torch.Generator(device).manual_seed(5)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    static = {n: torch.empty(T, *s, dtype=torch.bfloat16, device=device)
              for n, s in dict(u=(D,), delta=(D,), z=(D,), B=(1, N), C=(1, N), dO=(D,)).items()}
    A, weight, norm = -4 * torch.rand(D, N, device=device, generator=g), rnd(D, 4), 1 + 0.1 * rnd(D)
    cu = torch.tensor([0, 100, 100, 217, T], dtype=torch.int32, device=device)
    state, h = rnd(4, 3, D).bfloat16(), rnd(4, D, N)

    def calls(v):
        out = {}
        n, r = rla.rla_addnorm_forward(v["u"], norm)
        y, fin = rla.rla_conv_forward(n, weight, silu=True, state=state, cu_seqlens=cu)
        o, hf = rla.rla_ssm_forward(y, v["delta"], A, v["B"], v["C"], h0=h, cu_seqlens=cu)
        q = rla.rla_gatenorm_forward(o[:, None], v["z"][:, None], norm)
        back = rla.rla_gatenorm_backward(v["dO"][:, None], o[:, None], v["z"][:, None], norm)
        scan = rla.rla_ssm_backward(y, v["delta"], A, v["B"], v["C"], back["dx"][:, 0], h0=h, cu_seqlens=cu)
        conv = rla.rla_conv_backward(n, weight, scan["du"], silu=True, state=state, cu_seqlens=cu)
        add = rla.rla_addnorm_backward(conv["dx"], r, norm)
        y1, s1 = rla.rla_conv_decode(v["u"][:4, None], weight, silu=True, state=fin)
        o1, h1 = rla.rla_ssm_decode(y1, v["delta"][:4, None], A, v["B"][:4, None], v["C"][:4, None], h_in=hf)
        out.update(n=n, r=r, y=y, fin=fin, o=o, hf=hf, q=q, y1=y1, s1=s1, o1=o1, h1=h1)
        for name, grads in (("gate", back), ("scan", scan), ("conv", conv), ("add", add)):
            out.update({name + key: t for key, t in grads.items()})
        return out

    def fill():
        fresh = {n: rnd(*t.shape).bfloat16() for n, t in static.items()}
        for n, t in static.items():
            t.copy_(fresh[n])
        return fresh

    fill()
    calls(static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls(static)
    for _ in range(4):
        want = calls(fill())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)
