"""The operators at a model's ends with the gated linear recurrence between them: a small
language model with a shared table, trained, prefilled and decoded; captured in
graphs; on another stream; beside what is not theirs."""
import pytest
import torch

import paper_2509_25223_amd as rla
from paper_2509_25223_amd import model
from tests import layer_reference as lref
from tests import model_reference as ref

pytestmark = pytest.mark.gpu
V, W, D = 67, 40, 52   # vocabulary, width of the stream, channels of the mixer


def parameters(seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)   # noqa: E731
    return dict(table=rnd(V, W), norm1=1 + 0.1 * rnd(W), w1=rnd(W, 4 * D, scale=W ** -0.5), conv=rnd(D, 4, scale=0.5),
                A=-8 * torch.rand(D, generator=g), w2=rnd(D, W, scale=D ** -0.5), norm2=1 + 0.1 * rnd(W))


SCALE, HEAT = W ** 0.5, 0.8   # of the embedding; inverse temperature of the logits


def forward(p, tokens, cu=None, state=None, save=False):
    """Logits of packed [T] or dense [B, T] tokens, and the sequences' states."""
    n_of = lambda k: None if state is None else state[k]   # noqa: E731
    x0 = rla.rla_embed_forward(tokens, p["table"], scale=SCALE)
    n1, r1 = rla.rla_addnorm_forward(x0, p["norm1"])
    p1 = n1 @ p["w1"]
    u, r, i, z = p1.split(D, -1)
    y, cs = rla.rla_conv_forward(u, p["conv"], silu=True, cu_seqlens=cu, state=n_of("conv"))
    how = dict(i=i, z=z, h0=n_of("h"), cu_seqlens=cu)
    work = None
    if save:
        problem = rla.make_glr_problem(y, cu)
        work = torch.empty(rla.rla_glr_workspace_size(problem, rla.RLA_GLR_BACKWARD), dtype=torch.uint8, device=y.device)
    o, h = rla.rla_glr_forward(y, r, p["A"], **how, save_for_backward=save, workspace=work)
    n2, r2 = rla.rla_addnorm_forward(o @ p["w2"], p["norm2"], residual=r1)
    logits = n2 @ p["table"].t()
    return logits, dict(conv=cs, h=h), dict(tokens=tokens, cu=cu, n1=n1, r1=r1, u=u, r=r, y=y, how=how, work=work, o=o,
                                            n2=n2, r2=r2, state=state)


def gradients(p, dlogits, s):
    g = {}
    flat = lambda t: t.flatten(0, -2)   # noqa: E731
    dn2 = dlogits @ p["table"]
    b = rla.rla_addnorm_backward(dn2, s["r2"], p["norm2"])
    g["norm2"], dr1 = b["dweight"], b["dresidual"]
    g["w2"] = flat(s["o"]).t() @ flat(b["dx"])
    b = rla.rla_glr_backward(s["y"], s["r"], p["A"], b["dx"] @ p["w2"].t(), **s["how"], use_saved=True, workspace=s["work"])
    g["A"] = b["dA"]
    c = rla.rla_conv_backward(s["u"], p["conv"], b["dx"], silu=True, cu_seqlens=s["cu"],
                              state=None if s["state"] is None else s["state"]["conv"])
    g["conv"] = c["dweight"]
    dp1 = torch.cat([c["dx"], b["dr"], b["di"], b["dz"]], -1)
    g["w1"] = flat(s["n1"]).t() @ flat(dp1)
    b = rla.rla_addnorm_backward(dp1 @ p["w1"].t(), s["r1"], p["norm1"], dresidual_out=dr1)
    g["norm1"] = b["dweight"]
    head = flat(dlogits).t() @ flat(s["n2"])   # the table's part as the output projection
    g["table"] = rla.rla_embed_backward(s["tokens"], b["dx"], V, scale=SCALE, base=head, dtable=head)
    return g


def wide_loss(v, tokens, targets, spans, up, ent):
    """The loss in 64 bits: sum of up * log probability + ent * entropy."""
    x0 = SCALE * v["table"][tokens]
    n1, r1 = lref.addnorm(x0, None, v["norm1"], None)
    u, r, i, z = (n1 @ v["w1"]).split(D, -1)
    y, _ = lref.conv(u, v["conv"], None, True, None, spans)
    o, _ = ref.glr(y, r, v["A"], i, z, True, None, spans)
    n2, _ = lref.addnorm(o @ v["w2"], r1, v["norm2"], None)
    lp = torch.log_softmax(HEAT * (n2 @ v["table"].t()), -1)
    known = targets >= 0
    given = torch.where(known, lp.gather(1, targets.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lp[:, 0]))
    return (up * given - ent * (lp.exp() * lp).sum(-1)).sum()


def put(p, device):
    return {n: t.to(device) for n, t in p.items()}


def close(a, b, name=""):
    # fp32 through two norms, three products and the mixer: 1e-3 of the largest value
    a, b = a.detach().cpu().double(), b.detach().cpu().double()
    assert (a - b).abs().max().item() <= 1e-3 * b.abs().max().item(), name


@pytest.mark.parametrize("cu", [[0, 30, 30, 31, 140], [0, 140]])
def test_gradients(device, cu):
    p, g = put(parameters(), device), torch.Generator().manual_seed(1)
    T = cu[-1]
    tokens, targets = torch.randint(V, (T,), generator=g), torch.randint(V, (T,), generator=g)
    targets[::7] = -100
    up, ent = -torch.rand(T, generator=g), 0.1 * torch.randn(T, generator=g)
    offsets = torch.tensor(cu, dtype=torch.int32, device=device)
    logits, _, saved = forward(p, tokens.to(device), offsets, save=True)
    f = rla.rla_logprob_forward(logits, targets.to(device), scale=HEAT, entropy=True)
    d = rla.rla_logprob_backward(logits, f["lse"], targets.to(device), up.to(device), f["entropy"], ent.to(device), scale=HEAT,
                                 out=logits)
    got = gradients(p, d, saved)
    v = {n: lref.wide(t) for n, t in p.items()}
    loss = wide_loss(v, tokens, targets, lref.sequences(cu, T), up.double(), ent.double())
    close((up.to(device) * f["logprob"] + ent.to(device) * f["entropy"]).sum()[None], loss[None], "loss")
    for n, want in zip(v, torch.autograd.grad(loss, list(v.values()))):
        close(got[n], want, n)


def test_serving(device):
    """Packed prompts, then a token of each at a time onto the states, in place: the logits of
    whole sequences, and the same likeliest tokens."""
    p, g = put(parameters(), device), torch.Generator().manual_seed(2)
    lengths, more = [1, 40, 3, 150], 5
    rows = [torch.randint(V, (n + more,), generator=g).to(device) for n in lengths]
    cu = torch.tensor([0] + lengths).cumsum(0).to(device, torch.int32)
    logits, state, _ = forward(p, torch.cat([r[:n] for r, n in zip(rows, lengths)]), cu)
    whole = [forward(p, r[None])[0][0] for r in rows]
    for k, n in enumerate(lengths):
        close(logits[cu[k]:cu[k + 1]], whole[k][:n], k)
    for t in range(more):
        tokens = torch.stack([r[n + t] for r, n in zip(rows, lengths)])[:, None]
        n1, r1 = rla.rla_addnorm_forward(rla.rla_embed_forward(tokens, p["table"], scale=SCALE), p["norm1"])
        u, r, i, z = (n1 @ p["w1"]).split(D, -1)
        y, _ = rla.rla_conv_decode(u, p["conv"], silu=True, state=state["conv"], state_out=state["conv"])
        o, _ = rla.rla_glr_decode(y, r, p["A"], i=i, z=z, h_in=state["h"], h_out=state["h"])
        n2, _ = rla.rla_addnorm_forward(o @ p["w2"], p["norm2"], residual=r1)
        step = (n2 @ p["table"].t())[:, 0]
        want = torch.stack([w[n + t] for w, n in zip(whole, lengths)])
        close(step, want, t)
        best = rla.rla_logprob_forward(step, top=3)
        assert torch.equal(best["top_ids"].long(), step.topk(3).indices)


def calls(v, static):
    """Every entry point once, on inputs of one place; workspaces allocated by the calls."""
    out = {}
    x0 = rla.rla_embed_forward(v["ids"], static["table"], scale=0.5, out_dtype=torch.bfloat16)
    o, h = rla.rla_glr_forward(v["x"], v["r"], static["A"], i=v["i"], z=v["z"], h0=static["h0"], cu_seqlens=static["cu"])
    b = rla.rla_glr_backward(v["x"], v["r"], static["A"], x0, i=v["i"], z=v["z"], h0=static["h0"], cu_seqlens=static["cu"])
    o1, h1 = rla.rla_glr_decode(v["x"][:4, None], v["r"][:4, None], static["A"], z=v["z"][:4, None], h_in=h)
    f = rla.rla_logprob_forward(v["logits"], v["targets"], scale=0.7, entropy=True, top=9)
    d = rla.rla_logprob_backward(v["logits"], f["lse"], v["targets"], f["lse"], f["entropy"], f["entropy"], scale=0.7)
    e = rla.rla_embed_backward(v["ids"], b["dx"], 90, base=static["table"])
    out.update(x0=x0, o=o, h=h, o1=o1, h1=h1, d=d, e=e)
    out.update({"f" + n: t for n, t in f.items()})
    out.update({"b" + n: t for n, t in b.items()})
    return out


def make(device, T=500):
    g = torch.Generator(device).manual_seed(5)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g)   # noqa: E731
    static = dict(table=rnd(90, 72), A=-3 * torch.rand(72, device=device, generator=g), h0=rnd(4, 72),
                  cu=torch.tensor([0, 200, 200, 217, T], dtype=torch.int32, device=device))

    def fresh():
        v = {n: rnd(T, 72).bfloat16() for n in ("x", "r", "i", "z")}
        v.update(ids=torch.randint(-2, 92, (T,), device=device, generator=g), logits=3 * rnd(60, 140000),
                 targets=torch.randint(140000, (60,), device=device, generator=g))
        return v

    return static, fresh


def test_captured(device):
    """A graph of all calls, replayed on new inputs with other work in between: the results of
    plain calls.  A second graph, of the same inputs, between its replays."""
    static, fresh = make(device)
    place = fresh()
    calls(place, static)
    torch.cuda.synchronize()
    graphs, got = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(calls(place, static))
        graphs.append(graph)
    for turn in range(4):
        new = fresh()
        for n, t in place.items():
            t.copy_(new[n])
        want = calls(new, static)
        torch.cuda.synchronize()
        for k in (0, 1) if turn % 2 else (1, 0):
            graphs[k].replay()
        torch.cuda.synchronize()
        for res in got:
            for n in want:
                assert torch.equal(res[n], want[n]), n


def test_other_stream(device):
    """Calls on a stream of their own, inputs ready there: the same bits; twice at once too."""
    static, fresh = make(device)
    v = fresh()
    want = calls(v, static)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(calls(v, static))
    side = streams[0]
    f = rla.rla_logprob_forward(v["logits"], v["targets"], scale=0.7, stream=side)
    e = rla.rla_embed_backward(v["ids"], want["bdx"], 90, base=static["table"], stream=side)
    torch.cuda.synchronize()
    for res in got:
        for n in want:
            assert torch.equal(res[n], want[n]), n
    assert torch.equal(f["lse"], want["flse"]) and torch.equal(e, want["e"])


class Fenced:
    """Buffers with other values on both sides."""
    def __init__(self):
        self.all = []

    def __call__(self, shape, dtype, device, pad=37):
        n = 1
        for s in shape:
            n *= s
        big = torch.full((n + 2 * pad,), 77, dtype=dtype, device=device)
        self.all.append((big, n, pad))
        return big[pad:pad + n].view(shape)

    def check(self):
        for big, n, pad in self.all:
            assert (big[:pad] == 77).all() and (big[pad + n:] == 77).all()


@pytest.mark.parametrize("n,width,top", [(1, 1, 1), (3, 5, 4), (129, 33, 20), (70, 770, 64), (5, 20001, 7)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_beside_the_outputs(device, n, width, top, dtype):
    """Nothing is written outside the outputs, whatever their alignment."""
    new, f32 = Fenced(), torch.float32
    buf = lambda *s, t=dtype: new(s, t, device)   # noqa: E731
    g = torch.Generator(device).manual_seed(n)
    rnd = lambda *s: torch.randn(*s, device=device, generator=g).to(dtype)   # noqa: E731
    x, table = rnd(n, width), rnd(50, width)
    ids = torch.randint(50, (n,), device=device, generator=g)
    rla.rla_embed_forward(ids, table, out=buf(n, width))
    rla.rla_embed_backward(ids, x, 50, dtable=buf(50, width, t=f32))
    rla.rla_embed_backward(ids, x, 50, base=torch.ones(50, width, device=device), dtable=buf(50, width, t=f32))
    f = rla.rla_logprob_forward(x, torch.zeros(n, dtype=torch.int64, device=device), entropy=True, top=min(top, width),
                                out=buf(n, t=f32), lse=buf(n, t=f32), entropy_out=buf(n, t=f32),
                                top_logprobs=buf(n, min(top, width), t=f32), top_ids=buf(n, min(top, width), t=torch.int32))
    rla.rla_logprob_backward(x, f["lse"], torch.zeros(n, dtype=torch.int64, device=device), f["lse"], out=buf(n, width))
    A, cu = -torch.rand(width, device=device), torch.tensor([0, n // 3, n], dtype=torch.int32, device=device)
    for how in (dict(), dict(cu_seqlens=cu)):
        k = 2 if how else 1
        view = (lambda t: t) if how else (lambda t: t[None])
        xs = view(x)
        rla.rla_glr_forward(xs, xs, A, i=xs, z=xs, out=view(buf(n, width)), h_final=buf(k, width, t=f32), **how)
        grads = {m: view(buf(n, width)) for m in ("dx", "dr", "di", "dz")}
        grads.update(dA=buf(width, t=f32), dh0=buf(k, width, t=f32))
        rla.rla_glr_backward(xs, xs, A, xs, i=xs, z=xs, h0=torch.ones(k, width, device=device), grads=grads, **how)
    rla.rla_glr_decode(x[:, None], x[:, None], A, h_out=buf(n, width, t=f32), out=buf(n, 1, width))
    torch.cuda.synchronize()
    new.check()


def test_rows_far_apart(device):
    """Rows some 2^23 values apart: offsets of more than 32 bits give the same results."""
    T, D, apart = 600, 72, (1 << 23) - 1
    g = torch.Generator(device).manual_seed(4)
    space = torch.empty(T * apart, dtype=torch.bfloat16, device=device)
    near, far = {}, {}
    for k, n in enumerate(("x", "r", "i", "z", "dO", "logits")):
        width = 3000 if n == "logits" else D
        near[n] = torch.randn(T, width, device=device, generator=g).bfloat16()
        far[n] = space.as_strided((T, width), (apart, 1), 1 + 100 * k)
        far[n].copy_(near[n])
    A = -3 * torch.rand(D, device=device, generator=g)
    y = torch.randint(3000, (T,), device=device, generator=g)
    ids = torch.randint(200, (T,), device=device, generator=g)

    def results(v):
        o, h = rla.rla_glr_forward(v["x"], v["r"], A, i=v["i"], z=v["z"])
        b = rla.rla_glr_backward(v["x"], v["r"], A, v["dO"], i=v["i"], z=v["z"])
        o1, h1 = rla.rla_glr_decode(v["x"][:, None], v["r"][:, None], A, i=v["i"][:, None])
        f = rla.rla_logprob_forward(v["logits"], y, entropy=True, top=5)
        d = rla.rla_logprob_backward(v["logits"], f["lse"], y, f["lse"])
        e = rla.rla_embed_backward(ids, v["dO"], 200)
        return [o, h, o1, h1, d, e] + [t for r in (b, f) for _, t in sorted(r.items())]

    assert all(torch.equal(a, b) for a, b in zip(results(far), results(near)))


def test_more_rows_than_a_launch(device):
    """Rows of three logits and tokens of 2048 values beyond one launch's workgroups."""
    n = (1 << 25) + 5
    x = torch.randn(n, 3, device=device).bfloat16()
    y = torch.randint(3, (n,), device=device)
    f = rla.rla_logprob_forward(x, y)
    some = torch.tensor([0, 1, (1 << 25) - 1, 1 << 25, n - 1], device=device)
    want = ref.logprob(x[some].cpu().double(), y[some].cpu(), 1.0)
    assert (f["lse"][some].cpu().double() - want["lse"]).abs().max() < 1e-5
    assert (f["logprob"][some].cpu().double() - want["logprob"]).abs().max() < 1e-5
    d = rla.rla_logprob_backward(x, f["lse"], y, torch.ones(n, device=device))
    p = torch.softmax(x[some].float(), -1)
    p = torch.nn.functional.one_hot(y[some], 3) - p
    assert (d[some].float() - p).abs().max() < 2.0 ** -8
    del f, d, x, y
    n = (1 << 23) + 3
    table = torch.randn(1000, 2048, device=device).bfloat16()
    ids = torch.randint(1000, (n,), device=device)
    out = rla.rla_embed_forward(ids, table)
    some = torch.tensor([0, (1 << 23) - 1, 1 << 23, n - 1], device=device)
    assert torch.equal(out[some], table[ids[some]])


def test_calls_that_use_no_workspace(device):
    """Rows that a workgroup takes each, and whole sequences, need none from the caller, whatever room smaller calls
    have in one that is sized for them."""
    lib = model._lib()
    x = torch.randn(300, 65536, device=device)
    y = torch.zeros(300, dtype=torch.int64, device=device)
    problem = rla.make_logprob_problem(x)
    assert rla.rla_logprob_workspace_size(problem) > 0
    out, lse = torch.empty(2, 300, device=device)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.rla_logprob_forward(problem, x.data_ptr(), y.data_ptr(), out.data_ptr(), lse.data_ptr(), None, None, None, None, 0,
                                   stream) == 0
    want = rla.rla_logprob_forward(x, y)
    assert torch.equal(out, want["logprob"]) and torch.equal(lse, want["lse"])
    u, A = torch.randn(256, 30, 64, device=device), -torch.rand(64, device=device)
    problem, o = rla.make_glr_problem(u), torch.empty_like(u)
    assert rla.rla_glr_workspace_size(problem, rla.RLA_GLR_FORWARD) > 0
    assert lib.rla_glr_forward(problem, u.data_ptr(), u.data_ptr(), A.data_ptr(), None, None, None, o.data_ptr(), None, 0, None, 0,
                               stream) == 0
    assert torch.equal(o, rla.rla_glr_forward(u, u, A)[0])
