"""Performance cases of the operators at the ends of a language model and of a
recurrent mixer: the embedding lookup with its gradient, the gated linear
recurrence, and the log probabilities of given tokens with entropy, top
alternatives and their gradient.  Each case has its inputs, a plain form, its
work and a 64-bit reference.

A case is a dict of plain values:
  op        "embed", "glr" or "logprob"
  kind      "decode" (new tokens onto resident states), "forward" or "train"
            (forward, then every gradient)
  dtype     element type of the activations (embed: of the rows handed on;
            glr: x, gates, outputs; logprob: the logits)
  strided   activations are slices of wider rows
embed:
  tokens, V, D    token ids, rows of the table, values a row
  table     element type of the table
  add       the gradient is added to another's (a table shared with the output
            projection)
  pad       share of ids that are -1 (no token)
glr:
  B, T      dense [B, T, D]; or, packed (cu_seqlens),
  tokens, lo, hi, pack  sequences of lo..hi tokens drawn with the seed `pack`
            until they fill `tokens` (the last one is cut)
  D         channels
  i, z      input gate, output gate given
  norm      the input's factor sqrt(1 - a^2)
  states    initial states given (a continued sequence)
logprob:
  rows, V   rows of logits, tokens of the vocabulary
  scale     inverse temperature
  top       alternatives a row
  entropy   the rows' entropy (training: and its gradient)
  masked    share of the logits that are -inf
  ignored   share of the rows whose token is left out (-100)
"""
import math
import random

import torch

own = False
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _lib():
    import paper_2509_25223_amd as rla
    return rla


def _embed(name, kind, tokens, V, D, dtype="bf16", table="f32", scale=1.0, add=False, pad=0.0, strided=False):
    return dict(name=name, op="embed", kind=kind, dtype=dtype, tokens=tokens, V=V, D=D, table=table, scale=scale,
                add=add, pad=pad, strided=strided)


def _glr(name, kind, dtype="bf16", B=0, T=0, tokens=0, lo=0, hi=0, pack=0, D=2048, i=True, z=True, norm=True,
         states=False, strided=True):
    return dict(name=name, op="glr", kind=kind, dtype=dtype, B=B, T=T, tokens=tokens, lo=lo, hi=hi, pack=pack, D=D,
                i=i, z=z, norm=norm, states=states, strided=strided)


def _logprob(name, kind, rows, V, dtype="bf16", scale=1.0, top=0, entropy=False, masked=0.0, ignored=0.0,
             strided=False):
    return dict(name=name, op="logprob", kind=kind, dtype=dtype, rows=rows, V=V, scale=scale, top=top,
                entropy=entropy, masked=masked, ignored=ignored, strided=strided)


def listed():
    return [
        # one new token of each sequence of a full serving batch, bf16 table
        _embed("embed_decode", "forward", 256, 32768, 2048, table="bf16", scale=math.sqrt(2048.0)),
        # the training step's lookup out of the fp32 parameters, and their gradient
        _embed("embed_train", "train", 16384, 32768, 2048),
        # a table shared with the output projection, padded batch, odd sizes
        _embed("embed_train_shared", "train", 4099, 50001, 770, dtype="f32", scale=0.7, add=True, pad=0.1,
               strided=True),
        # one user's next token: the row's choice and alternatives, latency
        _logprob("logprob_b1", "forward", 1, 32768, dtype="f32", scale=1.25, top=20, entropy=True),
        # a serving batch over a large vocabulary, half of it not allowed by a grammar
        _logprob("logprob_decode", "forward", 64, 131072, top=8, entropy=True, masked=0.5),
        # scoring a prompt: each token's log probability and five alternatives; odd rows
        _logprob("logprob_prompt", "forward", 4001, 50001, top=5),
        # the training step's loss and its gradient: the largest
        _logprob("logprob_train", "train", 16384, 32768, ignored=0.05),
        # a policy's update: tempered log probabilities, entropy, both gradients
        _logprob("logprob_policy", "train", 3000, 20003, dtype="f32", scale=1.43, entropy=True, ignored=0.2),
        # a serving batch, one token each
        _glr("glr_decode", "decode", B=256, T=1, D=4096, states=True),
        # one long prompt onto given states: few channels, a long axis
        _glr("glr_prefill", "forward", B=1, T=16384, D=2048, states=True),
        # the training step of a layer
        _glr("glr_train", "train", B=4, T=4096, D=4096, strided=False),
        # a small fp32 model on packed documents, odd sizes
        _glr("glr_train_f32", "train", dtype="f32", tokens=3001, lo=1, hi=900, pack=5, D=514, z=False),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A row's width: a multiple of 64 more often than an odd one."""
    x = _between(rng, lo, hi)
    return x if rng.random() < 0.35 else max(64, (x + 32) // 64 * 64)


def draw(rng):
    op = rng.choice(["embed", "logprob", "logprob", "glr", "glr"])
    kind = rng.choice(["forward", "train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    strided = rng.random() < 0.4
    if op == "embed":
        V = _width(rng, 60, 131072)
        D = _width(rng, 20, min(8192, (1 << 26) // V))
        add = rng.random() < 0.4
        c = _embed("", kind, _between(rng, 1, min(20000, (1 << 25) // D)), V, D, dtype=dtype,
                   table=rng.choice(["f32", dtype]), scale=rng.choice([1.0, round(rng.uniform(0.1, 60.0), 3)]), add=add,
                   pad=rng.choice([0.0, 0.0, 0.15]), strided=strided)
    elif op == "logprob":
        V = _width(rng, 60, 200000)
        most = (1 << 28) // V if dtype == "f32" else (1 << 29) // V
        c = _logprob("", kind, _between(rng, 1, min(16384, most)), V, dtype=dtype,
                     scale=rng.choice([1.0, round(rng.uniform(0.3, 2.0), 3)]),
                     top=0 if kind == "train" else rng.choice([0, 1, 3, 8, 20, 50]), entropy=rng.random() < 0.5,
                     masked=rng.choice([0.0, 0.0, 0.5, 0.98]) if kind == "forward" else 0.0,
                     ignored=rng.choice([0.0, 0.1]), strided=strided)
    else:
        D = _width(rng, 32, 4096)
        how = dict(dtype=dtype, D=D, i=rng.random() < 0.8, z=rng.random() < 0.5, norm=rng.random() < 0.75,
                   states=rng.random() < 0.4, strided=strided)
        if rng.random() < 0.25:
            kind = "decode"
            how.update(B=_between(rng, 1, 300), T=rng.choice([1, 1, 1, 2, 5, 8]), states=True)
        elif rng.random() < 0.4:
            tokens = _between(rng, 300, min((1 << 25) // D, 20000))
            how.update(tokens=tokens, lo=rng.randint(1, 200), hi=_between(rng, 300, 4000), pack=rng.randrange(1 << 20))
        else:
            T = _between(rng, 1, min((1 << 25) // D, 12000))
            how.update(T=T, B=_between(rng, 1, max(1, min(32, (1 << 25) // (D * T)))))
        c = _glr("", kind, **how)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(c):
    if not c["tokens"]:
        return [c["T"]] * c["B"]
    r, got = random.Random(c["pack"]), []
    while sum(got) < c["tokens"]:
        got.append(min(r.randint(c["lo"], c["hi"]), c["tokens"] - sum(got)))
    return got


def _inputs(c, seed):
    dev = torch.device("cuda")
    g = torch.Generator(dev).manual_seed(seed)
    dt = TYPES[c["dtype"]]
    x = {"case": dict(c)}

    def normal(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    def uniform(*shape):
        return torch.rand(*shape, device=dev, generator=g)

    def rows(lead, *widths, factor=1.0):
        """Activations of these widths: slices of one wider tensor, or tensors of their own."""
        if not c["strided"]:
            return [(factor * normal(*lead, w)).to(dt) for w in widths]
        wide, at = (factor * normal(*lead, sum(widths) + 64)).to(dt), 32
        out = []
        for w in widths:
            out.append(wide[..., at:at + w])
            at += w
        return out

    def text(n, V):
        """Token ids as frequent as words are: the k-th in proportion to 1 / k, over a fixed shuffle."""
        rank = torch.exp(uniform(n) * math.log(V + 1.0)).long().clamp_(1, V) - 1
        return torch.randperm(V, device=dev, generator=torch.Generator(dev).manual_seed(1))[rank]

    if c["op"] == "embed":
        n, V, D = c["tokens"], c["V"], c["D"]
        ids = text(n, V)
        x["ids"] = torch.where(uniform(n) < c["pad"], torch.full_like(ids, -1), ids)
        x["table"] = normal(V, D).to(TYPES[c["table"]])
        if c["kind"] == "train":
            x["dout"], = rows((n,), D)
            x["before"] = normal(V, D) if c["add"] else None
    elif c["op"] == "logprob":
        n, V = c["rows"], c["V"]
        x["logits"], = rows((n,), V, factor=2.5)
        x["targets"] = text(n, V)
        # half of the rows know their token
        known = x["targets"][:(n + 1) // 2, None]
        x["logits"][:(n + 1) // 2].scatter_add_(1, known, torch.full_like(known, 9, dtype=dt))
        if c["masked"]:
            x["logits"].masked_fill_(uniform(V) < c["masked"], float("-inf"))
        x["targets"] = torch.where(uniform(n) < c["ignored"], torch.full_like(x["targets"], -100), x["targets"])
        if c["kind"] == "train":
            x["dlogprob"] = -(0.5 + uniform(n)) / n
            x["dentropy"] = 0.01 * normal(n) / n if c["entropy"] else None
    else:
        lens, D = _lengths(c), c["D"]
        lead, N = ((sum(lens),) if c["tokens"] else (c["B"], c["T"])), len(lens)
        x["lens"] = lens
        x["cu"] = torch.tensor([0] + lens, device=dev).cumsum(0).to(torch.int32) if c["tokens"] else None
        r, i, z = rows(lead, D, D, D)
        x["x"] = normal(*lead, D).to(dt)                    # the convolution's output
        x["r"], x["i"], x["z"] = r, i if c["i"] else None, z if c["z"] else None
        # decays of 0.9 to 0.999 at an open gate, a power of 8 of them
        base = 0.9 + 0.099 * uniform(D)
        x["A"] = 8.0 * torch.log(base)
        x["h0"] = 0.5 * normal(N, D) if c["states"] else None
        if c["kind"] == "train":
            x["dO"] = normal(*lead, D).to(dt)
    return x


def prepare(case, seed):
    """The inputs and the buffers that a serving or training loop keeps between calls."""
    c, x = case, _inputs(case, seed)
    dev = torch.device("cuda")

    def new(shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=dev)

    train = c["kind"] == "train"
    x["workspace"] = None
    if c["op"] == "embed":
        x["buffers"] = {"out": new((c["tokens"], c["D"]), TYPES[c["dtype"]])}
        if train:
            x["dtable"] = new((c["V"], c["D"]))
    elif c["op"] == "logprob":
        n = c["rows"]
        x["buffers"] = {"out": new(n), "lse": new(n)}
        if c["entropy"]:
            x["buffers"]["entropy_out"] = new(n)
        if c["top"]:
            x["buffers"].update(top_logprobs=new((n, c["top"])), top_ids=new((n, c["top"]), torch.int32))
        if train:
            x["dlogits"] = new(x["logits"].shape, x["logits"].dtype)
    else:
        state = "h_out" if c["kind"] == "decode" else "h_final"
        x["buffers"] = {"out": new(x["x"].shape, x["x"].dtype), state: new((len(x["lens"]), c["D"]))}
    if own:
        lib, size = _lib(), 0
        if c["op"] == "embed" and train:
            size = lib.rla_embed_workspace_size(lib.make_embed_problem(x["ids"], x["table"]))
        elif c["op"] == "logprob":
            size = lib.rla_logprob_workspace_size(lib.make_logprob_problem(x["logits"], top=c["top"]))
        elif c["op"] == "glr" and c["kind"] != "decode":
            size = lib.rla_glr_workspace_size(lib.make_glr_problem(x["x"], x["cu"]),
                                              lib.RLA_GLR_BACKWARD if train else lib.RLA_GLR_FORWARD)
        x["workspace"] = new(max(1, size), torch.uint8)
    return x


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(x):
    c = x["case"]
    if not own:
        with torch.no_grad():
            return {"embed": _plain_embed, "logprob": _plain_logprob, "glr": _plain_glr}[c["op"]](c, x)
    lib, buf, train = _lib(), x["buffers"], c["kind"] == "train"
    if c["op"] == "embed":
        out = {"out": lib.rla_embed_forward(x["ids"], x["table"], scale=c["scale"], **buf)}
        if train:
            out["dtable"] = lib.rla_embed_backward(x["ids"], x["dout"], c["V"], scale=c["scale"], base=x["before"],
                                                   dtable=x["dtable"], workspace=x["workspace"])
        return out
    if c["op"] == "logprob":
        got = lib.rla_logprob_forward(x["logits"], x["targets"], scale=c["scale"], entropy=c["entropy"], top=c["top"],
                                      workspace=x["workspace"], **buf)
        out = {k: v for k, v in got.items() if v is not None}
        if train:
            out["dlogits"] = lib.rla_logprob_backward(x["logits"], out["lse"], x["targets"], x["dlogprob"],
                                                      entropy=out.get("entropy"), dentropy=x["dentropy"],
                                                      scale=c["scale"], out=x["dlogits"])
        return out
    args, how = [x["x"], x["r"], x["A"]], dict(i=x["i"], z=x["z"], normalize=c["norm"])
    if c["kind"] == "decode":
        o, h = lib.rla_glr_decode(*args, **how, h_in=x["h0"], **buf)
        return {"o": o, "h": h}
    how.update(h0=x["h0"], cu_seqlens=x["cu"], workspace=x["workspace"])
    o, h = lib.rla_glr_forward(*args, **how, **buf, save_for_backward=train)
    out = {"o": o, "h": h}
    if train:
        out.update(lib.rla_glr_backward(*args, x["dO"], **how, use_saved=True))
    return out


# ---------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits, rounded once at the end
# ---------------------------------------------------------------------------

def _plain_embed(c, x):
    ids, there = x["ids"].clamp(min=0), (x["ids"] >= 0)[:, None]
    out = {"out": (c["scale"] * x["table"][ids].float() * there).to(TYPES[c["dtype"]])}
    if c["kind"] == "train":
        grad = torch.zeros(c["V"], c["D"], device=ids.device) if x["before"] is None else x["before"].clone()
        out["dtable"] = grad.index_add_(0, ids, c["scale"] * x["dout"].float() * there)
    return out


def _plain_logprob(c, x):
    z = x["logits"].float() * c["scale"]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    there = (x["targets"] >= 0)[:, None]
    at = x["targets"].clamp(min=0)[:, None]
    lp = z - lse
    got = {"logprob": torch.where(there, lp.gather(1, at), 0.0)[:, 0], "lse": lse[:, 0]}
    if c["entropy"]:
        plogp = torch.where(e > 0, e * lp, 0.0)
        entropy = -plogp.sum(-1, keepdim=True) / total
        got["entropy"] = entropy[:, 0]
    if c["top"]:
        # whole-number keys in the order of the values, equal values by their place
        bits = (x["logits"].float() + 0.0).view(torch.int32).long()
        keys = torch.where(bits < 0, -2147483648 - bits, bits) * (1 << 32) + (c["V"] - 1 - torch.arange(
            c["V"], device=z.device))
        best = torch.topk(keys, c["top"], -1).values
        ids = c["V"] - 1 - (best & ((1 << 32) - 1))
        alternatives = lp.gather(1, ids)
        got["top_logprobs"] = alternatives
        got["top_ids"] = torch.where(alternatives > float("-inf"), ids, -1).to(torch.int32)
    if c["kind"] == "train":
        p = e / total
        g = torch.where(there, x["dlogprob"][:, None], 0.0)
        d = -g * p
        if c["entropy"]:
            d -= x["dentropy"][:, None] * torch.where(p > 0, p * (lp + entropy), 0.0)
        got["dlogits"] = (c["scale"] * d.scatter_add(1, at, g)).to(x["logits"].dtype)
    return got


def _places(lens, dev):
    """[sequences, longest]: the token at each place of each sequence, and whether there is one."""
    n = torch.tensor(lens, device=dev)
    t = torch.arange(max(lens), device=dev)
    there = t < n[:, None]
    return torch.where(there, n.cumsum(0)[:, None] - n[:, None] + t, 0), there


def _spread(x, y, empty=0.0):
    """Token rows as [sequences, longest, width] in 32 bits, `empty` past a sequence's end."""
    if x["cu"] is None:
        return y.float()
    at, there = _places(x["lens"], y.device)
    return torch.where(there[..., None], y[at].float(), empty)


def _gather(x, y, like):
    """_spread undone, in the type of `like`."""
    return (y if x["cu"] is None else y[_places(x["lens"], y.device)[1]]).to(like.dtype)


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the second dimension, from 0: steps of 1, 2, 4, .. tokens."""
    step = 1
    while step < a.shape[1]:
        b = torch.cat([b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def _sigmoid(t):
    return 1 / (1 + torch.exp(-t))


def _plain_glr(c, x):
    u, A = _spread(x, x["x"]), x["A"]
    sr = _sigmoid(_spread(x, x["r"], float("-inf")))          # (past an end: the state stays)
    si = 1.0 if x["i"] is None else _sigmoid(_spread(x, x["i"]))
    a = torch.exp(A * sr)
    m = torch.sqrt(-torch.expm1(2 * A * sr)) if c["norm"] else torch.ones_like(a)
    b = m * si * u
    first = x["h0"]
    if first is not None:
        b = torch.cat([b[:, :1] + a[:, :1] * first[:, None], b[:, 1:]], 1)
    h = _scan(a, b)
    out = {"h": h[:, -1]}
    if x["z"] is not None:
        z = _spread(x, x["z"])
        sz = _sigmoid(z)
    out["o"] = _gather(x, h if x["z"] is None else h * z * sz, x["x"])
    if c["kind"] != "train":
        return out
    d = _spread(x, x["dO"])
    if x["z"] is not None:
        out["dz"] = _gather(x, d * h * sz * (1 + z * (1 - sz)), x["z"])
        d = d * z * sz
    behind = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    lam = _scan(behind.flip(1), d.flip(1)).flip(1)
    before = torch.cat([torch.zeros_like(h[:, :1]) if first is None else first[:, None], h[:, :-1]], 1)
    dlog = lam * before * a
    if c["norm"]:
        dlog = dlog - torch.where(m > 0, lam * si * u * a * a / m, 0.0)
    out["dx"] = _gather(x, lam * m * si, x["x"])
    out["dr"] = _gather(x, dlog * A * sr * (1 - sr), x["r"])
    out["dA"] = (dlog * sr).sum((0, 1))
    if x["i"] is not None:
        out["di"] = _gather(x, lam * m * u * si * (1 - si), x["i"])
    if first is not None:
        out["dh0"] = a[:, 0] * lam[:, 0]
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once and each output written once (a table's gradient, and what it is added to, whole).
    A logit is 5 operations (factor, maximum, exponential, two sums) and 7 in the gradient; a value of the recurrence 24
    (three gates, the decay, the factor, a multiply-add), its gradient twice as many."""
    c, el = case, 2 if case["dtype"] == "bf16" else 4
    train = c["kind"] == "train"
    if c["op"] == "embed":
        n, V, D = c["tokens"], c["V"], c["D"]
        b, f = n * D * (el + (2 if c["table"] == "bf16" else 4)) + 8 * n, n * D
        if train:
            b += n * D * el + 8 * n + 4 * V * D + (4 * V * D if c["add"] else 0)
            f += n * D
        return {"bytes": b, "flops": f}
    if c["op"] == "logprob":
        n, V = c["rows"], c["V"]
        b, f = n * V * el + n * (16 + 4 * c["entropy"] + 8 * c["top"]), n * V * 5
        if train:
            b, f = b + n * V * el + n * (4 + 4 * c["entropy"]), f + n * V * 7
        return {"bytes": b, "flops": f}
    lens, D = _lengths(c), c["D"]
    tok, state, rows = sum(lens), 4 * len(lens) * D, 2 + c["i"] + c["z"]
    b, f = tok * D * el * (rows + 1) + state * (2 if c["states"] else 1) + 4 * D, tok * D * 24
    if train:
        b, f = b + tok * D * el * (rows + 1) + 4 * D + (state if c["states"] else 0), f * 3
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

def _exact_embed(c, v):
    known = v["ids"] >= 0
    pick = v["ids"][known]
    out = torch.zeros(c["tokens"], c["D"], dtype=torch.float64, device=pick.device)
    out[known] = v["table"].index_select(0, pick) * c["scale"]
    got = {"out": out}
    if c["kind"] == "train":
        # the rows of equal ids side by side, their sums as differences between the ids' places
        order = torch.argsort(pick)
        rows = v["dout"][known].index_select(0, order) * c["scale"]
        run_, count = torch.unique_consecutive(pick[order], return_counts=True)
        sums = torch.segment_reduce(rows, "sum", lengths=count, axis=0) if count.numel() else rows
        grad = torch.zeros(c["V"], c["D"], dtype=torch.float64, device=pick.device)
        grad[run_] = sums
        got["dtable"] = grad if v["before"] is None else grad + v["before"]
    return got


def _exact_logprob(c, v):
    """A block of rows at a time."""
    parts = []
    for a in range(0, c["rows"], 1024):
        z = (v["logits"][a:a + 1024].double() * c["scale"]).requires_grad_(c["kind"] == "train")
        y = v["targets"][a:a + 1024]
        lp = torch.log_softmax(z, -1)
        given = torch.where(y >= 0, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lp[:, 0]))
        got = {"logprob": given, "lse": torch.logsumexp(z, -1)}
        if c["entropy"]:
            got["entropy"] = torch.special.entr(torch.exp(lp)).sum(-1) if c["kind"] != "train" else \
                -(torch.exp(lp) * lp).sum(-1)
        if c["top"]:
            order = torch.sort(v["logits"][a:a + 1024].float(), dim=-1, descending=True,
                               stable=True).indices[:, :c["top"]]
            best = lp.gather(1, order)
            got["top_logprobs"] = best
            got["top_ids"] = torch.where(torch.isinf(best), -1, order).to(torch.int32)
        if c["kind"] == "train":
            up = (given * v["dlogprob"][a:a + 1024]).sum()
            if c["entropy"]:
                up = up + (got["entropy"] * v["dentropy"][a:a + 1024]).sum()
            got["dlogits"] = torch.autograd.grad(up, z)[0] * c["scale"]
        parts.append({n: t.detach() for n, t in got.items()})
    return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}


def _exact_glr(c, v, lens):
    """Token after token, the sequences side by side."""
    train, L, dev = c["kind"] == "train", max(lens), v["x"].device
    start = torch.tensor([0] + lens[:-1], device=dev).cumsum(0)
    inside = torch.arange(L, device=dev) < torch.tensor(lens, device=dev)[:, None]
    at = torch.where(inside, start[:, None] + torch.arange(L, device=dev), 0)
    flat = {n: v[n].reshape(sum(lens), -1) for n in ("x", "r", "i", "z") if v[n] is not None}
    log_a = torch.sigmoid(flat["r"]) * v["A"]
    into = flat["x"]
    if "i" in flat:
        into = into * torch.sigmoid(flat["i"])
    if c["norm"]:
        into = into * torch.sqrt(1 - torch.exp(2 * log_a))
    a_of, b_of = torch.exp(log_a)[at], into[at]
    h = torch.zeros(len(lens), c["D"], dtype=torch.float64, device=dev) if v["h0"] is None else v["h0"]
    leaves = a_of.detach(), b_of.detach(), h.detach()
    hs, h_now = [], leaves[2]
    for t in range(L):
        h_now = torch.where(inside[:, t, None], leaves[0][:, t] * h_now + leaves[1][:, t], h_now)
        hs.append(h_now)
    states = torch.stack(hs, 1).requires_grad_(train)
    y = torch.empty_like(flat["x"])
    y = y.index_put((at[inside],), states[inside])
    o = y if "z" not in flat else y * flat["z"] * torch.sigmoid(flat["z"])
    out = {"o": o.detach().reshape(v["x"].shape), "h": h_now}
    if not train:
        return out
    # the adjoint of h_t = a h + b, from the last token on
    wanted = [states] + ([v["z"]] if v["z"] is not None else [])
    dstates, *dz = torch.autograd.grad(o, wanted, v["dO"].reshape(o.shape))
    carry, da, db = torch.zeros_like(h_now), torch.zeros_like(a_of), torch.zeros_like(b_of)
    for t in reversed(range(L)):
        live = inside[:, t, None]
        total = carry + dstates[:, t]
        prev = hs[t - 1] if t else leaves[2]
        da[:, t], db[:, t] = total * prev * live, total * live
        carry = torch.where(live, total * leaves[0][:, t], carry)
    names = ["x", "r", "A"] + (["i"] if v["i"] is not None else [])
    out.update(zip(["d" + n for n in names], torch.autograd.grad([a_of, b_of], [v[n] for n in names], [da, db])))
    if dz:
        out["dz"] = dz[0]
    if v["h0"] is not None:
        out["dh0"] = carry
    return out


def exact(case, seed):
    c, v = case, {}
    if c["op"] == "glr" and max(_lengths(c)) > 60000:
        return None
    for n, t in _inputs(c, seed).items():
        # (logits are taken to 64 bits a block at a time)
        if isinstance(t, torch.Tensor) and t.is_floating_point() and n != "logits":
            t = t.double()
            if c["op"] == "glr" and c["kind"] == "train" and n != "dO":
                t = t.clone().requires_grad_(True)
        v[n] = t
    if c["op"] == "embed":
        return _exact_embed(c, v)
    if c["op"] == "logprob":
        return _exact_logprob(c, v)
    got = _exact_glr(c, v, _lengths(c))
    return {n: t.detach() for n, t in got.items()}
