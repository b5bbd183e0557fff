"""A small language model from the package's operators, trained and then served.

One residual stream (fp32) and two mixing blocks on it:

  n, r = addnorm(embed(tokens))
  block 1   q, k, v, gate, four gates = n W1;  q, k, v through a short convolution;
            Residual Delta Net;  gated norm per head;  x = .. W2
  n, r = addnorm(x, r)
  block 2   u, delta, z, B, C = n W3;  u through a short convolution;  selective
            scan;  gated norm;  x = .. W4
  n, r = addnorm(x, r);  logits = n W5;  loss: their log probabilities of the next tokens

`Model.forward` takes a batch [B, T] or packed sequences [T] with their offsets, and
returns each sequence's state; `Model.decode` carries such states one token on, in
place; `Model.gradients` is the training step's backward.  The projections are torch;
what is between them, the lookup of the tokens and the loss are the package's calls.

  python examples/hybrid_model.py [--steps 400]

trains on periodic sequences and continues prompts of several lengths.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_25223_amd as rla  # noqa: E402

RAW = rla.RLA_FLAG_QK_SILU_L2NORM | rla.RLA_FLAG_GATE_PREACT   # q, k and gates as projected


class Model:
    def __init__(self, vocab=64, width=256, heads=2, head=128, channels=256, states=16, taps=4, dtype=torch.bfloat16,
                 device="cuda", seed=0):
        self.vocab, self.width, self.H, self.d = vocab, width, heads, head
        self.D, self.N, self.taps, self.dtype, self.device = channels, states, taps, dtype, device
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g)).to(device)   # noqa: E731
        Hd, D, N = heads * head, channels, states
        # parameters in fp32; projections are used in `dtype`
        self.p = dict(
            embed=rnd(vocab, width), norm1=torch.ones(width, device=device),
            w1=rnd(width, 4 * Hd + 4 * heads, scale=width ** -0.5), conv1=rnd(3 * Hd, taps, scale=taps ** -0.5),
            decay=torch.tensor([[0.5] * heads, [-3.0] * heads], device=device), gate1=torch.ones(head, device=device),
            w2=rnd(Hd, width, scale=Hd ** -0.5), scale2=torch.ones(width, device=device),
            norm2=torch.ones(width, device=device), w3=rnd(width, 3 * D + 2 * N, scale=width ** -0.5),
            conv2=rnd(D, taps, scale=taps ** -0.5), conv2_bias=torch.zeros(D, device=device),
            A=-torch.arange(1, N + 1, device=device).float().repeat(D, 1), skip=torch.ones(D, device=device),
            step=torch.full((D,), -3.0, device=device), gate2=torch.ones(D, device=device),
            w4=rnd(D, width, scale=D ** -0.5), scale3=torch.ones(width, device=device),
            norm3=torch.ones(width, device=device), w5=rnd(width, vocab, scale=width ** -0.5))

    def _cast(self, name):
        return self.p[name].to(self.dtype)

    def _split1(self, x):
        """q, k, v, gate [.., H d] and the four gates [.., H] of block 1's projection."""
        Hd, H = self.H * self.d, self.H
        parts = x.split([Hd] * 4 + [H] * 4, -1)
        return parts[:4], [t.float().contiguous() for t in parts[4:]]

    def _split3(self, x):
        """u, delta, z [.., D] and B, C [.., 1, N]: rows of the projection as they lie"""
        u, delta, z, B, C = x.split([self.D] * 3 + [self.N] * 2, -1)
        return u, delta, z, B.unflatten(-1, (1, self.N)), C.unflatten(-1, (1, self.N))

    def _heads(self, x):
        return x.unflatten(-1, (self.H, self.d))

    def _conv1(self, i):
        Hd = self.H * self.d
        return self.p["conv1"][i * Hd:(i + 1) * Hd]

    def forward(self, tokens, cu_seqlens=None, state=None, save=False):
        """(logits, state) of tokens [B, T], or packed [T]; `state`: the one that the
        sequences continue.  With save, also what `gradients` needs."""
        p, n_of = self.p, (lambda s, key: None if s is None else s[key])
        tokens = tokens.contiguous()   # (slices of a batch)
        x0 = rla.rla_embed_forward(tokens, p["embed"], out_dtype=self.dtype)
        n1, r1 = rla.rla_addnorm_forward(x0, p["norm1"])
        p1 = n1 @ self._cast("w1")
        (q, k, v, gate), gates = self._split1(p1)
        mixed, new = [], {}
        for i, t in enumerate((q, k, v)):   # q and k take their SiLU with their norm
            y, new["conv1.%d" % i] = rla.rla_conv_forward(t, self._conv1(i), silu=i == 2, cu_seqlens=cu_seqlens,
                                                          state=n_of(state, "conv1.%d" % i))
            mixed.append(self._heads(y))
        rdn = dict(S0=n_of(state, "S"), R0=n_of(state, "R"), cu_seqlens=cu_seqlens, variants=RAW, decay_param=p["decay"],
                   out_dtype=self.dtype)
        work = None
        if save:
            problem = rla.make_problem(mixed[0], mixed[2], cu_seqlens, out_dtype=self.dtype,
                                       flags=rla.RLA_FLAG_SAVE_FOR_BACKWARD | RAW, decay_param=p["decay"])
            work = torch.empty(rla.rla_workspace_size(problem, rla.RLA_OP_RDN_BACKWARD), dtype=torch.uint8,
                               device=self.device)
        o1, new["S"], new["R"] = rla.rdn_forward(*mixed, *gates, save_for_backward=save, workspace=work, **rdn)
        y1 = rla.rla_gatenorm_forward(o1, self._heads(gate), p["gate1"])
        x1 = y1.flatten(-2) @ self._cast("w2")

        n2, r2 = rla.rla_addnorm_forward(x1, p["norm2"], residual=r1, scale=p["scale2"])
        p3 = n2 @ self._cast("w3")
        u, delta, z, B, C = self._split3(p3)
        u2, new["conv2"] = rla.rla_conv_forward(u, p["conv2"], bias=p["conv2_bias"], silu=True, cu_seqlens=cu_seqlens,
                                                state=n_of(state, "conv2"))
        scan = dict(D=p["skip"], delta_bias=p["step"], h0=n_of(state, "h"), cu_seqlens=cu_seqlens)
        o2, new["h"] = rla.rla_ssm_forward(u2, delta, p["A"], B, C, **scan)
        y2 = rla.rla_gatenorm_forward(o2[..., None, :], z[..., None, :], p["gate2"], gate_first=True)
        x2 = y2[..., 0, :] @ self._cast("w4")

        n3, r3 = rla.rla_addnorm_forward(x2, p["norm3"], residual=r2, scale=p["scale3"])
        logits = (n3 @ self._cast("w5")).float()
        if not save:
            return logits, new
        return logits, new, dict(tokens=tokens, cu=cu_seqlens, n1=n1, r1=r1, p1=p1, mixed=mixed, gates=gates, work=work,
                                 rdn=rdn, o1=o1, y1=y1, x1=x1, n2=n2, r2=r2, p3=p3, u2=u2, scan=scan, o2=o2, y2=y2,
                                 x2=x2, n3=n3, r3=r3)

    def decode(self, tokens, state):
        """Logits [B, vocab] of the token behind tokens [B]; `state` moves on in place."""
        p = self.p
        x0 = rla.rla_embed_forward(tokens.contiguous()[:, None], p["embed"], out_dtype=self.dtype)
        n1, r = rla.rla_addnorm_forward(x0, p["norm1"])
        (q, k, v, gate), gates = self._split1(n1 @ self._cast("w1"))
        mixed = []
        for i, t in enumerate((q, k, v)):
            s = state["conv1.%d" % i]
            mixed.append(self._heads(rla.rla_conv_decode(t, self._conv1(i), silu=i == 2, state=s, state_out=s)[0]))
        S, R = state["S"], state["R"]
        o1, _, _ = rla.rdn_decode(*mixed, *gates, S_in=S, R_in=R, S_out=S, R_out=R, variants=RAW, decay_param=p["decay"],
                                  out_dtype=self.dtype)
        y1 = rla.rla_gatenorm_forward(o1, self._heads(gate), p["gate1"])
        n2, _ = rla.rla_addnorm_forward(y1.flatten(-2) @ self._cast("w2"), p["norm2"], residual=r, scale=p["scale2"],
                                        residual_out=r)
        u, delta, z, B, C = self._split3(n2 @ self._cast("w3"))
        s, h = state["conv2"], state["h"]
        u2, _ = rla.rla_conv_decode(u, p["conv2"], bias=p["conv2_bias"], silu=True, state=s, state_out=s)
        o2, _ = rla.rla_ssm_decode(u2, delta, p["A"], B, C, D=p["skip"], delta_bias=p["step"], h_in=h, h_out=h)
        y2 = rla.rla_gatenorm_forward(o2[..., None, :], z[..., None, :], p["gate2"], gate_first=True)
        n3, _ = rla.rla_addnorm_forward(y2[..., 0, :] @ self._cast("w4"), p["norm3"], residual=r, scale=p["scale3"],
                                        residual_out=r)
        return (n3[:, 0] @ self._cast("w5")).float()

    def loss(self, logits, targets):
        """Mean cross entropy, and its gradient by the logits."""
        if logits.dtype == torch.float64:   # (for differences: the definition)
            lp = torch.log_softmax(logits, -1)
            p = lp.exp().scatter_add(-1, targets[..., None], torch.full_like(lp[..., :1], -1))
            return -lp.gather(-1, targets[..., None]).mean(), p / targets.numel()
        logits, targets = logits.contiguous(), targets.contiguous()
        f = rla.rla_logprob_forward(logits, targets)
        up = torch.full_like(f["lse"], -1.0 / targets.numel())
        return -f["logprob"].mean(), rla.rla_logprob_backward(logits, f["lse"], targets, up)

    def gradients(self, dlogits, s):
        """Gradients of every parameter, from the gradient by the logits and what
        `forward` saved."""
        p, g = self.p, {}

        def through(name, x, dy):   # y = x W
            flat, up = x.flatten(0, -2), dy.flatten(0, -2)
            g[name] = (flat.t() @ up).float()
            return dy @ self._cast(name).t()

        dn3 = through("w5", s["n3"], dlogits.to(self.dtype))
        b = rla.rla_addnorm_backward(dn3, s["r3"], p["norm3"], x=s["x2"], scale=p["scale3"])
        g["norm3"], g["scale3"], dr = b["dweight"], b["dscale"], b["dresidual"]
        dy2 = through("w4", s["y2"][..., 0, :], b["dx"])
        u, delta, z, B, C = self._split3(s["p3"])
        b = rla.rla_gatenorm_backward(dy2[..., None, :], s["o2"][..., None, :], z[..., None, :], p["gate2"],
                                      gate_first=True)
        g["gate2"], dz = b["dweight"], b["dgate"][..., 0, :]
        b = rla.rla_ssm_backward(s["u2"], delta, p["A"], B, C, b["dx"][..., 0, :], **s["scan"])
        g["A"], g["skip"], g["step"] = b["dA"], b["dD"], b["ddelta_bias"]
        c = rla.rla_conv_backward(u, p["conv2"], b["du"], bias=p["conv2_bias"], silu=True, cu_seqlens=s["cu"])
        g["conv2"], g["conv2_bias"] = c["dweight"], c["dbias"]
        dp3 = torch.cat([c["dx"], b["ddelta"], dz, b["dB"][..., 0, :], b["dC"][..., 0, :]], -1)
        dn2 = through("w3", s["n2"], dp3)
        b = rla.rla_addnorm_backward(dn2, s["r2"], p["norm2"], x=s["x1"], scale=p["scale2"], dresidual_out=dr)
        g["norm2"], g["scale2"], dr = b["dweight"], b["dscale"], b["dresidual"]

        dy1 = through("w2", s["y1"].flatten(-2), b["dx"])
        (q, k, v, gate), _ = self._split1(s["p1"])
        b = rla.rla_gatenorm_backward(self._heads(dy1), s["o1"], self._heads(gate), p["gate1"])
        g["gate1"], dgate = b["dweight"], b["dgate"].flatten(-2)
        b = rla.rdn_backward(*s["mixed"], *s["gates"], b["dx"], use_saved=True, workspace=s["work"], **s["rdn"])
        g["decay"] = b["ddecay_param"]
        dx, dw = [], []
        for i, (t, name) in enumerate(zip((q, k, v), ("dq", "dk", "dv"))):
            c = rla.rla_conv_backward(t, self._conv1(i), b[name].flatten(-2), silu=i == 2, cu_seqlens=s["cu"])
            dx.append(c["dx"])
            dw.append(c["dweight"])
        g["conv1"] = torch.cat(dw)
        dgates = [b[name].to(self.dtype) for name in ("dalpha_s", "dbeta", "dalpha_r", "dgamma")]
        dn1 = through("w1", s["n1"], torch.cat(dx + [dgate] + dgates, -1))
        b = rla.rla_addnorm_backward(dn1, s["r1"], p["norm1"], dresidual_out=dr)
        g["norm1"] = b["dweight"]
        g["embed"] = rla.rla_embed_backward(s["tokens"], b["dx"], self.vocab)
        return g


def periodic(vocab, batch, length, generator):
    """Sequences that repeat a random word of 3 to 8 tokens."""
    rows = []
    for _ in range(batch):
        word = torch.randint(vocab, (int(torch.randint(3, 9, (1,), generator=generator)),), generator=generator)
        rows.append(word.repeat(length // len(word) + 1)[:length])
    return torch.stack(rows)


def train(model, steps, batch=16, length=128, rate=3e-3, seed=1, report=None):
    """Adam on periodic sequences; the losses."""
    gen, losses = torch.Generator().manual_seed(seed), []
    m = {n: torch.zeros_like(t) for n, t in model.p.items()}
    v = {n: torch.zeros_like(t) for n, t in model.p.items()}
    for i in range(1, steps + 1):
        data = periodic(model.vocab, batch, length + 1, gen).to(model.device)
        logits, _, saved = model.forward(data[:, :-1], save=True)
        loss, dlogits = model.loss(logits, data[:, 1:])
        for n, grad in model.gradients(dlogits, saved).items():
            m[n].lerp_(grad, 0.1)
            v[n].lerp_(grad * grad, 0.02)
            model.p[n] -= rate * (m[n] / (1 - 0.9 ** i)) / ((v[n] / (1 - 0.98 ** i)).sqrt() + 1e-8)
        model.p["A"].clamp_(max=-1e-3)                # states decay
        model.p["decay"][0].clamp_(min=1e-3)
        losses.append(loss.item())
        if report and i % report == 0:
            print("step %4d  loss %.3f" % (i, losses[-1]), flush=True)
    return losses


def likeliest(logits):
    return rla.rla_logprob_forward(logits, top=1)["top_ids"][..., 0]


def generate(model, prompts, count):
    """The `count` likeliest tokens behind each prompt: the prompts packed in one call,
    then a token of each at a time."""
    ends = torch.tensor([0] + [len(t) for t in prompts]).cumsum(0)
    cu = ends.to(model.device, torch.int32)
    logits, state = model.forward(torch.cat(prompts).to(model.device), cu_seqlens=cu)
    token = likeliest(logits[(ends[1:] - 1).to(model.device)])
    out = [token]
    for _ in range(count - 1):
        token = likeliest(model.decode(token, state))
        out.append(token)
    return torch.stack(out, 1).long().cpu()


def main():
    args = argparse.ArgumentParser()
    args.add_argument("--steps", type=int, default=400)
    args = args.parse_args()
    model = Model()
    train(model, args.steps, report=max(1, args.steps // 10))
    gen = torch.Generator().manual_seed(99)
    whole = periodic(model.vocab, 8, 96, gen)
    cuts = [int(torch.randint(24, 64, (1,), generator=gen)) for _ in range(8)]
    got = generate(model, [row[:c] for row, c in zip(whole, cuts)], 32)
    right = sum((g == row[c:c + 32]).float().mean().item() for g, row, c in zip(got, whole, cuts)) / 8
    print("continued 8 prompts of %d to %d tokens by 32: %.0f %% right" % (min(cuts), max(cuts), 100 * right))


if __name__ == "__main__":
    main()
