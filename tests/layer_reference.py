"""The operators around a mixing layer, written from their definitions in 64 bits
on the CPU, one sequence and one token at a time (gradients: torch autograd), and
what their GPU tests share."""
import torch

EPS = 1e-6


def silu(x):
    return x / (1 + torch.exp(-x))


def sequences(cu, ntok):
    """[start, end) of each sequence: running maxima of the clamped offsets."""
    m, out = 0, []
    for i, o in enumerate(cu):
        o = min(max(int(o), 0), ntok)
        if i:
            out.append((m, max(m, o)))
        m = max(m, o)
    return out


def conv(x, weight, bias, act, state, spans):
    """(y, final states) for token rows x [tokens, D]."""
    W = weight.shape[1]
    y, final = torch.zeros_like(x), []
    for n, (a, b) in enumerate(spans):
        before = x.new_zeros(W - 1, x.shape[1]) if state is None else state[n]
        rows = torch.cat([before, x[a:b]])
        pre = sum(weight[:, i] * rows[i:i + b - a] for i in range(W))
        if bias is not None:
            pre = pre + bias
        y = torch.cat([y[:a], silu(pre) if act else pre, y[b:]])
        final.append(rows[b - a:])
    return y, torch.stack(final) if final else x.new_zeros(0, W - 1, x.shape[1])


def ssm(u, delta, A, B, C, D, z, bias, softplus, h0, spans):
    """(o, final states) for token rows; B, C [tokens, G, states]."""
    G = B.shape[1]
    raw = delta if bias is None else delta + bias
    step = torch.where(raw > 30, raw, torch.log1p(torch.exp(raw.clamp(max=30)))) if softplus else raw
    rows, final = {}, []
    for n, (a, b) in enumerate(spans):
        h = A.new_zeros(A.shape) if h0 is None else h0[n]
        for t in range(a, b):
            Bt, Ct = (m[t].repeat_interleave(A.shape[0] // G, 0) for m in (B, C))
            h = torch.exp(step[t, :, None] * A) * h + (step[t] * u[t])[:, None] * Bt
            y = (h * Ct).sum(1)
            if D is not None:
                y = y + D * u[t]
            rows[t] = y if z is None else y * silu(z[t])
        final.append(h)
    zero = torch.zeros(A.shape[0], dtype=A.dtype)
    o = torch.stack([rows.get(t, zero) for t in range(u.shape[0])]) if u.shape[0] else u.clone()
    return o, torch.stack(final) if final else A.new_zeros(0, *A.shape)


def rms(y):
    return y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS)


def addnorm(x, residual, weight, scale):
    r = x if scale is None else scale * x
    r = r if residual is None else residual + r
    return rms(r) * weight, r


def gatenorm(x, gate, weight, first):
    return rms(x * silu(gate)) * weight if first else rms(x) * weight * silu(gate)


def wide(t, grad=True):
    """A tensor's values in 64 bits on the CPU, as a leaf."""
    return None if t is None else t.detach().cpu().double().requires_grad_(grad)


def gradients(outputs, upstream, leaves):
    """Gradients of sum <upstream, output> for the named leaves (zeros where unused)."""
    total = sum((o * g).sum() for o, g in zip(outputs, upstream) if g is not None)
    names = [n for n, t in leaves.items() if t is not None]
    got = torch.autograd.grad(total, [leaves[n] for n in names], allow_unused=True)
    return {n: torch.zeros_like(leaves[n]) if g is None else g for n, g in zip(names, got)}


def check(name, got, ref, terms=1):
    """Each value within its type's rounding of the reference, plus the error of fp32
    arithmetic: a value is a sum of `terms` products whose partial sums are of the
    size of the largest values, each step off by 2^-24 of that, with a factor of 8 for
    the functions inside (exponentials and reciprocals of a few ulp)."""
    ref = ref.detach()
    g = got.detach().cpu().double()
    assert g.shape == ref.shape, (name, g.shape, ref.shape)
    if not ref.numel():
        return
    top = ref.abs().max().item()
    allowed = 8 * terms ** 0.5 * 2.0 ** -24 * (top + 1e-30) + (2.0 ** -8 * ref.abs() if got.dtype == torch.bfloat16 else 0)
    over = ((g - ref).abs() - allowed).max().item()
    assert over <= 0 and torch.isfinite(g).all(), "%s: off by %.3e over the bound, largest %.3e" % (name, over, top)


def strided(t, lead):
    """The same values as a slice of wider rows."""
    inner = t.shape[lead:]
    flat = t.reshape(*t.shape[:lead], -1)
    big = torch.full((*t.shape[:lead], flat.shape[-1] + 13), float("nan"), dtype=t.dtype, device=t.device)
    big[..., 5:5 + flat.shape[-1]] = flat
    return big[..., 5:5 + flat.shape[-1]].unflatten(-1, inner) if inner else big


# packed tokens: lengths of one and less than the taps, empty sequences; offsets that
# leave tokens out in front and behind; offsets out of order and out of range
PACKED = {
    "ragged": ([0, 5, 5, 6, 8, 11, 51, 68], 68),
    "gaps": ([3, 3, 40, 41, 44], 60),
    "disorder": ([-4, 20, 10, 25, 99, 30], 70),
    "ones": (list(range(0, 41)), 40),
    "none": ([7], 9),
}
DENSE = {"one token": (1, 1), "ones": (5, 1), "short": (3, 2), "odd": (2, 37), "tiles": (1, 96)}


def layout(name):
    """(leading shape, spans, cu offsets or None)"""
    if name in PACKED:
        cu, ntok = PACKED[name]
        return (ntok,), sequences(cu, ntok), cu
    B, T = DENSE[name]
    return (B, T), [(b * T, (b + 1) * T) for b in range(B)], None


LAYOUTS = list(DENSE) + list(PACKED)
