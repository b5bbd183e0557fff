"""The operators around a mixing layer with more values than a launch holds threads
(2^32)."""
import pytest
import torch

import paper_2509_25223_amd as rla
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


def test_scan_gradients(device):
    """dB and dC of 2^25 tokens of 64 states: 2^32 values and more, all written, those of
    the last sequences right."""
    B, T, N = (1 << 19) + 3, 64, 64
    g = torch.Generator(device).manual_seed(0)
    rnd = lambda *s, dt=torch.bfloat16: torch.randn(*s, dtype=dt, device=device, generator=g)   # noqa: E731
    u, delta, dO, Bm, C = rnd(B, T, 1), rnd(B, T, 1), rnd(B, T, 1), rnd(B, T, N), rnd(B, T, N)
    A = -4 * torch.rand(1, N, device=device, generator=g)
    like = dict(du=u, ddelta=delta, dA=A, dB=Bm, dC=C)
    grads = {n: torch.full_like(t, float("nan")) for n, t in like.items()}
    rla.rla_ssm_backward(u, delta, A, Bm, C, dO, grads=grads)
    torch.cuda.synchronize()
    for n, t in grads.items():
        assert not torch.isnan(t).any(), n
    last = 3
    v = {n: ref.wide(t[-last:]) for n, t in dict(u=u, delta=delta, B=Bm, C=C).items()}
    rows = {n: t.reshape(last * T, -1) for n, t in v.items()}
    o, _ = ref.ssm(rows["u"], rows["delta"], ref.wide(A, False), rows["B"][:, None], rows["C"][:, None], None, None, None,
                   True, None, [(i * T, (i + 1) * T) for i in range(last)])
    want = ref.gradients([o], [dO[-last:].cpu().double().reshape(last * T, 1)], v)
    for n in ("u", "delta", "B", "C"):
        ref.check("d" + n, grads["d" + n][-last:], want[n], 8 * N + T)


def test_addnorm(device):
    """Rows of two values, a wave each: more of them than one launch takes."""
    rows, D = (1 << 26) + 77, 2
    g = torch.Generator(device).manual_seed(1)
    x = torch.randn(rows, D, dtype=torch.bfloat16, device=device, generator=g)
    res = torch.randn(rows, D, device=device, generator=g)
    weight, scale = torch.tensor([0.9, 1.3], device=device), torch.tensor([0.5, -2.0], device=device)
    n, r = torch.full_like(x, float("nan")), torch.full_like(res, float("nan"))
    rla.rla_addnorm_forward(x, weight, residual=res, scale=scale, out=n, residual_out=r)
    for at in range(0, rows, 1 << 24):   # (all of them, some at a time)
        part = slice(at, at + (1 << 24))
        want_n, want_r = ref.addnorm(x[part].double(), res[part].double(), weight.double(), scale.double())
        ref.check("n", n[part], want_n.cpu(), 4)
        ref.check("residual", r[part], want_r.cpu())
    same = res.clone()
    n2, _ = rla.rla_addnorm_forward(x, weight, residual=same, scale=scale, residual_out=same)
    assert torch.equal(n, n2) and torch.equal(r, same)


@pytest.mark.parametrize("first", [False, True])
def test_gatenorm(device, first):
    """Heads of one value, 8 lanes each: more of them than one launch takes."""
    T, H = (1 << 29) // 3 + 50, 3
    g = torch.Generator(device).manual_seed(2)
    x = torch.randn(T, H, 1, dtype=torch.bfloat16, device=device, generator=g)
    gate = torch.randn(T, H, 1, dtype=torch.bfloat16, device=device, generator=g)
    weight = torch.tensor([[0.9], [1.3], [-2.0]], device=device)
    o = torch.full_like(x, float("nan"))
    rla.rla_gatenorm_forward(x, gate, weight, gate_first=first, out=o)
    for part in (slice(0, 1 << 20), slice(T // 2, T // 2 + 10007), slice(T - (1 << 20), T)):
        want = ref.gatenorm(x[part].double(), gate[part].double(), weight.double(), first)
        ref.check("o", o[part], want.cpu(), 4)
    assert not torch.isnan(o).any()


def test_gatenorm_weights(device):
    """A gradient of more than 2^28 weights per head, from one token."""
    H, d = 1 << 20, 260
    g = torch.Generator(device).manual_seed(3)
    x, gate, dO = (torch.randn(1, H, d, dtype=torch.bfloat16, device=device, generator=g) for _ in range(3))
    weight = 1 + 0.1 * torch.randn(H, d, device=device, generator=g)
    grads = dict(dx=torch.full_like(x, float("nan")), dgate=torch.full_like(x, float("nan")),
                 dweight=torch.full_like(weight, float("nan")))
    rla.rla_gatenorm_backward(dO, x, gate, weight, grads=grads)
    for part in (slice(0, 2000), slice(H // 2, H // 2 + 2000), slice(H - 30000, H)):
        # the sum over one token: its gradient times the normalised, gated value
        want = dO[0, part].double() * ref.rms(x[0, part].double()) * ref.silu(gate[0, part].double())
        ref.check("dweight", grads["dweight"][part], want.cpu(), 8)
    assert not any(torch.isnan(t).any() for t in grads.values())
