"""The operators together, in the example's model: prefill, single tokens, gradients."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_model.py")
_spec = importlib.util.spec_from_file_location("hybrid_model", _path)
hybrid = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(hybrid)
# a pass of the mixing layer keeps 1e-4 (fp32) and 2e-2 (bf16) of the largest value; two
# blocks, their norms and three projections behind them: ten times that
CLOSE = {torch.float32: 1e-3, torch.bfloat16: 2e-1}


def close(a, b, dtype):
    return (a - b).abs().max().item() <= CLOSE[dtype] * b.abs().max().item()


def model(device, dtype):
    return hybrid.Model(vocab=48, width=72, heads=2, head=64, channels=104, states=16, dtype=dtype, device=device)


@pytest.mark.parametrize("dtype", list(CLOSE))
def test_serving(device, dtype):
    """Packed prompts, then a token of each at a time: the logits of each whole sequence."""
    m = model(device, dtype)
    g = torch.Generator().manual_seed(0)
    lengths, more = [1, 37, 2, 130, 64], 6
    rows = [torch.randint(m.vocab, (n + more,), generator=g).to(device) for n in lengths]
    cu = torch.tensor([0] + lengths).cumsum(0).to(device, torch.int32)
    logits, state = m.forward(torch.cat([r[:n] for r, n in zip(rows, lengths)]), cu_seqlens=cu)
    whole = [m.forward(r[None])[0][0] for r in rows]
    for i, n in enumerate(lengths):
        assert close(logits[cu[i]:cu[i + 1]], whole[i][:n], dtype), i
    for t in range(more):
        step = m.decode(torch.stack([r[n + t] for r, n in zip(rows, lengths)]), state)
        assert close(step, torch.stack([w[n + t] for w, n in zip(whole, lengths)]), dtype), t


def test_continued_prefill(device):
    """A prompt in two calls, the second onto the first one's state."""
    m = model(device, torch.float32)
    tokens = torch.randint(m.vocab, (2, 200), generator=torch.Generator().manual_seed(1)).to(device)
    whole, end = m.forward(tokens)
    first, state = m.forward(tokens[:, :90].contiguous())
    second, state = m.forward(tokens[:, 90:].contiguous(), state=state)
    assert close(torch.cat([first, second], 1), whole, torch.float32)
    assert set(state) == set(end) and all(close(state[n], end[n], torch.float32) for n in end)


@pytest.mark.parametrize("packed", [False, True])
def test_gradients(device, packed):
    """The loss along each parameter's own gradient, by differences."""
    m = model(device, torch.float32)
    g = torch.Generator().manual_seed(2)
    shape = (150,) if packed else (2, 75)
    tokens, targets = (torch.randint(m.vocab, shape, generator=g).to(device) for _ in range(2))
    cu = torch.tensor([0, 20, 20, 21, 150], dtype=torch.int32, device=device) if packed else None
    logits, _, saved = m.forward(tokens, cu_seqlens=cu, save=True)
    grads = m.gradients(m.loss(logits, targets)[1], saved)
    assert set(grads) == set(m.p)

    def loss():
        return m.loss(m.forward(tokens, cu_seqlens=cu)[0].double(), targets)[0].item()

    for n, grad in grads.items():
        assert grad.shape == m.p[n].shape and torch.isfinite(grad).all(), n
        size = grad.double().norm().item()
        assert size > 0, n
        # a step that changes the loss by about 0.02: far above its fp32 rounding (1e-5), and
        # small against the loss (4), so that the next term is a few percent at most
        e = min(0.01 / size, 0.02 * m.p[n].norm().item() or 1.0)   # (a bias may be zero)
        base, d = m.p[n].clone(), grad / size
        m.p[n].copy_(base + e * d)
        up = loss()
        m.p[n].copy_(base - e * d)
        down = loss()
        m.p[n].copy_(base)
        assert abs((up - down) / (2 * e) - size) <= 0.05 * size + 2e-5 / e, n


def test_training(device):
    """bf16: the loss of periodic sequences falls."""
    m = hybrid.Model(device=device)
    losses = hybrid.train(m, 240)
    assert all(torch.isfinite(torch.tensor(losses)))
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0]


def test_slices_of_a_batch(device):
    """Tokens and targets as a training loop has them, slices of one batch: the same as their copies."""
    m = model(device, torch.float32)
    data = torch.randint(m.vocab, (3, 41), generator=torch.Generator().manual_seed(4)).to(device)
    tokens, targets = data[:, :-1], data[:, 1:]
    logits, state, saved = m.forward(tokens, save=True)
    want, same, kept = m.forward(tokens.contiguous(), save=True)
    assert torch.equal(logits, want)
    loss, grad = m.loss(logits, targets)
    assert torch.equal(loss, m.loss(logits, targets.contiguous())[0])
    apart = m.loss(logits.transpose(0, 1), targets.t())[1]
    assert torch.equal(apart.transpose(0, 1), grad)
    got, twin = m.gradients(grad, saved), m.gradients(grad, kept)
    assert all(torch.equal(got[n], twin[n]) for n in got)
    assert torch.equal(m.decode(data[:, 40], state), m.decode(data[:, 40].contiguous(), same))
