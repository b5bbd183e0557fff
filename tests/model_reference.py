"""The operators at a language model's ends and the gated linear recurrence, written
from their definitions in 64 bits on the CPU (gradients: torch autograd)."""
import torch

from tests.layer_reference import silu


def embed(ids, table, scale):
    known = (ids >= 0) & (ids < table.shape[0])
    rows = [scale * table[i] if k else torch.zeros_like(table[0]) for i, k in zip(ids.tolist(), known.tolist())]
    return torch.stack(rows) if rows else table[:0]


def logprob(logits, targets, scale, top=0):
    """dict of the forward's outputs for logits [n, V] in 64 bits, row by row."""
    out = {"logprob": [], "lse": [], "entropy": [], "top_logprobs": [], "top_ids": []}
    for row, y in zip(logits * scale, targets.tolist()):
        there = [j for j, v in enumerate(row.tolist()) if v > float("-inf")]
        z = row[there]
        if there:
            ln = torch.log(torch.exp(z - z.max()).sum())
            lse, lp = z.max() + ln, z - z.max() - ln   # (z - lse would lose ln beside a far maximum)
            entropy = -(torch.exp(lp) * lp).sum()
        else:
            lse, lp, entropy = row.new_full((), float("-inf")), z, row.new_zeros(())
        full = torch.full_like(row, float("-inf"))
        full[there] = lp
        out["lse"].append(lse)
        out["entropy"].append(entropy)
        out["logprob"].append(full[y] if 0 <= y < len(row) else row.new_zeros(()))
        order = sorted(there, key=lambda j: (-row[j].item(), j))[:top]
        pad = top - len(order)
        out["top_ids"].append(torch.tensor(order + [-1] * pad, dtype=torch.int32))
        out["top_logprobs"].append(torch.cat([full[order], full.new_full((pad,), float("-inf"))]))
    return {n: torch.stack(t) if t else torch.zeros(0, *([top] if "top" in n else [])) for n, t in out.items()}


def glr(x, r, A, i, z, normalize, h0, spans):
    """(o, final states) for token rows [tokens, D]."""
    log_a = A / (1 + torch.exp(-r))
    a = torch.exp(log_a)
    b = x if i is None else x / (1 + torch.exp(-i))
    if normalize:
        b = b * torch.sqrt(-torch.expm1(2 * log_a))
    rows, final = {}, []
    for n, (first, end) in enumerate(spans):
        h = torch.zeros_like(A) if h0 is None else h0[n]
        for t in range(first, end):
            h = a[t] * h + b[t]
            rows[t] = h if z is None else h * silu(z[t])
        final.append(h)
    zero = torch.zeros_like(A)
    o = torch.stack([rows.get(t, zero) for t in range(x.shape[0])]) if x.shape[0] else x.clone()
    return o, torch.stack(final) if final else A.new_zeros(0, A.shape[0])
