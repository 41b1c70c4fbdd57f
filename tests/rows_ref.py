"""Plain 64-bit references of linear attention, projections and embeddings, on the CPU:
position after position, differentiable by autograd; and the bars that outputs are held
to beside seq_ref.close."""
import math

import torch

import seq_ref as ref

# A 16-bit input's product with an fp32 value takes 2^-17 of the value (128 units of
# 2^-24), or twice that where both are split in two; three such values follow each other
# in an output (weights, state, weights of the state).  Errors of a sum's terms add up as
# the terms do, to their share of the result's root mean square, which the worst of some
# 10^5 elements passes six times: 3 x 2 x 128 x 6 / 2 (an error spreads evenly over its
# range: its root mean square is under half of its bound).  fp32 rounds some hundred sums
# in order: 10 x 6 by the same count, and 2 units each of exp2 and its argument.
CHAIN = {torch.float32: 96, torch.bfloat16: 2304, torch.float16: 2304}


def close(got, want, what, kind):
    """An output of a call with activations of `kind`.  What rounds past fp16's largest
    value (65504, the next step of 32 from its middle on) is infinite."""
    if got.dtype == torch.float16:
        want = torch.where(want.abs() >= 65520, want.sign() * math.inf, want)
    ref.close(got, want, what, chain=CHAIN[kind])


def attention(q, k, v, g, decay, scale, state, lengths):
    """(y, state after) of float64 tensors."""
    B, L, H, DV = v.shape
    G, DK = q.shape[2:]
    ends = ref.ends(lengths, B, L)
    ys, after = [], []
    for b, n in enumerate(ends):
        S = torch.zeros(H, DK, DV, dtype=v.dtype) if state is None else state[b]
        rows = []
        for t in range(n):
            a = torch.zeros(H, dtype=v.dtype) if decay is None else decay
            a = a if g is None else a + g[b, t]
            heads = lambda x: x[b, t].repeat_interleave(H // G, dim=0)  # noqa: E731
            S = torch.exp(a)[:, None, None] * S + heads(k)[:, :, None] * v[b, t][:, None, :]
            rows.append(scale * (heads(q)[:, :, None] * S).sum(1))
        rows += [torch.zeros(H, DV, dtype=v.dtype)] * (L - n)
        ys.append(torch.stack(rows) if rows else torch.zeros(0, H, DV, dtype=v.dtype))
        after.append(S)
    if not ends:
        return torch.zeros(0, L, H, DV, dtype=v.dtype), torch.zeros(0, H, DK, DV, dtype=v.dtype)
    return torch.stack(ys), torch.stack(after)


def act(name, p):
    return {None: lambda p: p, "relu": torch.relu, "silu": ref.silu,
            "gelu": lambda p: p * 0.5 * torch.erfc(-p * math.sqrt(0.5))}[name](p)


def embed(ids, table, scale):
    V = table.shape[0]
    rows = [table[i] * scale if 0 <= i < V else torch.zeros_like(table[0])
            for i in ids.flatten().tolist()]
    rows = torch.stack(rows) if rows else table[:0]
    return rows.reshape(*ids.shape, table.shape[1])
