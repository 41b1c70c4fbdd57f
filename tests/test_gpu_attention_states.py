"""States that leave linear attention, and their gradients, are fp32 in full beside inputs of
16 bits too: a single key (or query) whose weight is all of an entry, which two bf16 parts
of that weight would miss."""
import pytest
import torch

import seq_ref as ref
from gpu_util import DEV
from paper_2301_09266_amd import finc

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UNIT = 2.0 ** -24
# What stands between an entry and its value, in units of 2^-24 of it: the exponent's rounding
# (below 4: 1.4) and exp2's ulp (2), the product with v (1), the parts' sums (1 each of three,
# cut off rather than rounded at most: 2), and where the state passes to the next part that
# part's decay (3.4) and a multiply-add (1).  In fp16 the second part is off by half a unit.
BAR = 20 * UNIT


def inputs(L, H, D, kind, at):
    """One position's k and v (or q and dy), and decays whose sum is 0.2 to 2.5."""
    r = torch.Generator().manual_seed(L + D)
    one, rows = torch.zeros(1, L, H, D), torch.zeros(1, L, H, D)
    one[:, at, :, 3] = 1.0
    rows[:, at] = torch.randn(1, H, D, generator=r)
    decay = -(0.2 + 2.3 * torch.rand(H, generator=r)) / max(L - 1, 1)
    return one.to(kind), rows.to(kind), decay


def weighted(rows, decay, at, steps):
    return torch.exp(decay.double() * steps)[:, None] * rows[0, at].double()


def off(got, want):
    return float(((got.double().cpu() - want).abs() / want.abs())[want != 0].max())


CASES = [(2, 16), (40, 64), (200, 128), (600, 64), (600, 20), (600, 128), (1100, 100)]
# where the key lies: in the last block of a part, or the query in the first one of the second
KEY = {2: 0, 40: 1, 200: 195, 600: 500, 1100: 1010}
QUERY = {2: 1, 40: 30, 200: 20, 600: 270, 1100: 520}


@pytest.mark.parametrize("L,D", CASES)
def test_two_parts_would_be_seen(L, D):
    """The same entries from weights of two bf16 parts, or of one and a half in fp16."""
    for at, steps in ((KEY[L], L - 1 - KEY[L]), (QUERY[L], QUERY[L] + 1)):
        _, rows, decay = inputs(L, 48, D, BF16, at)
        want = weighted(rows, decay, at, steps)
        w = want.float()
        hi = w.bfloat16().float()
        assert off(hi + (w - hi).bfloat16().float(), want) > 2 * BAR
        three = hi + (w - hi).bfloat16().float()
        assert off(three + (w - three).bfloat16().float(), want) < BAR / 8


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("L,D", CASES)
def test_the_state_after_a_row(L, D, kind):
    H, at = 48, KEY[L]
    k, v, decay = inputs(L, H, D, kind, at)
    end = torch.empty(1, H, D, D, device=DEV)
    for states in (None, finc.linear_attention_states(1, L, H, D, D, DEV)):
        finc.linear_attention_forward(k.to(DEV), k.to(DEV), v.to(DEV), decay=decay.to(DEV),
                                      states=states, state_out=end)
        want = weighted(v, decay, at, L - 1 - at)
        assert off(end[0, :, 3], want) <= BAR
        rest = end.clone()
        rest[:, :, 3] = 0
        assert not rest.any()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("L,D", CASES)
def test_the_gradient_of_the_state_before_a_row(L, D, kind):
    H, at = 48, QUERY[L]
    q, dy, decay = inputs(L, H, D, kind, at)
    states = finc.linear_attention_states(1, L, H, D, D, DEV)
    x = [t.to(DEV) for t in (q, torch.zeros_like(q), torch.zeros_like(dy))]
    finc.linear_attention_forward(*x, decay=decay.to(DEV), states=states)
    o = finc.linear_attention_backward(*x, dy.to(DEV), states, decay=decay.to(DEV))
    want = weighted(dy, decay, at, at + 1)
    assert off(o["dstate"][0, :, 3], want) <= BAR
    o["dstate"][:, :, 3] = 0
    assert not o["dstate"].any()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("L", [64, 512, 700])
def test_states_of_whole_rows(L, kind):
    """Sums of many positions, to a bar of fp32 alone: some hundred roundings in order, as
    rows_ref has it (96 units), and in fp16 half a unit of a column's largest of ten times a
    term's size or less (10, as bounds of a result's size)."""
    r = torch.Generator().manual_seed(L)
    n = lambda *s: torch.randn(*s, generator=r)  # noqa: E731
    H, D = 2, 64
    q, k, v, dy = (n(1, L, H, D).to(kind) for _ in range(4))
    state, dend = n(1, H, D, D), n(1, H, D, D)
    decay = torch.tensor([-0.01, -0.3])
    kw = dict(decay=decay.to(DEV), scale=0.25)
    end = torch.empty(1, H, D, D, device=DEV)
    states = finc.linear_attention_states(1, L, H, D, D, DEV)
    x = [t.to(DEV) for t in (q, k, v)]
    finc.linear_attention_forward(*x, state=state.to(DEV), state_out=end, states=states, **kw)
    o = finc.linear_attention_backward(*x, dy.to(DEV), states, dstate_out=dend.to(DEV), **kw)
    t = torch.arange(L, dtype=torch.float64)
    after, before = (torch.exp(decay.double()[:, None] * s) for s in (L - 1 - t, t + 1))
    heads = lambda u: u[0].double().transpose(0, 1)   # noqa: E731  (H, L, D)
    whole = torch.exp(decay.double() * L)[:, None, None]
    want = (heads(k) * after[..., None]).transpose(1, 2) @ heads(v) + whole * state[0].double()
    ref.close(end[0], want, "end", 106)
    want = 0.25 * (heads(q) * before[..., None]).transpose(1, 2) @ heads(dy) + whole * dend[0].double()
    ref.close(o["dstate"][0], want, "dstate", 106)
