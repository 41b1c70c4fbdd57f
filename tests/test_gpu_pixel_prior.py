"""The pixel prior of examples/pixel_prior.py: its gradients against a plain one in 64 bits,
whole rasters against single positions, a captured step, and that it trains."""
import math
import os
import sys

import pytest
import torch

import rows_ref as rows
import seq_ref as ref
from gpu_util import DEV

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
import pixel_prior as ex  # noqa: E402

pytestmark = pytest.mark.gpu


def plain(prior, codes):
    """(loss, gradients) of the model in 64 bits on the CPU."""
    def leaf(t):
        return t.detach().double().cpu().requires_grad_()

    top = [leaf(t) for t in (prior.codes, prior.places, prior.norm, prior.head_w)]
    blocks = [{n: leaf(t) for n, t in b.items()} for b in prior.blocks]
    B, L = codes.shape
    ids = codes.cpu()
    before = torch.cat([torch.full((B, 1), prior.V), ids[:, :-1]], 1)
    s = math.sqrt(prior.D)
    x = rows.embed(before, top[0], s) + rows.embed(torch.arange(L).expand(B, L), top[1], s)
    for b in blocks:
        mixed = ref.norm(x, b["norm"], ex.EPS) @ b["w_in"].T
        q, k, v, g = prior.split(mixed)
        y, _ = rows.attention(q, k, v, g, prior.decay.double().cpu(), prior.E ** -0.5, None, None)
        x = x + y.flatten(2) @ b["w_out"].T
        y = rows.act("silu", ref.norm(x, b["norm2"], ex.EPS) @ b["w_up"].T + b["b_up"])
        x = x + y @ b["w_down"].T
    logits = ref.norm(x, top[2], ex.EPS) @ top[3].T
    loss = torch.nn.functional.cross_entropy(logits.flatten(0, 1), ids.flatten()) / math.log(2)
    leaves = top + [t for b in blocks for t in b.values()]
    return logits.detach(), loss.detach(), torch.autograd.grad(loss, leaves)


# What a rounding to the type between the operators adds: some thirty of them on a path, each
# half a step, as independent errors of the values' size, three times their root mean square;
# gradients go through them twice.
BAR = {t: 3 * math.sqrt(30) * ref.U[t] for t in (torch.float32, torch.bfloat16)}


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_gradients_are_the_plain_models(kind):
    codes = ex.pixels(3, side=9, levels=20)
    prior = ex.Prior(20, 81, width=32, heads=2, head=12, dtype=kind, seed=1)
    logits, loss, want = plain(prior, codes)
    got = prior.forward(codes).detach()
    mine = prior.bits(codes)
    mine.backward()
    off = (got.double().cpu() - logits).square().mean().sqrt() / logits.square().mean().sqrt()
    assert float(off) <= BAR[kind]
    assert abs(float(mine.detach()) - float(loss)) <= BAR[kind] * float(loss)
    for p, w in zip(prior.parameters(), want):
        g = p.grad.double().cpu()
        assert g.shape == w.shape
        err = (g - w).square().sum().sqrt()
        assert float(err) <= 2 * BAR[kind] * float(w.square().sum().sqrt())


def test_positions_one_by_one_are_the_raster():
    codes = ex.pixels(4, side=8, levels=16)
    prior = ex.Prior(16, 64, seed=2)
    with torch.no_grad():
        want = prior.forward(codes)
    cache = prior.start(6)
    slots = torch.tensor([5, 0, 3, 2], dtype=torch.int32, device=DEV)
    for t in range(64):
        before = codes[:, t - 1].contiguous() if t else torch.full((4,), 16, device=DEV)
        got = prior.step(before, t, cache, slots)
        off = (got - want[:, t]).square().mean().sqrt() / want.square().mean().sqrt()
        assert float(off) <= BAR[torch.float32], t
    assert not cache[0][[1, 4]].any()
    out = prior.sample(3)
    assert out.shape == (3, 64) and int(out.min()) >= 0 and int(out.max()) < 16


def test_a_captured_position_replays():
    """A step of the sampler in a graph: codes and states change in place between replays."""
    codes = ex.pixels(2, side=8, levels=16)
    prior = ex.Prior(16, 64, seed=3)
    before = codes[:, 0].contiguous()
    eager, cache = prior.start(2), prior.start(2)
    prior.step(before, 1, prior.start(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = prior.step(before, 1, cache)
    for s in cache:
        s.zero_()
    for t in range(1, 5):
        before.copy_(codes[:, t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, prior.step(codes[:, t].contiguous(), 1, eager)), t
        assert all(torch.equal(a, b) for a, b in zip(cache, eager))


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_it_trains(kind):
    codes = ex.pixels(16, side=8, levels=16)
    losses = ex.train(ex.Prior(16, 64, dtype=kind), codes, steps=6, batch=8)
    assert all(math.isfinite(v) for v in losses)
