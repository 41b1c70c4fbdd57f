"""The example's raster prior: the sequence operators together, trained over whole
rasters and run one position at a time."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "raster_prior", os.path.join(ROOT, "examples", "raster_prior.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_likelihood_rises(example):
    z = example.flow_latents(64)
    losses = example.train(example.Prior(z.shape[2]), z, steps=40, batch=32)
    again = example.train(example.Prior(z.shape[2]), z, steps=3, batch=32)
    assert losses[-1] < losses[0] - 0.3, losses
    assert losses[:3] == again, "the same bits from run to run"


def test_single_positions_follow_the_raster(example):
    z = example.flow_latents(8)
    prior = example.Prior(z.shape[2], seed=3)
    with torch.no_grad():
        prior.head.normal_()
        mean, logsd = prior.forward(z)
    # eight rasters in the entries of a larger cache, one more row idle
    slots = torch.tensor([5, 0, 9, 3, 7, 1, 11, 2, -1], dtype=torch.int32, device=z.device)
    cache = prior.start(12)
    size = float(mean.abs().max())
    for t in range(z.shape[1]):
        before = torch.zeros(9, z.shape[2], device=z.device)
        if t:
            before[:8] = z[:, t - 1]
        m, s = prior.step(before, cache, slots)
        # fp32 through two blocks: some hundred roundings of values of this size
        assert float((m[:8] - mean[:, t]).abs().max()) <= 1e-4 * size
        assert float((s[:8] - logsd[:, t]).abs().max()) <= 1e-4 * size
    for taps, state in cache:
        used = slots[:8].long()
        idle = [i for i in range(12) if i not in used.tolist()]
        assert not taps[idle].any() and not state[idle].any()


def test_eight_bits_before_the_head(example):
    z = example.flow_latents(4)
    prior = example.Prior(z.shape[2], seed=4)
    with torch.no_grad():
        prior.head.normal_(0, prior.D ** -0.5)
    full, _ = prior.step(z[:, 0], prior.start(4))
    small, _ = prior.step(z[:, 0], prior.start(4), eight_bits=True)
    # e4m3 rounds by at most 1/16, at random over 64 terms of a product
    assert 0 < float((small - full).abs().max()) <= 0.25
    assert torch.isfinite(prior.sample(3, 20)).all()
