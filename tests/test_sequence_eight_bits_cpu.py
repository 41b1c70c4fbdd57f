"""That the inputs beside the middles of two 8-bit values tell the norm's fp64 from fp32:
the form in fp32 throughout, computed here, takes other values of them."""
import pytest
import torch

import seq_ref as ref
from test_gpu_sequence import BF16, F32, Rand, d64
from test_gpu_sequence_edges import beside_the_middles, codes


@pytest.mark.parametrize("D", [7, 128, 1000, 4096])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_an_fp32_norm_takes_other_values(D, kind):
    x, res, w = beside_the_middles(40000 // D + 2, D, kind, Rand(D))
    want, _ = codes(ref.norm(d64(x) if res is None else d64(x) + d64(res), d64(w), 1e-5))
    s = x.float() if res is None else x.float() + res
    y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-5) * w
    got = (y / (y.abs().amax(1, keepdim=True) / 448)).to(torch.float8_e4m3fn)
    other = (got.view(torch.uint8) != want.view(torch.uint8)).sum()
    assert other > 0.01 * want.numel(), f"{other} of {want.numel()}"
