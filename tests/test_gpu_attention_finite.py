"""Where an input of linear attention that is not finite is felt: y, the last state and dq
from its block on, dk, dv and the first state's gradient up to its block's end, dg anywhere,
all in its row and heads alone."""
import pytest
import torch

from gpu_util import DEV
from paper_2301_09266_amd import finc

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
BLOCK = 64


@pytest.mark.parametrize("L,at", [(200, 70), (640, 300), (640, 511)])
@pytest.mark.parametrize("what", [NAN, INF])
@pytest.mark.parametrize("name", ["q", "k", "v", "g", "dy"])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
def test_what_is_not_finite_reaches(L, at, what, name, kind):
    r = torch.Generator().manual_seed(L)
    n = lambda *s: torch.randn(*s, generator=r).to(kind)  # noqa: E731
    B, H, D = 2, 2, 16
    t = dict(q=n(B, L, H, D), k=n(B, L, H, D), v=n(B, L, H, D), dy=n(B, L, H, D),
             g=-0.05 * n(B, L, H).exp())

    def run():
        d = {m: x.to(DEV) for m, x in t.items()}
        states = finc.linear_attention_states(B, L, H, D, D, DEV)
        end = torch.empty(B, H, D, D, device=DEV)
        y = finc.linear_attention_forward(d["q"], d["k"], d["v"], g=d["g"], scale=0.3,
                                          states=states, state_out=end)
        o = finc.linear_attention_backward(d["q"], d["k"], d["v"], d["dy"], states, g=d["g"],
                                           scale=0.3)
        return dict(o, y=y, end=end)

    clean = run()
    t[name][1, at, 1] = what
    bad = run()
    first, past = at // BLOCK * BLOCK, at // BLOCK * BLOCK + BLOCK
    for m, x in bad.items():
        # other rows and heads keep their bits
        assert torch.equal(x[0], clean[m][0]), m
        if m in ("end", "dstate"):
            assert torch.equal(x[1, 0], clean[m][1, 0]), m
        else:
            assert torch.equal(x[1, :, 0], clean[m][1, :, 0]), m
        fine = {"y": slice(0, first), "dq": slice(0, first), "dk": slice(past, L),
                "dv": slice(past, L)}.get(m)
        if fine is not None:
            assert bool(torch.isfinite(x[1, fine, 1]).all()), m
    # and it does reach what its values are summed into
    felt = {"q": ("y", "dk", "dstate"), "k": ("y", "end", "dq", "dv"), "v": ("y", "end", "dq"),
            "dy": ("dk", "dv", "dstate")}.get(name, ())
    for m in felt:
        x = bad[m][1, 1] if m in ("end", "dstate") else bad[m][1, :, 1]
        assert not bool(torch.isfinite(x).all()), m
    # as far as its block's sums go, on to the row's end and back to its start
    if name == "v":
        assert not bool(torch.isfinite(bad["dq"][1, -1, 1]).any())
    if name == "dy":
        assert not bool(torch.isfinite(bad["dv"][1, 0, 1]).any())
