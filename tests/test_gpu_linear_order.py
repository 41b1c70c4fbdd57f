"""A projection's sums have an order that follows from the sizes alone: the same bits
whatever the addresses of its operands and the steps between their rows."""
import pytest
import torch

from gpu_util import DEV
from paper_2301_09266_amd import finc

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = float("nan")


def normal(seed, *shape, kind=F32, scale=1.0):
    r = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=r) * scale).to(kind).to(DEV)


def beside(t, front, more):
    """The same values `front` elements into rows of `more` further ones."""
    if t is None:
        return None
    big = torch.full((t.shape[0], t.shape[1] + more), NAN, dtype=t.dtype, device=DEV)
    big[:, front:front + t.shape[1]] = t
    return big[:, front:front + t.shape[1]]


# Few rows, sums in one part and in several, tiles of each size, with edges; rows that are
# whole chunks of 16 bytes and rows that are not.
SIZES = [(1, 2048, 512, BF16), (1, 4096, 1000, F32), (20, 1024, 304, F16), (32, 512, 96, F32),
         (64, 2048, 2048, BF16), (64, 2048, 64, F16), (256, 4096, 256, BF16), (100, 4096, 64, F32),
         (300, 1000, 72, F32), (1531, 336, 1000, F32), (5000, 256, 2056, BF16), (4096, 64, 128, F16),
         (65, 1001, 130, BF16), (700, 333, 250, F32)]
# offset and extra elements of x, w, dy and pre
PLACES = [((1, 5), (0, 0), (0, 0)), ((0, 0), (1, 5), (3, 8)), ((1, 8), (3, 7), (1, 1)), ((8, 8), (8, 16), (16, 24))]


@pytest.mark.parametrize("M,K,N,kind", SIZES)
def test_bits_do_not_depend_on_the_place(M, K, N, kind):
    x, w = normal(1, M, K, kind=kind), normal(2, N, K, kind=kind, scale=K ** -0.5)
    b, r = normal(3, N), normal(4, M, N, kind=kind)
    dy, pre = normal(5, M, N, kind=kind), normal(6, M, N, kind=kind)

    def run(px, pw, pn):
        u, v = beside(x, *px), beside(w, *pw)
        y = [finc.linear_forward(u, v)]
        for act in ("silu", "gelu"):
            kept = torch.empty_like(r)
            y.append(finc.linear_forward(u, v, b, act=act, residual=beside(r, *pn), pre_out=kept))
            y.append(kept)
        return [*y, *finc.linear_backward(beside(dy, *pn), u, v),
                *finc.linear_backward(beside(dy, *pn), u, v, beside(pre, *pn), act="silu")]

    want = run((0, 0), (0, 0), (0, 0))
    for p in PLACES:
        for i, (a, c) in enumerate(zip(run(*p), want)):
            assert torch.equal(a, c), (p, i)
