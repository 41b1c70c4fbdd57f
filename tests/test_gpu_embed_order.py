"""The order of the sums of a table's gradient: it follows from the sorted list of codes
alone, in which equal codes keep the order of the list."""
import pytest
import torch

from gpu_util import DEV
from paper_2301_09266_amd import finc

pytestmark = pytest.mark.gpu
D = 16


def rows(M, seed):
    """Sums of these depend on their order: sizes from 1 to 2^24 of either sign."""
    r = torch.Generator().manual_seed(seed)
    return torch.randn(M, D, generator=r) * torch.exp2(24 * torch.rand(M, 1, generator=r))


# M with tiles of 8 and of 32 entries, sorted in one launch and in several; codes before the
# one that is looked at, so that its run begins inside a tile, and its own number
LISTS = [(400, 13, 40), (3000, 101, 900), (9000, 1003, 70), (20000, 37, 5000)]


def listed(M, front, own, seed):
    """Codes 0 (front of them), 1 (own) and 2 in any order."""
    ids = torch.full((M,), 2)
    ids[:front] = 0
    ids[front:front + own] = 1
    return ids[torch.randperm(M, generator=torch.Generator().manual_seed(seed))]


@pytest.mark.parametrize("M,front,own", LISTS)
def test_equal_codes_keep_their_order(M, front, own):
    dy = rows(M, M)
    ids = listed(M, front, own, 1)
    want = finc.embed_backward(ids.to(DEV), dy.to(DEV), 3)
    # the same sorted list, whose codes stand elsewhere among each other
    other = listed(M, front, own, 2)
    moved = torch.empty_like(dy)
    moved[torch.argsort(other, stable=True)] = dy[torch.argsort(ids, stable=True)]
    assert torch.equal(finc.embed_backward(other.to(DEV), moved.to(DEV), 3), want)
    # the list already sorted, of 32-bit codes
    order = torch.argsort(ids, stable=True)
    got = finc.embed_backward(ids[order].to(torch.int32).to(DEV), dy[order].to(DEV), 3)
    assert torch.equal(got, want)
    # these sums do depend on the order: the code's rows the other way round
    at = torch.nonzero(ids == 1)[:, 0]
    turned = dy.clone()
    turned[at] = dy[at.flip(0)]
    got = finc.embed_backward(ids.to(DEV), turned.to(DEV), 3)
    assert not torch.equal(got[1], want[1]) and torch.equal(got[[0, 2]], want[[0, 2]])


@pytest.mark.parametrize("M,front,own", LISTS)
def test_a_run_within_tiles_is_the_sum(M, front, own):
    """In fp32: an addition rounds a running sum, which the terms' sizes bound, by a unit of
    2^-24 at most.  One behind the other stand a tile's 32, those of a share of the tiles (M /
    32 of them in 128 shares) and the shares' 128, and a product with the scale."""
    dy, ids = rows(M, M + 1), listed(M, front, own, 3)
    got = finc.embed_backward(ids.to(DEV), dy.to(DEV), 3, scale=0.5).double().cpu()
    want = torch.zeros(3, D, dtype=torch.float64).index_add_(0, ids, dy.double()) * 0.5
    size = torch.zeros(3, D, dtype=torch.float64).index_add_(0, ids, dy.double().abs()) * 0.5
    assert bool(((got - want).abs() <= (162 + M / 4096) * 2.0 ** -24 * size).all())
