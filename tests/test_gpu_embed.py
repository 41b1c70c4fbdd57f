"""Rows of a table by codes and the table's gradient through the binding, against 64-bit
references: types, padding, runs that pass tiles and blocks, streams and graphs."""
import pytest
import torch

import rows_ref as rows
import seq_ref as ref
from gpu_util import DEV
from paper_2301_09266_amd import finc

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = float("nan")


def normal(seed, *shape, kind=F32):
    r = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=r, dtype=torch.float64).to(kind)


def codes(seed, M, V, how):
    """"any", "few" (half of them one code), "one" (all of them), "order", "padding"."""
    r = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (M,), generator=r)
    if how == "few":
        ids[torch.rand(M, generator=r) < 0.5] = V // 2
    elif how == "one":
        ids[:] = V - 1
    elif how == "order":
        ids = torch.arange(M) % V
    elif how == "padding":
        ids[torch.rand(M, generator=r) < 0.3] = -1
        ids[::7] = V
        ids[::11] = -(1 << 31)
        ids[5::31] = (1 << 31) - 1
    return ids


CASES = [  # M, V, D, type, wide ids, how
    (1, 1, 1, F32, True, "any"), (5, 3, 7, BF16, False, "any"), (33, 2, 8, F16, True, "one"),
    (64, 300, 9, F32, False, "padding"), (31, 40, 64, BF16, True, "order"),
    (1000, 256, 33, BF16, False, "few"), (2048, 17, 16, F32, True, "one"),
    (2049, 70000, 24, F16, False, "padding"), (5000, 255, 512, BF16, True, "few"),
    (5000, 256, 100, F32, True, "any"), (4100, 257, 520, F16, False, "order"),
    (10000, 3, 40, BF16, False, "any"), (7000, 65536, 12, F32, True, "few"),
    (300, 20, 1100, BF16, True, "one"), (0, 5, 16, F32, True, "any"),
    (2500, 65537, 4, BF16, False, "order"),
    # tiles of 32 entries: many codes, and fewer of wide rows
    (9000, 30, 512, BF16, False, "padding"), (17000, 300, 5, F32, True, "few"),
    (20000, 5000, 33, F16, False, "any"), (8300, 2, 530, F32, False, "one"),
]


@pytest.mark.parametrize("M,V,D,kind,wide,how", CASES)
def test_forward_and_gradient(M, V, D, kind, wide, how):
    ids = codes(M, M, V, how) if M else torch.zeros(0, dtype=torch.int64)
    there = (ids if wide else ids.to(torch.int32)).to(DEV)
    for table_kind in {kind, F32}:
        table = normal(V, V, D, kind=table_kind)
        y = finc.embed_forward(there, table.to(DEV), scale=1.7, dtype=kind)
        ok = (ids >= 0) & (ids < V)
        want = torch.zeros(M, D, dtype=torch.float64)
        want[ok] = table.double()[ids[ok]] * 1.7
        ref.close(y, want, "y", 2)
    dy = normal(D, M, D, kind=kind)
    if M:
        dy[~ok] = NAN
    wide_rows = torch.full((M, 2 * D + 1), NAN, dtype=kind, device=DEV)
    wide_rows[:, 1:1 + D] = dy.to(DEV)
    out = torch.full((V, D), NAN, device=DEV)
    d = finc.embed_backward(there, wide_rows[:, 1:1 + D], V, scale=1.7, dtable=out)
    want = torch.zeros(V, D, dtype=torch.float64).index_add_(0, ids[ok], dy[ok].double()) * 1.7
    # fp32 sums of a code's rows: a unit a term in the worst order, of which the runs' tiles
    # leave some 32 + 8 + M / 256 in a row, of errors that go by the sum's size
    ref.close(d, want, "dtable", 64)
    untouched = torch.ones(V, dtype=torch.bool)
    untouched[ids[ok]] = False
    assert not bool(d.cpu()[untouched].any())
    again = finc.embed_backward(there, wide_rows[:, 1:1 + D], V, scale=1.7)
    assert torch.equal(d, again)


def test_sums_keep_the_order_of_equal_codes():
    """1 + 2^-24 ... would depend on the order: the same rows at other places of the list,
    with other codes between them, have the same bits."""
    dy = normal(3, 40, 16)
    ids = torch.zeros(40, dtype=torch.int64)
    one = finc.embed_backward(ids.to(DEV), dy.to(DEV), 2)
    spread, at = normal(4, 400, 16), torch.arange(40) * 10
    spread[at] = dy
    other = torch.ones(400, dtype=torch.int64)
    other[at] = 0
    two = finc.embed_backward(other.to(DEV), spread.to(DEV), 2)
    assert torch.equal(one[0], two[0])


def test_leading_dimensions_and_views():
    ids = torch.tensor([[1, 4, 2], [0, -1, 4]], device=DEV)
    big = normal(1, 5, 20).to(DEV)
    y = finc.embed_forward(ids, big[:, 3:10], scale=2.0)
    assert y.shape == (2, 3, 7) and torch.equal(y[0, 1], 2 * big[4, 3:10])
    assert not y[1, 1].any()
    out = torch.full((2, 3, 9), NAN, device=DEV)
    finc.embed_forward(ids, big[:, 3:10], scale=2.0, out=out[..., 1:8])
    assert torch.equal(out[..., 1:8], y) and bool(out[..., 0].isnan().all())
    d = finc.embed_backward(ids, y, 5)
    assert torch.allclose(d[4], y[0, 1] + y[1, 2]) and not d[3].any()
    # an empty table takes padding alone
    assert not finc.embed_forward(ids, torch.zeros(0, 7, device=DEV)).any()
    assert finc.embed_backward(ids, y, 0).shape == (0, 7)


def test_values_that_are_not_finite_stay_in_their_row():
    dy = normal(5, 100, 8)
    ids = torch.arange(100) % 10
    clean = finc.embed_backward(ids.to(DEV), dy.to(DEV), 10)
    dy[33, 2] = NAN
    bad = finc.embed_backward(ids.to(DEV), dy.to(DEV), 10)
    keep = torch.ones(10, 8, dtype=torch.bool)
    keep[3, 2] = False
    assert torch.equal(clean.cpu()[keep], bad.cpu()[keep]) and bool(bad[3, 2].isnan())


def test_graphs_replay_the_calls_and_streams_keep_them():
    M, V, D = 9000, 700, 40
    ids, table = codes(1, M, V, "few").to(DEV), normal(2, V, D, kind=BF16).to(DEV)
    dy = normal(3, M, D, kind=BF16).to(DEV)

    def call():
        return [finc.embed_forward(ids, table, scale=3.0), finc.embed_backward(ids, dy, V),
                finc.embed_backward(ids[:100], dy[:100], V)]

    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for i in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), f"replay {i}"
        assert all(torch.equal(a, b) for a, b in zip(want, call())), "eager work between replays"
    # new codes in the same place
    ids.copy_(codes(9, M, V, "any").to(DEV))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[1], finc.embed_backward(ids, dy, V))


def test_offsets_past_31_bits():
    V, D = 70000, 1 << 15
    table = torch.zeros(V, D, dtype=BF16, device=DEV)
    table[V - 1] = 3
    ids = torch.tensor([V - 1, 0], device=DEV)
    y = finc.embed_forward(ids, table)
    assert bool((y[0] == 3).all()) and not y[1].any()
    del table
    d = finc.embed_backward(ids, y, V)
    assert bool((d[V - 1] == 3).all()) and not d[:V - 1].any()


def test_the_binding_refuses():
    ids, table = torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(5, 8, device=DEV)
    dy = torch.zeros(4, 8, device=DEV)
    for f, what in [
            (lambda: finc.embed_forward(ids.float(), table), "int32 or int64"),
            (lambda: finc.embed_forward(ids.cpu(), table), "device tensor"),
            (lambda: finc.embed_forward(ids, table[0]), "expected \\(V, D\\)"),
            (lambda: finc.embed_forward(ids, table.T), "contiguous"),
            (lambda: finc.embed_forward(ids, table.bfloat16(), dtype=F32), "table must be"),
            (lambda: finc.embed_forward(ids, table.double()), "table must be"),
            (lambda: finc.embed_forward(ids, table, out=dy[:2]), "out has shape"),
            (lambda: finc.embed_forward(ids[::2], table), "contiguous"),
            (lambda: finc.embed_backward(ids, dy[:2], 5), "dy has shape"),
            (lambda: finc.embed_backward(ids, dy.double(), 5), "must be float32"),
            (lambda: finc.embed_backward(ids, dy, 5, dtable=table.bfloat16()), "dtable must be"),
            (lambda: finc.embed_backward(ids, dy, 6, dtable=table), "dtable has shape")]:
        with pytest.raises(ValueError, match=what):
            f()
    with pytest.raises(finc.FincError):
        finc.embed_forward(ids, table, out=table[:4])
    with pytest.raises(finc.FincError):
        finc.embed_backward(ids, table[:4], 5, dtable=table)
