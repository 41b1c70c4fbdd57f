"""Projections through the binding against 64-bit references: types, odd sizes, views,
activations, residuals in place, long sums in parts, streams and graphs."""
import math

import pytest
import torch

import rows_ref as rows
import seq_ref as ref
from gpu_util import DEV
from paper_2301_09266_amd import finc

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN, INF = float("nan"), float("inf")
# Products of 16 bits are exact in fp32: what is left is the fp32 sums' rounding, a unit a
# term in the worst order, of which some tens add up, and a few of the activation.
CHAIN = 64


def normal(seed, *shape, kind=F32, scale=1.0):
    r = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=r, dtype=torch.float64) * scale).to(kind)


def place(t, wide):
    """On the device; wide: beside NaN in rows of more elements, at an odd address."""
    if t is None or not wide:
        return None if t is None else t.to(DEV)
    big = torch.full((t.shape[0], t.shape[1] + 5), NAN, dtype=t.dtype, device=DEV)
    big[:, 1:1 + t.shape[1]] = t.to(DEV)
    return big[:, 1:1 + t.shape[1]]


def kept_beside(view):
    """Whether what lies beside a view made by `place` is still NaN."""
    base = view._base
    return bool(base[:, 0].isnan().all()) and bool(base[:, 1 + view.shape[1]:].isnan().all())


SIZES = [  # M, K, N, type, wide
    (1, 1, 1, F32, False), (1, 8, 3, BF16, True), (3, 7, 5, F16, True), (2, 31, 33, F32, True),
    (64, 64, 64, BF16, False), (65, 63, 66, BF16, True), (17, 129, 130, F32, False),
    (100, 200, 300, F16, False), (1, 2048, 512, BF16, False), (64, 2048, 512, BF16, False),
    (63, 1031, 70, F32, True), (700, 64, 40, BF16, True), (1531, 333, 250, F32, False),
    (2100, 96, 2050, BF16, False), (2049, 40, 2056, F32, True), (2049, 130, 2055, F16, True),
    (20, 12, 9, F32, False), (5, 20, 64, F32, False), (17, 40, 130, BF16, False),
    (1, 4096, 33, F16, False), (32, 1000, 100, F32, False), (300, 5000, 17, F16, False), (5, 16, 4097, BF16, False), (129, 257, 16, F32, True),
]


@pytest.mark.parametrize("M,K,N,kind,wide", SIZES)
def test_forward(M, K, N, kind, wide):
    for i, (act, bias, res, keep) in enumerate([(None, False, False, False),
                                                ("silu", True, True, True),
                                                ("gelu", True, False, True),
                                                ("relu", False, True, False)]):
        x, w = normal(M, M, K, kind=kind), normal(N + 1, N, K, kind=kind, scale=K ** -0.5)
        b = normal(K, N, scale=0.5) if bias else None
        r = normal(i, M, N, kind=kind) if res else None
        pre = place(torch.full((M, N), NAN, dtype=kind), wide) if keep else None
        out = place(torch.full((M, N), NAN, dtype=kind), wide)
        y = finc.linear_forward(place(x, wide), place(w, wide), None if b is None else b.to(DEV),
                                act=act, residual=place(r, wide), out=out, pre_out=pre)
        p = x.double() @ w.double().T + (0 if b is None else b.double())
        want = rows.act(act, p) + (0 if r is None else r.double())
        ref.close(y, want, f"y {act}", CHAIN)
        if keep:
            ref.close(pre, p, f"pre {act}", CHAIN)
        if wide:
            assert kept_beside(out) and (pre is None or kept_beside(pre))


@pytest.mark.parametrize("M,K,N,kind,wide", SIZES)
@pytest.mark.parametrize("act", [None, "silu", "gelu", "relu"])
def test_gradients(M, K, N, kind, wide, act):
    x, w = normal(M, M, K, kind=kind), normal(N + 1, N, K, kind=kind, scale=K ** -0.5)
    dy, pre = normal(K + 2, M, N, kind=kind), normal(K + 3, M, N, kind=kind) if act else None
    dx, dw, db = finc.linear_backward(place(dy, wide), place(x, wide), place(w, wide),
                                      place(pre, wide), act=act)
    d = dy.double()
    if act:
        p = pre.double().requires_grad_()
        d, = torch.autograd.grad(rows.act(act, p), p, d)
    ref.close(db, d.sum(0), "dbias", CHAIN)
    # d is rounded to the type before the products: half a step of every term, whose errors
    # add up as the terms do; six times their root mean square, which is under 0.6 of the
    # bound, in units of 2^-24
    chain = CHAIN + (0 if act is None else 6 * 0.6 * ref.U[kind] * 2.0 ** 24)
    ref.close(dx, d @ w.double(), "dx", chain)
    ref.close(dw, d.T @ x.double(), "dw", chain)
    without = finc.linear_backward(place(dy, wide), place(x, wide), place(w, wide),
                                   place(pre, wide), act=act, bias=False)
    assert without[2] is None and torch.equal(without[0], dx) and torch.equal(without[1], dw)


@pytest.mark.parametrize("M,K,N,kind", [(5000, 256, 2056, BF16), (4999, 264, 2050, F16),
                                        (8000, 2040, 512, BF16), (512, 2040, 8000, F16),
                                        (2040, 512, 2048, F32), (2048, 2044, 516, F32)])
def test_large_tiles(M, K, N, kind):
    """Products that fill the card with the largest tiles, with edges, in each place."""
    x, w = normal(1, M, K, kind=kind), normal(2, N, K, kind=kind, scale=K ** -0.5)
    b, r, dy = normal(3, N), normal(4, M, N, kind=kind), normal(5, M, N, kind=kind)
    pre = torch.full((M, N), NAN, dtype=kind, device=DEV)
    y = finc.linear_forward(x.to(DEV), w.to(DEV), b.to(DEV), act="silu", residual=r.to(DEV),
                            pre_out=pre)

    # A sum of n terms one after another: the i-th addition rounds a partial sum of sqrt(i / n)
    # of the result's root mean square by up to 2^-24 of it, evenly, 2^-24 / sqrt(3) in the
    # root mean square; all n make sqrt(n / 2) / sqrt(3) of it, which the worst of some 10^6
    # sums passes six times.
    def chain(n):
        return max(CHAIN, 6 * math.sqrt(n / 6))

    p = x.double() @ w.double().T + b.double()
    ref.close(pre, p, "pre", chain(K))
    ref.close(y, rows.act("silu", p) + r.double(), "y", chain(K))
    dx, dw, db = finc.linear_backward(dy.to(DEV), x.to(DEV), w.to(DEV))
    ref.close(dx, dy.double() @ w.double(), "dx", chain(N))
    ref.close(dw, dy.double().T @ x.double(), "dw", chain(M))
    ref.close(db, dy.double().sum(0), "dbias", chain(M))


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", None])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_activations_at_their_ends(act, kind):
    """Infinities, the type's ends, values near 0 and NaN, through w = 1."""
    top = torch.finfo(kind).max
    v = torch.tensor([0.0, -0.0, 1e-5, -1e-5, 1.0, -1.0, 5.0, -5.0, 12.0, -12.0, 60.0, -60.0, top,
                      -top, INF, -INF, NAN], dtype=torch.float64).to(kind)
    one = torch.ones(1, 1, dtype=kind, device=DEV)
    y = finc.linear_forward(v[:, None].to(DEV), one, act=act)[:, 0]
    p = v.double()
    want = {"silu": torch.where(p == -INF, 0.0, ref.silu(p)),
            "gelu": torch.where(p == -INF, 0.0, rows.act("gelu", p)),
            "relu": torch.relu(p), None: p}[act]
    got = y.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].isnan(), want[~fine].isnan())
    assert torch.equal(got[p == INF], want[p == INF])
    assert bool(((got - want)[fine].abs() <= ref.U[kind] * 1.01 * want[fine].abs()
                 + 64 * 2.0 ** -24 * want[fine].abs() + 2.0 ** -25).all())
    if act is None:
        return
    d = finc.linear_backward(torch.ones_like(y)[:, None], v[:, None].to(DEV), one,
                             v[:, None].to(DEV), act=act)[0][:, 0].double().cpu()
    q = p.clamp(-1e4, 1e4).requires_grad_()
    slope, = torch.autograd.grad(rows.act(act, q).sum(), q)
    fine = ~p.isnan()
    assert bool(d[~fine].isnan().all())
    assert bool(((d - slope)[fine].abs() <= ref.U[kind] * 1.01 * slope[fine].abs()
                 + 64 * 2.0 ** -24 * (1 + slope[fine].abs())).all())


def test_residual_in_place_and_leading_dimensions():
    x, w = normal(1, 2, 3, 40, kind=BF16), normal(2, 24, 40, kind=BF16, scale=0.2)
    r = normal(3, 2, 3, 24, kind=BF16)
    here = r.to(DEV)
    y = finc.linear_forward(x.to(DEV), w.to(DEV), residual=here, out=here)
    assert y.data_ptr() == here.data_ptr() and y.shape == (2, 3, 24)
    ref.close(y, x.double() @ w.double().T + r.double(), "y", CHAIN)
    dx, dw, db = finc.linear_backward(r.to(DEV), x.to(DEV), w.to(DEV))
    ref.close(dx, r.double() @ w.double(), "dx", CHAIN)
    ref.close(dw, r.double().flatten(0, 1).T @ x.double().flatten(0, 1), "dw", CHAIN)
    ref.close(db, r.double().sum((0, 1)), "dbias", CHAIN)
    # rows that are one row
    one = x[0, :1].to(DEV).expand(5, 40)
    y = finc.linear_forward(one, w.to(DEV))
    assert torch.equal(y, y[:1].expand(5, 24))


@pytest.mark.parametrize("M,K,N,kind", [(129, 96, 72, BF16), (37, 45, 50, F32), (300, 33, 64, F16),
                                        (1000, 600, 520, F32), (4096, 128, 64, BF16)])
@pytest.mark.parametrize("act", [0, 2])
def test_each_gradient_alone_is_the_same(M, K, N, kind, act):
    """Any of dx, dw and dbias may be absent from the call; the others keep their bits."""
    dy, x, w, pre = (normal(i, *s, kind=kind).to(DEV) for i, s in
                     enumerate(((M, N), (M, K), (N, K), (M, N))))
    full = finc.linear_backward(dy, x, w, pre, act="silu" if act else None)
    lib, code = finc._require_lib(), {F32: 0, BF16: 1, F16: 2}[kind]
    ws = torch.empty(lib.finc_linear_grad_workspace_bytes(code, act, M, K, N) // 4 + 64, device=DEV)
    for keep in ((0,), (1,), (2,), (0, 2), (1, 2), (0, 1), ()):
        out = [torch.full_like(t, NAN) if i in keep else None for i, t in enumerate(full)]
        at = [0 if t is None else t.data_ptr() for t in out]
        a = finc.LINEAR_GRAD_ARGS.pack(code, act, M, K, N, dy.data_ptr(),
                                       x.data_ptr() if 1 in keep else 0,
                                       w.data_ptr() if 0 in keep else 0,
                                       pre.data_ptr() if act else 0, at[0], at[1],
                                       N, K, K, N, K, K, at[2], ws.data_ptr())
        assert lib.finc_linear_backward(a, finc._stream()) == 0
        for t, want in zip(out, full):
            assert t is None or torch.equal(t, want), keep


def test_no_rows():
    x, w = torch.zeros(0, 16, device=DEV), torch.ones(8, 16, device=DEV)
    assert finc.linear_forward(x, w, act="silu").shape == (0, 8)
    dx, dw, db = finc.linear_backward(torch.zeros(0, 8, device=DEV), x, w)
    assert dx.shape == (0, 16) and not dw.any() and not db.any()


def test_gradients_are_the_differences():
    x, w, b = normal(1, 20, 12), normal(2, 9, 12), normal(3, 9)
    dy = normal(4, 20, 9)
    d = [v.to(DEV) for v in (x, w, b)]
    for act in ("silu", "gelu"):
        pre = torch.empty(20, 9, device=DEV)
        finc.linear_forward(*d, act=act, pre_out=pre)
        grads = finc.linear_backward(dy.to(DEV), d[0], d[1], pre, act=act)
        for i, g in enumerate(grads):
            u, h = normal(5 + i, *d[i].shape).to(DEV), 2.0 ** -7
            v = []
            for s in (1, -1):
                at = [t + s * h * u if j == i else t for j, t in enumerate(d)]
                v.append(float((finc.linear_forward(*at, act=act).double()
                                * dy.to(DEV).double()).sum()))
            want = float((g.double() * u.double()).sum())
            # the third derivative's share (h^2) and the sums' rounding over h
            size = float(g.double().square().sum().sqrt())
            assert abs((v[0] - v[1]) / (2 * h) - want) <= 5e-3 * size, (act, i)


def everything():
    d = {n: normal(i, *s, kind=BF16).to(DEV) for i, (n, s) in enumerate(
        dict(x=(300, 1100), w=(70, 1100), r=(300, 70), one=(3, 1100)).items())}
    b = normal(9, 70).to(DEV)

    def call():
        pre = torch.empty(300, 70, dtype=BF16, device=DEV)
        y = finc.linear_forward(d["x"], d["w"], b, act="silu", residual=d["r"], pre_out=pre)
        return [y, pre, finc.linear_forward(d["one"], d["w"], b),
                *finc.linear_backward(d["r"], d["x"], d["w"], pre, act="silu"),
                *finc.linear_backward(d["r"], d["x"], d["w"])]

    return call


def test_graphs_replay_the_calls_and_streams_keep_them():
    call = everything()
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


def test_offsets_past_31_bits():
    K, N, M = 64, 32, 3
    far = torch.zeros(((M - 1) << 30) + 256, dtype=BF16, device=DEV)
    x = far.as_strided((M, K), (1 << 30, 1))
    y = far.as_strided((M, N), (1 << 30, 1), K)
    xs, w = normal(1, M, K, kind=BF16), normal(2, N, K, kind=BF16)
    x.copy_(xs.to(DEV))
    finc.linear_forward(x, w.to(DEV), out=y)
    ref.close(y, xs.double() @ w.double().T, "y", CHAIN)
    dx = far.as_strided((M, K), (1 << 30, 1), K + N)
    finc.linear_backward(y, x, w.to(DEV), dx=dx)
    ref.close(dx, y.cpu().double() @ w.double(), "dx", CHAIN)


def test_more_columns_than_a_row_of_the_grid():
    N = (1 << 28) + 65
    dy = torch.ones(1, 1, dtype=BF16, device=DEV).expand(1, N).contiguous()
    dy[0, -1] = 3.0
    x, w = torch.ones(1, 1, dtype=BF16, device=DEV), torch.ones(N, 1, dtype=BF16, device=DEV)
    dx, dw, db = finc.linear_backward(dy, x, w)
    assert bool((dw[:, 0] == dy[0]).all()) and float(dx) > N / 2
    assert float(db[-1]) == 3.0 and bool((db[:-1] == 1).all())
    del dx, dw, db
    # 129 rows in two blocks, whose sums are joined
    N = (1 << 26) + 65
    dy = dy[:, -N:].expand(129, N)
    dx, dw, db = finc.linear_backward(dy, x.expand(129, 1), w[:N])
    assert float(db[-1]) == 387.0 and bool((db[:-1] == 129).all())
    assert bool((dw[:-1] == 129).all())


def test_the_binding_refuses():
    x, w = torch.zeros(4, 16, device=DEV), torch.zeros(8, 16, device=DEV)
    y = torch.zeros(4, 8, device=DEV)
    for a, kw, what in [
            ((x, w[:, :8]), {}, "expected \\(N, 16\\)"), ((x, w.bfloat16()), {}, "w must be"),
            ((x, w[0]), {}, "expected \\(N, K\\)"), ((x.cpu(), w), {}, "device tensor"),
            ((x.double(), w), {}, "must be float32"), ((x.T, w), {}, "contiguous"),
            ((x, w, torch.zeros(7, device=DEV)), {}, "bias has shape"),
            ((x, w, torch.zeros(8, device=DEV, dtype=BF16)), {}, "bias must be"),
            ((x, w), dict(act="tanh"), "expected one of"), ((x, w), dict(residual=x), "residual has"),
            ((x, w), dict(out=y[:2]), "out has shape"), ((x, w), dict(pre_out=y.bfloat16()), "pre_out"),
            ((x, w), dict(workspace=torch.zeros(3, device=DEV)), "workspace")]:
        if "workspace" in kw:
            a = (torch.zeros(4, 4096, device=DEV), torch.zeros(8, 4096, device=DEV))
        with pytest.raises(ValueError, match=what):
            finc.linear_forward(*a, **kw)
    with pytest.raises(finc.FincError):
        finc.linear_forward(x, w, out=x[:, :8])
    with pytest.raises(finc.FincError):
        finc.linear_forward(x, w, out=y, pre_out=y)
    with pytest.raises(finc.FincError):
        finc.linear_forward(x, w, out=torch.zeros(1, 8, device=DEV).expand(4, 8))
    with pytest.raises(ValueError, match="need pre"):
        finc.linear_backward(y, x, w, act="silu")
    with pytest.raises(ValueError, match="dy has shape"):
        finc.linear_backward(x, x, w)
