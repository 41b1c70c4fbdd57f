"""The sequence operators where inputs, sizes and layouts are at their ends: empty
rows beside others, infinities, magnitudes, the 8-bit norm code for code, outputs in
other orders, streams, launches and offsets past 32 bits."""
import pytest
import torch

import seq_ref as ref
from gpu_util import DEV
from paper_2301_09266_amd import finc
from test_gpu_sequence import BF16, F16, F32, NAN, Rand, d64, dev, same_bits, scan_inputs, scan_kw

pytestmark = pytest.mark.gpu
INF = float("inf")


def grads(loss, leaves):
    """Gradients of float64 leaves, 0 where the loss does not depend on one."""
    got = torch.autograd.grad(loss, leaves, allow_unused=True)
    return [torch.zeros_like(t) if g is None else g for g, t in zip(got, leaves)]


# ---- causal convolution ----------------------------------------------------------


@pytest.mark.parametrize("K,silu,kind", [(2, False, F32), (4, True, BF16), (8, True, F16)])
@pytest.mark.parametrize("what", [NAN, INF])
def test_conv_gradients_take_nothing_from_an_empty_rows_state(K, silu, kind, what):
    """A row of length 0 hands its state on and adds nothing to dw and dbias."""
    r = Rand(K)
    B, D, L = 4, 5, 40
    n = torch.tensor([L, 0, 3, 0], dtype=torch.int32)
    x, dy = (r.normal(B, D, L, kind=kind) for _ in range(2))
    w, bias = r.normal(D, K, scale=K ** -0.5), r.normal(D, scale=0.1)
    st, dso = (r.normal(B, D, K - 1, kind=kind) for _ in range(2))
    st[1], st[3, :, 0] = what, what
    leaves = [d64(t, True) for t in (x, w, bias, st)]
    y, after = ref.conv(leaves[0], leaves[1], leaves[2], silu, leaves[3], n)
    want = grads((y * d64(dy)).sum() + (after * d64(dso)).sum(), leaves)
    got = finc.causal_conv_backward(dev(x), dev(w), dev(dy), dev(bias), silu=silu, state=dev(st),
                                    lengths=dev(n), dstate_out=dev(dso))
    # sums over the positions: fp32 roundings in quadrature, of sqrt(B L) terms' size
    chain = 64 + 4 * (B * L) ** 0.5
    for g, v, name in zip(got, want, ("dx", "dw", "dbias", "dstate")):
        assert torch.isfinite(g).all(), name
        ref.close(g, v, name, chain if name in ("dw", "dbias") else 64)


@pytest.mark.parametrize("n", [1, 8, 37, 40])
def test_conv_gradients_of_an_infinite_last_input(n):
    """The taps that no position has over it stay finite."""
    r = Rand(n)
    B, D, L, K = 2, 3, 40, 4
    x, dy = r.normal(B, D, L), r.normal(B, D, L)
    x[0, 1, n - 1] = INF
    w, lens = r.normal(D, K), torch.tensor([n, L], dtype=torch.int32)
    leaves = [d64(t, True) for t in (x, w)]
    y, _ = ref.conv(leaves[0], leaves[1], None, False, None, lens)
    used = (torch.arange(L) < lens[:, None]).double()[:, None]
    want = grads((torch.where(used > 0, y, 0.0) * d64(dy)).sum(), leaves)
    assert torch.isinf(want[1][1, K - 1]) and torch.isfinite(want[1][1, :K - 1]).all()
    got = finc.causal_conv_backward(dev(x), dev(w), dev(dy), lengths=dev(lens))
    ref.close(got[0], want[0], "dx")
    ref.close(got[1], want[1], "dw", 64 + 4 * (B * L) ** 0.5)


# ---- selective scan --------------------------------------------------------------


@pytest.mark.parametrize("L,n", [(40, 5), (64, 50), (200, 130), (300, 7)])
@pytest.mark.parametrize("N", [3, 16, 40])
def test_scan_of_states_without_memory_takes_nothing_from_padding(L, n, N):
    """A decay of minus infinity keeps nothing from one position to the next, and the
    step of 0 that stands for padding does not meet it."""
    B, D = 2, 6
    t, _, r = scan_inputs(B, D, L, N, 1, "gsldbp", F32, L + N)
    t["A"][2], t["A"][4, N // 2] = -INF, -INF
    lens = torch.tensor([n, L], dtype=torch.int32)
    for k in ("x", "dt", "Bm", "Cm", "z"):
        t[k] = r.normal(*t[k].shape)
    g, kw = scan_kw(t, lens, "gsldbp", None)
    states, end = finc.selective_scan_states(B, D, L, N, DEV), torch.empty(B, D, N, device=DEV)
    y = finc.selective_scan_forward(**g, **kw, state_out=end, states=states)
    leaf = {k: d64(v, True) for k, v in t.items()}
    yr, er = ref.scan(**leaf, softplus=True, lengths=lens)
    chain = 64 + 2 * L ** 0.5
    ref.close(y, yr, "y", chain)
    ref.close(end, er, "state after", chain)
    dy, dend = r.normal(B, D, L), r.normal(B, D, N)
    kw.pop("state")
    got = finc.selective_scan_backward(**g, **kw, dy=dev(dy), states=states, dstate_out=dev(dend))
    names = [k for k in leaf if k != "dt_bias"]
    want = dict(zip(names, grads((yr * d64(dy)).sum() + (er * d64(dend)).sum(),
                                 [leaf[k] for k in names])))
    key = dict(x="dx", dt="ddt", A="dA", Bm="dB", Cm="dC", D="dD", z="dz", state="dstate")
    for k in names:
        a, b = got[key[k]], want[k]
        if k == "dt":   # -inf exp(-inf) has no value: of the other channels
            a, b = a[:, [0, 1, 3, 5]], b[:, [0, 1, 3, 5]]
        ref.close(a, b, key[k], 2 * chain + (4 * (B * L * D) ** 0.5
                                             if k in ("A", "D", "Bm", "Cm") else 0))


@pytest.mark.parametrize("L,at", [(30, 11), (66, 40), (128, 0), (300, 129), (300, 299)])
@pytest.mark.parametrize("N", [5, 16, 33])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
def test_scan_of_one_infinite_input_leaves_the_rest(L, at, N, what):
    """No finite value of its channel from its position on, and the same bits elsewhere."""
    t, _, _ = scan_inputs(2, 20, L, N, 1, "gsdbp", F32, L + N)
    g, kw = scan_kw(t, None, "gsdbp", None)
    end, end2 = (torch.empty(2, 20, N, device=DEV) for _ in range(2))
    y = finc.selective_scan_forward(**g, **kw, state_out=end)
    g["x"][1, 7, at] = what
    y2 = finc.selective_scan_forward(**g, **kw, state_out=end2)
    assert not torch.isfinite(y2[1, 7, at:]).any() and not torch.isfinite(end2[1, 7]).any()
    y2[1, 7, at:], end2[1, 7] = y[1, 7, at:], end[1, 7]
    assert torch.equal(y2, y) and torch.equal(end2, end)


# ---- norm ------------------------------------------------------------------------


@pytest.mark.parametrize("D", [3, 100, 333, 1000, 2063, 4096, 8200])
@pytest.mark.parametrize("kind,size", [(F32, 1e22), (BF16, 3e36), (F32, 1e-25), (BF16, 1e-30)])
def test_norm_of_large_and_small_rows(D, kind, size):
    """Rows whose squares leave fp32's range."""
    r = Rand(D)
    x, w = r.normal(9, D, kind=kind, scale=size), 1 + r.normal(D, scale=0.1)
    y, s = finc.add_norm_forward(dev(x), dev(w), eps=0.0)
    assert torch.equal(s.cpu(), x)
    ref.close(y, ref.norm(d64(x), d64(w), 0.0), "y", 64 + 2 * D ** 0.5)


@pytest.mark.parametrize("D", [3, 333, 1000, 4096])
@pytest.mark.parametrize("size", [1e22, 1e-25])
def test_gradients_and_eight_bits_of_large_and_small_rows(D, size):
    r = Rand(D)
    x, dy, w = r.normal(9, D, scale=size), r.normal(9, D), 1 + r.normal(D, scale=0.1)
    chain = 64 + 2 * D ** 0.5
    x6, w6 = d64(x, True), d64(w, True)
    want = grads((ref.norm(x6, w6, 0.0) * d64(dy)).sum(), [x6, w6])
    dx, _, dw = finc.add_norm_backward(dev(dy), dev(x), dev(w), eps=0.0)
    ref.close(dx, want[0], "dx", chain)
    ref.close(dw, want[1], "dw", chain + 4 * 9 ** 0.5)
    q, scale, _ = finc.add_norm_forward(dev(x), dev(w), eps=0.0, fp8=True)
    want, ws = codes(ref.norm(d64(x), d64(w), 0.0))
    same_codes(q.cpu(), want)
    assert torch.equal(scale.cpu(), ws.float())


# ---- norm in 8 bits --------------------------------------------------------------


def codes(y):
    """The 8-bit values and scales of float64 rows, by their definition."""
    s = (y.abs().amax(-1, keepdim=True) / 448).clamp(min=2.0 ** -126)
    return (y / s).float().to(torch.float8_e4m3fn), s[..., 0]


def same_codes(got, want):
    a, b = got.view(torch.uint8), want.view(torch.uint8)
    n = int((a != b).sum())
    assert n == 0, f"{n} of {a.numel()} 8-bit values are other ones"


EIGHT = [(20000, 5), (9000, 100), (8000, 128), (3000, 333), (2000, 512), (1100, 1000), (1000, 1024),
         (500, 2048), (500, 2063), (250, 4096), (200, 5000), (130, 8192), (130, 8200), (64, 16384)]


@pytest.mark.parametrize("M,D", EIGHT)
@pytest.mark.parametrize("kind,rkind,p", [(BF16, BF16, 0.0), (BF16, F32, 0.1), (F16, F32, 0.3),
                                          (F32, F32, 0.5)])
def test_norm_in_eight_bits_code_for_code(M, D, kind, rkind, p):
    r = Rand(M + D)
    x, res = r.normal(M, D, kind=kind), r.normal(M, D, kind=rkind)
    w = 1 + r.normal(D, scale=0.1)
    drop = dict(p=p, seed=D << 40, offset=M << 35)
    q, scale, s = finc.add_norm_forward(dev(x), dev(w), dev(res), fp8=True, **drop)
    f = ref.dropout_factor(M, D, p, drop["seed"], drop["offset"]).to(DEV)
    rr = dev(x).double() * f + dev(res).double()
    ref.close(s, rr, "r")
    want, ws = codes(ref.norm(rr, dev(w).double(), 1e-5))
    same_codes(q, want)
    assert torch.equal(scale, ws.float())


def beside_the_middles(M, D, kind, r):
    """(x, residual or None, w) whose sums are a few fp32 steps from the middle of two 8-bit
    values of their row."""
    w = (1 + r.normal(D, scale=0.1)).abs() + 0.25
    w[0] = w.max() * 1.01
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    mid = ((every[1:] + every[:-1]) / 2)[torch.randint(0, 126, (M, D), generator=r.g)]
    top = torch.rand(M, 1, generator=r.g, dtype=torch.float64) * 7 + 1
    sign = torch.randint(0, 2, (M, D), generator=r.g) * 2 - 1
    s = (sign * mid * top * d64(w)[0] / (448 * d64(w))).float()
    s = (s.view(torch.int32) + torch.randint(-3, 4, (M, D), generator=r.g, dtype=torch.int32)) \
        .view(F32)
    s[:, 0] = top[:, 0].float()
    if kind == F32:
        return s, None, w
    x = r.normal(M, D, kind=kind, scale=0.01)
    return x, (s.double() - d64(x)).float(), w


@pytest.mark.parametrize("D", [7, 128, 500, 1000, 2063, 4096, 8000, 16384])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_norm_in_eight_bits_beside_the_middles(D, kind):
    x, res, w = beside_the_middles(40000 // D + 2, D, kind, Rand(D))
    q, scale, _ = finc.add_norm_forward(dev(x), dev(w), dev(res), fp8=True)
    rr = d64(x) if res is None else d64(x) + d64(res)
    want, ws = codes(ref.norm(rr, d64(w), 1e-5))
    same_codes(q.cpu(), want)
    assert torch.equal(scale.cpu(), ws.float())


# ---- layouts of outputs ----------------------------------------------------------


def channels_first(t):
    """The (B, D, L) view of a (D, B, L) tensor that is NaN."""
    B, D, L = t.shape
    return torch.full((D, B, L), NAN, dtype=t.dtype, device=DEV).transpose(0, 1)


@pytest.mark.parametrize("L,kind", [(40, F32), (150, BF16)])
def test_outputs_with_the_channels_outside(L, kind):
    """(D, B, L) in memory, as a channel-major projection writes it."""
    B, D, N = 3, 10, 16
    t, _, r = scan_inputs(B, D, L, N, 1, "gdbp", kind, L)
    g, kw = scan_kw(t, None, "gdbp", None)
    kw.pop("state")
    w, dy = r.normal(D, 4).to(DEV), r.normal(B, D, L, kind=kind).to(DEV)
    swapped = {k: channels_first(v).copy_(v) if k in ("x", "dt", "z") else v for k, v in g.items()}
    new = lambda: channels_first(dy)  # noqa: E731
    want = finc.causal_conv_forward(g["x"], w, silu=True)
    assert torch.equal(finc.causal_conv_forward(swapped["x"], w, silu=True, out=new()), want)
    want = finc.causal_conv_backward(g["x"], w, dy, silu=True)
    got = finc.causal_conv_backward(swapped["x"], w, dy, silu=True, dx=new())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    states = finc.selective_scan_states(B, D, L, N, DEV)
    want = finc.selective_scan_forward(**g, **kw, states=states)
    assert torch.equal(finc.selective_scan_forward(**swapped, **kw, out=new()), want)
    want = finc.selective_scan_backward(**g, **kw, dy=dy, states=states)
    got = finc.selective_scan_backward(**swapped, **kw, dy=dy, states=states, dx=new(), ddt=new(),
                                       dz=new())
    assert all(torch.equal(got[k], want[k]) for k in want if want[k] is not None)


def test_outputs_that_share_elements_are_refused():
    x, w = torch.zeros(3, 10, 40, device=DEV), torch.zeros(10, 4, device=DEV)
    space = torch.zeros(10 * 3 * 40, device=DEV)
    for steps in ((40, 119), (39, 120), (0, 120), (399, 40), (400, 39), (40, 40)):
        with pytest.raises(finc.FincError) as e:
            finc.causal_conv_forward(x, w, out=space.as_strided(x.shape, (*steps, 1)))
        assert e.value.code == finc.EINVAL, steps


# ---- launches of many workgroups -------------------------------------------------


def repeated(t, B):
    """B batch rows at one address."""
    return None if t is None else t.to(DEV).expand(B, *t.shape[1:])


def all_rows_equal(t, one):
    for part in t.split(max(1, (1 << 28) // max(1, one.numel()))):
        assert torch.equal(part, one.expand_as(part))


def test_conv_of_many_workgroups():
    """2^24 of them: 2^30 rows of 17 positions."""
    r = Rand(1)
    B, D, L = 1 << 15, 1 << 15, 17
    x, w = r.normal(1, D, L, kind=BF16), r.normal(D, 4).to(DEV)
    all_rows_equal(finc.causal_conv_forward(repeated(x, B), w, silu=True),
                   finc.causal_conv_forward(x.to(DEV), w, silu=True))


def test_conv_gradients_of_many_channels():
    """2^24 and some, a workgroup each."""
    D, L = (1 << 24) + 7, 3
    x, dy = (torch.empty(1, D, L, dtype=BF16, device=DEV).normal_() for _ in range(2))
    w = torch.empty(D, 2, device=DEV).normal_()
    dx, dw, _, _ = finc.causal_conv_backward(x, w, dy, silu=True)
    for at in (slice(0, 1000), slice((1 << 21) - 500, (1 << 21) + 500), slice(D - 1000, D)):
        one = finc.causal_conv_backward(x[:, at], w[at], dy[:, at], silu=True)
        assert torch.equal(dx[:, at], one[0]) and torch.equal(dw[at], one[1])


@pytest.mark.parametrize("L,B", [(65, 1 << 13), (1, 1 << 14)])
def test_scan_of_many_workgroups(L, B):
    """2^23 and 2^24 of them: a group a channel."""
    D = 1 << 10
    t, _, _ = scan_inputs(1, D, L, 1, D, "gsdbp", BF16, L)
    g, kw = scan_kw(t, None, "gsdbp", None)
    one_end, end = torch.empty(1, D, 1, device=DEV), torch.empty(B, D, 1, device=DEV)
    one = finc.selective_scan_forward(**g, **kw, state_out=one_end)
    for k in ("x", "dt", "z", "Bm", "Cm"):
        g[k] = repeated(g[k], B)
    kw["state"] = kw["state"].expand(B, D, 1).contiguous()
    y = finc.selective_scan_forward(**g, **kw, state_out=end)
    all_rows_equal(y, one)
    all_rows_equal(end, one_end)


def back(t, B, L, D, N, dy):
    g, kw = scan_kw(t, None, "gdbp", None)
    kw.pop("state")
    for k in ("x", "dt", "z", "Bm", "Cm"):
        g[k] = repeated(g[k], B)
    states = finc.selective_scan_states(B, D, L, N, DEV)
    finc.selective_scan_forward(**g, **kw, states=states)
    return finc.selective_scan_backward(**g, **kw, dy=repeated(dy, B), states=states)


@pytest.mark.parametrize("B,D,G,N,L", [(1 << 14, 16, 16, 32, 64),
                                       (1 << 13, 1 << 10, 1 << 10, 1, 65),
                                       (1 << 17, 64, 64, 64, 1)])
def test_scan_gradients_of_many_rows(B, D, G, N, L):
    """2^24 workgroups' worth of sums of dB and dC, 2^23 workgroups, and 2^30 of sums."""
    t, _, r = scan_inputs(1, D, L, N, G, "gdbp", BF16, N)
    dy = r.normal(1, D, L, kind=BF16)
    one, many = back(t, 1, L, D, N, dy), back(t, B, L, D, N, dy)
    for k in ("dx", "ddt", "dz", "dB", "dC", "dstate"):
        all_rows_equal(many[k], one[k])
    for k in ("dA", "dD", "ddt_bias"):   # B equal terms, each sum of them one rounding
        bar = B * 2.0 ** -24 * B * one[k].abs()
        assert ((many[k] - B * one[k]).abs() <= bar).all(), k


def test_scan_gradients_of_many_channels():
    """2^24 workgroups' worth of sums of the parameters."""
    D, N = 1 << 23, 62
    mk = lambda *s, kind=BF16: torch.empty(*s, dtype=kind, device=DEV).normal_()  # noqa: E731
    x, dt, dy = (mk(1, D, 1) for _ in range(3))
    Bm, Cm, A = mk(1, 1, N, 1), mk(1, 1, N, 1), mk(D, N, kind=F32).abs_().neg_()
    skip = mk(D, kind=F32)

    def run(at):
        c = slice(at.start, at.stop)
        v = dict(x=x[:, c], dt=dt[:, c], A=A[c], Bm=Bm, Cm=Cm, D=skip[c])
        states = finc.selective_scan_states(1, at.stop - at.start, 1, N, DEV)
        finc.selective_scan_forward(**v, states=states)
        return finc.selective_scan_backward(**v, dy=dy[:, c], states=states)

    whole = run(slice(0, D))
    for at in (slice(0, 64), slice(1 << 22, (1 << 22) + 128), slice(D - 64, D)):
        part = run(at)
        for k in ("dA", "dD"):
            assert torch.equal(whole[k][at], part[k]), (k, at)
        for k in ("dx", "ddt"):
            assert torch.equal(whole[k][:, at], part[k]), (k, at)


# ---- streams and offsets ---------------------------------------------------------


def test_calls_read_what_their_own_stream_writes_last():
    """Inputs that are NaN until a stream's copies, behind some milliseconds of its other
    work, have filled them: a call on any other stream would read them before."""
    r = Rand(77)
    B, D, L, N = 3, 24, 150, 16
    t, _, _ = scan_inputs(B, D, L, N, 1, "gdbp", BF16, 77)
    g, _ = scan_kw(t, None, "gdbp", None)
    rows = {k: r.normal(B, D, kind=BF16).to(DEV) for k in ("x", "dt")}
    Bm, Cm = (r.normal(B, 1, N, kind=BF16).to(DEV) for _ in range(2))
    wide = {k: r.normal(50, 333, kind=BF16).to(DEV) for k in ("x", "res", "dy")}
    w, nw, A = r.normal(D, 4).to(DEV), r.normal(333).to(DEV), g.pop("A")
    skip, bias = g.pop("D"), g.pop("dt_bias")
    inputs = dict(**{"s" + k: v for k, v in g.items()}, **{"r" + k: v for k, v in rows.items()},
                  **{"w" + k: v for k, v in wide.items()}, Bm=Bm, Cm=Cm)
    states = finc.selective_scan_states(B, D, L, N, DEV)

    def call(i):
        x, dt, z, sB, sC = (i["s" + k] for k in ("x", "dt", "z", "Bm", "Cm"))
        out = [finc.causal_conv_forward(x, w, silu=True),
               *finc.causal_conv_backward(x, w, z, silu=True)[:2],
               finc.causal_conv_step(i["rx"], w, torch.zeros(B, D, 3, dtype=BF16, device=DEV)),
               finc.selective_scan_forward(x, dt, A, sB, sC, skip, z, bias, states=states)]
        back = finc.selective_scan_backward(x, dt, A, sB, sC, z, states, skip, z, bias)
        out += [v for v in back.values() if v is not None]
        out.append(finc.selective_scan_step(i["rx"], i["rdt"], A, i["Bm"], i["Cm"],
                                            torch.zeros(B, D, N, device=DEV)))
        out += finc.add_norm_forward(i["wx"], nw, i["wres"], p=0.1, seed=3)
        out += finc.add_norm_forward(i["wx"], nw, i["wres"], fp8=True)
        out += finc.add_norm_backward(i["wdy"], i["wx"], nw, i["wres"], p=0.1, seed=3)
        out.append(finc.dropout(i["wx"], 0.2, 9, residual=i["wres"]))
        return out

    want = [v.clone() for v in call(inputs)]
    late = {k: torch.full_like(v, NAN) for k, v in inputs.items()}
    work = torch.zeros(2, 1 << 29, device=DEV)   # 2 GiB each
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(30):
            work[0].copy_(work[1])
        for k, v in late.items():
            v.copy_(inputs[k])
        got = call(late)
    side.synchronize()
    assert same_bits(want, got)


def far(shape, kind, space, at):
    """A view whose channels lie 2^31 elements and more apart."""
    B, D, L = shape
    return space.view(kind).as_strided(shape, ((1 << 31) + 8 * L, (1 << 31) + 4096, 1)
                                       if D > 1 else ((1 << 31) + 4096, L, 1), at)


@pytest.mark.parametrize("L", [40, 200])
@pytest.mark.parametrize("B,D", [(1, 2), (2, 1)])
def test_scan_offsets_past_31_bits(L, B, D):
    """Channels, batch rows and states' rows 2^31 elements apart, in inputs and outputs."""
    N = 2
    t, _, r = scan_inputs(B, D, L, N, 1, "gdbp", BF16, L)
    g, kw = scan_kw(t, None, "gdbp", None)
    kw.pop("state")
    dy = r.normal(B, D, L, kind=BF16).to(DEV)
    space = [torch.empty((1 << 31) + (1 << 20), dtype=BF16, device=DEV) for _ in range(4)]
    wide = dict(g)
    for i, k in enumerate(("x", "dt", "z")):
        wide[k] = far((B, D, L), BF16, space[0], 1000 * i + 1).copy_(g[k])
    for i, k in enumerate(("Bm", "Cm")):
        wide[k] = space[0].as_strided((B, 1, N, L), ((1 << 30) + 4096 if B > 1 else 0, 0,
                                                     (1 << 31) - 4096 if B == 1 else L, 1),
                                      5000 + 1000 * i).copy_(g[k])
    states = finc.selective_scan_states(B, D, L, N, DEV)
    want = finc.selective_scan_forward(**g, **kw, states=states)
    y = finc.selective_scan_forward(**wide, **kw, out=far((B, D, L), BF16, space[1], 0))
    assert torch.equal(y, want)
    want = finc.selective_scan_backward(**g, **kw, dy=dy, states=states)
    got = finc.selective_scan_backward(
        **wide, **kw, dy=far((B, D, L), BF16, space[0], 8001).copy_(dy), states=states,
        dx=far((B, D, L), BF16, space[1], 0), ddt=far((B, D, L), BF16, space[2], 0),
        dz=far((B, D, L), BF16, space[3], 0))
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("L,B,D", [(64, 33000, 1024), (129, 16400, 1024)])
def test_scan_of_more_than_2_31_elements(L, B, D):
    """The last rows of a tensor of more than 2^31 elements."""
    N, r = 4, Rand(L)
    x, dt = (torch.empty(B, D, L, dtype=BF16, device=DEV) for _ in range(2))
    x.normal_()
    dt.normal_(-2.0)
    Bm, Cm = (torch.empty(B, 1, N, L, dtype=BF16, device=DEV).normal_() for _ in range(2))
    A, end = -torch.exp(r.normal(D, N)).to(DEV), torch.empty(B, D, N, device=DEV)
    y = finc.selective_scan_forward(x, dt, A, Bm, Cm, state_out=end)
    for at in (slice(0, 2), slice(B // 2, B // 2 + 2), slice(B - 2, B)):
        one_end = torch.empty(2, D, N, device=DEV)
        one = finc.selective_scan_forward(x[at].clone(), dt[at].clone(), A, Bm[at].clone(),
                                          Cm[at].clone(), state_out=one_end)
        assert torch.equal(y[at], one) and torch.equal(end[at], one_end)
