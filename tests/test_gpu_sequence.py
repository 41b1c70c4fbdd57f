"""The sequence operators (causal convolution, selective scan, residual norm,
dropout) through the binding against 64-bit references: types, odd sizes, views,
padding that holds NaN, states, empty rows, idle slots, streams and graphs."""
import pytest
import torch

import seq_ref as ref
from gpu_util import DEV
from paper_2301_09266_amd import finc

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
NAN = float("nan")


class Rand:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)

    def normal(self, *shape, kind=F32, scale=1.0):
        return (torch.randn(*shape, generator=self.g, dtype=torch.float64) * scale).to(kind)

    def lengths(self, B, L):
        n = torch.randint(0, L + 1, (B,), generator=self.g, dtype=torch.int32)
        n[0] = L
        if B > 1:
            n[-1] = 0
        if B > 2:
            n[1] = L + 7     # clamped
        if B > 3:
            n[2] = -3
        return n


def dev(t, view=None):
    """On the device; view "half": the lower half of the rows of a wider tensor that
    is NaN elsewhere, "odd": that and an odd first address."""
    if t is None:
        return None
    if view is None:
        return t.to(DEV)
    B, D, L = t.shape
    pad = 1 if view == "odd" else 0
    big = torch.full((B, 2 * D, L + pad), NAN, dtype=t.dtype, device=DEV)
    big[:, :D, pad:] = t.to(DEV)
    return big[:, :D, pad:]


def out_like(t, view=None):
    """NaN-filled output of the layout of `dev`."""
    big = dev(torch.zeros_like(t, device="cpu"), view)
    big.fill_(NAN)
    return big


def poison(t, lengths):
    """Padding filled with NaN, the largest and the lowest value."""
    if lengths is None:
        return t
    t = t.clone()
    for b, n in enumerate(ref.ends(lengths, t.shape[0], t.shape[-1])):
        t[b, ..., n:] = torch.tensor(NAN)
        t[b, ..., n + 1::3] = torch.finfo(t.dtype).min
        t[b, ..., n + 2::3] = torch.tensor(float("inf"))
    return t


def d64(t, grad=False):
    return None if t is None else t.double().requires_grad_(grad)


# ---- causal convolution ---------------------------------------------------------

CONV = [  # B, D, L, K, silu, bias, state, lengths, type, view
    (1, 1, 1, 1, False, False, False, False, F32, None),
    (2, 3, 1, 4, True, True, True, False, BF16, None),
    (3, 5, 2, 4, True, True, True, True, F16, "odd"),
    (4, 7, 0, 3, True, True, True, False, F32, None),
    (5, 2, 7, 8, True, True, True, True, F32, "half"),
    (4, 3, 8, 2, False, True, False, True, BF16, "odd"),
    (2, 9, 9, 5, True, False, True, False, BF16, None),
    (3, 4, 63, 3, False, True, True, True, F32, "odd"),
    (2, 6, 257, 6, True, True, True, True, F16, "half"),
    (6, 3, 130, 7, True, True, False, True, BF16, "half"),
    (2, 2, 2050, 4, True, True, True, False, BF16, "odd"),
    (3, 2, 1031, 8, True, True, True, True, F16, None),
    (1, 300, 20, 4, True, True, False, False, F32, None),
    (70, 1, 33, 4, True, True, True, True, BF16, None),
]


@pytest.mark.parametrize("B,D,L,K,silu,bias,state,lens,kind,view", CONV)
def test_conv_forward_and_gradients(B, D, L, K, silu, bias, state, lens, kind, view):
    r = Rand(B * 1000 + L * 10 + K)
    n = r.lengths(B, L) if lens else None
    x, dy = (poison(r.normal(B, D, L, kind=kind), n) for _ in range(2))
    w = r.normal(D, K, scale=K ** -0.5)
    bs = r.normal(D, scale=0.1) if bias else None
    st, dso = (r.normal(B, D, K - 1, kind=kind) if state else None for _ in range(2))
    after = torch.full((B, D, K - 1), NAN, dtype=kind, device=DEV)
    kw = dict(silu=silu, state=dev(st), lengths=dev(n))
    y = finc.causal_conv_forward(dev(x, view), dev(w), dev(bs), out=out_like(x, view),
                                 state_out=after, **kw)
    leaves = [d64(t, True) for t in (torch.nan_to_num(x, 0.0), w, bs, st) if t is not None]
    it = iter(leaves)
    x6, w6 = next(it), next(it)
    b6 = next(it) if bias else None
    s6 = next(it) if state else None
    yr, ar = ref.conv(x6, w6, b6, silu, s6, n)
    ref.close(y, yr, "y")
    ref.close(after, ar, "state after")
    assert torch.equal(after.cpu().double(), ar.detach()), "the state is copied"
    dx, dw, db, ds = finc.causal_conv_backward(dev(x, view), dev(w), dev(dy, view), dev(bs),
                                               dstate_out=dev(dso), dx=out_like(x, view), **kw)
    loss = (yr * mask(d64(dy), n)).sum() + (0 if dso is None else (ar * d64(dso)).sum())
    want = torch.autograd.grad(loss, leaves, allow_unused=True)
    want = [torch.zeros_like(t) if g is None else g for g, t in zip(want, leaves)]
    # sums over the positions: fp32 roundings in quadrature, of sqrt(B L) terms' size
    chain = 64 + 4 * (B * L) ** 0.5
    for got, g, what in zip([dx, dw] + [t for t in (db, ds) if t is not None], want,
                            ["dx", "dw"] + ["dbias"] * bias + ["dstate"] * state):
        ref.close(got, g, what, chain if what in ("dw", "dbias") else 64)


def mask(t, lengths):
    if lengths is None:
        return t
    t = t.clone()
    for b, n in enumerate(ref.ends(lengths, t.shape[0], t.shape[-1])):
        t[b, ..., n:] = 0.0
    return t


def test_conv_in_pieces_is_the_whole():
    """A raster in pieces that hand on the state has the bits of one call."""
    r = Rand(3)
    x, w = r.normal(2, 5, 200, kind=BF16).to(DEV), r.normal(5, 4).to(DEV)
    whole = finc.causal_conv_forward(x, w, silu=True)
    state = torch.zeros(2, 5, 3, dtype=BF16, device=DEV)
    pieces = []
    for lo, hi in ((0, 1), (1, 3), (3, 90), (90, 200)):
        nxt = torch.empty_like(state)
        pieces.append(finc.causal_conv_forward(x[:, :, lo:hi], w, silu=True, state=state,
                                               state_out=nxt))
        state = nxt
    assert torch.equal(torch.cat(pieces, dim=2), whole)


@pytest.mark.parametrize("K,kind", [(1, F32), (2, BF16), (4, F16), (4, BF16), (8, F32)])
def test_conv_steps_are_the_forward(K, kind):
    """Single positions, slots in any order and idle rows among them."""
    r = Rand(K)
    B, D, S, L = 5, 300, 9, 6
    slots = torch.tensor([4, -1, 0, 8, S], dtype=torch.int32)
    x = r.normal(B, D, L, kind=kind)
    w, bias = r.normal(D, K), r.normal(D)
    state = r.normal(S, D, K - 1, kind=kind)
    st = state.to(DEV)
    live = [0, 2, 3]
    at = slots[live].long()
    y, after = ref.conv(d64(x[live]), d64(w), d64(bias), True, d64(state[at]), None)
    for t in range(L):
        wide = torch.full((B, 2 * D), NAN, dtype=kind, device=DEV)
        wide[:, :D] = x[:, :, t].to(DEV)
        got = finc.causal_conv_step(wide[:, :D], w.to(DEV), st, bias.to(DEV), silu=True,
                                    slots=slots.to(DEV))
        ref.close(got.cpu()[live], y[:, :, t], f"position {t}")
        assert not got.cpu()[[1, 4]].any(), "an idle row's output is 0"
    assert torch.equal(st.cpu()[at].double(), after.double())
    idle = [i for i in range(S) if i not in at.tolist()]
    assert torch.equal(st.cpu()[idle], state[idle]), "no other entry changes"


# ---- selective scan --------------------------------------------------------------

SCAN = [  # B, D, L, N, G, options (g gate, s state, l lengths, d skip, b bias, p softplus), type, view
    (1, 1, 1, 1, 1, "p", F32, None),
    (2, 5, 1, 16, 1, "gsdbp", BF16, None),
    (3, 6, 2, 5, 2, "gsldbp", F16, "odd"),
    (2, 4, 0, 16, 1, "gsdbp", F32, None),
    (4, 7, 5, 3, 7, "sl", F32, "half"),
    (2, 20, 63, 16, 4, "gsdbp", F32, "odd"),
    (2, 33, 64, 8, 1, "gdbp", BF16, None),
    (4, 18, 65, 4, 2, "gsldbp", F32, "half"),
    (2, 9, 127, 16, 1, "gsdbp", F32, None),
    (3, 40, 128, 16, 1, "gsldbp", BF16, "half"),
    (2, 17, 129, 20, 1, "gsdp", F16, "odd"),
    (1, 70, 300, 16, 1, "gdbp", F32, None),
    (5, 12, 260, 32, 3, "sldbp", BF16, "odd"),
    (2, 10, 200, 33, 1, "gsldbp", F32, None),
    (1, 6, 140, 64, 2, "gsdbp", F32, None),
    (2, 8, 50, 64, 1, "gsldbp", BF16, None),
    (3, 8, 1030, 16, 1, "gsldbp", F32, None),
    (1, 132, 150, 16, 2, "gdbp", F16, None),
    (300, 30, 3, 16, 1, "gsldbp", F32, None),    # many rows: a wave keeps all the states
    (130, 64, 70, 8, 1, "gldbp", BF16, None),
]


def scan_inputs(B, D, L, N, G, opt, kind, seed):
    r = Rand(seed)
    n = r.lengths(B, L) if "l" in opt else None
    p = lambda t: poison(t, n)  # noqa: E731
    t = dict(x=p(r.normal(B, D, L, kind=kind)), dt=p(r.normal(B, D, L, kind=kind, scale=0.5)),
             A=-torch.exp(r.normal(D, N, scale=0.3)) * torch.arange(1, N + 1),
             Bm=p(r.normal(B, G, N, L, kind=kind)), Cm=p(r.normal(B, G, N, L, kind=kind)),
             D=r.normal(D) if "d" in opt else None,
             z=p(r.normal(B, D, L, kind=kind)) if "g" in opt else None,
             dt_bias=r.normal(D) - 2 if "b" in opt else None,
             state=r.normal(B, D, N) if "s" in opt else None)
    if "p" not in opt:   # the steps themselves
        t["dt"] = p(torch.rand(B, D, L, generator=r.g).to(kind) * 0.2)
    return t, n, r


def scan_kw(t, n, opt, view):
    g = {k: dev(v, view if k in ("x", "dt", "z") else None) for k, v in t.items()}
    state = g.pop("state")
    return g, dict(state=state, lengths=dev(n), softplus="p" in opt)


@pytest.mark.parametrize("B,D,L,N,G,opt,kind,view", SCAN)
def test_scan_forward_and_gradients(B, D, L, N, G, opt, kind, view):
    t, n, r = scan_inputs(B, D, L, N, G, opt, kind, B + 10 * L + N)
    g, kw = scan_kw(t, n, opt, view)
    end = torch.full((B, D, N), NAN, device=DEV)
    states = finc.selective_scan_states(B, D, L, N, DEV).fill_(NAN)
    y = finc.selective_scan_forward(**g, **kw, out=out_like(t["x"], view), state_out=end,
                                    states=states)
    plain = {k: (torch.nan_to_num(v, 0.0, 0.0, 0.0) if v is not None else None)
             for k, v in t.items()}
    names = [k for k, v in plain.items() if v is not None]
    leaf = {k: d64(plain[k], True) for k in names}
    full = {k: leaf.get(k) for k in t}
    yr, er = ref.scan(**full, softplus="p" in opt, lengths=n)
    # each of the positions before adds a few roundings
    chain = 64 + 2 * L ** 0.5
    ref.close(y, yr, "y", chain)
    ref.close(end, er, "state after", chain)
    again = finc.selective_scan_forward(**g, **kw)
    assert torch.equal(again, y), "the same bits without states"
    dy = poison(r.normal(B, D, L, kind=kind), n)
    dend = r.normal(B, D, N) if "s" in opt else None
    kw.pop("state")
    grads = finc.selective_scan_backward(
        **{k: g[k] for k in ("x", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias")}, **kw,
        dy=dev(dy, view), states=states, dstate_out=dev(dend), dx=out_like(dy, view),
        ddt=out_like(dy, view), dz=out_like(dy, view) if "g" in opt else None)
    loss = (yr * torch.nan_to_num(mask(d64(dy), n))).sum()
    if dend is not None:
        loss = loss + (er * d64(dend)).sum()
    want = torch.autograd.grad(loss, list(leaf.values()), allow_unused=True)
    want = {k: torch.zeros_like(leaf[k]) if w is None else w for k, w in zip(names, want)}
    key = dict(x="dx", dt="ddt", A="dA", Bm="dB", Cm="dC", D="dD", z="dz", dt_bias="ddt_bias",
               state="dstate")
    for k in names:
        many = k in ("A", "D", "dt_bias", "Bm", "Cm")
        ref.close(grads[key[k]], want[k], key[k],
                  2 * chain + (4 * (B * L * D) ** 0.5 if many else 0))
    for k in ("D", "z", "dt_bias"):
        if t[k] is None:
            assert grads[key[k]] is None


SHORT = [  # short rasters and last parts of every length, rows that end before them
    (3, 37, 3, 16, 1, "gsldbp", BF16, None),
    (2, 70, 4, 1, 1, "gsdbp", F32, "odd"),
    (4, 20, 8, 5, 2, "gsldbp", F16, "half"),
    (2, 66, 15, 64, 1, "gsdbp", F32, None),
    (3, 18, 16, 2, 1, "sldp", BF16, "odd"),
    (5, 33, 17, 16, 3, "gsldbp", F32, None),
    (2, 64, 31, 33, 1, "gdbp", F16, None),
    (6, 24, 49, 7, 2, "gsldbp", BF16, "half"),
    (130, 505, 20, 8, 1, "gsldbp", BF16, None),   # whole workgroups
    (5, 10, 66, 16, 1, "gsldbp", F32, "odd"),
    (5, 10, 71, 16, 2, "gsldbp", BF16, "odd"),
    (4, 9, 133, 40, 1, "gsldbp", F16, "half"),
    (6, 9, 135, 16, 1, "gsldbp", F32, None),
    (5, 8, 257, 9, 2, "sldbp", BF16, "odd"),
]


@pytest.mark.parametrize("B,D,L,N,G,opt,kind,view", SHORT)
def test_scan_short_rasters_and_ends(B, D, L, N, G, opt, kind, view):
    test_scan_forward_and_gradients(B, D, L, N, G, opt, kind, view)


@pytest.mark.parametrize("L,N", [(1, 3), (20, 5), (20, 16), (40, 33)])
def test_scan_infinite_inputs_stay_infinite(L, N):
    """An infinite input's row, N filling its lanes or not: the formula's values in a
    short raster (in a longer one the lanes' maps may multiply it by 0)."""
    t, _, _ = scan_inputs(2, 6, L, N, 1, "sdbp", F32, L + N)
    t["Bm"], t["Cm"] = t["Bm"].abs() + 0.1, t["Cm"].abs() + 0.1
    t["x"][0, 2, L // 2] = float("inf")
    t["x"][1, 3, L - 1] = -float("inf")
    t["D"] = t["D"].abs() + 0.1
    g, kw = scan_kw(t, None, "sdbp", None)
    end = torch.empty(2, 6, N, device=DEV)
    y = finc.selective_scan_forward(**g, **kw, state_out=end)
    yr, er = ref.scan(**{k: d64(v) if v is not None else None for k, v in t.items()},
                      softplus=True, lengths=None)
    assert bool(torch.isinf(yr).any()) and bool(torch.isinf(er).any())
    ref.close(y, yr, "y", 64 + 2 * L ** 0.5)
    ref.close(end, er, "state after", 64 + 2 * L ** 0.5)


def test_scan_bits_of_short_rasters_do_not_depend_on_the_number_of_rows():
    t, _, _ = scan_inputs(1, 520, 40, 16, 2, "gsdbp", BF16, 11)
    g, kw = scan_kw(t, None, "gsdbp", None)
    one = finc.selective_scan_forward(**g, **kw)
    wide = {k: v.expand(130, *v.shape[1:]) if k in ("x", "dt", "Bm", "Cm", "z") else v
            for k, v in g.items()}
    many = dict(kw, state=kw["state"].expand(130, 520, 16).contiguous())
    assert torch.equal(finc.selective_scan_forward(**wide, **many), one.expand(130, 520, 40))
    states = finc.selective_scan_states(1, 520, 40, 16, DEV)
    assert torch.equal(finc.selective_scan_forward(**g, **kw, states=states), one)


def test_scan_gradients_are_the_differences():
    """The change of the fp32 forward along a direction, against the gradients."""
    t, n, r = scan_inputs(2, 12, 90, 16, 2, "gsdbp", F32, 5)
    g, kw = scan_kw(t, n, "gsdbp", None)
    state = kw.pop("state")
    g["state"] = state
    weight = r.normal(2, 12, 90).to(DEV)

    def loss(v):
        return float((finc.selective_scan_forward(**v, **kw) * weight).double().sum())

    states = finc.selective_scan_states(2, 12, 90, 16, DEV)
    finc.selective_scan_forward(**g, **kw, states=states)
    got = finc.selective_scan_backward(**{k: v for k, v in g.items() if k != "state"}, **kw,
                                       dy=weight, states=states)
    key = dict(x="dx", dt="ddt", A="dA", Bm="dB", Cm="dC", D="dD", z="dz", dt_bias="ddt_bias",
               state="dstate")
    for k in key:
        v = r.normal(*g[k].shape).to(DEV)
        e = 1e-3 if k != "A" else 1e-4
        up, down = (loss(dict(g, **{k: g[k] + s * e * v})) for s in (1, -1))
        slope = (up - down) / (2 * e)
        inner = float((got[key[k]].double() * v.double()).sum())
        size = float(got[key[k]].double().norm() * v.double().norm())
        # the differences' own error: e^2 of the third derivative and the loss's fp32
        assert abs(slope - inner) <= 0.02 * abs(inner) + 2e-3 * size, (k, slope, inner, size)


@pytest.mark.parametrize("N,G,kind", [(1, 1, F32), (4, 2, BF16), (5, 1, F16), (16, 1, F32),
                                      (16, 4, BF16), (33, 1, F32), (64, 2, F32)])
def test_scan_steps_are_the_forward(N, G, kind):
    B, D, S, L = 5, 72, 9, 4
    slots = torch.tensor([4, -1, 0, 8, S], dtype=torch.int32)
    t, _, r = scan_inputs(B, D, L, N, G, "gdbp", kind, N)
    state = r.normal(S, D, N)
    st = state.to(DEV)
    live = [0, 2, 3]
    at = slots[live].long()
    full = {k: d64(v[live] if v is not None and k in ("x", "dt", "Bm", "Cm", "z") else v)
            for k, v in t.items()}
    full["state"] = d64(state[at])
    y, after = ref.scan(**full, softplus=True, lengths=None)
    par = {k: dev(t[k]) for k in ("A", "D", "dt_bias")}
    for i in range(L):
        wide = torch.full((B, 2 * D + 2 * G * N + 1), NAN, dtype=kind, device=DEV)
        wide[:, 1:D + 1] = t["x"][:, :, i].to(DEV)
        wide[:, D + 1:2 * D + 1] = t["z"][:, :, i].to(DEV)
        wide[:, 2 * D + 1:] = torch.cat([t["Bm"][..., i].flatten(1), t["Cm"][..., i].flatten(1)],
                                        dim=1).to(DEV)
        Bm, Cm = (wide[:, 2 * D + 1 + k * G * N:][:, :G * N].unflatten(1, (G, N)) for k in (0, 1))
        got = finc.selective_scan_step(wide[:, 1:D + 1], dev(t["dt"][:, :, i].contiguous()),
                                       par["A"], Bm, Cm, st, par["D"], wide[:, D + 1:2 * D + 1],
                                       par["dt_bias"], slots=slots.to(DEV))
        ref.close(got.cpu()[live], y[:, :, i], f"position {i}")
        assert not got.cpu()[[1, 4]].any(), "an idle row's output is 0"
    ref.close(st.cpu()[at], after, "state")
    idle = [i for i in range(S) if i not in at.tolist()]
    assert torch.equal(st.cpu()[idle], state[idle]), "no other entry changes"


def test_scan_state_in_place_and_shared_inputs():
    """state_out over state; one B and C, and one step, for every batch row."""
    t, _, r = scan_inputs(3, 8, 40, 16, 1, "sdbp", F32, 8)
    g, kw = scan_kw(t, None, "sdbp", None)
    g["Bm"], g["Cm"] = (g[k][:1].expand(3, 1, 16, 40) for k in ("Bm", "Cm"))
    g["dt"] = g["dt"][:, :1].expand(3, 8, 40)
    end = torch.empty(3, 8, 16, device=DEV)
    y = finc.selective_scan_forward(**g, **kw, state_out=end)
    st = kw["state"].clone()
    y2 = finc.selective_scan_forward(**g, **{**kw, "state": st}, state_out=st)
    assert torch.equal(y, y2) and torch.equal(st, end)
    full = {k: d64(v.cpu()) if v is not None else None for k, v in g.items()}
    yr, er = ref.scan(**full, softplus=True, state=d64(t["state"]), lengths=None)
    ref.close(y, yr, "y")
    ref.close(end, er, "state")


def test_scan_rows_do_not_depend_on_the_batch():
    t, _, _ = scan_inputs(4, 20, 150, 16, 1, "gsdbp", BF16, 9)
    g, kw = scan_kw(t, None, "gsdbp", None)
    whole = finc.selective_scan_forward(**g, **kw)
    cut = {k: v[2:3] if k in ("x", "dt", "Bm", "Cm", "z") else v for k, v in g.items()}
    one = finc.selective_scan_forward(**cut, **{**kw, "state": kw["state"][2:3].contiguous()})
    assert torch.equal(one[0], whole[2])


def test_scan_bits_do_not_depend_on_the_number_of_rows():
    """One row alone and among enough rows to fill the card, states kept or not."""
    t, _, _ = scan_inputs(1, 520, 200, 16, 2, "gsdbp", BF16, 10)
    g, kw = scan_kw(t, None, "gsdbp", None)
    one = finc.selective_scan_forward(**g, **kw)
    wide = {k: v.expand(40, *v.shape[1:]) if k in ("x", "dt", "Bm", "Cm", "z") else v
            for k, v in g.items()}
    many = dict(kw, state=kw["state"].expand(40, 520, 16).contiguous())
    got = finc.selective_scan_forward(**wide, **many)
    assert torch.equal(got, one.expand_as(got))
    states = finc.selective_scan_states(1, 520, 200, 16, DEV)
    assert torch.equal(finc.selective_scan_forward(**g, **kw, states=states), one)


# ---- norm ------------------------------------------------------------------------

NORM = [  # M, D, residual, type, rtype, p
    (1, 1, True, F32, F32, 0.0),
    (3, 7, True, BF16, BF16, 0.25),
    (17, 16, True, BF16, F32, 0.0),
    (100, 100, False, F16, F16, 0.5),
    (33, 128, True, F32, F32, 0.1),
    (9, 129, True, BF16, F32, 0.1),
    (5, 512, True, F16, F32, 0.0),
    (70, 513, True, BF16, BF16, 0.0),
    (13, 1000, True, BF16, BF16, 0.1),
    (2500, 264, True, F32, F32, 0.3),
    (6, 2048, True, BF16, F32, 0.1),
    (3, 2049, True, F32, F32, 0.1),
    (520, 4097, True, BF16, BF16, 0.0),
    (2, 8192, False, F32, F32, 0.0),
    (3, 8200, True, F16, F32, 0.1),
    (2, 16384, True, BF16, BF16, 0.1),
    (0, 64, True, F32, F32, 0.1),
]


def wide_rows(t):
    """Rows of a wider tensor at an odd address."""
    M, D = t.shape
    big = torch.full((M, D + 5), NAN, dtype=t.dtype, device=DEV)
    big[:, 1:D + 1] = t.to(DEV)
    return big[:, 1:D + 1]


@pytest.mark.parametrize("M,D,residual,kind,rkind,p", NORM)
@pytest.mark.parametrize("view", [False, True])
def test_norm_forward_and_gradients(M, D, residual, kind, rkind, p, view):
    r = Rand(M + D)
    put = wide_rows if view else dev
    x, dy = (r.normal(M, D, kind=kind) for _ in range(2))
    res = r.normal(M, D, kind=rkind) if residual else None
    w = 1 + r.normal(D, scale=0.1)
    drop = dict(p=p, seed=(M << 33) + D, offset=(1 << 40) + 3)
    f = ref.dropout_factor(M, D, p, drop["seed"], drop["offset"])
    y, got_r = finc.add_norm_forward(put(x), dev(w), None if res is None else put(res), **drop)
    rr = d64(x) * f + (0 if res is None else d64(res))
    ref.close(got_r, rr, "r")
    # the mean square of D terms
    chain = 64 + 2 * D ** 0.5
    ref.close(y, ref.norm(rr, d64(w), 1e-5), "y", chain)
    assert got_r.dtype == (rkind if residual else kind)
    rs, dr = r.normal(M, D, kind=rkind), r.normal(M, D, kind=rkind)
    for extra in (dr, None):
        dx, dres, dw = finc.add_norm_backward(put(dy), put(rs), dev(w),
                                              None if extra is None else put(extra), **drop)
        r6, w6 = d64(rs, True), d64(w, True)
        loss = (ref.norm(r6, w6, 1e-5) * d64(dy)).sum()
        if extra is not None:
            loss = loss + (r6 * d64(extra)).sum()
        want_r, want_w = torch.autograd.grad(loss, (r6, w6))
        assert dres.dtype == rkind and dx.dtype == kind
        ref.close(dres, want_r, "dresidual", chain)
        ref.close(dx, want_r * f, "dx", chain)
        ref.close(dw, want_w, "dw", chain + 4 * M ** 0.5)


def test_norm_in_place():
    r = Rand(2)
    x, res, w = r.normal(50, 333).to(DEV), r.normal(50, 333).to(DEV), r.normal(333).to(DEV)
    y, s = finc.add_norm_forward(x, w, res, p=0.2, seed=3)
    x2, res2 = x.clone(), res.clone()
    finc.add_norm_forward(x2, w, res2, p=0.2, seed=3, out=x2, residual_out=res2)
    assert torch.equal(x2, y) and torch.equal(res2, s)
    dy, dr = r.normal(50, 333).to(DEV), r.normal(50, 333).to(DEV)
    dx, dres, dw = finc.add_norm_backward(dy, s, w, dr, p=0.2, seed=3)
    dy2, dr2 = dy.clone(), dr.clone()
    _, _, dw2 = finc.add_norm_backward(dy2, s, w, dr2, p=0.2, seed=3, dx=dy2, dresidual=dr2)
    assert torch.equal(dy2, dx) and torch.equal(dr2, dres) and torch.equal(dw2, dw)
    # without dropout the two gradients are one tensor: over dy, over dr, or new
    want, same, _ = finc.add_norm_backward(dy, s, w, dr)
    assert want is same
    dy3, dr3 = dy.clone(), dr.clone()
    assert torch.equal(finc.add_norm_backward(dy3, s, w, dr, dx=dy3)[1], want)
    assert torch.equal(finc.add_norm_backward(dy, s, w, dr3, dresidual=dr3)[0], want)
    assert torch.equal(dy3, want) and torch.equal(dr3, want)
    a, b, _ = finc.add_norm_backward(dy, s, w, dr, dx=torch.empty_like(dy),
                                     dresidual=torch.empty_like(dy))
    assert a is not b and torch.equal(a, want) and torch.equal(b, want)


@pytest.mark.parametrize("D", [9, 131, 515, 1030, 2063, 4099, 8201])
def test_norm_in_place_over_rows_of_many_waves(D):
    """The last elements of a row are loaded with some of the neighbouring wave's."""
    r = Rand(D)
    x, res, dr = (r.normal(70, D, kind=BF16).to(DEV) for _ in range(3))
    w = 1 + r.normal(D, scale=0.1).to(DEV)
    y, s = finc.add_norm_forward(x, w, res)
    dx, dres, dw = finc.add_norm_backward(x, s, w, dr, p=0.1, seed=4)
    y8, scale, _ = finc.add_norm_forward(x, w, res, fp8=True)
    for _ in range(3):
        x2, res2 = x.clone(), res.clone()
        finc.add_norm_forward(x2, w, res2, out=x2, residual_out=res2)
        assert torch.equal(x2, y) and torch.equal(res2, s)
        x2, dr2 = x.clone(), dr.clone()
        dw2 = finc.add_norm_backward(x2, s, w, dr2, p=0.1, seed=4, dx=x2, dresidual=dr2)[2]
        assert torch.equal(x2, dx) and torch.equal(dr2, dres) and torch.equal(dw2, dw)
        res2 = res.clone()
        got8, scale2, _ = finc.add_norm_forward(x, w, res2, fp8=True, residual_out=res2)
        assert torch.equal(got8.view(torch.uint8), y8.view(torch.uint8))
        assert torch.equal(scale2, scale) and torch.equal(res2, s)


@pytest.mark.parametrize("M,D,kind", [(1, 5, F32), (40, 64, BF16), (9, 1000, BF16), (7, 2048, F16),
                                      (3, 5000, F32), (2, 16384, BF16)])
def test_norm_in_eight_bits(M, D, kind):
    r = Rand(D)
    x, res, w = r.normal(M, D, kind=kind), r.normal(M, D), 1 + r.normal(D, scale=0.1)
    q, scale, got_r = finc.add_norm_forward(dev(x), dev(w), dev(res), fp8=True)
    rr = d64(x) + d64(res)
    y = ref.norm(rr, d64(w), 1e-5)
    ref.close(got_r, rr, "r")
    ref.close(scale, y.abs().max(1).values / 448, "scale", 64 + 2 * D ** 0.5)
    v = q.float().cpu().double()
    s = scale.cpu().double()[:, None]
    assert (v.abs().max(1).values == 448).all(), "the largest takes the last step"
    # half a step of e4m3: 2^-4 of the value, 2^-10 below the least normal 2^-6
    bar = (y / s).abs().clamp(min=2.0 ** -6) * 2.0 ** -4 * 1.0001
    assert ((v - y / s).abs() <= bar).all()


def test_norm_of_zeros_infinities_and_nan():
    x = torch.zeros(4, 40)
    x[1, 3], x[2, 5] = float("inf"), NAN
    x[3] = torch.finfo(F32).tiny
    w = torch.ones(40)
    for kind in TYPES:
        y, _ = finc.add_norm_forward(dev(x.to(kind)), dev(w))
        q, scale, _ = finc.add_norm_forward(dev(x.to(kind)), dev(w), fp8=True)
        y, q, scale = y.float().cpu(), q.float().cpu(), scale.cpu()
        assert not y[0].any() and not q[0].any() and scale[0] == 2.0 ** -126
        # an infinite root mean square: 0 beside the infinity, which has no value
        assert torch.isnan(y[1, 3]) and not y[1, :3].any() and not y[1, 4:].any()
        assert torch.isnan(scale[1]) and torch.isnan(q[1]).all()
        assert torch.isnan(y[2]).all() and torch.isnan(q[2]).all() and torch.isnan(scale[2])
        assert torch.isfinite(y[3]).all() and torch.isfinite(q[3]).all()


# ---- dropout ---------------------------------------------------------------------


@pytest.mark.parametrize("M,D,kind,residual,p", [(1, 1, F32, False, 0.5), (5, 7, BF16, True, 0.1),
                                                 (100, 64, F16, True, 0.3),
                                                 (33, 333, F32, False, 0.25),
                                                 (4100, 129, BF16, True, 0.05),
                                                 (3, 70000, F32, True, 0.9),
                                                 (9, 20, F32, False, 0.0), (0, 8, F32, False, 0.1)])
def test_dropout_is_the_generator(M, D, kind, residual, p):
    r = Rand(M + D)
    x = r.normal(M, D, kind=kind)
    res = r.normal(M, D, kind=kind) if residual else None
    for seed, offset in ((0, 0), (0xFEDCBA9876543210, (1 << 32) - 3), (7, (1 << 64) - 1)):
        f = ref.dropout_factor(M, D, p, seed, offset)
        y = finc.dropout(wide_rows(x), p, seed, offset, residual=dev(res))
        want = d64(x) * f
        if residual:
            ref.close(y, want + d64(res), "y")
        else:
            ref.close(y, want, "y")
            assert torch.equal(y.cpu() == 0, want == 0), "the same elements are dropped"
    again = dev(x)
    finc.dropout(again, p, 3, out=again)
    assert torch.equal(again, finc.dropout(dev(x), p, 3)), "in place"


def test_dropout_goes_on_at_the_next_counter():
    x = torch.ones(6, 20, device=DEV)
    whole = finc.dropout(x, 0.5, 11)
    used = finc.dropout_counters(4, 20)
    assert used == 12
    assert torch.equal(finc.dropout(x[4:], 0.5, 11, used), whole[4:])


# ---- streams, graphs, order, size ----------------------------------------------------


def everything(seed, B=3, D=24, L=150, N=16):
    """One call of each entry point; the outputs."""
    t, n, r = scan_inputs(B, D, L, N, 1, "gsldbp", BF16, seed)
    g, kw = scan_kw(t, n, "gsldbp", None)
    w, rows = r.normal(D, 4).to(DEV), r.normal(B * L, D, kind=BF16).to(DEV)
    nw, dy = r.normal(D).to(DEV), r.normal(B, D, L, kind=BF16).to(DEV)
    state = kw.pop("state")
    cs = torch.zeros(B, D, 3, dtype=BF16, device=DEV)
    rec = {k: v for k, v in g.items()}

    def call():
        st, cst = state.clone(), cs.clone()
        out = [finc.causal_conv_forward(g["x"], w, silu=True, lengths=kw["lengths"])]
        out += [v for v in finc.causal_conv_backward(g["x"], w, dy, silu=True,
                                                     lengths=kw["lengths"]) if v is not None]
        out.append(finc.causal_conv_step(rows[:B], w, cst))
        keep = finc.selective_scan_states(B, D, L, N, DEV)
        out.append(finc.selective_scan_forward(**rec, **kw, state=st, state_out=st, states=keep))
        back = finc.selective_scan_backward(**rec, **kw, dy=dy, states=keep)
        out += [v for v in back.values() if v is not None]
        Bm, Cm = (rows[:B, :N].unflatten(1, (1, N)) for _ in range(2))
        out.append(finc.selective_scan_step(rows[:B], rows[B:2 * B], g["A"], Bm, Cm, st))
        y, res = finc.add_norm_forward(rows, nw, rows, p=0.1, seed=5)
        out += [y, res, st, cst, *finc.add_norm_forward(rows, nw, fp8=True)[:2]]
        out += list(finc.add_norm_backward(rows, res, nw, rows, p=0.1, seed=5))
        out.append(finc.dropout(rows, 0.4, 9, residual=rows))
        return out

    return call


def same_bits(a, b):
    return all(torch.equal(u.contiguous().view(torch.uint8), v.contiguous().view(torch.uint8))
               for u, v in zip(a, b))


def test_repeated_calls_have_the_same_bits():
    call = everything(21)
    first = [t.clone() for t in call()]
    assert same_bits(first, call())


def test_calls_run_on_the_current_stream():
    """Inputs that another stream still writes, in order on that stream alone."""
    call = everything(22)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert same_bits(want, got)


def test_graphs_replay_the_calls():
    call = everything(23)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for i in range(3):
        for t in got:
            t.view(torch.uint8).zero_() if t.is_contiguous() else t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(want, got), f"replay {i}"
        assert same_bits(want, call()), "eager work between replays"


def test_outputs_beside_their_inputs():
    """A projection's two halves: the output of one in the other's place, and two
    gradients side by side."""
    t, _, r = scan_inputs(3, 10, 70, 16, 1, "gdbp", BF16, 31)
    g, kw = scan_kw(t, None, "gdbp", None)
    w = r.normal(10, 4).to(DEV)
    both = torch.full((3, 20, 70), NAN, dtype=BF16, device=DEV)
    both[:, :10] = g["x"]
    y = finc.causal_conv_forward(both[:, :10], w, out=both[:, 10:])
    assert torch.equal(both[:, 10:], finc.causal_conv_forward(g["x"], w))
    assert torch.equal(both[:, :10], g["x"]) and y.data_ptr() == both[:, 10:].data_ptr()
    with pytest.raises(finc.FincError):
        finc.causal_conv_forward(both[:, :10], w, out=both[:, 5:15])
    states = finc.selective_scan_states(3, 10, 70, 16, DEV)
    kw.pop("state")
    finc.selective_scan_forward(**g, **kw, states=states)
    dy = r.normal(3, 10, 70, kind=BF16).to(DEV)
    args = {k: v for k, v in g.items()}
    apart = finc.selective_scan_backward(**args, **kw, dy=dy, states=states)
    pair = torch.full((3, 20, 70), NAN, dtype=BF16, device=DEV)
    finc.selective_scan_backward(**args, **kw, dy=dy, states=states, dx=pair[:, :10],
                                 dz=pair[:, 10:])
    assert torch.equal(pair, torch.cat([apart["dx"], apart["dz"]], dim=1))


def test_empty_batches():
    x = torch.empty(0, 6, 40, device=DEV)
    w, bias = torch.ones(6, 4, device=DEV), torch.ones(6, device=DEV)
    assert finc.causal_conv_forward(x, w, bias).shape == x.shape
    dx, dw, db, _ = finc.causal_conv_backward(x, w, x, bias)
    assert dx.shape == x.shape and not dw.any() and not db.any()
    A, Bm = -torch.ones(6, 16, device=DEV), torch.empty(0, 2, 16, 40, device=DEV)
    states = finc.selective_scan_states(0, 6, 40, 16, DEV)
    assert finc.selective_scan_forward(x, x, A, Bm, Bm, bias, x, bias,
                                       states=states).shape == x.shape
    grads = finc.selective_scan_backward(x, x, A, Bm, Bm, x, states, bias, x, bias)
    assert not grads["dA"].any() and not grads["dD"].any() and not grads["ddt_bias"].any()
    assert finc.causal_conv_step(x[:, :, 0], w, torch.ones(2, 6, 3, device=DEV)).shape == (0, 6)
    assert finc.selective_scan_step(x[:, :, 0], x[:, :, 0], A, Bm[..., 0], Bm[..., 0],
                                    torch.ones(2, 6, 16, device=DEV)).shape == (0, 6)
    q, scale, _ = finc.add_norm_forward(x, torch.ones(40, device=DEV), fp8=True)
    assert q.shape == x.shape and scale.shape == (0, 6)


def test_the_binding_refuses():
    t, _, r = scan_inputs(2, 6, 40, 16, 2, "gsdbp", F32, 41)
    g, kw = scan_kw(t, None, "gsdbp", None)
    w = r.normal(6, 4).to(DEV)
    x = g["x"]

    def refused(text, call, *args, **more):
        with pytest.raises(ValueError, match=text):
            call(*args, **more)

    conv, scan = finc.causal_conv_forward, finc.selective_scan_forward
    refused("x must be float32, bfloat16 or float16", conv, x.double(), w)
    refused("x must be contiguous in its last", conv, x.transpose(1, 2), r.normal(40, 4).to(DEV))
    refused("w has shape", conv, x, w[:5])
    refused("w must be torch.float32", conv, x, w.bfloat16())
    refused("w must be on the device", conv, x, w.cpu())
    refused("w must be contiguous", conv, x, w.t().contiguous().t())
    refused("state has shape", conv, x, w, state=torch.zeros(2, 6, 4, device=DEV))
    refused("state must be", conv, x, w, state=torch.zeros(2, 6, 3, device=DEV, dtype=BF16))
    refused("lengths must be torch.int32", conv, x, w, lengths=torch.zeros(2, device=DEV))
    refused("out has shape", conv, x, w, out=x[:, :, 1:])
    refused("dy has shape", finc.causal_conv_backward, x, w, x[:1])
    refused("workspace holds", finc.causal_conv_backward, x, w, x,
            workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    refused("state has 1 entries for 2", finc.causal_conv_step, x[:, :, 0].contiguous(), w,
            torch.zeros(1, 6, 3, device=DEV))
    refused("dt must be", scan, **dict(g, dt=g["dt"].bfloat16()), **kw)
    refused("Cm has shape", scan, **dict(g, Cm=g["Cm"][:, :1]), **kw)
    refused("groups of a", scan, **dict(g, Bm=torch.zeros(2, 3, 16, 40, device=DEV)[:, ::2]), **kw)
    refused("D has shape", scan, **dict(g, D=w[0]), **kw)
    refused("state must be", scan, **g, **dict(kw, state=kw["state"].bfloat16()))
    refused("states holds", scan, **g, **kw, states=torch.empty(8, device=DEV))
    refused("slots must be", finc.selective_scan_step, x[:, :, 0].contiguous(),
            x[:, :, 0].contiguous(), g["A"], g["Bm"][..., 0].contiguous(),
            g["Cm"][..., 0].contiguous(), kw["state"], slots=torch.zeros(2, device=DEV))
    rows, nw = r.normal(8, 40).to(DEV), torch.ones(40, device=DEV)
    refused("expected 0 <= p", finc.dropout, rows, 1.0, 0)
    refused("expected 0 <= p", finc.dropout, rows, -0.5, 0)
    refused("seed must be", finc.dropout, rows, 0.5, -1)
    refused("offset must be", finc.dropout, rows, 0.5, 0, 1 << 64)
    refused("must lie evenly", finc.dropout, torch.zeros(4, 6, 5, 40, device=DEV)[:, :2, :3], 0.5, 0)
    refused("residual must be", finc.add_norm_forward, rows, nw, rows.bfloat16())
    refused("residual_out must be", finc.add_norm_forward, rows.bfloat16(), nw, rows.bfloat16(),
            residual_out=rows)
    refused("scale goes with fp8", finc.add_norm_forward, rows, nw,
            scale=torch.zeros(8, device=DEV))
    refused("out must be", finc.add_norm_forward, rows, nw, fp8=True, out=rows.bfloat16())
    refused("r must be", finc.add_norm_backward, rows, rows.half(), nw)
    refused("dr must be", finc.add_norm_backward, rows, rows, nw, rows.bfloat16())
    wide = torch.zeros(2, 16385, device=DEV)
    with pytest.raises(finc.FincError) as e:
        finc.add_norm_forward(wide, torch.zeros(16385, device=DEV))
    assert e.value.code == finc.EUNSUPPORTED


def test_offsets_past_31_bits():
    """Rows of one tensor of more than 2^31 elements."""
    D, L = 3, (1 << 30) - 8
    x = torch.zeros(1, D, L, dtype=BF16, device=DEV)
    x[0, 2, -5:] = 1
    w = torch.tensor([[1.0, 2.0]] * D, device=DEV)
    y = finc.causal_conv_forward(x, w)
    assert y[0, 2, -6:].tolist() == [0, 2, 3, 3, 3, 3] and not y[0, 0, -6:].any()
    del y
    rows = x.view(-1)[: (x.numel() // 1024) * 1024].view(-1, 1024)
    rows[-1] = 1
    nw = torch.ones(1024, device=DEV)
    out, _ = finc.add_norm_forward(rows[-40000:], nw)
    assert (out[-1] == 1).all() and not out[0].any()
    part = finc.dropout(rows, 0.0, 1)
    assert torch.equal(part[-1], rows[-1]) and not part[-3].any()
