"""Linear attention through the binding against 64-bit references: types, odd heads,
shared heads, views, padding that holds NaN, states, empty rows, idle slots, decays that
clear the state, streams and graphs."""
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


def lengths_of(r, B, L):
    n = torch.randint(0, L + 1, (B,), generator=r, dtype=torch.int32)
    n[:1] = L
    if B > 1:
        n[-1] = 0
    if B > 2:
        n[1] = L + 7     # clamped
    if B > 3:
        n[2] = -3
    return n


def inputs(B, L, H, G, DK, DV, opt, kind, seed=0):
    """q, k, v, g, decay, state, lengths, dy, dend on the CPU (None without their letter)."""
    r = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=r, dtype=torch.float64)  # noqa: E731
    t = dict(q=normal(B, L, G, DK).to(kind), k=(normal(B, L, G, DK) * DK ** -0.5).to(kind),
             v=normal(B, L, H, DV).to(kind),
             g=(-normal(B, L, H).exp() * 0.05).to(kind) if "g" in opt else None,
             decay=-torch.exp2(-1 - 6 * torch.rand(H, generator=r)) if "d" in opt else None,
             state=normal(B, H, DK, DV).float() if "s" in opt else None,
             lengths=lengths_of(r, B, L) if "l" in opt else None,
             dy=normal(B, L, H, DV).to(kind), dend=normal(B, H, DK, DV).float())
    return t


def poison(t, lengths):
    if t is None or lengths is None:
        return t
    t = t.clone()
    for b, n in enumerate(ref.ends(lengths, t.shape[0], t.shape[1])):
        t[b, n:] = NAN
        t[b, n + 1::3] = torch.finfo(t.dtype).min
        t[b, n + 2::3] = INF
    return t


def place(t, view):
    """On the device, "rows": beside NaN in rows of twice the width and an odd address;
    "heads": the heads outside the positions."""
    if t is None or view is None:
        return None if t is None else t.to(DEV)
    if view == "heads":
        return t.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)
    flat = t.flatten(2)
    big = torch.full((*t.shape[:2], 2 * flat.shape[2] + 1), NAN, dtype=t.dtype, device=DEV)
    big[..., 1:1 + flat.shape[2]] = flat.to(DEV)
    return big[..., 1:1 + flat.shape[2]].unflatten(2, t.shape[2:])


def run(t, kind, view=None, scale=0.3, train=True):
    """(y, state after, gradients) of the device and of the reference."""
    n = t["lengths"]
    names = ("q", "k", "v", "g")
    x = {m: place(poison(t[m], n), view) for m in names}
    p = {m: None if t[m] is None else t[m].to(DEV) for m in ("decay", "state", "lengths")}
    B, L, H, DV = t["v"].shape
    DK = t["q"].shape[3]
    keep = finc.linear_attention_states(B, L, H, DK, DV, DEV)
    keep.fill_(NAN)
    end = torch.full((B, H, DK, DV), NAN, device=DEV)
    out = place(torch.full_like(t["v"], NAN), view)
    kw = dict(g=x["g"], decay=p["decay"], scale=scale, lengths=p["lengths"])
    y = finc.linear_attention_forward(x["q"], x["k"], x["v"], state=p["state"], state_out=end,
                                      states=keep, out=out, **kw)
    got = dict(y=y, end=end)
    leaves = {m: t[m].double().requires_grad_(train) for m in (*names, "state")
              if t[m] is not None}
    decay = None if t["decay"] is None else t["decay"].double()
    ry, rend = rows.attention(leaves["q"], leaves["k"], leaves["v"], leaves.get("g"), decay, scale,
                              leaves.get("state"), n)
    want = dict(y=ry, end=rend)
    if train:
        dy = place(poison(t["dy"], n), view)
        got.update(finc.linear_attention_backward(x["q"], x["k"], x["v"], dy, keep,
                                                  dstate_out=t["dend"].to(DEV), **kw))
        loss = (ry * t["dy"].double()).sum() + (rend * t["dend"].double()).sum()
        loss = loss + sum(0 * leaf.sum() for leaf in leaves.values())   # of an empty batch
        d = torch.autograd.grad(loss, list(leaves.values()), allow_unused=True)
        for m, v in zip(leaves, d):
            want["d" + m] = torch.zeros_like(leaves[m]) if v is None else v
    return got, want


def check(got, want, kind, t):
    for m, w in want.items():
        if m != "dg":
            rows.close(got[m], w, m, kind)
            continue
        # a sum over the part behind a position of products that mostly cancel: the bar
        # goes by their size
        x = (t["q"].double() * want["dq"]).sum(-1)
        if x.numel() == 0:
            continue
        size = float(x.square().mean().sqrt()) + float(
            (t["k"].double() * want["dk"]).sum(-1).square().mean().sqrt())
        S = want["end"].detach()
        size += float((S * t["dend"].double()).sum((-1, -2)).square().mean().sqrt())
        L = w.shape[1]
        bar = ref.U[kind] * 1.01 * w.abs() + ref.TINY[kind] + rows.CHAIN[kind] * 2.0 ** -24 * (
            size * math.sqrt(min(L, 512)) + w.abs())
        off = (got[m].double().cpu() - w).abs()
        assert bool((off <= bar).all()), (m, float((off / bar).max()))


CASES = [  # B, L, H, G, DK, DV, options, type, view
    (1, 1, 1, 1, 1, 1, "", F32, None),
    (1, 1, 1, 1, 1, 1, "gds", BF16, None),
    (2, 2, 2, 1, 3, 5, "gdsl", F16, "rows"),
    (2, 63, 1, 1, 16, 16, "d", F32, None),
    (1, 64, 2, 2, 64, 64, "gds", BF16, None),
    (4, 65, 2, 2, 33, 65, "gdsl", F32, "rows"),
    (3, 130, 4, 2, 100, 72, "gdsl", BF16, "rows"),
    (2, 100, 3, 3, 128, 128, "gs", F32, "heads"),
    (2, 200, 2, 2, 128, 128, "gdsl", BF16, None),
    (2, 150, 2, 1, 127, 128, "dsl", F16, "heads"),
    (1, 512, 1, 1, 17, 40, "gd", F32, None),
    (2, 513, 2, 2, 64, 32, "gdsl", F32, "rows"),
    (5, 700, 2, 1, 24, 64, "gdsl", BF16, "heads"),
    (1, 1100, 2, 2, 128, 128, "gds", BF16, None),
    (2, 1030, 1, 1, 72, 100, "gsl", F16, "rows"),
    (3, 1025, 2, 2, 40, 9, "sl", F32, None),
    (2, 200, 2, 2, 128, 64, "gds", BF16, None),
    (2, 300, 4, 2, 64, 128, "gdsl", F16, None),
    (2, 600, 2, 2, 128, 64, "gdl", F16, None),
    (3, 130, 2, 1, 40, 100, "gdsl", BF16, "rows"),
    (1, 560, 2, 2, 64, 128, "gds", F32, "heads"),
    (2, 140, 3, 3, 101, 61, "gdsl", F32, "rows"),
    (2, 700, 2, 2, 128, 128, "gds", F16, None),
    (0, 5, 2, 1, 8, 8, "gdsl", BF16, None),
    (3, 0, 2, 1, 8, 12, "gdsl", F32, None),
]


@pytest.mark.parametrize("B,L,H,G,DK,DV,opt,kind,view", CASES)
def test_forward_and_gradients(B, L, H, G, DK, DV, opt, kind, view):
    t = inputs(B, L, H, G, DK, DV, opt, kind, seed=L + DK)
    got, want = run(t, kind, view)
    check(got, want, kind, t)


@pytest.mark.parametrize("L,D", [(200, 128), (600, 64)])
def test_fp16_columns_of_all_sizes(L, D):
    """Values that differ by 2^30 from column to column and from block to block, columns of
    zeros, states far above fp16's range, an empty column that fills later."""
    t = inputs(2, L, 2, 2, D, D, "gds", F16, seed=D)
    size = torch.exp2(torch.randint(-12, 13, (2, 1, 2, D), generator=torch.Generator().manual_seed(1)))
    t["v"] = (t["v"].double() * size).to(F16)
    t["v"][:, 64:128] *= 2.0 ** -10
    t["v"][:, :, :, 3] = 0
    t["v"][:, : L // 2, :, 5] = 0
    t["state"][:, :, :, 1] *= 2.0 ** 60
    t["state"][:, :, :, 2:6] = 0
    t["state"][:, :, :, 6] *= 2.0 ** -90
    t["g"][:, 130] = -3.0
    got, want = run(t, F16, train=False)
    # column by column: each has its own size
    for d in range(D):
        y, end = want["y"][..., d], want["end"][..., d]
        if d == 1:      # past fp16's largest value from the start on
            assert not torch.isfinite(got["y"][:, 0, :, 1]).any()
        else:
            rows.close(got["y"][..., d], y, f"y {d}", F16)
        rows.close(got["end"][..., d], end, f"end {d}", F16)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("L", [70, 600])
def test_decays_that_clear_and_that_keep(kind, L):
    """Log decays of minus infinity and of the type's lowest value clear the state, 0
    keeps all of it, and strong ones leave hardly anything of the position before."""
    t = inputs(1, L, 3, 3, 16, 16, "gs", kind, seed=3)
    t["g"][:, :, 0] = 0
    t["g"][:, 5::37, 1] = -INF
    t["g"][:, 11::50, 1] = torch.finfo(kind).min
    t["g"][:, :, 2] = -9.0
    got, want = run(t, kind)
    check(got, want, kind, t)
    x = dict(t, state=t["state"] * 0 + 7)
    other, _ = run(x, kind, train=False)
    assert torch.equal(other["y"][:, 5:, 1], got["y"][:, 5:, 1])


def test_constant_decays_are_repeated_ones():
    """g with steps of 0 over positions and batch is the decay itself."""
    t = inputs(2, 300, 4, 2, 32, 32, "ds", F32, seed=4)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    one = finc.linear_attention_forward(d["q"], d["k"], d["v"], decay=d["decay"], state=d["state"])
    g = d["decay"].expand(2, 300, 4)
    assert torch.equal(one, finc.linear_attention_forward(d["q"], d["k"], d["v"], g=g,
                                                          state=d["state"]))
    # and a gate of one head, as a column of a projection
    wide = torch.full((2, 300, 9), NAN, device=DEV)
    wide[..., 2:6] = d["decay"]
    assert torch.equal(one, finc.linear_attention_forward(d["q"], d["k"], d["v"],
                                                          g=wide[..., 2:6], state=d["state"]))


@pytest.mark.parametrize("L,kind", [(100, BF16), (600, F32), (1100, F16)])
def test_pieces_are_the_whole(L, kind):
    """A row in two calls, the state handed on in place."""
    t = inputs(2, L, 2, 2, 48, 40, "gds", kind, seed=5)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    _, want = run(t, kind, train=False)
    state, at, out = d["state"].clone(), 0, []
    for n in (L // 3, 1, L - L // 3 - 1):
        p = {m: d[m][:, at:at + n] for m in "qkvg"}
        out.append(finc.linear_attention_forward(p["q"], p["k"], p["v"], g=p["g"],
                                                 decay=d["decay"], scale=0.3, state=state,
                                                 state_out=state))
        at += n
    rows.close(torch.cat(out, 1), want["y"], "y", kind)
    rows.close(state, want["end"], "state", kind)


@pytest.mark.parametrize("H,G,DK,DV,kind", [(1, 1, 1, 1, F32), (4, 2, 64, 64, BF16),
                                            (3, 3, 127, 33, F16), (2, 1, 128, 128, F32),
                                            (6, 2, 20, 101, BF16)])
def test_steps_are_the_forward(H, G, DK, DV, kind):
    """Single positions through slots in another order, an idle row beside them, views."""
    B, L, S = 3, 6, 5
    t = inputs(B, L, H, G, DK, DV, "gds", kind, seed=DK)
    _, want = run(t, kind, train=False)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    cache = torch.full((S, H, DK, DV), 3.0, device=DEV)
    slots = torch.tensor([4, 0, 2, -1, 5], dtype=torch.int32, device=DEV)
    cache[slots[:B].long()] = d["state"]
    pad = lambda x: torch.cat([x, torch.full_like(x[:2], NAN)])  # noqa: E731
    for i in range(L):
        y = torch.full((B + 2, 2, H, DV + 3), NAN, dtype=kind, device=DEV)[:, 1, :, :DV]
        got = finc.linear_attention_step(pad(d["q"][:, i]), pad(d["k"][:, i]), pad(d["v"][:, i]),
                                         cache, g=pad(d["g"][:, i]), decay=d["decay"], scale=0.3,
                                         slots=slots, out=y)
        rows.close(got[:B], want["y"][:, i], f"y {i}", F32)
        assert bool((got[B:] == 0).all())
    rows.close(cache[slots[:B].long()], want["end"], "state", F32)
    assert bool((cache[[1, 3]] == 3).all())


def test_steps_without_slots_and_with_more_entries():
    t = inputs(2, 1, 2, 1, 8, 8, "s", F32, seed=9)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    cache = torch.cat([d["state"], torch.full_like(d["state"], 5.0)])
    y = finc.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], cache, scale=0.3)
    _, want = run(t, F32, train=False)
    rows.close(y, want["y"][:, 0], "y", F32)
    rows.close(cache[:2], want["end"], "state", F32)
    assert bool((cache[2:] == 5).all())


@pytest.mark.parametrize("L", [90, 600])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_rows_do_not_depend_on_the_batch(L, kind):
    """Bits of a row and of its gradients alone and beside others."""
    t = inputs(5, L, 4, 2, 64, 72, "gds", kind, seed=7)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}

    def both(rows_):
        x = {m: v if v is None or m == "decay" else v[rows_] for m, v in d.items()}
        B = x["q"].shape[0]
        keep = finc.linear_attention_states(B, L, 4, 64, 72, DEV)
        end = torch.empty(B, 4, 64, 72, device=DEV)
        kw = dict(g=x["g"], decay=x["decay"], scale=0.3)
        y = finc.linear_attention_forward(x["q"], x["k"], x["v"], state=x["state"], states=keep,
                                          state_out=end, **kw)
        o = finc.linear_attention_backward(x["q"], x["k"], x["v"], x["dy"], keep, **kw)
        return [y, end, *o.values()]

    whole, alone = both(slice(0, 5)), both(slice(3, 4))
    for a, b in zip(whole, alone):
        assert torch.equal(a[3:4], b)
    # and without kept states
    y = finc.linear_attention_forward(d["q"], d["k"], d["v"], g=d["g"], decay=d["decay"], scale=0.3,
                                      state=d["state"])
    assert torch.equal(y, whole[0])


@pytest.mark.parametrize("L", [100, 640])
@pytest.mark.parametrize("what", [NAN, INF])
@pytest.mark.parametrize("name", ["q", "k", "v", "g"])
def test_what_is_not_finite_stays_in_its_row_and_heads(L, what, name):
    """From its block of 64 positions on forward, up to that block's end in the
    gradients' order; other rows and heads keep their bits."""
    t = inputs(3, L, 4, 2, 16, 16, "gd", F32, seed=8)
    at = 70
    clean, _ = run(t, F32)
    t[name][1, at, 1] = what     # heads 2 and 3 of the groups, or head 1
    bad, _ = run(t, F32)
    heads = [1] if name in "vg" else [2, 3]
    for m in ("y", "dq", "dk", "dv", "dg", "end", "dstate"):
        a, b = clean.get(m), bad.get(m)
        if a is None:
            continue
        keep = torch.ones_like(a, dtype=torch.bool)
        if m in ("end", "dstate"):
            keep[1, heads] = False
        elif m in ("dq", "dk"):
            keep[1, :, sorted({h // 2 for h in heads})] = False
        else:
            keep[1, :, heads] = False
        assert torch.equal(a[keep], b[keep]), m
    assert torch.equal(clean["y"][1, :64], bad["y"][1, :64])


def test_large_values_of_fp16():
    """Scores, weights and states past fp16's range, and inputs at its ends."""
    t = inputs(1, 130, 2, 2, 64, 64, "d", F16, seed=10)
    t["q"] *= 300
    t["k"] *= 2000
    t["v"] *= 1e-5
    got, want = run(t, F16, scale=0.01)
    check(got, want, F16, t)


def test_gradients_are_the_differences():
    """Central differences of the fp32 call in some directions."""
    L, kw = 90, dict(scale=0.5)
    t = inputs(1, L, 2, 1, 8, 8, "gds", F32, seed=11)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    keep = finc.linear_attention_states(1, L, 2, 8, 8, DEV)
    r = torch.Generator().manual_seed(1)

    def loss(x):
        end = torch.empty(1, 2, 8, 8, device=DEV)
        y = finc.linear_attention_forward(x["q"], x["k"], x["v"], g=x["g"], decay=x["decay"],
                                          state=x["state"], state_out=end, states=keep, **kw)
        return float((y.double() * d["dy"].double()).sum()
                     + (end.double() * d["dend"].double()).sum())

    loss(d)
    o = finc.linear_attention_backward(d["q"], d["k"], d["v"], d["dy"], keep, g=d["g"],
                                       decay=d["decay"], dstate_out=d["dend"], **kw)
    for m in ("q", "k", "v", "g", "state"):
        u = torch.randn(d[m].shape, generator=r).to(DEV)
        h = 2.0 ** -7 * float(d[m].abs().max())
        up, down = (loss(dict(d, **{m: d[m] + s * h * u})) for s in (1, -1))
        want = float((o["d" + m].double() * u.double()).sum())
        # the third derivative's share (h^2) and the fp32 sums' rounding over h
        size = float((o["d" + m].double().square().sum()).sqrt())
        assert abs((up - down) / (2 * h) - want) <= 2e-2 * size, m


def test_gradients_beside_each_other():
    """dq, dk and dv as parts of one projection's gradient."""
    B, L, H, D = 2, 70, 2, 16
    t = inputs(B, L, H, H, D, D, "g", BF16, seed=12)
    got, want = run(t, BF16)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    keep = finc.linear_attention_states(B, L, H, D, D, DEV)
    finc.linear_attention_forward(d["q"], d["k"], d["v"], g=d["g"], scale=0.3, states=keep)
    whole = torch.full((B, L, 3, H, D), NAN, dtype=BF16, device=DEV)
    o = finc.linear_attention_backward(d["q"], d["k"], d["v"], d["dy"], keep, g=d["g"], scale=0.3,
                                       dstate_out=d["dend"], dq=whole[:, :, 0],
                                       dk=whole[:, :, 1], dv=whole[:, :, 2])
    for i, m in enumerate(("dq", "dk", "dv")):
        assert torch.equal(whole[:, :, i], got[m]) and torch.equal(o[m], got[m])


def test_shared_rows_of_a_batch():
    """Inputs that are one row for the whole batch (steps of 0)."""
    t = inputs(1, 80, 2, 2, 24, 24, "gd", F32, seed=13)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}
    x = {m: d[m].expand(3, *d[m].shape[1:]) for m in "qkvg"}
    y = finc.linear_attention_forward(x["q"], x["k"], x["v"], g=x["g"], decay=d["decay"])
    one = finc.linear_attention_forward(d["q"], d["k"], d["v"], g=d["g"], decay=d["decay"])
    assert torch.equal(y, one.expand_as(y))


def everything(L):
    t = inputs(2, L, 4, 2, 40, 48, "gdsl", BF16, seed=14)
    d = {m: None if v is None else v.to(DEV) for m, v in t.items()}

    def call():
        state = d["state"].clone()
        keep = finc.linear_attention_states(2, L, 4, 40, 48, DEV)
        kw = dict(g=d["g"], decay=d["decay"], lengths=d["lengths"])
        y = finc.linear_attention_forward(d["q"], d["k"], d["v"], state=state, state_out=state,
                                          states=keep, **kw)
        o = finc.linear_attention_backward(d["q"], d["k"], d["v"], d["dy"], keep,
                                           dstate_out=d["dend"], **kw)
        s = finc.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], state,
                                       g=d["g"][:, 0], decay=d["decay"])
        return [y, state, s, *o.values()]

    return call


@pytest.mark.parametrize("L", [100, 600])
def test_graphs_replay_the_calls(L):
    call = everything(L)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
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


def test_calls_run_on_the_current_stream():
    call = everything(600)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_offsets_past_31_bits():
    """Rows and cache entries that lie more than 2^31 elements apart."""
    t = inputs(2, 70, 1, 1, 16, 16, "g", BF16, seed=15)
    far = torch.zeros((1 << 31) + 70 * 64 + 64, dtype=BF16, device=DEV)
    step = 1 << 31
    views = {}
    for i, m in enumerate("qkv"):
        views[m] = far.as_strided((2, 70, 1, 16), (step, 64, 16, 1), 16 * i)
        views[m].copy_(t[m].to(DEV))
    out = far.as_strided((2, 70, 1, 16), (step, 64, 16, 1), 48)
    finc.linear_attention_forward(views["q"], views["k"], views["v"], g=t["g"].to(DEV), scale=0.3,
                                  out=out)
    _, want = run(t, BF16, train=False)
    rows.close(out, want["y"], "y", BF16)
    del far
    S, H, D = 140000, 1, 128
    cache = torch.zeros(S, H, D, D, device=DEV)
    one = torch.ones(1, 1, D, dtype=BF16, device=DEV)
    slot = torch.tensor([S - 1], dtype=torch.int32, device=DEV)
    y = finc.linear_attention_step(one, one, one, cache, slots=slot)
    assert bool((y == D).all()) and bool((cache[S - 1] == 1).all())
    assert float(cache[:S - 1].abs().max()) == 0.0


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("L", [40, 600])
def test_an_empty_rows_state_goes_on_as_it_is(kind, L):
    """All of fp32's range beside each other in a column, and what is not finite."""
    t = inputs(2, L, 1, 1, 16, 16, "gs", kind, seed=21)
    state = t["state"].to(DEV)
    state[0, 0, 0] = 2.0 ** 100
    state[0, 0, 1] = 2.0 ** -100
    state[0, 0, 2, 3] = INF
    state[0, 0, 4, 5] = NAN
    end = torch.empty_like(state)
    n = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    y = finc.linear_attention_forward(
        t["q"].to(DEV), t["k"].to(DEV), t["v"].to(DEV), g=t["g"].to(DEV), state=state,
        lengths=n, states=finc.linear_attention_states(2, L, 1, 16, 16, DEV), state_out=end)
    assert torch.equal(end[0].view(torch.int32), state[0].view(torch.int32))
    assert not y[0].any() and not y[1, 1:].any() and torch.isfinite(y[1]).all()


def test_more_workgroups_than_a_row_of_the_grid():
    """Launches past 2^21 workgroups lie in rows of the grid, the last one partly without
    work: parts, their join and the decays' gradient; single positions.  All rows are the
    same, and so are their bits."""
    B, L = (1 << 21) + 5, 513
    x = [torch.randn(1, L, 1, 1, dtype=BF16, device=DEV).expand(B, L, 1, 1) for _ in range(4)]
    g = -x[3][..., 0].exp() * 0.05
    few = [t[:2].contiguous() for t in (*x, g)]

    def run(q, k, v, dy, g):
        n = q.shape[0]
        states = finc.linear_attention_states(n, L, 1, 1, 1, DEV)
        guard = torch.full((n + 64,), 7.0, device=DEV)
        end = guard[:n].view(n, 1, 1, 1)
        y = finc.linear_attention_forward(q, k, v, g=g, states=states, state_out=end)
        assert bool((guard[n:] == 7.0).all())
        o = finc.linear_attention_backward(q, k, v, dy, states, g=g)
        return y, end, o["dq"], o["dk"], o["dv"], o["dg"]

    want = run(*few)
    for t, w in zip(run(*x, g), want):
        assert bool((t == w[:1]).all())
    del t
    B, H, D = (1 << 19) + 3, 1, 128
    guard = torch.zeros((B + 8) * H * D, device=DEV)
    cache = guard[:B * D].view(B, H, 1, D)
    slots = torch.arange(B + 4096, dtype=torch.int32, device=DEV).clamp_(max=B)[:B].contiguous()
    one = torch.ones(1, 1, 1, dtype=BF16, device=DEV).expand(B, 1, 1)
    v = torch.ones(1, 1, D, dtype=BF16, device=DEV).expand(B, 1, D)
    y = finc.linear_attention_step(one, one, v, cache, slots=slots)
    assert bool((y == 1).all()) and bool((cache == 1).all()) and not guard[B * D:].any()


def test_the_binding_refuses():
    x = torch.zeros(2, 8, 2, 16, device=DEV)
    S = torch.zeros(2, 2, 16, 16, device=DEV)
    f = finc.linear_attention_forward
    keep = finc.linear_attention_states(2, 8, 2, 16, 16, DEV)
    bad = [
        (dict(q=x[0]), "expected \\(B, L, G, DK\\)"), (dict(v=x[..., 0]), "expected \\(B, L, H, DV\\)"),
        (dict(k=x[:, :4]), "k has shape"), (dict(v=x[:1]), "v has shape"),
        (dict(q=x.double()), "must be float32"), (dict(k=x.bfloat16()), "k must be"),
        (dict(v=x.bfloat16()), "v must be"), (dict(q=x.cpu()), "device tensor"),
        (dict(q=x.transpose(2, 3)), "16 groups|contiguous"),
        (dict(g=x[..., 0].bfloat16()), "g must be"), (dict(g=x[:1, :, :, 0]), "g has shape"),
        (dict(decay=torch.zeros(3, device=DEV)), "decay has shape"),
        (dict(state=S[:1]), "state has shape"), (dict(state=S.bfloat16()), "state must be"),
        (dict(state_out=S.transpose(2, 3)), "contiguous"),
        (dict(lengths=torch.zeros(2, device=DEV)), "lengths must be"),
        (dict(out=x[:1]), "out has shape"), (dict(states=keep[:100]), "bytes|small|states"),
    ]
    for change, what in bad:
        a = dict(q=x, k=x, v=x)
        a.update(change)
        with pytest.raises(ValueError, match=what):
            f(a.pop("q"), a.pop("k"), a.pop("v"), **a)
    with pytest.raises(ValueError, match="129"):
        wide = torch.zeros(1, 1, 1, 129, device=DEV)
        f(wide, wide, wide)
    with pytest.raises(ValueError, match="2 groups do not divide 3"):
        f(x, x, torch.zeros(2, 8, 3, 16, device=DEV))
    with pytest.raises(finc.FincError):
        f(x, x, x, out=x)
    with pytest.raises(finc.FincError):
        f(x, x, x, out=torch.zeros(1, 8, 2, 16, device=DEV).expand(2, 8, 2, 16))
    with pytest.raises(ValueError, match="1 entries for 2 rows"):
        finc.linear_attention_step(x[:, 0], x[:, 0], x[:, 0], S[:1])
