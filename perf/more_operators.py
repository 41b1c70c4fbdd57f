"""The operators of a sequence model over pixels or codes, as cases to measure.

A prior over a raster of codes looks its rows up in a table, projects them,
mixes them along the raster and projects back.  A case is one pass through one
of these operators, for prompts and training or for a single token:

* attn_forward, attn_train (forward and gradients), attn_step: linear attention
  whose state S = e^a S + k v decays by a factor of its own at every head and
  position, y = scale q S;
* linear_forward, linear_backward: a projection act(x w^T + bias) + residual;
* embed_forward, embed_backward: rows of a table by their codes, scaled, and
  the table's gradient.

Positions are rows: q and k are (B, L, G, DK), v is (B, L, H, DV), with G
groups of heads that share q and k.  States are fp32, activations of the
case's type.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
KINDS = ("attn_forward", "attn_forward", "attn_train", "attn_train", "attn_step", "linear_forward",
         "linear_forward", "linear_backward", "embed_forward", "embed_backward")
CHUNK = 64


def listed():
    return [
        # one position of a single raster that is being sampled
        dict(name="attn_step_b1_h16_d128_bf16", op="attn_step", B=1, H=16, G=16, DK=128, DV=128,
             gate=True, type="bf16"),
        # one position of 64 rasters, eight heads to a query
        dict(name="attn_step_b64_h32_g4_d64_fp32", op="attn_step", B=64, H=32, G=4, DK=64, DV=64,
             gate=True, type="fp32"),
        # one long prompt, a raster of 128 x 128
        dict(name="attn_b1_h16_d128_128x128_bf16", op="attn_forward", B=1, L=16384, H=16, G=16,
             DK=128, DV=128, gate=False, ragged=False, state=False, type="bf16"),
        # prompts of odd and unequal lengths that go on from earlier states, odd heads
        dict(name="attn_b6_h12_g4_l1531_ragged_fp16", op="attn_forward", B=6, L=1531, H=12, G=4,
             DK=72, DV=100, gate=True, ragged=True, state=True, type="fp16"),
        # a training batch of 64 x 64 rasters: forward and all the gradients
        dict(name="attn_train_b4_h16_d128_64x64_bf16", op="attn_train", B=4, L=4096, H=16, G=16,
             DK=128, DV=128, gate=True, ragged=False, state=False, type="bf16"),
        # training on 64 latents of 16 x 16 positions
        dict(name="attn_train_b64_h8_d64_16x16_fp32", op="attn_train", B=64, L=256, H=8, G=8,
             DK=64, DV=64, gate=True, ragged=False, state=False, type="fp32"),
        # the projection back of one position of 64 rasters
        dict(name="linear_m64_k2048_n2048_bf16", op="linear_forward", M=64, K=2048, N=2048,
             act=None, bias=False, residual=True, keep=False, type="bf16"),
        # the projection of eight 64 x 64 rasters in training, which keeps what its gradient needs
        dict(name="linear_m32768_k1024_n4096_bf16", op="linear_forward", M=32768, K=1024, N=4096,
             act="silu", bias=True, residual=False, keep=True, type="bf16"),
        # all the gradients of a projection of four 64 x 64 rasters
        dict(name="linear_grad_m16384_c2048_bf16", op="linear_backward", M=16384, K=2048, N=2048,
             act="silu", bias=True, type="bf16"),
        # the same of odd sizes
        dict(name="linear_grad_m1531_k333_n1000_fp32", op="linear_backward", M=1531, K=333, N=1000,
             act="gelu", bias=True, type="fp32"),
        # the pixels of 64 images of 16 x 16 positions
        dict(name="embed_m16384_v256_c512_fp32", op="embed_forward", M=16384, V=256, D=512,
             wide=True, table="fp32", type="fp32"),
        # the table's gradient from eight 64 x 64 rasters of codes, some far more frequent
        dict(name="embed_grad_m32768_v16384_c1024_bf16", op="embed_backward", M=32768, V=16384,
             D=1024, wide=False, type="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(KINDS)
    kind = rng.choice(("fp32", "bf16", "bf16", "fp16"))
    case = dict(op=op, type=kind)
    if op.startswith("embed"):
        D = _log(rng, 16, 4096)
        case.update(M=_log(rng, 1, min(65536, (1 << 25) // D)),
                    V=_log(rng, 2, min(65536, (1 << 25) // D)), D=D,
                    wide=rng.choice((True, False)))
        if op == "embed_forward":
            case.update(table=rng.choice((kind, "fp32")))
        return case
    if op.startswith("linear"):
        most = (1 << 37) if op == "linear_forward" else (1 << 36)
        most = most >> 3 if kind == "fp32" else most
        K, N = _log(rng, 16, 4096), _log(rng, 16, 4096)
        case.update(M=_log(rng, 1, min(32768, most // (K * N))), K=K, N=N,
                    act=rng.choice((None, "relu", "silu", "gelu")), bias=rng.choice((True, False)))
        if op == "linear_forward":
            case.update(residual=rng.choice((True, False)), keep=rng.choice((True, False)))
        return case
    G = rng.choice((1, 2, 4, 8))
    H = G * rng.choice((1, 1, 1, 2, 4))
    DK, DV = (rng.choice((64, 128, 128, _log(rng, 8, 128))) for _ in range(2))
    case.update(H=H, G=G, DK=DK, DV=DV, gate=rng.choice((True, True, False)))
    if op == "attn_step":
        case.update(B=_log(rng, 1, 256))
        return case
    most = (1 << 32) // (DK * DV) // H
    L = _log(rng, 1, min(16384, most, (1 << 20) // H))
    case.update(B=_log(rng, 1, max(1, min(64, most // L, (1 << 20) // (H * L)))), L=L,
                ragged=rng.choice((True, False)), state=rng.choice((True, False)))
    return case


# ---- inputs ------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    T, f32 = TYPES[case["type"]], torch.float32

    def normal(*shape, scale=1.0, kind=T):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(kind)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    s, op = dict(case), case["op"]
    if op.startswith("embed"):
        M, V, D = case["M"], case["V"], case["D"]
        # codes whose frequencies fall off, and a few rows of padding
        ids = (uniform(M) ** 3 * V).long().clamp(max=V - 1)
        ids = torch.where(uniform(M) < 0.02, -1, torch.randperm(V, generator=g, device=DEV)[ids])
        s.update(ids=ids if case["wide"] else ids.to(torch.int32), scale=math.sqrt(D))
        if op == "embed_forward":
            s["table"] = normal(V, D, scale=0.02, kind=TYPES[case["table"]])
        else:
            s["dy"] = normal(M, D)
        return s
    if op.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        s.update(x=normal(M, K), w=normal(N, K, scale=K ** -0.5),
                 bias=normal(N, scale=0.1, kind=f32) if case["bias"] else None)
        if op == "linear_forward":
            s["res"] = normal(M, N) if case["residual"] else None
        else:
            s.update(dy=normal(M, N), pre=normal(M, N) if case["act"] else None)
        return s
    B, H, G, DK, DV = (case[k] for k in ("B", "H", "G", "DK", "DV"))
    n = 2 * G * DK + H * DV
    # windows from some eight to a thousand positions, and a part of the position's own
    s.update(decay=-torch.exp2(-3 - 7 * uniform(H)), scale=DK ** -0.5)
    rows = (B,) if op == "attn_step" else (B, case["L"])
    proj = normal(*rows, n)
    at = len(rows)
    s.update(q=proj[..., :G * DK].unflatten(at, (G, DK)),
             k=proj[..., G * DK:2 * G * DK].unflatten(at, (G, DK)),
             v=proj[..., 2 * G * DK:].unflatten(at, (H, DV)),
             g=(normal(*rows, H, kind=f32).exp() * -0.02).to(T) if case["gate"] else None)
    if op == "attn_step":
        S = B + B // 4 + 1
        s.update(state=normal(S, H, DK, DV, kind=f32),
                 slots=torch.randperm(S, generator=g, device=DEV)[:B].to(torch.int32))
        return s
    L = case["L"]
    s.update(state=normal(B, H, DK, DV, kind=f32) if case["state"] else None, lengths=None)
    if case["ragged"]:
        ends = (uniform(B) * (L + 1)).to(torch.int32)
        ends[0] = L
        if B > 1:
            ends[B - 1] = 0
        s["lengths"] = ends
    if op == "attn_train":
        s.update(dy=normal(B, L, H, DV),
                 dend=normal(B, H, DK, DV, kind=f32) if case["state"] else None)
    return s


# ---- the plain forms, in 32 bits ------------------------------------------------


def _log_decays(s, g):
    """(B, L, H) or (B, H) in 64 bits."""
    own_part = 0 if g is None else g.double()
    return s["decay"].double() + own_part + torch.zeros(*s["v"].shape[:-1], device=DEV,
                                                        dtype=torch.float64)


def _chunks(t):
    """(B, L, H, D) as (B, H, chunks, CHUNK, D), the last one filled with zeros."""
    t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, -t.shape[1] % CHUNK))
    return t.transpose(1, 2).unflatten(2, (-1, CHUNK)).contiguous()


def _attn(s, q, k, v, g, state):
    """(y, the state after) of fp32 q, k, v, the gradients' way through by torch's graph."""
    B, L, H, DV = v.shape
    share = H // s["G"]
    inside = torch.ones(1, L, dtype=torch.bool, device=DEV) if s["lengths"] is None else (
        torch.arange(L, device=DEV) < s["lengths"][:, None])
    a = torch.where(inside[..., None], _log_decays(s, g), 0.0)
    k = torch.where(inside[..., None, None], k, 0.0)
    q, k, v = _chunks(q.repeat_interleave(share, 2)), _chunks(k.repeat_interleave(share, 2)), _chunks(v)
    G = _chunks(a[..., None])[..., 0].cumsum(-1)                       # (B, H, chunks, CHUNK)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).tril()
    apart = (G[..., :, None] - G[..., None, :]).masked_fill(~lower, -math.inf)
    weights = torch.exp(apart).float() * (q @ k.transpose(-1, -2))
    ends = G[..., -1:]
    local = (k * torch.exp(ends - G).float()[..., None]).transpose(-1, -2).contiguous() @ v
    # the states before every chunk and after the last one
    E = torch.nn.functional.pad(ends[..., 0].cumsum(-1), (1, 0))        # (B, H, chunks + 1)
    before = torch.arange(E.shape[-1], device=DEV)[:, None] > torch.arange(E.shape[-1] - 1, device=DEV)
    carry = torch.exp((E[..., :, None] - E[..., None, 1:]).masked_fill(~before, -math.inf)).float()
    states = (carry @ local.flatten(3)).unflatten(3, local.shape[3:])
    if state is not None:
        states = states + torch.exp(E).float()[..., None, None] * state[:, :, None]
    y = weights @ v + torch.exp(G).float()[..., None] * (q @ states[:, :, :-1])
    y = (s["scale"] * y).flatten(2, 3)[:, :, :L].transpose(1, 2)
    return torch.where(inside[..., None, None], y, 0.0), states[:, :, -1]


def _attn_forward(s):
    y, end = _attn(s, s["q"].float(), s["k"].float(), s["v"].float(), s["g"], s["state"])
    return y.to(s["v"].dtype).contiguous(), end.contiguous()


def _attn_train(s):
    T, names = s["v"].dtype, ("q", "k", "v", "g", "state")
    leaves = {n: s[n].detach().float().requires_grad_() for n in names if s[n] is not None}
    y, end = _attn(s, *(leaves.get(n) for n in names))
    outs, grads = (y, end), (s["dy"].float(), s["dend"])
    if s["dend"] is None:
        outs, grads = outs[:1], grads[:1]
    found = dict(zip(leaves, torch.autograd.grad(outs, list(leaves.values()), grads)))
    d = {"d" + n: found[n].to(T) if n in found else None for n in names[:4]}
    return dict(d, y=y.detach().to(T), end=end.detach().contiguous(), dstate=found.get("state"))


def _attn_step(s):
    T, at, share = s["v"].dtype, s["slots"].long(), s["H"] // s["G"]
    q, k = (s[n].float().repeat_interleave(share, 1) for n in ("q", "k"))
    factor = torch.exp(_log_decays(s, s["g"])).float()
    S = factor[..., None, None] * s["state"][at] + k[..., None] * s["v"].float()[..., None, :]
    s["state"][at] = S
    return (s["scale"] * (q[..., None] * S).sum(2)).to(T), s["state"]


def _act(name, p):
    if name == "relu":
        return torch.clamp(p, min=0)
    if name == "silu":
        return p / (1 + torch.exp(-p))
    if name == "gelu":
        return p * 0.5 * (1 + torch.erf(p * math.sqrt(0.5)))
    return p


def _act_grad(name, p):
    if name == "relu":
        return (p > 0).float()
    if name == "silu":
        e = 1 / (1 + torch.exp(-p))
        return e * (1 + p * (1 - e))
    return 0.5 * (1 + torch.erf(p * math.sqrt(0.5))) + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)


def _linear_forward(s):
    T = s["x"].dtype
    p = s["x"].float() @ s["w"].float().T
    p = p if s["bias"] is None else p + s["bias"]
    y = _act(s["act"], p)
    y = y if s["res"] is None else y + s["res"].float()
    return y.to(T), p.to(T) if s["keep"] else None


def _linear_backward(s):
    T, d = s["x"].dtype, s["dy"].float()
    if s["act"]:
        d = d * _act_grad(s["act"], s["pre"].float())
    return ((d @ s["w"].float()).to(T), (d.T @ s["x"].float()).to(T),
            d.double().sum(0).float() if s["bias"] is not None else None)


def _embed_forward(s):
    ids = s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
    return torch.where(ids[:, None] >= 0, rows, 0.0).to(TYPES[s["type"]])


def _embed_backward(s):
    # the padding's rows go to one of their own, behind the table
    at = torch.where(s["ids"] < 0, s["V"], s["ids"].long())
    sums = torch.zeros(s["V"] + 1, s["D"], device=DEV).index_add_(0, at, s["dy"].float())
    return sums[:-1] * s["scale"]


_PLAIN = dict(attn_forward=_attn_forward, attn_train=_attn_train, attn_step=_attn_step,
              linear_forward=_linear_forward, linear_backward=_linear_backward,
              embed_forward=_embed_forward, embed_backward=_embed_backward)


# ---- the framework's calls ------------------------------------------------------


def _own(s):
    from paper_2301_09266_amd import finc

    op = s["op"]
    if op == "embed_forward":
        return finc.embed_forward(s["ids"], s["table"], scale=s["scale"], dtype=TYPES[s["type"]])
    if op == "embed_backward":
        return finc.embed_backward(s["ids"], s["dy"], s["V"], scale=s["scale"])
    if op == "linear_forward":
        pre = None
        if s["keep"]:
            pre = torch.empty(s["M"], s["N"], dtype=s["x"].dtype, device=DEV)
        y = finc.linear_forward(s["x"], s["w"], s["bias"], act=s["act"], residual=s["res"],
                                pre_out=pre)
        return y, pre
    if op == "linear_backward":
        return finc.linear_backward(s["dy"], s["x"], s["w"], s["pre"], act=s["act"],
                                    bias=s["bias"] is not None)
    args = (s["q"], s["k"], s["v"])
    more = dict(g=s["g"], decay=s["decay"], scale=s["scale"])
    if op == "attn_step":
        return finc.linear_attention_step(*args, s["state"], slots=s["slots"], **more), s["state"]
    B, L, H, DK, DV = (s[n] for n in ("B", "L", "H", "DK", "DV"))
    end, states = torch.empty(B, H, DK, DV, device=DEV), None
    more["lengths"] = s["lengths"]
    if op == "attn_train":
        states = finc.linear_attention_states(B, L, H, DK, DV, DEV)
    y = finc.linear_attention_forward(*args, state=s["state"], state_out=end, states=states, **more)
    if states is None:
        return y, end
    grads = finc.linear_attention_backward(*args, s["dy"], states, dstate_out=s["dend"], **more)
    if s["state"] is None:
        grads["dstate"] = None
    return dict(grads, y=y, end=end)


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------


def work(case):
    op = case["op"]
    e = 4 if case["type"] == "fp32" else 2
    if op.startswith("embed"):
        M, V, D = case["M"], case["V"], case["D"]
        ids = M * (8 if case["wide"] else 4)
        if op == "embed_backward":
            return {"bytes": ids + M * D * e + V * D * 4, "flops": 2 * M * D}
        rows = min(M, V) * D * (4 if case["table"] == "fp32" else 2)
        return {"bytes": ids + rows + M * D * e, "flops": M * D}
    if op.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        bias = 4 * N if case["bias"] else 0
        if op == "linear_forward":
            more = (2 if case["keep"] else 1) + (1 if case["residual"] else 0)
            return {"bytes": (M * K + N * K + more * M * N) * e + bias, "flops": 2 * M * N * K}
        # dy, x, w, pre -> dx, dw
        return {"bytes": (2 * (M * K + N * K) + (2 if case["act"] else 1) * M * N) * e + bias,
                "flops": 4 * M * N * K}
    B, H, G, DK, DV = (case[k] for k in ("B", "H", "G", "DK", "DV"))
    n = B * case.get("L", 1)
    reads = n * (2 * G * DK + H * DV + (H if case["gate"] else 0)) * e + 4 * H
    y, state = n * H * DV * e, B * H * DK * DV * 4
    if op == "attn_train":
        # the inputs again and dy, their gradients, the state's
        return {"bytes": 3 * reads + 2 * y + state * (4 if case["state"] else 1),
                "flops": 14 * n * H * DK * DV}
    both = op == "attn_step" or case["state"]
    return {"bytes": reads + y + state * (2 if both else 1), "flops": 4 * n * H * DK * DV}


# ---- the same in 64 bits, from the definitions --------------------------------------


def _exact_attn(s, train):
    """Every pair of positions of one head of one row after another."""
    B, L, H, DV = s["v"].shape
    per, names = H // s["G"], ("q", "k", "v", "g", "state")
    leaves = {n: s[n].detach().double() for n in names if s[n] is not None}
    found = {n: torch.zeros_like(t) for n, t in leaves.items()}
    y = torch.zeros(B, L, H, DV, dtype=torch.float64, device=DEV)
    end = torch.zeros(B, H, s["DK"], DV, dtype=torch.float64, device=DEV)
    pick = dict(q=lambda b, n, h: (b, slice(n), h // per), k=lambda b, n, h: (b, slice(n), h // per),
                v=lambda b, n, h: (b, slice(n), h), g=lambda b, n, h: (b, slice(n), h),
                state=lambda b, n, h: (b, h))
    ends = [L] * B if s["lengths"] is None else s["lengths"].tolist()
    for b, n in enumerate(ends):
        for h in range(H):
            at = {m: pick[m](b, n, h) for m in leaves}
            t = {m: leaves[m][at[m]].clone().requires_grad_(train) for m in leaves}
            a = torch.cumsum(s["decay"][h].double() + t["g"], 0) if "g" in t else (
                s["decay"][h].double() * torch.arange(1, n + 1, device=DEV))
            span = a[:, None] - a[None, :]
            far = torch.triu(torch.full((n, n), math.inf, device=DEV, dtype=torch.float64), 1)
            P = torch.mm(t["q"], t["k"].t().contiguous()) * torch.exp(span.clamp(max=80.0) - far)
            del span, far
            out = torch.mm(P, t["v"])
            left = torch.exp(a[-1] - a) if n else a
            after = torch.mm((t["k"] * left[:, None]).t().contiguous(), t["v"])
            if "state" in t:
                out = out + torch.exp(a)[:, None] * torch.mm(t["q"], t["state"])
                after = after + (torch.exp(a[-1]) if n else 1.0) * t["state"]
            out = s["scale"] * out
            y[b, :n, h], end[b, h] = out.detach(), after.detach()
            if train:
                loss = (out * s["dy"][b, :n, h].double()).sum()
                if s["dend"] is not None:
                    loss = loss + (after * s["dend"][b, h].double()).sum()
                if loss.requires_grad:
                    got = torch.autograd.grad(loss, list(t.values()), allow_unused=True)
                    for m, d in zip(t, got):
                        if d is not None:
                            found[m][at[m]] += d
    if not train:
        return y, end
    return dict({"d" + m: found.get(m) for m in names[:4]}, y=y, end=end, dstate=found.get("state"))


def _exact_step(s):
    per, at = s["H"] // s["G"], s["slots"].long()
    heads = torch.arange(s["H"], device=DEV) // per
    a = s["decay"].double().expand(s["B"], s["H"])
    if s["g"] is not None:
        a = a + s["g"].double()
    new = s["state"][at].double() * a.exp()[:, :, None, None]
    new += s["k"].double()[:, heads, :, None] * s["v"].double()[:, :, None, :]
    after = s["state"].double()
    after[at] = new
    return torch.matmul(s["q"].double()[:, heads, None, :], new)[:, :, 0] * s["scale"], after


def _exact_linear(s, op):
    functions = {None: lambda p: p, "relu": torch.relu, "silu": torch.nn.functional.silu,
                 "gelu": torch.nn.functional.gelu}
    f, x, w = functions[s["act"]], s["x"].double(), s["w"].double()
    if op == "linear_forward":
        p = torch.nn.functional.linear(x, w, None if s["bias"] is None else s["bias"].double())
        y = f(p)
        if s["res"] is not None:
            y = y + s["res"].double()
        return y, p if s["keep"] else None
    d = s["dy"].double()
    if s["act"]:
        p = s["pre"].double().requires_grad_()
        d, = torch.autograd.grad(f(p), p, d)
    return torch.mm(d, w), torch.mm(d.t().contiguous(), x), d.sum(0) if s["bias"] is not None else None


def _exact_embed(s, op):
    ids = s["ids"].long()
    some = torch.nonzero(ids >= 0)[:, 0]
    if op == "embed_forward":
        y = torch.zeros(s["M"], s["D"], dtype=torch.float64, device=DEV)
        y[some] = s["table"].double()[ids[some]] * s["scale"]
        return y
    # sums of runs of equal codes, as differences of the running sum over the sorted rows
    order = torch.argsort(ids[some], stable=True)
    rows = s["dy"].double()[some[order]]
    run_up = torch.cat([torch.zeros_like(s["dy"][:1], dtype=torch.float64), rows.cumsum(0)])
    edges = torch.searchsorted(ids[some[order]].contiguous(), torch.arange(s["V"] + 1, device=DEV))
    return (run_up[edges[1:]] - run_up[edges[:-1]]) * s["scale"]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op.startswith("embed"):
        return _exact_embed(s, op)
    if op.startswith("linear"):
        return _exact_linear(s, op)
    if op == "attn_step":
        return _exact_step(s)
    # pairs of positions, over all rows and heads: some 20 seconds' worth at most
    if case["B"] * case["H"] * case["L"] ** 2 * (3 if op == "attn_train" else 1) > 1 << 34:
        return None
    return _exact_attn(s, op == "attn_train")
