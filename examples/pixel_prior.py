"""An autoregressive prior over quantised pixels, in raster order.

Codes of pixels are looked up in a table beside their position's, and go through blocks of

    x += W_out attention(q, k, v; decay, g),   q, k, v, gate = W_in norm(x);
    x += W_down silu(W_up norm(x) + b)

with linear attention, whose state decays by a factor of its own at every head (a constant)
and position (the gate).  A last norm and projection give the next code's logits.  Training
runs over whole rasters; sampling one position at a time from the blocks' carried states.

    python examples/pixel_prior.py [--steps 200] [--batch 32] [--bf16]

prints the negative log-likelihood (bits a pixel) as it falls, and the agreement of the two
ways to run the model.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2301_09266_amd import finc  # noqa: E402

DEV = "cuda:0"
EPS = 1e-5


# ---- the operators under autograd ---------------------------------------------------


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale, dtype):
        ctx.save_for_backward(ids)
        ctx.rows, ctx.scale = table.shape[0], scale
        return finc.embed_forward(ids, table, scale=scale, dtype=dtype)

    @staticmethod
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        return None, finc.embed_backward(ids, dy.contiguous(), ctx.rows, scale=ctx.scale), None, None


class Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, act):
        pre = None if act is None else x.new_empty(*x.shape[:-1], w.shape[0])
        y = finc.linear_forward(x, w, bias, act=act, residual=residual, pre_out=pre)
        ctx.save_for_backward(x, w, pre)
        ctx.act, ctx.bias, ctx.residual = act, bias is not None, residual is not None
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, pre = ctx.saved_tensors
        dy = dy.contiguous()
        dx, dw, db = finc.linear_backward(dy, x, w, pre, act=ctx.act, bias=ctx.bias)
        return dx, dw, db, dy if ctx.residual else None, None


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, decay, scale):
        B, L, H, DV = v.shape
        states = finc.linear_attention_states(B, L, H, q.shape[3], DV, q.device)
        ctx.save_for_backward(q, k, v, g, decay, states)
        ctx.scale = scale
        return finc.linear_attention_forward(q, k, v, g=g, decay=decay, scale=scale, states=states)

    @staticmethod
    def backward(ctx, dy):
        q, k, v, g, decay, states = ctx.saved_tensors
        o = finc.linear_attention_backward(q, k, v, dy.contiguous(), states, g=g, decay=decay,
                                           scale=ctx.scale)
        return o["dq"], o["dk"], o["dv"], o["dg"], None, None


class AddNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        y, r = finc.add_norm_forward(x, w, eps=EPS)
        ctx.save_for_backward(r, w)
        return y

    @staticmethod
    def backward(ctx, dy):
        r, w = ctx.saved_tensors
        dx, _, dw = finc.add_norm_backward(dy.contiguous(), r, w, eps=EPS)
        return dx, dw


# ---- the model ------------------------------------------------------------------------


class Prior:
    """Of rasters of L codes below V; the code before the first position is V."""

    def __init__(self, V, L, width=64, blocks=2, heads=4, head=16, dtype=torch.float32, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.V, self.L, self.D, self.H, self.E, self.T = V, L, width, heads, head, dtype
        self.inner = heads * head

        def normal(*shape, scale, kind=dtype):
            return (torch.randn(*shape, generator=gen) * scale).to(DEV, kind).requires_grad_()

        def const(value, *shape):
            return torch.full(shape, value, device=DEV, requires_grad=True)

        fan = width ** -0.5
        self.codes = normal(V + 1, width, scale=0.02, kind=torch.float32)
        self.places = normal(L, width, scale=0.02, kind=torch.float32)
        # windows from some four to 256 positions
        self.decay = -torch.exp2(-torch.linspace(2, 8, heads)).to(DEV)
        self.blocks = [dict(
            norm=const(1.0, width), w_in=normal(3 * self.inner + heads, width, scale=fan),
            w_out=normal(width, self.inner, scale=0.5 * self.inner ** -0.5),
            norm2=const(1.0, width), w_up=normal(4 * width, width, scale=fan),
            b_up=const(0.0, 4 * width), w_down=normal(width, 4 * width, scale=0.25 * fan),
        ) for _ in range(blocks)]
        self.norm = const(1.0, width)
        self.head_w = normal(V, width, scale=0.02)

    def parameters(self):
        return [self.codes, self.places, self.norm, self.head_w] + \
            [p for b in self.blocks for p in b.values()]

    def split(self, mixed):
        """q, k, v (..., H, E) and the log gate (..., H) of a projection's rows."""
        n, at = self.inner, mixed.dim() - 1
        heads = [mixed[..., i * n:(i + 1) * n].unflatten(at, (self.H, self.E)) for i in range(3)]
        return (*heads, -torch.nn.functional.softplus(mixed[..., 3 * n:] - 4.0))

    def look_up(self, before, places):
        """Rows of the codes before, beside their position's."""
        scale = math.sqrt(self.D)
        return Embed.apply(before, self.codes, scale, self.T) + \
            Embed.apply(places, self.places, scale, self.T)

    def forward(self, codes):
        """Logits (B, L, V) of every position of codes (B, L)."""
        B, L = codes.shape
        before = torch.cat([torch.full_like(codes[:, :1], self.V), codes[:, :-1]], dim=1)
        x = self.look_up(before, torch.arange(L, device=DEV).expand(B, L).contiguous())
        for b in self.blocks:
            q, k, v, g = self.split(Linear.apply(AddNorm.apply(x, b["norm"]), b["w_in"], None, None,
                                                 None))
            y = Attention.apply(q, k, v, g, self.decay, self.E ** -0.5)
            x = Linear.apply(y.flatten(2), b["w_out"], None, x, None)
            y = Linear.apply(AddNorm.apply(x, b["norm2"]), b["w_up"], b["b_up"], None, "silu")
            x = Linear.apply(y, b["w_down"], None, x, None)
        return Linear.apply(AddNorm.apply(x, self.norm), self.head_w, None, None, None)

    def bits(self, codes):
        """Bits a pixel."""
        logits = self.forward(codes).float()
        return torch.nn.functional.cross_entropy(logits.flatten(0, 1), codes.flatten()) / math.log(2)

    # ---- one position at a time --------------------------------------------------------

    def start(self, entries):
        """Zero states of `entries` rasters, entry by entry."""
        return [torch.zeros(entries, self.H, self.E, self.E, device=DEV) for _ in self.blocks]

    @torch.no_grad()
    def step(self, before, place, cache, slots=None):
        """Logits (B, V) of position `place` after the codes `before` (B)."""
        x = self.look_up(before, torch.full_like(before, place))
        for b, state in zip(self.blocks, cache):
            y, _ = finc.add_norm_forward(x, b["norm"], eps=EPS)
            q, k, v, g = self.split(finc.linear_forward(y, b["w_in"]))
            y = finc.linear_attention_step(q, k, v, state, g=g, decay=self.decay,
                                           scale=self.E ** -0.5, slots=slots)
            finc.linear_forward(y.flatten(1), b["w_out"], residual=x, out=x)
            y, _ = finc.add_norm_forward(x, b["norm2"], eps=EPS)
            y = finc.linear_forward(y, b["w_up"], b["b_up"], act="silu")
            finc.linear_forward(y, b["w_down"], residual=x, out=x)
        y, _ = finc.add_norm_forward(x, self.norm, eps=EPS)
        return finc.linear_forward(y, self.head_w)

    def sample(self, B, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        cache, out = self.start(B), torch.empty(B, self.L, dtype=torch.int64, device=DEV)
        before = torch.full((B,), self.V, device=DEV)
        for t in range(self.L):
            p = torch.softmax(self.step(before, t, cache).float(), dim=1)
            before = torch.multinomial(p, 1, generator=gen)[:, 0]
            out[:, t] = before
        return out


# ---- pixels, and training -------------------------------------------------------------


def pixels(images, side=16, levels=32, seed=0):
    """Codes (images, side^2) of smooth random images."""
    gen = torch.Generator().manual_seed(seed)
    at = torch.arange(side) / side
    f = torch.randn(images, 3, 2, generator=gen)
    x = sum(torch.sin(2 * math.pi * (f[:, i, 0, None, None] * at[:, None]
                                     + f[:, i, 1, None, None] * at + i / 3.0)) for i in range(3))
    return ((x / 6 + 0.5) * levels).long().clamp(0, levels - 1).flatten(1).to(DEV)


def train(prior, codes, steps, batch, lr=3e-3, report=None):
    """Losses of `steps` steps on batches of codes."""
    opt = torch.optim.Adam(prior.parameters(), lr=lr)
    losses = []
    for i in range(steps):
        at = (i * batch) % (len(codes) - batch + 1)
        loss = prior.bits(codes[at:at + batch])
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if report and i % report == 0:
            print(f"step {i}: {float(losses[-1]):.4f} bits a pixel", flush=True)
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--bf16", action="store_true")
    args = ap.parse_args()
    torch.cuda.set_device(torch.device(DEV))
    codes = pixels(4 * args.batch)
    prior = Prior(32, codes.shape[1], dtype=torch.bfloat16 if args.bf16 else torch.float32)
    train(prior, codes, args.steps, args.batch, report=20)
    with torch.no_grad():
        want = prior.forward(codes[:8]).float()
    cache, off = prior.start(8), 0.0
    for t in range(codes.shape[1]):
        before = codes[:8, t - 1].contiguous() if t else torch.full((8,), 32, device=DEV)
        off = max(off, float((prior.step(before, t, cache).float() - want[:, t]).abs().max()))
    print(f"prompt against single positions: {off:.2e}")
    print(f"samples: mean code {float(prior.sample(16).float().mean()):.2f}, "
          f"pixels {float(codes.float().mean()):.2f}")


if __name__ == "__main__":
    main()
