"""Plain 64-bit references of the sequence operators, on the CPU: position after
position, tap after tap, differentiable by autograd; and the bar their outputs are
held to."""
import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def close(got, ref, what, chain=64):
    """Elementwise: one rounding to the output's type, and `chain` fp32 roundings of
    values of the result's own size or of its root mean square (a sum's terms)."""
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    g, r = got.detach().double().cpu(), ref.detach().double().cpu()
    assert torch.equal(torch.isnan(g), torch.isnan(r)), f"{what}: NaN in other places"
    fine = torch.isfinite(r)
    assert torch.equal(g[~fine & ~torch.isnan(r)], r[~fine & ~torch.isnan(r)]), what
    g, r = g[fine], r[fine]
    if r.numel() == 0:
        return
    rms = r.square().mean().sqrt()
    bar = U[got.dtype] * 1.01 * r.abs() + TINY[got.dtype] + chain * 2.0 ** -24 * (r.abs() + rms)
    err = (g - r).abs()
    bad = err > bar
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {r.numel()} out of tolerance, "
                           f"largest {float((err / bar.clamp(min=1e-300)).max()):.2f} times it")


def silu(v):
    return v * torch.sigmoid(v)


def ends(lengths, B, L):
    return [L] * B if lengths is None else [min(max(int(n), 0), L) for n in lengths]


def conv(x, w, bias, act, state, lengths):
    """(y, state after) of float64 tensors."""
    B, D, L = x.shape
    K = w.shape[1]
    y = [torch.zeros(D, 0, dtype=x.dtype)] * B
    after = []
    for b, n in enumerate(ends(lengths, B, L)):
        before = torch.zeros(D, K - 1, dtype=x.dtype) if state is None else state[b]
        e = torch.cat([before, x[b, :, :n]], dim=1)
        p = sum(w[:, j:j + 1] * e[:, j:j + n] for j in range(K))
        p = p if bias is None else p + bias[:, None]
        y[b] = torch.cat([silu(p) if act else p, torch.zeros(D, L - n, dtype=x.dtype)], dim=1)
        after.append(e[:, n:n + K - 1])
    return torch.stack(y), torch.stack(after)


def scan(x, dt, A, Bm, Cm, D, z, dt_bias, softplus, state, lengths):
    """(y, state after) of float64 tensors."""
    B, C, L = x.shape
    G, N = Bm.shape[1:3]
    v = dt if dt_bias is None else dt + dt_bias[:, None]
    delta = torch.nn.functional.softplus(v, threshold=60.0) if softplus else v
    out, after = [], []
    for b, n in enumerate(ends(lengths, B, L)):
        h = torch.zeros(C, N, dtype=x.dtype) if state is None else state[b]
        cols = []
        for t in range(n):
            rows = lambda m: m[b, :, :, t].repeat_interleave(C // G, dim=0)  # noqa: E731
            h = torch.exp(delta[b, :, t, None] * A) * h \
                + (delta[b, :, t] * x[b, :, t])[:, None] * rows(Bm)
            y = (rows(Cm) * h).sum(1)
            if D is not None:
                y = y + D * x[b, :, t]
            if z is not None:
                y = y * silu(z[b, :, t])
            cols.append(y)
        cols += [torch.zeros(C, dtype=x.dtype)] * (L - n)
        out.append(torch.stack(cols, dim=1) if cols else torch.zeros(C, 0, dtype=x.dtype))
        after.append(h)
    return torch.stack(out), torch.stack(after)


def norm(r, w, eps):
    return r / (r.square().mean(-1, keepdim=True) + eps).sqrt() * w


def philox(ctr, key):
    """Philox4x32-10 of uint64 counters (the upper 64 bits 0): four uint32 words."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    ctr = np.asarray(ctr, dtype=u)
    return philox_words([ctr & low, ctr >> u(32), np.zeros_like(ctr), np.zeros_like(ctr)], key)


def philox_words(c, key):
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=u) for v in c]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(q >> u(32)) ^ c[1] ^ u(k[0]), q & low, (p >> u(32)) ^ c[3] ^ u(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_factor(rows, D, p, seed, offset):
    """What every element of (rows, D) is multiplied by (float64)."""
    per = -(-D // 8)
    with np.errstate(over="ignore"):
        at = np.arange(rows * per, dtype=np.uint64) + np.uint64(offset)
    words = philox(at, seed)
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1)
    cut = int(np.rint(p * 65536))
    keep = bits.reshape(rows, per * 8)[:, :D] >= cut
    return torch.from_numpy(keep * (65536.0 / (65536 - cut)))
