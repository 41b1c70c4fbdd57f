"""Linear attention, projections and embeddings without a GPU: the references' pins, the
argument structures against the header, refusals before any HIP call, workspace sizes."""
import os
import re
import shutil
import subprocess

import pytest
import torch

import rows_ref as rows
import test_kernel_resources_cpu
from paper_2301_09266_amd import finc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL = finc.EINVAL


# ---- pins of the references -------------------------------------------------------


def test_attention_reference_is_the_sum_over_pairs():
    r = torch.Generator().manual_seed(0)
    n = lambda *s: torch.randn(*s, generator=r).double()  # noqa: E731
    B, L, H, G, DK, DV = 2, 9, 4, 2, 3, 5
    q, k, v, g, d, S = (n(B, L, G, DK), n(B, L, G, DK), n(B, L, H, DV), -n(B, L, H).abs(),
                        -n(H).abs(), n(B, H, DK, DV))
    y, end = rows.attention(q, k, v, g, d, 0.7, S, torch.tensor([9, 4]))
    for b, count in ((0, 9), (1, 4)):
        for h in range(H):
            at = torch.cumsum(g[b, :, h] + d[h], 0)
            for i in range(L):
                want = torch.zeros(DV).double()
                if i < count:
                    want = torch.exp(at[i]) * (q[b, i, h // 2] @ S[b, h])
                    for j in range(i + 1):
                        want = want + torch.exp(at[i] - at[j]) * (
                            q[b, i, h // 2] @ k[b, j, h // 2]) * v[b, j, h]
                assert torch.allclose(y[b, i, h], 0.7 * want, rtol=1e-12, atol=1e-12)
            want = torch.exp(at[count - 1]) * S[b, h] + sum(
                torch.exp(at[count - 1] - at[j]) * torch.outer(k[b, j, h // 2], v[b, j, h])
                for j in range(count))
            assert torch.allclose(end[b, h], want, rtol=1e-12, atol=1e-12)


def test_activation_references_are_torchs():
    p = torch.linspace(-9, 9, 101, dtype=torch.float64)
    assert torch.allclose(rows.act("gelu", p), torch.nn.functional.gelu(p), rtol=1e-9, atol=1e-15)
    assert torch.allclose(rows.act("silu", p), torch.nn.functional.silu(p), rtol=1e-12)
    assert torch.equal(rows.act("relu", p), torch.relu(p)) and rows.act(None, p) is p


# ---- the ABI -----------------------------------------------------------------------

PACKED = {"finc_attention_args": finc.ATTENTION_ARGS, "finc_attention_grads": finc.ATTENTION_GRADS,
          "finc_attention_step_args": finc.ATTENTION_STEP_ARGS, "finc_linear_args": finc.LINEAR_ARGS,
          "finc_linear_grad_args": finc.LINEAR_GRAD_ARGS}


def struct_fields(name):
    """(type, field) of a structure in the header, heads as their four fields."""
    text = open(os.path.join(ROOT, "include", "finc.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text).group(1)
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        kind, names = re.match(r"(const void|void|const float|float|const int|int|finc_heads|"
                               r"long long|double)\s*(.*)", decl, flags=re.S).groups()
        for field in names.split(","):
            plain = field.replace("*", "").strip()
            if kind == "finc_heads":
                yield from (("P", plain + ".p"), *(("q", f"{plain}.{s}") for s in ("sb", "st", "sh")))
            else:
                yield "P" if "*" in field else {"int": "i", "long long": "q", "double": "d"}[kind], plain


@pytest.mark.parametrize("name", sorted(PACKED))
def test_packed_arguments_have_the_headers_fields(name):
    kinds = "".join(k for k, _ in struct_fields(name))
    fmt = re.sub(r"(\d+)([a-zA-Z])", lambda m: m.group(2) * int(m.group(1)),
                 PACKED[name].format.lstrip("@").replace(" ", ""))
    assert fmt == kinds


def test_packed_arguments_have_the_compilers_layout(tmp_path):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers not found")
    lines = []
    for name, packed in PACKED.items():
        lines.append(f'static_assert(sizeof({name}) == {packed.size}, "{name}");')
        at = 0
        for kind, field in struct_fields(name):
            size = {"i": 4}.get(kind, 8)
            at = -(-at // size) * size
            lines.append(f'static_assert(offsetof({name}, {field}) == {at}, "{name}.{field}");')
            at += size
    src = tmp_path / "layout.cpp"
    src.write_text('#include <stddef.h>\n#include "finc.h"\n' + "\n".join(lines) + "\n")
    subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-D__HIP_PLATFORM_AMD__",
                    "-Wno-invalid-offsetof", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), str(src)], check=True)


# Addresses that are never used: every call below is refused on the host.
P = [0x100000000 * (i + 1) for i in range(24)]
ODD = 0x100000001


def lib():
    return finc.lib()


# B = 2, L = 600, H = 4, G = 2, DK = 8, DV = 16, bf16
QK = (600 * 16, 16, 8)
VY = (600 * 64, 64, 16)
GG = (600 * 4, 4, 1)


def attention(kind=1, B=2, L=600, H=4, G=2, DK=8, DV=16, q=(P[0], *QK), k=(P[1], *QK),
              v=(P[2], *VY), g=(P[3], *GG), y=(P[4], *VY), decay=P[5], state=P[6], after=P[7],
              states=P[8], lengths=P[9], scale=1.0):
    return finc.ATTENTION_ARGS.pack(kind, B, L, H, G, DK, DV, *q, *k, *v, *g, *y, decay, state,
                                    after, states, lengths, scale)


@pytest.mark.parametrize("change", [
    dict(kind=3), dict(kind=-1), dict(B=-1), dict(L=-1), dict(H=0), dict(G=0), dict(G=3), dict(DK=0),
    dict(DK=129), dict(DV=0), dict(DV=129), dict(B=1 << 23), dict(q=(0, *QK)), dict(q=(ODD, *QK)),
    dict(k=(0, *QK)), dict(v=(0, *VY)), dict(v=(P[2] + 1, *VY)), dict(y=(0, *VY)),
    dict(y=(ODD, *VY)), dict(q=(P[0], -1, 16, 8)), dict(q=(P[0], 600 * 16, -16, 8)),
    dict(k=(P[1], 600 * 16, 16, -8)), dict(v=(P[2], 1 << 62, 64, 16)), dict(g=(ODD, *GG)),
    dict(g=(P[3], -4, 4, 1)), dict(y=(P[4], 0, 64, 16)), dict(y=(P[4], 600 * 64, 63, 16)),
    dict(y=(P[4], 600 * 64, 64, 15)), dict(y=(P[4], 64, 64, 16)), dict(y=(P[2], *VY)),
    dict(y=(P[0] + 64, *VY)), dict(y=(P[3], *VY)), dict(decay=ODD), dict(state=ODD),
    dict(after=ODD), dict(after=P[6] + 4), dict(after=P[2]), dict(states=0), dict(states=P[8] + 128),
    dict(states=P[6]), dict(states=P[4]), dict(lengths=ODD), dict(after=P[9]), dict(states=P[7])])
def test_attention_refusals(change):
    assert lib().finc_linear_attention_forward(attention(**change), None) == EINVAL
    assert lib().finc_linear_attention_forward(None, None) == EINVAL


def attention_grads(dy=(P[10], *VY), dq=(P[11], *QK), dk=(P[12], *QK), dv=(P[13], *VY),
                    dg=(P[14], *GG), dso=P[15], ds=P[16], ws=P[17]):
    return finc.ATTENTION_GRADS.pack(*dy, *dq, *dk, *dv, *dg, dso, ds, ws)


@pytest.mark.parametrize("change", [
    dict(dy=(0, *VY)), dict(dy=(ODD, *VY)), dict(dq=(0, *QK)), dict(dq=(P[11], 0, 16, 8)),
    dict(dk=(P[11], *QK)), dict(dk=(P[12], 600 * 16, 15, 8)), dict(dv=(P[10], *VY)),
    dict(dv=(P[2], *VY)), dict(dv=(0, *VY)), dict(dg=(P[3], *GG)), dict(dg=(P[14], 600 * 4, 3, 1)),
    dict(ds=P[15]), dict(ds=P[8]), dict(dso=ODD), dict(ws=0), dict(ws=P[17] + 64), dict(ws=P[8]),
    dict(dq=(P[10] + 32, *QK))])
def test_attention_gradient_refusals(change):
    f = lib().finc_linear_attention_backward
    assert f(attention(), attention_grads(**change), None) == EINVAL
    assert f(attention(states=0), attention_grads(), None) == EINVAL
    assert f(attention(DK=129), attention_grads(), None) == EINVAL
    assert f(attention(), None, None) == EINVAL
    assert f(None, attention_grads(), None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(kind=3), dict(B=-1), dict(S=-1), dict(H=0), dict(G=3), dict(DK=129), dict(DV=0),
    dict(q=(0, 16, 0, 8)), dict(k=(ODD, 16, 0, 8)), dict(v=(0, 64, 0, 16)), dict(y=(0, 64, 0, 16)),
    dict(y=(P[4], 63, 0, 16)), dict(y=(P[2], 64, 0, 16)), dict(y=(P[4], 64, 0, 15)),
    dict(y=(P[6], 64, 0, 16)), dict(state=0), dict(state=ODD), dict(state=P[2]), dict(slots=0, S=1),
    dict(slots=ODD), dict(decay=ODD), dict(g=(ODD, 4, 0, 1)), dict(q=(P[0], -16, 0, 8))])
def test_attention_step_refusals(change):
    a = dict(kind=1, B=2, S=4, H=4, G=2, DK=8, DV=16, q=(P[0], 16, 0, 8), k=(P[1], 16, 0, 8),
             v=(P[2], 64, 0, 16), g=(P[3], 4, 0, 1), y=(P[4], 64, 0, 16), decay=P[5], state=P[6],
             slots=P[7], scale=1.0)
    a.update(change)
    flat = [x for v in a.values() for x in (v if isinstance(v, tuple) else (v,))]
    assert lib().finc_linear_attention_step(finc.ATTENTION_STEP_ARGS.pack(*flat), None) == EINVAL
    assert lib().finc_linear_attention_step(None, None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=3), dict(act=4), dict(act=-1), dict(M=-1), dict(K=0), dict(N=0), dict(M=1 << 30),
    dict(M=1 << 29, K=1 << 20, sx=1 << 20), dict(x=0), dict(x=ODD), dict(w=0), dict(w=ODD),
    dict(res=ODD), dict(y=0), dict(y=ODD), dict(pre=ODD), dict(sx=-1), dict(sw=-1), dict(sres=-1),
    dict(sy=7), dict(sy=-8), dict(spre=7), dict(y=P[0]), dict(y=P[1]), dict(pre=P[2]),
    dict(pre=P[3]), dict(y=P[2], sy=16), dict(y=P[2] + 2), dict(bias=ODD), dict(y=P[5]),
    dict(ws=P[6] + 8)])
def test_linear_refusals(change):
    a = dict(type=1, act=2, M=4, K=16, N=8, x=P[0], w=P[1], res=P[2], y=P[3], pre=P[4], sx=16,
             sw=16, sres=8, sy=8, spre=8, bias=P[5], ws=P[6])
    a.update(change)
    assert lib().finc_linear_forward(finc.LINEAR_ARGS.pack(*a.values()), None) == EINVAL
    assert lib().finc_linear_forward(None, None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=3), dict(act=4), dict(M=-1), dict(K=0), dict(N=0), dict(dy=0), dict(x=0), dict(w=0),
    dict(pre=0), dict(pre=ODD), dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(sdy=-1),
    dict(sdx=15), dict(sdw=15), dict(dx=P[0]), dict(dx=P[1]), dict(dw=P[2]), dict(dw=P[4]),
    dict(db=P[5]), dict(ws=0), dict(ws=P[7] + 8), dict(ws=P[3])])
def test_linear_gradient_refusals(change):
    a = dict(type=1, act=2, M=4, K=16, N=8, dy=P[0], x=P[1], w=P[2], pre=P[3], dx=P[4], dw=P[5],
             sdy=8, sx=16, sw=16, spre=8, sdx=16, sdw=16, db=P[6], ws=P[7])
    a.update(change)
    assert lib().finc_linear_backward(finc.LINEAR_GRAD_ARGS.pack(*a.values()), None) == EINVAL
    assert lib().finc_linear_backward(None, None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=3), dict(ttype=2), dict(ids=0), dict(ids=P[0] + 4), dict(table=0), dict(table=ODD),
    dict(st=-1), dict(y=0), dict(y=ODD), dict(sy=7), dict(y=P[1]), dict(y=P[0]), dict(M=-1),
    dict(V=-1), dict(D=0), dict(M=1 << 30), dict(V=1 << 30), dict(M=1 << 28, D=100)])
def test_embed_refusals(change):
    a = dict(type=1, ttype=0, ids=P[0], wide=1, table=P[1], st=8, y=P[2], sy=8, M=4, V=10, D=8,
             scale=1.0)
    a.update(change)
    assert lib().finc_embed_forward(*a.values(), None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=3), dict(ids=0), dict(ids=P[0] + 4), dict(dy=0), dict(dy=ODD), dict(sdy=-8),
    dict(dtable=0), dict(dtable=ODD), dict(dtable=P[1]), dict(dtable=P[0]), dict(M=-1), dict(V=-1),
    dict(D=0), dict(ws=0), dict(ws=P[3] + 4), dict(ws=P[2]), dict(ws=P[1]), dict(M=1 << 28, D=100)])
def test_embed_gradient_refusals(change):
    a = dict(type=1, ids=P[0], wide=1, dy=P[1], sdy=8, dtable=P[2], M=4, V=10, D=8, scale=1.0,
             ws=P[3])
    a.update(change)
    assert lib().finc_embed_backward(*a.values(), None) == EINVAL


def test_nothing_to_do_is_no_error():
    none = (0, 0, 0, 0)
    assert lib().finc_linear_attention_forward(
        attention(B=0, q=none, k=none, v=none, g=none, y=none, state=0, after=0, states=0,
                  lengths=0, decay=0), None) == finc.OK
    assert lib().finc_linear_attention_forward(
        attention(L=0, q=none, k=none, v=none, g=none, y=none, state=0, after=0, states=0,
                  lengths=0, decay=0), None) == finc.OK
    assert lib().finc_embed_forward(1, 1, None, 1, P[0], 8, None, 8, 0, 4, 8, 1.0, None) == finc.OK
    a = (1, 2, 0, 16, 8, 0, P[1], 0, 0, 0, 16, 16, 8, 8, 8, 0, 0)
    assert lib().finc_linear_forward(finc.LINEAR_ARGS.pack(*a), None) == finc.OK


def test_sizes():
    L = lib()
    part = finc.ATTENTION_PART
    assert L.finc_linear_attention_states_bytes(2, 64, 3, 129, 8) == 0
    assert L.finc_linear_attention_workspace_bytes(2, 64, 3, 2, 8, 8) == 0
    # parts of half the length in rows of up to four
    for n, parts in ((1, 1), (part, 1), (part + 1, 3), (4 * part, 8), (4 * part + 1, 5),
                     (10 * part, 10)):
        size = L.finc_linear_attention_states_bytes(4, n, 8, 32, 16)
        assert size == 4 * 8 * (parts + 1) * 32 * 16 * 4 + -(-4 * 8 * parts * 4 // 256) * 256
        for G in (1, 8):
            assert L.finc_linear_attention_workspace_bytes(4, n, 8, G, 32, 16) % 256 == 0
    assert L.finc_linear_workspace_bytes(3, 4, 4, 4) == 0
    assert L.finc_linear_grad_workspace_bytes(1, 9, 4, 4, 4) == 0
    assert L.finc_linear_grad_workspace_bytes(1, 2, 100, 40, 30) >= 100 * 30 * 2
    assert L.finc_embed_workspace_bytes(-1, 4, 4) == 0 and L.finc_embed_workspace_bytes(4, 4, 0) == 0
    assert L.finc_embed_workspace_bytes(1000, 4, 64) % 256 == 0


def test_kernels_keep_their_registers():
    """No scratch in the kernels of heads that fill their tiles, of aligned projections and
    of the tables' gradients; little where heads of 128 do not."""
    ks = {n: k for n, k in test_kernel_resources_cpu.kernels().items()
          if re.search("attention_kernel|gemm_fast_kernel|gemm_few|10sum_kernel|join", n)}
    assert sum("16attention_kernelI" in n for n in ks) == 48
    for n, k in ks.items():
        some = re.search("16attention_kernelI.*Li128ELi128ELi2ELb0ELb0", n)
        assert k[".private_segment_fixed_size"] <= (128 if some else 0), n


def test_host_tensors_are_refused():
    x, w = torch.zeros(2, 6, 4, 8), torch.zeros(5, 8)
    with pytest.raises(ValueError, match="q must be a device tensor"):
        finc.linear_attention_forward(x, x, x)
    with pytest.raises(ValueError, match="expected \\(B, L, G, DK\\)"):
        finc.linear_attention_forward(x[0], x, x)
    with pytest.raises(ValueError, match="3 groups do not divide 4"):
        finc.linear_attention_forward(x[:, :, :3], x[:, :, :3], x)
    with pytest.raises(ValueError, match="expected 1 to 128"):
        finc.linear_attention_step(torch.zeros(2, 1, 200), torch.zeros(2, 1, 200), x[:, 0], x)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        finc.linear_forward(w, w)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        finc.linear_backward(w, w, w)
    with pytest.raises(ValueError, match="ids must be a device tensor"):
        finc.embed_forward(torch.zeros(3, dtype=torch.int64), w)
    with pytest.raises(ValueError, match="dy must be a device tensor"):
        finc.embed_backward(torch.zeros(5, dtype=torch.int64), w, 4)
