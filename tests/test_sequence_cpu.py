"""The sequence operators without a GPU: the references' pins, the argument
structures against the header, refusals before any HIP call, workspace sizes, and
the kernels' registers."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch
from scipy.signal import lfilter

import seq_ref as ref
from paper_2301_09266_amd import finc
from test_kernel_resources_cpu import kernels, waves

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED = finc.EINVAL, finc.EUNSUPPORTED

# ---- pins of the references -------------------------------------------------------


def test_generator_known_answers():
    """The published known answers of Philox4x32-10: zeros, ones, digits of pi."""
    cases = [((0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
             ((0xffffffff,) * 4, (0xffffffff,) * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
             ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
              "d16cfe09 94fdcceb 5001e420 24126ea1")]
    for ctr, key, want in cases:
        got = ref.philox_words(ctr, key[0] | key[1] << 32)
        assert " ".join(f"{int(v):08x}" for v in got) == want


def test_dropout_keeps_the_mean_and_the_share():
    f = ref.dropout_factor(1000, 1003, 0.3, 5, 9)
    cut = round(0.3 * 65536)
    assert set(np.unique(f)) == {0.0, 65536 / (65536 - cut)}
    assert abs(float((f == 0).double().mean()) - cut / 65536) < 5 * (0.21 / f.numel()) ** 0.5


def test_conv_reference_is_the_padded_convolution():
    g = torch.Generator().manual_seed(0)
    x, w = torch.randn(2, 3, 9, generator=g).double(), torch.randn(3, 4, generator=g).double()
    b, s = torch.randn(3, generator=g).double(), torch.randn(2, 3, 3, generator=g).double()
    y, after = ref.conv(x, w, b, False, s, None)
    want = torch.nn.functional.conv1d(torch.cat([s, x], 2), w[:, None], b, groups=3)
    assert torch.allclose(y, want, rtol=1e-12, atol=1e-12)
    assert torch.equal(after, x[:, :, -3:])


def test_scan_reference_is_a_filter_where_the_steps_are_equal():
    """Constant steps make the scan a sum of first-order filters."""
    g = torch.Generator().manual_seed(1)
    L, N = 50, 3
    x = torch.randn(1, 1, L, generator=g).double()
    A = -torch.rand(1, N, generator=g).double()
    Bm, Cm = (torch.randn(1, 1, N, 1, generator=g).double().expand(1, 1, N, L) for _ in range(2))
    dt = torch.full((1, 1, L), 0.3, dtype=torch.float64)
    y, h = ref.scan(x, dt, A, Bm, Cm, None, None, None, False, None, None)
    want = sum(Cm[0, 0, n, 0].item() * lfilter([0.3 * Bm[0, 0, n, 0].item()],
                                               [1, -np.exp(0.3 * A[0, n].item())], x[0, 0].numpy())
               for n in range(N))
    assert np.allclose(y[0, 0].numpy(), want, rtol=1e-12, atol=1e-12)
    assert h.shape == (1, 1, N)


# ---- the ABI ---------------------------------------------------------------------

PACKED = {"finc_conv_args": finc.CONV_ARGS, "finc_conv_grads": finc.CONV_GRADS,
          "finc_scan_args": finc.SCAN_ARGS, "finc_scan_grads": finc.SCAN_GRADS,
          "finc_scan_step_args": finc.SCAN_STEP_ARGS, "finc_norm_args": finc.NORM_ARGS,
          "finc_norm_grad_args": finc.NORM_GRAD_ARGS}


def struct_fields(name):
    """(type, field) of a structure in the header, rasters as their three fields."""
    text = open(os.path.join(ROOT, "include", "finc.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text).group(1)
    for decl in body.split(";"):
        decl = decl.strip()
        if not decl:
            continue
        m = re.match(r"(const void|void|const float|float|const int|int|finc_raster|long long|"
                     r"double|unsigned long long)\s*(.*)", decl, flags=re.S)
        for field in m.group(2).split(","):
            pointer = "*" in field
            field = field.replace("*", "").strip()
            if m.group(1) == "finc_raster":
                yield from (("P", field + ".p"), ("q", field + ".sb"), ("q", field + ".sd"))
            elif pointer:
                yield "P", field
            else:
                yield {"int": "i", "long long": "q", "double": "d",
                       "unsigned long long": "Q"}[m.group(1)], field


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
P = [0x10000000 * (i + 1) for i in range(24)]
ODD = 0x10000001


def lib():
    return finc.lib()


def conv(kind=1, B=2, D=6, L=40, K=4, silu=1, x=(P[0], 240, 40), y=(P[1], 240, 40), w=P[2],
         bias=P[3], state=P[4], after=P[5], lengths=P[6]):
    return finc.CONV_ARGS.pack(kind, B, D, L, K, silu, *x, *y, w, bias, state, after, lengths)


@pytest.mark.parametrize("change", [
    dict(kind=3), dict(kind=-1), dict(B=-1), dict(D=0), dict(L=-1), dict(L=1 << 30), dict(K=0),
    dict(K=9), dict(B=1 << 20, D=1 << 11), dict(x=(0, 240, 40)), dict(x=(ODD, 240, 40)),
    dict(x=(P[0], -240, 40)), dict(x=(P[0], 240, -40)), dict(x=(P[0], 1 << 62, 40)),
    dict(y=(0, 240, 40)), dict(y=(P[1], 240, 39)), dict(y=(P[1], 239, 40)), dict(y=(P[1], 0, 40)),
    dict(y=(P[0], 240, 40)), dict(y=(P[0] + 400, 240, 40)), dict(y=(P[0] + 100, 480, 40)),
    dict(w=0), dict(w=ODD), dict(bias=ODD), dict(state=ODD), dict(after=P[4]), dict(after=P[0] + 2),
    dict(y=(P[6], 240, 40)), dict(lengths=P[6] + 2)])
def test_conv_refusals(change):
    assert lib().finc_causal_conv_forward(conv(**change), None) == EINVAL
    assert lib().finc_causal_conv_forward(None, None) == EINVAL


def conv_grads(dy=(P[7], 240, 40), dx=(P[8], 240, 40), dw=P[9], dbias=P[10], dso=P[11], ds=P[12],
               ws=P[13]):
    return finc.CONV_GRADS.pack(*dy, *dx, dw, dbias, dso, ds, ws)


@pytest.mark.parametrize("change", [
    dict(dy=(0, 240, 40)), dict(dx=(0, 240, 40)), dict(dx=(P[8], 240, 0)), dict(dx=(P[7], 240, 40)),
    dict(dx=(P[0], 240, 40)), dict(dw=0), dict(dw=P[2]), dict(dbias=P[9] + 16), dict(ds=P[11]),
    dict(ws=0), dict(ws=P[13] + 128), dict(ws=P[8]), dict(dso=ODD)])
def test_conv_gradient_refusals(change):
    assert lib().finc_causal_conv_backward(conv(), conv_grads(**change), None) == EINVAL
    assert lib().finc_causal_conv_backward(conv(K=9), conv_grads(), None) == EINVAL
    assert lib().finc_causal_conv_backward(conv(), None, None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=7), dict(x=0), dict(y=0), dict(sy=5), dict(w=0), dict(state=0), dict(B=-1),
    dict(S=-1), dict(D=0), dict(K=9), dict(y=P[0]), dict(state=P[0]), dict(slots=0, S=1),
    dict(slots=ODD), dict(sx=-6)])
def test_conv_step_refusals(change):
    a = dict(type=1, x=P[0], sx=6, y=P[1], sy=6, w=P[2], bias=P[3], state=P[4], slots=P[5], B=2,
             S=4, D=6, K=4, silu=1)
    a.update(change)
    assert lib().finc_causal_conv_step(*a.values(), None) == EINVAL


def scan(kind=0, B=2, D=6, L=40, N=16, G=2, softplus=1, x=(P[0], 240, 40), dt=(P[1], 240, 40),
         z=(P[2], 240, 40), Bm=(P[3], 1280, 40), Cm=(P[4], 1280, 40), y=(P[5], 240, 40), A=P[6],
         D_=P[7], bias=P[8], state=P[9], after=P[10], states=P[11], lengths=P[12]):
    return finc.SCAN_ARGS.pack(kind, B, D, L, N, G, softplus, *x, *dt, *z, *Bm, *Cm, *y, A, D_,
                               bias, state, after, states, lengths)


@pytest.mark.parametrize("change", [
    dict(kind=5), dict(B=-1), dict(D=0), dict(L=-1), dict(L=1 << 30), dict(N=0), dict(N=65),
    dict(G=0), dict(G=4), dict(x=(0, 240, 40)), dict(dt=(0, 240, 40)), dict(Bm=(0, 1280, 40)),
    dict(Cm=(0, 1280, 40)), dict(Bm=(P[3] + 1, 1280, 40)), dict(z=(ODD, 240, 40)),
    dict(y=(0, 240, 40)), dict(y=(P[5], 240, 20)), dict(y=(P[2], 240, 40)),
    dict(y=(P[3] + 64, 240, 40)), dict(A=0), dict(A=ODD), dict(D_=ODD), dict(bias=ODD),
    dict(state=ODD), dict(after=P[9] + 4), dict(after=P[0]), dict(states=P[11] + 4),
    dict(states=P[9]), dict(after=P[11] + 16), dict(lengths=ODD)])
def test_scan_refusals(change):
    assert lib().finc_selective_scan_forward(scan(**change), None) == EINVAL
    assert lib().finc_selective_scan_forward(None, None) == EINVAL


def scan_grads(dy=(P[13], 240, 40), dx=(P[14], 240, 40), ddt=(P[15], 240, 40), dz=(P[16], 240, 40),
               dB=(P[17], 1280, 40), dC=(P[18], 1280, 40), dA=P[19], dD=P[20], db=P[21], dso=0,
               ds=P[22], ws=P[23]):
    return finc.SCAN_GRADS.pack(*dy, *dx, *ddt, *dz, *dB, *dC, dA, dD, db, dso, ds, ws)


@pytest.mark.parametrize("change", [
    dict(dy=(0, 240, 40)), dict(dx=(0, 240, 40)), dict(ddt=(0, 240, 40)), dict(dz=(0, 240, 40)),
    dict(dB=(0, 1280, 40)), dict(dC=(P[17], 1280, 40)), dict(dx=(P[13], 240, 40)),
    dict(dx=(P[15], 240, 40)), dict(dB=(P[17], 1280, 10)), dict(dA=0), dict(dA=P[6]),
    dict(dD=P[19] + 4), dict(db=ODD), dict(dso=P[22]), dict(ds=P[11]), dict(ws=0),
    dict(ws=P[23] + 64), dict(ws=P[11])])
def test_scan_gradient_refusals(change):
    assert lib().finc_selective_scan_backward(scan(), scan_grads(**change), None) == EINVAL
    assert lib().finc_selective_scan_backward(scan(states=0), scan_grads(), None) == EINVAL
    assert lib().finc_selective_scan_backward(scan(N=65), scan_grads(), None) == EINVAL
    assert lib().finc_selective_scan_backward(scan(), None, None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=3), dict(B=-1), dict(S=-1), dict(D=0), dict(N=65), dict(G=5), dict(x=0), dict(dt=0),
    dict(Bm=0), dict(Cm=0), dict(sx=-1), dict(sy=3), dict(y=0), dict(y=P[0]), dict(A=0),
    dict(state=0), dict(state=P[1]), dict(slots=0, S=1), dict(slots=ODD)])
def test_scan_step_refusals(change):
    a = dict(type=1, B=2, S=4, D=6, N=16, G=2, softplus=1, x=P[0], dt=P[1], z=P[2], Bm=P[3],
             Cm=P[4], sx=6, sdt=6, sz=6, sB=32, sC=32, sy=6, y=P[5], A=P[6], D_=P[7], bias=P[8],
             state=P[9], slots=P[10])
    a.update(change)
    assert lib().finc_selective_scan_step(finc.SCAN_STEP_ARGS.pack(*a.values()), None) == EINVAL


@pytest.mark.parametrize("change", [
    dict(type=3), dict(x=0), dict(y=0), dict(sx=-8), dict(sy=7), dict(M=-1), dict(D=0),
    dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=65535.6 / 65536),
    dict(y=P[0], sy=16), dict(y=P[0] + 2), dict(y=P[1], sy=9), dict(M=1 << 30, D=100)])
def test_dropout_refusals(change):
    a = dict(type=1, x=P[0], sx=8, res=P[1], sr=8, y=P[2], sy=8, M=4, D=8, p=0.1, seed=1, offset=2)
    a.update(change)
    assert lib().finc_dropout(*a.values(), None) == EINVAL


@pytest.mark.parametrize("change,want", [
    (dict(type=4), EINVAL), (dict(rtype=2), EINVAL), (dict(M=-1), EINVAL), (dict(D=0), EINVAL),
    (dict(D=16385, sx=16385, sres=16385, sy=16385, sr=16385), EUNSUPPORTED), (dict(x=0), EINVAL),
    (dict(y=0), EINVAL), (dict(w=0), EINVAL), (dict(w=ODD), EINVAL), (dict(sy=7), EINVAL),
    (dict(sr=7), EINVAL), (dict(scale=ODD), EINVAL), (dict(scale=P[0]), EINVAL),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(p=1.0), EINVAL),
    (dict(y=P[0], sy=16), EINVAL), (dict(y=P[0] + 4), EINVAL), (dict(r=P[0]), EINVAL),
    (dict(r=P[1], sr=16), EINVAL), (dict(r=P[2]), EINVAL), (dict(y=P[4]), EINVAL)])
def test_norm_refusals(change, want):
    a = dict(type=1, rtype=0, M=4, D=8, x=P[0], res=P[1], y=P[2], r=P[3], sx=8, sres=8, sy=8, sr=8,
             w=P[4], scale=0, eps=1e-5, p=0.0, seed=0, offset=0)
    a.update(change)
    assert lib().finc_add_norm_forward(finc.NORM_ARGS.pack(*a.values()), None) == want
    assert lib().finc_add_norm_forward(None, None) == EINVAL


@pytest.mark.parametrize("change,want", [
    (dict(type=4), EINVAL), (dict(rtype=2), EINVAL), (dict(M=-1), EINVAL), (dict(D=0), EINVAL),
    (dict(D=16385, sdy=16385, sr=16385, sdr=16385, sdx=16385, sds=16385), EUNSUPPORTED),
    (dict(dy=0), EINVAL), (dict(r=0), EINVAL), (dict(w=0), EINVAL), (dict(dw=0), EINVAL),
    (dict(ws=0), EINVAL), (dict(ws=P[7] + 16), EINVAL), (dict(ws=P[0]), EINVAL),
    (dict(dw=P[5]), EINVAL), (dict(dx=P[0], sdx=16), EINVAL), (dict(dx=P[1]), EINVAL),
    (dict(ds=P[1]), EINVAL), (dict(ds=P[3]), EINVAL), (dict(ds=P[2], sds=16), EINVAL),
    (dict(sdx=7), EINVAL), (dict(p=-1.0), EINVAL), (dict(eps=-1.0), EINVAL)])
def test_norm_gradient_refusals(change, want):
    a = dict(type=1, rtype=0, M=4, D=8, dy=P[0], r=P[1], dr=P[2], dx=P[3], ds=P[4], sdy=8, sr=8,
             sdr=8, sdx=8, sds=8, w=P[5], dw=P[6], eps=1e-5, p=0.0, seed=0, offset=0, ws=P[7])
    a.update(change)
    assert lib().finc_add_norm_backward(finc.NORM_GRAD_ARGS.pack(*a.values()), None) == want
    assert lib().finc_add_norm_backward(None, None) == EINVAL


def test_nothing_to_do_is_no_error():
    """Empty batches: no HIP call, whatever the addresses."""
    none = (0, 0, 0)
    assert lib().finc_causal_conv_forward(conv(B=0, x=none, y=none, state=0, after=0, lengths=0),
                                          None) == finc.OK
    assert lib().finc_selective_scan_forward(
        scan(B=0, x=none, dt=none, z=none, Bm=none, Cm=none, y=none, state=0, after=0, states=0,
             lengths=0), None) == finc.OK
    assert lib().finc_dropout(1, None, 8, None, 8, None, 8, 0, 8, 0.1, 0, 0, None) == finc.OK


def test_sizes():
    L = lib()
    assert L.finc_causal_conv_workspace_bytes(2, 6, 40, 9) == 0
    assert L.finc_causal_conv_workspace_bytes(2, 6, 40, 4) % 256 == 0
    assert L.finc_selective_scan_states_bytes(2, 6, 40, 65) == 0
    assert L.finc_selective_scan_workspace_bytes(2, 6, 40, 16, 4) == 0
    assert L.finc_add_norm_workspace_bytes(4, 16385) == 0
    for n, parts in ((64, 1), (65, 1), (128, 1), (129, 2), (1000, 8)):
        assert L.finc_selective_scan_states_bytes(4, 8, n, 16) == 4 * 8 * parts * 16 * 4, n
    assert L.finc_selective_scan_states_bytes(4, 8, 129, 5) == 4 * 8 * 2 * 8 * 4
    assert L.finc_selective_scan_states_bytes(4, 8, 129, 20) == 4 * 8 * 3 * 32 * 4
    assert L.finc_dropout_counters(5, 17) == 15 and L.finc_dropout_counters(0, 8) == 0
    assert L.finc_dropout_counters(-1, 8) == 0 and L.finc_dropout_counters(4, 0) == 0


def test_host_tensors_are_refused():
    x, w = torch.zeros(2, 6, 40), torch.zeros(6, 4)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        finc.causal_conv_forward(x, w)
    with pytest.raises(ValueError, match="expected \\(B, D, L\\)"):
        finc.causal_conv_forward(x[0], w)
    with pytest.raises(ValueError, match="9 taps"):
        finc.causal_conv_forward(x, torch.zeros(6, 9))
    with pytest.raises(ValueError, match="x must be a device tensor"):
        finc.dropout(x, 0.1, 0)
    with pytest.raises(ValueError, match="must be a device tensor"):
        finc.add_norm_forward(x, w)
    A, Bm = torch.zeros(6, 16), torch.zeros(2, 4, 16, 40)
    with pytest.raises(ValueError, match="4 groups do not divide 6"):
        finc.selective_scan_forward(x, x, A, Bm, Bm)
    with pytest.raises(ValueError, match="65 states"):
        finc.selective_scan_forward(x, x, torch.zeros(6, 65), Bm, Bm)


# ---- registers ----------------------------------------------------------------------


def test_sequence_kernels_keep_their_registers():
    """Four waves a SIMD forward, two in the scan's gradients, and no spills but for
    the widest instances."""
    ks = {n: k for n, k in kernels().items()
          if re.search("scan_|conv_forward|conv_backward|norm_|dropout", n) and "finc" not in n[:6]}
    fwd = [k for n, k in ks.items() if "19scan_forward_kernelI" in n]
    back = [k for n, k in ks.items() if "20scan_backward_kernelI" in n]
    assert len(fwd) == 6 and len(back) == 24
    for k in fwd:
        assert waves(k) >= 4 and k[".vgpr_spill_count"] == 0, k[".name"]
    for k in back:   # sixteen states a lane do not fit beside their gradients
        many = re.search("Li4ELi16EE", k[".name"])
        assert waves(k) >= 2 and k[".vgpr_spill_count"] <= (64 if many else 0), k[".name"]
    for n, k in ks.items():
        if "norm_" in n:
            assert k[".vgpr_spill_count"] <= (8 if "Li1024ELi2E" in n else 0), n
        elif "scan_backward" not in n:
            assert k[".vgpr_spill_count"] == 0, n
