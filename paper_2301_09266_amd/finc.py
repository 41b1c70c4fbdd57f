"""Python binding of libfinc (include/finc.h): argument marshalling only.

Every function takes and returns torch tensors on the current HIP device and
enqueues on torch's current stream; all arithmetic runs in the HIP kernels of
csrc/.  There is no fallback: if the library is missing or a call
fails, FincError is raised.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc", "libfinc.so")

TL, TR, BL, BR = 0, 1, 2, 3
OK, EINVAL, ESINGULAR, EUNSUPPORTED, EHIP = 0, -1, -2, -3, -4
PLAN_LAYER, PLAN_UNIT, PLAN_SPLIT, PLAN_STACK = 0, 1, 2, 3

_vp = ctypes.c_void_p
_i = ctypes.c_int
_sz = ctypes.c_size_t

_ll = ctypes.c_longlong
_ull = ctypes.c_ulonglong
_d = ctypes.c_double
F32, BF16, F16 = 0, 1, 2
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
MAX_TAPS, MAX_STATE, MAX_ROW, MAX_HEAD, ATTENTION_PART = 8, 64, 16384, 128, 512
_ACTS = {None: 0, "relu": 1, "silu": 2, "gelu": 3}

# The sequence operators' argument structures, in the header's order of fields and
# with the platform's alignment (packing takes a fraction of a ctypes structure's
# time, which counts where a call takes a few microseconds).  A raster is "Pqq", heads
# are "Pqqq".
CONV_ARGS = struct.Struct("@6i Pqq Pqq 5P")
CONV_GRADS = struct.Struct("@Pqq Pqq 5P")
SCAN_ARGS = struct.Struct("@7i Pqq Pqq Pqq Pqq Pqq Pqq 7P")
SCAN_GRADS = struct.Struct("@Pqq Pqq Pqq Pqq Pqq Pqq 6P")
SCAN_STEP_ARGS = struct.Struct("@7i 5P 6q 6P")
NORM_ARGS = struct.Struct("@4i 4P 4q 2P 2d 2Q")
NORM_GRAD_ARGS = struct.Struct("@4i 5P 5q 2P 2d 2Q P")
ATTENTION_ARGS = struct.Struct("@7i Pqqq Pqqq Pqqq Pqqq Pqqq 5P d")
ATTENTION_GRADS = struct.Struct("@Pqqq Pqqq Pqqq Pqqq Pqqq 3P")
ATTENTION_STEP_ARGS = struct.Struct("@7i Pqqq Pqqq Pqqq Pqqq Pqqq 3P d")
LINEAR_ARGS = struct.Struct("@5i 5P 5q 2P")
LINEAR_GRAD_ARGS = struct.Struct("@5i 6P 6q 2P")

# name -> (restype, argtypes); mirrors include/finc.h
SIGNATURES = {
    "finc_version": (_i, []),
    "finc_strerror": (ctypes.c_char_p, [_i]),
    "finc_inverse_plan": (_i, [_i, _i, _i, _i, _i, _i, _i, ctypes.POINTER(_i), _i]),
    "finc_forward_plan": (_i, [_i, _i, _i, _i, _i, _i, _i, ctypes.POINTER(_i)]),
    "finc_inverse_steps": (_i, [_i, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _i, _vp]),
    "finc_inverse_timeline": (_i, [_i, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _i, _vp]),
    "finc_banded_plan": (_i, [_i, _i, _i, _i, ctypes.POINTER(_i)]),
    "finc_banded_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "finc_inverse_banded": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_unit_inverse_banded": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_workspace_bytes": (_sz, [_i, _i, _i]),
    "finc_prepare": (_i, [_vp, _i, ctypes.POINTER(_i), _i, _i, _vp, _vp]),
    "finc_forward": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "finc_logdet": (_i, [_vp, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_inverse": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_inverse_prepared": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "finc_inverse_noalloc": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp]),
    "finc_backward_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_backward": (_i, [_vp, _vp, _vp, _vp, _vp, ctypes.c_double, _i, _i, _i, _i, _i, _i,
                           _vp, _vp]),
    "finc_unit_backward_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_unit_backward": (_i, [_vp, _vp, _vp, _vp, _vp, ctypes.c_double, _i, _i, _i, _i, _i,
                                _vp, _vp]),
    "finc_split_backward_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_split_backward": (_i, [_vp, _vp, _vp, _vp, _vp, ctypes.c_double, _i, _i, _i, _i, _i,
                                 _vp, _vp]),
    "finc_actnorm_backward_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "finc_actnorm_backward": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_double, _i, _i, _i,
                                   _i, _vp, _vp]),
    "finc_gauss_nll": (_i, [ctypes.POINTER(_vp), ctypes.POINTER(ctypes.c_longlong), _i, _i, _vp,
                            _vp, _vp, _vp]),
    "finc_stack_train_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "finc_stack_forward": (_i, [_vp, ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, _i, _i, _i, _i,
                                _i, _i, _i, _vp, _vp]),
    "finc_stack_backward": (_i, [_vp, ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                 ctypes.c_double, _i, _i, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_unit_forward": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "finc_unit_logdet": (_i, [_vp, _i, _i, _i, _i, _vp, _vp]),
    "finc_unit_inverse": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_unit_inverse_prepared": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "finc_split_forward": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "finc_split_logdet": (_i, [_vp, _i, _i, _i, _i, _vp, _vp]),
    "finc_split_inverse": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_split_inverse_prepared": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "finc_stack_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "finc_stack_inverse": (_i, [ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i,
                                _i, _i, _vp, _vp]),
    "finc_stack_prepare": (_i, [_vp, _i, _i, _i, _i, _vp, _vp]),
    "finc_stack_inverse_prepared": (_i, [ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, _i, _i,
                                         _i, _i, _i, _i, _i, _vp]),
    "finc_step_param_count": (_sz, [_i, _i, _i]),
    "finc_step_prepared_bytes": (_sz, [_i, _i]),
    "finc_step_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_step_prepare": (_i, [_vp, _i, _i, _i, _vp, _vp]),
    "finc_step_forward": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_step_inverse": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_flow_param_count": (_sz, [_i, _i, _i, _i, _i]),
    "finc_flow_prepared_bytes": (_sz, [_i, _i, _i, _i]),
    "finc_flow_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "finc_flow_prepare": (_i, [_vp, _i, _i, _i, _i, _i, _vp, _vp]),
    "finc_flow_forward": (_i, [_vp, ctypes.POINTER(_vp), _vp, _vp, _vp, _i, _i, _i, _i, _i, _i,
                               _i, _i, _vp, _vp]),
    "finc_flow_sample": (_i, [ctypes.POINTER(_vp), _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i,
                              _i, _vp, _vp]),
    "finc_conv1x1_workspace_bytes": (_sz, [_i]),
    "finc_conv1x1_forward": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _vp]),
    "finc_conv1x1_inverse": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _vp, _vp]),
    "finc_causal_conv_forward": (_i, [_vp, _vp]),
    "finc_causal_conv_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "finc_causal_conv_backward": (_i, [_vp, _vp, _vp]),
    "finc_causal_conv_step": (_i, [_i, _vp, _ll, _vp, _ll, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i,
                                   _vp]),
    "finc_selective_scan_states_bytes": (_sz, [_i, _i, _i, _i]),
    "finc_selective_scan_forward": (_i, [_vp, _vp]),
    "finc_selective_scan_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_selective_scan_backward": (_i, [_vp, _vp,
                                          _vp]),
    "finc_selective_scan_step": (_i, [_vp, _vp]),
    "finc_dropout_counters": (_ull, [_i, _i]),
    "finc_dropout": (_i, [_i, _vp, _ll, _vp, _ll, _vp, _ll, _i, _i, _d, _ull, _ull, _vp]),
    "finc_add_norm_forward": (_i, [_vp, _vp]),
    "finc_add_norm_workspace_bytes": (_sz, [_i, _i]),
    "finc_add_norm_backward": (_i, [_vp, _vp]),
    "finc_linear_attention_states_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_linear_attention_forward": (_i, [_vp, _vp]),
    "finc_linear_attention_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "finc_linear_attention_backward": (_i, [_vp, _vp, _vp]),
    "finc_linear_attention_step": (_i, [_vp, _vp]),
    "finc_linear_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "finc_linear_forward": (_i, [_vp, _vp]),
    "finc_linear_grad_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "finc_linear_backward": (_i, [_vp, _vp]),
    "finc_embed_forward": (_i, [_i, _i, _vp, _i, _vp, _ll, _vp, _ll, _i, _i, _i, _d, _vp]),
    "finc_embed_workspace_bytes": (_sz, [_i, _i, _i]),
    "finc_embed_backward": (_i, [_i, _vp, _i, _vp, _ll, _vp, _i, _i, _i, _d, _vp, _vp]),
}


class FincError(RuntimeError):
    def __init__(self, code: int, what: str):
        msg = _lib.finc_strerror(code).decode() if _lib is not None else str(code)
        super().__init__(f"{what}: {msg} ({code})")
        self.code = code


_lib = None


def lib(path: str = LIB_PATH):
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(
            f"libfinc is not built ({path}); run __graft_entry__.build() first")
    handle = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(handle, name)
        fn.restype = res
        fn.argtypes = args
    _lib = handle
    return _lib


def _require_lib():
    return lib()


def _check(code: int, what: str):
    if code != OK:
        raise FincError(code, what)


def _ptr(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# torch's current stream and device without the objects around them (2.8 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def _dev(t: torch.Tensor, name: str, shape=None):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != torch.float32:
        raise ValueError(f"{name} must be float32")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _logdet_out(t: torch.Tensor | None):
    if t is None:
        return None
    if not t.is_cuda or t.dtype != torch.float64 or t.numel() < 1:
        raise ValueError("logdet must be a device float64 tensor with at least one element")
    return t


def _bytes_buf(t: torch.Tensor, nbytes: int, name: str):
    """A device buffer of at least nbytes (prepared weights, workspaces)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{name} holds {t.numel() * t.element_size()} bytes, needs {nbytes}")
    return t


def _workspace(nbytes: int, device, ws):
    if ws is None:
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    return _bytes_buf(ws, nbytes, "workspace")


# ---------------------------------------------------------------------------

def version() -> int:
    return _require_lib().finc_version()


def inverse_plan(kind: int, C: int, H: int, W: int, k: int, L: int = 1, U: int = 1):
    """The inverse kernel launches a call would make (finc_inverse_plan): a
    list of dicts (threads, mode, groups, streamed, lds, compact), one per
    distinct launch, or the negative status (EUNSUPPORTED, EINVAL)."""
    info = (ctypes.c_int * (6 * 8))()
    n = _require_lib().finc_inverse_plan(kind, L, U, C, H, W, k, info, 8)
    if n < 0:
        return n
    keys = ("threads", "mode", "groups", "streamed", "lds", "compact")
    return [dict(zip(keys, info[6 * i:6 * i + 6])) for i in range(n)]


def forward_plan(kind: int, B: int, C: int, H: int, W: int, k: int, in_place: bool = False):
    """The forward's row blocks (finc_forward_plan): dict(blocks, rows, lds),
    or the negative status (EUNSUPPORTED when a block does not fit)."""
    info = (ctypes.c_int * 3)()
    rc = _require_lib().finc_forward_plan(kind, B, C, H, W, k, int(in_place), info)
    if rc < 0:
        return rc
    return dict(blocks=info[0], rows=info[1], lds=info[2])


def workspace_bytes(C: int, k: int, n_layers: int = 1) -> int:
    return int(_require_lib().finc_workspace_bytes(C, k, n_layers))


def stack_workspace_bytes(L: int, U: int, C1: int, k: int) -> int:
    return int(_require_lib().finc_stack_workspace_bytes(L, U, C1, k))


def prepare(K: torch.Tensor, corners, out: torch.Tensor | None = None) -> torch.Tensor:
    """K: (n, C, C, k, k) or (C, C, k, k); corners: one id per layer."""
    L = _require_lib()
    _dev(K, "K")
    if K.dim() not in (4, 5) or K.shape[-4] != K.shape[-3] or K.shape[-2] != K.shape[-1]:
        raise ValueError(f"K has shape {tuple(K.shape)}, expected ([n,] C, C, k, k)")
    n = 1 if K.dim() == 4 else K.shape[0]
    C, k = K.shape[-3], K.shape[-1]
    corners = [int(c) for c in (corners if hasattr(corners, "__len__") else [corners])]
    if len(corners) != n:
        raise ValueError("one corner per layer")
    out = _workspace(workspace_bytes(C, k, n), K.device, out)
    arr = (ctypes.c_int * n)(*corners)
    _check(L.finc_prepare(_ptr(K), n, arr, C, k, _ptr(out), _stream()), "finc_prepare")
    return out


def forward(x: torch.Tensor, K: torch.Tensor, corner: int, out: torch.Tensor | None = None,
            logdet: torch.Tensor | None = None, prepared: torch.Tensor | None = None):
    """y = layer(x); with `logdet` (a device float64 tensor of one element) the
    same launch also writes the layer's log|det|; with `prepared` (a uint8
    device tensor of workspace_bytes(C, k, 1)) it also writes the weights
    prepared for inverse_prepared."""
    L = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    k = K.shape[-1]
    _dev(K, "K", (C, C, k, k))
    y = torch.empty_like(x) if out is None else _dev(out, "out", x.shape)
    pp = None if prepared is None else _workspace(workspace_bytes(C, k, 1), x.device, prepared)
    _check(L.finc_forward(_ptr(x), _ptr(y), _ptr(K), _ptr(_logdet_out(logdet)), _ptr(pp), B, C,
                          H, W, k, corner, _stream()), "finc_forward")
    return y


def logdet(K: torch.Tensor, corner: int, H: int, W: int, out: torch.Tensor | None = None):
    L = _require_lib()
    _dev(K, "K")
    out = torch.empty(1, dtype=torch.float64, device=K.device) if out is None else out
    _check(L.finc_logdet(_ptr(K), K.shape[0], K.shape[-1], corner, H, W, _ptr(out),
                         _stream()), "finc_logdet")
    return out


def inverse(y: torch.Tensor, K: torch.Tensor, corner: int, out: torch.Tensor | None = None,
            workspace: torch.Tensor | None = None):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    k = K.shape[-1]
    _dev(K, "K", (C, C, k, k))
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    ws = _workspace(workspace_bytes(C, k, 1), y.device, workspace)
    _check(L.finc_inverse(_ptr(y), _ptr(x), _ptr(K), B, C, H, W, k, corner, _ptr(ws),
                          _stream()), "finc_inverse")
    return x


def inverse_noalloc(y: torch.Tensor, K: torch.Tensor, corner: int,
                    out: torch.Tensor | None = None):
    """finc_inverse with the library's own device array for the prepared
    weights (no workspace); calls on one device must not overlap."""
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    k = K.shape[-1]
    _dev(K, "K", (C, C, k, k))
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    _check(L.finc_inverse_noalloc(_ptr(y), _ptr(x), _ptr(K), B, C, H, W, k, corner, _stream()),
           "finc_inverse_noalloc")
    return x


def inverse_prepared(y: torch.Tensor, prepared: torch.Tensor, k: int, corner: int,
                     out: torch.Tensor | None = None):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    _bytes_buf(prepared, workspace_bytes(C, k, 1), "prepared")
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    _check(L.finc_inverse_prepared(_ptr(y), _ptr(x), _ptr(prepared), B, C, H, W, k, corner,
                                   _stream()), "finc_inverse_prepared")
    return x


def inverse_steps(y: torch.Tensor, prepared: torch.Tensor, k: int, corner: int = TL,
                  split: bool = False):
    """(x, steps): the inverse of a prepared layer (or, split=True, of a
    prepared channel-split unit) and the number of diagonal steps every wave
    of every workgroup ran, as (workgroups, waves) int32 (see
    finc_inverse_steps)."""
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    kind = PLAN_SPLIT if split else PLAN_LAYER
    _bytes_buf(prepared, workspace_bytes(C // 4 if split else C, k, 4 if split else 1),
               "prepared")
    info = inverse_plan(kind, C, H, W, k)
    if isinstance(info, int):
        _check(info, "finc_inverse_steps")
    waves = info[0]["threads"] // 64
    nwg = (4 * B if split else B)
    steps = torch.full((nwg, waves), -1, dtype=torch.int32, device=y.device)
    x = torch.empty_like(y)
    n = L.finc_inverse_steps(kind, _ptr(y), _ptr(x), _ptr(prepared), B, C, H, W, k, corner,
                             _ptr(steps), steps.numel(), _stream())
    if n < 0:
        _check(n, "finc_inverse_steps")
    return x, steps


def inverse_timeline(y: torch.Tensor, prepared: torch.Tensor, k: int, corner: int = TL,
                     split: bool = False):
    """(x, stamps): the inverse of a prepared layer (or, split=True, of a
    prepared channel-split unit) and, for every wave of every workgroup, the
    GPU's 100 MHz clock when its arguments arrived, its set-up was done, its
    last step was done and its store was issued, as (workgroups, waves, 4)
    int64 (see finc_inverse_timeline)."""
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    kind = PLAN_SPLIT if split else PLAN_LAYER
    _bytes_buf(prepared, workspace_bytes(C // 4 if split else C, k, 4 if split else 1),
               "prepared")
    info = inverse_plan(kind, C, H, W, k)
    if isinstance(info, int):
        _check(info, "finc_inverse_timeline")
    waves = info[0]["threads"] // 64
    nwg = (4 * B if split else B)
    stamps = torch.full((nwg, waves, 4), -1, dtype=torch.int64, device=y.device)
    x = torch.empty_like(y)
    n = L.finc_inverse_timeline(kind, _ptr(y), _ptr(x), _ptr(prepared), B, C, H, W, k, corner,
                                _ptr(stamps), stamps.numel(), _stream())
    if n < 0:
        _check(n, "finc_inverse_timeline")
    return x, stamps


def banded_plan(C: int, H: int, W: int, k: int):
    """dict(threads, rows, bands, lds) of the banded stream form
    (finc_banded_plan), or the negative status."""
    info = (ctypes.c_int * 4)()
    rc = _require_lib().finc_banded_plan(C, H, W, k, info)
    if rc < 0:
        return rc
    return dict(threads=info[0], rows=info[1], bands=info[2], lds=info[3])


def _banded(fn, y, K, n_layers, corner, out, workspace):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    k = K.shape[-1]
    _dev(K, "K", (C, C, k, k) if n_layers == 1 else (4, C, C, k, k))
    nbytes = int(L.finc_banded_workspace_bytes(B, C, H, W, k, n_layers))
    if nbytes == 0:
        raise FincError(EUNSUPPORTED if isinstance(banded_plan(C, H, W, k), int) else EINVAL, fn)
    ws = _workspace(nbytes, y.device, workspace)
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    args = (_ptr(y), _ptr(x), _ptr(K), B, C, H, W, k) + ((corner,) if n_layers == 1 else ())
    _check(getattr(L, fn)(*args, _ptr(ws), _stream()), fn)
    return x, ws


def inverse_banded(y, K, corner: int, out=None, workspace=None):
    """(x, workspace) of finc_inverse_banded; the workspace's int at byte
    offset workspace_bytes(C, k, 1) is the timeout flag."""
    return _banded("finc_inverse_banded", y, K, 1, corner, out, workspace)


def unit_inverse_banded(y, K4, out=None, workspace=None):
    """(x, workspace) of finc_unit_inverse_banded (timeout flag at byte
    offset workspace_bytes(C, k, 4))."""
    return _banded("finc_unit_inverse_banded", y, K4, 4, TL, out, workspace)


def backward(x: torch.Tensor, dy: torch.Tensor, K: torch.Tensor, corner: int,
             gld: float = 0.0, want_dx: bool = True, want_dK: bool = True,
             dx: torch.Tensor | None = None, dK: torch.Tensor | None = None,
             workspace: torch.Tensor | None = None):
    """(dx, dK) of one layer for the loss gradient dy (see finc_backward);
    either is None when not wanted."""
    L = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    _dev(dy, "dy", x.shape)
    k = K.shape[-1]
    _dev(K, "K", (C, C, k, k))
    if want_dx:
        dx = torch.empty_like(x) if dx is None else _dev(dx, "dx", x.shape)
    else:
        dx = None
    if want_dK:
        dK = torch.empty_like(K) if dK is None else _dev(dK, "dK", K.shape)
    else:
        dK = None
    ws = _workspace(int(L.finc_backward_workspace_bytes(B, C, H, W, k)), x.device, workspace)
    _check(L.finc_backward(_ptr(x), _ptr(dy), _ptr(K), _ptr(dx), _ptr(dK), float(gld), B, C, H,
                           W, k, corner, _ptr(ws), _stream()), "finc_backward")
    return dx, dK


def _unit_grads(fn, wsfn, x, dy, Kw, wshape, gld, want_dx, want_dK, dx, dKw, workspace):
    L = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    _dev(dy, "dy", x.shape)
    k = Kw.shape[-1]
    _dev(Kw, "K", wshape(C, k))
    dx = (torch.empty_like(x) if dx is None else _dev(dx, "dx", x.shape)) if want_dx else None
    dKw = ((torch.empty_like(Kw) if dKw is None else _dev(dKw, "dK", Kw.shape))
           if want_dK else None)
    nbytes = int(getattr(L, wsfn)(B, C, H, W, k))
    if nbytes == 0:
        raise FincError(EINVAL, fn)
    ws = _workspace(nbytes, x.device, workspace)
    _check(getattr(L, fn)(_ptr(x), _ptr(dy), _ptr(Kw), _ptr(dx), _ptr(dKw), float(gld), B, C, H,
                          W, k, _ptr(ws), _stream()), fn)
    return dx, dKw


def unit_backward(x, dy, K4, gld: float = 0.0, want_dx: bool = True, want_dK: bool = True,
                  dx=None, dK4=None, workspace=None):
    """(dx, dK4) of the sequential unit (see finc_unit_backward); K4 is
    (4, C, C, k, k)."""
    return _unit_grads("finc_unit_backward", "finc_unit_backward_workspace_bytes", x, dy, K4,
                       lambda C, k: (4, C, C, k, k), gld, want_dx, want_dK, dx, dK4, workspace)


def split_backward(x, dy, Kq4, gld: float = 0.0, want_dx: bool = True, want_dK: bool = True,
                   dx=None, dKq4=None, workspace=None):
    """(dx, dKq4) of the channel-split unit (see finc_split_backward); Kq4 is
    (4, C/4, C/4, k, k)."""
    return _unit_grads("finc_split_backward", "finc_split_backward_workspace_bytes", x, dy,
                       Kq4, lambda C, k: (4, C // 4, C // 4, k, k), gld, want_dx, want_dK, dx,
                       dKq4, workspace)


def actnorm_backward(x, dy, s, gld: float = 0.0, workspace=None):
    """(dx, ds, db) of actnorm y = s x + b (see finc_actnorm_backward)."""
    L = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    _dev(dy, "dy", x.shape)
    _dev(s, "s", (C,))
    dx, ds, db = torch.empty_like(x), torch.empty_like(s), torch.empty_like(s)
    nbytes = int(L.finc_actnorm_backward_workspace_bytes(B, C, H, W))
    if nbytes == 0:
        raise FincError(EINVAL, "finc_actnorm_backward")
    ws = _workspace(nbytes, x.device, workspace)
    _check(L.finc_actnorm_backward(_ptr(x), _ptr(dy), _ptr(s), _ptr(dx), _ptr(ds), _ptr(db),
                                   float(gld), B, C, H, W, _ptr(ws), _stream()),
           "finc_actnorm_backward")
    return dx, ds, db


def _stack_latents(B, L_levels, C1, H1, W1, device):
    return [torch.empty((B, (C1 << l) if l == L_levels - 1 else (C1 << l) // 2, H1 >> l, W1 >> l),
                        device=device) for l in range(L_levels)]


def stack_forward(x, K, scale, bias, L_levels: int, U: int, k: int, workspace=None):
    """(latents, logdet) of the stack's forward direction (finc_stack_forward);
    K, scale, bias flat in the stack's layout."""
    L = _require_lib()
    _dev(x, "x")
    B, C1, H1, W1 = x.shape
    _stack_params(L_levels, U, C1, k, scale, bias, K)
    z = _stack_latents(B, L_levels, C1, H1, W1, x.device)
    zp = (ctypes.c_void_p * L_levels)(*[t.data_ptr() for t in z])
    ld = torch.empty(B, dtype=torch.float64, device=x.device)
    nbytes = int(L.finc_stack_train_workspace_bytes(B, L_levels, U, C1, H1, W1, k))
    if nbytes == 0:
        raise FincError(EINVAL, "finc_stack_forward")
    ws = _workspace(nbytes, x.device, workspace)
    _check(L.finc_stack_forward(_ptr(x), zp, _ptr(ld), _ptr(K), _ptr(scale), _ptr(bias), B,
                                L_levels, U, C1, H1, W1, k, _ptr(ws), _stream()),
           "finc_stack_forward")
    return z, ld


def stack_backward(x, dz, K, scale, bias, L_levels: int, U: int, k: int, gld: float = 0.0,
                   want_dx: bool = True, workspace=None):
    """(dx, dK, dscale, dbias) of the stack's forward direction for latent
    gradients dz (finc_stack_backward); dx is None when not wanted."""
    L = _require_lib()
    _dev(x, "x")
    B, C1, H1, W1 = x.shape
    _stack_params(L_levels, U, C1, k, scale, bias, K)
    zp = _stack_args(dz, L_levels, C1, H1, W1)
    dx = torch.empty_like(x) if want_dx else None
    dK, ds, db = torch.empty_like(K), torch.empty_like(scale), torch.empty_like(bias)
    nbytes = int(L.finc_stack_train_workspace_bytes(B, L_levels, U, C1, H1, W1, k))
    if nbytes == 0:
        raise FincError(EINVAL, "finc_stack_backward")
    ws = _workspace(nbytes, x.device, workspace)
    _check(L.finc_stack_backward(_ptr(x), zp, _ptr(K), _ptr(scale), _ptr(bias), _ptr(dx),
                                 _ptr(dK), _ptr(ds), _ptr(db), float(gld), B, L_levels, U, C1,
                                 H1, W1, k, _ptr(ws), _stream()), "finc_stack_backward")
    return dx, dK, ds, db


def gauss_nll(zs, logdet):
    """(nll, bpd) per image (device float64, B each) for latents zs (float32
    tensors with the batch first) and per-image log|det| (float64, B); see
    finc_gauss_nll."""
    L = _require_lib()
    if not logdet.is_cuda or logdet.dtype != torch.float64 or logdet.dim() != 1:
        raise ValueError("logdet must be a 1-d float64 device tensor")
    B = logdet.shape[0]
    for z in zs:
        _dev(z, "z")
        if z.shape[0] != B:
            raise ValueError(f"latent has batch {z.shape[0]}, expected {B}")
    n = (ctypes.c_longlong * len(zs))(*[math.prod(z.shape[1:]) for z in zs])
    ptrs = (_vp * len(zs))(*[z.data_ptr() for z in zs])
    nll = torch.empty(B, dtype=torch.float64, device=logdet.device)
    bpd = torch.empty_like(nll)
    _check(L.finc_gauss_nll(ptrs, n, len(zs), B, _ptr(logdet), _ptr(nll), _ptr(bpd), _stream()),
           "finc_gauss_nll")
    return nll, bpd


def unit_forward(x: torch.Tensor, K4: torch.Tensor, out: torch.Tensor | None = None,
                 logdet: torch.Tensor | None = None, prepared: torch.Tensor | None = None):
    """The unit (TL, TR, BL, BR); optional side outputs as for forward, with
    `prepared` of workspace_bytes(C, k, 4) for unit_inverse_prepared."""
    L = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    k = K4.shape[-1]
    _dev(K4, "K4", (4, C, C, k, k))
    y = torch.empty_like(x) if out is None else _dev(out, "out", x.shape)
    pp = None if prepared is None else _workspace(workspace_bytes(C, k, 4), x.device, prepared)
    _check(L.finc_unit_forward(_ptr(x), _ptr(y), _ptr(K4), _ptr(_logdet_out(logdet)), _ptr(pp),
                               B, C, H, W, k, _stream()), "finc_unit_forward")
    return y


def unit_logdet(K4: torch.Tensor, H: int, W: int, out: torch.Tensor | None = None):
    L = _require_lib()
    _dev(K4, "K4")
    out = torch.empty(1, dtype=torch.float64, device=K4.device) if out is None else out
    _check(L.finc_unit_logdet(_ptr(K4), K4.shape[1], K4.shape[-1], H, W, _ptr(out),
                              _stream()), "finc_unit_logdet")
    return out


def unit_inverse(y: torch.Tensor, K4: torch.Tensor, out: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    k = K4.shape[-1]
    _dev(K4, "K4", (4, C, C, k, k))
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    ws = _workspace(workspace_bytes(C, k, 4), y.device, workspace)
    _check(L.finc_unit_inverse(_ptr(y), _ptr(x), _ptr(K4), B, C, H, W, k, _ptr(ws),
                               _stream()), "finc_unit_inverse")
    return x


def unit_inverse_prepared(y: torch.Tensor, prepared4: torch.Tensor, k: int,
                          out: torch.Tensor | None = None):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    _bytes_buf(prepared4, workspace_bytes(C, k, 4), "prepared4")
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    _check(L.finc_unit_inverse_prepared(_ptr(y), _ptr(x), _ptr(prepared4), B, C, H, W, k,
                                        _stream()), "finc_unit_inverse_prepared")
    return x


# channel-split unit (four quarter-channel PCBs side by side; quarter g has
# corner g): Kq4 of shape (4, C/4, C/4, k, k)

def split_forward(x: torch.Tensor, Kq4: torch.Tensor, out: torch.Tensor | None = None,
                  logdet: torch.Tensor | None = None, prepared: torch.Tensor | None = None):
    """Optional side outputs as for forward, with `prepared` of
    workspace_bytes(C/4, k, 4) for split_inverse_prepared."""
    L = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    k = Kq4.shape[-1]
    _dev(Kq4, "Kq4", (4, C // 4, C // 4, k, k))
    y = torch.empty_like(x) if out is None else _dev(out, "out", x.shape)
    pp = None if prepared is None else _workspace(workspace_bytes(C // 4, k, 4), x.device,
                                                  prepared)
    _check(L.finc_split_forward(_ptr(x), _ptr(y), _ptr(Kq4), _ptr(_logdet_out(logdet)), _ptr(pp),
                                B, C, H, W, k, _stream()), "finc_split_forward")
    return y


def split_logdet(Kq4: torch.Tensor, H: int, W: int, out: torch.Tensor | None = None):
    L = _require_lib()
    _dev(Kq4, "Kq4")
    out = torch.empty(1, dtype=torch.float64, device=Kq4.device) if out is None else out
    _check(L.finc_split_logdet(_ptr(Kq4), 4 * Kq4.shape[1], Kq4.shape[-1], H, W, _ptr(out),
                               _stream()), "finc_split_logdet")
    return out


def split_inverse(y: torch.Tensor, Kq4: torch.Tensor, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    k = Kq4.shape[-1]
    _dev(Kq4, "Kq4", (4, C // 4, C // 4, k, k))
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    ws = _workspace(workspace_bytes(C // 4, k, 4), y.device, workspace)
    _check(L.finc_split_inverse(_ptr(y), _ptr(x), _ptr(Kq4), B, C, H, W, k, _ptr(ws),
                                _stream()), "finc_split_inverse")
    return x


def split_inverse_prepared(y: torch.Tensor, prepared4: torch.Tensor, k: int,
                           out: torch.Tensor | None = None):
    L = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    _bytes_buf(prepared4, workspace_bytes(C // 4, k, 4), "prepared4")
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    _check(L.finc_split_inverse_prepared(_ptr(y), _ptr(x), _ptr(prepared4), B, C, H, W, k,
                                         _stream()), "finc_split_inverse_prepared")
    return x


def _stack_args(z, L_levels, C1, H1, W1):
    """Latents z[l]: (B, C_l / 2, H_l, W_l) below the top, (B, C_top, H_top,
    W_top) at the top, C_l = C1 2^l, H_l = H1 / 2^l."""
    if len(z) != L_levels:
        raise ValueError("one latent per level")
    B = z[0].shape[0] if z[0].dim() == 4 else -1
    for l, t in enumerate(z):
        C = C1 << l
        _dev(t, f"z[{l}]", (B, C if l == L_levels - 1 else C // 2, H1 >> l, W1 >> l))
    return (ctypes.c_void_p * L_levels)(*[t.data_ptr() for t in z])


def _stack_params(L_levels, U, C1, k, scale, bias, K=None):
    """scale, bias: U * sum_l C_l floats; K: U * 4 * sum_l C_l^2 k^2 floats."""
    chans = sum(C1 << l for l in range(L_levels))
    for name, t in (("scale", scale), ("bias", bias)):
        _dev(t, name)
        if t.numel() != U * chans:
            raise ValueError(f"{name} has {t.numel()} elements, expected {U * chans}")
    if K is not None:
        _dev(K, "K")
        n = U * 4 * sum((C1 << l) ** 2 for l in range(L_levels)) * k * k
        if K.numel() != n:
            raise ValueError(f"K has {K.numel()} elements, expected {n}")


def stack_prepare(K: torch.Tensor, L: int, U: int, C1: int, k: int,
                  out: torch.Tensor | None = None):
    lb = _require_lib()
    _dev(K, "K")
    n = U * 4 * sum((C1 << l) ** 2 for l in range(L)) * k * k
    if K.numel() != n:
        raise ValueError(f"K has {K.numel()} elements, expected {n}")
    out = _workspace(stack_workspace_bytes(L, U, C1, k), K.device, out)
    _check(lb.finc_stack_prepare(_ptr(K), L, U, C1, k, _ptr(out), _stream()),
           "finc_stack_prepare")
    return out


def stack_inverse(z, K: torch.Tensor, scale: torch.Tensor, bias: torch.Tensor, L: int,
                  U: int, C1: int, H1: int, W1: int, k: int, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None):
    """z: list of L latents (see finc.h); K, scale, bias: flat device tensors."""
    lb = _require_lib()
    zp = _stack_args(z, L, C1, H1, W1)
    _stack_params(L, U, C1, k, scale, bias, K)
    B = z[0].shape[0]
    x = (torch.empty((B, C1, H1, W1), dtype=torch.float32, device=z[0].device)
         if out is None else _dev(out, "out", (B, C1, H1, W1)))
    ws = _workspace(stack_workspace_bytes(L, U, C1, k), z[0].device, workspace)
    _check(lb.finc_stack_inverse(zp, _ptr(x), _ptr(K), _ptr(scale), _ptr(bias), B, L, U, C1,
                                 H1, W1, k, _ptr(ws), _stream()), "finc_stack_inverse")
    return x


def stack_inverse_prepared(z, prepared: torch.Tensor, scale: torch.Tensor,
                           bias: torch.Tensor, L: int, U: int, C1: int, H1: int, W1: int,
                           k: int, out: torch.Tensor | None = None):
    lb = _require_lib()
    zp = _stack_args(z, L, C1, H1, W1)
    _stack_params(L, U, C1, k, scale, bias)
    _bytes_buf(prepared, stack_workspace_bytes(L, U, C1, k), "prepared")
    B = z[0].shape[0]
    x = (torch.empty((B, C1, H1, W1), dtype=torch.float32, device=z[0].device)
         if out is None else _dev(out, "out", (B, C1, H1, W1)))
    _check(lb.finc_stack_inverse_prepared(zp, _ptr(x), _ptr(prepared), _ptr(scale),
                                          _ptr(bias), B, L, U, C1, H1, W1, k, _stream()),
           "finc_stack_inverse_prepared")
    return x


# ---------------------------------------------------------------------------
# The full FInC Flow (Step and multi-scale flow; parameter layout in finc.h)

def conv1x1_forward(x: torch.Tensor, Wm: torch.Tensor, out: torch.Tensor | None = None,
                    logdet: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    lb = _require_lib()
    _dev(x, "x")
    B, C, H, W = x.shape
    _dev(Wm, "Wm", (C, C))
    y = torch.empty_like(x) if out is None else _dev(out, "out", x.shape)
    ws = _workspace(int(lb.finc_conv1x1_workspace_bytes(C)), x.device, workspace)
    _check(lb.finc_conv1x1_forward(_ptr(x), _ptr(y), _ptr(Wm), _ptr(_logdet_out(logdet)), B, C,
                                   H, W, _ptr(ws), _stream()), "finc_conv1x1_forward")
    return y


def conv1x1_inverse(y: torch.Tensor, Wm: torch.Tensor, out: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None):
    lb = _require_lib()
    _dev(y, "y")
    B, C, H, W = y.shape
    _dev(Wm, "Wm", (C, C))
    x = torch.empty_like(y) if out is None else _dev(out, "out", y.shape)
    ws = _workspace(int(lb.finc_conv1x1_workspace_bytes(C)), y.device, workspace)
    _check(lb.finc_conv1x1_inverse(_ptr(y), _ptr(x), _ptr(Wm), B, C, H, W, _ptr(ws), _stream()),
           "finc_conv1x1_inverse")
    return x


def step_param_count(C: int, k: int, hid: int) -> int:
    return int(_require_lib().finc_step_param_count(C, k, hid))


def step_prepare(sp: torch.Tensor, C: int, k: int, hid: int, out: torch.Tensor | None = None):
    lb = _require_lib()
    _dev(sp, "sp")
    if sp.numel() != step_param_count(C, k, hid):
        raise ValueError(f"sp has {sp.numel()} elements, expected {step_param_count(C, k, hid)}")
    pp = _workspace(int(lb.finc_step_prepared_bytes(C, k)), sp.device, out)
    _check(lb.finc_step_prepare(_ptr(sp), C, k, hid, _ptr(pp), _stream()), "finc_step_prepare")
    return pp


def _step_call(name, a, sp, prepared, k, hid, out, workspace, logdet=None):
    lb = _require_lib()
    _dev(a, "input")
    B, C, H, W = a.shape
    _dev(sp, "sp")
    if sp.numel() != step_param_count(C, k, hid):
        raise ValueError("sp does not match (C, k, hid)")
    _bytes_buf(prepared, int(lb.finc_step_prepared_bytes(C, k)), "prepared")
    b = torch.empty_like(a) if out is None else _dev(out, "out", a.shape)
    ws = _workspace(int(lb.finc_step_workspace_bytes(B, C, H, W, hid)), a.device, workspace)
    if name == "finc_step_forward":
        if logdet is not None and (not logdet.is_cuda or logdet.dtype != torch.float64 or
                                   logdet.numel() < B):
            raise ValueError("logdet must be a device float64 tensor of B elements")
        rc = lb.finc_step_forward(_ptr(a), _ptr(b), _ptr(logdet), _ptr(sp), _ptr(prepared), B, C,
                                  H, W, k, hid, _ptr(ws), _stream())
    else:
        rc = lb.finc_step_inverse(_ptr(a), _ptr(b), _ptr(sp), _ptr(prepared), B, C, H, W, k, hid,
                                  _ptr(ws), _stream())
    _check(rc, name)
    return b


def step_forward(x, sp, prepared, k: int, hid: int, out=None, logdet=None, workspace=None):
    """y = Step(x); logdet (B float64, device) is incremented if given."""
    return _step_call("finc_step_forward", x, sp, prepared, k, hid, out, workspace, logdet)


def step_inverse(y, sp, prepared, k: int, hid: int, out=None, workspace=None):
    return _step_call("finc_step_inverse", y, sp, prepared, k, hid, out, workspace)


def flow_param_count(L: int, K: int, C0: int, k: int, hid: int) -> int:
    return int(_require_lib().finc_flow_param_count(L, K, C0, k, hid))


def flow_latent_shapes(B: int, L: int, C0: int, H0: int, W0: int):
    return [(B, ((4 * C0) << l) // (1 if l == L - 1 else 2), H0 >> (l + 1), W0 >> (l + 1))
            for l in range(L)]


def flow_prepare(params: torch.Tensor, L: int, K: int, C0: int, k: int, hid: int,
                 out: torch.Tensor | None = None):
    lb = _require_lib()
    _dev(params, "params")
    if params.numel() != flow_param_count(L, K, C0, k, hid):
        raise ValueError("params does not match (L, K, C0, k, hid)")
    pp = _workspace(int(lb.finc_flow_prepared_bytes(L, K, C0, k)), params.device, out)
    _check(lb.finc_flow_prepare(_ptr(params), L, K, C0, k, hid, _ptr(pp), _stream()),
           "finc_flow_prepare")
    return pp


def _flow_common(params, prepared, L, K, C0, k, hid):
    lb = _require_lib()
    _dev(params, "params")
    if params.numel() != flow_param_count(L, K, C0, k, hid):
        raise ValueError("params does not match (L, K, C0, k, hid)")
    _bytes_buf(prepared, int(lb.finc_flow_prepared_bytes(L, K, C0, k)), "prepared")
    return lb


def flow_forward(x: torch.Tensor, params: torch.Tensor, prepared: torch.Tensor, L: int, K: int,
                 k: int, hid: int, workspace: torch.Tensor | None = None):
    """(latents z[0..L-1], logdet per image) of images x."""
    _dev(x, "x")
    B, C0, H0, W0 = x.shape
    lb = _flow_common(params, prepared, L, K, C0, k, hid)
    z = [torch.empty(s, dtype=torch.float32, device=x.device)
         for s in flow_latent_shapes(B, L, C0, H0, W0)]
    ld = torch.empty(B, dtype=torch.float64, device=x.device)
    ws = _workspace(int(lb.finc_flow_workspace_bytes(B, L, C0, H0, W0, hid)), x.device, workspace)
    zp = (ctypes.c_void_p * L)(*[t.data_ptr() for t in z])
    _check(lb.finc_flow_forward(_ptr(x), zp, _ptr(ld), _ptr(params), _ptr(prepared), B, L, K, C0,
                                H0, W0, k, hid, _ptr(ws), _stream()), "finc_flow_forward")
    return z, ld


def flow_sample(z, params: torch.Tensor, prepared: torch.Tensor, L: int, K: int, C0: int,
                H0: int, W0: int, k: int, hid: int, out: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None):
    """Images from latents z[0..L-1] (shapes as flow_latent_shapes)."""
    if len(z) != L:
        raise ValueError("one latent per level")
    B = z[0].shape[0]
    for l, (t, shp) in enumerate(zip(z, flow_latent_shapes(B, L, C0, H0, W0))):
        _dev(t, f"z[{l}]", shp)
    lb = _flow_common(params, prepared, L, K, C0, k, hid)
    x = (torch.empty((B, C0, H0, W0), dtype=torch.float32, device=z[0].device)
         if out is None else _dev(out, "out", (B, C0, H0, W0)))
    ws = _workspace(int(lb.finc_flow_workspace_bytes(B, L, C0, H0, W0, hid)), z[0].device,
                    workspace)
    zp = (ctypes.c_void_p * L)(*[t.data_ptr() for t in z])
    _check(lb.finc_flow_sample(zp, _ptr(x), _ptr(params), _ptr(prepared), B, L, K, C0, H0, W0, k,
                               hid, _ptr(ws), _stream()), "finc_flow_sample")
    return x


# ---- sequence operators -----------------------------------------------------
# A model that reads a raster position by position (include/finc.h, "Sequence
# operators").  Inner tensors are (B, D, L) with contiguous positions -- views
# such as a projection's halves are taken as they are -- and rows are (..., D).
# Activations are float32, bfloat16 or float16, parameters and scan states float32.


_NO_RASTER = (0, 0, 0)


def _empty(like: torch.Tensor, dtype) -> torch.Tensor:
    """A contiguous tensor of the shape of like (a third of torch.empty's time)."""
    return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)


def _type(x: torch.Tensor, name: str = "x"):
    """(device, type id) of a call's first activations, contiguous in their last
    dimension."""
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    dev = x.get_device()
    if dev != _current_device():
        raise ValueError(f"{name} must be on the current device")
    kind = _TYPES.get(x.dtype)
    if kind is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16")
    if not (x.is_contiguous() or x.stride(-1) == 1 or x.shape[-1] <= 1):
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return dev, kind


def _act(t: torch.Tensor, name: str, dev: int, dtype, shape):
    """A tensor of activations, contiguous in its last dimension."""
    if t.get_device() == dev and t.dtype == dtype and t.shape == shape \
            and (t.is_contiguous() or t.stride(-1) == 1 or shape[-1] <= 1):
        return t
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the device of the other tensors")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name} must be contiguous in its last dimension")


def _param(t: torch.Tensor | None, name: str, dev: int, shape, dtype=torch.float32) -> int:
    """The address of a contiguous tensor, or 0 for None."""
    if t is None:
        return 0
    if t.get_device() == dev and t.dtype == dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the device of the other tensors")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name} must be contiguous")


def _raster(t: torch.Tensor | None):
    """A (B, D, L) or (B, G, N, L) tensor as the ABI's finc_raster."""
    if t is None:
        return _NO_RASTER
    st = t.stride()
    if len(st) == 3:
        return t.data_ptr(), st[0], st[1]
    G, N = t.shape[1], t.shape[2]
    if G > 1 and N > 1 and st[1] != N * st[2] and t.numel():
        raise ValueError("the groups of a (B, G, N, L) tensor must follow each other")
    return t.data_ptr(), st[0], st[2] if N > 1 else st[1]


def _out(t: torch.Tensor | None, like: torch.Tensor, name: str, dev: int):
    """An output of the shape and type of `like`, contiguous unless given."""
    if t is None:
        return _empty(like, like.dtype)
    return _act(t, name, dev, like.dtype, like.shape)


def _space(t: torch.Tensor | None, nbytes: int, dev: int, name: str = "workspace"):
    """A buffer of at least nbytes."""
    if t is None:
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the device of the other tensors")
    return _bytes_buf(t, nbytes, name)


def _dims(t: torch.Tensor, name: str, form: str):
    """The shape of t, which is of the form "(B, D, L)"."""
    if t.dim() != form.count(",") + 1:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {form}")
    return t.shape


def _conv_dims(x, w):
    B, D, L = _dims(x, "x", "(B, D, L)")
    K = _dims(w, "w", "(D, K)")[1]
    if not 1 <= K <= MAX_TAPS:
        raise ValueError(f"w has {K} taps, expected 1 to {MAX_TAPS}")
    return B, D, L, K


def causal_conv_forward(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, *,
                        silu: bool = False, state: torch.Tensor | None = None,
                        lengths: torch.Tensor | None = None, out: torch.Tensor | None = None,
                        state_out: torch.Tensor | None = None):
    """y = act(bias + the causal convolution of x (B, D, L) with w (D, K)) (see
    finc_causal_conv_forward); state_out (B, D, K - 1) is written if given."""
    lib_ = _require_lib()
    B, D, L, K = _conv_dims(x, w)
    dev, kind = _type(x)
    y = _out(out, x, "out", dev)
    st = (B, D, K - 1)
    a = CONV_ARGS.pack(kind, B, D, L, K, bool(silu), *_raster(x), *_raster(y),
                       _param(w, "w", dev, (D, K)), _param(bias, "bias", dev, (D,)),
                       _param(state, "state", dev, st, x.dtype),
                       _param(state_out, "state_out", dev, st, x.dtype),
                       _param(lengths, "lengths", dev, (B,), torch.int32))
    _check(lib_.finc_causal_conv_forward(a, _stream()), "finc_causal_conv_forward")
    return y


def causal_conv_backward(x: torch.Tensor, w: torch.Tensor, dy: torch.Tensor,
                         bias: torch.Tensor | None = None, *, silu: bool = False,
                         state: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                         dstate_out: torch.Tensor | None = None, dx: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None):
    """(dx, dw, dbias, dstate) of causal_conv_forward for the gradients dy and
    dstate_out of its outputs; dbias and dstate are None without bias and state."""
    lib_ = _require_lib()
    B, D, L, K = _conv_dims(x, w)
    dev, kind = _type(x)
    _act(dy, "dy", dev, x.dtype, x.shape)
    st = (B, D, K - 1)
    a = CONV_ARGS.pack(kind, B, D, L, K, bool(silu), *_raster(x), *_NO_RASTER,
                       _param(w, "w", dev, (D, K)), _param(bias, "bias", dev, (D,)),
                       _param(state, "state", dev, st, x.dtype), 0,
                       _param(lengths, "lengths", dev, (B,), torch.int32))
    dx = _out(dx, x, "dx", dev)
    dw = torch.empty_like(w)
    dbias = None if bias is None else torch.empty_like(bias)
    dstate = None if state is None else torch.empty_like(state)
    ws = _space(workspace, lib_.finc_causal_conv_workspace_bytes(B, D, L, K), dev)
    g = CONV_GRADS.pack(*_raster(dy), *_raster(dx), dw.data_ptr(),
                        0 if dbias is None else dbias.data_ptr(),
                        _param(dstate_out, "dstate_out", dev, st, x.dtype),
                        0 if dstate is None else dstate.data_ptr(), ws.data_ptr())
    _check(lib_.finc_causal_conv_backward(a, g, _stream()), "finc_causal_conv_backward")
    return dx, dw, dbias, dstate


def _slots(slots, dev, B, S):
    if slots is None and S < B:
        raise ValueError(f"state has {S} entries for {B} rows")
    return _param(slots, "slots", dev, (B,), torch.int32)


def causal_conv_step(x: torch.Tensor, w: torch.Tensor, state: torch.Tensor,
                     bias: torch.Tensor | None = None, *, silu: bool = False,
                     slots: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """One position: y (B, D) of x (B, D), whose row b's last inputs are entry
    slots[b] (or b) of state (S, D, K - 1), which takes the new one in place.  A
    slot outside [0, S) is an idle row (y 0)."""
    lib_ = _require_lib()
    B, D = _dims(x, "x", "(B, D)")
    K, S = _dims(w, "w", "(D, K)")[1], _dims(state, "state", "(S, D, K - 1)")[0]
    dev, kind = _type(x)
    y = _out(out, x, "out", dev)
    _check(lib_.finc_causal_conv_step(
        kind, x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), _param(w, "w", dev, (D, K)),
        _param(bias, "bias", dev, (D,)), _param(state, "state", dev, (S, D, K - 1), x.dtype),
        _slots(slots, dev, B, S), B, S, D, K, bool(silu), _stream()), "finc_causal_conv_step")
    return y


def _scan_counts(A, Bm, C):
    """(states, groups)."""
    N, G = _dims(A, "A", "(D, N)")[1], Bm.shape[1]
    if not 1 <= N <= MAX_STATE:
        raise ValueError(f"A has {N} states, expected 1 to {MAX_STATE}")
    if G < 1 or C % G:
        raise ValueError(f"{G} groups do not divide {C} channels")
    return N, G


def _scan_inputs(x, dt, A, Bm, Cm, D, z, dt_bias, softplus, lengths):
    """(device, sizes, SCAN_ARGS' fields up to y, those after it up to dt_bias, lengths)."""
    B, C, L = _dims(x, "x", "(B, D, L)")
    _dims(Bm, "Bm", "(B, G, N, L)")
    N, G = _scan_counts(A, Bm, C)
    dev, kind = _type(x)
    T, shape, shared = x.dtype, x.shape, (B, G, N, L)
    _act(dt, "dt", dev, T, shape)
    _act(Bm, "Bm", dev, T, shared)
    _act(Cm, "Cm", dev, T, shared)
    if z is not None:
        _act(z, "z", dev, T, shape)
    head = (kind, B, C, L, N, G, bool(softplus), *_raster(x), *_raster(dt), *_raster(z),
            *_raster(Bm), *_raster(Cm))
    params = (_param(A, "A", dev, (C, N)), _param(D, "D", dev, (C,)),
              _param(dt_bias, "dt_bias", dev, (C,)))
    return dev, (B, C, L, N, G), head, params, _param(lengths, "lengths", dev, (B,), torch.int32)


def selective_scan_states(B: int, D: int, L: int, N: int, device) -> torch.Tensor:
    """A buffer for the states that a forward keeps for its backward."""
    n = _require_lib().finc_selective_scan_states_bytes(B, D, L, N)
    return torch.empty(max(n, 256) // 4, dtype=torch.float32, device=device)


def selective_scan_forward(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor,
                           Cm: torch.Tensor, D: torch.Tensor | None = None,
                           z: torch.Tensor | None = None, dt_bias: torch.Tensor | None = None, *,
                           softplus: bool = True, state: torch.Tensor | None = None,
                           lengths: torch.Tensor | None = None, out: torch.Tensor | None = None,
                           state_out: torch.Tensor | None = None,
                           states: torch.Tensor | None = None):
    """y (B, D, L) of the selective scan of x with steps dt, decays A (D, N), Bm
    and Cm (B, G, N, L), skip D, gate z (see finc_selective_scan_forward).
    state_out (B, D, N) is written if given, and may be state; states
    (selective_scan_states) is what selective_scan_backward reads."""
    lib_ = _require_lib()
    dev, (B, C, L, N, G), head, params, rows = _scan_inputs(x, dt, A, Bm, Cm, D, z, dt_bias,
                                                            softplus, lengths)
    y = _out(out, x, "out", dev)
    keep = 0
    if states is not None:
        n = lib_.finc_selective_scan_states_bytes(B, C, L, N)
        keep = _space(states, n, dev, "states").data_ptr()
    a = SCAN_ARGS.pack(*head, *_raster(y), *params, _param(state, "state", dev, (B, C, N)),
                       _param(state_out, "state_out", dev, (B, C, N)), keep, rows)
    _check(lib_.finc_selective_scan_forward(a, _stream()), "finc_selective_scan_forward")
    return y


def selective_scan_backward(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor,
                            Cm: torch.Tensor, dy: torch.Tensor, states: torch.Tensor,
                            D: torch.Tensor | None = None, z: torch.Tensor | None = None,
                            dt_bias: torch.Tensor | None = None, *, softplus: bool = True,
                            lengths: torch.Tensor | None = None,
                            dstate_out: torch.Tensor | None = None,
                            dx: torch.Tensor | None = None, ddt: torch.Tensor | None = None,
                            dz: torch.Tensor | None = None,
                            workspace: torch.Tensor | None = None) -> dict:
    """The gradients of a selective_scan_forward that wrote `states`, for the
    gradients dy and dstate_out of its outputs: a dict of dx, ddt, dA, dB, dC, dD,
    dz, ddt_bias (None without D, z, dt_bias) and dstate."""
    lib_ = _require_lib()
    dev, (B, C, L, N, G), head, params, rows = _scan_inputs(x, dt, A, Bm, Cm, D, z, dt_bias,
                                                            softplus, lengths)
    _act(dy, "dy", dev, x.dtype, x.shape)
    n = lib_.finc_selective_scan_states_bytes(B, C, L, N)
    keep = _space(states, n, dev, "states").data_ptr()
    dx, ddt = _out(dx, x, "dx", dev), _out(ddt, x, "ddt", dev)
    dz = None if z is None else _out(dz, x, "dz", dev)
    dB, dC = _out(None, Bm, "dB", dev), _out(None, Cm, "dC", dev)
    dA = torch.empty_like(A)
    dD = None if D is None else torch.empty_like(D)
    db = None if dt_bias is None else torch.empty_like(dt_bias)
    dstate = torch.empty((B, C, N), dtype=torch.float32, device=x.device)
    ws = _space(workspace, lib_.finc_selective_scan_workspace_bytes(B, C, L, N, G), dev)
    a = SCAN_ARGS.pack(*head, *_NO_RASTER, *params, 0, 0, keep, rows)
    g = SCAN_GRADS.pack(*_raster(dy), *_raster(dx), *_raster(ddt), *_raster(dz), *_raster(dB),
                        *_raster(dC), dA.data_ptr(), 0 if dD is None else dD.data_ptr(),
                        0 if db is None else db.data_ptr(),
                        _param(dstate_out, "dstate_out", dev, (B, C, N)), dstate.data_ptr(),
                        ws.data_ptr())
    _check(lib_.finc_selective_scan_backward(a, g, _stream()), "finc_selective_scan_backward")
    return dict(dx=dx, ddt=ddt, dA=dA, dB=dB, dC=dC, dD=dD, dz=dz, ddt_bias=db, dstate=dstate)


def selective_scan_step(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor,
                        Cm: torch.Tensor, state: torch.Tensor, D: torch.Tensor | None = None,
                        z: torch.Tensor | None = None, dt_bias: torch.Tensor | None = None, *,
                        softplus: bool = True, slots: torch.Tensor | None = None,
                        out: torch.Tensor | None = None):
    """One position: y (B, D) of x, dt, z (B, D) and Bm, Cm (B, G, N); row b's
    state is entry slots[b] (or b) of state (S, D, N), updated in place.  A slot
    outside [0, S) is an idle row (y 0)."""
    lib_ = _require_lib()
    B, C = _dims(x, "x", "(B, D)")
    _dims(Bm, "Bm", "(B, G, N)")
    N, G = _scan_counts(A, Bm, C)
    S = _dims(state, "state", "(S, D, N)")[0]
    dev, kind = _type(x)
    T, shape = x.dtype, x.shape
    _act(dt, "dt", dev, T, shape)
    zp = zs = 0
    if z is not None:
        zp, zs = _act(z, "z", dev, T, shape).data_ptr(), z.stride(0)
    for t, name in ((Bm, "Bm"), (Cm, "Cm")):
        _act(t, name, dev, T, (B, G, N))
        if B > 0 and G > 1 and t.stride(1) != N:
            raise ValueError(f"the groups of {name} must follow each other")
    y = _out(out, x, "out", dev)
    a = SCAN_STEP_ARGS.pack(kind, B, S, C, N, G, bool(softplus), x.data_ptr(), dt.data_ptr(), zp,
                            Bm.data_ptr(), Cm.data_ptr(), x.stride(0), dt.stride(0), zs,
                            Bm.stride(0), Cm.stride(0), y.stride(0), y.data_ptr(),
                            _param(A, "A", dev, (C, N)), _param(D, "D", dev, (C,)),
                            _param(dt_bias, "dt_bias", dev, (C,)),
                            _param(state, "state", dev, (S, C, N)), _slots(slots, dev, B, S))
    _check(lib_.finc_selective_scan_step(a, _stream()), "finc_selective_scan_step")
    return y


def _rows(t: torch.Tensor, name: str) -> int:
    """The step between the rows of a (..., D) tensor, which lie evenly."""
    if t.is_contiguous():
        return t.shape[-1]
    outer = [(n, st) for n, st in zip(t.shape[:-1], t.stride()[:-1]) if n != 1]
    for (_, st), (n, inner) in zip(outer, outer[1:]):
        if st != n * inner:
            raise ValueError(f"the rows of {name} must lie evenly")
    return outer[-1][1] if outer else t.shape[-1]


def _row_dims(x, name="x"):
    """(rows, columns) of a (..., D) tensor."""
    shape = x.shape
    if not shape:
        raise ValueError(f"{name} must have a last dimension")
    D = shape[-1]
    return (x.numel() // D if D else 0), D


def _philox_args(p, seed, offset):
    if not 0.0 <= p < 1.0 or round(p * 65536) > 65535:
        raise ValueError(f"p is {p}, expected 0 <= p <= 65535 / 65536")
    if not 0 <= seed < 1 << 64:
        raise ValueError("seed must be an unsigned 64-bit number")
    if not 0 <= offset < 1 << 64:
        raise ValueError("offset must be an unsigned 64-bit number")


def dropout_counters(rows: int, D: int) -> int:
    """Counters that one dropout of (rows, D) uses, from its offset on."""
    return int(_require_lib().finc_dropout_counters(rows, D))


def dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0,
            residual: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """dropout(x), or residual + dropout(x), of (..., D) rows: which elements are
    kept follows from seed, offset and the element's place alone (see finc_dropout),
    so the gradient is the same call on dy.  out may be x or residual."""
    lib_ = _require_lib()
    M, D = _row_dims(x)
    dev, kind = _type(x)
    _philox_args(p, seed, offset)
    y = _out(out, x, "out", dev)
    rp = rs = 0
    if residual is not None:
        rp = _act(residual, "residual", dev, x.dtype, x.shape).data_ptr()
        rs = _rows(residual, "residual")
    _check(lib_.finc_dropout(kind, x.data_ptr(), _rows(x, "x"), rp, rs, y.data_ptr(),
                             _rows(y, "out"), M, D, p, seed, offset, _stream()), "finc_dropout")
    return y


def _residual_type(t, name, dtype):
    if t.dtype != dtype and t.dtype != torch.float32:
        raise ValueError(f"{name} must be {dtype} or float32, not {t.dtype}")
    return t.dtype


def add_norm_forward(x: torch.Tensor, w: torch.Tensor, residual: torch.Tensor | None = None, *,
                     eps: float = 1e-5, p: float = 0.0, seed: int = 0, offset: int = 0,
                     fp8: bool = False, out: torch.Tensor | None = None,
                     residual_out: torch.Tensor | None = None,
                     scale: torch.Tensor | None = None):
    """(y, r) of rows x (..., D): r = residual + dropout(x), y = r / rms(r) * w.
    residual is of x's type or float32, and r of the residual's (of x's without
    one); residual_out may be residual, and out x.  fp8: (q, scale, r) with y as
    float8_e4m3fn and a float32 scale a row (see finc_add_norm_forward)."""
    lib_ = _require_lib()
    M, D = _row_dims(x)
    dev, kind = _type(x)
    shape = x.shape
    _philox_args(p, seed, offset)
    R, sp, ss = x.dtype, 0, 0
    if residual is not None:
        R = _residual_type(residual, "residual", x.dtype)
        sp = _act(residual, "residual", dev, R, shape).data_ptr()
        ss = _rows(residual, "residual")
    elif residual_out is not None:
        R = _residual_type(residual_out, "residual_out", x.dtype)
    r = _empty(x, R) if residual_out is None else _act(residual_out, "residual_out", dev, R, shape)
    wp = _param(w, "w", dev, (D,))
    T, cp = x.dtype, 0
    if fp8:
        T = torch.float8_e4m3fn
        if scale is None:
            scale = w.new_empty(shape[:-1])
        cp = _param(scale, "scale", dev, shape[:-1])
    elif scale is not None:
        raise ValueError("scale goes with fp8")
    if out is None:
        out = _empty(x, T)
    else:
        _act(out, "out", dev, T, shape)
    a = NORM_ARGS.pack(kind, _TYPES[R], M, D, x.data_ptr(), sp, out.data_ptr(), r.data_ptr(),
                       _rows(x, "x"), ss, _rows(out, "out"), _rows(r, "residual_out"), wp, cp,
                       eps, p, seed, offset)
    # the ABI takes a scale's presence for the 8-bit output: an empty one has no address
    if M > 0:
        _check(lib_.finc_add_norm_forward(a, _stream()), "finc_add_norm_forward")
    return (out, scale, r) if fp8 else (out, r)


def add_norm_backward(dy: torch.Tensor, r: torch.Tensor, w: torch.Tensor,
                      dr: torch.Tensor | None = None, *, eps: float = 1e-5, p: float = 0.0,
                      seed: int = 0, offset: int = 0, dx: torch.Tensor | None = None,
                      dresidual: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None):
    """(dx, dresidual, dw) of add_norm_forward from its r, for the gradient dy of y
    and dr (or None for 0) of r.  Without dropout and with one type dx and dresidual
    are the same values: one tensor, unless both are given."""
    lib_ = _require_lib()
    M, D = _row_dims(dy, "dy")
    dev, kind = _type(dy, "dy")
    shape = dy.shape
    _philox_args(p, seed, offset)
    R = _residual_type(r, "r", dy.dtype)
    _act(r, "r", dev, R, shape)
    gp = gs = 0
    if dr is not None:
        gp, gs = _act(dr, "dr", dev, R, shape).data_ptr(), _rows(dr, "dr")
    one = p == 0.0 and dy.dtype == R and (dx is None or dresidual is None)
    xp = xs = rp = rs = 0
    if one and dx is None:
        dx = dresidual = _out(dresidual, r, "dresidual", dev)
        rp, rs = dresidual.data_ptr(), _rows(dresidual, "dresidual")
    else:
        dx = _out(dx, dy, "dx", dev)
        xp, xs = dx.data_ptr(), _rows(dx, "dx")
        if one:
            dresidual = dx
        else:
            dresidual = _out(dresidual, r, "dresidual", dev)
            rp, rs = dresidual.data_ptr(), _rows(dresidual, "dresidual")
    dw = torch.empty_like(w)
    ws = _space(workspace, lib_.finc_add_norm_workspace_bytes(M, D), dev)
    a = NORM_GRAD_ARGS.pack(kind, _TYPES[R], M, D, dy.data_ptr(), r.data_ptr(), gp, xp,
                            rp, _rows(dy, "dy"), _rows(r, "r"), gs, xs, rs,
                            _param(w, "w", dev, (D,)), dw.data_ptr(), eps, p, seed, offset,
                            ws.data_ptr())
    _check(lib_.finc_add_norm_backward(a, _stream()), "finc_add_norm_backward")
    return dx, dresidual, dw


# Rows of positions: q and k are (B, L, G, DK), v and y (B, L, H, DV), g (B, L, H); any
# steps between rows and heads, so that a projection's parts are taken as they are.

_NO_HEADS = (0, 0, 0, 0)


def _heads(t: torch.Tensor | None):
    """A (B, L, H, D) tensor, or (B, L, H) of single elements, as the ABI's finc_heads."""
    if t is None:
        return _NO_HEADS
    st = t.stride()
    return t.data_ptr(), st[0], st[1], st[2]


def _step_heads(t: torch.Tensor | None):
    """A (B, H, D) tensor, or (B, H), of one position."""
    if t is None:
        return _NO_HEADS
    st = t.stride()
    return t.data_ptr(), st[0], 0, st[1]


def _element(t: torch.Tensor, name: str, dev: int, dtype, shape):
    """A tensor of single elements, with any steps."""
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the device of the other tensors")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _attention_inputs(q, k, v, g, decay, rows, form):
    """(device, type id, groups, DK, heads, DV, the address of decay) of q, k (rows, G, DK),
    v (rows, H, DV) and g (rows, H)."""
    G, DK = _dims(q, "q", f"({form}, G, DK)")[rows:]
    H, DV = _dims(v, "v", f"({form}, H, DV)")[rows:]
    if not 1 <= DK <= MAX_HEAD or not 1 <= DV <= MAX_HEAD:
        raise ValueError(f"heads of {DK} and {DV} elements, expected 1 to {MAX_HEAD}")
    if G < 1 or H < 1 or H % G:
        raise ValueError(f"{G} groups do not divide {H} heads")
    dev, kind = _type(q, "q")
    T = q.dtype
    _act(k, "k", dev, T, q.shape)
    _act(v, "v", dev, T, (*q.shape[:rows], H, DV))
    if g is not None:
        _element(g, "g", dev, T, (*q.shape[:rows], H))
    return dev, kind, G, DK, H, DV, _param(decay, "decay", dev, (H,))


def linear_attention_states(B: int, L: int, H: int, DK: int, DV: int, device) -> torch.Tensor:
    """A buffer for the states that a forward keeps for its backward."""
    n = _require_lib().finc_linear_attention_states_bytes(B, L, H, DK, DV)
    return torch.empty(max(n, 256) // 4, dtype=torch.float32, device=device)


def linear_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *,
                             g: torch.Tensor | None = None, decay: torch.Tensor | None = None,
                             scale: float = 1.0, state: torch.Tensor | None = None,
                             lengths: torch.Tensor | None = None,
                             out: torch.Tensor | None = None,
                             state_out: torch.Tensor | None = None,
                             states: torch.Tensor | None = None):
    """y (B, L, H, DV) of linear attention with the log decays decay (H) + g (B, L, H):
    q and k (B, L, G, DK) shared by groups of heads, v (B, L, H, DV) (see
    finc_linear_attention_forward).  state_out (B, H, DK, DV) is written if given, and
    may be state; states (linear_attention_states) is what
    linear_attention_backward reads."""
    lib_ = _require_lib()
    dev, kind, G, DK, H, DV, dp = _attention_inputs(q, k, v, g, decay, 2, "B, L")
    B, L = q.shape[:2]
    y = _out(out, v, "out", dev)
    n = lib_.finc_linear_attention_states_bytes(B, L, H, DK, DV)
    if states is None and L > ATTENTION_PART:
        states = _space(None, n, dev)
    sp = 0 if states is None else _space(states, n, dev, "states").data_ptr()
    st = (B, H, DK, DV)
    a = ATTENTION_ARGS.pack(kind, B, L, H, G, DK, DV, *_heads(q), *_heads(k), *_heads(v),
                            *_heads(g), *_heads(y), dp, _param(state, "state", dev, st),
                            _param(state_out, "state_out", dev, st), sp,
                            _param(lengths, "lengths", dev, (B,), torch.int32), scale)
    _check(lib_.finc_linear_attention_forward(a, _stream()), "finc_linear_attention_forward")
    return y


def linear_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              dy: torch.Tensor, states: torch.Tensor, *,
                              g: torch.Tensor | None = None, decay: torch.Tensor | None = None,
                              scale: float = 1.0, lengths: torch.Tensor | None = None,
                              dstate_out: torch.Tensor | None = None,
                              dq: torch.Tensor | None = None, dk: torch.Tensor | None = None,
                              dv: torch.Tensor | None = None,
                              workspace: torch.Tensor | None = None) -> dict:
    """The gradients of a linear_attention_forward that wrote `states`, for the gradients
    dy and dstate_out of its outputs: a dict of dq, dk, dv, dg (None without g) and
    dstate."""
    lib_ = _require_lib()
    dev, kind, G, DK, H, DV, dp = _attention_inputs(q, k, v, g, decay, 2, "B, L")
    B, L = q.shape[:2]
    _act(dy, "dy", dev, v.dtype, v.shape)
    st = (B, H, DK, DV)
    n = lib_.finc_linear_attention_states_bytes(B, L, H, DK, DV)
    sp = _space(states, n, dev, "states").data_ptr()
    dq, dk, dv = _out(dq, q, "dq", dev), _out(dk, k, "dk", dev), _out(dv, v, "dv", dev)
    dg = None if g is None else _empty(g, g.dtype)
    dstate = torch.empty(st, dtype=torch.float32, device=q.device)
    ws = _space(workspace, lib_.finc_linear_attention_workspace_bytes(B, L, H, G, DK, DV), dev)
    a = ATTENTION_ARGS.pack(kind, B, L, H, G, DK, DV, *_heads(q), *_heads(k), *_heads(v),
                            *_heads(g), *_NO_HEADS, dp, 0, 0, sp,
                            _param(lengths, "lengths", dev, (B,), torch.int32), scale)
    o = ATTENTION_GRADS.pack(*_heads(dy), *_heads(dq), *_heads(dk), *_heads(dv), *_heads(dg),
                             _param(dstate_out, "dstate_out", dev, st), dstate.data_ptr(),
                             ws.data_ptr())
    _check(lib_.finc_linear_attention_backward(a, o, _stream()), "finc_linear_attention_backward")
    return dict(dq=dq, dk=dk, dv=dv, dg=dg, dstate=dstate)


def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                          state: torch.Tensor, *, g: torch.Tensor | None = None,
                          decay: torch.Tensor | None = None, scale: float = 1.0,
                          slots: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """One position: y (B, H, DV) of q, k (B, G, DK), v (B, H, DV) and g (B, H); row b's
    state is entry slots[b] (or b) of state (S, H, DK, DV), updated in place.  A slot
    outside [0, S) is an idle row (y 0)."""
    lib_ = _require_lib()
    dev, kind, G, DK, H, DV, dp = _attention_inputs(q, k, v, g, decay, 1, "B")
    B, S = q.shape[0], _dims(state, "state", "(S, H, DK, DV)")[0]
    y = _out(out, v, "out", dev)
    a = ATTENTION_STEP_ARGS.pack(kind, B, S, H, G, DK, DV, *_step_heads(q), *_step_heads(k),
                                 *_step_heads(v), *_step_heads(g), *_step_heads(y), dp,
                                 _param(state, "state", dev, (S, H, DK, DV)),
                                 _slots(slots, dev, B, S), scale)
    _check(lib_.finc_linear_attention_step(a, _stream()), "finc_linear_attention_step")
    return y


def _act_id(act):
    if act not in _ACTS:
        raise ValueError(f"act is {act!r}, expected one of {tuple(_ACTS)}")
    return _ACTS[act]


def _matrix(t: torch.Tensor, name: str, dev: int, dtype, shape=None):
    """A matrix of activations' type, contiguous in its last dimension: its rows' step."""
    _dims(t, name, "(N, K)")
    _act(t, name, dev, dtype, t.shape if shape is None else shape)
    return t.stride(0)


def linear_forward(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, *,
                   act: str | None = None, residual: torch.Tensor | None = None,
                   out: torch.Tensor | None = None, pre_out: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None):
    """act(x w^T + bias) + residual of rows x (..., K) and w (N, K) of one type, bias (N)
    float32; act is None, "relu", "silu" or "gelu" (see finc_linear_forward).  pre_out
    (..., N) takes x w^T + bias, which linear_backward reads where there is an act; out
    may be residual."""
    lib_ = _require_lib()
    M, K = _row_dims(x)
    dev, kind = _type(x)
    sw, N = _matrix(w, "w", dev, x.dtype), w.shape[0]
    if w.shape[1] != K:
        raise ValueError(f"w has shape {tuple(w.shape)}, expected (N, {K})")
    shape = (*x.shape[:-1], N)
    if out is None:
        y = torch.empty(shape, dtype=x.dtype, device=x.device)
    else:
        y = _act(out, "out", dev, x.dtype, shape)
    rp = rs = pp = ps = 0
    if residual is not None:
        rp = _act(residual, "residual", dev, x.dtype, shape).data_ptr()
        rs = _rows(residual, "residual")
    if pre_out is not None:
        pp = _act(pre_out, "pre_out", dev, x.dtype, shape).data_ptr()
        ps = _rows(pre_out, "pre_out")
    n, ws = lib_.finc_linear_workspace_bytes(kind, M, K, N), 0
    if n or workspace is not None:
        ws = _space(workspace, n, dev).data_ptr()
    a = LINEAR_ARGS.pack(kind, _act_id(act), M, K, N, x.data_ptr(), w.data_ptr(), rp, y.data_ptr(),
                         pp, _rows(x, "x"), sw, rs, _rows(y, "out"), ps,
                         _param(bias, "bias", dev, (N,)), ws)
    _check(lib_.finc_linear_forward(a, _stream()), "finc_linear_forward")
    return y


def linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor,
                    pre: torch.Tensor | None = None, *, act: str | None = None,
                    bias: bool = True, dx: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None):
    """(dx, dw, dbias) of linear_forward for the gradient dy (..., N) of its output, which
    is the residual's too; pre is what pre_out took, needed with an act.  dx and dw are of
    x's type, dbias is float32, or None without bias."""
    lib_ = _require_lib()
    M, K = _row_dims(x)
    dev, kind = _type(x)
    sw, N = _matrix(w, "w", dev, x.dtype), w.shape[0]
    if w.shape[1] != K:
        raise ValueError(f"w has shape {tuple(w.shape)}, expected (N, {K})")
    shape, act = (*x.shape[:-1], N), _act_id(act)
    _act(dy, "dy", dev, x.dtype, shape)
    pp = ps = 0
    if act:
        if pre is None:
            raise ValueError("the gradients of an act need pre")
        pp, ps = _act(pre, "pre", dev, x.dtype, shape).data_ptr(), _rows(pre, "pre")
    dx = _out(dx, x, "dx", dev)
    dw = _empty(w, w.dtype)
    db = torch.empty(N, dtype=torch.float32, device=x.device) if bias else None
    ws = _space(workspace, lib_.finc_linear_grad_workspace_bytes(kind, act, M, K, N), dev)
    a = LINEAR_GRAD_ARGS.pack(kind, act, M, K, N, dy.data_ptr(), x.data_ptr(), w.data_ptr(), pp,
                              dx.data_ptr(), dw.data_ptr(), _rows(dy, "dy"), _rows(x, "x"), sw, ps,
                              _rows(dx, "dx"), K, 0 if db is None else db.data_ptr(),
                              ws.data_ptr())
    _check(lib_.finc_linear_backward(a, _stream()), "finc_linear_backward")
    return dx, dw, db


def _ids(t: torch.Tensor, dev: int | None = None):
    """(device, whether ids are 64-bit) of a contiguous tensor of ids."""
    if not t.is_cuda:
        raise ValueError("ids must be a device tensor")
    at = t.get_device()
    if at != (_current_device() if dev is None else dev):
        raise ValueError("ids must be on the current device")
    if t.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"ids must be int32 or int64, not {t.dtype}")
    if not t.is_contiguous():
        raise ValueError("ids must be contiguous")
    return at, int(t.dtype == torch.int64)


def embed_forward(ids: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, dtype=None,
                  out: torch.Tensor | None = None):
    """scale table[ids] (..., D) of ids (...), int32 or int64, and a table (V, D) of the
    output's type (dtype, or the table's) or float32.  An id outside [0, V) is padding:
    its row is 0."""
    lib_ = _require_lib()
    dev, wide = _ids(ids)
    V, D = _dims(table, "table", "(V, D)")
    T = (table.dtype if out is None else out.dtype) if dtype is None else dtype
    if T not in _TYPES or table.dtype not in (T, torch.float32):
        raise ValueError(f"table must be {T} or float32, not {table.dtype}")
    st, shape = _matrix(table, "table", dev, table.dtype), (*ids.shape, D)
    if out is None:
        y = torch.empty(shape, dtype=T, device=ids.device)
    else:
        y = _act(out, "out", dev, T, shape)
    _check(lib_.finc_embed_forward(_TYPES[T], _TYPES[table.dtype], ids.data_ptr(), wide,
                                   table.data_ptr(), st, y.data_ptr(), _rows(y, "out"),
                                   ids.numel(), V, D, scale, _stream()), "finc_embed_forward")
    return y


def embed_backward(ids: torch.Tensor, dy: torch.Tensor, V: int, *, scale: float = 1.0,
                   dtable: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """The gradient (V, D), float32, of embed_forward's table for the gradient dy (..., D)
    of its output: every row is written, those that no id names with 0."""
    lib_ = _require_lib()
    dev, kind = _type(dy, "dy")
    _, wide = _ids(ids, dev)
    M, D = _row_dims(dy, "dy")
    if dy.shape[:-1] != ids.shape:
        raise ValueError(f"dy has shape {tuple(dy.shape)}, expected {(*ids.shape, D)}")
    if dtable is None:
        dtable = torch.empty((V, D), dtype=torch.float32, device=dy.device)
    ws = _space(workspace, lib_.finc_embed_workspace_bytes(M, V, D), dev)
    _check(lib_.finc_embed_backward(kind, ids.data_ptr(), wide, dy.data_ptr(), _rows(dy, "dy"),
                                    _param(dtable, "dtable", dev, (V, D)), M, V, D, scale,
                                    ws.data_ptr(), _stream()), "finc_embed_backward")
    return dtable
