"""ctypes binding of libvitattn.so (argument marshalling only).

Raw entry points (`library().vitattn_fwd(...)` etc.) take integer device
pointers exactly like the C ABI. The tensor helpers below allocate outputs
with PyTorch, pass `data_ptr()`s and the current HIP stream, and raise
VitattnError on a non-zero status.
"""
from __future__ import annotations

import ctypes
import functools
import math
import operator
import os
import threading

from ._build import LIB_PATH

_lock = threading.Lock()
_lib = None

c_int, c_float, c_size_t, c_void_p = ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p


class Strides(ctypes.Structure):
    """vitattn_strides: element strides of an operand viewed as [B, H, N, d]."""
    _fields_ = [("batch", ctypes.c_longlong), ("head", ctypes.c_longlong), ("row", ctypes.c_longlong)]


class Forms(ctypes.Structure):
    """vitattn_forms: the kernel forms a call takes."""
    _fields_ = [(n, ctypes.c_int) for n in ("fwd_waves", "dq_waves", "dkdv_keys", "dkdv_whole", "dkdv_split",
                                              "dkdv_rest64")]


_S = Strides


class Int:
    """A C int argument. ctypes would keep the low 32 bits of a larger value and
    the entry would compute a part of the call; it gets the lowest int instead,
    which every entry refuses (a workspace size is then 0)."""

    @staticmethod
    def from_param(x):
        if isinstance(x, int):
            return x if -0x80000000 <= x <= 0x7fffffff else -0x80000000
        return c_int.from_param(x) if isinstance(x, c_int) else Int.from_param(operator.index(x))


_I = Int

_SIGNATURES = {
    "vitattn_fwd": (c_int, [c_void_p] * 5 + [_I] * 4 + [c_float, c_void_p]),
    "vitattn_bwd_workspace_bytes": (c_size_t, [_I] * 4),
    "vitattn_bwd": (c_int, [c_void_p] * 9 + [_I] * 4 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_bwd_rowdot": (c_int, [c_void_p] * 3 + [_I] * 4 + [c_void_p, c_size_t, c_void_p]),
    "vitattn_bwd_dkdv": (c_int, [c_void_p] * 7 + [_I] * 4 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_bwd_dq": (c_int, [c_void_p] * 6 + [_I] * 4 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_fwd_kv": (c_int, [c_void_p] * 5 + [_I] * 5 + [c_float, c_void_p]),
    "vitattn_bwd_kv": (c_int, [c_void_p] * 9 + [_I] * 5 + [c_float, _I, c_void_p, c_size_t, c_void_p]),
    "vitattn_bwd_workspace_bytes_kv": (c_size_t, [_I] * 6),
    "vitattn_bwd_dkdv_ds": (c_int, [c_void_p] * 7 + [_I] * 4 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_bwd_dq_from_ds": (c_int, [c_void_p] * 2 + [_I] * 4 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_fwd_strided": (c_int, [c_void_p, _S] * 4 + [c_void_p] + [_I] * 5 + [c_float, c_void_p]),
    "vitattn_bwd_strided": (c_int, [c_void_p, _S] * 5 + [c_void_p] + [c_void_p, _S] * 3 + [_I] * 5
                            + [c_float, _I, c_void_p, c_size_t, c_void_p]),
    "vitattn_bwd_train_bf16_kv": (c_int, [_I]),
    "vitattn_bwd_train": (c_int, [c_void_p, _S] * 5 + [c_void_p] * 5 + [_I] * 5
                          + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_launch_forms": (c_int, [_I] * 6 + [ctypes.POINTER(Forms)]),
    "vitattn_merge": (c_int, [c_void_p] * 2 + [_I] + [c_void_p] * 2 + [_I] * 4 + [c_void_p]),
    "vitattn_agg_fwd": (c_int, [c_void_p] * 5 + [_I] * 4 + [c_float, c_void_p]),
    "vitattn_agg_bwd_workspace_bytes": (c_size_t, [_I] * 4),
    "vitattn_agg_bwd": (c_int, [c_void_p] * 9 + [_I] * 4 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_ulysses_pack": (c_int, [c_void_p] * 2 + [_I] * 5 + [c_void_p]),
    "vitattn_ulysses_unpack": (c_int, [c_void_p] * 2 + [_I] * 5 + [c_void_p]),
    "vitattn_ulysses_pack_out": (c_int, [c_void_p] * 2 + [_I] * 5 + [c_void_p]),
    "vitattn_ulysses_unpack_out": (c_int, [c_void_p] * 2 + [_I] * 5 + [c_void_p]),
    "vitattn_bwd_noalloc": (c_int, [c_void_p] * 9 + [_I] * 4 + [c_float, c_void_p]),
    "vitattn_layer_norm_fwd": (c_int, [c_void_p, _S] + [c_void_p] * 3 + [_S] + [c_void_p] * 2 + [_I] * 4
                               + [c_float, _I, _I, c_void_p]),
    "vitattn_layer_norm_bwd_workspace_bytes": (c_size_t, [_I] * 5),
    "vitattn_layer_norm_bwd": (c_int, [c_void_p, _S] + [c_void_p] * 4 + [_S, c_void_p, _S] + [c_void_p] * 2
                               + [_I] * 6 + [c_void_p, c_size_t, c_void_p]),
    "vitattn_rotary": (c_int, ([c_void_p, _S] * 2 + [_I]) * 2 + [c_void_p] + [ctypes.c_longlong] * 3 + [_I]
                       + [ctypes.POINTER(c_int), _I, ctypes.c_double] + [_I] * 5 + [c_void_p]),
    "vitattn_diff_fwd_workspace_bytes": (c_size_t, [_I] * 6),
    "vitattn_diff_fwd": (c_int, [c_void_p, _S] * 3 + [c_void_p, _I, c_void_p] + [c_void_p, _S] + [c_void_p] * 2
                         + [_I] * 6 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_diff_bwd_workspace_bytes": (c_size_t, [_I] * 6),
    "vitattn_diff_bwd": (c_int, [c_void_p, _S] * 3 + [c_void_p, _I] + [c_void_p] * 3
                         + [c_void_p, _S] * 4 + [c_void_p] + [_I] * 6 + [c_float, c_void_p, c_size_t, c_void_p]),
    "vitattn_status_str": (ctypes.c_char_p, [c_int]),
    "vitattn_version": (ctypes.c_char_p, []),
}


class VitattnError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(status_str(status))


def open_library(path):
    """ctypes handle of a built library at `path` with every entry point's
    signature set (library() uses it for the package's own build)."""
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


def library():
    """Load libvitattn.so once. Raises if it has not been built."""
    global _lib
    if _lib is None:
        with _lock:
            if _lib is None:
                if not os.path.exists(LIB_PATH):
                    raise ImportError(f"{LIB_PATH} is missing: build it with paper_2405_15780_amd._build.build()")
                _lib = open_library(LIB_PATH)
    return _lib


def status_str(status: int) -> str:
    return library().vitattn_status_str(status).decode()


def version() -> str:
    return library().vitattn_version().decode()


def workspace_bytes(B: int, H: int, N: int, d: int) -> int:
    return int(library().vitattn_bwd_workspace_bytes(B, H, N, d))


def _check(status: int):
    if status != 0:
        raise VitattnError(status)


@functools.lru_cache(maxsize=None)
def _torch():
    import torch

    return torch


@functools.lru_cache(maxsize=None)
def _raw_stream():
    """The current stream's handle by device index (without making a Stream of
    it, where torch offers that: 0.1 us instead of 1.9)."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream_ptr(t) -> int:
    return _raw_stream()(t.device.index)


def _as_input(t, name, device=None):
    torch = _torch()
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.bfloat16 and t.dim() == 4
            and (t.shape[3] == 1 or t.stride(3) == 1) and (device is None or t.device == device)):
        raise TypeError(f"{name} must be a 4-D bfloat16 CUDA tensor [B, H, N, d] with unit stride along d, on the "
                        "device of q (other strides are free, e.g. a [B, N, H, d] tensor passed as .transpose(1, 2))")
    return t


def _expect(t, name, dtype, shape, device, dense=False):
    """Raise TypeError unless t is a CUDA tensor of this dtype and exact shape
    on `device`, with unit stride along its last dim (contiguous if dense).
    A mismatch would otherwise become an out-of-bounds access on the GPU."""
    ok = (isinstance(t, _torch().Tensor) and t.is_cuda and t.device == device and t.dtype == dtype
          and t.shape == shape)
    if ok:
        ok = t.is_contiguous() if dense else (shape[-1] == 1 or t.stride(-1) == 1)
    if not ok:
        layout = "contiguous" if dense else "unit stride along the last dim"
        shape = tuple(int(n) for n in shape)
        raise TypeError(f"{name} must be a {dtype} CUDA tensor of shape {shape} on {device} ({layout})")
    return t


def _expect_workspace(ws, device):
    torch = _torch()
    if not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.device == device and ws.is_contiguous()):
        raise TypeError(f"workspace must be a contiguous CUDA tensor on {device}")
    return ws


def strides_of(t):
    """vitattn_strides of a [B, H, N, d] view (d contiguous)."""
    return Strides(t.stride(0), t.stride(1), t.stride(2))


def _dense(*ts):
    return all(t.is_contiguous() for t in ts)


def _default_scale(d, scale):
    return 1.0 / math.sqrt(d) if scale is None else float(scale)


VITATTN_BWD_ACCUMULATE_DQ = 1
VITATTN_BWD_STORE_DS = 2


def workspace_bytes_kv(B: int, H: int, Nq: int, Nk: int, d: int, flags: int = 0) -> int:
    """Workspace bytes of the backward pass for these sizes and flags (0 if invalid)."""
    return int(library().vitattn_bwd_workspace_bytes_kv(B, H, Nq, Nk, d, flags))


def _kv_shapes(q, k, v):
    B, H, Nq, d = q.shape
    if k.shape != v.shape or k.shape[:2] != q.shape[:2] or k.shape[3] != d:
        raise ValueError("k and v must be [B, H, Nk, d] with the B, H and d of q")
    return B, H, Nq, k.shape[2], d


def fwd(q, k, v, scale=None, out=None):
    """O (fp32 [B,H,Nq,d]) and LSE (fp32 [B,H,Nq]) of softmax(scale Q K^T) V;
    k and v may hold a different number of rows Nk (one key segment)."""
    torch = _torch()
    _as_input(q, "q")
    for t, n in ((k, "k"), (v, "v")):
        _as_input(t, n, q.device)
    B, H, Nq, Nk, d = _kv_shapes(q, k, v)
    if out is None:
        o = torch.empty((B, H, Nq, d), dtype=torch.float32, device=q.device)
        lse = torch.empty((B, H, Nq), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
        _expect(o, "o", torch.float32, (B, H, Nq, d), q.device)
        _expect(lse, "lse", torch.float32, (B, H, Nq), q.device, dense=True)
    lib = library()
    if not _dense(q, k, v, o):
        st = lib.vitattn_fwd_strided(q.data_ptr(), strides_of(q), k.data_ptr(), strides_of(k), v.data_ptr(),
                                     strides_of(v), o.data_ptr(), strides_of(o), lse.data_ptr(), B, H, Nq, Nk, d,
                                     _default_scale(d, scale), _stream_ptr(q))
    elif Nq == Nk:
        st = lib.vitattn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, Nq, d,
                             _default_scale(d, scale), _stream_ptr(q))
    else:
        st = lib.vitattn_fwd_kv(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, Nq, Nk,
                                d, _default_scale(d, scale), _stream_ptr(q))
    _check(st)
    return o, lse


def _workspace(q, k, workspace, flags=0):
    torch = _torch()
    B, H, N, d = q.shape
    need = workspace_bytes_kv(B, H, N, k.shape[2], d, flags)
    if workspace is None:
        workspace = torch.empty(max(need, 4) // 4, dtype=torch.float32, device=q.device)
    _expect_workspace(workspace, q.device)
    return workspace, workspace.numel() * workspace.element_size()


def bwd(q, k, v, o, lse, dout, scale=None, workspace=None, out=None, accumulate_dq=False, store_ds=False):
    """dQ (fp32 [B,H,Nq,d]), dK, dV (fp32 [B,H,Nk,d]) for the upstream gradient
    dout (bf16). For one key segment pass the merged o and lse of all keys;
    accumulate_dq adds this segment's share to out[0] instead of overwriting.
    store_ds selects the dS mode (dQ from stored dS; a workspace of about
    B*H*Nq*Nk*2 bytes, see workspace_bytes_kv)."""
    torch = _torch()
    _as_input(q, "q")
    for t, n in ((k, "k"), (v, "v"), (dout, "dout")):
        _as_input(t, n, q.device)
    B, H, Nq, Nk, d = _kv_shapes(q, k, v)
    _expect(dout, "dout", torch.bfloat16, (B, H, Nq, d), q.device)
    _expect(o, "o", torch.float32, (B, H, Nq, d), q.device)
    _expect(lse, "lse", torch.float32, (B, H, Nq), q.device, dense=True)
    flags = (VITATTN_BWD_ACCUMULATE_DQ if accumulate_dq else 0) | (VITATTN_BWD_STORE_DS if store_ds else 0)
    ws, ws_bytes = _workspace(q, k, workspace, flags)
    if out is None:
        if accumulate_dq:
            raise ValueError("accumulate_dq needs out=(dq, dk, dv) holding the running dq")
        dq = torch.empty((B, H, Nq, d), dtype=torch.float32, device=q.device)
        dk, dv = (torch.empty((B, H, Nk, d), dtype=torch.float32, device=q.device) for _ in range(2))
    else:
        dq, dk, dv = out
        _expect(dq, "dq", torch.float32, (B, H, Nq, d), q.device)
        _expect(dk, "dk", torch.float32, (B, H, Nk, d), q.device)
        _expect(dv, "dv", torch.float32, (B, H, Nk, d), q.device)
    lib = library()
    if not _dense(q, k, v, o, dout, dq, dk, dv):
        st = lib.vitattn_bwd_strided(q.data_ptr(), strides_of(q), k.data_ptr(), strides_of(k), v.data_ptr(),
                                     strides_of(v), o.data_ptr(), strides_of(o), dout.data_ptr(), strides_of(dout),
                                     lse.data_ptr(), dq.data_ptr(), strides_of(dq), dk.data_ptr(), strides_of(dk),
                                     dv.data_ptr(), strides_of(dv), B, H, Nq, Nk, d, _default_scale(d, scale),
                                     flags, ws.data_ptr(), ws_bytes, _stream_ptr(q))
    elif Nq == Nk and flags == 0:
        st = lib.vitattn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), dout.data_ptr(), lse.data_ptr(),
                             dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Nq, d, _default_scale(d, scale),
                             ws.data_ptr(), ws_bytes, _stream_ptr(q))
    else:
        st = lib.vitattn_bwd_kv(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), dout.data_ptr(),
                                lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Nq, Nk, d,
                                _default_scale(d, scale), flags, ws.data_ptr(), ws_bytes, _stream_ptr(q))
    _check(st)
    return dq, dk, dv


def bwd_train(q, k, v, o, lse, grad, scale=None):
    """Gradients of q, k and v in bf16 for an fp32 upstream gradient: bwd() with
    grad rounded to bf16 before and its outputs after, the conversions done in
    its kernels where they can be. None if grad's layout needs the general path."""
    torch = _torch()
    _as_input(q, "q")
    for t, n in ((k, "k"), (v, "v")):
        _as_input(t, n, q.device)
    B, H, Nq, Nk, d = _kv_shapes(q, k, v)
    _expect(o, "o", torch.float32, (B, H, Nq, d), q.device)
    _expect(lse, "lse", torch.float32, (B, H, Nq), q.device, dense=True)
    s = grad.stride()
    if not (grad.is_cuda and grad.device == q.device and grad.dtype == torch.float32 and grad.shape == q.shape
            and s[3] == 1 and s[2] >= grad.shape[3] and all(x >= 0 and x % 4 == 0 for x in s[:3])
            and (grad.shape[2] + 256) * s[2] * 2 <= 0x7fffffff and not grad.is_neg() and grad.data_ptr() != 0
            and grad.data_ptr() % 16 == 0):
        # The pitch bound is the bf16 operands': past it the conversion lays the
        # rows out anew. It also negates a lazily negated view (the memory holds
        # the opposite signs) and fills in zeros that have no memory yet.
        return None
    lib = library()
    dout, dq = (torch.empty((B, H, Nq, d), dtype=torch.bfloat16, device=q.device) for _ in range(2))
    kv_type = torch.bfloat16 if lib.vitattn_bwd_train_bf16_kv(Nq) else torch.float32
    dk, dv = (torch.empty((B, H, Nk, d), dtype=kv_type, device=q.device) for _ in range(2))
    ws, ws_bytes = _workspace(q, k, None)
    _check(lib.vitattn_bwd_train(q.data_ptr(), strides_of(q), k.data_ptr(), strides_of(k), v.data_ptr(),
                                 strides_of(v), o.data_ptr(), strides_of(o), grad.data_ptr(), strides_of(grad),
                                 lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H,
                                 Nq, Nk, d, _default_scale(d, scale), ws.data_ptr(), ws_bytes, _stream_ptr(q)))
    return dq, dk.to(torch.bfloat16), dv.to(torch.bfloat16)


def launch_forms(B, H, Nq, Nk, d, flags=0):
    """The kernel forms (a Forms) that calls of these sizes take on the current device."""
    forms = Forms()
    _check(library().vitattn_launch_forms(B, H, Nq, Nk, d, flags, ctypes.byref(forms)))
    return forms


VITATTN_NOALLOC_MAX_ROWS = 4194304


def bwd_noalloc(q, k, v, o, lse, dout, scale=None, out=None):
    """The backward pass through vitattn_bwd_noalloc (no workspace: the
    library's static scratch; B*H*N at most VITATTN_NOALLOC_MAX_ROWS; calls on
    one device must not overlap). Dense [B,H,N,d] operands; out=(dq, dk, dv)
    to write into existing tensors."""
    torch = _torch()
    B, H, N, d = _shape4(q, "q")
    dev = q.device
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (dout, "dout")):
        _expect(t, n, torch.bfloat16, (B, H, N, d), dev, dense=True)
    _expect(o, "o", torch.float32, (B, H, N, d), dev, dense=True)
    _expect(lse, "lse", torch.float32, (B, H, N), dev, dense=True)
    if out is None:
        dq, dk, dv = (torch.empty((B, H, N, d), dtype=torch.float32, device=dev) for _ in range(3))
    else:
        dq, dk, dv = out
        for t, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
            _expect(t, n, torch.float32, (B, H, N, d), dev, dense=True)
    _check(library().vitattn_bwd_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), dout.data_ptr(),
                                         lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, N, d,
                                         _default_scale(d, scale), _stream_ptr(q)))
    return dq, dk, dv


def merge(o_parts, lse_parts, out=None):
    """Merge partial results over disjoint key segments: o_parts fp32
    [P,B,H,N,d], lse_parts fp32 [P,B,H,N] -> (o [B,H,N,d], lse [B,H,N])."""
    torch = _torch()
    if not (o_parts.is_cuda and o_parts.dtype == torch.float32 and o_parts.dim() == 5 and o_parts.is_contiguous()):
        raise TypeError("o_parts must be a contiguous 5-D float32 CUDA tensor [P, B, H, N, d]")
    P, B, H, N, d = o_parts.shape
    _expect(lse_parts, "lse_parts", torch.float32, (P, B, H, N), o_parts.device, dense=True)
    if out is None:
        o = torch.empty((B, H, N, d), dtype=torch.float32, device=o_parts.device)
        lse = torch.empty((B, H, N), dtype=torch.float32, device=o_parts.device)
    else:
        o, lse = out
        _expect(o, "o", torch.float32, (B, H, N, d), o_parts.device, dense=True)
        _expect(lse, "lse", torch.float32, (B, H, N), o_parts.device, dense=True)
    _check(library().vitattn_merge(o_parts.data_ptr(), lse_parts.data_ptr(), P, o.data_ptr(), lse.data_ptr(), B, H,
                                   N, d, _stream_ptr(o_parts)))
    return o, lse


def _stage_args(q, names_bf16, names_f32_rows, names_f32_out, lse, workspace, B, H, N, d):
    """Checks for the dense stage entry points: bf16 operands and fp32 outputs
    of shape [B, H, N, d], lse [B, H, N], all contiguous on q's device."""
    torch = _torch()
    dev = q.device
    for t, n in names_bf16:
        _expect(t, n, torch.bfloat16, (B, H, N, d), dev, dense=True)
    for t, n in names_f32_rows + names_f32_out:
        _expect(t, n, torch.float32, (B, H, N, d), dev, dense=True)
    if lse is not None:
        _expect(lse, "lse", torch.float32, (B, H, N), dev, dense=True)
    _expect_workspace(workspace, dev)


def _shape4(t, name):
    torch = _torch()
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 4):
        raise TypeError(f"{name} must be a 4-D CUDA tensor [B, H, N, d]")
    return tuple(int(n) for n in t.shape)


def bwd_rowdot(o, dout, lse, workspace):
    B, H, N, d = _shape4(dout, "dout")
    _stage_args(dout, [(dout, "dout")], [(o, "o")], [], lse, workspace, B, H, N, d)
    _check(library().vitattn_bwd_rowdot(o.data_ptr(), dout.data_ptr(), lse.data_ptr(), B, H, N, d, workspace.data_ptr(),
                                        workspace.numel() * workspace.element_size(), _stream_ptr(dout)))


def bwd_dkdv(q, k, v, dout, lse, dk, dv, workspace, scale=None):
    B, H, N, d = _shape4(q, "q")
    _stage_args(q, [(q, "q"), (k, "k"), (v, "v"), (dout, "dout")], [], [(dk, "dk"), (dv, "dv")], lse, workspace,
                B, H, N, d)
    _check(library().vitattn_bwd_dkdv(q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(), lse.data_ptr(),
                                      dk.data_ptr(), dv.data_ptr(), B, H, N, d, _default_scale(d, scale),
                                      workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                      _stream_ptr(q)))


def bwd_dkdv_ds(q, k, v, dout, lse, dk, dv, workspace, scale=None):
    """The dK/dV stage of the dS mode (also writes the dS blocks into workspace)."""
    B, H, N, d = _shape4(q, "q")
    _stage_args(q, [(q, "q"), (k, "k"), (v, "v"), (dout, "dout")], [], [(dk, "dk"), (dv, "dv")], lse, workspace,
                B, H, N, d)
    _check(library().vitattn_bwd_dkdv_ds(q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(), lse.data_ptr(),
                                         dk.data_ptr(), dv.data_ptr(), B, H, N, d, _default_scale(d, scale),
                                         workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                         _stream_ptr(q)))


def bwd_dq_from_ds(k, dq, workspace, scale=None):
    """The dQ stage of the dS mode, from the dS blocks bwd_dkdv_ds stored."""
    B, H, N, d = _shape4(k, "k")
    _stage_args(k, [(k, "k")], [], [(dq, "dq")], None, workspace, B, H, N, d)
    _check(library().vitattn_bwd_dq_from_ds(k.data_ptr(), dq.data_ptr(), B, H, N, d, _default_scale(d, scale),
                                            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                            _stream_ptr(k)))


def bwd_dq(q, k, v, dout, lse, dq, workspace, scale=None):
    B, H, N, d = _shape4(q, "q")
    _stage_args(q, [(q, "q"), (k, "k"), (v, "v"), (dout, "dout")], [], [(dq, "dq")], lse, workspace, B, H, N, d)
    _check(library().vitattn_bwd_dq(q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(), lse.data_ptr(),
                                    dq.data_ptr(), B, H, N, d, _default_scale(d, scale), workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), _stream_ptr(q)))


def _rows(t, lead, name):
    """(leading dims, row shape, row_bytes) of a contiguous CUDA tensor whose
    first `lead` dims index rows."""
    if not (t.is_cuda and t.is_contiguous() and t.dim() > lead):
        raise TypeError(f"{name} must be a contiguous CUDA tensor with more than {lead} dims")
    row_shape = tuple(t.shape[lead:])
    row_bytes = t.element_size()
    for n in row_shape:
        row_bytes *= n
    return tuple(t.shape[:lead]), row_shape, row_bytes


def _ulysses(status, dst):
    _check(status)
    return dst


def _dst(out, shape, like):
    """`out` if given (checked), else a new tensor of `shape` like `like`."""
    torch = _torch()
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    if not (isinstance(out, torch.Tensor) and out.is_cuda and out.device == like.device and out.dtype == like.dtype
            and out.is_contiguous() and tuple(out.shape) == tuple(shape)):
        raise TypeError(f"out must be a contiguous {like.dtype} CUDA tensor of shape {tuple(shape)} on {like.device}")
    return out


def ulysses_pack(x, P, out=None):
    """x [B, Nl, H, *row] -> send [P, B, H/P, Nl, *row] (head group p in chunk p)."""
    (B, Nl, H), row, rb = _rows(x, 3, "x")
    if P < 1 or H % P != 0:
        raise ValueError("H must be a multiple of P")
    send = _dst(out, (P, B, H // P, Nl) + row, x)
    return _ulysses(library().vitattn_ulysses_pack(x.data_ptr(), send.data_ptr(), B, Nl, H, P, rb, _stream_ptr(x)),
                    send)


def ulysses_unpack(recv, out=None):
    """recv [P, B, Hl, Nl, *row] (chunk r from rank r) -> y [B, Hl, P*Nl, *row]."""
    (P, B, Hl, Nl), row, rb = _rows(recv, 4, "recv")
    y = _dst(out, (B, Hl, P * Nl) + row, recv)
    return _ulysses(library().vitattn_ulysses_unpack(recv.data_ptr(), y.data_ptr(), B, Nl, Hl * P, P, rb,
                                                     _stream_ptr(recv)), y)


def ulysses_pack_out(y, P, out=None):
    """y [B, Hl, P*Nl, *row] -> send [P, B, Hl, Nl, *row] (the inverse of unpack)."""
    (B, Hl, N), row, rb = _rows(y, 3, "y")
    if P < 1 or N % P != 0:
        raise ValueError("the sequence length must be divisible by P")
    send = _dst(out, (P, B, Hl, N // P) + row, y)
    return _ulysses(library().vitattn_ulysses_pack_out(y.data_ptr(), send.data_ptr(), B, N // P, Hl * P, P, rb,
                                                       _stream_ptr(y)), send)


def ulysses_unpack_out(recv, out=None):
    """recv [P, B, Hl, Nl, *row] -> x [B, Nl, P*Hl, *row] (the inverse of pack)."""
    (P, B, Hl, Nl), row, rb = _rows(recv, 4, "recv")
    x = _dst(out, (B, Nl, P * Hl) + row, recv)
    return _ulysses(library().vitattn_ulysses_unpack_out(recv.data_ptr(), x.data_ptr(), B, Nl, Hl * P, P, rb,
                                                         _stream_ptr(recv)), x)


def _agg_shapes(q, k, v):
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        if not (isinstance(t, _torch().Tensor) and t.is_cuda and t.dtype == _torch().bfloat16 and t.is_contiguous()
                and t.device == k.device):
            raise TypeError(f"{n} must be a contiguous bfloat16 CUDA tensor on the device of k")
    if q.dim() != 2 or k.dim() != 4 or k.shape != v.shape or k.shape[1] != q.shape[0] or k.shape[3] != q.shape[1]:
        raise ValueError("q must be [H, d] and k, v [M, H, C, d]")
    M, H, C, d = k.shape
    return M, H, C, d


def agg_fwd(q, k, v, scale=None):
    """Channel aggregation: o (fp32 [M,H,d]) and lse (fp32 [M,H]) of one shared
    query per head (q [H,d]) over each patch's C channel keys (k, v [M,H,C,d])."""
    torch = _torch()
    M, H, C, d = _agg_shapes(q, k, v)
    o = torch.empty((M, H, d), dtype=torch.float32, device=k.device)
    lse = torch.empty((M, H), dtype=torch.float32, device=k.device)
    _check(library().vitattn_agg_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), M, H, C,
                                     d, _default_scale(d, scale), _stream_ptr(k)))
    return o, lse


def agg_bwd(q, k, v, o, lse, dout, scale=None):
    """Gradients of the channel aggregation: dq (fp32 [H,d], summed over all
    patches), dk and dv (fp32 [M,H,C,d])."""
    torch = _torch()
    M, H, C, d = _agg_shapes(q, k, v)
    _expect(dout, "dout", torch.bfloat16, (M, H, d), k.device, dense=True)
    _expect(o, "o", torch.float32, (M, H, d), k.device, dense=True)
    _expect(lse, "lse", torch.float32, (M, H), k.device, dense=True)
    lib = library()
    wsb = int(lib.vitattn_agg_bwd_workspace_bytes(M, H, C, d))
    ws = torch.empty(max(wsb, 4) // 4, dtype=torch.float32, device=k.device)
    dq = torch.empty((H, d), dtype=torch.float32, device=k.device)
    dk = torch.empty((M, H, C, d), dtype=torch.float32, device=k.device)
    dv = torch.empty_like(dk)
    _check(lib.vitattn_agg_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), dout.data_ptr(),
                               lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), M, H, C, d,
                               _default_scale(d, scale), ws.data_ptr(), ws.numel() * 4, _stream_ptr(k)))
    return dq, dk, dv


# ------------------------------------------------------------------ layer norm, rotary positions

VITATTN_BF16, VITATTN_FP16, VITATTN_FP32 = 0, 1, 2
VITATTN_ROTARY_INTERLEAVED, VITATTN_ROTARY_INVERSE, VITATTN_ROTARY_JOINT = 1, 2, 4


_ALL_TYPES, _LAM_TYPES = (VITATTN_BF16, VITATTN_FP16, VITATTN_FP32), (VITATTN_BF16, VITATTN_FP32)


@functools.lru_cache(maxsize=None)
def _type_codes():
    torch = _torch()
    return {torch.bfloat16: VITATTN_BF16, torch.float16: VITATTN_FP16, torch.float32: VITATTN_FP32}


def _type_code(t, name, allowed=_ALL_TYPES):
    code = _type_codes().get(t.dtype) if isinstance(t, _torch().Tensor) and t.is_cuda else None
    if code is None or code not in allowed:
        names = ", ".join(str(d) for d, c in _type_codes().items() if c in allowed)
        raise TypeError(f"{name} must be a CUDA tensor of one of {names}")
    if t.is_neg():
        _negated(name)
    return code


def _negated(name):
    """Of a tensor whose memory holds its values negated (the imaginary part of a
    conjugate, which torch negates when it reads it)."""
    raise TypeError(f"{name} is a lazily negated view: pass {name}.resolve_neg()")


def _as_it_is(t, name):
    if t.is_neg():
        _negated(name)
    return t


def _call(t, fn, *args):
    """fn(*args, stream) on t's device and its current stream."""
    device = t.device.index
    cuda = _torch().cuda
    if device == cuda.current_device():
        status = fn(*args, _raw_stream()(device))
    else:
        with cuda.device(device):
            status = fn(*args, _raw_stream()(device))
    if status != 0:
        raise VitattnError(status)


def _expect_out(t, name, dtype, shape, device, dense=False):
    """_expect for a tensor that a call writes: as in torch, one that requires a
    gradient is refused where gradients are recorded."""
    _as_it_is(_expect(t, name, dtype, shape, device, dense), name)
    if t.requires_grad and _torch().is_grad_enabled():
        raise ValueError(f"{name} requires a gradient: it is written outside autograd (detach it, or call under no_grad)")
    return t


def _written(*ts):
    """Tells autograd that these were written, as torch's own in-place operations do: the backward of an operation that
    saved one raises instead of reading what it has become."""
    _torch().autograd.graph.increment_version(ts)


def plain_memory(t):
    """t, or a copy where its memory does not hold its values as they are: a
    lazily negated view, zeros without memory, a last dim that is not contiguous."""
    if (t.shape[-1] != 1 and t.stride(-1) != 1) or t.is_neg() or (t.numel() and t.data_ptr() == 0):
        return _torch().empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)
    return t


def _new_like(t):
    """A new tensor in t's order of dims, the last one contiguous: torch's order of
    a sliding window's (whose rows start one element apart) may put another there."""
    y = _torch().empty_like(t)
    if y.is_contiguous() or y.stride(-1) == 1 or y.shape[-1] == 1:
        return y
    return _torch().empty(t.shape, dtype=t.dtype, device=t.device)


def _norm_view(t, name):
    """t as the rows of a layer norm; more than three leading dims become one (by
    a copy where t's layout needs it)."""
    n = t.dim()
    if n < 1 or (t.stride(-1) != 1 and t.shape[-1] != 1):
        raise TypeError(f"{name} must have at least one dim, the last with unit stride")
    return t if n <= 4 else t.reshape(-1, t.shape[-1])


def _norm_rows(*ts):
    """The row dimensions of tensors of one shape (up to three): the order in
    which the first tensor's memory has them (None: one dimension, all of them
    contiguous) and their sizes padded to three."""
    x = ts[0]
    for t in ts:
        if not t.is_contiguous():
            break
    else:
        return None, (1, 1, x.numel() // x.shape[-1])
    lead = x.dim() - 1
    order = sorted(range(lead), key=lambda i: (-x.stride(i), i))
    return order, (1,) * (3 - lead) + tuple(x.shape[i] for i in order)


@functools.lru_cache(maxsize=1024)
def _strides(batch, head, row):
    """Strides(batch, head, row), which nobody writes."""
    return Strides(batch, head, row)


def _norm_strides(t, order, D):
    if order is None:
        return _strides(0, 0, D)
    return _strides(*[0] * (3 - len(order)), *(0 if t.shape[i] == 1 else t.stride(i) for i in order))


def _norm_weights(x, D, weight, bias):
    """The type of weight and bias, checked (x's without any)."""
    wt, dtype, device, torch = None, x.dtype, x.device, _torch()
    for t, n in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        if not (isinstance(t, torch.Tensor) and (t.dtype == dtype or t.dtype == torch.float32) and t.shape == (D,)
                and t.device == device and t.is_contiguous()):
            raise TypeError(f"{n} must be a contiguous {dtype} or torch.float32 CUDA tensor of shape ({D},) on {device}")
        if wt is not None and t.dtype != wt:
            raise TypeError("weight and bias must be of one type")
        if t.is_neg():
            _negated(n)
        wt = t.dtype
    return dtype if wt is None else wt


def _ptr(t):
    return None if t is None else t.data_ptr()


def layer_norm_fwd(x, weight=None, bias=None, eps=1e-5, out=None, stats=True):
    """Layer norm over the last dim of x (bf16, fp16 or fp32; any strides with
    that dim contiguous): y like x, and the rows' mean and 1/sqrt(var + eps) in
    fp32 (x.shape[:-1]; None, None without stats). weight and bias: [D], of x's
    type or fp32. out: the tensor to write, may be x."""
    torch = _torch()
    code = _type_code(x, "x")
    x4 = _norm_view(x, "x")
    D = x4.shape[-1]
    wt = _norm_weights(x, D, weight, bias)
    if x.numel() == 0:
        raise ValueError("layer_norm needs at least one row and one column")
    if out is None:
        y = _new_like(x) if x4 is x else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        y = _expect_out(out, "out", x.dtype, x.shape, x.device, dense=x4 is not x)
    y4 = y if x4 is x else y.view(x4.shape)
    order, n = _norm_rows(x4, y4)
    mean = rstd = None
    if stats:
        mean = torch.empty(x.shape[:-1] if order is None else n, dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
    _call(x, library().vitattn_layer_norm_fwd, x4.data_ptr(), _norm_strides(x4, order, D), _ptr(weight), _ptr(bias),
          y.data_ptr(), _norm_strides(y4, order, D), _ptr(mean), _ptr(rstd), *n, D, eps, code,
          VITATTN_FP32 if wt == torch.float32 else code)
    if out is not None:
        _written(out)
    if order is not None and stats:
        mean, rstd = _norm_stat_out(mean, order, x4, x.shape), _norm_stat_out(rstd, order, x4, x.shape)
    return y, mean, rstd


def _norm_stat_out(t, order, x4, shape):
    """A statistic in the kernel's order of rows, as x.shape[:-1]."""
    t = t.view([x4.shape[i] for i in order]).permute(sorted(range(len(order)), key=lambda i: order[i]))
    return t.reshape(shape[:-1])


def layer_norm_bwd(x, weight, mean, rstd, dy, want_dweight=True, want_dbias=True, bias_dtype=None, workspace=None):
    """dx, dweight and dbias of layer_norm_fwd for the upstream gradient dy (x's
    shape and type); dweight is None without a weight or if not wanted, dbias if
    not wanted. Without a weight dbias has bias_dtype (default x's)."""
    torch = _torch()
    code = _type_code(x, "x")
    x4 = _norm_view(x, "x")
    shape, device = x.shape, x.device
    D, rows = shape[-1], shape[:-1]
    _as_it_is(_expect(dy, "dy", x.dtype, shape, device), "dy")
    for t, n in ((mean, "mean"), (rstd, "rstd")):
        if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype == torch.float32 and t.shape == rows):
            raise TypeError(f"{n} must be a torch.float32 CUDA tensor of shape {tuple(rows)} on {device}")
    wt = _norm_weights(x, D, weight, None)
    if weight is None and bias_dtype is not None:
        if bias_dtype not in (x.dtype, torch.float32):
            raise TypeError(f"bias_dtype must be {x.dtype} or torch.float32")
        wt = bias_dtype
    if x.numel() == 0:
        raise ValueError("layer_norm needs at least one row and one column")
    dx = _new_like(x) if x4 is x else torch.empty(shape, dtype=x.dtype, device=x.device)
    dy4, dx4 = _norm_view(dy, "dy"), dx if x4 is x else dx.view(x4.shape)
    order, n = _norm_rows(x4, dy4, dx4)
    if order is not None:
        mean, rstd = (t.reshape(x4.shape[:-1]).permute(order) for t in (mean, rstd))
    mean, rstd = mean.contiguous(), rstd.contiguous()  # (rows of x in memory order)
    dw = torch.empty(D, dtype=wt, device=device) if want_dweight and weight is not None else None
    db = torch.empty(D, dtype=wt, device=device) if want_dbias else None
    lib, size = library(), 0
    if workspace is not None:
        size = _expect_workspace(workspace, device).numel() * workspace.element_size()
    elif dw is not None or db is not None:
        size = lib.vitattn_layer_norm_bwd_workspace_bytes(*n, D, code)
        workspace = torch.empty(size // 4, dtype=torch.float32, device=device)
    _call(x, lib.vitattn_layer_norm_bwd, x4.data_ptr(), _norm_strides(x4, order, D), _ptr(weight), mean.data_ptr(),
          rstd.data_ptr(), dy4.data_ptr(), _norm_strides(dy4, order, D), dx4.data_ptr(), _norm_strides(dx4, order, D),
          _ptr(dw), _ptr(db), *n, D, code, VITATTN_FP32 if wt == torch.float32 else code, _ptr(workspace), size)
    return dx, dw, db


def _strides_any(t):
    """Strides of a [B, H, N, d] view, zeros for dims of size one."""
    (b, h, r, _), (B, H, N, _) = t.stride(), t.shape
    return _strides(b if B != 1 else 0, h if H != 1 else 0, r if N != 1 else 0)


@functools.lru_cache(maxsize=None)
def _pos_codes():
    torch = _torch()
    return {torch.int32: 0, torch.int64: 1, torch.float32: 2}


@functools.lru_cache(maxsize=256)
def _c_ints(values):
    """A C array of these ints, which nobody writes."""
    return (c_int * max(len(values), 1))(*map(Int.from_param, values))


def rotary_fwd(q, k, positions, sections, base=10000.0, interleaved=False, joint=False, inverse=False, out=None):
    """q [B,Hq,N,d] and k [B,Hk,N,d] (or None) with pairs of columns turned by
    their positions: sections[a] pairs for axis a, positions [N, A] or [B, N, A]
    (int32, int64 or fp32). Pair p is columns p and R + p of the first 2 R (2p and
    2p + 1 if interleaved); frequencies base^(-i/n) over an axis's n pairs, or
    over all R (joint). inverse turns back: the gradient. out=(q', k') to write
    into, which may be q and k. Returns q', or (q', k') if there is a k."""
    torch = _torch()
    code = _type_code(q, "q")
    device, dtype = q.device, q.dtype
    for t, n in ((q, "q"), (k, "k")):
        if t is None:
            continue
        if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.device == device and t.dim() == 4
                and (t.stride(3) == 1 or t.shape[3] == 1)):
            raise TypeError(f"{n} must be a 4-D CUDA tensor [B, H, N, d] of q's type and device with unit stride along d")
    B, Hq, N, d = q.shape
    Hk = 0
    if k is not None:
        Bk, Hk, Nk, dk = k.shape
        if (Bk, Nk, dk) != (B, N, d):
            raise ValueError("k must be [B, Hk, N, d] with the B, N and d of q")
    sections = tuple(sections)
    try:
        sections = tuple(map(operator.index, sections))
    except TypeError:
        if sections != tuple(map(int, sections)):
            raise ValueError("sections must be whole numbers") from None
        sections = tuple(map(int, sections))
    A = len(sections)
    pos_code = _pos_codes().get(positions.dtype) if isinstance(positions, torch.Tensor) else None
    if pos_code is None or positions.device != device or positions.shape not in ((N, A), (B, N, A)):
        raise TypeError(f"positions must be an int32, int64 or float32 tensor [{N}, {A}] or [{B}, {N}, {A}] on {device}")
    if positions.is_neg() or k is not None and k.is_neg():
        _negated("positions" if positions.is_neg() else "k")
    k_out, sk, sk_out = None, _NO_STRIDES, _NO_STRIDES
    if out is None:
        q_out = _new_like(q)
        if k is not None:
            k_out = _new_like(k)
    else:
        q_out, k_out = out if k is not None else ((out[0] if isinstance(out, (tuple, list)) else out), None)
        for t, like, n in ((q_out, q, "out q"), (k_out, k, "out k")):
            if like is not None:
                _expect_out(t, n, dtype, like.shape, device)
    if k is not None:
        sk, sk_out = _strides_any(k), _strides_any(k_out)
    sp = positions.stride()
    flags = ((VITATTN_ROTARY_INTERLEAVED if interleaved else 0) | (VITATTN_ROTARY_INVERSE if inverse else 0)
             | (VITATTN_ROTARY_JOINT if joint else 0))
    _call(q, library().vitattn_rotary, q.data_ptr(), _strides_any(q), q_out.data_ptr(), _strides_any(q_out), Hq,
          _ptr(k), sk, _ptr(k_out), sk_out, Hk, positions.data_ptr(), sp[0] if len(sp) == 3 else 0, sp[-2], sp[-1],
          pos_code, _c_ints(sections), A, float(base), B, N, d, code, flags)
    if out is not None:
        _written(q_out) if k is None else _written(q_out, k_out)
    return q_out if k is None else (q_out, k_out)


_NO_STRIDES = Strides(0, 0, 0)

# ------------------------------------------------------------------ differential attention


def _diff_strides(t):
    """Strides of a [B, H, N, d] view as the attention takes them; those of dims
    of size one do not matter and are replaced."""
    (b, h, r, _), (B, H, N, d) = t.stride(), t.shape
    return _strides(b if B != 1 else 0, h if H != 1 else 0, r if N != 1 else d)


def _diff_args(q, k, v, lam, key_lens):
    _as_input(q, "q")
    device = q.device
    _as_input(k, "k", device)
    _as_input(v, "v", device)
    if q.is_neg() or k.is_neg() or v.is_neg():
        _negated("q" if q.is_neg() else "k" if k.is_neg() else "v")
    B, H2, Nq, d = q.shape
    Bv, H, Nk, e = v.shape
    if H2 != 2 * H or Bv != B or tuple(k.shape) != (B, H2, Nk, d):
        raise ValueError("q must be [B, 2H, Nq, d], k [B, 2H, Nk, d] and v [B, H, Nk, e]")
    lam_code = _type_code(lam, "lam", _LAM_TYPES)
    _expect(lam, "lam", lam.dtype, (H,), device, dense=True)
    if key_lens is not None:
        _expect(key_lens, "key_lens", _torch().int32, (B,), device, dense=True)
    return (B, H, Nq, Nk, d, e), lam_code


def _like_layout(t, shape):
    """A new tensor [B, H, N, e] in t's order of heads and rows."""
    torch = _torch()
    B, H, N, e = shape
    s, n = t.stride(), t.shape
    if n[1] > 1 and n[2] > 1 and s[1] < s[2]:
        return torch.empty((B, N, H, e), dtype=t.dtype, device=t.device).transpose(1, 2)
    return torch.empty(shape, dtype=t.dtype, device=t.device)


def _diff_workspace(workspace, need, device):
    torch = _torch()
    if workspace is None:
        return torch.empty(max(need, 4) // 4, dtype=torch.float32, device=device)
    return _expect_workspace(workspace, device)


def diff_fwd(q, k, v, lam, scale=None, key_lens=None, out=None, save=True, workspace=None):
    """Differential attention: o (bf16 [B,H,Nq,e], in q's order of heads and rows)
    = softmax(scale Q1 K1^T) V - lam softmax(scale Q2 K2^T) V for q [B,2H,Nq,d], k
    [B,2H,Nk,d] (heads 2h and 2h + 1 are the two maps of head h), v [B,H,Nk,e] and
    lam [H] (fp32 or bf16). key_lens: int32 [B], sample b attends to its first
    key_lens[b] keys. Returns o and what diff_bwd needs: o2 (fp32 [B,2H,Nq,e], each
    map's output before the difference) and lse (fp32 [B,2H,Nq]); None, None
    unless save."""
    torch = _torch()
    sizes, lam_code = _diff_args(q, k, v, lam, key_lens)
    B, H, Nq, Nk, d, e = sizes
    o = (_like_layout(q, (B, H, Nq, e)) if out is None
         else _expect_out(out, "out", torch.bfloat16, (B, H, Nq, e), q.device))
    o2 = lse = None
    if save:
        o2 = torch.empty((B, 2 * H, Nq, e), dtype=torch.float32, device=q.device)
        lse = torch.empty((B, 2 * H, Nq), dtype=torch.float32, device=q.device)
    lib = library()
    need = int(lib.vitattn_diff_fwd_workspace_bytes(*sizes))
    ws = _diff_workspace(workspace, need, q.device) if need or workspace is not None else None
    _call(q, lib.vitattn_diff_fwd, q.data_ptr(), _diff_strides(q), k.data_ptr(), _diff_strides(k), v.data_ptr(),
          _diff_strides(v), lam.data_ptr(), lam_code, _ptr(key_lens), o.data_ptr(), _diff_strides(o), _ptr(o2), _ptr(lse),
          *sizes, _default_scale(d, scale), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())
    if out is not None:
        _written(out)
    return o, o2, lse


def diff_bwd(q, k, v, lam, o, o2, lse, dout, scale=None, key_lens=None, want_dlam=True, workspace=None):
    """dq, dk, dv (bf16, like q, k and v) and dlam (lam's type, or None) of
    diff_fwd for the upstream gradient dout (bf16 [B,H,Nq,e]). The kernels read
    the unrounded outputs in o2; o (or None) is only checked to belong to the same
    call's sizes."""
    torch = _torch()
    sizes, lam_code = _diff_args(q, k, v, lam, key_lens)
    B, H, Nq, Nk, d, e = sizes
    if o is not None:
        _expect(o, "o", torch.bfloat16, (B, H, Nq, e), q.device)
    _expect(o2, "o2", torch.float32, (B, 2 * H, Nq, e), q.device, dense=True)
    _expect(lse, "lse", torch.float32, (B, 2 * H, Nq), q.device, dense=True)
    _as_it_is(_expect(dout, "dout", torch.bfloat16, (B, H, Nq, e), q.device), "dout")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dlam = torch.empty_like(lam) if want_dlam else None
    lib = library()
    ws = _diff_workspace(workspace, int(lib.vitattn_diff_bwd_workspace_bytes(*sizes)), q.device)
    _call(q, lib.vitattn_diff_bwd, q.data_ptr(), _diff_strides(q), k.data_ptr(), _diff_strides(k), v.data_ptr(),
          _diff_strides(v), lam.data_ptr(), lam_code, _ptr(key_lens), o2.data_ptr(), lse.data_ptr(), dout.data_ptr(),
          _diff_strides(dout), dq.data_ptr(), _diff_strides(dq), dk.data_ptr(), _diff_strides(dk), dv.data_ptr(),
          _diff_strides(dv), _ptr(dlam), *sizes, _default_scale(d, scale), ws.data_ptr(), ws.numel() * ws.element_size())
    return dq, dk, dv, dlam
