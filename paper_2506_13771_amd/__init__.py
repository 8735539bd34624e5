"""LittleBit linear layer on MI355X (gfx950): Python binding of liblittlebit.so.

This module only marshals arguments into the C ABI declared in
include/littlebit.h: every step of the computation runs in the library's HIP
kernels.  PyTorch provides device memory and the current stream.  If the
library is not built, or a tensor is not on a GPU, calls raise instead of
falling back to anything else.

The names follow the C ABI:
  lb_pack_signs, lb_linear_forward, lb_dense_reference_weight,
  lb_packed_bytes, lb_bits_per_weight, lb_rank_for_bpw,
  lb_forward_workspace_bytes, lb_workspace_init, lb_workspace_status, lb_decode_max_tokens,
  lb_linear_forward_many, lb_forward_many_workspace_bytes,
  lb_list_workspace_bytes, lb_list_init, lb_list_forward (class LittleBitList),
  lb_linear_latent, lb_latent_workspace_bytes,
  lb_linear_from_latent, lb_from_latent_workspace_bytes,
  lb_linear_backward, lb_backward_workspace_bytes,
  lb_rotate, lb_latent_row, lb_latent_append, lb_latent_attention, lb_latent_attention_workspace_bytes
  (class LatentCache), lb_attention_forward, lb_attention_backward, lb_attention_backward_workspace_bytes.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblittlebit.so")

LB_OK, LB_ERR_NULL, LB_ERR_SHAPE, LB_ERR_DTYPE, LB_ERR_ALIGN, LB_ERR_WORKSPACE, LB_ERR_HIP, LB_ERR_ARG = range(8)
LB_F32, LB_F16, LB_BF16 = 0, 1, 2
LB_ROLE_U, LB_ROLE_V = 0, 1
LB_KERNEL_AUTO, LB_KERNEL_DECODE, LB_KERNEL_PREFILL, LB_KERNEL_DECODE_MFMA = 0, 1, 2, 3
ABI_VERSION = 8


class LittleBitError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {lb_status_str(status)} ({status})")
        self.status = status


class lb_path(ctypes.Structure):
    _fields_ = [("U", ctypes.c_void_p), ("V", ctypes.c_void_p), ("h", ctypes.c_void_p),
                ("g", ctypes.c_void_p), ("l", ctypes.c_void_p)]


class lb_linear_desc(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("act_dtype", ctypes.c_int), ("T", ctypes.c_int64),
                ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64), ("r", ctypes.c_int64),
                ("paths", lb_path * 2), ("scale_dtype", ctypes.c_int), ("y", ctypes.c_void_p)]


class lb_path_train(ctypes.Structure):
    _fields_ = [("U_latent", ctypes.c_void_p), ("V_latent", ctypes.c_void_p), ("Ut", ctypes.c_void_p),
                ("Vt", ctypes.c_void_p), ("dU", ctypes.c_void_p), ("dV", ctypes.c_void_p), ("dh", ctypes.c_void_p),
                ("dg", ctypes.c_void_p), ("dl", ctypes.c_void_p)]


class lb_svid_out(ctypes.Structure):
    _fields_ = [("U_latent", ctypes.c_void_p), ("V_latent", ctypes.c_void_p), ("h", ctypes.c_void_p),
                ("g", ctypes.c_void_p), ("l", ctypes.c_void_p), ("sigma", ctypes.c_void_p)]


class lb_latent_cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int), ("n_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int64), ("r", ctypes.c_int64), ("d_rope", ctypes.c_int64),
                ("table", ctypes.c_void_p), ("n_seq", ctypes.c_int64), ("max_pages", ctypes.c_int64),
                ("lens", ctypes.c_void_p), ("cu", ctypes.c_void_p)]


class lb_attention(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_rope", ctypes.c_void_p),
                ("dtype", ctypes.c_int), ("Tq", ctypes.c_int64), ("Tk", ctypes.c_int64), ("H", ctypes.c_int64),
                ("Hk", ctypes.c_int64), ("d_nope", ctypes.c_int64), ("d_rope", ctypes.c_int64), ("d_v", ctypes.c_int64),
                ("q_t", ctypes.c_int64), ("q_h", ctypes.c_int64), ("k_t", ctypes.c_int64), ("k_h", ctypes.c_int64),
                ("v_t", ctypes.c_int64), ("v_h", ctypes.c_int64), ("kr_t", ctypes.c_int64), ("cu_q", ctypes.c_void_p),
                ("cu_k", ctypes.c_void_p), ("n_seq", ctypes.c_int64), ("causal", ctypes.c_int),
                ("scale", ctypes.c_float)]


class lb_attention_grads(ctypes.Structure):
    _fields_ = [("dq", ctypes.c_void_p), ("dk", ctypes.c_void_p), ("dv", ctypes.c_void_p), ("dk_rope", ctypes.c_void_p),
                ("dk_t", ctypes.c_int64), ("dk_h", ctypes.c_int64), ("dv_t", ctypes.c_int64), ("dv_h", ctypes.c_int64)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load liblittlebit.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"LittleBit HIP library not built: {path} is missing "
                           "(run __graft_entry__.build() or python paper_2506_13771_amd/_build.py)")
    lib = ctypes.CDLL(path)
    i64, sz, vp, i32 = ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int
    lib.lb_abi_version.restype = i32
    lib.lb_abi_version.argtypes = []
    lib.lb_status_str.restype = ctypes.c_char_p
    lib.lb_status_str.argtypes = [i32]
    lib.lb_packed_bytes.restype = sz
    lib.lb_packed_bytes.argtypes = [i32, i64, i64]
    lib.lb_bits_per_weight.restype = ctypes.c_double
    lib.lb_bits_per_weight.argtypes = [i64, i64, i64, i32]
    lib.lb_rank_for_bpw.restype = i64
    lib.lb_rank_for_bpw.argtypes = [i64, i64, ctypes.c_double, i64]
    lib.lb_pack_signs.restype = i32
    lib.lb_pack_signs.argtypes = [vp, i32, i64, i64, i32, vp, vp, vp]
    lib.lb_forward_workspace_bytes.restype = sz
    lib.lb_forward_workspace_bytes.argtypes = [i64, i64, i64, i64]
    lib.lb_workspace_init.restype = i32
    lib.lb_workspace_init.argtypes = [vp, sz, vp]
    lib.lb_workspace_status.restype = i32
    lib.lb_workspace_status.argtypes = [vp, sz, vp, vp]
    lib.lb_decode_max_tokens.restype = i64
    lib.lb_decode_max_tokens.argtypes = []
    lib.lb_linear_forward.restype = i32
    lib.lb_linear_forward.argtypes = [vp, i32, i64, i64, i64, i64, ctypes.POINTER(lb_path), i32, vp, vp, sz, vp]
    lib.lb_linear_forward_kernel.restype = i32
    lib.lb_linear_forward_kernel.argtypes = [vp, i32, i64, i64, i64, i64, ctypes.POINTER(lb_path), i32, vp, vp,
                                             sz, i32, vp]
    lib.lb_noalloc_scratch_bytes.restype = sz
    lib.lb_noalloc_scratch_bytes.argtypes = []
    lib.lb_linear_forward_noalloc.restype = i32
    lib.lb_linear_forward_noalloc.argtypes = [vp, i32, i64, i64, i64, i64, ctypes.POINTER(lb_path), i32, vp, vp]
    lib.lb_forward_many_workspace_bytes.restype = sz
    lib.lb_forward_many_workspace_bytes.argtypes = [ctypes.POINTER(lb_linear_desc), i64]
    lib.lb_linear_forward_many.restype = i32
    lib.lb_linear_forward_many.argtypes = [ctypes.POINTER(lb_linear_desc), i64, vp, sz, vp]
    lib.lb_list_workspace_bytes.restype = sz
    lib.lb_list_workspace_bytes.argtypes = [ctypes.POINTER(lb_linear_desc), i64]
    lib.lb_list_init.restype = i32
    lib.lb_list_init.argtypes = [ctypes.POINTER(lb_linear_desc), i64, vp, sz, vp]
    lib.lb_list_forward.restype = i32
    lib.lb_list_forward.argtypes = [ctypes.POINTER(lb_linear_desc), i64, vp, sz, vp]
    lib.lb_latent_workspace_bytes.restype = sz
    lib.lb_latent_workspace_bytes.argtypes = [i64, i64, i64]
    lib.lb_linear_latent.restype = i32
    lib.lb_linear_latent.argtypes = [vp, i32, i64, i64, i64, ctypes.POINTER(lb_path), i32, vp, i32, vp, sz, vp]
    lib.lb_from_latent_workspace_bytes.restype = sz
    lib.lb_from_latent_workspace_bytes.argtypes = [i64, i64]
    lib.lb_linear_from_latent.restype = i32
    lib.lb_linear_from_latent.argtypes = [vp, i32, i64, i64, i64, ctypes.POINTER(lb_path), i32, vp, i32, vp, sz,
                                          vp]
    lib.lb_backward_workspace_bytes.restype = sz
    lib.lb_backward_workspace_bytes.argtypes = [i64, i64, i64, i64]
    lib.lb_linear_backward.restype = i32
    lib.lb_linear_backward.argtypes = [vp, vp, i32, i64, i64, i64, i64, ctypes.POINTER(lb_path), i32,
                                       ctypes.POINTER(lb_path_train), ctypes.c_float, vp, vp, sz, vp]
    lib.lb_dense_reference_weight.restype = i32
    lib.lb_dense_reference_weight.argtypes = [ctypes.POINTER(lb_path), i32, i64, i64, i64, vp, vp]
    lib.lb_dual_svid_workspace_bytes.restype = sz
    lib.lb_dual_svid_workspace_bytes.argtypes = [i64, i64, i64, i64]
    lib.lb_dual_svid.restype = i32
    lib.lb_dual_svid.argtypes = [vp, i32, i64, i64, i64, i64, i32, ctypes.c_uint64, ctypes.POINTER(lb_svid_out), vp,
                                 vp, sz, vp]
    f32 = ctypes.c_float
    lib.lb_latent_row.restype = i64
    lib.lb_latent_row.argtypes = [i64, i64]
    lib.lb_rotate.restype = i32
    lib.lb_rotate.argtypes = [vp, i32, i64, i64, i64, i64, i64, vp, vp, i32, vp, i64, i64, vp]
    lib.lb_latent_append.restype = i32
    # (structures by address: the binding packs them as bytes, which takes a third of a ctypes object's time)
    lib.lb_latent_append.argtypes = [vp, vp, vp, i64, i32, i64, vp, vp]
    lib.lb_latent_attention_workspace_bytes.restype = sz
    lib.lb_latent_attention_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    lib.lb_latent_attention.restype = i32
    lib.lb_latent_attention.argtypes = [vp, i32, i64, i64, i64, i64, i64, i64, i64, vp, i32, vp, vp, f32, vp, vp, sz, vp]
    lib.lb_attention_forward.restype = i32
    lib.lb_attention_forward.argtypes = [vp, vp, vp, vp]
    lib.lb_attention_backward_workspace_bytes.restype = sz
    lib.lb_attention_backward_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    lib.lb_attention_backward.restype = i32
    lib.lb_attention_backward.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
    if lib.lb_abi_version() != ABI_VERSION:
        raise RuntimeError("liblittlebit.so ABI version mismatch")
    _lib = lib
    return lib


# ----------------------------------------------------------------------------
# pure host helpers
# ----------------------------------------------------------------------------
def lb_status_str(status: int) -> str:
    return load_library().lb_status_str(status).decode()


def lb_packed_bytes(role: int, rows: int, r: int) -> int:
    return int(load_library().lb_packed_bytes(role, rows, r))


def lb_bits_per_weight(d_in: int, d_out: int, r: int, npaths: int = 2) -> float:
    return float(load_library().lb_bits_per_weight(d_in, d_out, r, npaths))


def lb_rank_for_bpw(d_in: int, d_out: int, bpw: float, mult: int = 16) -> int:
    return int(load_library().lb_rank_for_bpw(d_in, d_out, bpw, mult))


def lb_forward_workspace_bytes(T: int, d_in: int, d_out: int, r: int) -> int:
    return int(load_library().lb_forward_workspace_bytes(T, d_in, d_out, r))


def lb_decode_max_tokens() -> int:
    return int(load_library().lb_decode_max_tokens())


# ----------------------------------------------------------------------------
# tensor marshalling
# ----------------------------------------------------------------------------
# torch, its dtypes' codes and its current-stream call, filled on first use (the
# package imports without torch).  A call's host work is these few lookups per
# tensor: with an import statement, a new dict and a Stream object per lookup it
# took 12.7 us per lb_linear_forward, twice the decode kernel's time.
_T = None
_CODES = {}
_current_stream = None


def _torch():
    global _T, _current_stream
    if _T is None:
        import torch
        _CODES.update({torch.float32: LB_F32, torch.float16: LB_F16, torch.bfloat16: LB_BF16})
        raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and dev is not None:
            _current_stream = lambda: raw(dev())  # noqa: E731
        else:
            _current_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
        _T = torch
    return _T


def _dtype_code(t) -> int:
    _torch()
    c = _CODES.get(t.dtype)
    if c is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return c


def _torch_dtype(code: int):
    torch = _torch()
    return {LB_F32: torch.float32, LB_F16: torch.float16, LB_BF16: torch.bfloat16}[code]


def _dev_ptr(t, name: str) -> int:
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    # (the first call initialises CUDA; the raw call needs that done)
    return _current_stream() if torch.cuda.is_initialized() else torch.cuda.current_stream().cuda_stream


def _check(status: int, what: str):
    if status != LB_OK:
        raise LittleBitError(status, what)


@dataclass
class LittleBitPath:
    """One path's packed signs (uint8 device tensors in LB layout v1) and scales."""
    U: object
    V: object
    h: object
    g: object
    l: object


_PathPair = lb_path * 2


def _paths_struct(paths: Sequence[LittleBitPath]):
    if len(paths) != 2:
        raise ValueError("exactly two paths (primary, residual) are required")
    p, q = paths
    arr = _PathPair((_dev_ptr(p.U, "U"), _dev_ptr(p.V, "V"), _dev_ptr(p.h, "h"), _dev_ptr(p.g, "g"),
                     _dev_ptr(p.l, "l")),
                    (_dev_ptr(q.U, "U"), _dev_ptr(q.V, "V"), _dev_ptr(q.h, "h"), _dev_ptr(q.g, "g"),
                     _dev_ptr(q.l, "l")))
    sc = {_dtype_code(t) for t in (p.h, p.g, p.l, q.h, q.g, q.l) if t is not None}
    if len(sc) != 1:
        raise TypeError("all scales must share one dtype")
    return arr, sc.pop()


def lb_pack_signs(src, role: int, dst=None, nan_count=None, stream=None):
    """Pack the signs of src [rows, r] (latent U or V) into dst (uint8, LB layout v1)."""
    torch = _torch()
    lib = load_library()
    rows, r = src.shape
    n = lb_packed_bytes(role, rows, r)
    if dst is None:
        dst = torch.empty(n, dtype=torch.uint8, device=src.device)
    if dst.numel() * dst.element_size() < n:
        raise ValueError("dst too small")
    st = lib.lb_pack_signs(_dev_ptr(src, "src"), _dtype_code(src), rows, r, role, _dev_ptr(dst, "dst"),
                           _dev_ptr(nan_count, "nan_count"), _stream(stream))
    _check(st, "lb_pack_signs")
    return dst


def lb_workspace_init(ws, stream=None):
    st = load_library().lb_workspace_init(_dev_ptr(ws, "workspace"), ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "lb_workspace_init")
    return ws


def lb_workspace_status(ws, stream=None) -> int:
    """Read and clear the workspace's error word (0: no bounded wait expired since the last clear);
    synchronises the stream to return the value."""
    torch = _torch()
    out = torch.full((1,), -1, dtype=torch.int32, device=ws.device)
    st = load_library().lb_workspace_status(_dev_ptr(ws, "workspace"), ws.numel() * ws.element_size(),
                                            _dev_ptr(out, "status"), _stream(stream))
    _check(st, "lb_workspace_status")
    return int(out.item())


def alloc_workspace(T: int, d_in: int, d_out: int, r: int, device="cuda"):
    """A zero-filled workspace tensor of lb_forward_workspace_bytes(T, d_in, d_out, r) bytes."""
    torch = _torch()
    n = lb_forward_workspace_bytes(T, d_in, d_out, r)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)
    return lb_workspace_init(ws)


def lb_linear_forward(x, paths: Sequence[LittleBitPath], r: int, y=None, workspace=None,
                      kernel: int = LB_KERNEL_AUTO, stream=None):
    """y [T, d_out] = LittleBit forward of x [T, d_in] with both paths; returns y."""
    torch = _torch()
    lib = load_library()
    T, d_in = x.shape
    d_out = paths[0].h.shape[0]
    arr, sc = _paths_struct(paths)
    if y is None:
        y = torch.empty((T, d_out), dtype=x.dtype, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(T, d_in, d_out, r, device=x.device)
    st = lib.lb_linear_forward_kernel(_dev_ptr(x, "x"), _dtype_code(x), T, d_in, d_out, r, arr, sc,
                                      _dev_ptr(y, "y"), _dev_ptr(workspace, "workspace"),
                                      workspace.numel() * workspace.element_size(), kernel, _stream(stream))
    _check(st, "lb_linear_forward")
    return y


def lb_linear_forward_noalloc(x, paths: Sequence[LittleBitPath], r: int, y=None, stream=None):
    """lb_linear_forward with the library's static per-GPU scratch as workspace (no workspace argument,
    nothing allocated by the call); y is allocated here when None."""
    torch = _torch()
    lib = load_library()
    T, d_in = x.shape
    d_out = paths[0].h.shape[0]
    arr, sc = _paths_struct(paths)
    if y is None:
        y = torch.empty((T, d_out), dtype=x.dtype, device=x.device)
    st = lib.lb_linear_forward_noalloc(_dev_ptr(x, "x"), _dtype_code(x), T, d_in, d_out, r, arr, sc,
                                       _dev_ptr(y, "y"), _stream(stream))
    _check(st, "lb_linear_forward_noalloc")
    return y


def make_descs(items):
    """A ctypes array of lb_linear_desc for items (x, paths, r, y) (y allocated when None); returns
    (array, list of y).  The tensors must outlive every call that uses the array."""
    torch = _torch()
    arr = (lb_linear_desc * max(len(items), 1))()
    ys = []
    for i, (x, paths, r, y) in enumerate(items):
        T, d_in = x.shape
        d_out = paths[0].h.shape[0]
        parr, sc = _paths_struct(paths)
        if y is None:
            y = torch.empty((T, d_out), dtype=x.dtype, device=x.device)
        arr[i] = lb_linear_desc(_dev_ptr(x, "x"), _dtype_code(x), T, d_in, d_out, r, parr, sc, _dev_ptr(y, "y"))
        ys.append(y)
    return arr, ys


def lb_forward_many_workspace_bytes(descs, n: int) -> int:
    return int(load_library().lb_forward_many_workspace_bytes(descs, n))


def lb_linear_forward_many(items, workspace=None, stream=None):
    """The LittleBit forward of every (x, paths, r, y) of items (independent linears) in as few launches as
    the library can; returns the list of y."""
    torch = _torch()
    lib = load_library()
    arr, ys = make_descs(items)
    n = len(items)
    if workspace is None:
        need = lb_forward_many_workspace_bytes(arr, n)
        workspace = lb_workspace_init(torch.empty(max(need, 256), dtype=torch.uint8, device=ys[0].device if ys else "cuda"))
    st = lib.lb_linear_forward_many(arr, n, _dev_ptr(workspace, "workspace"),
                                    workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "lb_linear_forward_many")
    return ys


def lb_list_workspace_bytes(descs, n: int) -> int:
    return int(load_library().lb_list_workspace_bytes(descs, n))


class LittleBitList:
    """A fixed list of decode-sized linears (items (x, paths, r, y), y allocated when None) run by the
    streaming list forward: the plan is written once into the list's workspace (lb_list_init) and every
    forward() is three launches (lb_list_forward).  The tensors must outlive the object and keep their
    storage (the plan holds their addresses)."""

    def __init__(self, items, stream=None):
        torch = _torch()
        self.items = items
        self.descs, self.ys = make_descs(items)
        self.n = len(items)
        lib = load_library()
        need = lb_list_workspace_bytes(self.descs, self.n)
        if need == 0:
            raise LittleBitError(LB_ERR_SHAPE, "lb_list_workspace_bytes (list out of scope or invalid)")
        dev = self.ys[0].device if self.ys else "cuda"
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        st = lib.lb_list_init(self.descs, self.n, _dev_ptr(self.workspace, "workspace"), need, _stream(stream))
        _check(st, "lb_list_init")

    def forward(self, stream=None):
        st = load_library().lb_list_forward(self.descs, self.n, _dev_ptr(self.workspace, "workspace"),
                                            self.workspace.numel(), _stream(stream))
        _check(st, "lb_list_forward")
        return self.ys


def lb_latent_workspace_bytes(T: int, d_in: int, r: int) -> int:
    return int(load_library().lb_latent_workspace_bytes(T, d_in, r))


def lb_from_latent_workspace_bytes(T: int, r: int) -> int:
    return int(load_library().lb_from_latent_workspace_bytes(T, r))


def _scratch(n: int, device):
    torch = _torch()
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def lb_linear_latent(x, paths: Sequence[LittleBitPath], r: int, w=None, latent_dtype=None, workspace=None,
                     stream=None):
    """The latent cache entries w [T, 2, r] of x [T, d_in] (only V, g, l of the paths are read; latent_dtype
    defaults to float32); returns w."""
    torch = _torch()
    lib = load_library()
    T, d_in = x.shape
    arr, sc = _paths_struct(paths)
    if w is None:
        w = torch.empty((T, 2, r), dtype=latent_dtype or torch.float32, device=x.device)
    if workspace is None:
        workspace = _scratch(lb_latent_workspace_bytes(T, d_in, r), x.device)
    st = lib.lb_linear_latent(_dev_ptr(x, "x"), _dtype_code(x), T, d_in, r, arr, sc, _dev_ptr(w, "w"),
                              _dtype_code(w), _dev_ptr(workspace, "workspace"),
                              workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "lb_linear_latent")
    return w


def lb_linear_from_latent(w, paths: Sequence[LittleBitPath], y=None, out_dtype=None, workspace=None, stream=None):
    """y [T, d_out] of the layer from cached latents w [T, 2, r] (only U, h of the paths are read; out_dtype
    defaults to w's dtype); returns y."""
    torch = _torch()
    lib = load_library()
    T, two, r = w.shape
    if two != 2:
        raise ValueError("w must be [T, 2, r]")
    d_out = paths[0].h.shape[0]
    arr, sc = _paths_struct(paths)
    if y is None:
        y = torch.empty((T, d_out), dtype=out_dtype or w.dtype, device=w.device)
    if workspace is None:
        workspace = _scratch(lb_from_latent_workspace_bytes(T, r), w.device)
    st = lib.lb_linear_from_latent(_dev_ptr(w, "w"), _dtype_code(w), T, d_out, r, arr, sc, _dev_ptr(y, "y"),
                                   _dtype_code(y), _dev_ptr(workspace, "workspace"),
                                   workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "lb_linear_from_latent")
    return y


def lb_backward_workspace_bytes(T: int, d_in: int, d_out: int, r: int) -> int:
    return int(load_library().lb_backward_workspace_bytes(T, d_in, d_out, r))


@dataclass
class LittleBitPathTrain:
    """One path's fp32 latent factors, their signs packed in the backward's orientation (Ut: U packed
    with LB_ROLE_V, Vt: V packed with LB_ROLE_U) and, after lb_linear_backward, the gradients."""
    U_latent: object
    V_latent: object
    Ut: object = None
    Vt: object = None
    dU: object = None
    dV: object = None
    dh: object = None
    dg: object = None
    dl: object = None


def lb_linear_backward(x, dy, paths: Sequence[LittleBitPath], train: Sequence[LittleBitPathTrain],
                       kappa: float = 100.0, dx=None, need_dx: bool = True, workspace=None, stream=None):
    """Gradients of one layer for x [T, d_in] and dy [T, d_out]: fills (allocating when None) Ut, Vt (packed
    from the latents), dU, dV, dh, dg, dl of each train entry; returns dx (None when need_dx is False)."""
    torch = _torch()
    lib = load_library()
    T, d_in = x.shape
    d_out = dy.shape[1]
    r = train[0].U_latent.shape[1]
    arr, sc = _paths_struct(paths)
    tarr = (lb_path_train * 2)()
    dev = x.device
    for i, q in enumerate(train):
        if q.Ut is None:
            q.Ut = lb_pack_signs(q.U_latent, LB_ROLE_V, stream=stream)
        if q.Vt is None:
            q.Vt = lb_pack_signs(q.V_latent, LB_ROLE_U, stream=stream)
        for name, shape in (("dU", (d_out, r)), ("dV", (d_in, r)), ("dh", (d_out,)), ("dg", (d_in,)), ("dl", (r,))):
            if getattr(q, name) is None:
                setattr(q, name, torch.empty(shape, dtype=torch.float32, device=dev))
        tarr[i] = lb_path_train(*[_dev_ptr(getattr(q, f), f) for f in ("U_latent", "V_latent", "Ut", "Vt", "dU",
                                                                         "dV", "dh", "dg", "dl")])
    if need_dx and dx is None:
        dx = torch.empty((T, d_in), dtype=x.dtype, device=dev)
    if workspace is None:
        workspace = _scratch(lb_backward_workspace_bytes(T, d_in, d_out, r), dev)
    st = lib.lb_linear_backward(_dev_ptr(x, "x"), _dev_ptr(dy, "dy"), _dtype_code(x), T, d_in, d_out, r, arr, sc,
                                tarr, float(kappa), _dev_ptr(dx, "dx") if need_dx else 0,
                                _dev_ptr(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                _stream(stream))
    _check(st, "lb_linear_backward")
    return dx if need_dx else None


# ----------------------------------------------------------------------------
# paged latent cache and attention
# ----------------------------------------------------------------------------
# The C structures as packed bytes (native sizes and alignment).
_PACK_CACHE = struct.Struct("@PiqqqqPqqPP").pack
_PACK_PATHS = struct.Struct("@10P").pack
_PACK_ATTN = struct.Struct("@PPPPi14qPPqif").pack
_PACK_GRADS = struct.Struct("@4P4q").pack


def _current_device() -> int:
    return _torch()._C._cuda_getDevice()


def _on_gpu(*tensors):
    """Every tensor on the current GPU (a launch goes to the current device's stream)."""
    cur = None
    for t in tensors:
        if t is None:
            continue
        d = t.get_device()
        if d < 0:
            raise ValueError(f"expected a GPU tensor, got one on {t.device}")
        if cur is None:
            cur = _current_device()
        if d != cur:
            raise ValueError(f"every tensor must be on the current GPU (cuda:{cur}), got one on {t.device}")


_NO_CONTEXT = contextlib.nullcontext()


def _memory_of(stream):
    """Where a call's new tensors are allocated: with the stream that it runs on, so that their memory is not
    handed on while that stream still uses it."""
    return _NO_CONTEXT if stream is None else _torch().cuda.stream(stream)


def _need(t, shape, dtype, name: str):
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _whole(t, shape, dtype, name: str) -> int:
    """The address of a contiguous tensor of this shape and type."""
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        _need(t, shape, dtype, name)
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _default_scale(width: int) -> float:
    return max(width, 1) ** -0.5


def _freqs(t, d: int) -> int:
    return 0 if t is None else _whole(t, (d // 2,), _T.float32, "freqs")


def _rows(t, name: str):
    """(address, strides) of a tensor whose last dimension is contiguous."""
    st = t.stride()
    if st[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return t.data_ptr(), st


def lb_rotate(x, positions, freqs, inverse: bool = False, out=None, stream=None):
    """x [T, H, d] turned by positions [T] (int32) and freqs [d / 2] (fp32 radians a position), pairs
    (i, i + d / 2); inverse=True turns back, which is also the gradient's map.  x and out may be strided
    (last dimension contiguous), out may be x; returns out."""
    torch = _torch()
    shape = x.shape
    T, H, d = shape
    if out is None:
        with _memory_of(stream):
            out = x.new_empty(shape)
    else:
        _need(out, shape, x.dtype, "out")
    _on_gpu(x, positions, freqs, out)
    px, sx = _rows(x, "x")
    py, sy = _rows(out, "out")
    st = load_library().lb_rotate(px, _dtype_code(x), T, H, d, sx[0], sx[1], _whole(positions, (T,), torch.int32, "positions"),
                                  _whole(freqs, (d // 2,), torch.float32, "freqs"), 1 if inverse else 0, py, sy[0], sy[1],
                                  _stream(stream))
    if st:
        _check(st, "lb_rotate")
    return out


def lb_latent_row(r: int, d_rope: int) -> int:
    """Elements of a paged latent cache's row: [w (2 r) | rotary key (d_rope) | zeros], a multiple of 32."""
    return int(load_library().lb_latent_row(r, d_rope))


@dataclass
class LatentCache:
    """A paged latent cache: data [n_pages, page_size, lb_latent_row(r, d_rope)] in fp32, fp16 or bf16."""
    data: object
    r: int
    d_rope: int = 0

    @classmethod
    def empty(cls, n_pages: int, page_size: int, r: int, d_rope: int = 0, dtype=None, device="cuda"):
        torch = _torch()
        return cls(torch.empty((n_pages, page_size, lb_latent_row(r, d_rope)), dtype=dtype or torch.bfloat16,
                               device=device), r, d_rope)

    def _packed(self, table, lens, cu) -> bytes:
        d = self.data
        row = (2 * self.r + self.d_rope + 31) // 32 * 32
        if d.dim() != 3 or d.shape[2] != row or not d.is_contiguous():
            raise ValueError("a cache's data must be contiguous [n_pages, page_size, lb_latent_row(r, d_rope)]")
        if table.dim() != 2:
            raise ValueError("table must be [sequences, pages]")
        B, M = table.shape
        i32 = _T.int32
        return _PACK_CACHE(d.data_ptr(), _dtype_code(d), d.shape[0], d.shape[1], self.r, self.d_rope,
                           _whole(table, (B, M), i32, "table"), B, M, _whole(lens, (B,), i32, "lens"),
                           _whole(cu, (B + 1,), i32, "cu"))


def lb_latent_append(cache: LatentCache, w, k_rope, freqs, table, lens, cu, stream=None):
    """Append latents w [T, 2, r] and rotary keys k_rope [T, d_rope] (None if d_rope is 0; turned by their
    positions with freqs, or stored as they are if it is None): sequence b's tokens are rows cu[b] ..
    cu[b + 1] - 1 and become its last positions below lens[b], on the pages table[b] names."""
    _torch()
    d = cache.d_rope
    _on_gpu(cache.data, w, k_rope if d else None, freqs, table, lens, cu)
    T = w.shape[0]
    pw = _whole(w, (T, 2, cache.r), w.dtype, "w")
    kp, kt = 0, 0
    if d:
        _need(k_rope, (T, d), w.dtype, "k_rope")
        kp, (kt, _) = _rows(k_rope, "k_rope")
    st = load_library().lb_latent_append(cache._packed(table, lens, cu), pw, kp, kt, _dtype_code(w), T,
                                         _freqs(freqs, d), _stream(stream))
    if st:
        _check(st, "lb_latent_append")


def lb_latent_attention_workspace_bytes(T: int, n_seq: int, H: int, r: int, d_rope: int) -> int:
    return int(load_library().lb_latent_attention_workspace_bytes(T, n_seq, H, r, d_rope))


def lb_latent_attention(q, cache: LatentCache, paths: Sequence[LittleBitPath], Hk: int, d_v: int, table, lens, cu,
                        freqs=None, scale=None, out=None, workspace=None, stream=None):
    """Attention of new query tokens q [T, H, d_nope + d_rope] over the paged latent cache, the up-projection
    absorbed; the tokens are already appended (table, lens and cu as for lb_latent_append).  paths: U and h of
    the fused layer, d_out = Hk (d_nope + d_v), keys first.  q's last d_rope values are turned by their
    positions with freqs (None: taken as they are).  scale defaults to (d_nope + d_rope) ** -0.5; returns
    out [T, H, d_v]."""
    _torch()
    if len(paths) != 2:
        raise ValueError("exactly two paths (primary, residual) are required")
    if q.dim() != 3:
        raise ValueError("q must be [T, H, d_nope + d_rope]")
    a, b = paths
    _on_gpu(q, cache.data, freqs, table, lens, cu, out, workspace, a.U, a.h, b.U, b.h)
    T, H, dq = q.shape
    r, dr = cache.r, cache.d_rope
    dn = dq - dr
    if dn < 0:
        raise ValueError("q's heads are narrower than the rotary key")
    n_out = Hk * (dn + d_v)
    nb, w = r // 32, r % 32
    need = n_out * (4 * nb + (0 if w == 0 else 2 if w <= 16 else 4))
    for U in (a.U, b.U):
        if U.numel() * U.element_size() < need or not U.is_contiguous():
            raise ValueError(f"U must hold the packed signs of d_out = Hk (d_nope + d_v) = {n_out} rows at r = {r}")
    sdt = a.h.dtype
    arr = _PACK_PATHS(a.U.data_ptr(), 0, _whole(a.h, (n_out,), sdt, "h"), 0, 0,
                      b.U.data_ptr(), 0, _whole(b.h, (n_out,), sdt, "h"), 0, 0)
    with _memory_of(stream):
        if out is None:
            out = q.new_empty((T, H, d_v))
        if workspace is None:
            workspace = _scratch(lb_latent_attention_workspace_bytes(T, lens.shape[0], H, r, dr), q.device)
    pq, sq = _rows(q, "q")
    st = load_library().lb_latent_attention(
        pq, _dtype_code(q), T, H, Hk, dn, d_v, sq[0], sq[1], arr, _dtype_code(a.h), cache._packed(table, lens, cu),
        _freqs(freqs, dr), _default_scale(dq) if scale is None else scale, _whole(out, (T, H, d_v), q.dtype, "out"),
        _dev_ptr(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream(stream))
    if st:
        _check(st, "lb_latent_attention")
    return out


def _packed_attention(q, k, v, k_rope, cu_q, cu_k, causal, scale):
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k and v must be [tokens, heads, width]")
    dt = q.dtype
    Tq, H, dq = q.shape
    Tk, Hk, dn = k.shape
    d_v = v.shape[2]
    dr, pr, kr_t = 0, 0, 0
    if k_rope is not None:
        dr = k_rope.shape[-1]
        _need(k_rope, (Tk, dr), dt, "k_rope")
        pr, (kr_t, _) = _rows(k_rope, "k_rope")
    if dn + dr != dq:
        raise ValueError("q's heads must be as wide as k's and k_rope's together")
    _need(k, (Tk, Hk, dn), dt, "k")
    _need(v, (Tk, Hk, d_v), dt, "v")
    pq, sq = _rows(q, "q")
    pk, sk = _rows(k, "k")
    pv, sv = _rows(v, "v")
    if (cu_q is None) != (cu_k is None):
        raise ValueError("cu_q and cu_k are given together")
    n, pcq, pck = 0, 0, 0
    if cu_q is not None:
        if cu_q.dim() != 1 or cu_q.shape[0] < 1:
            raise ValueError("cu_q must hold the sequences' prefix sums")
        n = cu_q.shape[0] - 1
        pcq = _whole(cu_q, (n + 1,), _T.int32, "cu_q")
        pck = _whole(cu_k, (n + 1,), _T.int32, "cu_k")
    return _PACK_ATTN(pq, pk, pv, pr, _dtype_code(q), Tq, Tk, H, Hk, dn, dr, d_v, sq[0], sq[1], sk[0], sk[1], sv[0], sv[1],
                      kr_t, pcq, pck, n, 1 if causal else 0, _default_scale(dq) if scale is None else scale), (
                          Tq, Tk, H, Hk, dn, dr, d_v)


def lb_attention_forward(q, k, v, k_rope=None, cu_q=None, cu_k=None, causal: bool = True, scale=None, o=None, lse=None,
                         stream=None):
    """Attention over expanded keys and values: q [Tq, H, d_nope + d_rope], k [Tk, Hk, d_nope], v [Tk, Hk, d_v],
    k_rope [Tk, d_rope] (one rotary key a token for all heads, or None), any strides with a contiguous last
    dimension; cu_q, cu_k int32 prefix sums of packed sequences (None: one sequence).  scale defaults to
    (d_nope + d_rope) ** -0.5.  Returns (o [Tq, H, d_v], lse [Tq, H] fp32)."""
    torch = _torch()
    _on_gpu(q, k, v, k_rope, cu_q, cu_k, o, lse)
    a, (Tq, _, H, _, _, _, d_v) = _packed_attention(q, k, v, k_rope, cu_q, cu_k, causal, scale)
    with _memory_of(stream):
        if o is None:
            o = q.new_empty((Tq, H, d_v))
        if lse is None:
            lse = q.new_empty((Tq, H), dtype=torch.float32)
    st = load_library().lb_attention_forward(a, _whole(o, (Tq, H, d_v), q.dtype, "o"),
                                             _whole(lse, (Tq, H), torch.float32, "lse"), _stream(stream))
    if st:
        _check(st, "lb_attention_forward")
    return o, lse


def lb_attention_backward_workspace_bytes(Tq: int, Tk: int, H: int, Hk: int, d_rope: int) -> int:
    return int(load_library().lb_attention_backward_workspace_bytes(Tq, Tk, H, Hk, d_rope))


def lb_attention_backward(q, k, v, k_rope, o, lse, d_o, cu_q=None, cu_k=None, causal: bool = True, scale=None, dq=None,
                          dk=None, dv=None, dk_rope=None, workspace=None, stream=None):
    """Gradients of lb_attention_forward for d_o [Tq, H, d_v] (contiguous); dk and dv may be strided views (the
    two parts of the fused layer's dy).  Returns (dq, dk, dv, dk_rope) (dk_rope None without a rotary key)."""
    torch = _torch()
    _on_gpu(q, k, v, k_rope, o, lse, d_o, cu_q, cu_k, dq, dk, dv, dk_rope, workspace)
    a, (Tq, Tk, H, Hk, dn, dr, d_v) = _packed_attention(q, k, v, k_rope, cu_q, cu_k, causal, scale)
    dt = q.dtype
    with _memory_of(stream):
        dq = q.new_empty((Tq, H, dn + dr)) if dq is None else dq
        dk = q.new_empty((Tk, Hk, dn)) if dk is None else dk
        dv = q.new_empty((Tk, Hk, d_v)) if dv is None else dv
        if dr and dk_rope is None:
            dk_rope = q.new_empty((Tk, dr))
        if workspace is None:
            workspace = _scratch(lb_attention_backward_workspace_bytes(Tq, Tk, H, Hk, dr), q.device)
    _need(dk, (Tk, Hk, dn), dt, "dk")
    _need(dv, (Tk, Hk, d_v), dt, "dv")
    pr = _whole(dk_rope, (Tk, dr), dt, "dk_rope") if dr else 0
    pk, sk = _rows(dk, "dk")
    pv, sv = _rows(dv, "dv")
    g = _PACK_GRADS(_whole(dq, (Tq, H, dn + dr), dt, "dq"), pk, pv, pr, sk[0], sk[1], sv[0], sv[1])
    st = load_library().lb_attention_backward(
        a, _whole(o, (Tq, H, d_v), dt, "o"), _whole(lse, (Tq, H), torch.float32, "lse"),
        _whole(d_o, (Tq, H, d_v), dt, "d_o"), g, _dev_ptr(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(stream))
    if st:
        _check(st, "lb_attention_backward")
    return dq, dk, dv, dk_rope if dr else None


def lb_dense_reference_weight(paths: Sequence[LittleBitPath], d_in: int, d_out: int, r: int, W=None, stream=None):
    """Dense fp32 W_hat [d_out, d_in] from the packed buffers (checking path)."""
    torch = _torch()
    lib = load_library()
    arr, sc = _paths_struct(paths)
    if W is None:
        W = torch.empty((d_out, d_in), dtype=torch.float32, device=paths[0].h.device)
    st = lib.lb_dense_reference_weight(arr, sc, d_in, d_out, r, _dev_ptr(W, "W"), _stream(stream))
    _check(st, "lb_dense_reference_weight")
    return W


def lb_dual_svid_workspace_bytes(d_out: int, d_in: int, r: int, oversample: int) -> int:
    return int(load_library().lb_dual_svid_workspace_bytes(d_out, d_in, r, oversample))


def svid_defaults(r: int, d_out: int, d_in: int):
    """(oversample, iters) used when lb_dual_svid is not given them: a block of about 1.5 r vectors
    (at least r + 16) and 12 rounds of subspace iteration."""
    return max(16, r // 2), 12


def lb_dual_svid(W, r: int, oversample=None, iters=None, seed: int = 0, residual: bool = False, workspace=None,
                 stream=None) -> dict:
    """Dual-SVID of a dense weight W [d_out, d_in] (device, f32 / f16 / bf16) at rank r.  Returns
    {"U": [U'_0, U'_1], "V": [...], "h": [...], "g": [...], "l": [...], "sigma": [...]} (fp32 device
    tensors; U' [d_out, r], V' [d_in, r]) and, with residual=True, "W_res" = W - W_hat_pri,0 (fp32)."""
    torch = _torch()
    lib = load_library()
    d_out, d_in = W.shape
    ov, it = svid_defaults(r, d_out, d_in)
    oversample = ov if oversample is None else oversample
    iters = it if iters is None else iters
    dev = W.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = {"U": [torch.empty((d_out, r), **f32) for _ in range(2)],
           "V": [torch.empty((d_in, r), **f32) for _ in range(2)],
           "h": [torch.empty(d_out, **f32) for _ in range(2)], "g": [torch.empty(d_in, **f32) for _ in range(2)],
           "l": [torch.empty(r, **f32) for _ in range(2)], "sigma": [torch.empty(r, **f32) for _ in range(2)]}
    arr = (lb_svid_out * 2)()
    for p in range(2):
        arr[p] = lb_svid_out(*(_dev_ptr(out[k][p], k) for k in ("U", "V", "h", "g", "l", "sigma")))
    W_res = torch.empty((d_out, d_in), **f32) if residual else None
    need = lb_dual_svid_workspace_bytes(d_out, d_in, r, oversample)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    st = lib.lb_dual_svid(_dev_ptr(W, "W"), _dtype_code(W), d_out, d_in, r, oversample, iters,
                          ctypes.c_uint64(seed), arr, _dev_ptr(W_res, "W_res"), _dev_ptr(workspace, "workspace"),
                          workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "lb_dual_svid")
    if residual:
        out["W_res"] = W_res
    return out


def littlebit_from_dense(W, r: int, scale_dtype=None, **kw):
    """A LittleBit linear initialised from the dense W [d_out, d_in] by Dual-SVID: the two paths with
    packed signs (LB layout v1) and scales in scale_dtype (default fp16), ready for lb_linear_forward."""
    torch = _torch()
    sd = torch.float16 if scale_dtype is None else scale_dtype
    s = lb_dual_svid(W, r, **kw)
    paths = []
    for p in range(2):
        paths.append(LittleBitPath(U=lb_pack_signs(s["U"][p], LB_ROLE_U), V=lb_pack_signs(s["V"][p], LB_ROLE_V),
                                   h=s["h"][p].to(sd), g=s["g"][p].to(sd), l=s["l"][p].to(sd)))
    return paths


__all__ = [
    "LB_OK", "LB_ERR_NULL", "LB_ERR_SHAPE", "LB_ERR_DTYPE", "LB_ERR_ALIGN", "LB_ERR_WORKSPACE", "LB_ERR_HIP",
    "LB_ERR_ARG", "LB_F32", "LB_F16", "LB_BF16", "LB_ROLE_U", "LB_ROLE_V", "LB_KERNEL_AUTO", "LB_KERNEL_DECODE",
    "LB_KERNEL_PREFILL", "LB_KERNEL_DECODE_MFMA", "LittleBitError", "LittleBitPath", "lb_path", "load_library", "lb_status_str",
    "lb_packed_bytes", "lb_bits_per_weight", "lb_rank_for_bpw", "lb_forward_workspace_bytes",
    "lb_decode_max_tokens", "lb_pack_signs", "lb_workspace_init", "lb_workspace_status", "alloc_workspace", "lb_linear_forward",
    "lb_dense_reference_weight", "lb_linear_forward_noalloc", "lb_linear_desc", "make_descs", "lb_forward_many_workspace_bytes",
    "lb_linear_forward_many", "lb_list_workspace_bytes", "LittleBitList", "lb_latent_workspace_bytes", "lb_from_latent_workspace_bytes", "lb_linear_latent",
    "lb_linear_from_latent", "lb_path_train", "LittleBitPathTrain", "lb_backward_workspace_bytes",
    "lb_linear_backward", "lb_svid_out", "lb_dual_svid_workspace_bytes", "svid_defaults", "lb_dual_svid",
    "littlebit_from_dense", "lb_rotate", "lb_latent_row", "LatentCache", "lb_latent_append",
    "lb_latent_attention_workspace_bytes", "lb_latent_attention", "lb_attention_forward",
    "lb_attention_backward_workspace_bytes", "lb_attention_backward",
]
