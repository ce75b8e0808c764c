"""Binding of ``libnmg.so`` (declared in ``include/nmg.h``): ctypes, and a compiled
module for the calls of every layer and token (the attention operators, the 8-bit
cache's, the residual norm), which are as short as their marshalling.

Argument marshalling only: torch allocates the outputs on the input's device
and supplies the current HIP stream; every step of the computation runs in the
library's HIP kernels.  There is no fallback: if the library is missing or a
call fails, the binding raises.

Paper: STen (arXiv 2304.07613), Section 5 (n:m:g layout), 5.1 (sparse x dense
product), 5.2 (magnitude converter and conversion back to dense).
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import re
import types

import torch

from . import build as _build

LIB_PATH = _build.LIB_PATH

F32, F16 = 0, 1
_DTYPE_CODE = {torch.float32: F32, torch.float16: F16}
KERNELS = {"auto": 0, "valu": 1, "mfma": 2, "mfma_general": 3, "mfma_scalar": 4, "mfma_f16": 5,
           "mfma_direct": 6, "smfmac_f16": 7, "valu_staged": 8, "mfma_wide": 9, "mfma_split": 10,
           "mfma_expand": 11, "sparse": 12}
_KERNEL_NAME = {v: k for k, v in KERNELS.items()}
EPILOGUES = {"none": 0, "gelu": 1, "add": 2}
ROTARY_PAIRS = {"half": 0, "interleaved": 1}
CACHE_FORMATS = {"e4m3": (0, torch.float8_e4m3fn), "int8": (1, torch.int8)}
NORMS = {"none": 0, "rms": 1, "layer": 2}
ROTARY_SCALING = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}

OK, ERR_NULL, ERR_PARAM, ERR_SHAPE, ERR_DTYPE, ERR_ALIGN, ERR_LAUNCH, ERR_UNSUPPORTED, ERR_CAPACITY = \
    range(9)


class NmgError(RuntimeError):
    """A libnmg call returned a status other than NMG_OK."""

    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_str(status)} (status {status})")
        self.status = status


class _Layout(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int32), ("K", ctypes.c_int32), ("n", ctypes.c_int32),
                ("m", ctypes.c_int32), ("g", ctypes.c_int32), ("C", ctypes.c_int32),
                ("dtype", ctypes.c_int)]


class _Rotary(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("pairs", ctypes.c_int), ("length", ctypes.c_int64),
                ("table", ctypes.c_void_p), ("positions", ctypes.c_void_p)]


class _Heads(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int)]


class _Sequences(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("q_offsets", ctypes.c_void_p),
                ("kv_begin", ctypes.c_void_p), ("kv_end", ctypes.c_void_p)]


class _Cache(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int), ("format", ctypes.c_int),
                ("block", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("sequences", ctypes.c_int32), ("row", ctypes.c_int32), ("room", ctypes.c_int32),
                ("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("k_open", ctypes.c_void_p), ("v_open", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("references", ctypes.c_void_p)]


class _Norm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("eps", ctypes.c_float)]


class _PLayout(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int32), ("K", ctypes.c_int32), ("n", ctypes.c_int32),
                ("m", ctypes.c_int32), ("g", ctypes.c_int32), ("P", ctypes.c_int32),
                ("S", ctypes.c_int32), ("B", ctypes.c_int32), ("dtype", ctypes.c_int)]


_lib = None


def header_functions() -> list:
    """Names of the functions ``include/nmg.h`` declares."""
    with open(_build.HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"^[A-Za-z_][\w \t\*]*?\b(nmg_\w+)\s*\(", text, re.M)))


def lib():
    """The loaded library; raises if it has not been built."""
    return _lib if _lib is not None else _load()


def _load():
    global _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, lp = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(_Layout)
    pp = ctypes.POINTER(_PLayout)
    rp, hp, sp = (ctypes.POINTER(t) for t in (_Rotary, _Heads, _Sequences))
    cp, np = ctypes.POINTER(_Cache), ctypes.POINTER(_Norm)
    ip = ctypes.POINTER(i32)
    f32, f64 = ctypes.c_float, ctypes.c_double
    sig = {
        "nmg_layout_init": ([lp, i32, i32, i32, i32, i32, ctypes.c_int], ctypes.c_int),
        "nmg_values_numel": ([lp], i64),
        "nmg_indices_numel": ([lp], i64),
        "nmg_compress": ([lp, vp, i64, vp, vp, vp], ctypes.c_int),
        "nmg_repack": ([lp, vp, i64, vp, vp, vp], ctypes.c_int),
        "nmg_spmm": ([lp, vp, vp, vp, i64, i64, vp, i64, vp], ctypes.c_int),
        "nmg_spmm_with": ([lp, ctypes.c_int, vp, vp, vp, i64, i64, vp, i64, vp], ctypes.c_int),
        "nmg_spmm_epilogue": ([lp, ctypes.c_int, ctypes.c_int, vp, vp, vp, i64, i64, vp, i64, vp,
                               i64, vp], ctypes.c_int),
        "nmg_spmm_epilogue_noalloc": ([lp, ctypes.c_int, ctypes.c_int, vp, vp, vp, i64, i64, vp,
                                       i64, vp, i64, vp], ctypes.c_int),
        "nmg_spmm_epilogue_ws": ([lp, ctypes.c_int, ctypes.c_int, vp, vp, vp, i64, i64, vp, i64, vp,
                                  i64, vp, i64, vp], ctypes.c_int),
        "nmg_spmm_workspace_bytes": ([lp, ctypes.c_int, i64], i64),
        "nmg_spmm_plan": ([lp, ctypes.c_int, vp, vp, vp, i64, i64, ctypes.POINTER(i64)],
                          ctypes.c_int),
        "nmg_p_spmm_ws": ([pp, ctypes.c_int, vp, vp, vp, i64, i64, vp, i64, vp, i64, vp],
                          ctypes.c_int),
        "nmg_p_spmm_workspace_bytes": ([pp, ctypes.c_int, i64], i64),
        "nmg_spmm_auto_kernel": ([lp, i64], ctypes.c_int),
        "nmg_densify": ([lp, vp, vp, vp, i64, vp], ctypes.c_int),
        "nmg_gelu": ([ctypes.c_int, vp, vp, i64, vp], ctypes.c_int),
        "nmg_add": ([ctypes.c_int, vp, vp, vp, i64, vp], ctypes.c_int),
        "nmg_p_layout_init": ([pp, i32, i32, i32, i32, i32, ctypes.c_int], ctypes.c_int),
        "nmg_p_compress": ([pp, vp, i64, vp, vp, vp], ctypes.c_int),
        "nmg_p_spmm": ([pp, vp, vp, vp, i64, i64, vp, i64, vp], ctypes.c_int),
        "nmg_p_spmm_with": ([pp, ctypes.c_int, vp, vp, vp, i64, i64, vp, i64, vp], ctypes.c_int),
        "nmg_p_refine": ([pp, vp, i64, vp, vp, vp], ctypes.c_int),
        "nmg_p_densify": ([pp, vp, vp, vp, i64, vp], ctypes.c_int),
        "nmg_x16_prepared_bytes": ([lp], i64),
        "nmg_x16_prepare": ([lp, vp, vp, vp, vp], ctypes.c_int),
        "nmg_spmm_x16": ([lp, vp, vp, i64, i64, vp, i64, vp], ctypes.c_int),
        "nmg_spmm_x16_epilogue": ([lp, vp, ctypes.c_int, vp, i64, i64, vp, i64, vp, i64, vp],
                                  ctypes.c_int),
        "nmg_rotary_table": ([i32, i64, f64, ctypes.c_int, f64, f64, f64, f64, f64, vp, vp],
                             ctypes.c_int),
        "nmg_rotary": ([ctypes.c_int, i32, i32, rp, vp, i64, i64, vp, i64, vp], ctypes.c_int),
        "nmg_qk_norm_rotary": ([ctypes.c_int, i32, i32, i32, rp, vp, vp, f32, vp, i64, vp, i64, i64,
                                vp, i64, vp, i64, vp], ctypes.c_int),
        "nmg_attention": ([hp, sp, vp, i64, i64, vp, i64, vp, i64, i64, vp, f32, vp, i64, vp, i64,
                           vp], ctypes.c_int),
        "nmg_tree_attention": ([hp, sp, vp, i64, i64, vp, i64, vp, i64, i64, vp, i64, i64, f32, vp,
                                i64, vp, i64, vp], ctypes.c_int),
        "nmg_attention_workspace_bytes": ([hp, i32, i64, i64], i64),
        "nmg_cache_append": ([cp, i32, vp, vp, vp, i64, vp, i64, i64, vp], ctypes.c_int),
        "nmg_cache_attention": ([cp, i32, i32, vp, vp, vp, i64, i64, vp, i64, i64, i64, f32, vp, i64,
                                 vp, i64, vp], ctypes.c_int),
        "nmg_cache_attention_workspace_bytes": ([cp, i32, i64, i64], i64),
        "nmg_cache_commit": ([cp, vp, vp, vp, i64, vp, vp], ctypes.c_int),
        "nmg_cache_reserve": ([cp, vp, vp, vp, vp], ctypes.c_int),
        "nmg_cache_fork": ([cp, vp, i32, ip, ip, vp], ctypes.c_int),
        "nmg_cache_free": ([cp, vp, i32, ip, vp], ctypes.c_int),
        "nmg_cache_compact": ([cp, vp, vp, vp, vp, i64, vp], ctypes.c_int),
        "nmg_cache_compact_workspace_bytes": ([cp], i64),
        "nmg_residual_norm": ([ctypes.c_int, i64, i64, vp, i64, np, vp, i64, f32, vp, i64, np, vp, i64,
                               vp, i64, vp], ctypes.c_int),
        "nmg_status_str": ([ctypes.c_int], ctypes.c_char_p),
        "nmg_version": ([], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    _lib = L
    return L


_calls = None


def _load_calls():
    """The compiled marshalling of the calls of every layer, bound to the library."""
    global _calls
    L = lib()
    path = _build.calls_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run __graft_entry__.build()")
    name = __package__ + "._calls"
    spec = importlib.util.spec_from_file_location(name, path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)

    names = ("nmg_rotary", "nmg_qk_norm_rotary", "nmg_attention", "nmg_tree_attention",
             "nmg_attention_workspace_bytes")
    module.bind({n: ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in names}, _check,
                torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
    more = ("nmg_cache_append", "nmg_cache_attention", "nmg_cache_attention_workspace_bytes",
            "nmg_cache_commit", "nmg_residual_norm")
    module.bind_more({n: ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in more})
    _calls = module
    return module


def status_str(status: int) -> str:
    return lib().nmg_status_str(status).decode()


def version() -> str:
    return lib().nmg_version().decode()


def _check(status: int, what: str):
    if status != OK:
        raise NmgError(status, what)


class Layout:
    """Shape of one n:m:g weight (``nmg_layout``)."""

    def __init__(self, M: int, K: int, n: int, m: int, g: int, dtype=torch.float32):
        if dtype not in _DTYPE_CODE:
            raise TypeError(f"unsupported dtype {dtype}")
        self.c = _Layout()
        _check(lib().nmg_layout_init(ctypes.byref(self.c), M, K, n, m, g, _DTYPE_CODE[dtype]),
               "nmg_layout_init")
        self.dtype = dtype
        self._derive()

    def _derive(self):
        c = self.c
        self.M, self.K, self.n, self.m, self.g, self.C = c.M, c.K, c.n, c.m, c.g, c.C
        self.values_shape = (self.M, self.C * self.n)
        self.indices_shape = (self.M // self.g, self.C * self.n)
        self._ws = (None, 0)     # what sized the last product's workspace, and its bytes

    def __setstate__(self, state):     # (also states of c and dtype alone)
        self.__dict__.update(state)
        self._derive()

    def __repr__(self):
        return (f"Layout(M={self.M}, K={self.K}, n={self.n}, m={self.m}, g={self.g}, "
                f"C={self.C}, dtype={self.dtype})")


def _stream(t: torch.Tensor) -> int:
    """The raw handle of the current stream of t's device."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _need_cuda(*ts):
    """Every tensor on the current GPU: the library launches on the current
    HIP device, on that device's current stream."""
    cur = -1
    for t in ts:
        dev = t.get_device()
        if dev < 0 or not t.is_cuda:
            raise ValueError("libnmg works on GPU tensors only")
        if cur < 0:
            cur = torch._C._cuda_getDevice()
        if dev != cur:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{cur} "
                             "(select it with torch.cuda.device)")


def _rows(t: torch.Tensor, name: str) -> int:
    """Leading dimension of a 2-D row-major tensor (unit stride along rows)."""
    st = t.stride()
    if len(st) != 2 or st[1] != 1:
        raise ValueError(f"{name} must be a 2-D tensor with unit column stride")
    return st[0]


def _packed_ok(layout, values, indices):
    if values.shape != layout.values_shape or not values.is_contiguous():
        raise ValueError(f"values must be contiguous {layout.values_shape}")
    if indices.shape != layout.indices_shape or not indices.is_contiguous():
        raise ValueError(f"indices must be contiguous {layout.indices_shape}")


def _workspace(nbytes: int, like: torch.Tensor):
    """Scratch memory of one call from torch's allocator: (tensor, pointer,
    bytes).  Freed after the call returns; the allocator hands it out again in
    stream order on the current stream only.  None when the memory is not there:
    the library then takes what it takes without a workspace."""
    if nbytes <= 0:
        return None, None, 0
    try:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    except torch.OutOfMemoryError:
        return None, None, 0
    return ws, ws.data_ptr(), nbytes


def _workspace_bytes(layout, code: int, vp: int, ip: int, xp: int, ldx: int, N: int) -> int:
    """The workspace of nmg_spmm_plan: a function of the layout, kernel, sizes and
    the pointers' alignment to 16 bytes."""
    at = (code, N, ldx, vp & 15, ip & 15, xp & 15)
    key, nbytes = layout._ws
    if key != at:
        out = ctypes.c_int64(0)
        lib().nmg_spmm_plan(layout.c, code, vp, ip, xp, ldx, N, ctypes.byref(out))
        nbytes = out.value
        layout._ws = (at, nbytes)
    return nbytes


def compress_into(layout: Layout, W: torch.Tensor, values: torch.Tensor, indices: torch.Tensor):
    """``nmg_compress`` into caller-allocated ``values`` / ``indices``."""
    _need_cuda(W, values, indices)
    if W.dtype != layout.dtype or values.dtype != layout.dtype or indices.dtype != torch.uint8:
        raise TypeError("dtype mismatch")
    if W.shape != (layout.M, layout.K):
        raise ValueError(f"W must be {layout.M} x {layout.K}")
    _packed_ok(layout, values, indices)
    _check(lib().nmg_compress(layout.c, W.data_ptr(), _rows(W, "W"), values.data_ptr(),
                              indices.data_ptr(), _stream(W)), "nmg_compress")


def compress(W: torch.Tensor, n: int, m: int, g: int):
    """Dense W (M x K, GPU) -> (values, indices, layout)."""
    layout = Layout(W.shape[0], W.shape[1], n, m, g, W.dtype)
    values = W.new_empty(layout.values_shape)
    indices = torch.empty(layout.indices_shape, dtype=torch.uint8, device=W.device)
    compress_into(layout, W, values, indices)
    return values, indices, layout


def repack(W: torch.Tensor, indices: torch.Tensor, layout: Layout) -> torch.Tensor:
    """Dense W (M x K, GPU) packed into the existing pattern `indices`
    (the fixed-mask path after a weight update) -> values."""
    _need_cuda(W, indices)
    if W.dtype != layout.dtype or indices.dtype != torch.uint8:
        raise TypeError("dtype mismatch")
    if W.shape != (layout.M, layout.K):
        raise ValueError(f"W must be {layout.M} x {layout.K}")
    if indices.shape != layout.indices_shape or not indices.is_contiguous():
        raise ValueError(f"indices must be contiguous {layout.indices_shape}")
    values = W.new_empty(layout.values_shape)
    _check(lib().nmg_repack(layout.c, W.data_ptr(), _rows(W, "W"), indices.data_ptr(),
                            values.data_ptr(), _stream(W)), "nmg_repack")
    return values


# kernel families that run on prepared operands (made per call by
# nmg_spmm_with, or once by nmg_x16_prepare for nmg_spmm_x16), and the element
# type each takes
X16_KERNELS = {"mfma_wide": torch.float16, "mfma_split": torch.float32}


def x16_prepare(values, indices, layout: Layout) -> torch.Tensor:
    """``nmg_x16_prepare``: the prepared operands of a packed weight (bytes)."""
    _need_cuda(values, indices)
    nbytes = lib().nmg_x16_prepared_bytes(layout.c)
    if nbytes < 0:
        raise NmgError(ERR_UNSUPPORTED, "nmg_x16_prepared_bytes")
    prepared = torch.empty(int(nbytes), dtype=torch.uint8, device=values.device)
    _check(lib().nmg_x16_prepare(layout.c, values.data_ptr(), indices.data_ptr(),
                                 prepared.data_ptr(), _stream(values)), "nmg_x16_prepare")
    return prepared


def spmm_x16_into(layout: Layout, prepared, X, Y):
    """``nmg_spmm_x16`` into a caller-allocated Y (M x N)."""
    _need_cuda(prepared, X, Y)
    if X.dtype != layout.dtype or Y.dtype != layout.dtype:
        raise TypeError("dtype mismatch")
    if X.shape[0] != layout.K or Y.shape[0] != layout.M or Y.shape[1] != X.shape[1]:
        raise ValueError("X must be K x N and Y M x N")
    _check(lib().nmg_spmm_x16(layout.c, prepared.data_ptr(), X.data_ptr(), _rows(X, "X"),
                              X.shape[1], Y.data_ptr(), _rows(Y, "Y"), _stream(X)), "nmg_spmm_x16")


def spmm_x16_epilogue(layout: Layout, prepared, X, epilogue: str = "none", R=None, Y=None):
    """``nmg_spmm_x16_epilogue``: Y = W_s X ("none") or W_s X + R ("add") from
    prepared operands, the sum taken as the product is stored."""
    _need_cuda(prepared, X)
    if X.dtype != layout.dtype or X.shape[0] != layout.K:
        raise ValueError("X must be K x N of the layout's dtype")
    N = X.shape[1]
    if Y is None:
        Y = X.new_empty((layout.M, N))
    _need_cuda(Y)
    if Y.dtype != layout.dtype or Y.shape != (layout.M, N):
        raise ValueError("Y must be M x N of the layout's dtype")
    rp, ldr = None, 0
    if epilogue == "add":
        if R is None:
            raise ValueError("the add epilogue needs R")
        _need_cuda(R)
        if R.dtype != layout.dtype or R.shape != (layout.M, N):
            raise ValueError("R must be M x N of the layout's dtype")
        rp, ldr = R.data_ptr(), _rows(R, "R")
    _check(lib().nmg_spmm_x16_epilogue(layout.c, prepared.data_ptr(),
                                       EPILOGUES[epilogue], X.data_ptr(), _rows(X, "X"), N, rp, ldr,
                                       Y.data_ptr(), _rows(Y, "Y"), _stream(X)),
           "nmg_spmm_x16_epilogue")
    return Y


def spmm_into(layout: Layout, values, indices, X, Y, kernel: str = "auto"):
    """``nmg_spmm_epilogue_ws`` without an epilogue into a caller-allocated Y
    (M x N), scratch memory from torch's allocator."""
    _need_cuda(values, indices, X, Y)
    if X.dtype != layout.dtype or Y.dtype != layout.dtype or values.dtype != layout.dtype:
        raise TypeError("dtype mismatch")
    if X.shape[0] != layout.K or Y.shape[0] != layout.M or Y.shape[1] != X.shape[1]:
        raise ValueError("X must be K x N and Y M x N")
    _packed_ok(layout, values, indices)
    L = lib()
    N, code = X.shape[1], KERNELS[kernel]
    vp, ip, xp, ldx = values.data_ptr(), indices.data_ptr(), X.data_ptr(), _rows(X, "X")
    ws, wp, wb = _workspace(_workspace_bytes(layout, code, vp, ip, xp, ldx, N), X)
    _check(L.nmg_spmm_epilogue_ws(layout.c, code, 0, vp, ip, xp, ldx, N, None, 0, Y.data_ptr(),
                                  _rows(Y, "Y"), wp, wb, _stream(X)), "nmg_spmm")


def spmm(values, indices, X, layout: Layout, kernel: str = "auto"):
    """Y = W_s X for the packed weight (values, indices)."""
    Y = X.new_empty((layout.M, X.shape[1]))
    spmm_into(layout, values, indices, X, Y, kernel)
    return Y


def spmm_epilogue(values, indices, X, layout: Layout, epilogue: str = "none", R=None,
                  kernel: str = "auto", Y=None):
    """Y = epilogue(W_s X): "none", "gelu" (GELU of the product) or "add"
    (product + R), bit for bit what spmm followed by gelu or add gives."""
    return _spmm_epilogue("nmg_spmm_epilogue_ws", values, indices, X, layout, epilogue, R, kernel, Y)


def spmm_epilogue_noalloc(values, indices, X, layout: Layout, epilogue: str = "none", R=None,
                          kernel: str = "auto", Y=None):
    """``nmg_spmm_epilogue_noalloc``: spmm_epilogue without device allocation
    in the library (the prepared operands of mfma_wide / mfma_split go to the
    library's fixed per-GPU array; overlapping calls on one GPU race).  "auto"
    never puts a layout into that array whose choice without a workspace has no
    scratch memory, so there spmm_epilogue, which brings a workspace, may take
    "sparse" where this call does not.  Y is
    allocated here when not given: pass Y to allocate nothing at all."""
    return _spmm_epilogue("nmg_spmm_epilogue_noalloc", values, indices, X, layout, epilogue, R,
                          kernel, Y)


def _spmm_epilogue(fn, values, indices, X, layout, epilogue, R, kernel, Y):
    _need_cuda(values, indices, X)
    if X.dtype != layout.dtype or values.dtype != layout.dtype:
        raise TypeError("dtype mismatch")
    if X.shape[0] != layout.K:
        raise ValueError("X must be K x N")
    _packed_ok(layout, values, indices)
    N = X.shape[1]
    if Y is None:
        Y = X.new_empty((layout.M, N))
    _need_cuda(Y)
    if Y.dtype != layout.dtype or Y.shape != (layout.M, N):
        raise ValueError("Y must be M x N of the layout's dtype")
    rp, ldr = None, 0
    if epilogue == "add":
        if R is None:
            raise ValueError("the add epilogue needs R")
        _need_cuda(R)
        if R.dtype != layout.dtype or R.shape != (layout.M, N):
            raise ValueError("R must be M x N of the layout's dtype")
        rp, ldr = R.data_ptr(), _rows(R, "R")
    L = lib()
    vp, ip, xp, ldx = values.data_ptr(), indices.data_ptr(), X.data_ptr(), _rows(X, "X")
    args = [layout.c, KERNELS[kernel], EPILOGUES[epilogue], vp, ip, xp, ldx, N, rp, ldr,
            Y.data_ptr(), _rows(Y, "Y")]
    if fn == "nmg_spmm_epilogue_ws":
        ws, wp, wb = _workspace(_workspace_bytes(layout, args[1], vp, ip, xp, ldx, N), X)
        args += [wp, wb]
    _check(getattr(L, fn)(*args, _stream(X)), fn)
    return Y


def auto_kernel(layout: Layout, N: int) -> str:
    """The family spmm / spmm_into / spmm_epilogue run for "auto" on aligned,
    contiguous operands (``nmg_spmm_plan``: they bring a workspace; the family
    without one is ``nmg_spmm_auto_kernel``)."""
    return _KERNEL_NAME[lib().nmg_spmm_plan(layout.c, KERNELS["auto"], None, None, None, N, N, None)]


def densify(values, indices, layout: Layout):
    """(values, indices) -> dense M x K weight (zeros at dropped positions)."""
    _need_cuda(values, indices)
    out = values.new_empty((layout.M, layout.K), dtype=layout.dtype)
    _check(lib().nmg_densify(layout.c, values.data_ptr(), indices.data_ptr(), out.data_ptr(),
                             layout.K, _stream(values)), "nmg_densify")
    return out


def gelu(x: torch.Tensor, out: torch.Tensor | None = None):
    _need_cuda(x)
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    out = torch.empty_like(x) if out is None else out
    _check(lib().nmg_gelu(_DTYPE_CODE[x.dtype], x.data_ptr(), out.data_ptr(), x.numel(), _stream(x)),
           "nmg_gelu")
    return out


def add(a: torch.Tensor, b: torch.Tensor, out: torch.Tensor | None = None):
    _need_cuda(a, b)
    if a.shape != b.shape or a.dtype != b.dtype or not (a.is_contiguous() and b.is_contiguous()):
        raise ValueError("a and b must be contiguous tensors of one shape and dtype")
    out = torch.empty_like(a) if out is None else out
    _check(lib().nmg_add(_DTYPE_CODE[a.dtype], a.data_ptr(), b.data_ptr(), out.data_ptr(), a.numel(),
                         _stream(a)), "nmg_add")
    return out


# ------------------------------------------------ the paper's chunked layout

class PLayout:
    """Shape of one weight in the paper's chunked layout (``nmg_p_layout``)."""

    def __init__(self, M: int, K: int, n: int, m: int, g: int, dtype=torch.float32):
        if dtype not in _DTYPE_CODE:
            raise TypeError(f"unsupported dtype {dtype}")
        self.c = _PLayout()
        _check(lib().nmg_p_layout_init(ctypes.byref(self.c), M, K, n, m, g, _DTYPE_CODE[dtype]),
               "nmg_p_layout_init")
        self.dtype = dtype
        self._derive()

    def _derive(self):
        c = self.c
        self.M, self.K, self.n, self.m, self.g = c.M, c.K, c.n, c.m, c.g
        self.P, self.S, self.B = c.P, c.S, c.B
        self.values_shape = (self.M, self.B * self.n)
        self.index_shape = (self.M, self.B)

    def __setstate__(self, state):     # (also states of c and dtype alone)
        self.__dict__.update(state)
        self._derive()


def p_compress(W: torch.Tensor, n: int, m: int, g: int):
    """Dense W (M x K, GPU) -> (values, index, layout) in the chunked layout."""
    _need_cuda(W)
    layout = PLayout(W.shape[0], W.shape[1], n, m, g, W.dtype)
    values = W.new_empty(layout.values_shape)
    index = torch.empty(layout.index_shape, dtype=torch.uint8, device=W.device)
    _check(lib().nmg_p_compress(layout.c, W.data_ptr(), _rows(W, "W"), values.data_ptr(),
                                index.data_ptr(), _stream(W)), "nmg_p_compress")
    return values, index, layout


def _p_check(layout: PLayout, values, index):
    _need_cuda(values, index)
    if values.dtype != layout.dtype or index.dtype != torch.uint8:
        raise TypeError("dtype mismatch")
    if values.shape != layout.values_shape or not values.is_contiguous():
        raise ValueError(f"values must be contiguous {layout.values_shape}")
    if index.shape != layout.index_shape or not index.is_contiguous():
        raise ValueError(f"index must be contiguous {layout.index_shape}")


def p_spmm(values, index, X, layout: PLayout, kernel: str = "auto"):
    """Y = W_s X for the chunked layout; kernel is "auto", "valu" or "mfma"."""
    _p_check(layout, values, index)
    _need_cuda(X)
    if X.dtype != layout.dtype or X.shape[0] != layout.K:
        raise ValueError("X must be K x N of the layout's dtype")
    if kernel not in ("auto", "valu", "mfma"):
        raise ValueError(f"unknown chunked-layout kernel {kernel!r}")
    Y = X.new_empty((layout.M, X.shape[1]))
    L = lib()
    N, code = X.shape[1], KERNELS[kernel]
    ws, wp, wb = _workspace(L.nmg_p_spmm_workspace_bytes(layout.c, code, N), X)
    _check(L.nmg_p_spmm_ws(layout.c, code, values.data_ptr(), index.data_ptr(), X.data_ptr(),
                           _rows(X, "X"), N, Y.data_ptr(), _rows(Y, "Y"), wp, wb, _stream(X)),
           "nmg_p_spmm_ws")
    return Y


def p_densify(values, index, layout: PLayout):
    """Chunked layout -> dense M x K weight."""
    _p_check(layout, values, index)
    out = values.new_empty((layout.M, layout.K), dtype=layout.dtype)
    _check(lib().nmg_p_densify(layout.c, values.data_ptr(), index.data_ptr(), out.data_ptr(),
                               layout.K, _stream(values)), "nmg_p_densify")
    return out


def p_refine(W: torch.Tensor, index: torch.Tensor, layout: PLayout):
    """The swap search of Section 5.2's GPU converter from the packing `index`:
    returns new (values, index); the inputs are not changed."""
    _need_cuda(W, index)
    if W.dtype != layout.dtype or index.dtype != torch.uint8:
        raise TypeError("dtype mismatch")
    if W.shape != (layout.M, layout.K):
        raise ValueError(f"W must be {layout.M} x {layout.K}")
    if index.shape != layout.index_shape:
        raise ValueError(f"index must be {layout.index_shape}")
    idx = index.contiguous().clone()
    values = W.new_empty(layout.values_shape)
    _check(lib().nmg_p_refine(layout.c, W.data_ptr(), _rows(W, "W"), values.data_ptr(),
                              idx.data_ptr(), _stream(W)), "nmg_p_refine")
    return values, idx


# ---------------------------------------- attention between sparse projections

def rotary_table(length: int, dim: int, base: float = 10000.0, scaling: str = "none",
                 factor: float = 1.0, original: float = 0.0, slow: float = 1.0, fast: float = 32.0,
                 magnitude: float = 1.0, device="cuda") -> torch.Tensor:
    """``nmg_rotary_table``: (2, dim / 2, length) binary32, cosines then sines
    of every position's angles; made once for a model and a length.  scaling
    "linear", "ntk" and "parts" stretch it to `factor` times the context,
    "parts" from the `original` length."""
    if scaling not in ROTARY_SCALING:
        raise ValueError(f"unknown scaling {scaling!r}")
    if dim < 2 or dim % 2 or length < 1:
        raise ValueError("dim must be even and length positive")
    table = torch.empty((2, dim // 2, length), dtype=torch.float32, device=device)
    _need_cuda(table)
    _check(lib().nmg_rotary_table(dim, length, base, ROTARY_SCALING[scaling], factor, original,
                                  slow, fast, magnitude, table.data_ptr(), _stream(table)),
           "nmg_rotary_table")
    return table


# These calls are made for every layer and token, so their marshalling is
# compiled (csrc/calls.cpp): the same checks, outputs and workspace from torch's
# allocator, and errors as above.

def rotary(X, heads: int, table, positions, layout: str = "half", out=None):
    """``nmg_rotary``: the first 2 * table.shape[1] rows of each of the `heads`
    heads of X (features x tokens) turned by their tokens' positions, the
    others copied.  out may be X."""
    return (_calls or _load_calls()).rotary(X, heads, table, positions, layout, out)


def qk_norm_rotary(Q, K, heads: int, kv_heads: int, q_weight, k_weight, table=None, positions=None,
                   layout: str = "half", eps: float = 1e-6, out=None):
    """``nmg_qk_norm_rotary``: RMS norm of every head's column of Q and K
    (weights float32 of head_dim, or None) and the rotation (none without a
    table).  out: (Q's, K's), which may be Q and K.  Returns both."""
    yq, yk = (None, None) if out is None else out
    return (_calls or _load_calls()).qk_norm_rotary(Q, K, heads, kv_heads, q_weight, k_weight, table,
                                                    positions, layout, eps, yq, yk)


def attention(Q, K, V, heads: int, kv_heads: int, q_offsets, kv_begin, kv_end, key_mask=None,
              scale: float | None = None, out=None):
    """``nmg_attention``: every sequence's query columns of Q (features x tokens)
    attend to its key columns of K and V; sequence b has queries q_offsets[b] ..
    q_offsets[b + 1] - 1 and keys kv_begin[b] .. kv_end[b] - 1 (int32 tensors on
    the device).  key_mask: uint8 or bool for every key column, 0 leaves it out.
    scale: head_dim ** -0.5 by default.  Scratch memory from torch's
    allocator."""
    return (_calls or _load_calls()).attention(Q, K, V, heads, kv_heads, q_offsets, kv_begin, kv_end,
                                               key_mask, None, scale, out)


def tree_attention(Q, K, V, heads: int, kv_heads: int, q_offsets, kv_begin, kv_end, tree,
                   scale: float | None = None, out=None):
    """``nmg_tree_attention``: the query columns are drafted tokens, whose keys and
    values are the last columns of their sequence's key range; tree (uint8 or
    bool, a row per query column) says which drafted tokens of its sequence each
    one attends to, itself included; all earlier columns it attends to."""
    if tree is None:
        raise ValueError("tree must be uint8 or bool with a row for every query column")
    return (_calls or _load_calls()).attention(Q, K, V, heads, kv_heads, q_offsets, kv_begin, kv_end,
                                               None, tree, scale, out)


# ------------------------------------------------------------ a cache in 8 bits

class _Fixed:
    """What the library knows by the addresses of its tensors: once it is made, its attributes stay."""

    def __setattr__(self, name, value):
        if self.__dict__.get("made"):
            raise AttributeError(f"a {type(self).__name__} stays as it was made: calls know its tensors by address")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        raise AttributeError(f"a {type(self).__name__} stays as it was made: calls know its tensors by address")


class Cache(_Fixed):
    """Buffers of a cache in 8 bits for several sequences and layers (``nmg_cache``);
    they are read by the attribute names below and cannot be exchanged afterwards (calls
    know their addresses).

        k_pages     layers x pages x kv_heads x block x dim16   float8_e4m3fn or int8
        v_pages     layers x pages x kv_heads x head_dim x block
        k_scales    layers x pages x kv_heads                   float32
        v_scales
        k_open      layers x sequences x kv_heads x room x dim16  float32 or float16
        v_open      layers x sequences x kv_heads x head_dim x room
        table       sequences x row                             int32, -1: no page
        references  pages                                       int32, rows that hold a page

    dim16 is head_dim rounded up to 16."""

    def __init__(self, k_pages, v_pages, k_scales, v_scales, k_open, v_open, table, references):
        if v_pages.dim() != 5 or v_open.dim() != 5 or table.dim() != 2:
            raise ValueError("pages and open tokens must have 5 dimensions and the table 2")
        layers, pages, heads, dim, block = v_pages.shape
        sequences, row, room, wide = *table.shape, v_open.shape[4], (dim + 15) // 16 * 16
        by_code = {t: (name, code) for name, (code, t) in CACHE_FORMATS.items()}
        if v_pages.dtype not in by_code or v_open.dtype not in _DTYPE_CODE:
            raise TypeError("pages must be float8_e4m3fn or int8, open tokens float32 or float16")
        want = {"k_pages": ((layers, pages, heads, block, wide), v_pages.dtype),
                "v_pages": ((layers, pages, heads, dim, block), v_pages.dtype),
                "k_scales": ((layers, pages, heads), torch.float32),
                "v_scales": ((layers, pages, heads), torch.float32),
                "k_open": ((layers, sequences, heads, room, wide), v_open.dtype),
                "v_open": ((layers, sequences, heads, dim, room), v_open.dtype),
                "table": ((sequences, row), torch.int32), "references": ((pages,), torch.int32)}
        given = locals()
        for name, (shape, dtype) in want.items():
            t = given[name]
            if t.dtype != dtype:
                raise TypeError(f"{name} must be {dtype}")
            if tuple(t.shape) != shape or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {shape}")
            if not t.is_cuda or t.device != v_pages.device:
                raise ValueError("a cache's tensors must be on one GPU")
        self.buffers = types.MappingProxyType({name: given[name] for name in want})
        self.format, code = by_code[v_pages.dtype]
        self.layers, self.pages, self.kv_heads, self.head_dim, self.block = v_pages.shape
        self.sequences, self.row, self.room, self.dtype = sequences, row, room, v_open.dtype
        self.device, self.index = v_pages.device, v_pages.get_device()
        self.c = _Cache(layers, heads, dim, _DTYPE_CODE[v_open.dtype], code, block, pages, sequences,
                        row, room, *(t.data_ptr() for t in self.buffers.values()))
        if lib().nmg_cache_compact_workspace_bytes(self.c) < 0:
            raise NmgError(ERR_UNSUPPORTED, "nmg_cache")
        self.address, self.made = ctypes.addressof(self.c), True

    def __getattr__(self, name):
        try:
            return self.__dict__["buffers"][name]
        except KeyError:
            raise AttributeError(name) from None

    @classmethod
    def empty(cls, layers: int, kv_heads: int, head_dim: int, sequences: int, pages: int, row: int,
              room: int, block: int = 64, format: str = "e4m3", dtype=torch.float16, device="cuda"):
        """A cache without tokens: every page free, every row of the table empty."""
        if format not in CACHE_FORMATS:
            raise ValueError(f"unknown cache format {format!r}")
        code, wide = CACHE_FORMATS[format][1], (head_dim + 15) // 16 * 16
        make = lambda shape, t, v=0: torch.full(shape, v, dtype=t, device=device)   # noqa: E731
        page = lambda *shape: make(shape, torch.uint8).view(code)                   # noqa: E731
        return cls(page(layers, pages, kv_heads, block, wide), page(layers, pages, kv_heads, head_dim, block),
                   make((layers, pages, kv_heads), torch.float32), make((layers, pages, kv_heads), torch.float32),
                   make((layers, sequences, kv_heads, room, wide), dtype),
                   make((layers, sequences, kv_heads, head_dim, room), dtype),
                   make((sequences, row), torch.int32, -1), make((pages,), torch.int32))


def _lengths(cache, t, name="lengths"):
    """Checks an int32 value for every sequence, on the cache's device, which is current."""
    _need_cuda(t, cache.table)
    if t.dtype != torch.int32 or tuple(t.shape) != (cache.sequences,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 values, one for every sequence")
    return t.data_ptr()


def cache_append(cache: Cache, layer: int, K, V, q_offsets, lengths):
    """``nmg_cache_append``: the drafted tokens' keys and values of one layer
    (features x tokens), sequence b's in columns q_offsets[b] .. q_offsets[b + 1] -
    1, behind its lengths[b] kept ones (int32 tensors on the device)."""
    (_calls or _load_calls()).cache_append(cache.address, cache.index, layer, K, V, q_offsets, lengths)


def cache_attention(cache: Cache, layer: int, Q, heads: int, q_offsets, lengths, tree=None,
                    longest: int | None = None, scale: float | None = None, out=None):
    """``nmg_cache_attention``: every drafted token (a column of Q) attends to its
    sequence's kept tokens and to the drafted ones that its row of `tree` (uint8 or
    bool) names, or without a tree to itself and those before it.  longest: the
    most kept tokens of a sequence, where the program knows it (it guides the
    split over the GPU).  scale: head_dim ** -0.5 by default.  Scratch memory from
    torch's allocator."""
    return (_calls or _load_calls()).cache_attention(cache.address, cache.index, layer, Q, heads, q_offsets,
                                                     lengths, tree, longest, scale, out)


def cache_commit(cache: Cache, lengths, kept_offsets, kept=None, out=None):
    """``nmg_cache_commit``: of sequence b's drafted tokens those numbered
    kept[kept_offsets[b]] .. kept[kept_offsets[b + 1] - 1] stay (int32, ascending), without
    `kept` the first kept_offsets[b + 1] - kept_offsets[b]; whole blocks become
    pages.  Returns the new lengths (out, which is not lengths)."""
    return (_calls or _load_calls()).cache_commit(cache.address, cache.index, lengths, kept_offsets, kept, out)


def cache_reserve(cache: Cache, lengths, tokens) -> torch.Tensor:
    """``nmg_cache_reserve``: pages for tokens[b] more tokens of every sequence.
    Returns the number of pages that were not there (int32, on the device)."""
    n, t = _lengths(cache, lengths), _lengths(cache, tokens, "tokens")
    missing = torch.empty(1, dtype=torch.int32, device=lengths.device)
    _check(lib().nmg_cache_reserve(cache.c, n, t, missing.data_ptr(), _stream(lengths)), "nmg_cache_reserve")
    return missing


def _list(values):
    values = [int(v) for v in values]
    if any(not 0 <= v < 1 << 31 for v in values):
        raise NmgError(ERR_PARAM, "a sequence's number")
    return (ctypes.c_int32 * len(values))(*values), len(values)


def cache_fork(cache: Cache, lengths, sources, targets):
    """``nmg_cache_fork``: sequences `targets` become copies of `sources` (lists of
    numbers), which share their pages.  Changes lengths."""
    n, (a, count), (b, other) = _lengths(cache, lengths), _list(sources), _list(targets)
    if count != other:
        raise ValueError("one target for every source")
    _check(lib().nmg_cache_fork(cache.c, n, count, a, b, _stream(lengths)), "nmg_cache_fork")


def cache_free(cache: Cache, lengths, sequences):
    """``nmg_cache_free``: the sequences of a list give their pages back and have no
    tokens.  Changes lengths."""
    n, (a, count) = _lengths(cache, lengths), _list(sequences)
    _check(lib().nmg_cache_free(cache.c, n, count, a, _stream(lengths)), "nmg_cache_free")


def cache_compact(cache: Cache, table=None, references=None) -> torch.Tensor:
    """``nmg_cache_compact``: the pages in use move to the front of the pool; the
    table and the references follow, into the cache's own or those given.  Returns
    the number of pages in use (int32, on the device)."""
    table = cache.table if table is None else table
    references = cache.references if references is None else references
    _need_cuda(table, references, cache.table)
    for t, like in ((table, cache.table), (references, cache.references)):
        if t.dtype != torch.int32 or t.shape != like.shape or not t.is_contiguous():
            raise ValueError("table and references must be contiguous int32 of the cache's shapes")
    live = torch.empty(1, dtype=torch.int32, device=table.device)
    nbytes = lib().nmg_cache_compact_workspace_bytes(cache.c)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=table.device)
    _check(lib().nmg_cache_compact(cache.c, table.data_ptr(), references.data_ptr(), live.data_ptr(),
                                   ws.data_ptr(), nbytes, _stream(table)), "nmg_cache_compact")
    return live


# ------------------------------------------------------- norms around a block

class Norm(_Fixed):
    """A norm over features (``nmg_norm``): kind "rms", "layer" or "none", weight and
    bias float32 with a value for every feature, or None.  Their values may change, the
    tensors and numbers themselves not: that is another Norm."""

    def __init__(self, kind: str = "rms", weight=None, bias=None, eps: float = 1e-6):
        if kind not in NORMS:
            raise ValueError(f"unknown norm {kind!r}")
        rows, device = -1, -1
        for t in (weight, bias):
            if t is None:
                continue
            if t.dtype != torch.float32 or t.dim() != 1 or not t.is_contiguous():
                raise ValueError("a norm's weight and bias must be contiguous float32 vectors")
            if not t.is_cuda:
                raise ValueError("libnmg works on GPU tensors only")
            if rows >= 0 and (t.numel() != rows or t.get_device() != device):
                raise ValueError("a norm's weight and bias must be of one size, on one GPU")
            rows, device = t.numel(), t.get_device()
        self.kind, self.weight, self.bias, self.eps = kind, weight, bias, eps
        self.c = _Norm(NORMS[kind], None if weight is None else weight.data_ptr(),
                       None if bias is None else bias.data_ptr(), eps)
        self.args, self.made = (ctypes.addressof(self.c), rows, device), True


def residual_norm(A, R=None, gate=None, scale: float = 1.0, after: Norm | None = None,
                  before: Norm | None = None, out=None, keep: bool = True):
    """``nmg_residual_norm``: H = R + scale * gate * after(A) and Y = before(H) of
    matrices features x tokens, one pass.  Returns (H, Y); Y is None without `before`, H
    with keep=False, where only Y is wanted.  out: (H, Y), each None or a tensor, which may be A, gate or R."""
    h, y = (None, None) if out is None else out
    if (before is None and y is not None) or (not keep and h is not None):
        raise ValueError("an output is given that the call does not have")
    return (_calls or _load_calls()).residual_norm(A, R, gate, scale, None if after is None else after.args,
                                                   None if before is None else before.args, h, y, keep)
