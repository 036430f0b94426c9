"""Thin ctypes binding of the C ABI in include/lmkan.h.

Argument marshalling only: every step of the layer runs in the HIP kernels of
liblmkan.so.  PyTorch appears here only as the owner of device memory and of
the current stream.  There is no CPU fallback: if the library is missing or a
call fails, an exception is raised.

The calls that a program makes per step (forward, backward, pack, the
convolution, the optimiser's step, the linear term, the norm, checkpoints, adapters) first go to ``_native`` (csrc/lmkan_torch.cpp), which does the same
marshalling in native code for the ordinary case and returns None for any
other; the code here then takes over and raises what there is to raise.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblmkan.so")

LMKAN_F32, LMKAN_F16, LMKAN_BF16 = 0, 1, 2
LMKAN_LAYOUT_PAPER, LMKAN_LAYOUT_PACKED = 0, 1
LMKAN_FLAG_ACCUMULATE_GRAD_COEF = 1
LMKAN_FLAG_WORKSPACE_HAS_RECORDS = 2
LMKAN_PACK_TILE = 64
LMKAN_MAX_GRID = 64
LMKAN_STATIC_SCRATCH_BYTES = 32 << 20
LMKAN_LINEAR_RELU = 1
LMKAN_LINEAR_ACCUMULATE = 2
LMKAN_NORM_ACCUMULATE = 1
LMKAN_CHECKPOINT_BLOCK = 32
LMKAN_MAX_ADAPTERS = 8192
LMKAN_MAX_ADAPTER_RANK = 256
LMKAN_MAX_ORTHO_STEPS = 32

_TORCH_DTYPE = {LMKAN_F32: torch.float32, LMKAN_F16: torch.float16, LMKAN_BF16: torch.bfloat16}
_DTYPE_CODE = {v: k for k, v in _TORCH_DTYPE.items()}


class LmkanError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().lmkan_status_string(status).decode()
        super().__init__(f"{where}: {msg} (status {status})")


class _Desc(C.Structure):
    _fields_ = [("n_in", C.c_int32), ("n_out", C.c_int32), ("grid", C.c_int32),
                ("spline_order", C.c_int32), ("coef_dtype", C.c_int32),
                ("coef_layout", C.c_int32), ("flags", C.c_int32)]


class _Conv2d(C.Structure):
    _fields_ = [("n", C.c_int32), ("h", C.c_int32), ("w", C.c_int32), ("c_in", C.c_int32),
                ("kh", C.c_int32), ("kw", C.c_int32), ("stride", C.c_int32)]


@dataclass
class Conv2d:
    """Mirror of ``lmkan_conv2d``: channels-last image [n][h][w][c_in], kh x kw windows, no padding."""
    n: int
    h: int
    w: int
    c_in: int
    kh: int
    kw: int
    stride: int

    def c(self) -> _Conv2d:
        return _Conv2d(self.n, self.h, self.w, self.c_in, self.kh, self.kw, self.stride)

    def image_shape(self):
        return (self.n, self.h, self.w, self.c_in)


@dataclass
class LayerDesc:
    """Mirror of ``lmkan_desc``."""
    n_in: int
    n_out: int
    grid: int
    spline_order: int = 2
    coef_dtype: int = LMKAN_F32
    coef_layout: int = LMKAN_LAYOUT_PAPER
    flags: int = 0

    def c(self) -> _Desc:
        return _Desc(self.n_in, self.n_out, self.grid, self.spline_order, self.coef_dtype,
                     self.coef_layout, self.flags)

    @property
    def pairs(self) -> int:
        return self.n_in // 2

    def coef_shape(self):
        return (self.grid + 1, self.grid + 1, self.pairs, self.n_out)


class _Matrices(C.Structure):
    _fields_ = [("batch", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("dtype", C.c_int32),
                ("eps", C.c_float)]


class _Muon(C.Structure):
    _fields_ = [("lr", C.c_float), ("momentum", C.c_float), ("weight_decay", C.c_float), ("scale", C.c_float),
                ("nesterov", C.c_int32)]


class _Linear(C.Structure):
    _fields_ = [("n_in", C.c_int32), ("n_out", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32),
                ("flags", C.c_int32)]


class _Norm(C.Structure):
    _fields_ = [("cols", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("flags", C.c_int32),
                ("eps", C.c_float)]


class _Adapters(C.Structure):
    _fields_ = [("count", C.c_int32), ("rank", C.c_int32), ("n_in", C.c_int32), ("n_out", C.c_int32),
                ("dtype", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("flags", C.c_int32)]


@dataclass
class MatrixDesc:
    """Mirror of ``lmkan_matrices``: a batch of dense matrices [batch][rows][cols].  A table in the layout of
    Alg. 1 is one of (G+1)^2 matrices of pairs x n_out."""
    batch: int
    rows: int
    cols: int
    dtype: int = LMKAN_F32
    eps: float = 1e-7

    def c(self) -> _Matrices:
        return _Matrices(self.batch, self.rows, self.cols, self.dtype, self.eps)

    def shape(self):
        return (self.batch, self.rows, self.cols)


@dataclass
class MuonParams:
    """Mirror of ``lmkan_muon``."""
    lr: float
    momentum: float = 0.95
    weight_decay: float = 0.0
    scale: float = 1.0
    nesterov: bool = True

    def c(self) -> _Muon:
        return _Muon(self.lr, self.momentum, self.weight_decay, self.scale, int(self.nesterov))


@dataclass
class LinearDesc:
    """Mirror of ``lmkan_linear``: Linear(x), or Linear(ReLU(x)) with ``relu``."""
    n_in: int
    n_out: int
    x_dtype: int = LMKAN_F32
    y_dtype: int = LMKAN_F32
    relu: bool = False

    def c(self) -> _Linear:
        return _Linear(self.n_in, self.n_out, self.x_dtype, self.y_dtype, LMKAN_LINEAR_RELU if self.relu else 0)


@dataclass
class NormDesc:
    """Mirror of ``lmkan_norm`` (its flag is an argument of the backward call)."""
    cols: int
    x_dtype: int = LMKAN_F32
    y_dtype: int = LMKAN_F32
    eps: float = 1e-5

    def c(self, accumulate: bool = False) -> _Norm:
        return _Norm(self.cols, self.x_dtype, self.y_dtype, LMKAN_NORM_ACCUMULATE if accumulate else 0, self.eps)


@dataclass
class AdapterDesc:
    """Mirror of ``lmkan_adapters``: ``count`` adapters of one rank for a linear term n_in -> n_out; ``dtype`` is that
    of the adapters."""
    count: int
    rank: int
    n_in: int
    n_out: int
    dtype: int = LMKAN_F32
    x_dtype: int = LMKAN_F32
    y_dtype: int = LMKAN_F32
    relu: bool = False

    def c(self) -> _Adapters:
        return _Adapters(self.count, self.rank, self.n_in, self.n_out, self.dtype, self.x_dtype, self.y_dtype,
                         LMKAN_LINEAR_RELU if self.relu else 0)

    def a_shape(self):
        return (self.count, self.rank, self.n_in)

    def b_shape(self):
        return (self.count, self.n_out, self.rank)


# five steps of the quintic that brings singular values from a few thousandths up near one
QUINTIC_SCHEDULE = ((3.4445, -4.7750, 2.0315),) * 5

_lib = None
_native = None   # the extension module, once the library is loaded


def lib() -> C.CDLL:
    """Load liblmkan.so (built in-tree by ``build.py``); fail loudly if it is absent."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2509_07103_amd.build` "
                          "(the layer has no fallback implementation)")
    L = C.CDLL(LIB_PATH)
    dp = C.POINTER(_Desc)
    L.lmkan_version.restype = C.c_int
    L.lmkan_version.argtypes = []
    L.lmkan_status_string.restype = C.c_char_p
    L.lmkan_status_string.argtypes = [C.c_int]
    L.lmkan_grid.restype = C.c_int
    L.lmkan_grid.argtypes = [C.c_int32, C.c_void_p, C.c_void_p]
    L.lmkan_packed_bytes.restype = C.c_size_t
    L.lmkan_packed_bytes.argtypes = [dp]
    L.lmkan_workspace_bytes.restype = C.c_size_t
    L.lmkan_workspace_bytes.argtypes = [dp, C.c_int64, C.c_int32]
    L.lmkan_pack.restype = C.c_int
    L.lmkan_pack.argtypes = [dp, C.c_void_p, C.c_void_p, C.c_void_p]
    L.lmkan_locate.restype = C.c_int
    L.lmkan_locate.argtypes = [dp, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
    L.lmkan_forward.restype = C.c_int
    L.lmkan_forward.argtypes = [dp, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                C.c_size_t, C.c_void_p]
    L.lmkan_forward_static.restype = C.c_int
    L.lmkan_forward_static.argtypes = [dp, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    L.lmkan_fold.restype = C.c_int
    L.lmkan_fold.argtypes = [dp, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    L.lmkan_hessian_reg.restype = C.c_int
    L.lmkan_hessian_reg.argtypes = [dp, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
    L.lmkan_backward.restype = C.c_int
    L.lmkan_backward.argtypes = [dp, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.lmkan_time_next_kernel.restype = C.c_int
    L.lmkan_time_next_kernel.argtypes = [C.c_void_p, C.c_void_p]
    L.lmkan_microbench.restype = C.c_int
    L.lmkan_microbench.argtypes = [C.c_int32, C.c_void_p, C.c_size_t, C.POINTER(C.c_double), C.c_void_p]
    mp, up, np_ = C.POINTER(_Matrices), C.POINTER(_Muon), C.POINTER(_Linear)
    L.lmkan_orthogonalize_workspace_bytes.restype = C.c_size_t
    L.lmkan_orthogonalize_workspace_bytes.argtypes = [mp]
    L.lmkan_orthogonalize.restype = C.c_int
    L.lmkan_orthogonalize.argtypes = [mp, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                      C.c_void_p]
    L.lmkan_muon_step.restype = C.c_int
    L.lmkan_muon_step.argtypes = [mp, up, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_size_t, C.c_void_p]
    L.lmkan_quantize_rows.restype = C.c_int
    L.lmkan_quantize_rows.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p]
    L.lmkan_linear_i8_workspace_bytes.restype = C.c_size_t
    L.lmkan_linear_i8_workspace_bytes.argtypes = [np_, C.c_int64]
    L.lmkan_linear_i8.restype = C.c_int
    L.lmkan_linear_i8.argtypes = [np_, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    vp, lp, ap = C.c_void_p, C.POINTER(_Norm), C.POINTER(_Adapters)
    L.lmkan_checkpoint_exps_bytes.restype = C.c_size_t
    L.lmkan_checkpoint_exps_bytes.argtypes = [C.c_int64, C.c_int32]
    L.lmkan_checkpoint_rows.restype = C.c_int
    L.lmkan_checkpoint_rows.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp]
    L.lmkan_restore_rows.restype = C.c_int
    L.lmkan_restore_rows.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp]
    L.lmkan_layer_norm.restype = C.c_int
    L.lmkan_layer_norm.argtypes = [lp, C.c_int64, vp, vp, vp, vp, vp, vp, vp, vp]
    L.lmkan_layer_norm_backward_workspace_bytes.restype = C.c_size_t
    L.lmkan_layer_norm_backward_workspace_bytes.argtypes = [lp, C.c_int64]
    L.lmkan_layer_norm_backward.restype = C.c_int
    L.lmkan_layer_norm_backward.argtypes = [lp, C.c_int64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.lmkan_linear_grad_workspace_bytes.restype = C.c_size_t
    L.lmkan_linear_grad_workspace_bytes.argtypes = [np_, C.c_int64]
    L.lmkan_linear_grad.restype = C.c_int
    L.lmkan_linear_grad.argtypes = [np_, C.c_int64, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.lmkan_adapters_workspace_bytes.restype = C.c_size_t
    L.lmkan_adapters_workspace_bytes.argtypes = [ap, C.c_int64]
    L.lmkan_adapters_add.restype = C.c_int
    L.lmkan_adapters_add.argtypes = [ap, C.c_int64, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    cp = C.POINTER(_Conv2d)
    L.lmkan_conv2d_rows.restype = C.c_int64
    L.lmkan_conv2d_rows.argtypes = [cp, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    L.lmkan_conv2d_forward.restype = C.c_int
    L.lmkan_conv2d_forward.argtypes = [dp, cp, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                       C.c_void_p]
    L.lmkan_conv2d_backward.restype = C.c_int
    L.lmkan_conv2d_backward.argtypes = [dp, cp, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_size_t, C.c_void_p]
    from . import _native as native   # ImportError when it has not been built
    native.init(*(C.cast(f, C.c_void_p).value for f in (
        L.lmkan_workspace_bytes, L.lmkan_packed_bytes, L.lmkan_forward, L.lmkan_backward, L.lmkan_conv2d_rows,
        L.lmkan_conv2d_forward, L.lmkan_conv2d_backward, L.lmkan_pack, L.lmkan_orthogonalize_workspace_bytes,
        L.lmkan_orthogonalize, L.lmkan_muon_step, L.lmkan_linear_i8_workspace_bytes, L.lmkan_linear_i8,
        L.lmkan_checkpoint_rows, L.lmkan_restore_rows, L.lmkan_layer_norm, L.lmkan_layer_norm_backward_workspace_bytes,
        L.lmkan_layer_norm_backward, L.lmkan_linear_grad_workspace_bytes, L.lmkan_linear_grad,
        L.lmkan_adapters_workspace_bytes, L.lmkan_adapters_add)))
    _native = native
    _lib = L
    return L


def _fast():
    """The extension module, loading the library first if need be."""
    if _native is None:
        lib()
    return _native


def _check(status: int, where: str) -> None:
    if status != 0:
        raise LmkanError(status, where)


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _used_on(stream, *tensors) -> None:
    """Tells torch's caching allocator that `tensors` (what a call allocated itself: the workspace it
    frees on return, the outputs it hands back) are in use on `stream` when that is not the current
    stream: their memory is then not given out again before the work queued there has finished."""
    if stream is None:
        return
    handle = _stream(stream)
    if handle == torch.cuda.current_stream().cuda_stream:
        return
    s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(handle)
    for t in tensors:
        if t is not None:
            t.record_stream(s)


def _dev(t: torch.Tensor | None, dtype, shape, name: str) -> int | None:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous() or t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected contiguous device tensor {dtype} {tuple(shape)}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def lmkan_version() -> int:
    return lib().lmkan_version()


def lmkan_status_string(status: int) -> str:
    return lib().lmkan_status_string(status).decode()


def lmkan_grid(grid: int):
    """(nodes[G+1], inv_h[G]) as float32 numpy arrays."""
    n = max(int(grid), 0)
    nodes = np.zeros(n + 1, dtype=np.float32)
    inv_h = np.zeros(n, dtype=np.float32)
    _check(lib().lmkan_grid(grid, nodes.ctypes.data, inv_h.ctypes.data), "lmkan_grid")
    return nodes, inv_h


def lmkan_packed_bytes(desc: LayerDesc) -> int:
    return lib().lmkan_packed_bytes(C.byref(desc.c()))


def lmkan_workspace_bytes(desc: LayerDesc, batch: int, backward: bool, need_grad_x: bool = True,
                          need_grad_coef: bool = True) -> int:
    """Workspace of a forward call, or of a backward call for the gradients it is asked for."""
    if not backward:
        code = 0
    else:
        code = 1 if (need_grad_x and need_grad_coef) else (2 if need_grad_x else 3)
    return lib().lmkan_workspace_bytes(C.byref(desc.c()), batch, code)


def _workspace(desc: LayerDesc, batch: int, backward: bool, device, workspace: torch.Tensor | None = None,
               need_grad_x: bool = True, need_grad_coef: bool = True):
    """(tensor or None, bytes): the caller's workspace when given (any dtype, contiguous, on the device;
    its size goes to the library, which checks it), else a fresh allocation of the size the library asks for."""
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace: expected a contiguous device tensor")
        return workspace, workspace.numel() * workspace.element_size()
    need = lmkan_workspace_bytes(desc, batch, backward, need_grad_x, need_grad_coef)
    if need == 0:
        return None, 0
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    return ws, need


def lmkan_pack(desc: LayerDesc, coef: torch.Tensor, stream=None) -> torch.Tensor:
    """Coefficients [G+1][G+1][K][n_out] -> packed tensor (flat, same dtype)."""
    if stream is None:
        out = (_native or _fast()).pack(desc, coef)
        if out is not None:
            return out
    dt = _TORCH_DTYPE[desc.coef_dtype]
    src = _dev(coef, dt, desc.coef_shape(), "coef")
    nbytes = lmkan_packed_bytes(desc)
    out = torch.empty(nbytes // coef.element_size(), dtype=dt, device=coef.device)
    _check(lib().lmkan_pack(C.byref(desc.c()), src, out.data_ptr(), _stream(stream)), "lmkan_pack")
    _used_on(stream, out)
    return out


def _coef_ptr(desc: LayerDesc, coef: torch.Tensor | None) -> int | None:
    if coef is None:
        return None
    dt = _TORCH_DTYPE[desc.coef_dtype]
    if desc.coef_layout == LMKAN_LAYOUT_PACKED:
        shape = (lmkan_packed_bytes(desc) // (4 if desc.coef_dtype == LMKAN_F32 else 2),)
    else:
        shape = desc.coef_shape()
    return _dev(coef, dt, shape, "coef")


def lmkan_locate(desc: LayerDesc, x: torch.Tensor, stream=None) -> torch.Tensor:
    batch = x.shape[0]
    xp = _dev(x, torch.float32, (batch, desc.n_in), "x")
    cell = torch.empty((batch, desc.pairs), dtype=torch.int32, device=x.device)
    _check(lib().lmkan_locate(C.byref(desc.c()), batch, xp, cell.data_ptr(), _stream(stream)),
           "lmkan_locate")
    _used_on(stream, cell)
    return cell


def lmkan_forward(desc: LayerDesc, x: torch.Tensor, coef: torch.Tensor, y: torch.Tensor | None = None,
                  stream=None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    if stream is None:
        out = (_native or _fast()).forward(desc, None, x, coef, y, workspace)
        if out is not None:
            return out
    batch = x.shape[0]
    xp = _dev(x, torch.float32, (batch, desc.n_in), "x")
    cp = _coef_ptr(desc, coef)
    if y is None:
        y = torch.empty((batch, desc.n_out), dtype=torch.float32, device=x.device)
    yp = _dev(y, torch.float32, (batch, desc.n_out), "y")
    ws, wsz = _workspace(desc, batch, False, x.device, workspace)
    _check(lib().lmkan_forward(C.byref(desc.c()), batch, xp, cp, yp,
                               ws.data_ptr() if ws is not None else None, wsz, _stream(stream)),
           "lmkan_forward")
    _used_on(stream, ws, y)
    return y


def lmkan_forward_static(desc: LayerDesc, x: torch.Tensor, coef: torch.Tensor, y: torch.Tensor,
                         stream=None) -> torch.Tensor:
    """lmkan_forward on the library's own static scratch: the caller brings x, coef and y, nothing is allocated."""
    batch = x.shape[0]
    xp = _dev(x, torch.float32, (batch, desc.n_in), "x")
    cp = _coef_ptr(desc, coef)
    yp = _dev(y, torch.float32, (batch, desc.n_out), "y")
    _check(lib().lmkan_forward_static(C.byref(desc.c()), batch, xp, cp, yp, _stream(stream)),
           "lmkan_forward_static")
    return y


def lmkan_backward(desc: LayerDesc, x: torch.Tensor, coef: torch.Tensor | None, grad_y: torch.Tensor,
                   need_grad_x: bool = True, need_grad_coef: bool = True,
                   grad_x: torch.Tensor | None = None, grad_coef: torch.Tensor | None = None,
                   stream=None, workspace: torch.Tensor | None = None):
    """Returns (grad_x or None, grad_coef or None); grad_coef is float32 in the layout of Alg. 1."""
    if stream is None:
        out = (_native or _fast()).backward(desc, None, x, coef, grad_y, need_grad_x, need_grad_coef, grad_x,
                                            grad_coef, workspace)
        if out is not None:
            return out
    batch = x.shape[0]
    xp = _dev(x, torch.float32, (batch, desc.n_in), "x")
    cp = _coef_ptr(desc, coef)
    gyp = _dev(grad_y, torch.float32, (batch, desc.n_out), "grad_y")
    if need_grad_x and grad_x is None:
        grad_x = torch.empty((batch, desc.n_in), dtype=torch.float32, device=x.device)
    if need_grad_coef and grad_coef is None:
        if desc.flags & LMKAN_FLAG_ACCUMULATE_GRAD_COEF:
            raise ValueError("accumulating into grad_coef needs an existing grad_coef tensor")
        grad_coef = torch.empty(desc.coef_shape(), dtype=torch.float32, device=x.device)
    gxp = _dev(grad_x, torch.float32, (batch, desc.n_in), "grad_x") if need_grad_x else None
    gcp = _dev(grad_coef, torch.float32, desc.coef_shape(), "grad_coef") if need_grad_coef else None
    ws, wsz = _workspace(desc, batch, True, x.device, workspace, need_grad_x, need_grad_coef)
    _check(lib().lmkan_backward(C.byref(desc.c()), batch, xp, cp, gyp, gxp, gcp,
                                ws.data_ptr() if ws is not None else None, wsz, _stream(stream)),
           "lmkan_backward")
    _used_on(stream, ws, grad_x, grad_coef)
    return (grad_x if need_grad_x else None), (grad_coef if need_grad_coef else None)


def lmkan_time_next_kernel(start: torch.cuda.Event | None, stop: torch.cuda.Event | None) -> None:
    """Arms two timing events (already created: record them once beforehand) for the main kernel of
    the next compute call of this thread; (None, None) disarms."""
    hs = None if start is None else start.cuda_event
    he = None if stop is None else stop.cuda_event
    if (start is not None and not hs) or (stop is not None and not he):
        raise ValueError("the events must exist already: record each once before arming them")
    _check(lib().lmkan_time_next_kernel(hs, he), "lmkan_time_next_kernel")


MICROBENCH = {"hbm_copy_GBps": 0, "hbm_read_GBps": 1, "fma_per_clk_cu": 2, "mfma_fma_per_clk_cu": 3,
              "lds_read_B_per_clk_cu": 4, "lds_write_B_per_clk_cu": 5, "l2_row_gather_B_per_clk_cu": 6,
              "nominal_clock_GHz": 7}


def lmkan_microbench(which: int, scratch: torch.Tensor, stream=None) -> float:
    """One of the machine measurements of ``lmkan_microbench`` (waits for its kernels)."""
    if not scratch.is_cuda or not scratch.is_contiguous():
        raise ValueError("scratch: expected a contiguous device tensor")
    out = C.c_double(0.0)
    _check(lib().lmkan_microbench(which, scratch.data_ptr(), scratch.numel() * scratch.element_size(),
                                  C.byref(out), _stream(stream)), "lmkan_microbench")
    return out.value


def lmkan_conv2d_rows(conv: Conv2d):
    """(rows, out_h, out_w) of the equivalent fully connected layer."""
    oh, ow = C.c_int32(0), C.c_int32(0)
    rows = lib().lmkan_conv2d_rows(C.byref(conv.c()), C.byref(oh), C.byref(ow))
    if rows < 0:
        raise ValueError(f"invalid convolution geometry {conv}")
    return rows, oh.value, ow.value


def lmkan_conv2d_forward(desc: LayerDesc, conv: Conv2d, x: torch.Tensor, coef: torch.Tensor,
                         y: torch.Tensor | None = None, stream=None,
                         workspace: torch.Tensor | None = None) -> torch.Tensor:
    """x[n][h][w][c_in] -> y[n][out_h][out_w][n_out]."""
    if stream is None:
        out = (_native or _fast()).forward(desc, conv, x, coef, y, workspace)
        if out is not None:
            return out
    rows, oh, ow = lmkan_conv2d_rows(conv)
    xp = _dev(x, torch.float32, conv.image_shape(), "x")
    cp = _coef_ptr(desc, coef)
    if y is None:
        y = torch.empty((conv.n, oh, ow, desc.n_out), dtype=torch.float32, device=x.device)
    yp = _dev(y, torch.float32, (conv.n, oh, ow, desc.n_out), "y")
    ws, wsz = _workspace(desc, rows, False, x.device, workspace)
    _check(lib().lmkan_conv2d_forward(C.byref(desc.c()), C.byref(conv.c()), xp, cp, yp,
                                      ws.data_ptr() if ws is not None else None, wsz, _stream(stream)),
           "lmkan_conv2d_forward")
    _used_on(stream, ws, y)
    return y


def lmkan_conv2d_backward(desc: LayerDesc, conv: Conv2d, x: torch.Tensor, coef: torch.Tensor | None,
                          grad_y: torch.Tensor, need_grad_x: bool = True, need_grad_coef: bool = True,
                          grad_x: torch.Tensor | None = None, grad_coef: torch.Tensor | None = None, stream=None,
                          workspace: torch.Tensor | None = None):
    """Returns (grad_x in the shape of the image or None, grad_coef in the layout of Alg. 1 or None)."""
    if stream is None:
        out = (_native or _fast()).backward(desc, conv, x, coef, grad_y, need_grad_x, need_grad_coef, grad_x,
                                            grad_coef, workspace)
        if out is not None:
            return out
    rows, oh, ow = lmkan_conv2d_rows(conv)
    xp = _dev(x, torch.float32, conv.image_shape(), "x")
    cp = _coef_ptr(desc, coef)
    gyp = _dev(grad_y, torch.float32, (conv.n, oh, ow, desc.n_out), "grad_y")
    if need_grad_x and grad_x is None:
        grad_x = torch.empty(conv.image_shape(), dtype=torch.float32, device=x.device)
    if need_grad_coef and grad_coef is None:
        if desc.flags & LMKAN_FLAG_ACCUMULATE_GRAD_COEF:
            raise ValueError("accumulating into grad_coef needs an existing grad_coef tensor")
        grad_coef = torch.empty(desc.coef_shape(), dtype=torch.float32, device=x.device)
    gxp = _dev(grad_x, torch.float32, conv.image_shape(), "grad_x") if need_grad_x else None
    gcp = _dev(grad_coef, torch.float32, desc.coef_shape(), "grad_coef") if need_grad_coef else None
    ws, wsz = _workspace(desc, rows, True, x.device, workspace, need_grad_x, need_grad_coef)
    _check(lib().lmkan_conv2d_backward(C.byref(desc.c()), C.byref(conv.c()), xp, cp, gyp, gxp, gcp,
                                       ws.data_ptr() if ws is not None else None, wsz, _stream(stream)),
           "lmkan_conv2d_backward")
    _used_on(stream, ws, grad_x, grad_coef)
    return (grad_x if need_grad_x else None), (grad_coef if need_grad_coef else None)


def lmkan_hessian_reg(desc: LayerDesc, coef: torch.Tensor, scale: float = 1.0, need_value: bool = True,
                      need_grad: bool = True, grad_coef: torch.Tensor | None = None, stream=None):
    """Returns (value tensor of one float64 or None, scale * gradient float32 in the layout of Alg. 1 or None)."""
    cp = _coef_ptr(desc, coef)
    value = torch.empty(1, dtype=torch.float64, device=coef.device) if need_value else None
    if need_grad and grad_coef is None:
        if desc.flags & LMKAN_FLAG_ACCUMULATE_GRAD_COEF:
            raise ValueError("accumulating into grad_coef needs an existing grad_coef tensor")
        grad_coef = torch.empty(desc.coef_shape(), dtype=torch.float32, device=coef.device)
    gcp = _dev(grad_coef, torch.float32, desc.coef_shape(), "grad_coef") if need_grad else None
    _check(lib().lmkan_hessian_reg(C.byref(desc.c()), cp, float(scale),
                                   value.data_ptr() if need_value else None, gcp, _stream(stream)),
           "lmkan_hessian_reg")
    _used_on(stream, value, grad_coef)
    return value, (grad_coef if need_grad else None)


def lmkan_fold(desc: LayerDesc, coef: torch.Tensor, gamma: float = 1.0, lin_w: torch.Tensor | None = None,
               lin_b: torch.Tensor | None = None, out_scale: torch.Tensor | None = None,
               out_shift: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Folds, in place, the ReLU-first preconditioning and an output affine into a float32 table."""
    cp = _coef_ptr(desc, coef)
    wp = _dev(lin_w, torch.float32, (desc.n_out, desc.n_in), "lin_w") if lin_w is not None else None
    bp = _dev(lin_b, torch.float32, (desc.n_out,), "lin_b") if lin_b is not None else None
    sp = _dev(out_scale, torch.float32, (desc.n_out,), "out_scale") if out_scale is not None else None
    tp = _dev(out_shift, torch.float32, (desc.n_out,), "out_shift") if out_shift is not None else None
    _check(lib().lmkan_fold(C.byref(desc.c()), cp, float(gamma), wp, bp, sp, tp, _stream(stream)), "lmkan_fold")
    return coef


@functools.lru_cache(maxsize=64)
def _schedule_bytes(schedule: tuple) -> bytes:
    if any(len(row) != 3 for row in schedule):
        raise ValueError("schedule: expected a sequence of (a, b, c)")
    return np.asarray(schedule, dtype=np.float32).tobytes()


def _schedule(schedule) -> bytes:
    """float32 [steps][3] of a sequence of (a, b, c)."""
    return _schedule_bytes(tuple(tuple(float(v) for v in row) for row in schedule))


def _call_workspace(workspace: torch.Tensor | None, need: int, device):
    """(tensor or None, bytes): the caller's workspace, else a fresh allocation of `need` bytes."""
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace: expected a contiguous device tensor")
        return workspace, workspace.numel() * workspace.element_size()
    return (torch.empty(need, dtype=torch.uint8, device=device), need) if need else (None, 0)


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def lmkan_orthogonalize_workspace_bytes(desc: MatrixDesc) -> int:
    return lib().lmkan_orthogonalize_workspace_bytes(C.byref(desc.c()))


def lmkan_orthogonalize(desc: MatrixDesc, x: torch.Tensor, schedule=QUINTIC_SCHEDULE, out: torch.Tensor | None = None,
                        stream=None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Each matrix of x [batch][rows][cols] brought near orthonormal rows (columns when rows > cols) by
    Newton-Schulz steps, one (a, b, c) of ``schedule`` each; ``out`` may be ``x``."""
    rows = _schedule(schedule)
    if stream is None:
        done = (_native or _fast()).orthogonalize(desc, rows, x, out, workspace)
        if done is not None:
            return done
    dt = _TORCH_DTYPE[desc.dtype]
    xp = _dev(x, dt, desc.shape(), "x")
    if out is None:
        out = torch.empty(desc.shape(), dtype=dt, device=x.device)
    op = _dev(out, dt, desc.shape(), "out")
    ws, wsz = _call_workspace(workspace, lmkan_orthogonalize_workspace_bytes(desc), x.device)
    _check(lib().lmkan_orthogonalize(C.byref(desc.c()), len(rows) // 12, rows, xp, op, _ptr(ws), wsz, _stream(stream)),
           "lmkan_orthogonalize")
    _used_on(stream, ws, out)
    return out


def lmkan_muon_step(desc: MatrixDesc, muon: MuonParams, grad: torch.Tensor, momentum: torch.Tensor,
                    weight: torch.Tensor, schedule=QUINTIC_SCHEDULE, stream=None,
                    workspace: torch.Tensor | None = None) -> torch.Tensor:
    """One optimiser step in place: ``momentum`` and ``weight`` (float32) change, ``weight`` is returned."""
    rows = _schedule(schedule)
    if stream is None:
        done = (_native or _fast()).muon_step(desc, muon, rows, grad, momentum, weight, workspace)
        if done is not None:
            return done
    gp = _dev(grad, _TORCH_DTYPE[desc.dtype], desc.shape(), "grad")
    mp = _dev(momentum, torch.float32, desc.shape(), "momentum")
    wp = _dev(weight, torch.float32, desc.shape(), "weight")
    ws, wsz = _call_workspace(workspace, lmkan_orthogonalize_workspace_bytes(desc), grad.device)
    _check(lib().lmkan_muon_step(C.byref(desc.c()), C.byref(muon.c()), len(rows) // 12, rows, gp, mp, wp, _ptr(ws),
                                 wsz, _stream(stream)), "lmkan_muon_step")
    _used_on(stream, ws)
    return weight


def lmkan_quantize_rows(x: torch.Tensor, relu: bool = False, stream=None):
    """x [rows][cols] -> (codes int8 [rows][cols], scale float32 [rows])."""
    if x.dim() != 2 or x.dtype not in _DTYPE_CODE:
        raise ValueError(f"x: expected a matrix of float32, float16 or bfloat16, got {x.dtype} {tuple(x.shape)}")
    rows, cols = x.shape
    xp = _dev(x, x.dtype, (rows, cols), "x")
    codes = torch.empty((rows, cols), dtype=torch.int8, device=x.device)
    scale = torch.empty((rows,), dtype=torch.float32, device=x.device)
    _check(lib().lmkan_quantize_rows(rows, cols, _DTYPE_CODE[x.dtype], LMKAN_LINEAR_RELU if relu else 0, xp,
                                     codes.data_ptr(), scale.data_ptr(), _stream(stream)), "lmkan_quantize_rows")
    _used_on(stream, codes, scale)
    return codes, scale


def lmkan_linear_i8_workspace_bytes(desc: LinearDesc, batch: int) -> int:
    return lib().lmkan_linear_i8_workspace_bytes(C.byref(desc.c()), batch)


def lmkan_linear_i8(desc: LinearDesc, x: torch.Tensor, w_codes: torch.Tensor, w_scale: torch.Tensor,
                    bias: torch.Tensor | None = None, beta: float = 0.0, y: torch.Tensor | None = None, stream=None,
                    workspace: torch.Tensor | None = None) -> torch.Tensor:
    """y = beta y + Linear(x) with rows quantised on the way and weights of ``lmkan_quantize_rows``."""
    if stream is None:
        done = (_native or _fast()).linear_i8(desc, x, w_codes, w_scale, bias, beta, y, workspace)
        if done is not None:
            return done
    batch = x.shape[0]
    xp = _dev(x, _TORCH_DTYPE[desc.x_dtype], (batch, desc.n_in), "x")
    wp = _dev(w_codes, torch.int8, (desc.n_out, desc.n_in), "w_codes")
    sp = _dev(w_scale, torch.float32, (desc.n_out,), "w_scale")
    bp = _dev(bias, torch.float32, (desc.n_out,), "bias")
    if y is None:
        if beta != 0.0:
            raise ValueError("beta != 0 adds to y: an existing y is needed")
        y = torch.empty((batch, desc.n_out), dtype=_TORCH_DTYPE[desc.y_dtype], device=x.device)
    yp = _dev(y, _TORCH_DTYPE[desc.y_dtype], (batch, desc.n_out), "y")
    ws, wsz = _call_workspace(workspace, lmkan_linear_i8_workspace_bytes(desc, batch), x.device)
    _check(lib().lmkan_linear_i8(C.byref(desc.c()), batch, xp, wp, sp, bp, beta, yp, _ptr(ws), wsz, _stream(stream)),
           "lmkan_linear_i8")
    _used_on(stream, ws, y)
    return y


def _rows(t: torch.Tensor, dtype: int, cols: int, name: str) -> int:
    """Rows of a matrix that is checked with ``_here`` later on."""
    if t.dim() != 2:
        raise ValueError(f"{name}: expected a matrix {_TORCH_DTYPE[dtype]} (rows, {cols}), got {t.dtype} {tuple(t.shape)}")
    return t.shape[0]


def _here(t: torch.Tensor | None, dtype, shape, name: str) -> int | None:
    """``_dev``, and the tensor is on the current device, where the library launches."""
    p = _dev(t, dtype, shape, name)
    if t is not None and t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return p


def _own_workspace(workspace: torch.Tensor | None, need: int, device):
    """``_call_workspace``; the caller's is on the current device."""
    if workspace is not None:
        _here(workspace, workspace.dtype, workspace.shape, "workspace")
    return _call_workspace(workspace, need, device)


def _exps_shape(rows: int, cols: int):
    return (rows, (cols + LMKAN_CHECKPOINT_BLOCK - 1) // LMKAN_CHECKPOINT_BLOCK)


def lmkan_checkpoint_exps_bytes(rows: int, cols: int) -> int:
    return lib().lmkan_checkpoint_exps_bytes(rows, cols)


def lmkan_checkpoint_rows(x: torch.Tensor, relu: bool = False, stream=None):
    """x [rows][cols] -> its 8-bit checkpoint (codes int8 [rows][cols], exps uint8 [rows][ceil(cols / 32)])."""
    if stream is None:
        done = (_native or _fast()).checkpoint_rows(x, relu)
        if done is not None:
            return done
    if x.dim() != 2 or x.dtype not in _DTYPE_CODE:
        raise ValueError(f"x: expected a matrix of float32, float16 or bfloat16, got {x.dtype} {tuple(x.shape)}")
    rows, cols = x.shape
    xp = _here(x, x.dtype, (rows, cols), "x")
    codes = torch.empty((rows, cols), dtype=torch.int8, device=x.device)
    exps = torch.empty(_exps_shape(rows, cols), dtype=torch.uint8, device=x.device)
    _check(lib().lmkan_checkpoint_rows(rows, cols, _DTYPE_CODE[x.dtype], LMKAN_LINEAR_RELU if relu else 0, xp,
                                       codes.data_ptr(), exps.data_ptr(), _stream(stream)), "lmkan_checkpoint_rows")
    _used_on(stream, codes, exps)
    return codes, exps


def lmkan_restore_rows(codes: torch.Tensor, exps: torch.Tensor, weight: torch.Tensor | None = None,
                       bias: torch.Tensor | None = None, relu: bool = False, dtype: int = LMKAN_F32,
                       y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Rows in ``dtype`` from a checkpoint: f(weight value + bias), f = max(., 0) with ``relu``."""
    if stream is None:
        done = (_native or _fast()).restore_rows(codes, exps, weight, bias, relu, dtype, y)
        if done is not None:
            return done
    if codes.dim() != 2:
        raise ValueError(f"codes: expected a matrix of int8, got {codes.dtype} {tuple(codes.shape)}")
    if dtype not in _TORCH_DTYPE:
        raise ValueError(f"dtype: expected LMKAN_F32, LMKAN_F16 or LMKAN_BF16, got {dtype}")
    rows, cols = codes.shape
    cp = _here(codes, torch.int8, (rows, cols), "codes")
    ep = _here(exps, torch.uint8, _exps_shape(rows, cols), "exps")
    wp = _here(weight, torch.float32, (cols,), "weight")
    bp = _here(bias, torch.float32, (cols,), "bias")
    if y is None:
        y = torch.empty((rows, cols), dtype=_TORCH_DTYPE[dtype], device=codes.device)
    yp = _here(y, _TORCH_DTYPE[dtype], (rows, cols), "y")
    _check(lib().lmkan_restore_rows(rows, cols, dtype, LMKAN_LINEAR_RELU if relu else 0, cp, ep, wp, bp, yp,
                                    _stream(stream)), "lmkan_restore_rows")
    _used_on(stream, y)
    return y


def lmkan_layer_norm(desc: NormDesc, x: torch.Tensor, weight: torch.Tensor | None = None,
                     bias: torch.Tensor | None = None, y: torch.Tensor | None = None, keep: bool = False, stream=None):
    """Returns (y, stats [rows][2], kept): rows normalised over their columns, what the backward call needs of the
    statistics, and with ``keep`` the checkpoint (codes, exps) of the normalised rows before weight and bias, else
    None.  ``y`` may be ``x``."""
    if stream is None:
        done = (_native or _fast()).layer_norm(desc, x, weight, bias, y, keep)
        if done is not None:
            return done
    rows = _rows(x, desc.x_dtype, desc.cols, "x")
    xp = _here(x, _TORCH_DTYPE[desc.x_dtype], (rows, desc.cols), "x")
    wp = _here(weight, torch.float32, (desc.cols,), "weight")
    bp = _here(bias, torch.float32, (desc.cols,), "bias")
    if y is None:
        y = torch.empty((rows, desc.cols), dtype=_TORCH_DTYPE[desc.y_dtype], device=x.device)
    yp = _here(y, _TORCH_DTYPE[desc.y_dtype], (rows, desc.cols), "y")
    stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device)
    codes = torch.empty((rows, desc.cols), dtype=torch.int8, device=x.device) if keep else None
    exps = torch.empty(_exps_shape(rows, desc.cols), dtype=torch.uint8, device=x.device) if keep else None
    _check(lib().lmkan_layer_norm(C.byref(desc.c()), rows, xp, wp, bp, yp, stats.data_ptr(), _ptr(codes), _ptr(exps),
                                  _stream(stream)), "lmkan_layer_norm")
    _used_on(stream, y, stats, codes, exps)
    return y, stats, ((codes, exps) if keep else None)


def lmkan_layer_norm_backward_workspace_bytes(desc: NormDesc, rows: int) -> int:
    return lib().lmkan_layer_norm_backward_workspace_bytes(C.byref(desc.c()), rows)


def lmkan_layer_norm_backward(desc: NormDesc, grad_y: torch.Tensor, stats: torch.Tensor, x: torch.Tensor | None = None,
                              kept=None, weight: torch.Tensor | None = None, need_grad_x: bool = True,
                              need_grad_weight: bool = True, need_grad_bias: bool = True,
                              grad_x: torch.Tensor | None = None, grad_weight: torch.Tensor | None = None,
                              grad_bias: torch.Tensor | None = None, accumulate: bool = False, stream=None,
                              workspace: torch.Tensor | None = None):
    """Returns (grad_x, grad_weight, grad_bias), None for those not needed, from the rows ``x`` of the forward call or
    from the checkpoint ``kept`` that it made (one of them).  With ``accumulate`` the last two are added to the tensors
    given."""
    if (x is None) == (kept is None):
        raise ValueError("the backward call takes the rows x or their checkpoint kept, one of the two")
    if accumulate and ((need_grad_weight and grad_weight is None) or (need_grad_bias and grad_bias is None)):
        raise ValueError("accumulating into grad_weight and grad_bias needs existing tensors")
    codes, exps = kept if kept is not None else (None, None)
    if stream is None:
        done = (_native or _fast()).layer_norm_backward(desc, grad_y, stats, x, codes, exps, weight, need_grad_x,
                                                        need_grad_weight, need_grad_bias, grad_x, grad_weight, grad_bias,
                                                        accumulate, workspace)
        if done is not None:
            return done
    rows, cols, dev = _rows(grad_y, desc.y_dtype, desc.cols, "grad_y"), desc.cols, grad_y.device
    gp = _here(grad_y, _TORCH_DTYPE[desc.y_dtype], (rows, cols), "grad_y")
    sp = _here(stats, torch.float32, (rows, 2), "stats")
    xp = _here(x, _TORCH_DTYPE[desc.x_dtype], (rows, cols), "x")
    cp = _here(codes, torch.int8, (rows, cols), "codes")
    ep = _here(exps, torch.uint8, _exps_shape(rows, cols), "exps")
    wp = _here(weight, torch.float32, (cols,), "weight")
    if need_grad_x and grad_x is None:
        grad_x = torch.empty((rows, cols), dtype=_TORCH_DTYPE[desc.x_dtype], device=dev)
    if need_grad_weight and grad_weight is None:
        grad_weight = torch.empty((cols,), dtype=torch.float32, device=dev)
    if need_grad_bias and grad_bias is None:
        grad_bias = torch.empty((cols,), dtype=torch.float32, device=dev)
    gxp = _here(grad_x, _TORCH_DTYPE[desc.x_dtype], (rows, cols), "grad_x") if need_grad_x else None
    gwp = _here(grad_weight, torch.float32, (cols,), "grad_weight") if need_grad_weight else None
    gbp = _here(grad_bias, torch.float32, (cols,), "grad_bias") if need_grad_bias else None
    need = lmkan_layer_norm_backward_workspace_bytes(desc, rows) if need_grad_weight or need_grad_bias else 0
    ws, wsz = _own_workspace(workspace, need, dev)
    _check(lib().lmkan_layer_norm_backward(C.byref(desc.c(accumulate)), rows, xp, cp, ep, sp, wp, gp, gxp, gwp, gbp,
                                           _ptr(ws), wsz, _stream(stream)), "lmkan_layer_norm_backward")
    _used_on(stream, ws, grad_x, grad_weight, grad_bias)
    return (grad_x if need_grad_x else None, grad_weight if need_grad_weight else None,
            grad_bias if need_grad_bias else None)


def _linear_grad_desc(desc: LinearDesc, accumulate: bool = False) -> _Linear:
    d = desc.c()
    d.flags |= LMKAN_LINEAR_ACCUMULATE if accumulate else 0
    return d


def lmkan_linear_grad_workspace_bytes(desc: LinearDesc, batch: int) -> int:
    return lib().lmkan_linear_grad_workspace_bytes(C.byref(_linear_grad_desc(desc)), batch)


def lmkan_linear_grad(desc: LinearDesc, codes: torch.Tensor, exps: torch.Tensor, grad_y: torch.Tensor,
                      need_grad_bias: bool = True, grad_weight: torch.Tensor | None = None,
                      grad_bias: torch.Tensor | None = None, accumulate: bool = False, stream=None,
                      workspace: torch.Tensor | None = None):
    """Returns (grad_weight [n_out][n_in], grad_bias [n_out] or None), float32, of the linear term whose input is held
    in the checkpoint (codes, exps); ``grad_y`` is in the descriptor's y_dtype.  With ``accumulate`` they are added to the
    tensors given."""
    if accumulate and (grad_weight is None or (need_grad_bias and grad_bias is None)):
        raise ValueError("accumulating into grad_weight and grad_bias needs existing tensors")
    if stream is None:
        done = (_native or _fast()).linear_grad(desc, codes, exps, grad_y, need_grad_bias, grad_weight, grad_bias,
                                                accumulate, workspace)
        if done is not None:
            return done
    batch, dev = _rows(grad_y, desc.y_dtype, desc.n_out, "grad_y"), grad_y.device
    gp = _here(grad_y, _TORCH_DTYPE[desc.y_dtype], (batch, desc.n_out), "grad_y")
    cp = _here(codes, torch.int8, (batch, desc.n_in), "codes")
    ep = _here(exps, torch.uint8, _exps_shape(batch, desc.n_in), "exps")
    if grad_weight is None:
        grad_weight = torch.empty((desc.n_out, desc.n_in), dtype=torch.float32, device=dev)
    if need_grad_bias and grad_bias is None:
        grad_bias = torch.empty((desc.n_out,), dtype=torch.float32, device=dev)
    gwp = _here(grad_weight, torch.float32, (desc.n_out, desc.n_in), "grad_weight")
    gbp = _here(grad_bias, torch.float32, (desc.n_out,), "grad_bias") if need_grad_bias else None
    ws, wsz = _own_workspace(workspace, lmkan_linear_grad_workspace_bytes(desc, batch), dev)
    _check(lib().lmkan_linear_grad(C.byref(_linear_grad_desc(desc, accumulate)), batch, cp, ep, gp, gwp, gbp, _ptr(ws),
                                   wsz, _stream(stream)), "lmkan_linear_grad")
    _used_on(stream, ws, grad_weight, grad_bias)
    return grad_weight, (grad_bias if need_grad_bias else None)


def lmkan_adapters_workspace_bytes(desc: AdapterDesc, batch: int) -> int:
    return lib().lmkan_adapters_workspace_bytes(C.byref(desc.c()), batch)


def lmkan_adapters_add(desc: AdapterDesc, x: torch.Tensor, index: torch.Tensor, a: torch.Tensor, b: torch.Tensor,
                       y: torch.Tensor, scale: torch.Tensor | None = None, stream=None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """y[n] += scale[r] B_r (A_r f(x[n])) in place, r = index[n] (int32); rows whose index is not in [0, count) stay."""
    if stream is None:
        done = (_native or _fast()).adapters_add(desc, x, index, a, b, y, scale, workspace)
        if done is not None:
            return done
    batch = _rows(x, desc.x_dtype, desc.n_in, "x")
    dt = _TORCH_DTYPE[desc.dtype]
    xp = _here(x, _TORCH_DTYPE[desc.x_dtype], (batch, desc.n_in), "x")
    ip = _here(index, torch.int32, (batch,), "index")
    ap = _here(a, dt, desc.a_shape(), "a")
    bp = _here(b, dt, desc.b_shape(), "b")
    yp = _here(y, _TORCH_DTYPE[desc.y_dtype], (batch, desc.n_out), "y")
    sp = _here(scale, torch.float32, (desc.count,), "scale")
    ws, wsz = _own_workspace(workspace, lmkan_adapters_workspace_bytes(desc, batch), x.device)
    _check(lib().lmkan_adapters_add(C.byref(desc.c()), batch, xp, ip, ap, bp, sp, yp, _ptr(ws), wsz, _stream(stream)),
           "lmkan_adapters_add")
    _used_on(stream, ws)
    return y
