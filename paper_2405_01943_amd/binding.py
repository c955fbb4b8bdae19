"""ctypes binding of libdass.so -- argument marshalling only.

Function names follow the C ABI in ``include/dass.h`` (``dass_`` prefix
dropped).  Tensors are torch CUDA tensors; their ``data_ptr()`` and the current
torch stream are handed to the library, which does all the work.  There is no
fallback: if the shared library cannot be loaded the call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libdass.so")

_F32 = torch.float32
DTYPE = {torch.float32: 0, torch.bfloat16: 1}
ACT = {"silu": 0, "gelu_tanh": 1, "gelu_erf": 2, "relu": 3}
LINEAR_ACT = {**ACT, "none": 4}      # of linear and its gradient
AXIS = {"rows": 0, "cols": 1}

EXPORTS = (
    "dass_calib_workspace_bytes", "dass_calib_norms",
    "dass_nm_workspace_bytes", "dass_score_mask_nm",
    "dass_nm_batched_workspace_bytes", "dass_score_mask_nm_batched",
    "dass_unstructured_workspace_bytes", "dass_score_mask_unstructured", "dass_score_mask_unstructured_static",
    "dass_input_norms_workspace_bytes", "dass_input_norms",
    "dass_mlp_forward_workspace_bytes", "dass_mlp_forward", "dass_compress_24", "dass_down_proj_sparse24",
    "dass_expert_sort_workspace_bytes", "dass_expert_sort", "dass_expert_gather", "dass_expert_combine",
    "dass_expert_combine_backward",
    "dass_linear_workspace_bytes", "dass_linear", "dass_linear_backward_workspace_bytes", "dass_linear_backward",
    "dass_status_string", "dass_last_error_string", "dass_version",
)


class NmTask(ctypes.Structure):
    """dass_nm_task of include/dass.h."""
    _fields_ = [("W", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("norms", ctypes.c_void_p), ("norm_axis", ctypes.c_int),
                ("group_axis", ctypes.c_int), ("alpha", ctypes.c_double), ("mask_out", ctypes.c_void_p)]


class LinearTask(ctypes.Structure):
    """dass_linear_task of include/dass.h."""
    _fields_ = [("X", ctypes.c_void_p), ("T", ctypes.c_int64), ("ldx", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("expert_stride", ctypes.c_int64),
                ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
                ("offsets", ctypes.c_void_p), ("n_experts", ctypes.c_int64), ("bias", ctypes.c_void_p),
                ("mul", ctypes.c_void_p), ("ldm", ctypes.c_int64), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("pre_out", ctypes.c_void_p), ("ldp", ctypes.c_int64), ("out", ctypes.c_void_p), ("ldo", ctypes.c_int64),
                ("dt", ctypes.c_int), ("act", ctypes.c_int)]


class LinearGradTask(ctypes.Structure):
    """dass_linear_grad_task of include/dass.h."""
    _fields_ = [("dout", ctypes.c_void_p), ("T", ctypes.c_int64), ("ldg", ctypes.c_int64),
                ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("expert_stride", ctypes.c_int64),
                ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
                ("offsets", ctypes.c_void_p), ("n_experts", ctypes.c_int64),
                ("pre", ctypes.c_void_p), ("ldp", ctypes.c_int64), ("mul", ctypes.c_void_p), ("ldm", ctypes.c_int64),
                ("dX", ctypes.c_void_p), ("lddx", ctypes.c_int64),
                ("dW", ctypes.c_void_p), ("lddw", ctypes.c_int64), ("dw_stride", ctypes.c_int64),
                ("dbias", ctypes.c_void_p), ("dmul", ctypes.c_void_p), ("lddm", ctypes.c_int64),
                ("dt", ctypes.c_int), ("act", ctypes.c_int)]


class DassError(RuntimeError):
    """A libdass call returned a status other than DASS_OK."""

    def __init__(self, status: int, name: str, detail: str):
        super().__init__(f"{name}: {detail}" if detail else name)
        self.status = status
        self.status_name = name


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libdass.so.  A library that is missing, or was built from other sources than the
    present ones (compared by content hash), is rebuilt with hipcc first; if that fails the
    call raises: a binary older than its sources is never used."""
    global _lib
    if _lib is not None:
        return _lib
    from . import build as _build
    if _build.is_stale():
        _build.build()
    lib = ctypes.CDLL(_LIB_PATH)
    i64, sz, vp, ci, dbl = (ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int,
                            ctypes.c_double)
    lib.dass_calib_workspace_bytes.restype = sz
    lib.dass_calib_workspace_bytes.argtypes = [i64, i64, i64, ci]
    lib.dass_calib_norms.restype = ci
    lib.dass_calib_norms.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, ci, ci, vp, ci, vp,
                                     vp, sz, vp]
    lib.dass_nm_workspace_bytes.restype = sz
    lib.dass_nm_workspace_bytes.argtypes = [i64, i64, ci]
    lib.dass_score_mask_nm.restype = ci
    lib.dass_score_mask_nm.argtypes = [vp, i64, i64, i64, ci, vp, ci, ci, dbl, ci, ci, vp,
                                       vp, sz, vp]
    lib.dass_nm_batched_workspace_bytes.restype = sz
    lib.dass_nm_batched_workspace_bytes.argtypes = [ctypes.POINTER(NmTask), i64]
    lib.dass_score_mask_nm_batched.restype = ci
    lib.dass_score_mask_nm_batched.argtypes = [ctypes.POINTER(NmTask), i64, ci, ci, ci, vp, sz, vp]
    lib.dass_unstructured_workspace_bytes.restype = sz
    lib.dass_unstructured_workspace_bytes.argtypes = [i64, i64, ci, ci, ci]
    lib.dass_score_mask_unstructured.restype = ci
    lib.dass_score_mask_unstructured.argtypes = [vp, i64, i64, i64, ci, vp, ci, ci, dbl, i64, vp,
                                                 vp, sz, vp]
    lib.dass_score_mask_unstructured_static.restype = ci
    lib.dass_score_mask_unstructured_static.argtypes = [vp, i64, i64, i64, ci, vp, ci, ci, dbl, i64, vp, vp]
    lib.dass_input_norms_workspace_bytes.restype = sz
    lib.dass_input_norms_workspace_bytes.argtypes = [i64, i64]
    lib.dass_input_norms.restype = ci
    lib.dass_input_norms.argtypes = [vp, i64, i64, i64, ci, vp, ci, vp, vp, sz, vp]
    lib.dass_mlp_forward_workspace_bytes.restype = sz
    lib.dass_mlp_forward_workspace_bytes.argtypes = [i64, i64, i64, ci]
    lib.dass_mlp_forward.restype = ci
    lib.dass_mlp_forward.argtypes = [vp, i64, i64, vp, vp, i64, vp, i64, i64, i64, ci, ci, vp, i64,
                                     vp, sz, vp]
    lib.dass_compress_24.restype = ci
    lib.dass_compress_24.argtypes = [vp, i64, i64, i64, ci, ci, vp, i64, vp, i64, vp, vp]
    lib.dass_down_proj_sparse24.restype = ci
    lib.dass_down_proj_sparse24.argtypes = [vp, i64, i64, vp, i64, vp, i64, i64, i64, ci, vp, i64, vp]
    lib.dass_expert_sort_workspace_bytes.restype = sz
    lib.dass_expert_sort_workspace_bytes.argtypes = [i64, i64, i64]
    lib.dass_expert_sort.restype = ci
    lib.dass_expert_sort.argtypes = [vp, ci, i64, i64, i64, vp, vp, vp, vp, sz, vp]
    lib.dass_expert_gather.restype = ci
    lib.dass_expert_gather.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp, i64, vp]
    lib.dass_expert_combine.restype = ci
    lib.dass_expert_combine.argtypes = [vp, i64, vp, i64, i64, vp, vp, i64, i64, ci, vp, i64, vp]
    lib.dass_expert_combine_backward.restype = ci
    lib.dass_expert_combine_backward.argtypes = [vp, i64, vp, i64, vp, i64, i64, vp, i64, ci, vp, i64, vp, vp]
    lib.dass_linear.restype = ci
    lib.dass_linear.argtypes = [ctypes.POINTER(LinearTask), vp, sz, vp]
    lib.dass_linear_workspace_bytes.restype = sz
    lib.dass_linear_workspace_bytes.argtypes = [i64, i64, i64, ci, i64]
    lib.dass_linear_backward_workspace_bytes.restype = sz
    lib.dass_linear_backward_workspace_bytes.argtypes = [i64, i64, i64, ci, i64]
    lib.dass_linear_backward.restype = ci
    lib.dass_linear_backward.argtypes = [ctypes.POINTER(LinearGradTask), vp, sz, vp]
    lib.dass_status_string.restype = ctypes.c_char_p
    lib.dass_status_string.argtypes = [ci]
    lib.dass_last_error_string.restype = ctypes.c_char_p
    lib.dass_last_error_string.argtypes = []
    lib.dass_version.restype = ci
    lib.dass_version.argtypes = []
    _lib = lib
    return lib


def version() -> int:
    return int(load_library().dass_version())


def _check(status: int) -> None:
    if status != 0:
        lib = load_library()
        raise DassError(status, lib.dass_status_string(status).decode(),
                        lib.dass_last_error_string().decode())


# The smallest calls are over on the GPU before the host has made the next one, so the wrappers below ask a tensor
# for as little as the checks need, and for each thing once: a whole shape and stride, no size query for a workspace
# that is there, addresses as plain integers (ctypes converts them).  dass_input_norms of 2048 x 4096, this side of the
# library call, on one host: 5.7 -> 4.2 us; dass_calib_norms 10.8 -> 6.8, dass_score_mask_unstructured 7.3 -> 4.8.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _nbytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.nbytes


# The raw handle of the current stream: building a torch.cuda.Stream takes 2.9 us a call, this 0.3.  It is
# none of torch's public functions, so that a torch without it goes by the public one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _matrix(t: torch.Tensor, name: str):
    stride = t.stride()
    if len(stride) != 2 or stride[1] != 1 or t.dtype not in DTYPE:
        raise TypeError(f"{name}: need a 2-D f32/bf16 tensor with unit column stride")
    rows, cols = t.shape
    return rows, cols, stride[0] if rows > 1 else max(stride[0], cols)


def _scratch(nbytes: int, device, stream=None) -> torch.Tensor:
    """A workspace for a caller that passed none.  This is a convenience of the binding (the
    library itself never allocates): the block comes from torch's caching allocator and is
    released when the call returns, so it is taken from the blocks of the stream the kernels run
    on: one of another stream's could still be in use by the kernels queued there.  A caller
    that wants no allocation on its path passes ``workspace`` itself."""
    # (the current stream given by name takes its blocks as they come: 7.3 us through the context, 1.5 without)
    if stream is None or (_raw_stream is not None and stream.cuda_stream == _raw_stream(stream.device_index)):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)


# ------------------------------------------------------------------ stage 1 --
def calib_workspace_bytes(T: int, d: int, d_int: int, dtype: torch.dtype) -> int:
    return int(load_library().dass_calib_workspace_bytes(T, d, d_int, DTYPE[dtype]))


def calib_norms(X: torch.Tensor, Wgate: torch.Tensor, Wup: torch.Tensor, act: str,
                sumsq: torch.Tensor, accumulate: bool = False,
                norms_out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_calib_norms: sumsq (+)= sum_t y[t, :]^2 with y = act(X Wgate^T) * (X Wup^T)."""
    lib = load_library()
    T, d, ldx = _matrix(X, "X")
    d_int, dg, ldw = _matrix(Wgate, "Wgate")
    d_int_u, du, ldw_u = _matrix(Wup, "Wup")
    if (d_int_u, du, ldw_u) != (d_int, dg, ldw) or dg != d or not (X.dtype == Wgate.dtype == Wup.dtype):
        raise ValueError("X, Wgate, Wup disagree in shape, stride or dtype")
    if sumsq.dtype != _F32 or sumsq.numel() != d_int or not sumsq.is_contiguous():
        raise TypeError("sumsq: need contiguous float32[d_int]")
    if norms_out is not None and (norms_out.dtype != _F32 or norms_out.numel() != d_int
                                  or not norms_out.is_contiguous()):
        raise TypeError("norms_out: need contiguous float32[d_int]")
    if workspace is None:
        need = int(lib.dass_calib_workspace_bytes(T, d, d_int, DTYPE[X.dtype]))
        if need > 0:
            workspace = _scratch(need, X.device, stream)
    ws_bytes = _nbytes(workspace)
    status = lib.dass_calib_norms(_ptr(X), T, ldx, _ptr(Wgate), _ptr(Wup), ldw, d, d_int,
                                  DTYPE[X.dtype], ACT[act], _ptr(sumsq), 1 if accumulate else 0,
                                  _ptr(norms_out), _ptr(workspace), ws_bytes, _stream(stream))
    if status:
        _check(status)


def input_norms_workspace_bytes(T: int, d: int) -> int:
    return int(load_library().dass_input_norms_workspace_bytes(T, d))


def input_norms(X: torch.Tensor, sumsq: torch.Tensor, accumulate: bool = False,
                norms_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream=None) -> None:
    """dass_input_norms: sumsq[j] (+)= sum_t X[t, j]^2 (the Wanda metric's input norms, Eq. 1)."""
    lib = load_library()
    T, d, ldx = _matrix(X, "X")
    for name, t in (("sumsq", sumsq), ("norms_out", norms_out)):
        if t is not None and (t.dtype != _F32 or t.numel() != d or not t.is_contiguous()):
            raise TypeError(f"{name}: need contiguous float32[d]")
    if workspace is None:
        workspace = _scratch(int(lib.dass_input_norms_workspace_bytes(T, d)), X.device, stream)
    ws_bytes = _nbytes(workspace)
    status = lib.dass_input_norms(_ptr(X), T, ldx, d, DTYPE[X.dtype], _ptr(sumsq), 1 if accumulate else 0,
                                  _ptr(norms_out), _ptr(workspace), ws_bytes, _stream(stream))
    if status:
        _check(status)


def mlp_forward_workspace_bytes(T: int, d: int, d_int: int, dtype=torch.bfloat16) -> int:
    return int(load_library().dass_mlp_forward_workspace_bytes(T, d, d_int, DTYPE[dtype]))


def mlp_forward(X: torch.Tensor, Wgate: torch.Tensor, Wup: torch.Tensor, Wdown: Optional[torch.Tensor], act: str,
                out: Optional[torch.Tensor], workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_mlp_forward: out = (act(X Wgate^T) * (X Wup^T)) Wdown^T (Eq. 2 then Eq. 3).

    With ``Wdown=None`` only Eq. 2 runs: y is left in ``workspace`` (required then) as [T, d_int].
    """
    lib = load_library()
    T, d, ldx = _matrix(X, "X")
    d_int, d2, ldw = _matrix(Wgate, "Wgate")
    if _matrix(Wup, "Wup") != (d_int, d2, ldw) or d2 != d:
        raise ValueError("Wgate and Wup must be [d_int, d] with one leading dimension")
    ldd = ldo = 0
    if Wdown is None:
        if workspace is None:
            raise ValueError("Wdown=None leaves y in the workspace: pass one")
        out = None
        dtypes = {X.dtype, Wgate.dtype, Wup.dtype}
    else:
        dd, di, ldd = _matrix(Wdown, "Wdown")
        To, do, ldo = _matrix(out, "out")
        if (dd, di) != (d, d_int) or (To, do) != (T, d):
            raise ValueError("Wdown must be [d, d_int] and out [T, d]")
        dtypes = {X.dtype, Wgate.dtype, Wup.dtype, Wdown.dtype, out.dtype}
    if len(dtypes) != 1:
        raise TypeError("X, the weights and out must share one dtype")
    if workspace is None:
        workspace = _scratch(int(lib.dass_mlp_forward_workspace_bytes(T, d, d_int, DTYPE[X.dtype])), X.device, stream)
    ws_bytes = _nbytes(workspace)
    status = lib.dass_mlp_forward(_ptr(X), T, ldx, _ptr(Wgate), _ptr(Wup), ldw, _ptr(Wdown), ldd, d, d_int,
                                  DTYPE[X.dtype], ACT[act], _ptr(out), ldo, _ptr(workspace), ws_bytes,
                                  _stream(stream))
    if status:
        _check(status)


# ------------------------------------------------------------------ stage 2 --
def nm_workspace_bytes(rows: int, cols: int, norm_axis: str) -> int:
    return int(load_library().dass_nm_workspace_bytes(rows, cols, AXIS[norm_axis]))


def score_mask_nm(W: torch.Tensor, norms: torch.Tensor, norm_axis: str, group_axis: str,
                  alpha: float, n_keep: int, m: int, mask_out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_score_mask_nm: in-place N:M pruning of W by |W| * norms^alpha."""
    lib = load_library()
    rows, cols, ld = _matrix(W, "W")
    if norms.dtype != _F32 or not norms.is_contiguous():
        raise TypeError("norms: need contiguous float32")
    if norms.numel() != (rows if norm_axis == "rows" else cols):
        raise ValueError("norms length does not match norm_axis")
    if mask_out is not None and (mask_out.dtype != torch.uint8 or not mask_out.is_contiguous()
                                 or mask_out.numel() != rows * (cols // 8)):
        raise TypeError("mask_out: need contiguous uint8[rows * cols / 8]")
    if workspace is None:
        workspace = _scratch(int(lib.dass_nm_workspace_bytes(rows, cols, AXIS[norm_axis])), W.device, stream)
    ws_bytes = _nbytes(workspace)
    status = lib.dass_score_mask_nm(_ptr(W), rows, cols, ld, DTYPE[W.dtype], _ptr(norms),
                                    AXIS[norm_axis], AXIS[group_axis], float(alpha), int(n_keep),
                                    int(m), _ptr(mask_out), _ptr(workspace), ws_bytes,
                                    _stream(stream))
    if status:
        _check(status)


def _nm_task_array(tasks):
    """tasks: sequence of (W, norms, norm_axis, group_axis, alpha[, mask_out]) -> (NmTask array, dtype, device)."""
    arr = (NmTask * max(len(tasks), 1))()
    dtype = device = None
    for i, t in enumerate(tasks):
        W, norms, norm_axis, group_axis, alpha = t[:5]
        mask_out = t[5] if len(t) > 5 else None
        rows, cols, ld = _matrix(W, f"tasks[{i}].W")
        if dtype is None:
            dtype, device = W.dtype, W.device
        elif W.dtype != dtype:
            raise TypeError("all matrices of a batched call must share one dtype")
        if norms.dtype != _F32 or not norms.is_contiguous():
            raise TypeError(f"tasks[{i}].norms: need contiguous float32")
        if norms.numel() != (rows if norm_axis == "rows" else cols):
            raise ValueError(f"tasks[{i}]: norms length does not match norm_axis")
        if mask_out is not None and (mask_out.dtype != torch.uint8 or not mask_out.is_contiguous()
                                     or mask_out.numel() != rows * (cols // 8)):
            raise TypeError(f"tasks[{i}].mask_out: need contiguous uint8[rows * cols / 8]")
        arr[i] = NmTask(W.data_ptr(), rows, cols, ld, norms.data_ptr(), AXIS[norm_axis], AXIS[group_axis],
                        float(alpha), None if mask_out is None else mask_out.data_ptr())
    return arr, dtype, device


def nm_batched_workspace_bytes(tasks) -> int:
    arr, _, _ = _nm_task_array(tasks)
    return int(load_library().dass_nm_batched_workspace_bytes(arr, len(tasks)))


def score_mask_nm_batched(tasks, n_keep: int, m: int, workspace: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    """dass_score_mask_nm_batched: score_mask_nm over many matrices, equal ones sharing launches.

    tasks: sequence of (W, norms, norm_axis, group_axis, alpha[, mask_out]).
    """
    lib = load_library()
    if len(tasks) == 0:
        return
    arr, dtype, device = _nm_task_array(tasks)
    if workspace is None:
        workspace = _scratch(int(lib.dass_nm_batched_workspace_bytes(arr, len(tasks))), device, stream)
    ws_bytes = _nbytes(workspace)
    status = lib.dass_score_mask_nm_batched(arr, len(tasks), DTYPE[dtype], int(n_keep), int(m),
                                            _ptr(workspace), ws_bytes, _stream(stream))
    if status:
        _check(status)


def unstructured_workspace_bytes(rows: int, cols: int, dtype: torch.dtype, norm_axis: str,
                                 group_axis: str) -> int:
    return int(load_library().dass_unstructured_workspace_bytes(
        rows, cols, DTYPE[dtype], AXIS[norm_axis], AXIS[group_axis]))


def score_mask_unstructured(W: torch.Tensor, norms: torch.Tensor, norm_axis: str, group_axis: str,
                            alpha: float, n_prune: int, mask_out: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_score_mask_unstructured: prune the n_prune lowest scores of every line."""
    lib = load_library()
    rows, cols, ld = _matrix(W, "W")
    if norms.dtype != _F32 or not norms.is_contiguous():
        raise TypeError("norms: need contiguous float32")
    if norms.numel() != (rows if norm_axis == "rows" else cols):
        raise ValueError("norms length does not match norm_axis")
    if mask_out is not None and (mask_out.dtype != torch.uint8 or not mask_out.is_contiguous()
                                 or mask_out.numel() != rows * (cols // 8)):
        raise TypeError("mask_out: need contiguous uint8[rows * cols / 8]")
    if workspace is None:
        workspace = _scratch(int(lib.dass_unstructured_workspace_bytes(rows, cols, DTYPE[W.dtype], AXIS[norm_axis],
                                                                       AXIS[group_axis])), W.device, stream)
    ws_bytes = _nbytes(workspace)
    status = lib.dass_score_mask_unstructured(_ptr(W), rows, cols, ld, DTYPE[W.dtype], _ptr(norms),
                                              AXIS[norm_axis], AXIS[group_axis], float(alpha),
                                              int(n_prune), _ptr(mask_out), _ptr(workspace), ws_bytes,
                                              _stream(stream))
    if status:
        _check(status)


def score_mask_unstructured_static(W: torch.Tensor, norms: torch.Tensor, norm_axis: str, group_axis: str,
                                   alpha: float, n_prune: int, mask_out: Optional[torch.Tensor] = None,
                                   stream=None) -> None:
    """dass_score_mask_unstructured_static: the same selection with the library's own device scratch."""
    lib = load_library()
    rows, cols, ld = _matrix(W, "W")
    if norms.dtype != _F32 or not norms.is_contiguous():
        raise TypeError("norms: need contiguous float32")
    if norms.numel() != (rows if norm_axis == "rows" else cols):
        raise ValueError("norms length does not match norm_axis")
    if mask_out is not None and (mask_out.dtype != torch.uint8 or not mask_out.is_contiguous()
                                 or mask_out.numel() != rows * (cols // 8)):
        raise TypeError("mask_out: need contiguous uint8[rows * cols / 8]")
    status = lib.dass_score_mask_unstructured_static(_ptr(W), rows, cols, ld, DTYPE[W.dtype], _ptr(norms),
                                                     AXIS[norm_axis], AXIS[group_axis], float(alpha),
                                                     int(n_prune), _ptr(mask_out), _stream(stream))
    if status:
        _check(status)


def compress_24(W: torch.Tensor, group_axis: str, values_out: torch.Tensor, meta_out: torch.Tensor,
                surplus_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_compress_24: kept values and 2-bit position codes of a 2:4 sparse matrix."""
    lib = load_library()
    rows, cols, ld = _matrix(W, "W")
    vr, vc, ldv = _matrix(values_out, "values_out")
    if values_out.dtype != W.dtype or (vr, vc) != ((rows // 2, cols) if group_axis == "rows" else (rows, cols // 2)):
        raise TypeError("values_out: need W's dtype and [rows / 2, cols] (rows) or [rows, cols / 2] (cols)")
    want = (rows // 4, cols // 2) if group_axis == "rows" else (rows, cols // 8)
    if meta_out.dtype != torch.uint8 or meta_out.dim() != 2 or tuple(meta_out.shape) != want or meta_out.stride(1) != 1:
        raise TypeError(f"meta_out: need uint8 {want}")
    ldm = meta_out.stride(0) if meta_out.shape[0] > 1 else max(meta_out.stride(0), meta_out.shape[1])
    if surplus_out is not None and (surplus_out.dtype != torch.int64 or surplus_out.numel() != 1):
        raise TypeError("surplus_out: need one int64")
    status = lib.dass_compress_24(_ptr(W), rows, cols, ld, DTYPE[W.dtype], AXIS[group_axis], _ptr(values_out), ldv,
                                  _ptr(meta_out), ldm, _ptr(surplus_out), _stream(stream))
    if status:
        _check(status)


def down_proj_sparse24(Y: torch.Tensor, values: torch.Tensor, meta: torch.Tensor, out: torch.Tensor,
                       stream=None) -> None:
    """dass_down_proj_sparse24: out = Y Wdown^T from the 2:4 compressed Down-Proj (sparse MFMA)."""
    lib = load_library()
    T, d_int, ldy = _matrix(Y, "Y")
    d, half, ldv = _matrix(values, "values")
    To, do, ldo = _matrix(out, "out")
    if half * 2 != d_int or (To, do) != (T, d) or values.dtype != Y.dtype or out.dtype != Y.dtype:
        raise ValueError("need values [d, d_int / 2] and out [T, d] in Y's dtype")
    if meta.dtype != torch.uint8 or meta.dim() != 2 or tuple(meta.shape) != (d, d_int // 8) or meta.stride(1) != 1:
        raise TypeError("meta: need uint8 [d, d_int / 8]")
    ldm = meta.stride(0) if meta.shape[0] > 1 else max(meta.stride(0), meta.shape[1])
    status = lib.dass_down_proj_sparse24(_ptr(Y), T, ldy, _ptr(values), ldv, _ptr(meta), ldm, d, d_int,
                                         DTYPE[Y.dtype], _ptr(out), ldo, _stream(stream))
    if status:
        _check(status)



# ------------------------------------------------- a mixture of GLU experts --
_I32 = torch.int32
_NEEDS_WORKSPACE = 6     # DASS_ERR_WORKSPACE


def _on_device(stream, *tensors) -> int:
    """The handle of the stream that a call goes to; every tensor must be on its GPU, and that the current one."""
    device = None
    for t in tensors:
        if t is not None:
            where = t.get_device()
            if where != device:
                if device is not None or where < 0:
                    raise ValueError("every tensor must be on the GPU" if where < 0 else f"tensors on GPUs {device} and {where}")
                device = where
    current = torch.cuda.current_device()
    if stream is not None and stream.device_index != device:
        raise ValueError(f"the tensors are on GPU {device}, the stream is of GPU {stream.device_index}")
    if current != device:       # the library's launches reserve LDS on the current GPU
        raise ValueError(f"the tensors are on GPU {device}, the current one is GPU {current}")
    return _raw_stream(current) if stream is None and _raw_stream is not None else _stream(stream)


def _integers(t: torch.Tensor, name: str, shape) -> None:
    if t.dtype != _I32 or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{name}: need contiguous int32 {tuple(shape)}")


def expert_sort_workspace_bytes(T: int, k: int, n_experts: int) -> int:
    return int(load_library().dass_expert_sort_workspace_bytes(T, k, n_experts))


def expert_sort(experts: torch.Tensor, n_experts: int, offsets: torch.Tensor, order: torch.Tensor, place: torch.Tensor,
                workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_expert_sort: the pairs of experts[T, k] (int32 or int64) numbered by expert.

    offsets int32[n_experts + 1], order int32[T * k], place int32[T, k].
    """
    lib = load_library()
    if experts.dtype not in (_I32, torch.int64) or experts.dim() != 2 or not experts.is_contiguous():
        raise TypeError("experts: need contiguous int32 or int64 [T, k]")
    T, k = experts.shape
    _integers(offsets, "offsets", (n_experts + 1,))
    _integers(order, "order", (T * k,))
    _integers(place, "place", (T, k))
    handle = _on_device(stream, experts, offsets, order, place, workspace)
    args = _ptr(experts), experts.element_size(), T, k, n_experts, _ptr(offsets), _ptr(order), _ptr(place)
    status = lib.dass_expert_sort(*args, _ptr(workspace), _nbytes(workspace), handle)
    if status == _NEEDS_WORKSPACE and workspace is None:    # few pairs need none, so they are not asked first
        workspace = _scratch(int(lib.dass_expert_sort_workspace_bytes(T, k, n_experts)), experts.device, stream)
        status = lib.dass_expert_sort(*args, _ptr(workspace), _nbytes(workspace), handle)
    if status:
        _check(status)


def _rows_of_pairs(t: torch.Tensor, name: str, pairs: int, d: int, dtype) -> int:
    rows, width, ld = _matrix(t, name)
    if (rows, width) != (pairs, d) or t.dtype != dtype:
        raise ValueError(f"{name}: need [{pairs}, {d}] in the dtype of the other rows")
    return ld


def expert_gather(X: torch.Tensor, place: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """dass_expert_gather: out[place[t, j]] = X[t]; place int32[T, k], out [T * k, d]."""
    lib = load_library()
    T, d, ldx = _matrix(X, "X")
    k = place.shape[-1]
    _integers(place, "place", (T, k))
    ldo = _rows_of_pairs(out, "out", T * k, d, X.dtype)
    handle = _on_device(stream, X, place, out)
    status = lib.dass_expert_gather(_ptr(X), T, ldx, d, DTYPE[X.dtype], _ptr(place), k, _ptr(out), ldo, handle)
    if status:
        _check(status)


def expert_combine(Y: torch.Tensor, place: torch.Tensor, out: torch.Tensor, weights: Optional[torch.Tensor] = None,
                   residual: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_expert_combine: out[t] = residual[t] + sum_j weights[t, j] Y[place[t, j]].

    Without weights and residual this is the gradient of expert_gather.
    """
    lib = load_library()
    T, d, ldo = _matrix(out, "out")
    k = place.shape[-1]
    _integers(place, "place", (T, k))
    ldy = _rows_of_pairs(Y, "Y", T * k, d, out.dtype)
    ldr = 0 if residual is None else _rows_of_pairs(residual, "residual", T, d, out.dtype)
    if weights is not None and (weights.dtype != _F32 or weights.shape != place.shape or not weights.is_contiguous()):
        raise TypeError("weights: need contiguous float32 [T, k]")
    handle = _on_device(stream, Y, place, out, weights, residual)
    status = lib.dass_expert_combine(_ptr(Y), ldy, _ptr(place), T, k, _ptr(weights), _ptr(residual), ldr, d, DTYPE[out.dtype],
                                     _ptr(out), ldo, handle)
    if status:
        _check(status)


def expert_combine_backward(dout: torch.Tensor, Y: torch.Tensor, place: torch.Tensor, weights: torch.Tensor, dY: torch.Tensor,
                            dweights: torch.Tensor, stream=None) -> None:
    """dass_expert_combine_backward: dY[place[t, j]] = weights[t, j] dout[t], dweights[t, j] = dout[t] . Y[place[t, j]]."""
    lib = load_library()
    T, d, ldg = _matrix(dout, "dout")
    k = place.shape[-1]
    _integers(place, "place", (T, k))
    ldy = _rows_of_pairs(Y, "Y", T * k, d, dout.dtype)
    lddy = _rows_of_pairs(dY, "dY", T * k, d, dout.dtype)
    for name, t in (("weights", weights), ("dweights", dweights)):
        if t.dtype != _F32 or t.shape != place.shape or not t.is_contiguous():
            raise TypeError(f"{name}: need contiguous float32 [T, k]")
    handle = _on_device(stream, dout, Y, place, weights, dY, dweights)
    status = lib.dass_expert_combine_backward(_ptr(dout), ldg, _ptr(Y), ldy, _ptr(place), T, k, _ptr(weights), d,
                                              DTYPE[dout.dtype], _ptr(dY), lddy, _ptr(dweights), handle)
    if status:
        _check(status)


def _weights(W: torch.Tensor, name: str, n_experts: int, dtype):
    """[d_out, d_in], or [n_experts, d_out, d_in] with offsets -> (d_out, d_in, row stride, expert stride)."""
    stride = W.stride()
    if len(stride) != (3 if n_experts else 2) or stride[-1] != 1 or W.dtype != dtype or (n_experts and W.shape[0] != n_experts):
        raise TypeError(f"{name}: need {f'[{n_experts}, d_out, d_in]' if n_experts else '[d_out, d_in]'} with unit column "
                        "stride in the dtype of X")
    d_out, d_in = W.shape[-2:]
    ld = stride[-2] if d_out > 1 else max(stride[-2], d_in)
    return d_out, d_in, ld, stride[0] if n_experts > 1 else d_out * ld


def _like(t: Optional[torch.Tensor], name: str, shape, dtype) -> int:
    """The row stride of an optional matrix of the given shape."""
    if t is None:
        return 0
    rows, cols, ld = _matrix(t, name)
    if (rows, cols) != shape or t.dtype != dtype:
        raise ValueError(f"{name}: need [{shape[0]}, {shape[1]}] in the dtype of X")
    return ld


def _expert_count(offsets: Optional[torch.Tensor]) -> int:
    """0 without offsets."""
    if offsets is None:
        return 0
    if offsets.dtype != _I32 or offsets.dim() != 1 or offsets.numel() < 2 or not offsets.is_contiguous():
        raise TypeError("offsets: need contiguous int32 [n_experts + 1]")
    return offsets.numel() - 1


def _bias(t: Optional[torch.Tensor], name: str, n_experts: int, d_out: int, dtype) -> None:
    if t is not None and (t.dtype != dtype or tuple(t.shape) != ((n_experts, d_out) if n_experts else (d_out,))
                          or not t.is_contiguous()):
        raise TypeError(f"{name}: need contiguous {'[n_experts, d_out]' if n_experts else '[d_out]'} in the dtype of X")


def linear_workspace_bytes(T: int, d_in: int, d_out: int, dtype: torch.dtype, n_experts: int = 1) -> int:
    return int(load_library().dass_linear_workspace_bytes(T, d_in, d_out, DTYPE[dtype], n_experts))


def linear(X: torch.Tensor, W: torch.Tensor, out: torch.Tensor, act: str = "none", bias: Optional[torch.Tensor] = None,
           mul: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
           pre_out: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_linear: out = act(X W^T + bias) * mul + residual.

    Dense: W [d_out, d_in], bias [d_out].  By expert: offsets int32[n_experts + 1] (as expert_sort leaves
    it), W [n_experts, d_out, d_in], bias [n_experts, d_out]; row t takes its expert's.  pre_out receives
    X W^T + bias for the gradient.
    """
    lib = load_library()
    T, d, ldx = _matrix(X, "X")
    E, dt, code = _expert_count(offsets), X.dtype, LINEAR_ACT[act]
    d_out, d_in, ldw, per_expert = _weights(W, "W", E, dt)
    if d_in != d:
        raise ValueError("W: rows must be as long as those of X")
    shape = (T, d_out)
    ldm, ldr = _like(mul, "mul", shape, dt), _like(residual, "residual", shape, dt)
    ldp, ldo = _like(pre_out, "pre_out", shape, dt), _like(out, "out", shape, dt)
    _bias(bias, "bias", E, d_out, dt)
    handle = _on_device(stream, X, W, out, bias, mul, residual, pre_out, offsets, workspace)
    task = LinearTask(_ptr(X), T, ldx, _ptr(W), ldw, per_expert, d_in, d_out, _ptr(offsets), max(E, 1), _ptr(bias), _ptr(mul),
                      ldm, _ptr(residual), ldr, _ptr(pre_out), ldp, _ptr(out), ldo, DTYPE[dt], code)
    status = lib.dass_linear(ctypes.byref(task), _ptr(workspace), _nbytes(workspace), handle)
    if status == _NEEDS_WORKSPACE and workspace is None:    # most calls need none, so they are not asked first
        workspace = _scratch(int(lib.dass_linear_workspace_bytes(T, d_in, d_out, DTYPE[dt], max(E, 1))), X.device, stream)
        status = lib.dass_linear(ctypes.byref(task), _ptr(workspace), _nbytes(workspace), handle)
    if status:
        _check(status)


def linear_backward_workspace_bytes(T: int, d_in: int, d_out: int, dtype: torch.dtype, n_experts: int = 1) -> int:
    return int(load_library().dass_linear_backward_workspace_bytes(T, d_in, d_out, DTYPE[dtype], n_experts))


def linear_backward(dout: torch.Tensor, X: Optional[torch.Tensor], W: torch.Tensor, act: str = "none",
                    pre: Optional[torch.Tensor] = None, mul: Optional[torch.Tensor] = None,
                    dX: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None,
                    dbias: Optional[torch.Tensor] = None, dmul: Optional[torch.Tensor] = None,
                    offsets: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dass_linear_backward: the gradients of linear that are given a tensor to go to.

    pre is linear's pre_out (not needed for act "none" unless dmul is asked for), X is needed for dW alone.
    """
    lib = load_library()
    T, d_out, ldg = _matrix(dout, "dout")
    E, dt, code = _expert_count(offsets), dout.dtype, LINEAR_ACT[act]
    do, d_in, ldw, per_expert = _weights(W, "W", E, dt)
    if do != d_out:
        raise ValueError("dout: rows must be as long as W has rows")
    lddw = dw_per = 0
    if dW is not None:
        if tuple(dW.shape) != tuple(W.shape):
            raise ValueError("dW: need the shape of W")
        _, _, lddw, dw_per = _weights(dW, "dW", E, dt)
    wide, narrow = (T, d_out), (T, d_in)
    ldx, lddx = _like(X, "X", narrow, dt), _like(dX, "dX", narrow, dt)
    ldp, ldm, lddm = _like(pre, "pre", wide, dt), _like(mul, "mul", wide, dt), _like(dmul, "dmul", wide, dt)
    _bias(dbias, "dbias", E, d_out, dt)
    handle = _on_device(stream, dout, X, W, pre, mul, dX, dW, dbias, dmul, offsets, workspace)
    if workspace is None:
        need = int(lib.dass_linear_backward_workspace_bytes(T, d_in, d_out, DTYPE[dt], max(E, 1)))
        workspace = _scratch(need, dout.device, stream)
    task = LinearGradTask(_ptr(dout), T, ldg, _ptr(X), ldx, _ptr(W), ldw, per_expert, d_in, d_out, _ptr(offsets), max(E, 1),
                          _ptr(pre), ldp, _ptr(mul), ldm, _ptr(dX), lddx, _ptr(dW), lddw, dw_per, _ptr(dbias), _ptr(dmul), lddm,
                          DTYPE[dt], code)
    status = lib.dass_linear_backward(ctypes.byref(task), _ptr(workspace), _nbytes(workspace), handle)
    if status:
        _check(status)
