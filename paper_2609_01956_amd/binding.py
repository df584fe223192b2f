"""Python binding of the C ABI in include/kan.h (ctypes).

Argument marshalling only: every step of the computation runs in the HIP
kernels of ``libkan.so``.  The raw entry points keep the C names
(``kan_basis_eval``, ``kan_layer_forward``, ``kan_status_string``) and take
device addresses as integers; ``basis``, ``layer_forward`` and ``mlp_forward``
accept torch tensors on a ROCm device and launch on torch's current stream.

The library must have been built (``python -m paper_2609_01956_amd.build``);
loading raises if it is missing.  There is no fallback of any kind.
"""
from __future__ import annotations

import array
import ctypes
import operator
import os
import threading
from typing import Iterable, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkan.so")

KAN_OK = 0
KAN_ERR_INVALID_ARG = 1
KAN_ERR_UNSUPPORTED = 2
KAN_ERR_DEVICE = 3
KAN_ERR_SCRATCH_LIMIT = 4
KAN_NOALLOC_SCRATCH_BYTES = 16 << 20

KAN_F32 = 0
KAN_BF16 = 1

EXPORTED_SYMBOLS = ("kan_basis_eval", "kan_basis_eval_cdb", "kan_layer_forward", "kan_layer_forward_workspace_bytes",
                    "kan_layer_packed_bytes", "kan_layer_pack", "kan_layer_forward_packed",
                    "kan_layer_forward_packed_workspace_bytes",
                    "kan_layer_forward_packed_full_workspace_bytes",
                    "kan_layer_plan", "kan_layer_forward_noalloc", "kan_layer_backward",
                    "kan_layer_backward_workspace_bytes", "kan_layer_forward_span",
                    "kan_layer_forward_span_workspace_bytes", "kan_layer_norm",
                    "kan_layer_norm_backward", "kan_layer_norm_backward_workspace_bytes",
                    "kan_token_logprobs", "kan_token_logprobs_workspace_bytes",
                    "kan_token_logprobs_backward", "kan_grad_norm", "kan_clip_grad_norm",
                    "kan_grad_norm_workspace_bytes", "kan_embedding", "kan_embedding_backward",
                    "kan_embedding_backward_workspace_bytes", "kan_linear_logprobs",
                    "kan_linear_logprobs_workspace_bytes", "kan_linear_logprobs_backward",
                    "kan_linear_logprobs_backward_workspace_bytes", "kan_status_string",
                    "kan_abi_version")

_VP = ctypes.c_void_p
_I32P = ctypes.POINTER(ctypes.c_int32)


class kan_grid(ctypes.Structure):
    _fields_ = [("grid_size", ctypes.c_int32), ("spline_order", ctypes.c_int32),
                ("grid_lo", ctypes.c_float), ("grid_hi", ctypes.c_float)]


class KanError(RuntimeError):
    pass


_lock = threading.Lock()
_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libkan.so once; raise if it has not been built."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(path):
                raise RuntimeError(
                    f"{path} is missing: build the HIP library first "
                    "(python -m paper_2609_01956_amd.build)")
            lib = ctypes.CDLL(path)
            lib.kan_basis_eval.argtypes = [ctypes.POINTER(kan_grid), ctypes.c_int, ctypes.c_void_p,
                                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
            lib.kan_basis_eval.restype = ctypes.c_int
            lib.kan_basis_eval_cdb.argtypes = lib.kan_basis_eval.argtypes
            lib.kan_basis_eval_cdb.restype = ctypes.c_int
            g = ctypes.POINTER(kan_grid)
            lib.kan_layer_forward.argtypes = [g, ctypes.c_int, ctypes.c_int64, ctypes.c_int32,
                                              ctypes.c_int32, _VP, _VP, _VP, _VP, ctypes.c_size_t,
                                              _VP, _VP]
            lib.kan_layer_forward.restype = ctypes.c_int
            lib.kan_layer_forward_workspace_bytes.argtypes = [g, ctypes.c_int, ctypes.c_int64,
                                                              ctypes.c_int32, ctypes.c_int32,
                                                              ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_layer_forward_workspace_bytes.restype = ctypes.c_int
            lib.kan_layer_packed_bytes.argtypes = [g, ctypes.c_int, ctypes.c_int32,
                                                   ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_layer_packed_bytes.restype = ctypes.c_int
            lib.kan_layer_pack.argtypes = [g, ctypes.c_int, ctypes.c_int32, ctypes.c_int32, _VP,
                                           _VP, _VP, ctypes.c_size_t, _VP]
            lib.kan_layer_pack.restype = ctypes.c_int
            lib.kan_layer_forward_packed.argtypes = [g, ctypes.c_int, ctypes.c_int64,
                                                     ctypes.c_int32, ctypes.c_int32, _VP, _VP,
                                                     ctypes.c_size_t, _I32P, _VP,
                                                     ctypes.c_size_t, _VP, _VP]
            lib.kan_layer_forward_packed.restype = ctypes.c_int
            lib.kan_layer_forward_packed_workspace_bytes.argtypes = [
                g, ctypes.c_int, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _I32P,
                ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_layer_forward_packed_workspace_bytes.restype = ctypes.c_int
            lib.kan_layer_forward_packed_full_workspace_bytes.argtypes = \
                lib.kan_layer_forward_workspace_bytes.argtypes
            lib.kan_layer_forward_packed_full_workspace_bytes.restype = ctypes.c_int
            lib.kan_layer_plan.argtypes = [g, ctypes.c_int, ctypes.c_int64, ctypes.c_int32,
                                           ctypes.c_int32, _I32P, _I32P]
            lib.kan_layer_plan.restype = ctypes.c_int
            lib.kan_layer_forward_noalloc.argtypes = [g, ctypes.c_int, ctypes.c_int64,
                                                      ctypes.c_int32, ctypes.c_int32, _VP, _VP,
                                                      _VP, _VP, _VP]
            lib.kan_layer_forward_noalloc.restype = ctypes.c_int
            lib.kan_layer_backward.argtypes = [g, ctypes.c_int, ctypes.c_int64, ctypes.c_int32,
                                               ctypes.c_int32, _VP, _VP, _VP, _VP, _VP, _VP, _VP,
                                               _VP, ctypes.c_size_t, _VP]
            lib.kan_layer_backward.restype = ctypes.c_int
            lib.kan_layer_backward_workspace_bytes.argtypes = [g, ctypes.c_int, ctypes.c_int64,
                                                               ctypes.c_int32, ctypes.c_int32,
                                                               ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_layer_backward_workspace_bytes.restype = ctypes.c_int
            lib.kan_layer_forward_span.argtypes = lib.kan_layer_forward.argtypes
            lib.kan_layer_forward_span.restype = ctypes.c_int
            lib.kan_layer_forward_span_workspace_bytes.argtypes = \
                lib.kan_layer_forward_workspace_bytes.argtypes
            lib.kan_layer_forward_span_workspace_bytes.restype = ctypes.c_int
            lib.kan_layer_norm.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int64,
                                           ctypes.c_int32, _VP, _VP, _VP, _VP, ctypes.c_float, _VP,
                                           _VP, _VP, _VP, _VP]
            lib.kan_layer_norm.restype = ctypes.c_int
            lib.kan_layer_norm_backward.argtypes = [
                ctypes.c_int, ctypes.c_int, ctypes.c_int64, ctypes.c_int32, _VP, _VP, _VP, _VP, _VP,
                _VP, _VP, _VP, _VP, _VP, ctypes.c_size_t, _VP]
            lib.kan_layer_norm_backward.restype = ctypes.c_int
            lib.kan_layer_norm_backward_workspace_bytes.argtypes = [
                ctypes.c_int, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_layer_norm_backward_workspace_bytes.restype = ctypes.c_int
            lib.kan_token_logprobs.argtypes = [
                ctypes.c_int, ctypes.c_int64, ctypes.c_int32, _VP, ctypes.c_int64, _VP,
                ctypes.c_int64, ctypes.c_int32, _VP, _VP, _VP, _VP, _VP, _VP, ctypes.c_size_t, _VP]
            lib.kan_token_logprobs.restype = ctypes.c_int
            lib.kan_token_logprobs_workspace_bytes.argtypes = [
                ctypes.c_int, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_token_logprobs_workspace_bytes.restype = ctypes.c_int
            lib.kan_token_logprobs_backward.argtypes = [
                ctypes.c_int, ctypes.c_int64, ctypes.c_int32, _VP, ctypes.c_int64, _VP,
                ctypes.c_int64, _VP, _VP, _VP, _VP, _VP, ctypes.c_int64, _VP]
            lib.kan_token_logprobs_backward.restype = ctypes.c_int
            lib.kan_grad_norm.argtypes = [ctypes.c_int32, _VP, _VP, _VP, _VP, ctypes.c_size_t, _VP,
                                          _VP]
            lib.kan_grad_norm.restype = ctypes.c_int
            lib.kan_clip_grad_norm.argtypes = [ctypes.c_int32, _VP, _VP, _VP, ctypes.c_float,
                                               ctypes.c_float, _VP, _VP, ctypes.c_size_t, _VP, _VP]
            lib.kan_clip_grad_norm.restype = ctypes.c_int
            lib.kan_grad_norm_workspace_bytes.argtypes = [ctypes.c_int32,
                                                          ctypes.POINTER(ctypes.c_size_t)]
            lib.kan_grad_norm_workspace_bytes.restype = ctypes.c_int
            c_int, i32, i64, f32 = ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
            size, sizep = ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
            lib.kan_embedding.argtypes = [c_int, c_int, i64, i32, i32, _VP, i64, _VP, i64, f32, _VP,
                                          _VP]
            lib.kan_embedding.restype = c_int
            lib.kan_embedding_backward.argtypes = [c_int, c_int, i64, i32, i32, _VP, i64, _VP, i64,
                                                   f32, _VP, _VP, _VP, size, _VP]
            lib.kan_embedding_backward.restype = c_int
            lib.kan_embedding_backward_workspace_bytes.argtypes = [i64, i32, i32, sizep]
            lib.kan_embedding_backward_workspace_bytes.restype = c_int
            lib.kan_linear_logprobs.argtypes = [c_int, i64, i32, i32, _VP, i64, _VP, i64, f32, _VP,
                                                i64, _VP, _VP, _VP, _VP, size, _VP]
            lib.kan_linear_logprobs.restype = c_int
            lib.kan_linear_logprobs_backward.argtypes = [c_int, i64, i32, i32, _VP, i64, _VP, i64,
                                                         f32, _VP, i64, _VP, _VP, _VP, _VP, _VP,
                                                         size, _VP]
            lib.kan_linear_logprobs_backward.restype = c_int
            for fn in (lib.kan_linear_logprobs_workspace_bytes,
                       lib.kan_linear_logprobs_backward_workspace_bytes):
                fn.argtypes = [c_int, i64, i32, i32, _VP, i64, _VP, i64, sizep]
                fn.restype = c_int
            lib.kan_status_string.argtypes = [ctypes.c_int]
            lib.kan_status_string.restype = ctypes.c_char_p
            lib.kan_abi_version.argtypes = []
            lib.kan_abi_version.restype = ctypes.c_int32
            _lib = lib
    return _lib


# ----------------------------------------------------------- raw C entry points

def make_grid(grid_size: int, grid_lo: float = -1.0, grid_hi: float = 1.0,
              spline_order: int = 3) -> kan_grid:
    return kan_grid(int(grid_size), int(spline_order), float(grid_lo), float(grid_hi))


def kan_status_string(status: int) -> str:
    return load_library().kan_status_string(int(status)).decode()


def kan_abi_version() -> int:
    return int(load_library().kan_abi_version())


def kan_basis_eval(grid: kan_grid, dtype: int, x: int, n: int, phi: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_basis_eval(ctypes.byref(grid), int(dtype), ctypes.c_void_p(x),
                                             int(n), ctypes.c_void_p(phi), ctypes.c_void_p(stream)))


def _shape_arg(shape):
    """None, or a forced workgroup shape (rf, wk, nw, cs) / "rf,wk[,nw[,cs]]"
    as an int32[4] (nw defaults to 4, cs to 1)."""
    if shape is None:
        return None
    if isinstance(shape, str):
        shape = [int(t) for t in shape.split(",")]
    v = list(shape) + [4, 1][len(shape) - 2:] if len(shape) < 4 else list(shape)
    if len(v) != 4:
        raise ValueError("a shape is (rf, wk[, nw[, cs]])")
    return (ctypes.c_int32 * 4)(*[int(t) for t in v])


def kan_basis_eval_cdb(grid: kan_grid, dtype: int, x: int, n: int, phi: int,
                       stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_basis_eval_cdb(ctypes.byref(grid), int(dtype), _VP(x), int(n),
                                                 _VP(phi), _VP(stream)))


def kan_layer_forward(grid: kan_grid, dtype: int, batch: int, in_features: int,
                      out_features: int, x: int, coef: int, base_w: int, workspace: int,
                      workspace_bytes: int, y: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_layer_forward(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        _VP(x), _VP(coef), _VP(base_w), _VP(workspace), ctypes.c_size_t(workspace_bytes),
        _VP(y), _VP(stream)))


def kan_layer_forward_noalloc(grid: kan_grid, dtype: int, batch: int, in_features: int,
                              out_features: int, x: int, coef: int, base_w: int, y: int,
                              stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_layer_forward_noalloc(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        _VP(x), _VP(coef), _VP(base_w), _VP(y), _VP(stream)))


def kan_layer_backward(grid: kan_grid, dtype: int, batch: int, in_features: int,
                       out_features: int, x: int, coef: int, base_w: int, dy: int, dx: int,
                       dcoef: int, dbase_w: int, workspace: int, workspace_bytes: int,
                       stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_layer_backward(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        _VP(x), _VP(coef), _VP(base_w), _VP(dy), _VP(dx), _VP(dcoef), _VP(dbase_w),
        _VP(workspace), ctypes.c_size_t(workspace_bytes), _VP(stream)))


def kan_layer_forward_span(grid: kan_grid, dtype: int, batch: int, in_features: int,
                           out_features: int, x: int, coef: int, base_w: int, workspace: int,
                           workspace_bytes: int, y: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_layer_forward_span(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        _VP(x), _VP(coef), _VP(base_w), _VP(workspace), ctypes.c_size_t(workspace_bytes),
        _VP(y), _VP(stream)))


def kan_layer_forward_span_workspace_bytes(grid: kan_grid, dtype: int, batch: int,
                                           in_features: int, out_features: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    n = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_forward_span_workspace_bytes(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        ctypes.byref(n)))
    return st, int(n.value)


def kan_layer_backward_workspace_bytes(grid: kan_grid, dtype: int, batch: int, in_features: int,
                                       out_features: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    n = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_backward_workspace_bytes(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        ctypes.byref(n)))
    return st, int(n.value)


def kan_layer_forward_workspace_bytes(grid: kan_grid, dtype: int, batch: int, in_features: int,
                                      out_features: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    n = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_forward_workspace_bytes(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        ctypes.byref(n)))
    return st, int(n.value)


def kan_layer_packed_bytes(grid: kan_grid, dtype: int, in_features: int,
                           out_features: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    n = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_packed_bytes(ctypes.byref(grid), int(dtype),
                                                   int(in_features), int(out_features),
                                                   ctypes.byref(n)))
    return st, int(n.value)


def kan_layer_plan(grid: kan_grid, dtype: int, batch: int, in_features: int,
                   out_features: int, shape=None) -> Tuple[int, Tuple[int, ...]]:
    """Raw call: returns (kan_status, (rf, wk, nw, cs, sparse, k_splits));
    `shape` forces a workgroup shape (see _shape_arg), None takes the
    library's choice."""
    plan = (ctypes.c_int32 * 6)()
    st = int(load_library().kan_layer_plan(ctypes.byref(grid), int(dtype), int(batch),
                                           int(in_features), int(out_features),
                                           _shape_arg(shape), plan))
    return st, tuple(int(v) for v in plan)


def kan_layer_pack(grid: kan_grid, dtype: int, in_features: int, out_features: int, coef: int,
                   base_w: int, packed: int, packed_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_layer_pack(
        ctypes.byref(grid), int(dtype), int(in_features), int(out_features), _VP(coef),
        _VP(base_w), _VP(packed), ctypes.c_size_t(packed_bytes), _VP(stream)))


def kan_layer_forward_packed(grid: kan_grid, dtype: int, batch: int, in_features: int,
                             out_features: int, x: int, packed: int, packed_bytes: int, y: int,
                             stream: int = 0, shape=None, workspace: int = 0,
                             workspace_bytes: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code.
    `shape` forces a workgroup shape (see _shape_arg); `workspace` (0: none)
    holds the partial sums of a split contraction."""
    return int(load_library().kan_layer_forward_packed(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        _VP(x), _VP(packed), ctypes.c_size_t(packed_bytes), _shape_arg(shape), _VP(workspace),
        ctypes.c_size_t(workspace_bytes), _VP(y), _VP(stream)))


def kan_layer_forward_packed_workspace_bytes(grid: kan_grid, dtype: int, batch: int,
                                             in_features: int, out_features: int,
                                             shape=None) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    n = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_forward_packed_workspace_bytes(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        _shape_arg(shape), ctypes.byref(n)))
    return st, int(n.value)


def kan_layer_forward_packed_full_workspace_bytes(grid: kan_grid, dtype: int, batch: int,
                                                  in_features: int,
                                                  out_features: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    n = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_forward_packed_full_workspace_bytes(
        ctypes.byref(grid), int(dtype), int(batch), int(in_features), int(out_features),
        ctypes.byref(n)))
    return st, int(n.value)


def kan_layer_norm(dtype: int, param_dtype: int, rows: int, n: int, x: int, residual: int,
                   weight: int, bias: int, eps: float, h: int, y: int, mean: int, rstd: int,
                   stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_layer_norm(
        int(dtype), int(param_dtype), int(rows), int(n), _VP(x), _VP(residual), _VP(weight),
        _VP(bias), float(eps), _VP(h), _VP(y), _VP(mean), _VP(rstd), _VP(stream)))


def kan_layer_norm_backward(dtype: int, param_dtype: int, rows: int, n: int, h: int, mean: int,
                            rstd: int, weight: int, dy: int, dh: int, dx: int, dweight: int,
                            dbias: int, workspace: int, workspace_bytes: int,
                            stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_layer_norm_backward(
        int(dtype), int(param_dtype), int(rows), int(n), _VP(h), _VP(mean), _VP(rstd),
        _VP(weight), _VP(dy), _VP(dh), _VP(dx), _VP(dweight), _VP(dbias), _VP(workspace),
        ctypes.c_size_t(workspace_bytes), _VP(stream)))


def kan_layer_norm_backward_workspace_bytes(dtype: int, rows: int, n: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    size = ctypes.c_size_t(0)
    st = int(load_library().kan_layer_norm_backward_workspace_bytes(
        int(dtype), int(rows), int(n), ctypes.byref(size)))
    return st, int(size.value)


def kan_token_logprobs(dtype: int, rows: int, classes: int, logits: int, row_stride: int,
                       targets: int, ignore_index: int, top_k: int, logp: int, stats: int,
                       entropy: int, top_logp: int, top_index: int, workspace: int,
                       workspace_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_token_logprobs(
        int(dtype), int(rows), int(classes), _VP(logits), int(row_stride), _VP(targets),
        int(ignore_index), int(top_k), _VP(logp), _VP(stats), _VP(entropy), _VP(top_logp),
        _VP(top_index), _VP(workspace), ctypes.c_size_t(workspace_bytes), _VP(stream)))


def kan_token_logprobs_workspace_bytes(dtype: int, rows: int, classes: int,
                                       top_k: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    size = ctypes.c_size_t(0)
    st = int(load_library().kan_token_logprobs_workspace_bytes(
        int(dtype), int(rows), int(classes), int(top_k), ctypes.byref(size)))
    return st, int(size.value)


def kan_token_logprobs_backward(dtype: int, rows: int, classes: int, logits: int, row_stride: int,
                                targets: int, ignore_index: int, stats: int, dlogp: int,
                                entropy: int, dentropy: int, dlogits: int, dlogits_stride: int,
                                stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_token_logprobs_backward(
        int(dtype), int(rows), int(classes), _VP(logits), int(row_stride), _VP(targets),
        int(ignore_index), _VP(stats), _VP(dlogp), _VP(entropy), _VP(dentropy), _VP(dlogits),
        int(dlogits_stride), _VP(stream)))


def _host(kind: str, values):
    """A host array and its address (0 for None)."""
    if values is None:
        return None, 0
    a = array.array(kind, values)
    return a, a.buffer_info()[0]


def kan_grad_norm(grads: Sequence[int], sizes: Sequence[int], dtypes: Sequence[int],
                  workspace: int, workspace_bytes: int, norm: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers, the host arrays as sequences; returns the
    kan_status code."""
    (g, pg), (n, pn), (d, pd) = _host("Q", grads), _host("q", sizes), _host("i", dtypes)
    return int(load_library().kan_grad_norm(len(g), pg, pn, pd, _VP(workspace),
                                            ctypes.c_size_t(workspace_bytes), _VP(norm),
                                            _VP(stream)))


def kan_clip_grad_norm(grads: Sequence[int], sizes: Sequence[int], dtypes: Sequence[int],
                       max_norm: float, eps: float, out: Optional[Sequence[int]], workspace: int,
                       workspace_bytes: int, norm: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers, the host arrays as sequences (out None: NULL);
    returns the kan_status code."""
    (g, pg), (n, pn), (d, pd) = _host("Q", grads), _host("q", sizes), _host("i", dtypes)
    o, po = _host("Q", out)
    return int(load_library().kan_clip_grad_norm(
        len(g), pg, pn, pd, float(max_norm), float(eps), po, _VP(workspace),
        ctypes.c_size_t(workspace_bytes), _VP(norm), _VP(stream)))


def kan_grad_norm_workspace_bytes(count: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    size = ctypes.c_size_t(0)
    st = int(load_library().kan_grad_norm_workspace_bytes(int(count), ctypes.byref(size)))
    return st, int(size.value)


def kan_embedding(dtype: int, table_dtype: int, rows: int, classes: int, n: int, tokens: int,
                  ignore_index: int, table: int, table_stride: int, scale: float, y: int,
                  stream: int = 0) -> int:
    """Raw call: device addresses as integers; returns the kan_status code."""
    return int(load_library().kan_embedding(
        int(dtype), int(table_dtype), int(rows), int(classes), int(n), _VP(tokens),
        int(ignore_index), _VP(table), int(table_stride), float(scale), _VP(y), _VP(stream)))


def kan_embedding_backward(dtype: int, table_dtype: int, rows: int, classes: int, n: int,
                           tokens: int, ignore_index: int, dy: int, dy_stride: int, scale: float,
                           base: int, dtable: int, workspace: int, workspace_bytes: int,
                           stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_embedding_backward(
        int(dtype), int(table_dtype), int(rows), int(classes), int(n), _VP(tokens),
        int(ignore_index), _VP(dy), int(dy_stride), float(scale), _VP(base), _VP(dtable),
        _VP(workspace), ctypes.c_size_t(workspace_bytes), _VP(stream)))


def kan_embedding_backward_workspace_bytes(rows: int, classes: int, n: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    size = ctypes.c_size_t(0)
    st = int(load_library().kan_embedding_backward_workspace_bytes(
        int(rows), int(classes), int(n), ctypes.byref(size)))
    return st, int(size.value)


def kan_linear_logprobs(dtype: int, rows: int, classes: int, n: int, x: int, x_stride: int,
                        weight: int, weight_stride: int, scale: float, targets: int,
                        ignore_index: int, logp: int, stats: int, best: int, workspace: int,
                        workspace_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_linear_logprobs(
        int(dtype), int(rows), int(classes), int(n), _VP(x), int(x_stride), _VP(weight),
        int(weight_stride), float(scale), _VP(targets), int(ignore_index), _VP(logp), _VP(stats),
        _VP(best), _VP(workspace), ctypes.c_size_t(workspace_bytes), _VP(stream)))


def kan_linear_logprobs_workspace_bytes(dtype: int, rows: int, classes: int, n: int, x: int,
                                        x_stride: int, weight: int,
                                        weight_stride: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    size = ctypes.c_size_t(0)
    st = int(load_library().kan_linear_logprobs_workspace_bytes(
        int(dtype), int(rows), int(classes), int(n), _VP(x), int(x_stride), _VP(weight),
        int(weight_stride), ctypes.byref(size)))
    return st, int(size.value)


def kan_linear_logprobs_backward(dtype: int, rows: int, classes: int, n: int, x: int, x_stride: int,
                                 weight: int, weight_stride: int, scale: float, targets: int,
                                 ignore_index: int, stats: int, dlogp: int, dx: int, dweight: int,
                                 workspace: int, workspace_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as integers (0 for NULL); returns the kan_status code."""
    return int(load_library().kan_linear_logprobs_backward(
        int(dtype), int(rows), int(classes), int(n), _VP(x), int(x_stride), _VP(weight),
        int(weight_stride), float(scale), _VP(targets), int(ignore_index), _VP(stats), _VP(dlogp),
        _VP(dx), _VP(dweight), _VP(workspace), ctypes.c_size_t(workspace_bytes), _VP(stream)))


def kan_linear_logprobs_backward_workspace_bytes(dtype: int, rows: int, classes: int, n: int,
                                                 x: int, x_stride: int, weight: int,
                                                 weight_stride: int) -> Tuple[int, int]:
    """Raw call: returns (kan_status, bytes)."""
    size = ctypes.c_size_t(0)
    st = int(load_library().kan_linear_logprobs_backward_workspace_bytes(
        int(dtype), int(rows), int(classes), int(n), _VP(x), int(x_stride), _VP(weight),
        int(weight_stride), ctypes.byref(size)))
    return st, int(size.value)


def check(status: int) -> None:
    """Map a kan_status to an exception."""
    if status == KAN_OK:
        return
    msg = kan_status_string(status)
    if status in (KAN_ERR_INVALID_ARG, KAN_ERR_SCRATCH_LIMIT):
        raise ValueError(msg)
    if status == KAN_ERR_UNSUPPORTED:
        raise NotImplementedError(msg)
    raise KanError(msg)


# ------------------------------------------------------------ torch marshalling

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return KAN_F32
    if t.dtype == torch.bfloat16:
        return KAN_BF16
    raise NotImplementedError(f"dtype {t.dtype} is not supported (float32 or bfloat16)")


def _require_device(*ts) -> None:
    for t in ts:
        if not t.is_cuda:
            raise ValueError("tensors must live on the GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")
    dev = ts[0].device
    for t in ts[1:]:
        if t.device != dev:
            raise ValueError("tensors must live on one device")


def _stream(device) -> int:
    """Handle of torch's current stream (read without building a Stream object: 0.1
    against 1.9 us)."""
    raw = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)
    if raw is not None:
        return raw(device.index)
    return int(_torch().cuda.current_stream(device).cuda_stream)


def _call(device, fn, *args) -> int:
    """fn(*args) with `device` current; a small layer's call is bound by the host, so
    the device is switched only where it is another one."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getDevice", None)
    if (torch.cuda.current_device() if raw is None else raw()) == device.index:
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _library() -> ctypes.CDLL:
    return _lib if _lib is not None else load_library()


def _fits(workspace, nbytes: int, device) -> bool:
    """Can a caller's workspace (or None) be used: nbytes side by side on the device (an expanded
    or strided tensor counts elements that it does not hold)."""
    return workspace is not None and workspace.device == device and \
        workspace.numel() >= nbytes and workspace.is_contiguous()


def _query(fn, grid, *args) -> int:
    """A size query's bytes."""
    n = ctypes.c_size_t(0)
    check(fn(ctypes.byref(grid), *args, ctypes.byref(n)))
    return n.value


def basis(x, grid_size: int, grid_lo: float = -1.0, grid_hi: float = 1.0, out=None,
          spline_order: int = 3, method: str = "tp"):
    """phi[..., j] = N_j(x[...]) for j < grid_size + spline_order: the
    truncated-power form (kan_basis_eval, method "tp") or the Cox-de Boor
    recursion (kan_basis_eval_cdb, method "cdb")."""
    if method not in ("tp", "cdb"):
        raise ValueError("method is 'tp' or 'cdb'")
    torch = _torch()
    _require_device(x)
    nb = int(grid_size) + int(spline_order)
    if out is None:
        out = torch.empty(tuple(x.shape) + (nb,), dtype=x.dtype, device=x.device)
    else:
        _require_device(x, out)
        if out.dtype != x.dtype or tuple(out.shape) != tuple(x.shape) + (nb,):
            raise ValueError("out must have shape x.shape + (G + k,) and x's dtype")
    lib = _library()
    g = make_grid(grid_size, grid_lo, grid_hi, spline_order)
    check(_call(x.device, lib.kan_basis_eval if method == "tp" else lib.kan_basis_eval_cdb,
                ctypes.byref(g), _dtype_code(x), x.data_ptr(), x.numel(), out.data_ptr(),
                _stream(x.device)))
    return out


class PackedLayer:
    """Weights of one layer packed by kan_layer_pack (device buffer + shape)."""

    def __init__(self, buf, grid_size, grid_lo, grid_hi, n_in, n_out, dtype, spline_order=3):
        self.buf = buf
        self.spline_order = int(spline_order)
        self.grid_size, self.grid_lo, self.grid_hi = int(grid_size), float(grid_lo), float(grid_hi)
        self.n_in, self.n_out = int(n_in), int(n_out)
        self.dtype = dtype

    @property
    def nbytes(self) -> int:
        return int(self.buf.numel())


def _check_weights(coef, base_w, grid_size, spline_order=3):
    _require_device(coef, base_w)
    if base_w.dim() != 2 or coef.dim() != 3:
        raise ValueError("expected coef [out, in, G+3], base_w [out, in]")
    n_out, n_in = base_w.shape
    if tuple(coef.shape) != (n_out, n_in, int(grid_size) + int(spline_order)):
        raise ValueError("coef / base_w shapes do not match each other and the grid")
    if coef.dtype != base_w.dtype:
        raise ValueError("coef and base_w must share one dtype")
    return n_in, n_out


def pack_layer(coef, base_w, grid_size: int, grid_lo: float = -1.0, grid_hi: float = 1.0,
               out: Optional[PackedLayer] = None, spline_order: int = 3) -> PackedLayer:
    """kan_layer_pack: coef [out, in, G + 3], base_w [out, in] -> PackedLayer
    (device buffer from torch's allocator, filled on torch's current stream)."""
    torch = _torch()
    n_in, n_out = _check_weights(coef, base_w, grid_size, spline_order)
    dt = _dtype_code(coef)
    g = make_grid(grid_size, grid_lo, grid_hi, spline_order)
    lib = _library()
    nbytes = _query(lib.kan_layer_packed_bytes, g, dt, n_in, n_out)
    if out is None:
        buf = torch.empty(nbytes, dtype=torch.uint8, device=coef.device)
        out = PackedLayer(buf, grid_size, grid_lo, grid_hi, n_in, n_out, coef.dtype, spline_order)
    elif out.nbytes < nbytes or out.buf.device != coef.device:
        raise ValueError("packed buffer too small or on another device")
    else:
        # the buffer now holds these weights: its geometry follows them
        out.grid_size, out.grid_lo, out.grid_hi = int(grid_size), float(grid_lo), float(grid_hi)
        out.n_in, out.n_out, out.dtype = int(n_in), int(n_out), coef.dtype
        out.spline_order = int(spline_order)
    check(_call(coef.device, lib.kan_layer_pack, ctypes.byref(g), dt, n_in, n_out, coef.data_ptr(),
                base_w.data_ptr(), out.buf.data_ptr(), out.nbytes, _stream(coef.device)))
    return out


def layer_forward_packed(x, packed: PackedLayer, out=None, shape=None, workspace=None,
                         split: bool = True):
    """kan_layer_forward_packed: x [B, in] with packed weights -> y [B, out].
    `shape` forces a workgroup shape (rf, wk[, nw[, cs]]) for tests and tuning.
    For batches too small to fill the GPU the contraction is split across
    workgroups, and large layers run on weights expanded for the call; the
    partial sums and expanded weights go to `workspace` (a uint8 device tensor)
    when large enough, else to a fresh one from torch's allocator; split=False
    runs the layer unsplit on the packed weights alone."""
    torch = _torch()
    _require_device(x)
    if x.dim() != 2 or x.shape[1] != packed.n_in:
        raise ValueError("x must be [B, in] with the packed layer's in")
    if x.dtype != packed.dtype or packed.buf.device != x.device:
        raise ValueError("x must match the packed layer's dtype and device")
    B = x.shape[0]
    if out is None:
        out = torch.empty((B, packed.n_out), dtype=x.dtype, device=x.device)
    else:
        _require_device(x, out)
        if out.dtype != x.dtype or tuple(out.shape) != (B, packed.n_out):
            raise ValueError("out must be [B, out] with x's dtype")
    g = make_grid(packed.grid_size, packed.grid_lo, packed.grid_hi, packed.spline_order)
    dt = _dtype_code(x)
    lib = _library()
    shape = _shape_arg(shape)
    ws_ptr, ws_bytes = 0, 0
    if split:
        if shape is None:
            need = _query(lib.kan_layer_forward_packed_full_workspace_bytes, g, dt, B, packed.n_in,
                          packed.n_out)
        else:
            need = _query(lib.kan_layer_forward_packed_workspace_bytes, g, dt, B, packed.n_in,
                          packed.n_out, shape)
        if need > 0:
            if not _fits(workspace, need, x.device):
                workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
            ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel()
    check(_call(x.device, lib.kan_layer_forward_packed, ctypes.byref(g), dt, B, packed.n_in,
                packed.n_out, x.data_ptr(), packed.buf.data_ptr(), packed.nbytes, shape, ws_ptr,
                ws_bytes, out.data_ptr(), _stream(x.device)))
    return out


def layer_forward(x, coef, base_w, grid_size: int, grid_lo: float = -1.0, grid_hi: float = 1.0,
                  out=None, packed: Optional[PackedLayer] = None, shape=None,
                  spline_order: int = 3):
    """One KAN layer: x [B, in], coef [out, in, G + 3], base_w [out, in] -> y
    [B, out], all of one dtype on one device.  Packs the weights (kan_layer_pack,
    into `packed` if given, else a fresh buffer) and runs
    kan_layer_forward_packed, both on torch's current stream; `shape` forces a
    workgroup shape."""
    _require_device(x)
    n_in, n_out = _check_weights(coef, base_w, grid_size, spline_order)
    if x.dim() != 2 or x.shape[1] != n_in:
        raise ValueError("x must be [B, in] with coef's in")
    if coef.dtype != x.dtype:
        raise ValueError("x, coef and base_w must share one dtype")
    if out is None and packed is None and shape is None and x.device == coef.device:
        # both steps in one call, in one workspace
        torch, lib = _torch(), _library()
        g, dt, B = make_grid(grid_size, grid_lo, grid_hi, spline_order), _dtype_code(x), x.shape[0]
        need = _query(lib.kan_layer_forward_workspace_bytes, g, dt, B, n_in, n_out)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device)
        out = torch.empty((B, n_out), dtype=x.dtype, device=x.device)
        check(_call(x.device, lib.kan_layer_forward, ctypes.byref(g), dt, B, n_in, n_out,
                    x.data_ptr(), coef.data_ptr(), base_w.data_ptr(), ws.data_ptr(), need,
                    out.data_ptr(), _stream(x.device)))
        return out
    p = pack_layer(coef, base_w, grid_size, grid_lo, grid_hi, out=packed,
                   spline_order=spline_order)
    return layer_forward_packed(x, p, out=out, shape=shape)


def mlp_forward(x, layers: Sequence[Tuple[object, object]], grid_size: int, grid_lo: float = -1.0,
                grid_hi: float = 1.0, return_all: bool = False, spline_order: int = 3):
    """Stacked KAN layers; each output feeds the next layer unchanged (values
    off the grid are handled by the clamp of the basis)."""
    h = x
    outs = []
    for coef, base_w in layers:
        h = layer_forward(h, coef, base_w, grid_size, grid_lo, grid_hi,
                          spline_order=spline_order)
        outs.append(h)
    return outs if return_all else h


def layer_backward(x, coef, base_w, dy, grid_size: int, grid_lo: float = -1.0,
                   grid_hi: float = 1.0, need_dx: bool = True, need_dw: bool = True,
                   workspace=None, out=None):
    """Gradients of one KAN layer (kan_layer_backward): x [B, in], coef [out,
    in, G + 3], base_w [out, in], dy [B, out], all of one dtype on one device
    -> (dx [B, in] or None, dcoef or None, dbase_w or None), enqueued on
    torch's current stream.  `workspace` (a uint8 device tensor) is used when
    large enough, else a fresh one is taken from torch's allocator; `out`, a
    (dx, dcoef, dbase_w) tuple of tensors shaped like x, coef and base_w,
    receives the gradients instead of fresh tensors."""
    torch = _torch()
    _require_device(x, dy)
    n_in, n_out = _check_weights(coef, base_w, grid_size)
    if x.dim() != 2 or x.shape[1] != n_in or dy.shape != (x.shape[0], n_out):
        raise ValueError("x must be [B, in] and dy [B, out] for the weights' in and out")
    if not (x.dtype == dy.dtype == coef.dtype):
        raise ValueError("x, dy and the weights must share one dtype")
    if not (need_dx or need_dw):
        raise ValueError("nothing to compute")
    B = x.shape[0]
    dt = _dtype_code(x)
    g = make_grid(grid_size, grid_lo, grid_hi)
    lib = _library()
    nbytes = _query(lib.kan_layer_backward_workspace_bytes, g, dt, B, n_in, n_out)
    if not _fits(workspace, nbytes, x.device):
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x.device)
    if out is not None:
        dx, dC, dW = out
        for t, like in ((dx, x), (dC, coef), (dW, base_w)):
            if t is not None and (t.shape != like.shape or t.dtype != like.dtype or
                                  t.device != like.device or not t.is_contiguous()):
                raise ValueError("out tensors must match x, coef and base_w")
        dx = dx if need_dx else None
        dC, dW = (dC, dW) if need_dw else (None, None)
    else:
        dx = torch.empty_like(x) if need_dx else None
        dC = torch.empty_like(coef) if need_dw else None
        dW = torch.empty_like(base_w) if need_dw else None
    ptr = lambda t: 0 if t is None else t.data_ptr()
    check(_call(x.device, lib.kan_layer_backward, ctypes.byref(g), dt, B, n_in, n_out,
                x.data_ptr(), coef.data_ptr(), base_w.data_ptr(), dy.data_ptr(), ptr(dx), ptr(dC),
                ptr(dW), workspace.data_ptr(), workspace.numel(), _stream(x.device)))
    return dx, dC, dW


def layer_forward_span(x, coef, base_w, grid_size: int, grid_lo: float = -1.0,
                       grid_hi: float = 1.0, out=None, spline_order: int = 3, workspace=None):
    """kan_layer_forward_span: the layer on its nonzero terms only (the k + 1
    bases whose support holds each input, and SiLU); x [B, in], coef [out, in,
    G + k], base_w [out, in] -> y [B, out], on torch's current stream."""
    torch = _torch()
    _require_device(x)
    n_in, n_out = _check_weights(coef, base_w, grid_size, spline_order)
    if x.dim() != 2 or x.shape[1] != n_in or x.dtype != coef.dtype:
        raise ValueError("x must be [B, in] with the weights' in and dtype")
    B = x.shape[0]
    dt = _dtype_code(x)
    g = make_grid(grid_size, grid_lo, grid_hi, spline_order)
    lib = _library()
    nbytes = _query(lib.kan_layer_forward_span_workspace_bytes, g, dt, B, n_in, n_out)
    if not _fits(workspace, nbytes, x.device):
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x.device)
    if out is None:
        out = torch.empty((B, n_out), dtype=x.dtype, device=x.device)
    elif out.dtype != x.dtype or tuple(out.shape) != (B, n_out):
        raise ValueError("out must be [B, out] with x's dtype")
    _require_device(x, coef, out)
    check(_call(x.device, lib.kan_layer_forward_span, ctypes.byref(g), dt, B, n_in, n_out,
                x.data_ptr(), coef.data_ptr(), base_w.data_ptr(), workspace.data_ptr(),
                workspace.numel(), out.data_ptr(), _stream(x.device)))
    return out


# ------------------------------------------------- the step around the layers

def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _same(what: str, like, *ts) -> None:
    """Tensors (or None) of one shape, dtype and device, contiguous."""
    for t in ts:
        if t is not None and (t.shape != like.shape or t.dtype != like.dtype or
                              t.device != like.device or not t.is_contiguous()):
            raise ValueError(f"{what} must match each other in shape, dtype and device and be "
                             "contiguous")


def _norm_params(x, n: int, first, second=None) -> int:
    """Checks a norm's parameters (or None) against x [..., n]: their dtype code."""
    like = second if first is None else first
    if like is None:
        return _dtype_code(x)
    for t in (first, second):
        if t is None:
            continue
        if t.device != x.device or not t.is_contiguous():
            raise ValueError("the norm's parameters must be contiguous, on the rows' device")
        if t.dim() != 1 or t.shape[0] != n or t.dtype != like.dtype:
            raise ValueError("the norm's parameters must be [n] of one dtype for rows of n")
    return _dtype_code(like)


def _rows(x) -> Tuple[int, int]:
    shape = x.shape
    if len(shape) < 1 or shape[-1] < 1:
        raise ValueError("expected rows [..., n] with n >= 1")
    return x.numel() // shape[-1], shape[-1]


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None,
               need_stats: bool = True, out=None):
    """kan_layer_norm over the last dimension of x [..., n], with `residual` (shaped like x)
    added first -> (y, h, mean, rstd): h = x + residual (x itself without one), mean and rstd
    [...] fp32 for layer_norm_backward (None without need_stats).  weight and bias [n] are
    fp32 or of x's dtype.  `out`, a (y, h) tuple (h None without a residual), receives the
    results instead of fresh tensors."""
    torch = _torch()
    _require_device(x)
    rows, n = _rows(x)
    pdt = _norm_params(x, n, weight, bias)
    if residual is not None:
        _same("x and residual", x, residual)
    if out is None:
        y = torch.empty_like(x)
        h = None if residual is None else torch.empty_like(x)
    else:
        y, h = out
        if (h is None) != (residual is None) or y is None:
            raise ValueError("out is (y, h), h with a residual only")
        _same("x and out", x, y, h)
    device = x.device
    mean = rstd = None
    if need_stats:
        mean = x.new_empty(x.shape[:-1], dtype=torch.float32)
        rstd = torch.empty_like(mean)
    check(_call(device, _library().kan_layer_norm, _dtype_code(x), pdt, rows, n, x.data_ptr(),
                _ptr(residual), _ptr(weight), _ptr(bias), eps, _ptr(h), y.data_ptr(), _ptr(mean),
                _ptr(rstd), _stream(device)))
    return y, x if residual is None else h, mean, rstd


def layer_norm_backward(h, mean, rstd, weight, dy, dh=None, need_dx: bool = True,
                        need_dw: bool = True, workspace=None, out=None):
    """Gradients of layer_norm (kan_layer_norm_backward): h, mean and rstd as it returned
    them, weight as it was given (None: 1), dy like h, dh (like h, or None) the gradient that
    reaches h on the residual stream -> (dx or None, dweight or None, dbias or None); dx is
    the gradient of x and of the residual.  dweight and dbias have weight's dtype (h's
    without a weight).  `workspace` (a uint8 device tensor) is used when large enough, else a
    fresh one is taken; `out`, a (dx, dweight, dbias) tuple, receives the gradients."""
    torch = _torch()
    _require_device(h, dy)
    rows, n = _rows(h)
    pdt = _norm_params(h, n, weight)
    _same("h, dy and dh", h, dy, dh)
    device, f32, lead = h.device, torch.float32, h.shape[:-1]
    for t in (mean, rstd):
        if t is None or t.dtype != f32 or t.shape != lead or t.device != device or \
                not t.is_contiguous():
            raise ValueError("mean and rstd are fp32, one value per row, on the rows' device")
    if not (need_dx or need_dw):
        raise ValueError("nothing to compute")
    dw_dtype = h.dtype if weight is None else weight.dtype
    if out is not None:
        dx, dw, db = out
        dx = dx if need_dx else None
        dw, db = (dw, db) if need_dw else (None, None)
        _same("h and dx", h, dx)
        for t in (dw, db):
            if t is not None and (tuple(t.shape) != (n,) or t.dtype != dw_dtype or
                                  t.device != device or not t.is_contiguous()):
                raise ValueError("dweight and dbias must be [n] with the weight's dtype")
    else:
        dx = torch.empty_like(h) if need_dx else None
        dw = h.new_empty((n,), dtype=dw_dtype) if need_dw else None
        db = torch.empty_like(dw) if need_dw else None
    lib, dt = _library(), _dtype_code(h)
    ws, nbytes = None, 0
    if dw is not None or db is not None:
        size = ctypes.c_size_t(0)
        check(lib.kan_layer_norm_backward_workspace_bytes(dt, rows, n, ctypes.byref(size)))
        nbytes, ws = size.value, workspace
        if not _fits(ws, nbytes, device):
            ws = h.new_empty((max(nbytes, 1),), dtype=torch.uint8)
    check(_call(device, lib.kan_layer_norm_backward, dt, pdt, rows, n, h.data_ptr(),
                mean.data_ptr(), rstd.data_ptr(), _ptr(weight), dy.data_ptr(), _ptr(dh), _ptr(dx),
                _ptr(dw), _ptr(db), _ptr(ws), nbytes, _stream(device)))
    return dx, dw, db


def _logits(z) -> Tuple[int, int, int]:
    """Checks logits [rows, classes]: (rows, classes, elements from row to row)."""
    if not z.is_cuda:
        raise ValueError("tensors must live on the GPU")
    shape = z.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError("logits must be [rows, classes]")
    rows, classes = shape
    stride, inner = z.stride()
    if rows <= 1:
        stride = classes
    if (classes > 1 and inner != 1) or stride < classes:
        raise ValueError("a row of logits must be contiguous, and rows must not overlap")
    return rows, classes, stride


def _row_values(what: str, z, *ts) -> None:
    """fp32 values (or None), one per row of the logits."""
    torch = _torch()
    rows, device, f32 = z.shape[0], z.device, torch.float32
    for t in ts:
        if t is not None and (t.dtype != f32 or t.dim() != 1 or t.shape[0] != rows or
                              t.device != device or not t.is_contiguous()):
            raise ValueError(f"{what} must be fp32 [rows], contiguous, on the logits' device")


def _check_targets(z, rows: int, targets) -> None:
    if targets.dtype != _torch().int64 or targets.dim() != 1 or targets.shape[0] != rows or \
            targets.device != z.device or not targets.is_contiguous():
        raise ValueError("targets must be int64 [rows], contiguous, on the logits' device")


def token_logprobs(logits, targets, top_k: int = 0, entropy: bool = False,
                   ignore_index: int = -100, workspace=None):
    """kan_token_logprobs: logits [rows, classes] (rows may be padded: any row stride of at
    least classes), targets [rows] int64 -> (logp [rows], stats [rows, 2], entropy [rows] or
    None, top_logp [rows, top_k] or None, top_index [rows, top_k] int64 or None), all values
    fp32.  stats goes to token_logprobs_backward.  `workspace` (a uint8 device tensor) is used
    when large enough, else a fresh one is taken."""
    torch = _torch()
    rows, classes, stride = _logits(logits)
    _check_targets(logits, rows, targets)
    dt, k, dev, lib = _dtype_code(logits), int(top_k), logits.device, _library()
    size = ctypes.c_size_t(0)
    check(lib.kan_token_logprobs_workspace_bytes(dt, rows, classes, k, ctypes.byref(size)))
    logp = logits.new_empty((rows,), dtype=torch.float32)
    stats = logp.new_empty((rows, 2))
    ent = torch.empty_like(logp) if entropy else None
    top = logp.new_empty((rows, k)) if k else None
    idx = targets.new_empty((rows, k)) if k else None
    ws = None
    if size.value:
        ws = workspace
        if not _fits(ws, size.value, dev):
            ws = logits.new_empty((size.value,), dtype=torch.uint8)
    check(_call(dev, lib.kan_token_logprobs, dt, rows, classes, logits.data_ptr(), stride,
                targets.data_ptr(), int(ignore_index), k, logp.data_ptr(), stats.data_ptr(),
                _ptr(ent), _ptr(top), _ptr(idx), _ptr(ws), size.value, _stream(dev)))
    return logp, stats, ent, top, idx


def token_logprobs_backward(logits, targets, stats, dlogp, entropy=None, dentropy=None,
                            ignore_index: int = -100, out=None):
    """The gradient of token_logprobs with respect to the logits
    (kan_token_logprobs_backward) for dlogp [rows] fp32, and for dentropy [rows] fp32 given
    the forward's entropy; stats as token_logprobs returned them.  `out` (like the logits; the
    logits themselves: in place) receives the gradient instead of a fresh tensor."""
    torch = _torch()
    rows, classes, stride = _logits(logits)
    _check_targets(logits, rows, targets)
    if stats is None or stats.dtype != torch.float32 or stats.shape != (rows, 2) or \
            stats.device != logits.device or not stats.is_contiguous():
        raise ValueError("stats must be fp32 [rows, 2], contiguous, on the logits' device")
    _row_values("dlogp, entropy and dentropy", logits, dlogp, entropy, dentropy)
    if dlogp is None or (entropy is None) != (dentropy is None):
        raise ValueError("dlogp is needed, and entropy and dentropy go together")
    if out is None:
        out, ostride = logits.new_empty((rows, classes)), classes
    else:
        if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device:
            raise ValueError("out must match the logits in shape, dtype and device")
        _, _, ostride = _logits(out)
    device = logits.device
    check(_call(device, _library().kan_token_logprobs_backward, _dtype_code(logits), rows,
                classes, logits.data_ptr(), stride, targets.data_ptr(), int(ignore_index),
                stats.data_ptr(), dlogp.data_ptr(), _ptr(entropy), _ptr(dentropy), out.data_ptr(),
                ostride, _stream(device)))
    return out


_dtype_of = operator.attrgetter("dtype")


def _many(grads):
    """Checks a list of tensors: host arrays of their addresses, sizes and dtypes."""
    Tensor = _torch().Tensor
    devices = set(map(Tensor.get_device, grads))
    if len(devices) > 1 or -1 in devices:
        raise ValueError("tensors must live on one GPU")
    if not all(map(Tensor.is_contiguous, grads)):
        raise ValueError("tensors must be contiguous")
    dtypes = list(map(_dtype_of, grads))
    if dtypes.count(dtypes[0]) == len(dtypes):
        codes = array.array("i", (_dtype_code(grads[0]),)) * len(dtypes)
    else:
        codes = array.array("i", map(_dtype_code, grads))
    return (array.array("Q", map(Tensor.data_ptr, grads)),
            array.array("q", map(Tensor.numel, grads)), codes)


def _norm_buffers(count: int, device, workspace):
    torch = _torch()
    size = ctypes.c_size_t(0)
    check(_library().kan_grad_norm_workspace_bytes(count, ctypes.byref(size)))
    if not _fits(workspace, size.value, device):
        workspace = torch.empty(size.value, dtype=torch.uint8, device=device)
    return torch.empty((), dtype=torch.float32, device=device), workspace


def grad_norm(grads: Iterable, workspace=None):
    """The global 2-norm of a list of tensors (fp32 or bf16, of any shapes, on one device):
    a scalar fp32 tensor on the device (kan_grad_norm; nothing is copied to the host)."""
    grads = list(grads)
    if not grads:
        raise ValueError("no tensors")
    ptrs, sizes, dtypes = _many(grads)
    dev = grads[0].device
    norm, ws = _norm_buffers(len(grads), dev, workspace)
    check(_call(dev, _library().kan_grad_norm, len(grads), ptrs.buffer_info()[0],
                sizes.buffer_info()[0], dtypes.buffer_info()[0], ws.data_ptr(), ws.numel(),
                norm.data_ptr(), _stream(dev)))
    return norm


def clip_grad_norm(grads: Iterable, max_norm: float, eps: float = 1e-6, out=None,
                   workspace=None):
    """Scales the tensors by min(1, max_norm / (norm + eps)) with their global 2-norm
    (kan_clip_grad_norm), in place, or into `out`, a list of tensors like them -> the norm
    before scaling, a scalar fp32 tensor on the device (nothing is copied to the host)."""
    grads = list(grads)
    if not grads:
        raise ValueError("no tensors")
    ptrs, sizes, dtypes = _many(grads)
    optrs = ptrs
    if out is not None:
        out = list(out)
        optrs, osizes, odtypes = _many(out)
        if osizes != sizes or odtypes != dtypes or out[0].device != grads[0].device:
            raise ValueError("out must match the gradients in sizes, dtypes and device")
    dev = grads[0].device
    norm, ws = _norm_buffers(len(grads), dev, workspace)
    check(_call(dev, _library().kan_clip_grad_norm, len(grads), ptrs.buffer_info()[0],
                sizes.buffer_info()[0], dtypes.buffer_info()[0], float(max_norm), float(eps),
                optrs.buffer_info()[0], ws.data_ptr(), ws.numel(), norm.data_ptr(), _stream(dev)))
    return norm


# ------------------------------------------------- the two ends of a token model

_MOST = 2 ** 31 - 1  # what a call's 32-bit sizes hold


def _tokens(tokens) -> int:
    if not tokens.is_cuda:
        raise ValueError("tensors must live on the GPU")
    if tokens.dtype != _torch().int64 or not tokens.is_contiguous():
        raise ValueError("tokens must be int64 and contiguous")
    return tokens.numel()


def _matrix(what: str, t, device) -> Tuple[int, int, int]:
    """Checks rows [rows, n] on `device`: (rows, n, elements from row to row)."""
    if t.device != device:
        raise ValueError("tensors must live on one device")
    shape = t.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError(f"{what} must be [rows, n] with n >= 1")
    rows, n = shape
    if rows > _MOST or n > _MOST:
        raise ValueError(f"{what} has more than 2^31 - 1 rows or columns")
    stride, inner = t.stride()
    if rows <= 1:
        stride = n
    if (n > 1 and inner != 1) or stride < n:
        raise ValueError(f"a row of {what} must be contiguous, and rows must not overlap")
    return rows, n, stride


def embedding(tokens, table, scale: float = 1.0, ignore_index: int = -100, dtype=None, out=None):
    """kan_embedding: tokens [...] int64, table [classes, n] (its rows may be padded) -> y [..., n]
    of `dtype` (the table's own by default; a float32 table also gives bfloat16 rows).  `out`
    receives the rows instead of a fresh tensor."""
    torch = _torch()
    rows = _tokens(tokens)
    device = tokens.device
    classes, n, stride = _matrix("the table", table, device)
    shape = tokens.shape + (n,)
    if out is None:
        out = table.new_empty(shape, dtype=table.dtype if dtype is None else dtype)
    elif out.shape != shape or out.device != device or not out.is_contiguous() or \
            out.dtype != (table.dtype if dtype is None else dtype):
        raise ValueError("out must be [..., n] of the rows' dtype, contiguous, on the tokens' device")
    check(_call(device, _library().kan_embedding, _dtype_code(out), _dtype_code(table), rows, classes,
                n, tokens.data_ptr(), int(ignore_index), table.data_ptr(), stride, scale,
                out.data_ptr(), _stream(device)))
    return out


def embedding_backward(tokens, dy, classes: int, scale: float = 1.0, ignore_index: int = -100,
                       dtype=None, base=None, out=None, workspace=None):
    """The gradient of embedding's table (kan_embedding_backward): tokens [...] int64, dy [..., n]
    -> [classes, n] of `dtype` (base's, out's or dy's by default; float32 goes with any dy), `base`
    [classes, n] (None: 0) added: a gradient that the table has already, as a head's weights.
    `out` receives it instead of a fresh tensor, and may be `base` itself.  `workspace` (a uint8
    device tensor) is used when large enough, else a fresh one is taken."""
    torch = _torch()
    rows, device, classes = _tokens(tokens), tokens.device, int(classes)
    if not 1 <= classes <= _MOST:
        raise ValueError("classes must be from 1 to 2^31 - 1")
    if dy.shape[:-1] != tokens.shape or dy.dim() != tokens.dim() + 1:
        raise ValueError("dy must be [..., n] for tokens [...]")
    if dy.dim() != 2:
        if not dy.is_contiguous():
            raise ValueError("dy must be contiguous, or [rows, n]")
        dy = dy.view(rows, dy.shape[-1]) if dy.shape[-1] else dy.reshape(rows, 0)
    _, n, stride = _matrix("dy", dy, device)
    for t in (base, out):
        if dtype is None and t is not None:
            dtype = t.dtype
    dtype = dy.dtype if dtype is None else dtype
    for t in (base, out):
        if t is not None and (t.shape != (classes, n) or t.dtype != dtype or t.device != device or
                              not t.is_contiguous()):
            raise ValueError("base and out must be [classes, n] of one dtype, contiguous, on the "
                             "tokens' device")
    lib, size = _library(), ctypes.c_size_t(0)
    check(lib.kan_embedding_backward_workspace_bytes(rows, classes, n, ctypes.byref(size)))
    if out is None:
        out = dy.new_empty((classes, n), dtype=dtype)
    if not _fits(workspace, size.value, device):
        workspace = dy.new_empty((size.value,), dtype=torch.uint8)
    check(_call(device, lib.kan_embedding_backward, _dtype_code(dy), _dtype_code(out), rows, classes, n,
                tokens.data_ptr(), int(ignore_index), dy.data_ptr(), stride, scale, _ptr(base),
                out.data_ptr(), workspace.data_ptr(), size.value, _stream(device)))
    return out


def _head(x, weight, targets):
    """Checks a head's tensors: the arguments that describe them."""
    if not x.is_cuda:
        raise ValueError("tensors must live on the GPU")
    rows, n, stride = _matrix("x", x, x.device)
    classes, width, wstride = _matrix("the weight", weight, x.device)
    if width != n or weight.dtype != x.dtype:
        raise ValueError("weight must be [classes, n] of x's dtype for x [rows, n]")
    _check_targets(x, rows, targets)
    return (_dtype_code(x), rows, classes, n, x.data_ptr(), stride, weight.data_ptr(), wstride)


def _head_workspace(fn, args, device, workspace):
    torch, size = _torch(), ctypes.c_size_t(0)
    check(fn(*args, ctypes.byref(size)))
    if not _fits(workspace, size.value, device):
        workspace = torch.empty((size.value,), dtype=torch.uint8, device=device)
    return workspace, size.value


def linear_logprobs(x, weight, targets, scale: float = 1.0, best: bool = False,
                    ignore_index: int = -100, workspace=None):
    """kan_linear_logprobs: log probabilities of targets [rows] int64 under the softmax of scale x
    weight^T, for x [rows, n] and weight [classes, n] (rows of both may be padded) -> (logp [rows],
    stats [rows, 2], best [rows] int64 or None: the most probable class), logp and stats fp32.
    stats goes to linear_logprobs_backward.  `workspace` (a uint8 device tensor) is used when large
    enough, else a fresh one is taken."""
    torch = _torch()
    args = _head(x, weight, targets)
    device, rows, lib = x.device, x.shape[0], _library()
    ws, nbytes = _head_workspace(lib.kan_linear_logprobs_workspace_bytes, args, device, workspace)
    logp = x.new_empty((rows,), dtype=torch.float32)
    stats = logp.new_empty((rows, 2))
    at = torch.empty_like(targets) if best else None
    check(_call(device, lib.kan_linear_logprobs, *args, scale, targets.data_ptr(), int(ignore_index),
                logp.data_ptr(), stats.data_ptr(), _ptr(at), ws.data_ptr(), nbytes,
                _stream(device)))
    return logp, stats, at


def linear_logprobs_backward(x, weight, targets, stats, dlogp, scale: float = 1.0,
                             ignore_index: int = -100, need_dx: bool = True, need_dw: bool = True,
                             workspace=None, out=None):
    """Gradients of linear_logprobs (kan_linear_logprobs_backward) for dlogp [rows] fp32; stats as
    linear_logprobs returned them -> (dx [rows, n] or None, dweight [classes, n] or None).  `out`, a
    (dx, dweight) tuple of contiguous tensors, receives the gradients instead of fresh ones.
    `workspace` (a uint8 device tensor) is used when large enough, else a fresh one is taken."""
    torch = _torch()
    args = _head(x, weight, targets)
    device, rows, lib = x.device, x.shape[0], _library()
    if stats is None or stats.dtype != torch.float32 or stats.shape != (rows, 2) or \
            stats.device != device or not stats.is_contiguous():
        raise ValueError("stats must be fp32 [rows, 2], contiguous, on x's device")
    if dlogp is None:
        raise ValueError("dlogp is needed")
    _row_values("dlogp", x, dlogp)
    if not (need_dx or need_dw):
        raise ValueError("nothing to compute")
    if out is not None:
        dx, dw = out
        for t, like in ((dx, x), (dw, weight)):
            if t is not None and (t.shape != like.shape or t.dtype != like.dtype or
                                  t.device != device or not t.is_contiguous()):
                raise ValueError("out tensors must match x and weight and be contiguous")
        dx, dw = dx if need_dx else None, dw if need_dw else None
    else:
        dx = x.new_empty(x.shape) if need_dx else None
        dw = weight.new_empty(weight.shape) if need_dw else None
    ws, nbytes = _head_workspace(lib.kan_linear_logprobs_backward_workspace_bytes, args, device,
                                 workspace)
    check(_call(device, lib.kan_linear_logprobs_backward, *args, scale, targets.data_ptr(),
                int(ignore_index), stats.data_ptr(), dlogp.data_ptr(), _ptr(dx), _ptr(dw),
                ws.data_ptr(), nbytes, _stream(device)))
    return dx, dw
