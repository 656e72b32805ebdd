"""ctypes binding of the token-row operators of libumap_layout.so (include/umap_rows.h).

Argument marshalling only: the work runs in the library's HIP kernels.  Matrices are
two-dimensional torch tensors on the GPU whose columns lie next to each other (rows may be
apart: views of a wider tensor are taken as they are); scales, ids and workspaces are
contiguous tensors.  Streams are ``torch.cuda.Stream`` objects, raw ``hipStream_t`` integers or
None (null stream); tensors that were made on another stream are for the caller to order and to
keep alive.  The calls do not block.  A tensor of another type or shape, or on another GPU than the
current one, raises ValueError, whatever the library refuses :class:`UmapLayoutError`.

Autograd does not record the calls (the gradients are calls of their own).  What they write counts
as changed in place: a backward pass that needs the values from before raises an error.
"""

from __future__ import annotations

import ctypes
import struct

import torch
from torch.autograd.graph import increment_version

from .umap_layout import UmapLayoutError, _check, _stream, lib as _layout_lib

UMAP_F32 = 0
UMAP_F16 = 1
UMAP_BF16 = 2
UMAP_I8 = 3
UMAP_F8 = 4
UMAP_I32 = 8
UMAP_I64 = 9

EXPORTS = ("umap_rows_lookup", "umap_rows_lookup_grad", "umap_rows_lookup_grad_workspace", "umap_rows_norm",
           "umap_rows_norm_grad", "umap_rows_norm_grad_workspace", "umap_rows_layer_norm",
           "umap_rows_layer_norm_grad", "umap_rows_layer_norm_grad_workspace",
           "umap_rows_cross_entropy", "umap_rows_cross_entropy_workspace",
           "umap_rows_cross_entropy_grad", "umap_rows_cross_entropy_grad_workspace",
           "umap_rows_distill", "umap_rows_distill_workspace", "umap_rows_distill_grad", "umap_rows_distill_grad_workspace")

_FLOAT = {torch.float32: UMAP_F32, torch.float16: UMAP_F16, torch.bfloat16: UMAP_BF16}
_ANY = {**_FLOAT, torch.int8: UMAP_I8, torch.float8_e4m3fn: UMAP_F8}
_IDS = {torch.int32: UMAP_I32, torch.int64: UMAP_I64}


class umap_rows(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("scales", ctypes.c_void_p),
        ("rows", ctypes.c_int64),
        ("stride", ctypes.c_int64),
        ("cols", ctypes.c_int32),
        ("type", ctypes.c_int32),
        ("group", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


_lib = None
_call: dict = {}   # the library's functions, taking packed umap_rows
_only = -2         # the GPU's number where the process sees just one: tensors on it are in place
_pack = struct.Struct("@PPqqiiii").pack


def lib() -> ctypes.CDLL:
    """The native library with this module's signatures set."""
    global _lib
    if _lib is None:
        L = _layout_lib()
        M, P, i32, i64, f32 = ctypes.POINTER(umap_rows), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        sig = {
            "umap_rows_lookup": ([M, P, i32, f32, M, P], ctypes.c_int),
            "umap_rows_lookup_grad": ([M, P, i32, f32, M, i32, P, i64, P], ctypes.c_int),
            "umap_rows_lookup_grad_workspace": ([i64, i64, i32], i64),
            "umap_rows_norm": ([M, P, i32, f32, M, M, P, i32, f32, M, P], ctypes.c_int),
            "umap_rows_norm_grad": ([M, M, M, P, i32, f32, M, P, P, i64, P], ctypes.c_int),
            "umap_rows_norm_grad_workspace": ([i64, i32], i64),
            "umap_rows_layer_norm": ([M, M, M, P, i32, P, i32, f32, M, P], ctypes.c_int),
            "umap_rows_layer_norm_grad": ([M, M, M, P, i32, f32, M, P, P, P, i64, P], ctypes.c_int),
            "umap_rows_layer_norm_grad_workspace": ([i64, i32], i64),
            "umap_rows_cross_entropy": ([M, M, P, i32, f32, P, P, P, i64, P], ctypes.c_int),
            "umap_rows_cross_entropy_workspace": ([i64, i64, i32, i32], i64),
            "umap_rows_cross_entropy_grad": ([M, M, P, i32, f32, P, P, f32, M, M, i32, P, i64, P], ctypes.c_int),
            "umap_rows_cross_entropy_grad_workspace": ([i64, i64, i32, i32], i64),
            "umap_rows_distill": ([M, M, P, i32, M, f32, f32, P, P, P, i64, P], ctypes.c_int),
            "umap_rows_distill_workspace": ([i64, i64, i32, i32, i32], i64),
            "umap_rows_distill_grad": ([M, M, P, i32, M, f32, f32, P, P, f32, M, M, i32, P, i64, P], ctypes.c_int),
            "umap_rows_distill_grad_workspace": ([i64, i64, i32, i32, i32], i64),
        }
        for name, (args, result) in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = result
            # a packed structure is passed in a fraction of the time that a Structure takes
            packed = [ctypes.c_char_p if a is M else a for a in args]
            _call[name] = ctypes.CFUNCTYPE(result, *packed)((name, L))
        _lib = L
    return _lib


def _place(x, name: str) -> None:
    """A tensor has to lie on the current GPU, which is where the kernels run."""
    global _only
    at = x.get_device()
    if at < 0:
        raise ValueError(f"{name} must be a GPU tensor, got one on {x.device}")
    here = torch.cuda.current_device()
    if at != here:
        raise ValueError(f"{name} lies on GPU {at}, the current one is {here}")
    if torch.cuda.device_count() == 1:
        _only = at


def _rows(x, name: str, types: dict, scales=None, group: int = 0) -> tuple:
    """A matrix as a packed umap_rows, its rows and its columns."""
    kind = types.get(x.dtype)
    if kind is None:
        raise ValueError(f"{name} must not hold {x.dtype}")
    if x.get_device() != _only:
        _place(x, name)
    if x.dim() != 2:
        raise ValueError(f"{name} must be two-dimensional")
    rows, cols = x.shape
    stride, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: the columns must lie next to each other")
    at = 0
    if scales is not None:
        at = _flat(scales, f"{name}'s scales", torch.float32, rows * (-(-cols // group) if group > 0 else 1))
    return _pack(x.data_ptr(), at, rows, stride, cols, kind, group, 0), rows, cols


def _flat(x, name: str, dtype, count: int) -> int:
    """Address of a contiguous GPU tensor of `count` elements at least (`dtype` None: any type)."""
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name} must hold {dtype}, got {x.dtype}")
    if x.get_device() != _only:
        _place(x, name)
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if x.numel() < count:
        raise ValueError(f"{name} holds {x.numel()} elements, the call needs {count}")
    return x.data_ptr()


def _id_args(ids, n: int) -> tuple:
    if ids is None:
        return None, 0
    kind = _IDS.get(ids.dtype)
    if kind is None:
        raise ValueError(f"ids must hold int32 or int64, got {ids.dtype}")
    if ids.numel() != n:
        raise ValueError(f"{ids.numel()} ids for {n} rows")
    return _flat(ids, "ids", None, n), kind


def _weight_args(weight, cols: int, name: str = "weight") -> tuple:
    if weight is None:
        return None, 0
    kind = _FLOAT.get(weight.dtype)
    if kind is None:
        raise ValueError(f"{name} must hold a float type, got {weight.dtype}")
    if weight.numel() != cols:
        raise ValueError(f"{weight.numel()} {name}{'' if name.endswith('s') else 's'} for {cols} columns")
    return _flat(weight, name, None, cols), kind


def _work(workspace) -> tuple:
    if workspace is None:
        return None, 0
    return _flat(workspace, "workspace", None, 0), workspace.numel() * workspace.element_size()


def _count(bytes_: int) -> int:
    _check(min(bytes_, 0))
    return bytes_


def umap_rows_lookup(table, ids, out, scale: float = 1.0, table_scales=None, group: int = 0, stream=None) -> None:
    """out[t] = scale * table[ids[t]] (zeros where an id is outside the table; ids None: table row t).

    An int8 or float8_e4m3fn table comes with `table_scales`, one fp32 per row and `group` columns (32, 64 or 128;
    0: one per row)."""
    t, _, _ = _rows(table, "table", _ANY, table_scales, group)
    o, n, _ = _rows(out, "out", _FLOAT)
    at, kind = _id_args(ids, n)
    lib()
    _check(_call["umap_rows_lookup"](t, at, kind, scale, o, _stream(stream)))
    increment_version(out)


def umap_rows_lookup_grad_workspace(n: int, rows: int, cols: int) -> int:
    """Bytes of umap_rows_lookup_grad's workspace."""
    return _count(lib().umap_rows_lookup_grad_workspace(n, rows, cols))


def umap_rows_lookup_grad(dout, ids, grad, workspace, scale: float = 1.0, accumulate: bool = False,
                          stream=None) -> None:
    """grad[v] = scale * (sum of dout[t] over ids[t] = v); with `accumulate` added to grad's rows."""
    d, n, _ = _rows(dout, "dout", _FLOAT)
    g, _, _ = _rows(grad, "grad", _FLOAT)
    at, kind = _id_args(ids, n)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_lookup_grad"](d, at, kind, scale, g, 1 if accumulate else 0, work, size, _stream(stream)))
    increment_version(grad)


def umap_rows_norm(x, y, weight=None, residual=None, h=None, ids=None, scale: float = 1.0, y_scales=None,
                   group: int = 0, eps: float = 1e-6, stream=None) -> None:
    """h = scale * x (or scale * x[ids]) + residual; y = h / sqrt(mean h^2 + eps) * weight, row by row.

    An int8 or float8_e4m3fn y is written with `y_scales` (see umap_rows_lookup).  h may be the residual itself or,
    without ids, x."""
    X, _, cols = _rows(x, "x", _FLOAT)
    Y, n, _ = _rows(y, "y", _ANY, y_scales, group)
    R = None if residual is None else _rows(residual, "residual", _FLOAT)[0]
    H = None if h is None else _rows(h, "h", _FLOAT)[0]
    at, kind = _id_args(ids, n)
    w, w_kind = _weight_args(weight, cols)
    lib()
    _check(_call["umap_rows_norm"](X, at, kind, scale, R, H, w, w_kind, eps, Y, _stream(stream)))
    increment_version([x for x in (y, y_scales, h) if x is not None])


def umap_rows_norm_grad_workspace(n: int, cols: int) -> int:
    """Bytes of umap_rows_norm_grad's workspace."""
    return _count(lib().umap_rows_norm_grad_workspace(n, cols))


def umap_rows_norm_grad(dy, h, dx, weight=None, dh=None, dweight=None, workspace=None, eps: float = 1e-6,
                        stream=None) -> None:
    """Gradient of y = h / sqrt(mean h^2 + eps) * weight for h (plus `dh`, what reaches h otherwise), into dx (which
    may be dy or dh itself), and for the weight, into dweight (fp32; needs the workspace).

    dx is the residual's gradient too; x's is dx times umap_rows_norm's scale."""
    Y, _, cols = _rows(dy, "dy", _FLOAT)
    H, _, _ = _rows(h, "h", _FLOAT)
    X, _, _ = _rows(dx, "dx", _FLOAT)
    U = None if dh is None else _rows(dh, "dh", _FLOAT)[0]
    w, w_kind = _weight_args(weight, cols)
    dw = None if dweight is None else _flat(dweight, "dweight", torch.float32, cols)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_norm_grad"](Y, H, U, w, w_kind, eps, X, dw, work, size, _stream(stream)))
    increment_version(dx if dweight is None else (dx, dweight))


def umap_rows_layer_norm(x, y, weight=None, bias=None, residual=None, h=None, eps: float = 1e-5, stream=None) -> None:
    """h = x + residual; y = (h - mean h) / sqrt(mean (h - mean h)^2 + eps) * weight + bias, row by row.

    h may be x or the residual itself."""
    X, _, cols = _rows(x, "x", _FLOAT)
    Y, _, _ = _rows(y, "y", _FLOAT)
    S = None if residual is None else _rows(residual, "residual", _FLOAT)[0]
    H = None if h is None else _rows(h, "h", _FLOAT)[0]
    w, w_kind = _weight_args(weight, cols)
    b, b_kind = _weight_args(bias, cols, "bias")
    lib()
    _check(_call["umap_rows_layer_norm"](X, S, H, w, w_kind, b, b_kind, eps, Y, _stream(stream)))
    increment_version(y if h is None else (y, h))


def umap_rows_layer_norm_grad_workspace(n: int, cols: int) -> int:
    """Bytes of umap_rows_layer_norm_grad's workspace."""
    return _count(lib().umap_rows_layer_norm_grad_workspace(n, cols))


def umap_rows_layer_norm_grad(dy, h, dx, weight=None, dh=None, dweight=None, dbias=None, workspace=None, eps: float = 1e-5,
                              stream=None) -> None:
    """Gradient of umap_rows_layer_norm for h (plus `dh`, what reaches h otherwise), into dx (which may be dy or dh
    itself), for the weight, into dweight, and for the bias, into dbias (both fp32; they need the workspace)."""
    Y, _, cols = _rows(dy, "dy", _FLOAT)
    H, _, _ = _rows(h, "h", _FLOAT)
    X, _, _ = _rows(dx, "dx", _FLOAT)
    U = None if dh is None else _rows(dh, "dh", _FLOAT)[0]
    w, w_kind = _weight_args(weight, cols)
    dw = None if dweight is None else _flat(dweight, "dweight", torch.float32, cols)
    db = None if dbias is None else _flat(dbias, "dbias", torch.float32, cols)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_layer_norm_grad"](Y, H, U, w, w_kind, eps, X, dw, db, work, size, _stream(stream)))
    increment_version([x for x in (dx, dweight, dbias) if x is not None])


def _type(dtype) -> int:
    kind = _FLOAT.get(dtype)
    if kind is None:
        raise ValueError(f"rows must not hold {dtype}")
    return kind


def _head_ids(ids, n: int, name: str) -> tuple:
    if ids is None:
        raise ValueError(f"{name} must be given")
    kind = _IDS.get(ids.dtype)
    if kind is None:
        raise ValueError(f"{name} must hold int32 or int64, got {ids.dtype}")
    if ids.numel() != n:
        raise ValueError(f"{name} holds {ids.numel()} ids, the call needs {n}")
    return _flat(ids, name, None, n), kind


def _head_grads(dh, dtable) -> tuple:
    return (None if dh is None else _rows(dh, "dh", _FLOAT)[0], None if dtable is None else _rows(dtable, "dtable", _FLOAT)[0])


def umap_rows_cross_entropy_workspace(n: int, rows: int, cols: int, dtype) -> int:
    """Bytes of umap_rows_cross_entropy's workspace, for n rows and a table of rows x cols of `dtype`."""
    return _count(lib().umap_rows_cross_entropy_workspace(n, rows, cols, _type(dtype)))


def umap_rows_cross_entropy(h, table, targets, loss, lse, workspace, scale: float = 1.0, stream=None) -> None:
    """loss[t] = lse[t] - z[t, targets[t]], lse = logsumexp(z), z = scale * h @ table.T (which is not kept).

    Rows whose target lies outside the table have loss 0."""
    H, n, _ = _rows(h, "h", _FLOAT)
    W, _, _ = _rows(table, "table", _FLOAT)
    at, kind = _head_ids(targets, n, "targets")
    f32 = torch.float32
    out, sums = _flat(loss, "loss", f32, n), _flat(lse, "lse", f32, n)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_cross_entropy"](H, W, at, kind, scale, out, sums, work, size, _stream(stream)))
    increment_version((loss, lse))


def umap_rows_cross_entropy_grad_workspace(n: int, rows: int, cols: int, dtype) -> int:
    """Bytes of umap_rows_cross_entropy_grad's workspace."""
    return _count(lib().umap_rows_cross_entropy_grad_workspace(n, rows, cols, _type(dtype)))


def umap_rows_cross_entropy_grad(h, table, targets, lse, workspace, dh=None, dtable=None, dloss=None, dscale: float = 1.0,
                                 scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """Gradient of dscale * sum(dloss * loss) for h, into dh, and for the table, into dtable (with `accumulate` added to
    it); dloss None: ones.  Either may be left out.  Rows without a target and rows of weight 0 take no part."""
    H, n, _ = _rows(h, "h", _FLOAT)
    W, _, _ = _rows(table, "table", _FLOAT)
    at, kind = _head_ids(targets, n, "targets")
    sums = _flat(lse, "lse", torch.float32, n)
    weights = None if dloss is None else _flat(dloss, "dloss", torch.float32, n)
    dH, dW = _head_grads(dh, dtable)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_cross_entropy_grad"](H, W, at, kind, scale, sums, weights, dscale, dH, dW,
                                                 1 if accumulate else 0, work, size, _stream(stream)))
    increment_version([x for x in (dh, dtable) if x is not None])


def umap_rows_distill_workspace(n: int, rows: int, cols: int, k: int, dtype) -> int:
    """Bytes of umap_rows_distill's workspace, for n rows with k tokens each and a table of rows x cols of `dtype`."""
    return _count(lib().umap_rows_distill_workspace(n, rows, cols, k, _type(dtype)))


def umap_rows_distill(h, table, ids, teacher, loss, lse, workspace, scale: float = 1.0, teacher_scale: float = 1.0,
                      stream=None) -> None:
    """loss[t] = sum over v of q[t, v] * (log q[t, v] - log p[t, v]), q = softmax(teacher_scale * teacher) over the row's
    tokens ids[t] (of a token that comes twice the sum), p = softmax(scale * h @ table.T); lse as for
    umap_rows_cross_entropy.

    Places whose id lies outside the table are empty; a row with empty places only has loss 0."""
    H, n, _ = _rows(h, "h", _FLOAT)
    W, _, _ = _rows(table, "table", _FLOAT)
    A, _, k = _rows(teacher, "teacher", _FLOAT)
    at, kind = _head_ids(ids, n * k, "ids")
    f32 = torch.float32
    out, sums = _flat(loss, "loss", f32, n), _flat(lse, "lse", f32, n)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_distill"](H, W, at, kind, A, scale, teacher_scale, out, sums, work, size, _stream(stream)))
    increment_version((loss, lse))


def umap_rows_distill_grad_workspace(n: int, rows: int, cols: int, k: int, dtype) -> int:
    """Bytes of umap_rows_distill_grad's workspace."""
    return _count(lib().umap_rows_distill_grad_workspace(n, rows, cols, k, _type(dtype)))


def umap_rows_distill_grad(h, table, ids, teacher, lse, workspace, dh=None, dtable=None, dloss=None, dscale: float = 1.0,
                           scale: float = 1.0, teacher_scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """Gradient of dscale * sum(dloss * loss) of umap_rows_distill for h and the table; the teacher is constant."""
    H, n, _ = _rows(h, "h", _FLOAT)
    W, _, _ = _rows(table, "table", _FLOAT)
    A, _, k = _rows(teacher, "teacher", _FLOAT)
    at, kind = _head_ids(ids, n * k, "ids")
    sums = _flat(lse, "lse", torch.float32, n)
    weights = None if dloss is None else _flat(dloss, "dloss", torch.float32, n)
    dH, dW = _head_grads(dh, dtable)
    work, size = _work(workspace)
    lib()
    _check(_call["umap_rows_distill_grad"](H, W, at, kind, A, scale, teacher_scale, sums, weights, dscale, dH, dW,
                                           1 if accumulate else 0, work, size, _stream(stream)))
    increment_version([x for x in (dh, dtable) if x is not None])


__all__ = [*EXPORTS, "UmapLayoutError", "umap_rows"]
