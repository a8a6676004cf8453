"""Binding of libaccept's stage operators (include/accept_stage.h): layer norm, blocks in 8-bit floating point, their product.

Argument marshalling only, as in binding.py: tensors are checked on the host against the descriptor, outputs that are not
given are allocated with ``torch.empty``, and the kernels run on the current stream of the current device, where the tensors
have to be.  csrc/native.cpp makes the same checks and calls without the interpreter; whatever it does not take comes to
the code here, which says what is wrong.  Codes are ``torch.float8_e4m3fn`` or ``torch.float8_e5m2``, scales ``torch.float8_e8m0fnu``.
"""
from __future__ import annotations

import ctypes

from . import binding as B
import torch  # after the binding, which decides the order in which the runtimes are loaded

E4M3, E5M2 = 0, 1
BLOCK = 128
_CODE_TYPES = (torch.float8_e4m3fn, torch.float8_e5m2)  # by E4M3 / E5M2
_SCALE_TYPE = torch.float8_e8m0fnu


class NormDesc(ctypes.Structure):
    """Mirror of accept_norm_desc."""
    _fields_ = [
        ("x_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32), ("param_dtype", ctypes.c_int32), ("code", ctypes.c_int32),
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
        ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64), ("dx_stride", ctypes.c_int64), ("eps", ctypes.c_double),
    ]


class BlockDesc(ctypes.Structure):
    """Mirror of accept_block_desc."""
    _fields_ = [
        ("in_dtype", ctypes.c_int32), ("code", ctypes.c_int32), ("group", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("x_stride", ctypes.c_int64),
    ]


class MatmulDesc(ctypes.Structure):
    """Mirror of accept_matmul_desc."""
    _fields_ = [
        ("out_dtype", ctypes.c_int32), ("a_code", ctypes.c_int32), ("b_code", ctypes.c_int32),
        ("a_group", ctypes.c_int32), ("b_group", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("m", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
        ("a_stride", ctypes.c_int64), ("b_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64),
    ]


def _declare(lib):
    P, V = ctypes.POINTER, ctypes.c_void_p
    sz = P(ctypes.c_size_t)
    for name, args in (("accept_layer_norm", [P(NormDesc), V, V, V, V, V, V]),
                       ("accept_layer_norm_quantize", [P(NormDesc), V, V, V, V, V, V, V]),
                       ("accept_norm_workspace_size", [P(NormDesc), sz]),
                       ("accept_layer_norm_backward", [P(NormDesc), V, V, V, V, V, V, V, V, V]),
                       ("accept_block_quantize", [P(BlockDesc), V, V, V, V, V, V]),
                       ("accept_matmul_workspace_size", [P(MatmulDesc), sz]),
                       ("accept_block_matmul", [P(MatmulDesc), V, V, V, V, V, V, V])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ctypes.c_int
    lib.accept_block_stride.argtypes = [ctypes.c_int64]
    lib.accept_block_stride.restype = ctypes.c_int64
    return lib


lib = _declare(B.lib)
_native = B._native


# ------------------------------------------------------------------------------- descriptors
def make_norm_desc(rows, cols, x_dtype=B.F32, y_dtype=B.F32, param_dtype=B.F32, eps=1e-5, code=E4M3, x_stride=0, y_stride=0,
                   dx_stride=0):
    return NormDesc(int(x_dtype), int(y_dtype), int(param_dtype), int(code), int(rows), int(cols), int(x_stride), int(y_stride),
                    int(dx_stride), float(eps))


def make_block_desc(rows, cols, group=1, in_dtype=B.F32, code=E4M3, x_stride=0):
    return BlockDesc(int(in_dtype), int(code), int(group), 0, int(rows), int(cols), int(x_stride))


def make_matmul_desc(m, n, k, out_dtype=B.F32, a_code=E4M3, b_code=E4M3, a_group=1, b_group=BLOCK, a_stride=0, b_stride=0,
                     y_stride=0):
    return MatmulDesc(int(out_dtype), int(a_code), int(b_code), int(a_group), int(b_group), 0, int(m), int(n), int(k),
                      int(a_stride), int(b_stride), int(y_stride))


def accept_block_stride(length):
    return lib.accept_block_stride(int(length))


def _size_of(function, desc, where):
    b = ctypes.c_size_t(0)
    B._check(function(ctypes.byref(desc), ctypes.byref(b)), where)
    return b.value


def accept_norm_workspace_size(desc):
    return _size_of(lib.accept_norm_workspace_size, desc, "accept_norm_workspace_size")


def accept_matmul_workspace_size(desc):
    return _size_of(lib.accept_matmul_workspace_size, desc, "accept_matmul_workspace_size")


# ------------------------------------------------------------------------------------ checks
def _refuse(where, what, why):
    raise B.AcceptError(B.INVALID_ARG, "%s: %s %s" % (where, what, why))


def _check_desc(desc, kind, where):
    if type(desc) is not kind:
        _refuse(where, "desc", "is not a %s" % kind.__name__)


def _check_place(t, where, what, dtype):
    if t is None:
        _refuse(where, what, "is missing")
    if not t.is_cuda:
        _refuse(where, what, "is not a device tensor")
    if t.device.index != torch.cuda.current_device():
        _refuse(where, what, "is on %s, the current device is %d" % (t.device, torch.cuda.current_device()))
    if t.dtype is not dtype:
        _refuse(where, what, "has dtype %s, the descriptor says %s" % (t.dtype, dtype))


def _check_matrix(t, where, what, dtype, rows, cols, stride):
    """(rows, cols) with rows `stride` apart, or, where that is `cols`, any contiguous tensor of as many elements."""
    _check_place(t, where, what, dtype)
    stride = stride or cols
    if t.dim() == 2 and t.shape[0] == rows and t.shape[1] == cols:
        if (rows <= 1 or cols == 0 or t.stride(0) == stride) and (cols <= 1 or rows == 0 or t.stride(1) == 1):
            return
        _refuse(where, what, "has strides %s, the descriptor says (%d, 1)" % (tuple(t.stride()), stride))
    if t.numel() != rows * cols:
        _refuse(where, what, "has %d elements, the descriptor says %d x %d" % (t.numel(), rows, cols))
    if stride != cols or not t.is_contiguous():
        _refuse(where, what, "is neither contiguous nor %d x %d" % (rows, cols))


def _check_flat(t, where, what, dtype, elems):
    _check_place(t, where, what, dtype)
    if t.numel() != elems:
        _refuse(where, what, "has %d elements, %d needed" % (t.numel(), elems))
    if not t.is_contiguous():
        _refuse(where, what, "is not contiguous")


def _check_table(t, where, what, dtype, rows, cols):
    """(rows, cols), contiguous: in another order they would be read as another's."""
    _check_place(t, where, what, dtype)
    if tuple(t.shape) != (rows, cols):
        _refuse(where, what, "is %s, %s needed" % (tuple(t.shape), (rows, cols)))
    if not t.is_contiguous():
        _refuse(where, what, "is not contiguous")


def _check_codes(t, where, what, dtype, rows, cols, stride):
    """(rows, cols) codes, rows `stride` bytes apart (one row: any) and readable up to a multiple of 16."""
    _check_place(t, where, what, dtype)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        _refuse(where, what, "is %s, the descriptor says %d x %d" % (tuple(t.shape), rows, cols))
    if rows == 0 or cols == 0:
        return
    if (rows > 1 and t.stride(0) != stride) or (cols > 1 and t.stride(1) != 1):
        _refuse(where, what, "has strides %s, the descriptor says (%d, 1)" % (tuple(t.stride()), stride))
    if t.data_ptr() % 16:
        _refuse(where, what, "is not 16-byte aligned")
    if t.storage_offset() + (rows - 1) * stride + (cols + 15) // 16 * 16 > t.untyped_storage().nbytes():
        raise B.AcceptError(B.BUFFER_TOO_SMALL, "%s: %s's last row is not readable up to a multiple of 16 bytes" % (where, what))


def _check_workspace(t, where, nbytes):
    if t is None or not t.is_cuda or not t.is_contiguous():
        _refuse(where, "workspace", "is not a contiguous device tensor")
    if t.device.index != torch.cuda.current_device():
        _refuse(where, "workspace", "is on %s" % t.device)
    if B._nbytes(t) < nbytes:
        raise B.AcceptError(B.BUFFER_TOO_SMALL, "%s: workspace has %d bytes, %d needed" % (where, B._nbytes(t), nbytes))


def _empty(size, dtype, device):
    return torch.empty(size, dtype=dtype, device=device)


def _empty_codes(rows, cols, dtype, device):
    return torch.empty((rows, accept_block_stride(cols)), dtype=dtype, device=device)[:, :cols]


def _blocks(length):
    return (length + BLOCK - 1) // BLOCK


# ----------------------------------------------------------------------------------- operators
def _check_norm_inputs(where, desc, x, weight, bias):
    _check_desc(desc, NormDesc, where)
    accept_norm_workspace_size(desc)  # raises on a bad descriptor
    _check_matrix(x, where, "x", B._DTYPES[desc.x_dtype], desc.rows, desc.cols, desc.x_stride)
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is not None:
            _check_flat(t, where, what, B._DTYPES[desc.param_dtype], desc.cols)


def accept_layer_norm(desc, x, weight=None, bias=None, y=None, stats=None):
    """Enqueue a layer norm of x's rows on the current stream; returns (y, stats).  y has x's shape, or is (rows, cols)
    where its rows are further apart; stats (2, rows) float32 are the means and reciprocal deviations that the backward
    pass takes."""
    if type(desc) is NormDesc:
        got = _native.layer_norm(desc, x, weight, bias, y, stats)
        if type(got) is tuple:
            return got
        if got > 0:
            raise B.AcceptError(got, "accept_layer_norm")
    where = "accept_layer_norm"
    _check_norm_inputs(where, desc, x, weight, bias)
    if y is None:
        if desc.y_stride in (0, desc.cols):
            y = _empty(x.shape, B._DTYPES[desc.y_dtype], x.device)
        else:
            y = _empty((desc.rows, desc.y_stride), B._DTYPES[desc.y_dtype], x.device)[:, :desc.cols]
    if stats is None:
        stats = _empty((2, desc.rows), torch.float32, x.device)
    _check_matrix(y, where, "y", B._DTYPES[desc.y_dtype], desc.rows, desc.cols, desc.y_stride)
    _check_table(stats, where, "stats", torch.float32, 2, desc.rows)
    B._check(lib.accept_layer_norm(ctypes.byref(desc), B._ptr(x), B._ptr(weight), B._ptr(bias), B._ptr(y), B._ptr(stats),
                                   B._stream_handle()), where)
    return y, stats


def accept_layer_norm_quantize(desc, x, weight=None, bias=None, codes=None, scales=None, stats=None):
    """The same with y as codes (rows, cols) and scales (blocks of columns, rows), as accept_block_quantize makes them
    from the float32 y; returns (codes, scales, stats)."""
    if type(desc) is NormDesc:
        got = _native.layer_norm_quantize(desc, x, weight, bias, codes, scales, stats)
        if type(got) is tuple:
            return got
        if got > 0:
            raise B.AcceptError(got, "accept_layer_norm_quantize")
    where = "accept_layer_norm_quantize"
    _check_norm_inputs(where, desc, x, weight, bias)
    if codes is None:
        codes = _empty_codes(desc.rows, desc.cols, _CODE_TYPES[desc.code], x.device)
    if scales is None:
        scales = _empty((_blocks(desc.cols), desc.rows), _SCALE_TYPE, x.device)
    if stats is None:
        stats = _empty((2, desc.rows), torch.float32, x.device)
    _check_out_codes(codes, where, "codes", _CODE_TYPES[desc.code], desc.rows, desc.cols)
    _check_table(scales, where, "scales", _SCALE_TYPE, _blocks(desc.cols), desc.rows)
    _check_table(stats, where, "stats", torch.float32, 2, desc.rows)
    B._check(lib.accept_layer_norm_quantize(ctypes.byref(desc), B._ptr(x), B._ptr(weight), B._ptr(bias), B._ptr(codes),
                                            B._ptr(scales), B._ptr(stats), B._stream_handle()), where)
    return codes, scales, stats


def accept_layer_norm_backward(desc, dy, x, weight, stats, dx=None, dweight=None, dbias=None, need_weight=True, need_bias=True,
                               workspace=None):
    """Gradients of accept_layer_norm: (dx, dweight, dbias); None where need_weight or need_bias is false.  weight None: ones."""
    if type(desc) is NormDesc:
        got = _native.layer_norm_backward(desc, dy, x, weight, stats, dx, dweight, dbias, need_weight, need_bias, workspace)
        if type(got) is tuple:
            return got
        if got > 0:
            raise B.AcceptError(got, "accept_layer_norm_backward")
    where = "accept_layer_norm_backward"
    _check_norm_inputs(where, desc, x, weight, None)
    _check_matrix(dy, where, "dy", B._DTYPES[desc.y_dtype], desc.rows, desc.cols, desc.y_stride)
    _check_table(stats, where, "stats", torch.float32, 2, desc.rows)
    if dx is None:
        if desc.dx_stride in (0, desc.cols):
            dx = _empty(x.shape, x.dtype, x.device)
        else:
            dx = _empty((desc.rows, desc.dx_stride), x.dtype, x.device)[:, :desc.cols]
    param = B._DTYPES[desc.param_dtype]
    dweight = (_empty(desc.cols, param, x.device) if dweight is None else dweight) if need_weight else None
    dbias = (_empty(desc.cols, param, x.device) if dbias is None else dbias) if need_bias else None
    _check_matrix(dx, where, "dx", B._DTYPES[desc.x_dtype], desc.rows, desc.cols, desc.dx_stride)
    for t, what in ((dweight, "dweight"), (dbias, "dbias")):
        if t is not None:
            _check_flat(t, where, what, param, desc.cols)
    if need_weight or need_bias:
        nbytes = accept_norm_workspace_size(desc)
        if workspace is None:
            workspace = _empty(nbytes, torch.uint8, x.device)
        _check_workspace(workspace, where, nbytes)
    B._check(lib.accept_layer_norm_backward(ctypes.byref(desc), B._ptr(dy), B._ptr(x), B._ptr(weight), B._ptr(stats), B._ptr(dx),
                                            B._ptr(dweight), B._ptr(dbias), B._ptr(workspace), B._stream_handle()), where)
    return dx, dweight, dbias


def _check_out_codes(t, where, what, dtype, rows, cols):
    """(rows, cols) codes whose rows are accept_block_stride(cols) bytes apart and as long."""
    stride = accept_block_stride(cols)
    _check_codes(t, where, what, dtype, rows, cols, stride)
    if rows and cols and t.storage_offset() + rows * stride > t.untyped_storage().nbytes():
        raise B.AcceptError(B.BUFFER_TOO_SMALL, "%s: %s's last row ends before %d bytes" % (where, what, stride))


def accept_block_quantize(desc, x, rowwise=True, colwise=False, codes=None, scales=None, codes_t=None, scales_t=None):
    """x's codes and scales along its rows, along its columns (transposed), or both from one read.

    Returns (codes, scales, codes_t, scales_t), None for what is not wanted.  codes: (rows, cols), scales: (blocks of 128
    columns, rows, or blocks of 128 rows for group 128); codes_t: (cols, rows), scales_t: (blocks of rows, columns or blocks
    of columns)."""
    if type(desc) is BlockDesc:
        got = _native.block_quantize(desc, x, rowwise, colwise, codes, scales, codes_t, scales_t)
        if type(got) is tuple:
            return got
        if got > 0:
            raise B.AcceptError(got, "accept_block_quantize")
    where = "accept_block_quantize"
    _check_desc(desc, BlockDesc, where)
    if (desc.in_dtype not in (B.F32, B.BF16) or desc.code not in (E4M3, E5M2) or desc.group not in (1, BLOCK) or desc.rows < 0
            or desc.cols < 0):
        raise B.AcceptError(B.INVALID_ARG, where + ": bad descriptor")
    rows, cols, group = desc.rows, desc.cols, desc.group
    _check_matrix(x, where, "x", B._DTYPES[desc.in_dtype], rows, cols, desc.x_stride)
    if not rowwise and not colwise:
        _refuse(where, "codes", "are wanted along neither rows nor columns")
    code = _CODE_TYPES[desc.code]
    if rowwise:
        codes = _empty_codes(rows, cols, code, x.device) if codes is None else codes
        scales = _empty((_blocks(cols), -(-rows // group)), _SCALE_TYPE, x.device) if scales is None else scales
        _check_out_codes(codes, where, "codes", code, rows, cols)
        _check_table(scales, where, "scales", _SCALE_TYPE, _blocks(cols), -(-rows // group))
    else:
        codes = scales = None
    if colwise:
        codes_t = _empty_codes(cols, rows, code, x.device) if codes_t is None else codes_t
        scales_t = _empty((_blocks(rows), -(-cols // group)), _SCALE_TYPE, x.device) if scales_t is None else scales_t
        _check_out_codes(codes_t, where, "codes_t", code, cols, rows)
        _check_table(scales_t, where, "scales_t", _SCALE_TYPE, _blocks(rows), -(-cols // group))
    else:
        codes_t = scales_t = None
    B._check(lib.accept_block_quantize(ctypes.byref(desc), B._ptr(x), B._ptr(codes), B._ptr(scales), B._ptr(codes_t),
                                       B._ptr(scales_t), B._stream_handle()), where)
    return codes, scales, codes_t, scales_t


def accept_block_matmul(desc, a, a_scales, b, b_scales, y=None, workspace=None):
    """y = a b^T of codes and scales (see accept_block_quantize), a (m, k), b (n, k); returns y (m, n)."""
    if type(desc) is MatmulDesc:
        got = _native.block_matmul(desc, a, a_scales, b, b_scales, y, workspace)
        if type(got) is tuple:
            return got[0]
        if got > 0:
            raise B.AcceptError(got, "accept_block_matmul")
    where = "accept_block_matmul"
    _check_desc(desc, MatmulDesc, where)
    nbytes = accept_matmul_workspace_size(desc)  # raises on a bad descriptor
    m, n, k = desc.m, desc.n, desc.k
    whole = accept_block_stride(k)
    _check_codes(a, where, "a", _CODE_TYPES[desc.a_code], m, k, desc.a_stride or whole)
    _check_codes(b, where, "b", _CODE_TYPES[desc.b_code], n, k, desc.b_stride or whole)
    _check_table(a_scales, where, "a_scales", _SCALE_TYPE, _blocks(k), -(-m // desc.a_group))
    _check_table(b_scales, where, "b_scales", _SCALE_TYPE, _blocks(k), -(-n // desc.b_group))
    out = B._DTYPES[desc.out_dtype]
    if y is None:
        y = _empty((m, n), out, a.device) if desc.y_stride in (0, n) else _empty((m, desc.y_stride), out, a.device)[:, :n]
    _check_matrix(y, where, "y", out, m, n, desc.y_stride)
    if nbytes:
        if workspace is None:
            workspace = _empty(nbytes, torch.uint8, a.device)
        _check_workspace(workspace, where, nbytes)
    else:
        workspace = None
    B._check(lib.accept_block_matmul(ctypes.byref(desc), B._ptr(a), B._ptr(a_scales), B._ptr(b), B._ptr(b_scales), B._ptr(y),
                                     B._ptr(workspace), B._stream_handle()), where)
    return y
