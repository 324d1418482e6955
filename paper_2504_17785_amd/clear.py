"""Binding of include/silenzio_clear.h: products of 8-bit integers, layers with 4-bit weights, softmax cross entropy of a linear layer,
orthogonalised updates, gradients clipped by their norm.

As in the rest of the binding the functions check their arguments, hand pointers and the current stream to the library and return at once.
Matrices are CUDA tensors on the current device with unit stride along their rows (any distance between rows).  Workspaces
come from torch's allocator on the current stream, so that their memory is not given away before the call's work on it is done.

The gradients are functions of their own (matmul_i8_grad, linear_i4_grad, linear_ce_grad) and autograd does not know them: results of tensors that require
a gradient raise an error when a backward pass comes to them."""
from __future__ import annotations

import ctypes
import functools

import torch

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_E_TOO_LARGE = -5


class SlzI8Shape(ctypes.Structure):
    """slz_i8_shape of include/silenzio_clear.h."""
    _fields_ = [("m", ctypes.c_uint32), ("n", ctypes.c_uint32), ("k", ctypes.c_uint32), ("type", ctypes.c_int),
                ("ld_a", ctypes.c_int64), ("ld_b", ctypes.c_int64), ("ld_y", ctypes.c_int64)]


class SlzCeShape(ctypes.Structure):
    """slz_ce_shape of include/silenzio_clear.h."""
    _fields_ = [("tokens", ctypes.c_uint32), ("inner", ctypes.c_uint32), ("vocab", ctypes.c_uint32), ("type", ctypes.c_int),
                ("ld_h", ctypes.c_int64), ("ld_w", ctypes.c_int64), ("ld_dh", ctypes.c_int64), ("ld_dw", ctypes.c_int64),
                ("ignore_index", ctypes.c_int64)]


class SlzI4Shape(ctypes.Structure):
    """slz_i4_shape of include/silenzio_clear.h."""
    _fields_ = [("m", ctypes.c_uint32), ("n", ctypes.c_uint32), ("k", ctypes.c_uint32), ("type", ctypes.c_int), ("group", ctypes.c_uint32),
                ("ld_x", ctypes.c_int64), ("ld_q", ctypes.c_int64), ("ld_scale", ctypes.c_int64), ("ld_y", ctypes.c_int64)]


class SlzGradTensor(ctypes.Structure):
    """slz_grad_tensor of include/silenzio_clear.h."""
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32),
                ("ld_g", ctypes.c_int64), ("ld_out", ctypes.c_int64), ("type", ctypes.c_int)]


class SlzOrthShape(ctypes.Structure):
    """slz_orth_shape of include/silenzio_clear.h."""
    _fields_ = [("batch", ctypes.c_uint32), ("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32), ("type", ctypes.c_int),
                ("ld_g", ctypes.c_int64), ("stride_g", ctypes.c_int64), ("ld_out", ctypes.c_int64), ("stride_out", ctypes.c_int64),
                ("steps", ctypes.c_uint32), ("a", ctypes.c_float), ("b", ctypes.c_float), ("c", ctypes.c_float), ("eps", ctypes.c_float)]


def declare(L):
    vp, u32, sz, i64, i, f = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    size = ctypes.POINTER(sz)
    i8, ce, orth = ctypes.POINTER(SlzI8Shape), ctypes.POINTER(SlzCeShape), ctypes.POINTER(SlzOrthShape)
    L.slz_quantize_i8.argtypes = [vp, i, u32, u32, i64, vp, i64, vp, vp]
    L.slz_matmul_i8_workspace.argtypes = [i8, vp, vp, size]
    L.slz_matmul_i8.argtypes = [i8, vp, vp, vp, vp, vp, vp, sz, vp]
    L.slz_linear_i8_workspace.argtypes = [i8, vp, vp, size]
    L.slz_linear_i8.argtypes = [i8, vp, vp, vp, vp, vp, sz, vp]
    L.slz_matmul_i8_grad_workspace.argtypes = [i8, vp, size]
    L.slz_matmul_i8_grad.argtypes = [i8, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    i4 = ctypes.POINTER(SlzI4Shape)
    L.slz_quantize_i4.argtypes = [vp, i, u32, u32, i64, u32, vp, i64, vp, i64, vp]
    L.slz_values_i4.argtypes = [vp, i64, vp, i64, u32, u32, u32, vp, i, i64, vp]
    L.slz_linear_i4_workspace.argtypes = [i4, vp, size]
    L.slz_linear_i4.argtypes = [i4, vp, vp, vp, vp, vp, sz, vp]
    L.slz_linear_i4_grad_workspace.argtypes = [i4, vp, vp, size]
    L.slz_linear_i4_grad.argtypes = [i4, vp, vp, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    L.slz_linear_ce_workspace.argtypes = [ce, vp, vp, size]
    L.slz_linear_ce.argtypes = [ce, vp, vp, vp, vp, vp, vp, sz, vp]
    L.slz_linear_ce_grad_workspace.argtypes = [ce, vp, vp, size]
    L.slz_linear_ce_grad.argtypes = [ce, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.slz_orthogonalize_workspace.argtypes = [orth, size]
    L.slz_orthogonalize.argtypes = [orth, vp, vp, vp, sz, vp]
    L.slz_clip_workspace.argtypes = [vp, u32, size]
    L.slz_grad_norm.argtypes = [vp, u32, vp, vp, sz, vp]
    L.slz_clip_by_norm.argtypes = [vp, u32, f, f, i, vp, vp, sz, vp]


@functools.lru_cache(maxsize=None)
def _lib():
    import paper_2504_17785_amd as slz
    return slz.lib()


@functools.lru_cache(maxsize=None)
def _tensors():
    """The reader of tensor lists (csrc/slz_tensors.cpp)."""
    import os
    from . import build
    lib = build.torch_lib()
    if not os.path.exists(lib):
        build._build_tensors()
    T = ctypes.PyDLL(lib)
    T.slz_tensors_table.argtypes = [ctypes.py_object, ctypes.py_object, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
    T.slz_tensors_written.argtypes = [ctypes.py_object]
    return T


def _check(rc: int, where: str):
    if rc != 0:
        import paper_2504_17785_amd as slz
        raise slz.SlzError(rc, where)


def _stream(t) -> int:
    """The current stream's handle; work is enqueued on the current device, so its tensors have to be there."""
    at = t.get_device()
    if at != torch._C._cuda_getDevice():
        raise ValueError("tensors are on device %d, the current device is %d" % (at, torch._C._cuda_getDevice()))
    return torch._C._cuda_getCurrentRawStream(at)


def _matrix(t, what: str, types, like=None, rows=None, cols=None, dims: int = 2):
    """Checks a matrix; its row distance in elements."""
    if not t.is_cuda or t.dtype not in types:
        raise TypeError("%s: need a CUDA tensor of %s, got %s on %s" % (what, " or ".join(str(d) for d in types), t.dtype, t.device))
    if t.dim() != dims:
        raise ValueError("%s: need %d dimensions, got %d" % (what, dims, t.dim()))
    shape, stride = t.shape, t.stride()
    if (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError("%s: shape %s, need (%s, %s)" % (what, tuple(shape), rows, cols))
    if max(shape) > 0x7fffffff:                        # the library takes 32 bits of a length, and refuses what it sees of longer ones
        _check(_E_TOO_LARGE, "%s: shape %s" % (what, tuple(shape)))
    if like is not None and t.get_device() != like.get_device():
        raise ValueError("%s: on device %d, others on %d" % (what, t.get_device(), like.get_device()))
    c, r = shape[-1], shape[-2]
    if c > 1 and stride[-1] != 1:
        raise ValueError("%s: need unit stride along the rows, got strides %s" % (what, tuple(stride)))
    if r < 2:
        return max(c, 1)
    if stride[-2] < c:
        raise ValueError("%s: rows overlap: strides %s" % (what, tuple(stride)))
    return stride[-2]


def _vector(t, what: str, dtype, count: int, like):
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError("%s: need a contiguous CUDA tensor of %s" % (what, dtype))
    if t.dim() != 1 or t.shape[0] != count:
        raise ValueError("%s: shape %s, need (%d,)" % (what, tuple(t.shape), count))
    if t.get_device() != like.get_device():
        raise ValueError("%s: on device %d, others on %d" % (what, t.get_device(), like.get_device()))
    return t.data_ptr()


def _workspace(fn, where: str, like, *args):
    """(tensor or None, address, bytes) of a call's workspace."""
    need = ctypes.c_size_t(0)
    _check(fn(*args, ctypes.byref(need)), where + "_workspace")
    if need.value == 0:
        return None, None, 0
    ws = torch.empty(need.value, dtype=torch.uint8, device=like.device)
    return ws, ws.data_ptr(), need.value


class _NoFormula(torch.autograd.Function):
    """Results of tensors that require a gradient: without it a backward pass would leave them out and say nothing."""

    @staticmethod
    def forward(ctx, where, count, *tensors):
        ctx.where = where
        ctx.mark_non_differentiable(*(t for t in tensors[:count] if t is not None and not t.is_floating_point()))
        return tensors[:count]

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("%s: autograd has no formula for it; call it on detached tensors, and matmul_i8_grad, linear_i4_grad or linear_ce_grad for gradients" % ctx.where)


def _results(where: str, inputs, *out):
    for t in inputs:
        if t.requires_grad and torch.is_grad_enabled():
            out = _NoFormula.apply(where, len(out), *out, *inputs)
            break
    return out if len(out) > 1 else out[0]


def quantize_i8(x):
    """slz_quantize_i8: x [rows][cols] -> (int8 [rows][cols], scale float32 [rows])."""
    ld = _matrix(x, "x", _TYPES)
    rows, cols = x.shape
    q = torch.empty((rows, cols), dtype=torch.int8, device=x.device)
    scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(_lib().slz_quantize_i8(x.data_ptr(), _TYPES[x.dtype], rows, cols, ld, q.data_ptr(), max(cols, 1), scale.data_ptr(), _stream(x)),
           "slz_quantize_i8")
    return _results("quantize_i8", (x,), q, scale)


def matmul_i8(a, a_scale, b, b_scale, dtype=torch.bfloat16):
    """slz_matmul_i8: a int8 [m][k], b int8 [n][k], a scale for each row of either -> y [m][n] of `dtype`."""
    if dtype not in _TYPES:
        raise TypeError("dtype: need float32, bfloat16 or float16, got %s" % dtype)
    ld_a = _matrix(a, "a", (torch.int8,))
    m, k = a.shape
    ld_b = _matrix(b, "b", (torch.int8,), a, None, k)
    n = b.shape[0]
    sa, sb = _vector(a_scale, "a_scale", torch.float32, m, a), _vector(b_scale, "b_scale", torch.float32, n, a)
    stream = _stream(a)
    y = torch.empty((m, n), dtype=dtype, device=a.device)
    sh = SlzI8Shape(m, n, k, _TYPES[dtype], ld_a, ld_b, max(n, 1))
    L = _lib()
    ws, at, need = _workspace(L.slz_matmul_i8_workspace, "slz_matmul_i8", a, ctypes.byref(sh), a.data_ptr(), b.data_ptr())
    _check(L.slz_matmul_i8(ctypes.byref(sh), a.data_ptr(), sa, b.data_ptr(), sb, y.data_ptr(), at, need, stream), "slz_matmul_i8")
    return _results("matmul_i8", (a_scale, b_scale), y)


def linear_i8(x, w, w_scale):
    """slz_linear_i8: x [m][k] floating, its rows quantised, times w int8 [n][k] -> y [m][n] of x's type."""
    ld_x = _matrix(x, "x", _TYPES)
    m, k = x.shape
    ld_w = _matrix(w, "w", (torch.int8,), x, None, k)
    n = w.shape[0]
    sw = _vector(w_scale, "w_scale", torch.float32, n, x)
    stream = _stream(x)
    y = torch.empty((m, n), dtype=x.dtype, device=x.device)
    sh = SlzI8Shape(m, n, k, _TYPES[x.dtype], ld_x, ld_w, max(n, 1))
    L = _lib()
    ws, at, need = _workspace(L.slz_linear_i8_workspace, "slz_linear_i8", x, ctypes.byref(sh), x.data_ptr(), w.data_ptr())
    _check(L.slz_linear_i8(ctypes.byref(sh), x.data_ptr(), w.data_ptr(), sw, y.data_ptr(), at, need, stream), "slz_linear_i8")
    return _results("linear_i8", (x, w_scale), y)


def matmul_i8_grad(dy, a, a_scale, b, b_scale, need_a: bool = True, need_b: bool = True):
    """slz_matmul_i8_grad: dy [m][n] -> (gradient of the values a_scale a [m][k], of b_scale b [n][k]), of dy's type; None for
    one that is not needed."""
    ld_y = _matrix(dy, "dy", _TYPES)
    m, n = dy.shape
    ld_a = _matrix(a, "a", (torch.int8,), dy, m)
    k = a.shape[1]
    ld_b = _matrix(b, "b", (torch.int8,), dy, n, k)
    sa, sb = _vector(a_scale, "a_scale", torch.float32, m, dy), _vector(b_scale, "b_scale", torch.float32, n, dy)
    stream = _stream(dy)
    da = torch.empty((m, k), dtype=dy.dtype, device=dy.device) if need_a else None
    db = torch.empty((n, k), dtype=dy.dtype, device=dy.device) if need_b else None
    sh = SlzI8Shape(m, n, k, _TYPES[dy.dtype], ld_a, ld_b, ld_y)
    L = _lib()
    ws, at, need = _workspace(L.slz_matmul_i8_grad_workspace, "slz_matmul_i8_grad", dy, ctypes.byref(sh), dy.data_ptr())
    _check(L.slz_matmul_i8_grad(ctypes.byref(sh), dy.data_ptr(), a.data_ptr(), sa, b.data_ptr(), sb, da.data_ptr() if need_a else None,
                                max(k, 1), db.data_ptr() if need_b else None, max(k, 1), at, need, stream), "slz_matmul_i8_grad")
    return _results("matmul_i8_grad", (dy, a_scale, b_scale), da, db)


def _rows_i4(q, scale, rows, cols, group, like):
    """Checks 4-bit rows and their scales; their row distances."""
    if group not in (32, 64, 128):
        raise ValueError("group: %s, need 32, 64 or 128" % (group,))
    ld_q = _matrix(q, "q", (torch.uint8,), like, rows, (cols + 127) // 128 * 64)
    return ld_q, _matrix(scale, "scale", (torch.float32,), q, q.shape[0], (cols + group - 1) // group)


# What has been found out of calls that are alike in all that the checks look at
_quantize_i4_known, _values_i4_known, _linear_i4_known, _linear_i4_grad_known = {}, {}, {}, {}


def _remember(known, alike, what):
    if len(known) >= 1024:
        known.clear()
    known[alike] = what
    return what


def _i4_plan(grad: bool, shape, *places):
    """A call's slz_i4_shape and workspace; places: addresses' last four bits, which is all that the library looks at."""
    sh, need = SlzI4Shape(*shape), ctypes.c_size_t(0)
    L = _lib()
    if grad:
        _check(L.slz_linear_i4_grad_workspace(ctypes.byref(sh), *places, ctypes.byref(need)), "slz_linear_i4_grad_workspace")
    else:
        _check(L.slz_linear_i4_workspace(ctypes.byref(sh), *places, ctypes.byref(need)), "slz_linear_i4_workspace")
    return ctypes.byref(sh), need.value


def quantize_i4(w, group: int = 128):
    """slz_quantize_i4: w [rows][cols] -> (4-bit rows, uint8 [rows][64 for every 128 columns], scale float32 [rows][one for every `group` columns])."""
    alike = (w.dtype, w.shape, w.stride(), w.get_device(), group)
    known = _quantize_i4_known.get(alike)
    if known is None:
        ld = _matrix(w, "w", _TYPES)
        rows, cols = w.shape
        if group not in (32, 64, 128):
            raise ValueError("group: %s, need 32, 64 or 128" % (group,))
        known = _remember(_quantize_i4_known, alike, (rows, cols, ld, _TYPES[w.dtype], (cols + 127) // 128 * 64, (cols + group - 1) // group))
    rows, cols, ld, code, row, groups = known
    stream, device = _stream(w), w.device
    q = torch.empty((rows, row), dtype=torch.uint8, device=device)
    scale = torch.empty((rows, groups), dtype=torch.float32, device=device)
    _check(_lib().slz_quantize_i4(w.data_ptr(), code, rows, cols, ld, group, q.data_ptr(), row, scale.data_ptr(), groups, stream), "slz_quantize_i4")
    return _results("quantize_i4", (w,), q, scale)


def values_i4(q, scale, cols: int, group: int = 128, dtype=torch.bfloat16):
    """slz_values_i4: 4-bit rows of `cols` entries and their scales -> the values [rows][cols] of `dtype`."""
    alike = (q.dtype, q.shape, q.stride(), q.get_device(), scale.dtype, scale.shape, scale.stride(), scale.get_device(), cols, group, dtype)
    known = _values_i4_known.get(alike)
    if known is None:
        if dtype not in _TYPES:
            raise TypeError("dtype: need float32, bfloat16 or float16, got %s" % dtype)
        if not 0 <= cols <= 0x7fffffff:
            raise ValueError("cols: %d" % cols)
        known = _remember(_values_i4_known, alike, (q.shape[0], *_rows_i4(q, scale, None, cols, group, None), _TYPES[dtype]))
    rows, ld_q, ld_scale, code = known
    stream = _stream(q)
    out = torch.empty((rows, cols), dtype=dtype, device=q.device)
    _check(_lib().slz_values_i4(q.data_ptr(), ld_q, scale.data_ptr(), ld_scale, group, rows, cols, out.data_ptr(), code, max(cols, 1), stream), "slz_values_i4")
    return _results("values_i4", (scale,), out)


def linear_i4(x, q, scale, group: int = 128):
    """slz_linear_i4: x [m][k] times the values of 4-bit rows q [n] with their scales -> y [m][n] of x's type.  For many rows (a thousand, about; nine
    where k is below 8) of bf16 or f16 the values are rounded to that type first; for few nothing of them is rounded."""
    at_x = x.data_ptr()
    alike = (x.dtype, x.shape, x.stride(), x.get_device(), q.dtype, q.shape, q.stride(), q.get_device(), scale.dtype, scale.shape, scale.stride(), scale.get_device(), group, at_x & 15)
    known = _linear_i4_known.get(alike)
    if known is None:
        ld_x = _matrix(x, "x", _TYPES)
        m, k = x.shape
        ld_q, ld_scale = _rows_i4(q, scale, None, k, group, x)
        n = q.shape[0]
        known = _remember(_linear_i4_known, alike, ((m, n), *_i4_plan(False, (m, n, k, _TYPES[x.dtype], group, ld_x, ld_q, ld_scale, max(n, 1)), at_x & 15)))
    shape, sh, need = known
    stream = _stream(x)
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _check(_lib().slz_linear_i4(sh, at_x, q.data_ptr(), scale.data_ptr(), y.data_ptr(), ws.data_ptr() if need else None, need, stream), "slz_linear_i4")
    return _results("linear_i4", (x, scale), y)


def linear_i4_grad(dy, x, q, scale, group: int = 128, need_x: bool = True, need_w: bool = True):
    """slz_linear_i4_grad: dy [m][n] and what linear_i4 was called with -> (gradient of x [m][k], of the weights' values [n][k]), of dy's type; None for one
    that is not needed.  For dx the values are rounded to bf16 or f16, if dy is of these."""
    at_dy, at_x = dy.data_ptr(), x.data_ptr()
    alike = (dy.dtype, dy.shape, dy.stride(), dy.get_device(), x.dtype, x.shape, x.stride(), x.get_device(), q.dtype, q.shape, q.stride(), q.get_device(),
             scale.dtype, scale.shape, scale.stride(), scale.get_device(), group, at_dy & 15, at_x & 15)
    known = _linear_i4_grad_known.get(alike)
    if known is None:
        ld_y = _matrix(dy, "dy", _TYPES)
        m, n = dy.shape
        ld_x = _matrix(x, "x", (dy.dtype,), dy, m)
        k = x.shape[1]
        ld_q, ld_scale = _rows_i4(q, scale, n, k, group, dy)
        known = _remember(_linear_i4_grad_known, alike, (m, n, k, *_i4_plan(True, (m, n, k, _TYPES[dy.dtype], group, ld_x, ld_q, ld_scale, ld_y), at_dy & 15, at_x & 15)))
    m, n, k, sh, need = known
    stream, device = _stream(dy), dy.device
    dx = torch.empty((m, k), dtype=dy.dtype, device=device) if need_x else None
    dw = torch.empty((n, k), dtype=dy.dtype, device=device) if need_w else None
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(_lib().slz_linear_i4_grad(sh, at_dy, at_x, q.data_ptr(), scale.data_ptr(), dx.data_ptr() if need_x else None, max(k, 1),
                                     dw.data_ptr() if need_w else None, max(k, 1), ws.data_ptr() if need else None, need, stream), "slz_linear_i4_grad")
    return _results("linear_i4_grad", (dy, x, scale), dx, dw)


def _ce_shape(h, w, labels, ignore_index):
    ld_h = _matrix(h, "h", _TYPES)
    tokens, inner = h.shape
    ld_w = _matrix(w, "w", (h.dtype,), h, None, inner)
    at = _vector(labels, "labels", torch.int64, tokens, h)
    return SlzCeShape(tokens, inner, w.shape[0], _TYPES[h.dtype], ld_h, ld_w, inner, inner, ignore_index), at


def linear_ce(h, w, labels, ignore_index: int = -100):
    """slz_linear_ce: hidden states h [tokens][inner], weights w [vocab][inner], labels int64 [tokens] -> (loss, lse), float32
    [tokens] each: the cross entropy of the softmax of h w^T, and the logarithm of the softmax's sum."""
    sh, at_labels = _ce_shape(h, w, labels, ignore_index)
    stream = _stream(h)
    both = torch.empty((2, h.shape[0]), dtype=torch.float32, device=h.device)
    loss, lse = both[0], both[1]
    L = _lib()
    ws, at, need = _workspace(L.slz_linear_ce_workspace, "slz_linear_ce", h, ctypes.byref(sh), h.data_ptr(), w.data_ptr())
    _check(L.slz_linear_ce(ctypes.byref(sh), h.data_ptr(), w.data_ptr(), at_labels, loss.data_ptr(), lse.data_ptr(), at, need, stream),
           "slz_linear_ce")
    return _results("linear_ce", (h, w), loss, lse)


def linear_ce_grad(h, w, labels, lse, dloss, ignore_index: int = -100):
    """slz_linear_ce_grad: with lse of linear_ce and dloss float32 [tokens] -> (dh [tokens][inner], dw [vocab][inner]) of h's type."""
    sh, at_labels = _ce_shape(h, w, labels, ignore_index)
    tokens = h.shape[0]
    at_lse, at_dloss = _vector(lse, "lse", torch.float32, tokens, h), _vector(dloss, "dloss", torch.float32, tokens, h)
    stream = _stream(h)
    dh = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    dw = torch.empty(w.shape, dtype=h.dtype, device=h.device)
    L = _lib()
    ws, at, need = _workspace(L.slz_linear_ce_grad_workspace, "slz_linear_ce_grad", h, ctypes.byref(sh), h.data_ptr(), w.data_ptr())
    _check(L.slz_linear_ce_grad(ctypes.byref(sh), h.data_ptr(), w.data_ptr(), at_labels, at_lse, at_dloss, dh.data_ptr(), dw.data_ptr(), at,
                                need, stream), "slz_linear_ce_grad")
    return _results("linear_ce_grad", (h, w, lse, dloss), dh, dw)


def orthogonalize(g, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7):
    """slz_orthogonalize: g [rows][cols] or [batch][rows][cols] -> the same shape, each matrix orthogonalised by `steps`
    Newton-Schulz steps with the given coefficients (a, b, c)."""
    ld = _matrix(g, "g", _TYPES, dims=g.dim() if g.dim() in (2, 3) else 2)
    rows, cols = g.shape[-2:]
    batch, stride = (g.shape[0], g.stride(0)) if g.dim() == 3 else (1, 0)
    if batch > 1 and stride < 0:
        raise ValueError("g: negative stride")
    if not 0 <= steps <= 64:
        raise ValueError("steps: %d, need 0 to 64" % steps)
    a, b, c = coefficients
    stream = _stream(g)
    out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
    sh = SlzOrthShape(batch, rows, cols, _TYPES[g.dtype], ld, stride, max(cols, 1), rows * cols, steps, a, b, c, eps)
    L = _lib()
    ws, at, need = _workspace(L.slz_orthogonalize_workspace, "slz_orthogonalize", g, ctypes.byref(sh))
    _check(L.slz_orthogonalize(ctypes.byref(sh), g.data_ptr(), out.data_ptr(), at, need, stream), "slz_orthogonalize")
    return _results("orthogonalize", (g,), out)


def _grad_place(t, what: str, device: int):
    """(rows, cols, row distance) of a tensor of any shape whose elements are one run, or of a matrix."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s: need a tensor, got %s" % (what, type(t).__name__))
    if t.dtype not in _TYPES or t.get_device() != device:
        raise TypeError("%s: need a CUDA tensor of float32, bfloat16 or float16 on device %d, got %s on %s" % (what, device, t.dtype, t.device))
    if t.is_contiguous():
        n = t.numel()
        if n <= 0x7fffffff:
            return 1, n, n
        cols = t.shape[-1]
        _check(_E_TOO_LARGE if max(cols, n // cols) > 0x7fffffff else 0, "%s: shape %s" % (what, tuple(t.shape)))
        return n // cols, cols, cols
    if t.dim() != 2:
        raise ValueError("%s: need a contiguous tensor, or a matrix with unit stride along its rows; got strides %s" % (what, t.stride()))
    return (*t.shape, _matrix(t, what, _TYPES))


_NO_FORMULA = "clip_by_norm: autograd has no formula for it; call it on detached tensors or under torch.no_grad()"


def _grad_table(grads, out, device: int, recording: bool = False):
    """An array of slz_grad_tensor; recording: autograd is, and would not know of what is written."""
    table = (SlzGradTensor * len(grads))()
    if _tensors().slz_tensors_table(grads, out, device, recording, table) == 0:
        return table
    for i, (g, o) in enumerate(zip(grads, out)):
        rows, cols, ld = _grad_place(g, "gradient %d" % i, device)
        if o is g:
            ld_o = ld
        else:
            if o.dtype != g.dtype or o.shape != g.shape:
                raise ValueError("output %d: need %s %s, got %s %s" % (i, g.dtype, tuple(g.shape), o.dtype, tuple(o.shape)))
            rows_o, cols_o, ld_o = _grad_place(o, "output %d" % i, device)
            if (rows, cols) != (rows_o, cols_o):               # one of them is a run, the other is not
                rows, cols = g.shape
                ld, ld_o = _matrix(g, "gradient %d" % i, _TYPES), _matrix(o, "output %d" % i, _TYPES)
        if recording and (g.requires_grad or o.requires_grad):
            raise RuntimeError(_NO_FORMULA)
        table[i] = SlzGradTensor(g.data_ptr(), o.data_ptr(), rows, cols, ld, ld_o, _TYPES[g.dtype])
    return table


def _clip_norm(grads, norm):
    """The list of gradients, and where their norm is to be or is."""
    grads = list(grads)
    device = torch._C._cuda_getDevice()
    if norm is None:
        return grads, torch.empty((), dtype=torch.float32, device="cuda:%d" % device), device
    if norm.dtype != torch.float32 or norm.get_device() != device or norm.numel() != 1:
        raise TypeError("norm: need one float32 on device %d" % device)
    return grads, norm, device


def grad_norm(grads):
    """slz_grad_norm: the norm that all tensors of a list have together, a float32 scalar tensor."""
    grads, norm, device = _clip_norm(grads, None)
    table, L = _grad_table(grads, grads, device), _lib()
    ws, at, need = _workspace(L.slz_clip_workspace, "slz_clip", norm, table, len(grads))
    _check(L.slz_grad_norm(table, len(grads), norm.data_ptr(), at, need, torch._C._cuda_getCurrentRawStream(device)), "slz_grad_norm")
    return _results("grad_norm", grads, norm) if grads else norm


def clip_by_norm(grads, max_norm: float, eps: float = 1e-6, norm=None, out=None):
    """slz_clip_by_norm: all tensors of a list times max_norm / (their common norm + eps) where that is below 1, in place or into the tensors of `out`.  The norm, a float32
    scalar tensor, is returned; one that is given is taken in its place (of gradients that are spread over several devices).  Gradients and outputs are contiguous tensors
    or matrices with unit stride along their rows; dense tensors in another order, such as a transposed matrix, are refused."""
    grads, at_norm, device = _clip_norm(grads, norm)
    out = grads if out is None else list(out)
    if len(out) != len(grads):
        raise ValueError("out: %d tensors for %d gradients" % (len(out), len(grads)))
    recording = torch.is_grad_enabled()
    if recording and at_norm.requires_grad:
        raise RuntimeError(_NO_FORMULA)
    table, L = _grad_table(grads, out, device, recording), _lib()
    ws, at, need = _workspace(L.slz_clip_workspace, "slz_clip", at_norm, table, len(grads))
    _check(L.slz_clip_by_norm(table, len(grads), max_norm, eps, norm is not None, at_norm.data_ptr(), at, need, torch._C._cuda_getCurrentRawStream(device)),
           "slz_clip_by_norm")
    if _tensors().slz_tensors_written(out):
        raise RuntimeError("clip_by_norm: the outputs' versions could not be counted up")
    return at_norm
