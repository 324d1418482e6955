"""Binding of include/silenzio_clear.h: products of 8-bit integers, softmax cross entropy of a linear layer, orthogonalised updates.

As in the rest of the binding the functions check their arguments, hand pointers and the current stream to the library and return at once.
Matrices are CUDA tensors on the current device with unit stride along their rows (any distance between rows).  Workspaces
come from torch's allocator on the current stream, so that their memory is not given away before the call's work on it is done.

The gradients are functions of their own (matmul_i8_grad, linear_ce_grad) and autograd does not know them: results of tensors that require
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


class SlzOrthShape(ctypes.Structure):
    """slz_orth_shape of include/silenzio_clear.h."""
    _fields_ = [("batch", ctypes.c_uint32), ("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32), ("type", ctypes.c_int),
                ("ld_g", ctypes.c_int64), ("stride_g", ctypes.c_int64), ("ld_out", ctypes.c_int64), ("stride_out", ctypes.c_int64),
                ("steps", ctypes.c_uint32), ("a", ctypes.c_float), ("b", ctypes.c_float), ("c", ctypes.c_float), ("eps", ctypes.c_float)]


def declare(L):
    vp, u32, sz, i64, i = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int
    size = ctypes.POINTER(sz)
    i8, ce, orth = ctypes.POINTER(SlzI8Shape), ctypes.POINTER(SlzCeShape), ctypes.POINTER(SlzOrthShape)
    L.slz_quantize_i8.argtypes = [vp, i, u32, u32, i64, vp, i64, vp, vp]
    L.slz_matmul_i8_workspace.argtypes = [i8, vp, vp, size]
    L.slz_matmul_i8.argtypes = [i8, vp, vp, vp, vp, vp, vp, sz, vp]
    L.slz_linear_i8_workspace.argtypes = [i8, vp, vp, size]
    L.slz_linear_i8.argtypes = [i8, vp, vp, vp, vp, vp, sz, vp]
    L.slz_matmul_i8_grad_workspace.argtypes = [i8, vp, size]
    L.slz_matmul_i8_grad.argtypes = [i8, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    L.slz_linear_ce_workspace.argtypes = [ce, vp, vp, size]
    L.slz_linear_ce.argtypes = [ce, vp, vp, vp, vp, vp, vp, sz, vp]
    L.slz_linear_ce_grad_workspace.argtypes = [ce, vp, vp, size]
    L.slz_linear_ce_grad.argtypes = [ce, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.slz_orthogonalize_workspace.argtypes = [orth, size]
    L.slz_orthogonalize.argtypes = [orth, vp, vp, vp, sz, vp]


@functools.lru_cache(maxsize=None)
def _lib():
    import paper_2504_17785_amd as slz
    return slz.lib()


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
        raise RuntimeError("%s: autograd has no formula for it; call it on detached tensors, and matmul_i8_grad or linear_ce_grad for gradients" % ctx.where)


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
