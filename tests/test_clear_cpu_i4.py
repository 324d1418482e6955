"""Refusals of the entry points for 4-bit layers and for clipped gradients that need no GPU: every bad argument comes back as a code, before anything is enqueued."""
import ctypes

import pytest

import paper_2504_17785_amd as slz
from paper_2504_17785_amd.clear import SlzGradTensor, SlzI4Shape

INVALID, TOO_LARGE = -1, -5
P = 0x100000          # an aligned address; nothing is read from it
ref = ctypes.byref


def test_quantize_and_values_refuse():
    L = slz.lib()

    def both(code, w=P, type=1, rows=4, cols=200, ld=200, group=64, q=P, ld_q=128, scale=P, ld_scale=4):
        assert L.slz_quantize_i4(w, type, rows, cols, ld, group, q, ld_q, scale, ld_scale, None) == code
        assert L.slz_values_i4(q, ld_q, scale, ld_scale, group, rows, cols, w, type, ld, None) == code

    for kw in (dict(type=3), dict(type=-1), dict(group=0), dict(group=16), dict(group=48), dict(group=256), dict(w=None), dict(q=None), dict(scale=None), dict(w=P + 1),
               dict(type=0, w=P + 2), dict(scale=P + 2), dict(q=P + 8), dict(ld=199), dict(ld_q=127), dict(ld_q=136), dict(ld_scale=3)):
        both(INVALID, **kw)
    for kw in (dict(rows=1 << 31), dict(cols=1 << 31, ld=1 << 31, ld_q=1 << 31, ld_scale=1 << 31), dict(ld=(1 << 22) + 1), dict(ld_q=(1 << 22) + 16), dict(ld_scale=(1 << 22) + 1)):
        both(TOO_LARGE, **kw)
    both(0, rows=0, w=None, q=None, scale=None)
    both(0, cols=0, w=None, q=None, scale=None)


def test_products_refuse():
    L = slz.lib()
    need = ctypes.c_size_t(7)
    ok = dict(m=5000, n=5000, k=200, type=1, group=64, ld_x=200, ld_q=128, ld_scale=4, ld_y=5000)

    def each(code, x=P, q=P, scale=P, y=P, ws=P, size=1 << 40, which="lxw", **kw):
        sh = SlzI4Shape(**{**ok, **kw})
        if "l" in which:
            assert L.slz_linear_i4(ref(sh), x, q, scale, y, ws, size, None) == code
        if "x" in which:
            assert L.slz_linear_i4_grad(ref(sh), y, x, q, scale, P, 200, None, 0, ws, size, None) == code
        if "w" in which:
            assert L.slz_linear_i4_grad(ref(sh), y, x, q, scale, None, 0, P, 200, ws, size, None) == code

    for kw in (dict(type=5), dict(group=65), dict(y=None), dict(y=P + 1), dict(ld_y=4999), dict(ws=None), dict(ws=P + 64), dict(size=64)):
        each(INVALID, **kw)
    for kw in (dict(x=None), dict(x=P + 1), dict(ld_x=199)):
        each(INVALID, which="lw", **kw)
    for kw in (dict(q=None), dict(q=P + 4), dict(scale=None), dict(scale=P + 1), dict(ld_q=112), dict(ld_q=129), dict(ld_scale=3)):
        each(INVALID, which="lx", **kw)
    for kw in (dict(m=1 << 31), dict(n=1 << 31), dict(k=1 << 31), dict(ld_y=(1 << 22) + 1)):
        each(TOO_LARGE, **kw)
    sh = SlzI4Shape(**ok)
    assert L.slz_linear_i4(None, P, P, P, P, P, 1 << 40, None) == INVALID
    assert L.slz_linear_i4_grad(None, P, P, P, P, P, 200, P, 200, P, 1 << 40, None) == INVALID
    assert L.slz_linear_i4_grad(ref(sh), P, P, P, P, P, 199, P, 200, P, 1 << 40, None) == INVALID
    assert L.slz_linear_i4_grad(ref(sh), P, P, P, P, P, 200, P, 199, P, 1 << 40, None) == INVALID
    assert L.slz_linear_i4_grad(ref(sh), P, P, P, P, P + 1, 200, P, 200, P, 1 << 40, None) == INVALID
    for f, args in ((L.slz_linear_i4_workspace, (P,)), (L.slz_linear_i4_grad_workspace, (P, P))):
        assert f(None, *args, ref(need)) == INVALID
        assert f(ref(sh), *args, None) == INVALID
        assert f(ref(SlzI4Shape(**{**ok, "group": 1})), *args, ref(need)) == INVALID
        assert f(ref(SlzI4Shape(**{**ok, "k": 1 << 31})), *args, ref(need)) == TOO_LARGE
        assert f(ref(sh), *args, ref(need)) == 0 and need.value > 0
    # nothing to compute
    for kw in (dict(m=0), dict(n=0)):
        need.value = 7
        assert L.slz_linear_i4_workspace(ref(SlzI4Shape(**{**ok, **kw})), P, ref(need)) == 0 and need.value == 0
    for kw in (dict(m=0), dict(n=0), dict(k=0), dict(m=0, n=0, k=0)):
        assert L.slz_linear_i4_workspace(ref(SlzI4Shape(**{**ok, **kw})), P, ref(need)) == 0
        assert L.slz_linear_i4_grad_workspace(ref(SlzI4Shape(**{**ok, **kw})), P, P, ref(need)) == 0
    each(0, which="l", m=0, x=None, y=None, ws=None, size=0)
    each(0, which="l", n=0, q=None, scale=None, y=None, ws=None, size=0)
    each(0, which="xw", k=0, x=None, q=None, scale=None, ws=None, size=0)


def tensors(*items):
    return (SlzGradTensor * len(items))(*(SlzGradTensor(**{**dict(g=P, out=P, rows=4, cols=8, ld_g=8, ld_out=8, type=0), **kw}) for kw in items))


def test_clip_refuses():
    L = slz.lib()
    need = ctypes.c_size_t(0)

    def clip(code, *items, max_norm=1.0, eps=1e-6, norm=P, ws=P, size=1 << 40):
        t = tensors(*items)
        assert L.slz_clip_by_norm(t, len(items), max_norm, eps, 0, norm, ws, size, None) == code
        assert L.slz_clip_by_norm(t, len(items), max_norm, eps, 1, norm, ws, size, None) == code

    for kw in (dict(type=3), dict(g=None), dict(out=None), dict(g=P + 2, out=P + 2), dict(out=P + 1), dict(ld_g=7), dict(ld_out=7)):
        clip(INVALID, kw)
    for kw in (dict(rows=1 << 31), dict(cols=1 << 31, ld_g=1 << 31, ld_out=1 << 31), dict(ld_g=1 << 49, ld_out=1 << 49)):
        clip(TOO_LARGE, kw)
    for kw in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("nan")), dict(norm=None), dict(norm=P + 2), dict(ws=None), dict(ws=P + 8), dict(size=4)):
        clip(INVALID, {}, **kw)
    assert L.slz_clip_by_norm(None, 1, 1.0, 0.0, 0, P, P, 1 << 40, None) == INVALID
    assert L.slz_clip_by_norm(None, 1 << 26, 1.0, 0.0, 0, P, P, 1 << 40, None) == INVALID
    assert L.slz_grad_norm(None, 1, P, P, 1 << 40, None) == INVALID
    assert L.slz_grad_norm(tensors({}), 1, None, P, 1 << 40, None) == INVALID
    assert L.slz_grad_norm(tensors({}), 1, P, P, 7, None) == INVALID
    assert L.slz_grad_norm(tensors(dict(g=None)), 1, P, P, 1 << 40, None) == INVALID
    assert L.slz_clip_workspace(tensors({}), 1, None) == INVALID
    assert L.slz_clip_workspace(None, 1, ref(need)) == INVALID
    assert L.slz_clip_workspace(tensors(dict(type=9)), 1, ref(need)) == INVALID
    assert L.slz_clip_workspace(None, 0, ref(need)) == 0 and need.value == 0
    assert L.slz_clip_workspace(tensors(dict(rows=0)), 1, ref(need)) == 0 and need.value == 0


# a matrix of 4 rows of 8 numbers of 4 bytes: 128 bytes
@pytest.mark.parametrize("items", [
    ({}, {}),                                                                      # the same twice
    ({}, dict(g=P + 64, out=P + 64)),
    ({}, dict(g=P + 0x1000, out=P + 124, rows=1)),
    (dict(out=P + 4),),                                                            # over its own gradient
    (dict(out=P - 32),),
    (dict(ld_out=9),),                                                             # in place, with another distance
    (dict(out=P + 0x1000), dict(g=P + 0x1000, out=P + 0x2000)),                    # over another one's
    (dict(g=P + 0x1000), dict(g=P, out=P + 0x2000)),
    (dict(ld_g=16, ld_out=16), dict(g=P + 28, out=P + 28, ld_g=16, ld_out=16)),    # columns 0 to 7 and 7 to 14
    (dict(ld_g=16, ld_out=16), dict(g=P + 36, out=P + 36, ld_g=16, ld_out=16)),    # columns 0 to 7, and 9 to 16: 16 is the next row's 0
    (dict(ld_g=16, ld_out=16), dict(g=P + 32, out=P + 32, rows=1, cols=9, ld_g=9, ld_out=9)),
    (dict(ld_g=16, ld_out=16), dict(g=P + 32, out=P + 32, rows=3, cols=8)),        # a run across the rows
])
def test_clip_refuses_outputs_that_overlap(items):
    for order in (items, items[::-1]):
        assert slz.lib().slz_clip_by_norm(tensors(*order), len(order), 1.0, 0.0, 0, P, P, 1 << 40, None) == INVALID


def test_clip_refuses_a_norm_inside_the_tensors():
    clip = slz.lib().slz_clip_by_norm
    Q = P + 0x1000
    for given in (0, 1):                                                           # written while others still read it
        for at in (P, P + 124):
            assert clip(tensors({}), 1, 1.0, 0.0, given, at, Q, 1 << 40, None) == INVALID
            assert clip(tensors(dict(g=Q)), 1, 1.0, 0.0, given, at, Q, 1 << 40, None) == INVALID
    assert clip(tensors(dict(out=Q)), 1, 1.0, 0.0, 0, P + 64, Q, 1 << 40, None) == INVALID


def test_binding_refuses_what_is_not_on_the_gpu():
    torch = pytest.importorskip("torch")
    x, q, s = torch.zeros(4, 128), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1)
    with pytest.raises(TypeError):
        slz.quantize_i4(x)
    with pytest.raises(TypeError):
        slz.values_i4(q, s, 128)
    with pytest.raises(TypeError):
        slz.linear_i4(x, q, s)
    with pytest.raises(TypeError):
        slz.linear_i4_grad(x[:, :4], x, q, s)
