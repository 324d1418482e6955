"""Refusals of the C entry points of include/silenzio_clear.h that need no GPU: every bad argument comes back as a code, before
anything is enqueued."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2504_17785_amd as slz
from paper_2504_17785_amd.clear import SlzCeShape, SlzI8Shape, SlzOrthShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, TOO_LARGE = -1, -5
P = 0x100000          # an aligned address; nothing is read from it


def ref(s):
    return ctypes.byref(s)


def test_header_is_plain_c():
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    r = subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", "-x", "c",
                        os.path.join(ROOT, "include", "silenzio_clear.h")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_quantize_refuses():
    f = slz.lib().slz_quantize_i8
    assert f(P, 3, 4, 8, 8, P, 8, P, None) == INVALID            # no such type
    assert f(None, 0, 4, 8, 8, P, 8, P, None) == INVALID
    assert f(P, 0, 4, 8, 8, None, 8, P, None) == INVALID
    assert f(P, 0, 4, 8, 8, P, 8, None, None) == INVALID
    assert f(P, 0, 4, 8, 7, P, 8, P, None) == INVALID            # rows overlap
    assert f(P, 0, 4, 8, 8, P, 7, P, None) == INVALID
    assert f(P + 2, 0, 4, 8, 8, P, 8, P, None) == INVALID        # misaligned for its type
    assert f(P + 1, 1, 4, 8, 8, P, 8, P, None) == INVALID
    assert f(P, 0, 1 << 31, 8, 8, P, 8, P, None) == TOO_LARGE
    assert f(P, 0, 4, 8, (1 << 22) + 1, P, 8, P, None) == TOO_LARGE
    assert f(None, 0, 0, 8, 8, None, 8, None, None) == 0         # no rows: nothing to do


def test_products_of_8_bit_integers_refuse():
    L = slz.lib()
    need = ctypes.c_size_t(7)
    ok = dict(m=4, n=8, k=32, type=1, ld_a=32, ld_b=32, ld_y=8)

    def both(code, a=P, sa=P, b=P, sb=P, y=P, ws=P, size=1 << 30, **kw):
        sh = SlzI8Shape(**{**ok, **kw})
        assert L.slz_matmul_i8(ref(sh), a, sa, b, sb, y, ws, size, None) == code
        assert L.slz_linear_i8(ref(sh), a, b, sb, y, ws, size, None) == code

    both(INVALID, type=5)
    both(INVALID, a=None)
    both(INVALID, b=None)
    both(INVALID, sb=None)
    both(INVALID, y=None)
    both(INVALID, sb=P + 2)
    both(INVALID, y=P + 1)
    both(INVALID, ld_a=31)
    both(INVALID, ld_b=31)
    both(INVALID, ld_y=7)
    both(TOO_LARGE, k=1 << 17, ld_a=1 << 17, ld_b=1 << 17)
    both(TOO_LARGE, m=1 << 31)
    sh = SlzI8Shape(**ok)
    assert L.slz_matmul_i8(ref(sh), P, None, P, P, P, P, 1 << 30, None) == INVALID
    assert L.slz_matmul_i8(None, P, P, P, P, P, P, 1 << 30, None) == INVALID
    assert L.slz_linear_i8(None, P, P, P, P, P, 1 << 30, None) == INVALID
    assert L.slz_matmul_i8_workspace(None, P, P, ref(need)) == INVALID
    assert L.slz_matmul_i8_workspace(ref(sh), P, P, None) == INVALID
    # a workspace that is missing, too small or misaligned, where one is needed (many rows, of 31 entries)
    odd = SlzI8Shape(**{**ok, "m": 64, "k": 31})
    odd.ld_a = odd.ld_b = 31
    assert L.slz_matmul_i8_workspace(ref(odd), P, P, ref(need)) == 0 and need.value > 0
    for ws, size in ((None, 1 << 30), (P, need.value - 1), (P + 128, need.value)):
        assert L.slz_matmul_i8(ref(odd), P, P, P, P, P, ws, size, None) == INVALID
    # gradient
    g = L.slz_matmul_i8_grad
    assert L.slz_matmul_i8_grad_workspace(ref(sh), P, ref(need)) == 0 and need.value > 0
    size = need.value
    for args in ((None, P, P, P, P, P), (P, None, P, P, P, P), (P, P, None, P, P, P), (P, P, P, None, P, P), (P, P, P, P, None, P),
                 (P, P, P, P, P, P + 1)):
        assert g(ref(sh), *args, 32, P, 32, P, size, None) == INVALID
    assert g(ref(sh), P, P, P, P, P, P, 31, P, 32, P, size, None) == INVALID
    assert g(ref(sh), P, P, P, P, P, P, 32, P, 31, P, size, None) == INVALID
    assert g(ref(sh), P, P, P, P, P, P, 32, P, 32, P, size - 1, None) == INVALID
    assert g(None, P, P, P, P, P, P, 32, P, 32, P, size, None) == INVALID
    # without elements nothing is enqueued
    assert L.slz_matmul_i8(ref(SlzI8Shape(**{**ok, "m": 0})), None, None, P, P, None, P, 1 << 30, None) == 0
    assert L.slz_matmul_i8(ref(SlzI8Shape(**{**ok, "n": 0})), P, P, None, None, None, P, 1 << 30, None) == 0


def test_cross_entropy_refuses():
    L = slz.lib()
    need = ctypes.c_size_t(0)
    ok = dict(tokens=4, inner=32, vocab=100, type=1, ld_h=32, ld_w=32, ld_dh=32, ld_dw=32, ignore_index=-100)

    def each(code, h=P, w=P, labels=P, lse=P, ws=P, size=1 << 40, **kw):
        sh = SlzCeShape(**{**ok, **kw})
        assert L.slz_linear_ce(ref(sh), h, w, labels, P, lse, ws, size, None) == code
        assert L.slz_linear_ce_grad(ref(sh), h, w, labels, lse, P, P, P, ws, size, None) == code

    for kw in (dict(type=-1), dict(inner=0), dict(vocab=0), dict(h=None), dict(w=None), dict(labels=None), dict(lse=None), dict(labels=P + 4),
               dict(lse=P + 2), dict(h=P + 1), dict(ld_h=31), dict(ld_w=31), dict(ws=None), dict(ws=P + 16), dict(size=0)):
        each(INVALID, **kw)
    for kw in (dict(tokens=1 << 31), dict(vocab=1 << 31), dict(ld_w=(1 << 22) + 1)):
        each(TOO_LARGE, **kw)
    sh = SlzCeShape(**ok)
    assert L.slz_linear_ce(ref(sh), P, P, P, None, P, P, 1 << 40, None) == INVALID
    assert L.slz_linear_ce_grad(ref(sh), P, P, P, P, None, P, P, P, 1 << 40, None) == INVALID
    assert L.slz_linear_ce_grad(ref(sh), P, P, P, P, P, None, P, P, 1 << 40, None) == INVALID
    assert L.slz_linear_ce_grad(ref(sh), P, P, P, P, P, P, None, P, 1 << 40, None) == INVALID
    assert L.slz_linear_ce_grad(ref(SlzCeShape(**{**ok, "ld_dh": 31})), P, P, P, P, P, P, P, P, 1 << 40, None) == INVALID
    assert L.slz_linear_ce_grad(ref(SlzCeShape(**{**ok, "ld_dw": 31})), P, P, P, P, P, P, P, P, 1 << 40, None) == INVALID
    for f in (L.slz_linear_ce_workspace, L.slz_linear_ce_grad_workspace):
        assert f(None, P, P, ref(need)) == INVALID
        assert f(ref(sh), P, P, None) == INVALID
        assert f(ref(SlzCeShape(**{**ok, "vocab": 0})), P, P, ref(need)) == INVALID
        assert f(ref(SlzCeShape(**{**ok, "tokens": 1 << 31})), P, P, ref(need)) == TOO_LARGE
    assert L.slz_linear_ce(ref(SlzCeShape(**{**ok, "tokens": 0})), None, P, None, None, None, P, 1 << 40, None) == 0


def test_cross_entropy_workspace_does_not_hold_the_logits():
    L = slz.lib()
    need = ctypes.c_size_t(0)
    sh = SlzCeShape(tokens=8192, inner=4096, vocab=262144, type=1, ld_h=4096, ld_w=4096, ld_dh=4096, ld_dw=4096, ignore_index=-100)
    for f in (L.slz_linear_ce_workspace, L.slz_linear_ce_grad_workspace):
        assert f(ref(sh), P, P, ref(need)) == 0
        assert need.value < 8192 * 262144 * 2 // 6


def test_orthogonalize_refuses():
    L = slz.lib()
    need = ctypes.c_size_t(0)
    ok = dict(batch=2, rows=200, cols=300, type=1, ld_g=300, stride_g=60000, ld_out=300, stride_out=60000, steps=5, a=3.4, b=-4.8, c=2.0, eps=1e-7)

    def each(code, g=P, out=P, ws=P, size=1 << 40, **kw):
        assert L.slz_orthogonalize(ref(SlzOrthShape(**{**ok, **kw})), g, out, ws, size, None) == code

    for kw in (dict(type=4), dict(steps=65), dict(ld_g=299), dict(ld_out=299), dict(g=None), dict(out=None), dict(g=P + 1), dict(out=P + 1), dict(ws=None),
               dict(ws=P + 64), dict(size=1000)):
        each(INVALID, **kw)
    for kw in (dict(batch=65536), dict(rows=1 << 22), dict(cols=(1 << 22) + 1, ld_g=1 << 23, ld_out=1 << 23)):
        each(TOO_LARGE, **kw)
    assert L.slz_orthogonalize(None, P, P, P, 1 << 40, None) == INVALID
    assert L.slz_orthogonalize_workspace(None, ref(need)) == INVALID
    assert L.slz_orthogonalize_workspace(ref(SlzOrthShape(**ok)), None) == INVALID
    for kw in (dict(batch=0), dict(rows=0), dict(cols=0)):
        each(0, g=None, out=None, ws=None, size=0, **kw)


def test_binding_refuses_what_is_not_on_the_gpu():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        slz.quantize_i8(x)
    with pytest.raises(TypeError):
        slz.linear_i8(x, x.to(torch.int8), torch.zeros(4))
    with pytest.raises(TypeError):
        slz.matmul_i8(x.to(torch.int8), torch.zeros(4), x.to(torch.int8), torch.zeros(4))
    with pytest.raises(TypeError):
        slz.matmul_i8_grad(x, x.to(torch.int8), torch.zeros(4), x.to(torch.int8), torch.zeros(4))
    with pytest.raises(TypeError):
        slz.linear_ce(x, x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(TypeError):
        slz.linear_ce_grad(x, x, torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4))
    with pytest.raises(TypeError):
        slz.orthogonalize(x)
