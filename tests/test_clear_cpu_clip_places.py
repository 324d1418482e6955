"""Which matrices have bytes in common (csrc/slz_clip_places.h), against a list of their bytes, and the entry point's refusals by it.  Whether it accepts is seen without a GPU by what it
refuses next: one more matrix makes the elements too many."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import paper_2504_17785_amd as slz
from tests.test_clear_cpu_i4 import INVALID, TOO_LARGE, P, tensors

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = r"""
#include "slz_clip_places.h"
static clip_place of(uint64_t at, uint64_t rows, uint64_t row, uint64_t step) {
    if (rows == 1 || row == step) return {(uintptr_t)at, (uintptr_t)(at + rows * row), rows * row, 0, 0};
    return {(uintptr_t)at, (uintptr_t)(at + (rows - 1) * step + row), row, step, 0};
}
extern "C" int meet(const uint64_t *a, const uint64_t *b) {
    const clip_place p = of(a[0], a[1], a[2], a[3]), q = of(b[0], b[1], b[2], b[3]);
    return p.begin <= q.begin ? clip_meet(p, q) : clip_meet(q, p);
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("places")
    (at / "host.cpp").write_text(HOST)
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "paper_2504_17785_amd", "csrc"), "-o", str(at / "host.so"), str(at / "host.cpp")], check=True)
    L = ctypes.CDLL(str(at / "host.so"))
    four = ctypes.c_uint64 * 4

    def of(a, b):
        both = bool(L.meet(four(*a), four(*b)))
        assert both == bool(L.meet(four(*b), four(*a))), (a, b)
        return both
    return of


def bytes_of(at, rows, row, step):
    return {at + i * step + c for i in range(rows) for c in range(row)}


def test_small_matrices_against_their_bytes(meet):
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for _ in range(60000):
        most = rng.choice((4, 12, 40))
        a, b = ((1000 + rng.randrange(3 * most), rng.randint(1, 9), row, row + rng.randrange(most)) for row in (rng.randint(1, most), rng.randint(1, rng.choice((2, most)))))
        want = bool(bytes_of(*a) & bytes_of(*b))
        assert meet(a, b) == want, (a, b)
        seen[want] += 1
    assert min(seen.values()) > 5000


def test_many_rows(meet):
    # rows of 1 and 2 bytes in steps without a common divisor meet somewhere, if there are enough of them
    for sa, sb in ((101, 103), (1024, 96), (4099, 4096), (77, 770), (1000, 999)):
        for offset in (1, 2, 50, 76):
            for rows in (1, 2, 30, 200, 2000):
                a, b = (10 ** 6, rows, 1, sa), (10 ** 6 + offset, rows, 2, sb)
                ends = {10 ** 6 + offset + j * sb + c for j in range(rows) for c in (0, 1)}
                assert meet(a, b) == any(10 ** 6 + i * sa in ends for i in range(rows)), (a, b)


def test_the_largest(meet):
    most = (1 << 31) - 1
    # columns of one matrix of 2^50 bytes
    step = (1 << 50) // most
    assert not meet((P, most, 1000, step), (P + 1000, most, 1000, step))
    assert meet((P, most, 1000, step), (P + 999, most, 1000, step))
    assert not meet((P, most, 1000, step), (P + 1000, most // 2, 1000, 2 * step))
    assert meet((P, most, 1000, step), (P + step - 1, most // 2, 2, 2 * step))
    # the last row of one lies in the first row of the other
    assert meet((P, most, 1, step), (P + (most - 1) * step, 1, 1, 1)) and not meet((P, most, 1, step), (P + (most - 1) * step + 1, 5, 1, 9))


LARGEST = dict(g=1 << 52, out=1 << 52, rows=(1 << 31) - 1, cols=1 << 18, ld_g=1 << 18, ld_out=1 << 18, type=1)


@pytest.mark.parametrize("items", [
    (dict(ld_g=64, ld_out=64, rows=40), dict(g=P + 32, out=P + 32, ld_g=128, ld_out=128, rows=20)),                             # columns of every row and of every second one
    (dict(ld_g=64, ld_out=64, rows=40), dict(g=P + 224, out=P + 224, ld_g=192, ld_out=192, rows=13)),
    (dict(ld_g=128, ld_out=128, rows=20), dict(g=P + 256, out=P + 256, ld_g=128, ld_out=128, rows=20)),                         # even rows and odd ones
    (dict(ld_g=16, ld_out=16), dict(g=P + 32, out=P + 32, rows=1, cols=8)),                                                     # a run between two rows
    (dict(ld_g=16, ld_out=16), dict(g=P + 32, out=P + 32, rows=2, cols=8, ld_g=32, ld_out=32)),
    (dict(ld_g=63, ld_out=63, rows=49), dict(g=P + 32, out=P + 32, ld_g=64, ld_out=64, rows=48)),                               # a row less than where they meet
])
def test_outputs_between_others_are_accepted(items):
    for order in (items, items[::-1]):
        # nothing is enqueued: one more tensor, far from them, has more elements than are taken
        assert slz.lib().slz_clip_by_norm(tensors(*order, LARGEST), len(order) + 1, 1.0, 0.0, 0, P - 256, P, 1 << 40, None) == TOO_LARGE


@pytest.mark.parametrize("items", [
    (dict(ld_g=64, ld_out=64, rows=40), dict(g=P + 28, out=P + 28, ld_g=128, ld_out=128, rows=20)),
    (dict(ld_g=64, ld_out=64, rows=40), dict(g=P + 32, out=P + 32, cols=57, ld_g=128, ld_out=128, rows=20)),
    # row j + 1 of one begins 220 - 4 j bytes behind row j of the other, which has 32: they meet from row 48 on
    (dict(ld_g=63, ld_out=63, rows=50), dict(g=P + 32, out=P + 32, ld_g=64, ld_out=64, rows=49)),
    (dict(ld_g=16, ld_out=16), dict(g=P + 32, out=P + 32, rows=1, cols=9)),
])
def test_outputs_that_meet_others_are_refused(items):
    for order in (items, items[::-1]):
        assert slz.lib().slz_clip_by_norm(tensors(*order, LARGEST), len(order) + 1, 1.0, 0.0, 0, P - 256, P, 1 << 40, None) == INVALID
