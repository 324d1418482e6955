"""The shapes of tests/clear_i4_routes.py take the kernels that stand beside them, and what the choice allows fits a launch."""
import ctypes
import os
import shutil
import subprocess

import pytest

from tests import clear_i4_routes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = r"""
#include "slz_i4_route.h"
extern "C" void route(uint32_t m, uint32_t n, uint32_t k, int wide, uint32_t group, int *out) {
    const i4_route R = i4_route_of(m, n, k, wide, group);
    out[0] = R.way;
    out[1] = R.kind;
    out[2] = (int)i4_thin_bytes(m < 9 ? m : 0, k, group, wide, 2);
    const i4_kind &of = wide ? I4_KINDS_WIDE[R.kind] : I4_KINDS[R.kind];
    const uint64_t tiles = (uint64_t)((m + of.tm - 1) / of.tm) * ((n + of.tn - 1) / of.tn);
    out[3] = tiles * I4_THREADS < 0x100000000ull;
}
"""
WAYS = ("thin", "rows", "tiles")


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("route")
    (at / "host.cpp").write_text(HOST)
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2504_17785_amd", "csrc"),
                    "-o", str(at / "host.so"), str(at / "host.cpp")], check=True)
    L = ctypes.CDLL(str(at / "host.so"))

    def of(m, n, k, group, wide):
        out = (ctypes.c_int * 4)()
        L.route(ctypes.c_uint32(m), ctypes.c_uint32(n), ctypes.c_uint32(k), int(wide), ctypes.c_uint32(group), out)
        return (WAYS[out[0]], out[1]), out[2], out[3]
    return of


def test_shapes_take_their_kernels(route):
    assert {(wide, taken) for _, wide, taken in clear_i4_routes.ROUTES} == {
        *((False, ("rows", i)) for i in range(5)), (True, ("rows", 0)), *((w, (way, 0)) for w in (False, True) for way in ("thin", "tiles"))}
    for shape, wide, taken in clear_i4_routes.ROUTES:
        assert route(*shape, wide)[0] == taken, (shape, wide)


def test_what_is_chosen_fits(route):
    sizes = (1, 2, 8, 9, 100, 5000, 1 << 17, 1 << 22)
    for wide in (False, True):
        for group in (32, 64, 128):
            for m in (*sizes, (1 << 22) + 1, 1 << 27, (1 << 31) - 1):
                for n in sizes:
                    for k in (0, 1, 7, 8, 1000, 20000, 1 << 22):
                        (way, _), thin, fits = route(m, n, k, group, wide)
                        if way == "thin":
                            assert m <= 8 and thin <= 160 << 10
                            assert (n + 15) // 16 * 512 < 1 << 32
                        if way == "rows":
                            assert k >= 8 and fits
