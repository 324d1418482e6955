"""What of the tiled matrix product needs no GPU (csrc/slz_tiling.h): every piece of a tile is read from where it was put, and the shapes of
tests/clear_tilings.py take the tilings that stand beside them."""
import ctypes
import os
import shutil
import subprocess

import pytest

from tests import clear_tilings

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = r"""
#include "slz_tiling.h"
template <int T> static int wrong_t() {
    // what the loads bring: place q of row r of shared memory holds piece slz_piece_t(r, q) of the row; what is read as piece p has to be p
    int wrong = 0;
    for (uint32_t row = 0; row < 64; row++)
        for (uint32_t p = 0; p < T / 8; p++) {
            const uint32_t q = slz_piece_t<T>(row, p);
            wrong += q >= T / 8 || slz_piece_t<T>(row, q) != p;
        }
    return wrong;
}
template <int T, int SPREAD> static int wrong_k() {
    int wrong = 0;
    for (uint32_t row = 0; row < T; row++)
        for (uint32_t p = 0; p < 8; p++) {
            const uint32_t q = slz_piece_k<SPREAD>(row, p);
            wrong += q >= 8 || slz_piece_k<SPREAD>(row, q) != p;
        }
    return wrong;
}
extern "C" int rows_are_k(int side) { return side == 64 ? wrong_t<64>() : side == 128 ? wrong_t<128>() : side == 192 ? wrong_t<192>() : wrong_t<256>(); }
extern "C" int k_in_a_row(int side) {
    return side == 64 ? wrong_k<64, 0>() + wrong_k<64, 8>() : side == 128 ? wrong_k<128, 0>() + wrong_k<128, 8>() + wrong_k<128, 16>()
         : side == 192 ? wrong_k<192, 0>() + wrong_k<192, 12>() : wrong_k<256, 0>() + wrong_k<256, 16>();
}
extern "C" void choose(uint32_t M, uint32_t N, uint32_t steps, uint32_t batches, int symmetric, uint32_t ranges, int rows_k, int any_side, uint32_t pieces,
                       double *out) {
    const slz_choice c = slz_choose(M, N, steps, batches, symmetric, ranges, rows_k, any_side, pieces);
    out[0] = c.side;
    out[1] = c.split;
    out[2] = c.us;
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("tiling")
    (at / "host.cpp").write_text(HOST)
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2504_17785_amd", "csrc"),
                    "-o", str(at / "host.so"), str(at / "host.cpp")], check=True)
    L = ctypes.CDLL(str(at / "host.so"))

    def choose(M, N, steps, batches=1, symmetric=False, ranges=1, rows_k=False, any_side=True, pieces=1):
        out = (ctypes.c_double * 3)()
        L.choose(M, N, steps, batches, symmetric, ranges, rows_k, any_side, pieces, out)
        return int(out[0]), int(out[1]), out[2]

    L.chosen = choose
    return L


@pytest.mark.parametrize("side", (64, 128, 192, 256))
def test_pieces_are_read_from_where_they_were_put(host, side):
    assert host.rows_are_k(side) == 0
    assert host.k_in_a_row(side) == 0


def over(a, b):
    return -(-a // b)


def test_choices_for_products(host):
    for (m, n, k), want in clear_tilings.PRODUCTS:
        assert host.chosen(m, n, over(k, 128), ranges=16)[:2] == want, (m, n, k)
    assert {t[0] for _, t in clear_tilings.PRODUCTS} == {64, 128, 192, 256}


def test_choices_for_gradients(host):
    seen = {False: set(), True: set()}
    for (m, n, k), wide, da, db in clear_tilings.GRADS:
        pairs = 6 if wide else 1
        assert host.chosen(m, k, over(n, 64) * pairs, ranges=16, rows_k=True)[:2] == da, (m, n, k)
        assert host.chosen(n, k, over(m, 64) * pairs, ranges=16, rows_k=True)[:2] == db, (m, n, k)
        seen[wide] |= {("da", da[0], da[1] > 1), ("db", db[0], db[1] > 1)}
    for which in ("da", "db"):
        assert {side for w, side, _ in seen[False] | seen[True] if w == which} == {64, 128, 192, 256}
        assert {side for w, side, cut in seen[False] | seen[True] if w == which and cut} == {64, 128, 192, 256}


def test_choices_for_losses(host):
    seen = set()
    for (tokens, inner, vocab), wide, pieces, z, dh, dw in clear_tilings.LOSSES:
        words = vocab
        if pieces:                                     # f32: words whose three pieces of w or g take 128 MiB
            words = min((128 << 20) // (6 * tokens), (128 << 20) // (6 * inner)) & ~255
            assert words < vocab
        pairs = 6 if wide else 1
        assert host.chosen(tokens, words, over(inner, 64) * pairs, any_side=False)[0] == z, (tokens, inner, vocab)
        assert host.chosen(tokens, inner, over(words, 64) * pairs, ranges=64, rows_k=True)[:2] == dh, (tokens, inner, vocab)
        assert host.chosen(words, inner, over(tokens, 64) * pairs, ranges=32, rows_k=True)[:2] == dw, (tokens, inner, vocab)
        seen |= {("z", z), ("dh", dh[0]), ("dw", dw[0])}
    assert seen == {("z", s) for s in (64, 128, 256)} | {(w, s) for w in ("dh", "dw") for s in (64, 128, 192, 256)}


def test_choices_for_updates(host):
    seen = set()
    for (batch, m, n), halves, gram, polynomial, apply in clear_tilings.UPDATES:
        def chosen(N, steps, symmetric, ranges, rows_k):
            if not halves:
                return (*host.chosen(m, N, steps, batch, symmetric, ranges, rows_k), 1)
            in_turn = host.chosen(m, N, steps * 3, batch, symmetric, ranges, rows_k)
            together = host.chosen(m, N, steps, batch, symmetric, ranges, rows_k, True, 2)
            return (*together, 2) if together[2] < in_turn[2] else (*in_turn, 1)

        def short(c):
            return c[:2] + c[3:]

        whole, cut = chosen(m, over(n, 64), True, 1, False), chosen(m, over(n, 64), False, 32, False)
        assert short(cut if cut[2] < whole[2] else whole) == gram, (batch, m, n)
        assert short(chosen(m, over(m, 64), True, 1, False)) == polynomial, (batch, m, n)
        assert short(chosen(n, over(m, 64), False, 1, True)) == apply, (batch, m, n)
        seen |= {("gram", gram[0], gram[2]), ("polynomial", polynomial[0], polynomial[2]), ("apply", apply[0], apply[2])}
    for which, sides in (("gram", (64, 128, 192)), ("polynomial", (64, 128, 192)), ("apply", (64, 128, 192, 256))):
        assert {side for w, side, _ in seen if w == which} == set(sides)
        assert (which, 64, 2) in seen
