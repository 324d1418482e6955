// What of the tiled matrix product (slz_gemm.h) needs no GPU: where a piece of a tile lies in shared memory, and which tiling a product takes.
#pragma once
#include <stdint.h>
#include <initializer_list>

// ---- places ------------------------------------------------------------------------------------------------------------------
// The place of a 16-byte piece within its tile row, from the piece's number, and the other way round: both XOR the same bits of the row number.
// Rows of 128 bytes (k contiguous), eight pieces.  SPREAD: the lanes of a read take rows r and (r >> 2) * SPREAD apart instead of consecutive ones.
template <int SPREAD> constexpr uint32_t slz_piece_k(uint32_t row, uint32_t piece) {
    return piece ^ (SPREAD == 0 ? row & 7u : (row & 3u) | ((row / (SPREAD ? SPREAD : 1)) & 1u) << 2);
}
// Rows of T elements (rows are k), whole 32-byte pairs of pieces.  The XOR must not leave the row: it stays within aligned groups of as many pieces as
// the largest power of two that divides their number (T = 192: 24 pieces, groups of 8).
template <int T> constexpr uint32_t slz_piece_t(uint32_t row, uint32_t piece) {
    constexpr uint32_t pieces = T / 8, group = pieces & (0u - pieces);
    return piece ^ ((((row & 3u) | ((row >> 3) & 1u) << 2) << 1) & (group - 1u));
}
// every row's pieces have places of their own within the row
template <int T, int SPREAD> constexpr bool slz_places_k() {
    for (uint32_t row = 0; row < T; row++) {
        uint32_t taken = 0;
        for (uint32_t p = 0; p < 8; p++) taken |= 1u << slz_piece_k<SPREAD>(row, p);
        if (taken != 0xffu) return false;
    }
    return true;
}
template <int T> constexpr bool slz_places_t() {
    static_assert(T % 8 == 0 && T / 8 <= 32, "");
    for (uint32_t row = 0; row < 64; row++) {
        uint64_t taken = 0;
        for (uint32_t p = 0; p < T / 8; p++) taken |= (uint64_t)1 << slz_piece_t<T>(row, p);
        if (taken != ((uint64_t)1 << T / 8) - 1) return false;
    }
    return true;
}

// ---- choice ------------------------------------------------------------------------------------------------------------------
// Which tiling and how many ranges of k.  A step of 128 bytes of k takes a compute unit 1.5 us with a tile of 256 a side, 0.95 with one of 192, 0.62
// with one of 128 and 0.88 with two at once, 0.33 with one of 64 and 0.18 for each of several (measured at 4096 deep: 3840^2 with 256: 99 us;
// 2688^2 with 192: 63, with 128: 57; 768^2 with 256, 192, 128: 85, 58, 43).  Large tiles read less for each product, small ones fill the chip with less
// and leave less of it idle at the end.  Ranges of k cost a second launch that reads their sums.
// rows_k: an operand's rows are k.  All sides then take longer, and 192 by more than the others: 2688^2 with 256, 192, 128, 64: 111, 81, 67, 93 us where
// 92, 62, 59, 83 with k contiguous, 5184^2 by 2048 deep 121, 129, 127, 165 (98, 102, 108, 151).  The estimate compares sides, so only 192 gets another figure.
// pieces: of a number that are loaded together, in tiles of 64 (0.5 us a step, 0.42 for each of several; one of 128 1.9, more than the four in its place)
struct slz_choice { uint32_t side, split; double us; uint32_t pieces = 1; };
static inline double slz_step_us(uint32_t side, double tiles, uint32_t pieces, bool rows_k) {
    const auto rounds = [&](double at_once) { return (double)(uint64_t)((tiles + at_once - 1) / at_once); };
    if (pieces == 2) return rounds(256) * 0.42 > 0.5 ? rounds(256) * 0.42 : 0.5;
    if (side == 256) return rounds(256) * 1.5;
    if (side == 192) return rounds(256) * (rows_k ? 1.1 : 0.95);
    if (side == 64) return rounds(256) * 0.18 > 0.33 ? rounds(256) * 0.18 : 0.33;
    const double pairs = (double)(uint64_t)(tiles / 512), rest = tiles - pairs * 512;
    return pairs * 0.88 + (rest > 256 ? 0.88 : rest > 0 ? 0.62 : 0.0);
}
static inline slz_choice slz_choose(uint32_t M, uint32_t N, uint32_t steps, uint32_t batches, bool symmetric, uint32_t most_ranges, bool rows_k = false,
                                    bool any_side = true, uint32_t pieces = 1) {
    slz_choice best = {64, 1, 1e30};
    for (const uint32_t side : {256u, 192u, 128u, 64u}) {
        if ((side == 192 && !any_side) || (side == 256 && symmetric) || (side > 64 && pieces == 2)) continue;
        const double tm = (M + side - 1) / side, tn = (N + side - 1) / side, tiles = (symmetric ? tm * (tm + 1) / 2 : tm * tn) * batches;
        for (uint32_t split = 1; split <= most_ranges && (split == 1 || steps >= 4 * split); split *= 2) {
            double us = ((steps + split - 1) / split) * slz_step_us(side, tiles * split, pieces, rows_k);
            if (split > 1) us += 4.0 + (double)M * N * batches * 4.0 * (split + 1) / 3e6;
            if (us < best.us) best = {side, split, us, pieces};
        }
    }
    return best;
}
