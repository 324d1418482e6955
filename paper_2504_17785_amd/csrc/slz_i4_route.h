// Which kernel takes a product with 4-bit weights (slz_i4.hip); host code that needs no GPU.
#pragma once
#include <stddef.h>
#include "slz_tiling.h"
#ifndef __HIPCC__
#define __host__
#define __device__
#endif

#define I4_BLOCK 128u                // entries of a block, 64 bytes
#define I4_THREADS 512u              // of a workgroup that streams weights
#define I4_LDS (128u << 10)          // shared memory for x and scales
__host__ __device__ static inline uint32_t i4_blocks(uint32_t cols) { return (cols + I4_BLOCK - 1) / I4_BLOCK; }
__host__ __device__ static inline uint32_t i4_groups(uint32_t cols, uint32_t group) { return (cols + group - 1) / group; }
// k_thin_i4: bytes of a row of x in shared memory, 16 bytes apart in the banks; floats of a row of scales: odd, and up to three past its end are there
__host__ __device__ static inline uint32_t i4_pitch(uint32_t k) { return i4_blocks(k) * 256u + 16u; }
__host__ __device__ static inline uint32_t i4_pitch_scales(uint32_t groups) { return (groups | 3u) + 2u; }
static inline size_t i4_thin_bytes(uint32_t m, uint32_t k, uint32_t group, bool wide, uint32_t nb) {
    return (size_t)m * i4_pitch(k) * (wide ? 3 : 1) + (size_t)i4_pitch_scales(i4_groups(k, group)) * 64 * nb;
}

// THIN: k_thin_i4; ROWS: k_rows_i4 with the tiles `kind`; TILES: the matrix product of the values, tiled as c says.
// A phase of k_rows_i4 takes 1.0 us with tiles of 16 by 32, 0.8 with 16 by 64, 1.0 with 32 by 64, 1.55 with 64 by 64 and 2.0 with 128 by 128, on every compute
// unit at once, and a tile's beginning and end together 0.6, 0.5, 0.6, 3.2 and 7.5 (f32: 1.25 and 0.4 with 16 by 64); the matrix product of the values, which
// are laid out for it at 4.2 TB/s, takes more launches.
// Measured and estimated, bf16, 4096 x 4096 with 64, 256, 512, 1024, 2048 rows: streamed 10.0, 17.8, 36, 44, 85 (12, 19, 35, 43, 83), laid out 29, 38, 52, 62,
// 75 (28, 38, 41, 58, 74); 8192 x 8192 with 512: 74 (75) and 107 (125); 4096 x 1024 with 1024 and 2048: 19.5, 36 (19, 35) and 28, 33 (20, 25); f32, 8192 x
// 8192 with 512 and 1024: 320, 642 (330, 656) and 451, 755 (432, 725).
struct i4_kind { uint32_t tm, tn, wk; double us, ends; };                         // wk: blocks of k in a phase
static const i4_kind I4_KINDS[] = {{16, 32, 8, 1.0, 0.6}, {16, 64, 4, 0.8, 0.5}, {32, 64, 4, 1.0, 0.6}, {64, 64, 4, 1.55, 3.2}, {128, 128, 2, 2.0, 7.5}}, I4_KINDS_WIDE[] = {{16, 64, 4, 1.25, 0.4}};
struct i4_route { enum { THIN, ROWS, TILES } way; int kind; slz_choice c; };
// wide: f32; n is at most 2^22, the longest row of y
static inline i4_route i4_route_of(uint32_t m, uint32_t n, uint32_t k, bool wide, uint32_t group) {
    i4_route R = {i4_route::TILES, 0, slz_choose(m, n, (k + 63) / 64 * (wide ? 6 : 1), 1, false, 16)};
    // k_thin_i4's time grows with each row, k_rows_i4's not within a tile, and with more than 16384 rows of weights the latter's wider tiles fill the chip
    // (bf16, one row by 32768 x 2048: 11.1 and 10.5 us; 8192 x 4096: one row 6.9 and 7.7, three 8.1 and 7.9; 4096 x 4096: one 5.5 and 7.2, eight 7.4 and 7.4;
    // f32, four rows by 4096 x 4096 8.0 and 13.3, by 8192 x 4096 14.1 and 13.6, eight by 8192 x 2048 11.8 and 8.9).  For long rows the border is early: one row by
    // 24576 x 4096 12.8 and 17.4.
    const bool few = m <= 2 ? n <= 16384 : m <= 8 && n <= 4096;
    if ((few || (m <= 8 && k < 8)) && i4_thin_bytes(m, k, group, wide, 2) <= I4_LDS) R.way = i4_route::THIN;
    else if (k >= 8 && n > 0) {
        double least = 8.0 + (double)n * k * (wide ? 6.5 : 2.5) / 4.2e6 + R.c.us;
        for (int i = 0; i < (wide ? 1 : 5); i++) {
            const i4_kind &of = wide ? I4_KINDS_WIDE[i] : I4_KINDS[i];
            const uint64_t tiles = (uint64_t)((m + of.tm - 1) / of.tm) * ((n + of.tn - 1) / of.tn), phases = (i4_blocks(k) + of.wk - 1) / of.wk;
            const double us = 3.5 + (double)((tiles + 255) / 256) * (phases * of.us + of.ends);
            if (us >= least || tiles > 0xffffffffu / I4_THREADS) continue;         // threads of a launch stay below 2^32
            least = us;
            R.way = i4_route::ROWS;
            R.kind = i;
        }
    }
    return R;
}
