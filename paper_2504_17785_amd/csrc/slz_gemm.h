// Tiled matrix product on the matrix cores for the operators of include/silenzio_clear.h.
//
//   C[m][n] = sum_k A(m, k) B(n, k)      bf16 or f16 with sums in f32, int8 with sums in int32
//
// An operand is stored with k contiguous (rows m or n) or with m / n contiguous (rows k).  A workgroup of WM x WN waves computes a
// TM x TN tile; in steps of 128 bytes of k (64 or 128 elements) both operands' tiles go from memory straight to shared memory in
// 16-byte pieces, double buffered: the next step's pieces are under way while the matrix instructions run on this step's.  Where an operand's rows are k only
// part of the step overlaps: the compiler lets all loads finish before the first transposing read after them, as it cannot tell which buffer they fill.
// Shared memory has no padding (the direct loads write a wave's 1 KiB in a row), so a piece's place within its row is its
// index XOR some bits of the row number, chosen so that the lanes that read together meet different banks (tiles of 192 and 64 whose rows are k: two meet; for
// 192 other bits without that took the same time): a matrix-instruction operand is eight (int8: sixteen) consecutive k of one row.  Where rows are k it is read through the transposing ds_read_b64_tr_b16.
// The instruction gets B's rows as its rows and A's as its columns: a lane then holds consecutive columns of C for one row.
//
// Bounds: each step's loads go through a buffer descriptor that begins at the tile's corner and ends with the matrix, so rows past
// its end read as zero; pieces past the end of k are sent past the descriptor's end.  Columns past a row's end, where rows are
// k, may read the next row; they only reach sums that no one stores.
#pragma once
#include "slz_clear.h"
#include "slz_tiling.h"
#include <type_traits>
#include <utility>

typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s16 __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

enum { SLZ_EL_BF16 = SLZ_BF16, SLZ_EL_F16 = SLZ_F16, SLZ_EL_I8 = 3 };
template <int EL> struct slz_el { static constexpr int bytes = EL == SLZ_EL_I8 ? 1 : 2; using acc = v4f; };
template <> struct slz_el<SLZ_EL_I8> { static constexpr int bytes = 1; using acc = v4i32; };

template <int EL> __device__ __forceinline__ typename slz_el<EL>::acc slz_mma(v4i32 a, v4i32 b, typename slz_el<EL>::acc c) {
    if constexpr (EL == SLZ_EL_I8) return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    else if constexpr (EL == SLZ_EL_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// What a product is of.  The sum may run over several pairs of pieces of the operands (numbers carried in two or three pieces):
// pair s adds a_piece[s] and b_piece[s] bytes to the operands' addresses.
struct slz_gemm {
    const char *a, *b;
    int64_t lda, ldb;                // bytes between rows
    int64_t a_batch, b_batch;        // bytes between the matrices of a batch (grid z / split)
    uint32_t M, N, K;
    uint32_t pairs;
    int64_t a_piece[6], b_piece[6];
    uint32_t split;                  // ranges of steps, each by workgroups of its own
    uint32_t range;                  // steps of a range
    uint32_t tiles_m, tiles_n;
    uint32_t first_tile;             // of this launch
    uint32_t symmetric;              // only tiles on and below the diagonal
};

// Where the sums of a workgroup belong, for the epilogues.
struct slz_place {
    uint32_t m0, n0;                 // the wave's first row and column
    uint32_t lane, wave_m, wave_n;
    uint32_t tile_m, tile_n;
    uint32_t batch, range;
};

#define SLZ_LDS(p) ((__attribute__((address_space(3))) void *)(p))

// One operand's share of a wave: which pieces it brings, and how it reads its matrix operands.
template <bool ROWS_ARE_K, int T, int WAVES, int SPREAD> struct slz_tile {
    static constexpr int BYTES = T * 128, LOADS = BYTES / 1024 / WAVES;
    static_assert(LOADS * WAVES * 1024 == BYTES, "each wave brings whole kilobytes");
    static_assert(ROWS_ARE_K ? slz_places_t<T>() : slz_places_k<T, SPREAD>(), "every piece has a place, and is read from it");
    uint32_t off[LOADS], piece[LOADS];
    __device__ __forceinline__ void init(uint32_t wave, uint32_t lane, uint32_t ld) {
#pragma unroll
        for (int j = 0; j < LOADS; j++) {
            const uint32_t at = (wave * LOADS + j) * 1024u + lane * 16u;
            if constexpr (!ROWS_ARE_K) {
                const uint32_t row = at / 128u;
                piece[j] = slz_piece_k<SPREAD>(row, at / 16u & 7u);
                off[j] = row * ld + piece[j] * 16u;
            } else {
                const uint32_t row = at / (T * 2u);
                off[j] = row * ld + slz_piece_t<T>(row, at / 16u % (T / 8u)) * 16u;
                piece[j] = 0;
            }
        }
    }
    // base: the tile's corner at this step; bytes: from there to the matrix's end; pieces: of k that are left
    __device__ __forceinline__ void load(const char *base, uint32_t bytes, uint32_t pieces, char *lds, uint32_t wave) const {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes, 0x00020000);
#pragma unroll
        for (int j = 0; j < LOADS; j++) {
            uint32_t o = off[j];
            if constexpr (!ROWS_ARE_K) o = piece[j] < pieces ? o : 0x80000000u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, SLZ_LDS(lds + (wave * LOADS + j) * 1024u), 16, o, 0, 0, 0);
        }
    }
    // matrix operand `i` of the wave whose first row is `first`, for the half `kk` of the step
    template <int COUNT> __device__ __forceinline__ v4i32 read(const char *lds, uint32_t first, int i, int kk, uint32_t lane) const {
        const uint32_t r = lane & 15u, g = lane >> 4;
        if constexpr (!ROWS_ARE_K) {
            const uint32_t row = first + (SPREAD ? (r >> 2) * (COUNT * 4u) + i * 4u + (r & 3u) : i * 16u + r);
            return *(const v4i32 *)(lds + row * 128u + slz_piece_k<SPREAD>(row, kk * 4u + g) * 16u);
        } else {
            v4i32 v;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint32_t row = kk * 32u + g * 8u + h * 4u + (r >> 2);
                const uint32_t at = (first + i * 16u + (r & 3u) * 4u) * 2u;
                const char *p = lds + row * (T * 2u) + slz_piece_t<T>(row, at >> 4) * 16u + (at & 15u);
                const v4s16 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s16 *)p);
                const uint64_t b = __builtin_bit_cast(uint64_t, x);
                v[2 * h] = (int)(uint32_t)b;
                v[2 * h + 1] = (int)(uint32_t)(b >> 32);
            }
            return v;
        }
    }
};

// Tile, range of k and matrix of a workgroup.  The eight XCDs take workgroups in turn and each has an L2 of its own, so each gets a run of consecutive
// tiles, all of a range and of a matrix before the next; within the order, four tile rows go along the columns together.
__device__ __forceinline__ void slz_tile_of(uint32_t tiles_m, uint32_t tiles_n, uint32_t first_tile, uint32_t symmetric, uint32_t &tm, uint32_t &tn, uint32_t &range, uint32_t &batch) {
    uint32_t x = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
    const uint32_t total = gridDim.x * gridDim.y * gridDim.z, even = total & ~7u;
    if (x < even) x = (x & 7u) * (even >> 3) + (x >> 3);
    const uint32_t which = x / gridDim.x;
    x += first_tile - which * gridDim.x;
    batch = which / gridDim.y;
    range = which - batch * gridDim.y;
    if (symmetric) {                                   // row tm has tm + 1 tiles
        uint32_t t = (uint32_t)((__builtin_sqrtf(8.0f * (float)x + 1.0f) - 1.0f) * 0.5f);
        while (t * (t + 1u) / 2u > x) t--;
        while ((t + 1u) * (t + 2u) / 2u <= x) t++;
        tm = t;
        tn = x - t * (t + 1u) / 2u;
        return;
    }
    const uint32_t band = 4u * tiles_n, first = x / band * 4u, rows = min(4u, tiles_m - first), in = x % band;
    tm = first + in % rows;
    tn = in / rows;
}

// The order in which the compiler is to issue what stands before: so many reads of shared memory, then so many matrix instructions.
template <int READS, int MATRIX> __device__ __forceinline__ void slz_order() {
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    if constexpr (MATRIX > 0) __builtin_amdgcn_sched_group_barrier(0x8, MATRIX, 0);
}
template <int MI, int NI, int A_LDS, int B_LDS, int... G> __device__ __forceinline__ void slz_order_groups(std::integer_sequence<int, G...>) {
    (slz_order<(G + 2 < 2 * MI ? A_LDS : 0) + (G < MI ? B_LDS * ((G + 1) * NI / MI - G * NI / MI) : 0), NI>(), ...);
}

// Measured, 4096^3 with tiles of 256 (a large library product: 1.40 P/s bf16, 2.15 int8): bf16 1.32 P/s where k is contiguous, 1.04 where B's rows are k,
// 0.99 where both operands' are, int8 2.07 (8192^3 2.5).  The matrix cores are busy 48 to 54 % of the time, waves wait 29 to 41 %, no bank conflicts.  Neither side
// alone is the bound: with the loads off an earlier form ran at 1.46 instead of 1.21, with the matrix instructions off at the time of 1.74; and a loop of
// matrix instructions alone reaches 1.6 to 2.0 on random data, where the clock falls.
template <int EL, bool A_ROWS_K, bool B_ROWS_K, int TM, int TN, int WM, int WN, int PIECES, class EPI>
__global__ void __launch_bounds__(WM *WN * 64) k_gemm(const slz_gemm p, const EPI epi) {
    constexpr int WAVES = WM * WN, MI = TM / WM / 16, NI = TN / WN / 16, ES = slz_el<EL>::bytes, KS = 128 / ES;
    constexpr int A_LDS = A_ROWS_K ? 2 : 1, B_LDS = B_ROWS_K ? 2 : 1;           // instructions per operand
    using acc_t = typename slz_el<EL>::acc;
    using tile_a = slz_tile<A_ROWS_K, TM, WAVES, 0>;
    using tile_b = slz_tile<B_ROWS_K, TN, WAVES, B_ROWS_K ? 0 : NI * 4>;
    __shared__ __attribute__((aligned(1024))) char lds[2][PIECES * (tile_a::BYTES + tile_b::BYTES)];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wave_m = wave / WN, wave_n = wave % WN;
    uint32_t tm, tn, range, batch;
    slz_tile_of(p.tiles_m, p.tiles_n, p.first_tile, p.symmetric, tm, tn, range, batch);
    const uint32_t steps_k = (p.K + KS - 1) / KS, steps = steps_k * p.pairs;
    const uint32_t begin = range * p.range, end = min(steps, begin + p.range);

    // corners of the tile and the bytes from there to the matrices' ends, at k = 0
    const uint32_t m0 = tm * TM, n0 = tn * TN;
    const char *a0 = p.a + batch * p.a_batch + (A_ROWS_K ? (int64_t)m0 * ES : (int64_t)m0 * p.lda);
    const char *b0 = p.b + batch * p.b_batch + (B_ROWS_K ? (int64_t)n0 * ES : (int64_t)n0 * p.ldb);
    const uint32_t lda = (uint32_t)p.lda, ldb = (uint32_t)p.ldb;

    tile_a ta;
    tile_b tb;
    ta.init(wave, lane, lda);
    tb.init(wave, lane, ldb);
    acc_t acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = acc_t{0, 0, 0, 0};

    uint32_t pair = steps_k ? begin / steps_k : 0u, kt = begin - pair * steps_k;
    constexpr int SECOND = tile_a::BYTES + tile_b::BYTES;           // second pieces' place
    const auto load_step = [&](int buffer) {
        const uint32_t k0 = kt * KS, left = p.K - k0;
        const uint32_t pieces = min((left * ES + 15u) / 16u, 8u), rows_k = min(left, (uint32_t)KS);
        const char *a = a0 + p.a_piece[pair] + (A_ROWS_K ? (int64_t)k0 * lda : (int64_t)k0 * ES);
        const char *b = b0 + p.b_piece[pair] + (B_ROWS_K ? (int64_t)k0 * ldb : (int64_t)k0 * ES);
        const uint32_t bytes_a = A_ROWS_K ? (rows_k - 1) * lda + ((p.M - m0) * ES + 15u) / 16u * 16u : (min(p.M - m0, (uint32_t)TM) - 1) * lda + (left * ES + 15u) / 16u * 16u;
        const uint32_t bytes_b = B_ROWS_K ? (rows_k - 1) * ldb + ((p.N - n0) * ES + 15u) / 16u * 16u : (min(p.N - n0, (uint32_t)TN) - 1) * ldb + (left * ES + 15u) / 16u * 16u;
        ta.load(a, bytes_a, pieces, lds[buffer], wave);
        tb.load(b, bytes_b, pieces, lds[buffer] + tile_a::BYTES, wave);
        if constexpr (PIECES == 2) {
            ta.load(a + p.a_piece[1], bytes_a, pieces, lds[buffer] + SECOND, wave);
            tb.load(b + p.b_piece[1], bytes_b, pieces, lds[buffer] + SECOND + tile_a::BYTES, wave);
        }
        if (++kt == steps_k) { kt = 0; pair++; }
    };
    if (begin < end) load_step(0);
    for (uint32_t s = begin; s < end; s++) {
        const int buffer = (s - begin) & 1;
        __syncthreads();                               // this step's pieces are there; everyone is done with the other buffer
        if ((A_ROWS_K || PIECES == 2) && s + 1 < end) load_step(buffer ^ 1);
        const char *la = lds[buffer], *lb = la + tile_a::BYTES;
        if constexpr (PIECES == 2) {
            // numbers in two pieces, both loaded at once: three products of what is read once, the small ones first
#pragma unroll
            for (int kk = 0; kk < 2; kk++) {
                v4i32 fb[2][NI], fa[2];
#pragma unroll
                for (int j = 0; j < NI; j++)
#pragma unroll
                    for (int q = 0; q < 2; q++) fb[q][j] = tb.template read<NI>(lb + q * SECOND, wave_n * (NI * 16), j, kk, lane);
#pragma unroll
                for (int i = 0; i < MI; i++) {
#pragma unroll
                    for (int q = 0; q < 2; q++) fa[q] = ta.template read<MI>(la + q * SECOND, wave_m * (MI * 16), i, kk, lane);
#pragma unroll
                    for (int j = 0; j < NI; j++) {
                        acc[i][j] = slz_mma<EL>(fb[0][j], fa[1], acc[i][j]);
                        acc[i][j] = slz_mma<EL>(fb[1][j], fa[0], acc[i][j]);
                        acc[i][j] = slz_mma<EL>(fb[0][j], fa[0], acc[i][j]);
                    }
                }
            }
            continue;
        }
        // 2 MI groups of NI matrix instructions, each with one operand of A; A's operands are read two groups ahead, B's for the
        // second half during the first: shared memory and the matrix cores are busy for about as long, and so at the same time
        v4i32 fa[3], fb[2][NI];
#pragma unroll
        for (int j = 0; j < NI; j++) fb[0][j] = tb.template read<NI>(lb, wave_n * (NI * 16), j, 0, lane);
#pragma unroll
        for (int g = 0; g < 2; g++) fa[g] = ta.template read<MI>(la, wave_m * (MI * 16), g % MI, g / MI, lane);
        if constexpr (A_ROWS_K) slz_order<B_LDS * NI + A_LDS * 2, 0>();
        else {
            // the next step's loads, behind the first reads (before them, where both operands' rows are k: 2 % either way)
            __builtin_amdgcn_sched_barrier(0);
            if (s + 1 < end) load_step(buffer ^ 1);
        }
#pragma unroll
        for (int g = 0; g < 2 * MI; g++) {
            if (g + 2 < 2 * MI) fa[(g + 2) % 3] = ta.template read<MI>(la, wave_m * (MI * 16), (g + 2) % MI, (g + 2) / MI, lane);
            if (g < MI)
#pragma unroll
                for (int j = g * NI / MI; j < (g + 1) * NI / MI; j++) fb[1][j] = tb.template read<NI>(lb, wave_n * (NI * 16), j, 1, lane);
#pragma unroll
            for (int j = 0; j < NI; j++) acc[g % MI][j] = slz_mma<EL>(fb[g / MI][j], fa[g % 3], acc[g % MI][j]);
        }
        slz_order_groups<MI, NI, A_LDS, B_LDS>(std::make_integer_sequence<int, 2 * MI>());
    }
    __syncthreads();                                   // the epilogue may use the shared memory
    const slz_place at{m0 + wave_m * (MI * 16), n0 + wave_n * (NI * 16), lane, wave_m, wave_n, tm, tn, batch, range};
    epi.template run<MI, NI, !B_ROWS_K, WM, WN>(acc, at, p, (float *)lds[0]);
}

// Row of acc[i][..] in this lane, and column of acc[..][j][e]: RUN (B's k contiguous) gives a lane NI * 4 consecutive columns, else 4.
__device__ __forceinline__ uint32_t slz_row(const slz_place &at, int i) { return at.m0 + i * 16u + (at.lane & 15u); }
template <int NI, bool RUN> __device__ __forceinline__ uint32_t slz_col(const slz_place &at, int j) {
    return at.n0 + (RUN ? (at.lane >> 4) * (NI * 4u) + j * 4u : j * 16u + (at.lane >> 4) * 4u);
}

// ---- epilogues ---------------------------------------------------------------------------------------------------------------
// What is done with a sum, with all that is the same for all of them read: a thread's stores might change it, as far as the compiler knows
template <class F> __device__ __forceinline__ F slz_ready(const F &f) { return f; }
// the sum times a constant and, if given, a number that the operand was divided by
struct slz_times { float by; __device__ __forceinline__ float operator()(uint32_t, uint32_t, uint32_t, float sum) const { return sum * by; } };
struct slz_times_unit {
    const float *unit;
    float by;
};
__device__ __forceinline__ slz_times slz_ready(const slz_times_unit &f) { return {f.unit ? *f.unit * f.by : 1.0f}; }

// out[m][n] = f(m, n, sum), rounded once to the type
template <class F> struct slz_store_epi {
    void *out;
    int type;
    int64_t ld, batch_stride;        // elements
    uint32_t aligned;                // rows begin at multiples of 16 bytes
    F f;
    static constexpr bool any_side = true;
    static constexpr int widest = 256;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *) const {
        constexpr int C = RUN ? NI * 4 : 4, PARTS = RUN ? 1 : NI;
        const uint32_t eb = slz_type_bytes(type);
        const auto value = slz_ready(f);
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
            if (m >= p.M) continue;
#pragma unroll
            for (int q = 0; q < PARTS; q++) {
                const uint32_t n = slz_col<NI, RUN>(at, q);
                if (n >= p.N) continue;
                float v[C];
#pragma unroll
                for (int c = 0; c < C; c++) v[c] = value(at.batch, m, min(n + c, p.N - 1), acc[i][q + c / 4][c % 4]);
                slz_put_run<C>((char *)out + (at.batch * batch_stride + (int64_t)m * ld + n) * eb, type, v, p.N - n, aligned);
            }
        }
    }
};

// the sums themselves, or added to what is there, of each range: ws[range][batch][M][ld], ld a multiple of 16
template <class T> struct slz_partial_epi {
    T *ws;
    uint32_t ld, batches, add;
    static constexpr bool any_side = true;
    static constexpr int widest = 256;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *) const {
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
            if (m >= p.M) continue;
            T *row = ws + (((size_t)at.range * batches + at.batch) * p.M + m) * ld;
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const uint32_t n = slz_col<NI, RUN>(at, j);
                if (n >= p.N) continue;
                ACC v = acc[i][j];
                if (add) v += *(const ACC *)(row + n);
                *(ACC *)(row + n) = v;
            }
        }
    }
};
// out[m][n] = f(m, n, sum of the ranges' sums in their order)
template <class T, class F>
__global__ void __launch_bounds__(256) k_join(const T *ws, uint32_t ranges, uint32_t M, uint32_t N, uint32_t ld, void *out, int type, int64_t ld_out, F f) {
    const size_t total = (size_t)M * ((N + 3) / 4), stride = (size_t)M * ld;
    typedef T t4 __attribute__((ext_vector_type(4)));
    const auto value = slz_ready(f);
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        const uint32_t m = (uint32_t)(g / ((N + 3) / 4)), n = (uint32_t)(g % ((N + 3) / 4)) * 4;
        t4 sum = *(const t4 *)(ws + (size_t)m * ld + n);
        for (uint32_t r = 1; r < ranges; r++) sum += *(const t4 *)(ws + r * stride + (size_t)m * ld + n);
        for (uint32_t c = 0; c < 4 && n + c < N; c++) slz_put(out, type, (size_t)m * ld_out + n + c, value(0, m, n + c, sum[c]));
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------
template <int TM_, int TN_, int WM_, int WN_> struct slz_tiling { static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_; };
using slz_tiles_256 = slz_tiling<256, 256, 2, 4>;
using slz_tiles_192 = slz_tiling<192, 192, 2, 4>;
using slz_tiles_128 = slz_tiling<128, 128, 2, 2>;
using slz_tiles_64 = slz_tiling<64, 64, 2, 2>;

// workspace of the ranges' sums
static inline uint32_t slz_ranges_ld(uint32_t N) { return (N + 15u) & ~15u; }
static inline size_t slz_ranges_bytes(const slz_choice &c, uint32_t M, uint32_t N) { return c.split > 1 ? up256((size_t)c.split * M * slz_ranges_ld(N) * 4) : 0; }

static inline slz_gemm slz_gemm_of(const slz_operand &a, const slz_operand &b, uint32_t M, uint32_t N, uint32_t K) {
    slz_gemm p = {};
    p.a = a.p; p.b = b.p; p.lda = a.ld; p.ldb = b.ld;
    p.M = M; p.N = N; p.K = K;
    p.split = 1;
    // three pieces each: the products whose share of the result is 2^-16 and more, the small ones first
    static const int order[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
    p.pairs = a.pieces == 3 ? 6 : 1;
    for (uint32_t i = 0; i < p.pairs && p.pairs == 6; i++) {
        p.a_piece[i] = order[i][0] * a.piece;
        p.b_piece[i] = order[i][1] * b.piece;
    }
    return p;
}
static inline uint32_t slz_gemm_steps(const slz_gemm &p, int element_bytes) {
    const uint32_t ks = 128 / element_bytes;
    return (p.K + ks - 1) / ks * p.pairs;
}

template <class T, int EL, bool A_ROWS_K, bool B_ROWS_K, int PIECES = 1, class EPI>
static int slz_gemm_launch(slz_gemm p, const EPI &epi, uint32_t batches, hipStream_t s) {
    p.tiles_m = (p.M + T::TM - 1) / T::TM;
    p.tiles_n = (p.N + T::TN - 1) / T::TN;
    p.range = (slz_gemm_steps(p, slz_el<EL>::bytes) + p.split - 1) / p.split;
    const uint64_t tiles = p.symmetric ? (uint64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (uint64_t)p.tiles_m * p.tiles_n;
    if (tiles == 0 || batches == 0) return SLZ_OK;
    if (tiles * p.split * batches > 0x7fffffffu) return SLZ_E_TOO_LARGE;
    constexpr uint32_t threads = T::WM * T::WN * 64;
    for (p.first_tile = 0; p.first_tile < tiles; p.first_tile += slz_most_blocks(threads)) {
        const uint32_t left = (uint32_t)tiles - p.first_tile, most = slz_most_blocks(threads);
        hipLaunchKernelGGL((k_gemm<EL, A_ROWS_K, B_ROWS_K, T::TM, T::TN, T::WM, T::WN, PIECES, EPI>), dim3(left < most ? left : most, p.split, batches),
                           dim3(threads), 0, s, p, epi);
    }
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}
// operands of two pieces (a_piece[1] and b_piece[1]: the second ones)
template <int EL, bool A_ROWS_K, bool B_ROWS_K, class EPI>
static int slz_gemm_run2(const slz_gemm &p, const EPI &epi, uint32_t batches, hipStream_t s) {
    return slz_gemm_launch<slz_tiles_64, EL, A_ROWS_K, B_ROWS_K, 2>(p, epi, batches, s);
}
template <int EL, bool A_ROWS_K, bool B_ROWS_K, class EPI>
static int slz_gemm_run(const slz_gemm &p, const EPI &epi, uint32_t side, uint32_t batches, hipStream_t s) {
    if constexpr (EPI::widest == 256)
        if (side == 256) return slz_gemm_launch<slz_tiles_256, EL, A_ROWS_K, B_ROWS_K>(p, epi, batches, s);
    if constexpr (EPI::any_side)
        if (side == 192) return slz_gemm_launch<slz_tiles_192, EL, A_ROWS_K, B_ROWS_K>(p, epi, batches, s);
    // eight waves where an operand's rows are k: 768^2 by 4096 deep 58 us, with four 67; 43 and 45 where k is contiguous, but 4096^3 141 and 133
    if (side == 128) return slz_gemm_launch<typename std::conditional<B_ROWS_K, slz_tiling<128, 128, 2, 4>, slz_tiles_128>::type, EL, A_ROWS_K, B_ROWS_K>(p, epi, batches, s);
    return slz_gemm_launch<slz_tiles_64, EL, A_ROWS_K, B_ROWS_K>(p, epi, batches, s);
}
// out = f(sums): at once, or where the choice has several ranges of k by their sums in `ranges` (slz_ranges_bytes) and a second launch
template <int EL, bool A_ROWS_K, bool B_ROWS_K, class F>
static int slz_gemm_to(slz_gemm p, const slz_choice &c, const F &f, void *out, int type, int64_t ld, char *ranges, hipStream_t s) {
    using sum_t = typename std::conditional<EL == SLZ_EL_I8, int, float>::type;
    if (c.split == 1)
        return slz_gemm_run<EL, A_ROWS_K, B_ROWS_K>(p, slz_store_epi<F>{out, type, ld, 0, slz_in_place(out, 16, ld, slz_type_bytes(type)), f}, c.side, 1, s);
    p.split = c.split;
    const uint32_t ld_r = slz_ranges_ld(p.N);
    const int rc = slz_gemm_run<EL, A_ROWS_K, B_ROWS_K>(p, slz_partial_epi<sum_t>{(sum_t *)ranges, ld_r, 1, 0}, c.side, 1, s);
    if (rc != SLZ_OK || p.M == 0 || p.N == 0) return rc;
    hipLaunchKernelGGL((k_join<sum_t, F>), ew_grid((size_t)p.M * ((p.N + 3) / 4)), dim3(256), 0, s, (const sum_t *)ranges, c.split, p.M, p.N, ld_r, out, type, ld, f);
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}
