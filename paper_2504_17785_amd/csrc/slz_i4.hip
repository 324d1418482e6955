// Layers whose weights have 4 bits (include/silenzio_clear.h): quantisation by groups, the values, the product and its gradient.
//
// A word of a 4-bit row has eight consecutive entries, which is what a lane feeds to a matrix instruction, and a block of 128 entries lies so that the
// four words that a lane needs for the block's four instructions are 16 bytes in a row.
#include "slz_gemm.h"
#include "slz_i4_route.h"

#define THIN_WAVES (I4_THREADS / 64)

// four entries of a word (half 0 or 1) in the order of k, times a scale: as bytes they are subnormal e4m3 numbers (i4_operand)
__device__ __forceinline__ void i4_numbers(uint32_t word, int half, float scale, float *v) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const uint32_t w = half ? word >> 4 : word, b = (w & 0x07070707u) | (w << 4 & 0x80808080u);
    const f2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(b, 512.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(b, 512.0f, true);
    v[0] = lo[0] * scale;
    v[1] = lo[1] * scale;
    v[2] = hi[0] * scale;
    v[3] = hi[1] * scale;
}
// place of the word with the entries 8 i to 8 i + 7 of a row
__device__ __forceinline__ uint32_t i4_place(uint32_t i) { return (i & ~15u) + (i & 3u) * 4u + (i >> 2 & 3u); }

// ---- quantisation ------------------------------------------------------------------------------------------------------------------
// How the kernels that go over whole matrices share them: a wave has 64 words of a row, or 32 or 16 of two or four rows where a row has no more, and as many
// of the three rows (or twos, or fours) that follow.  In rows further apart 8192 x 8192 took 34.6 us instead of 32.6 (quantisation of bf16) and 91 instead of
// 83 (f32 values), in runs of 256 words of one row 37 and 83.
#define I4_DOWN 4u
struct i4_walk {
    uint32_t i, row, next, step;     // the lane's word within a row; its first row, those that follow it, and the distance to the next ones
    __device__ __forceinline__ i4_walk(uint32_t wide) {                            // log2 of the words of a row that a wave has
        const uint32_t lane = threadIdx.x & 63u, rows = 64u >> wide;
        i = (blockIdx.x << wide) + (lane & ((1u << wide) - 1u));
        row = (blockIdx.y * 4u + (threadIdx.x >> 6)) * I4_DOWN * rows + (lane >> wide);
        next = rows;
        step = gridDim.y * 4u * I4_DOWN * rows;
    }
};
static inline uint32_t walk_wide(uint32_t words) { return words <= 16 ? 4u : words <= 32 ? 5u : 6u; }
static inline dim3 walk_grid(uint32_t rows, uint32_t words) {
    const uint32_t wide = walk_wide(words), x = (words + (1u << wide) - 1) >> wide;
    const uint64_t of_block = (4u << (6 - wide)) * I4_DOWN, y = (rows + of_block - 1) / of_block, most = 16384u / x ? 16384u / x : 1u;
    return dim3(x, (unsigned)(y < most ? y : most));
}
__device__ __forceinline__ uint32_t i4_max(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int CONTROL> __device__ __forceinline__ uint32_t i4_dpp_max(uint32_t x) { return i4_max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CONTROL, 0xf, 0xf, true)); }

// The eight entries of a word.  7 |v| / top, ties to even, exactly: for 16-bit types the quotient is a half exactly or at least 2^-15 from one (14 v - (2 n +
// 1) top is a whole number of eighths of top's last place, of 2^12 of them at most), so the product with a reciprocal, less than 2^-19 off, is rounded to
// multiples of 2^-17 by adding 64: halves become exact, nothing else becomes one.  Adding 2^23 rounds it to a whole number in the last bits.  For f32 the same
// in 64 bits: 2^-28, 2^-30 by adding 2^22, and 2^52.
template <int TYPE> __device__ __forceinline__ uint32_t i4_word(const row8<TYPE> &q, const float (&v)[8], float top) {
    uint32_t w = 0, sign;
    if constexpr (TYPE == SLZ_F32) {
        const double inv = 7.0 / (double)top;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const double s = __builtin_fma((double)fabsf(v[e]), inv, 0x1p22) + 0x1p52;
            w += ((uint32_t)__builtin_bit_cast(uint64_t, s) & 7u) << (8 * (e & 3) + 4 * (e >> 2));
        }
        sign = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) sign |= (__builtin_bit_cast(uint32_t, v[e]) >> 31) << (8 * (e & 3) + 4 * (e >> 2) + 3);
    } else {
        // moved to where 1 / top is an ordinary number
        const float up = TYPE == SLZ_F16 ? 1.0f : top < 0x1p-100f ? 0x1p100f : top > 0x1p100f ? 0x1p-100f : 1.0f, inv = 7.0f * __builtin_amdgcn_rcpf(top * up);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float s = __builtin_fmaf(fabsf(TYPE == SLZ_BF16 ? v[e] * up : v[e]), inv, 64.0f) + 0x1p23f;
            w += __builtin_bit_cast(uint32_t, s) << (8 * (e & 3) + 4 * (e >> 2));
        }
        // what the numbers of 64 + 2^23 are in 32 bits
        constexpr uint32_t base = __builtin_bit_cast(uint32_t, 0x1p23f + 64.0f);
        constexpr uint32_t all = (base << 0) + (base << 8) + (base << 16) + (base << 24) + (base << 4) + (base << 12) + (base << 20) + (base << 28);
        w -= all;
        const uint32_t a = __builtin_amdgcn_perm((uint32_t)q.w[0][1], (uint32_t)q.w[0][0], 0x07050301u), b = __builtin_amdgcn_perm((uint32_t)q.w[0][3], (uint32_t)q.w[0][2], 0x07050301u);
        sign = (a >> 4 & 0x08080808u) | (b & 0x80808080u);
    }
    return w | (sign & ((w + 0x77777777u) & 0x88888888u));                         // zeros have none
}
// A lane makes a word, a group is 4, 8 or 16 lanes.  Bound by memory: 8192 x 8192 bf16 32.6 us (5.2 TB/s), f32 60 (5.1).
template <int TYPE>
__global__ void __launch_bounds__(256)
k_quantize_i4(const void *__restrict__ w, uint32_t rows, uint32_t cols, int64_t ld_w, uint32_t group, char *__restrict__ q, int64_t ld_q, float *__restrict__ scale,
              int64_t ld_scale, uint32_t wide) {
    const i4_walk at(wide);
    const uint32_t c = at.i * 8u;
    if (at.i >= (cols + I4_BLOCK - 1) / I4_BLOCK * 16u) return;                    // a block's 16 lanes together
    for (uint32_t r0 = at.row; r0 < rows; r0 += at.step) {
        row8<TYPE> x[I4_DOWN];
#pragma unroll
        for (uint32_t d = 0; d < I4_DOWN; d++) x[d] = row8_load<TYPE>(w, (size_t)min(r0 + d * at.next, rows - 1) * ld_w, c, cols);
#pragma unroll
        for (uint32_t d = 0; d < I4_DOWN; d++) {
            const size_t r = r0 + d * at.next;
            if (r >= rows) break;
            float v[8];
            row8_values<TYPE>(x[d], c, cols, v);
            if (TYPE != SLZ_F32 && c + 8u > cols)      // as they were moved down
#pragma unroll
                for (int i = 0; i < 4; i++) x[d].w[0][i] = (int)(slz_half(v[2 * i], TYPE) | (uint32_t)slz_half(v[2 * i + 1], TYPE) << 16);
            // magnitudes as whole numbers, so that infinities and NaN are the largest
            uint32_t m = 0;
            if constexpr (TYPE == SLZ_F32) {
#pragma unroll
                for (int e = 0; e < 8; e++) m = i4_max(m, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
            } else {
                typedef unsigned short us2 __attribute__((ext_vector_type(2)));
                us2 p = {0, 0};
#pragma unroll
                for (int i = 0; i < 4; i++) p = __builtin_elementwise_max(p, __builtin_bit_cast(us2, (uint32_t)x[d].w[0][i] & 0x7fff7fffu));
                m = i4_max(p[0], p[1]);
            }
            m = i4_dpp_max<0x4e>(i4_dpp_max<0xb1>(m));
            if (group > 32) m = i4_dpp_max<0x141>(m);
            if (group > 64) m = i4_dpp_max<0x140>(m);
            const bool finite = m < (TYPE == SLZ_F32 ? 0x7f800000u : TYPE == SLZ_BF16 ? 0x7f80u : 0x7c00u);
            const float top = TYPE == SLZ_F32 ? __builtin_bit_cast(float, m) : TYPE == SLZ_BF16 ? slz_bf16_to_f32((uint16_t)m) : slz_f16_to_f32((uint16_t)m);
            const uint32_t word = finite && m ? i4_word<TYPE>(x[d], v, top) : 0u;
            *(uint32_t *)(q + r * ld_q + i4_place(at.i) * 4u) = word;
            // top / 7 correctly rounded: it is never within 2^-30 of halfway between two numbers
            if ((c & (group - 1u)) == 0 && c < cols) scale[r * ld_scale + c / group] = finite ? (float)((double)top * (1.0 / 7.0)) : __builtin_nanf("");
        }
    }
}

static int i4_group_check(uint32_t group) { return group == 32 || group == 64 || group == 128 ? SLZ_OK : SLZ_E_INVALID_ARG; }
// 4-bit rows and their scales
static int i4_check(const void *q, int64_t ld_q, const float *scale, int64_t ld_scale, uint32_t rows, uint32_t cols, uint32_t group) {
    int rc = i4_group_check(group);
    if (rc != SLZ_OK) return rc;
    if (rows > SLZ_CLEAR_MAX_LEN || cols > SLZ_CLEAR_MAX_LEN) return SLZ_E_TOO_LARGE;
    rc = slz_matrix_check(q, rows, i4_blocks(cols) * 64u, ld_q, 16);
    if (rc == SLZ_OK && rows > 1 && cols && (ld_q & 15)) rc = SLZ_E_INVALID_ARG;
    if (rc == SLZ_OK) rc = slz_matrix_check(scale, rows, i4_groups(cols, group), ld_scale, 4);
    return rc;
}

extern "C" int slz_quantize_i4(const void *w, int type, uint32_t rows, uint32_t cols, int64_t ld_w, uint32_t group, uint8_t *q, int64_t ld_q, float *scale,
                               int64_t ld_scale, void *stream) {
    if (!slz_type_ok(type)) return SLZ_E_INVALID_ARG;
    int rc = i4_check(q, ld_q, scale, ld_scale, rows, cols, group);
    if (rc == SLZ_OK) rc = slz_matrix_check(w, rows, cols, ld_w, slz_type_bytes(type));
    if (rc != SLZ_OK || rows == 0 || cols == 0) return rc;
    const auto k = type == SLZ_F32 ? k_quantize_i4<SLZ_F32> : type == SLZ_BF16 ? k_quantize_i4<SLZ_BF16> : k_quantize_i4<SLZ_F16>;
    const uint32_t words = i4_blocks(cols) * 16u;
    hipLaunchKernelGGL(k, walk_grid(rows, words), dim3(256), 0, (hipStream_t)stream, w, rows, cols, ld_w, group, (char *)q, ld_q, scale, ld_scale, walk_wide(words));
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- values ------------------------------------------------------------------------------------------------------------------------
// Bound by memory: 8192 x 8192 bf16 29 us (5.8 TB/s), f32 83 (3.6, most of it written).  A lane has 16 bytes of the result: a word's eight entries, or four.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_values_i4(const char *__restrict__ q, int64_t ld_q, const float *__restrict__ scale, int64_t ld_scale, uint32_t group, uint32_t rows, uint32_t cols, char *__restrict__ out,
            int64_t ld_out, uint32_t aligned, uint32_t wide) {
    constexpr uint32_t E = TYPE == SLZ_F32 ? 4 : 8;
    const i4_walk at(wide);
    const uint32_t c = at.i * E;
    if (c >= cols) return;
    for (uint32_t r0 = at.row; r0 < rows; r0 += at.step) {
        uint32_t word[I4_DOWN];
        float sc[I4_DOWN];
#pragma unroll
        for (uint32_t d = 0; d < I4_DOWN; d++) {
            const size_t r = min(r0 + d * at.next, rows - 1);
            word[d] = *(const uint32_t *)(q + r * ld_q + i4_place(c / 8u) * 4u);
            sc[d] = scale[r * ld_scale + c / group];
        }
#pragma unroll
        for (uint32_t d = 0; d < I4_DOWN; d++) {
            const size_t r = r0 + d * at.next;
            if (r >= rows) break;
            float v[E];
            if constexpr (E == 8) {
                i4_numbers(word[d], 0, sc[d], v);
                i4_numbers(word[d], 1, sc[d], v + 4);
            } else i4_numbers(word[d], c >> 2 & 1, sc[d], v);
            slz_put_run<E>(out + (r * ld_out + c) * slz_type_bytes(TYPE), TYPE, v, cols - c, aligned);
        }
    }
}

extern "C" int slz_values_i4(const uint8_t *q, int64_t ld_q, const float *scale, int64_t ld_scale, uint32_t group, uint32_t rows, uint32_t cols, void *out, int type,
                             int64_t ld_out, void *stream) {
    if (!slz_type_ok(type)) return SLZ_E_INVALID_ARG;
    int rc = i4_check(q, ld_q, scale, ld_scale, rows, cols, group);
    if (rc == SLZ_OK) rc = slz_matrix_check(out, rows, cols, ld_out, slz_type_bytes(type));
    if (rc != SLZ_OK || rows == 0 || cols == 0) return rc;
    const uint32_t words = type == SLZ_F32 ? (cols + 3u) / 4u : (cols + 7u) / 8u;
    const auto k = type == SLZ_F32 ? k_values_i4<SLZ_F32> : type == SLZ_BF16 ? k_values_i4<SLZ_BF16> : k_values_i4<SLZ_F16>;
    hipLaunchKernelGGL(k, walk_grid(rows, words), dim3(256), 0, (hipStream_t)stream, (const char *)q, ld_q, scale, ld_scale, group, rows, cols, (char *)out, ld_out,
                       slz_in_place(out, 16, ld_out, slz_type_bytes(type)) ? 1u : 0u, walk_wide(words));
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- few rows ------------------------------------------------------------------------------------------------------------------------
// The entries of a word as eight numbers of a matrix operand, exact.  As a byte, sign and magnitude in the lowest bits of its fields, an entry is a subnormal
// e4m3 number, 2^-9 times the entry; the conversion to two bf16 or f16 takes a factor `by`, 512 or what i4_by says.  10 instructions a word (tables of the
// numbers' bytes by permutation: 15).
template <int EL> __device__ __forceinline__ v4i32 i4_operand(uint32_t word, float by) {
    v4i32 o;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint32_t b = h ? (word >> 4 & 0x07070707u) | (word & 0x80808080u) : (word & 0x07070707u) | (word << 4 & 0x80808080u);
        if constexpr (EL == SLZ_EL_BF16) {
            o[2 * h] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, by, false));
            o[2 * h + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, by, true));
        } else {
            o[2 * h] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, by, false));
            o[2 * h + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, by, true));
        }
    }
    return o;
}

// What follows streams the weights past the matrix instructions with the entries as whole numbers; what a group sums up to in 32 bits is multiplied by its
// scale, so that no value is rounded.  x lies in shared memory as operands.
struct i4_args {
    const char *x, *q;
    const float *scale;
    char *y;
    int64_t ld_x, ld_q, ld_scale, ld_y;                // of q in bytes
    uint32_t M, N, K, group;
};
template <int TYPE> constexpr int i4_pieces = TYPE == SLZ_F32 ? 3 : 1;
// A group's sum is up to 7 * 128 times the largest element of x, which for bf16 and f32 may be more than 32 bits hold.  So their entries are multiplied times
// 2^-10 (exactly: elements of x are multiples of 2^-133, and 2^-143 is one of 32 bits' numbers), and bf16's results times 2^10 at the end, where sums to
// multiples of 2^-139 are enough.  f32's are not to lose that, so there each scale is taken times 2^10, and one of 2^100 or more as it is with whole entries:
// where x is large enough for its group's sum to overflow, its products do too.
template <int EL, int PIECES> __device__ __forceinline__ float i4_by(float scale) { return EL == SLZ_EL_F16 || (PIECES > 1 && !(fabsf(scale) < 0x1p100f)) ? 512.0f : 0.5f; }
template <int PIECES> __device__ __forceinline__ float i4_scale(float scale) { return PIECES > 1 && fabsf(scale) < 0x1p100f ? scale * 0x1p10f : scale; }
template <int TYPE> constexpr float i4_sums_by = TYPE == SLZ_BF16 ? 0x1p10f : 1.0f;
// Eight entries of a row of x at c as operands, zeros past its end: one, or three that 32-bit numbers are cut into, the large ones first
template <int TYPE> __device__ __forceinline__ void i4_octet(const row8<TYPE> &q, uint32_t c, uint32_t cols, v4i32 (&o)[i4_pieces<TYPE>]) {
    if constexpr (TYPE != SLZ_F32)
        if (c + 8u <= cols) {
            o[0] = q.w[0];
            return;
        }
    float v[8];
    row8_values<TYPE>(q, c, cols, v);
    if constexpr (TYPE == SLZ_F32) {
        // the leading 8 bits, the next 8 and the last, of what is left exactly; an infinity is all in the first.  6 instructions an entry
        uint32_t u[3][8];
        float top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float r = v[i] - __int_as_float(__float_as_int(v[i]) & (int)0xffff0000u), l = r - __int_as_float(__float_as_int(r) & (int)0xffff0000u);
            u[0][i] = __float_as_int(v[i]);
            u[1][i] = __float_as_int(r);
            u[2][i] = __float_as_int(l);
            top = fmaxf(top, fabsf(v[i]));
        }
        if (top == INFINITY)
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (fabsf(v[i]) == INFINITY) u[1][i] = u[2][i] = 0;
#pragma unroll
        for (int k = 0; k < 3; k++)
#pragma unroll
            for (int i = 0; i < 4; i++) o[k][i] = (int)__builtin_amdgcn_perm(u[k][2 * i + 1], u[k][2 * i], 0x07060302u);
    } else
#pragma unroll
        for (int i = 0; i < 4; i++) o[0][i] = (int)(slz_half(v[2 * i], TYPE) | (uint32_t)slz_half(v[2 * i + 1], TYPE) << 16);
}
// A wave's share of the weights: 16 NB rows, a block's entries at a time.  Rows of a workgroup begin at uniform addresses, lanes' places are below 2^32 from there.
template <int NB> struct i4_stream {
    const char *q0;
    uint32_t at_q[NB];
    __device__ __forceinline__ void init(const i4_args &p, uint32_t first, uint32_t lane) {
        const uint32_t n0 = min(first, p.N - 1);       // a wave without rows reads the last one
        q0 = p.q + (int64_t)n0 * p.ld_q;
#pragma unroll
        for (int j = 0; j < NB; j++) {
            const uint32_t row = min(j * 16 + (lane & 15u), p.N - 1 - n0);
            at_q[j] = row * (uint32_t)p.ld_q + (lane >> 4) * 16u;
        }
    }
    __device__ __forceinline__ void load(uint32_t block, v4i32 (&w)[NB]) const {
#pragma unroll
        for (int j = 0; j < NB; j++) w[j] = *(const v4i32 *)(q0 + (at_q[j] + block * 64u));
    }
};
// Sums of a block's four steps: part collects a group (of 2^SHIFT entries), acc the groups times their scales.  read(step, i, o): x's operands.  A step's operands are read and
// its entries converted while the matrix instructions of the step before run; of more than four tiles of x's rows, four at a time, for which the entries are converted once.
template <int EL, int PIECES, int SHIFT, int MI, int NB, class READ>
__device__ __forceinline__ void i4_block(const v4i32 (&w)[NB], const v4f (&s)[NB], v4f (&acc)[MI][NB], const READ &read) {
    constexpr int OF = 1 << (SHIFT - 5), PART = MI < 4 ? MI : 4;                   // steps of a group, tiles at a time
    constexpr bool KEPT = MI > PART;
    static_assert(MI % PART == 0, "");
    v4i32 b[KEPT ? 4 : 2][NB];
#pragma unroll
    for (int first = 0; first < MI; first += PART) {
        v4f part[PART][NB];
        v4i32 o[2][PART][PIECES];
        const auto prepare = [&](int step) {
#pragma unroll
            for (int i = 0; i < PART; i++) read(step, first + i, o[step & 1][i]);
            __builtin_amdgcn_sched_barrier(0);
            if (first == 0)
#pragma unroll
                for (int j = 0; j < NB; j++) b[KEPT ? step : step & 1][j] = i4_operand<EL>((uint32_t)w[j][step], i4_by<EL, PIECES>(s[j][step / OF]));
        };
        prepare(0);
#pragma unroll
        for (int step = 0; step < 4; step++) {
            if (step < 3) prepare(step + 1);
#pragma unroll
            for (int i = 0; i < PART; i++)
#pragma unroll
                for (int k = PIECES - 1; k >= 0; k--)
#pragma unroll
                    for (int j = 0; j < NB; j++)
                        part[i][j] = slz_mma<EL>(o[step & 1][i][k], b[KEPT ? step : step & 1][j], step % OF == 0 && k == PIECES - 1 ? v4f{0, 0, 0, 0} : part[i][j]);
            if (step % OF == OF - 1)
#pragma unroll
                for (int i = 0; i < PART; i++)
#pragma unroll
                    for (int j = 0; j < NB; j++)
#pragma unroll
                        for (int e = 0; e < 4; e++) acc[first + i][j][e] = __builtin_fmaf(part[i][j][e], i4_scale<PIECES>(s[j][step / OF]), acc[first + i][j][e]);
        }
    }
}

// A few rows, all of x and of the scales that a workgroup needs in shared memory.  A workgroup of eight waves has 16 NB rows of weights, each wave an eighth
// of the blocks of k.
// Loads return in order, so those of x and the scales go first, then the wave's first blocks, before anything is looked at; the eight waves' sums meet in
// shared memory.
// One row by 8192 x 4096 bf16: 6.5 us (launch included; 17.9 MB), by 16384 x 4096 8.9; the waves wait for their loads 64 % of the time.  With x read where it
// is used by each wave 9.9 and 15.5, with the scales also 12.4 and 16.1.
#define THIN_SLOTS 2                 // octets of x, and scales, that a thread has under way
template <int TYPE, int NB, int SHIFT>
__global__ void __launch_bounds__(THIN_WAVES * 64) k_thin_i4(const i4_args p) {
    constexpr int EL = TYPE == SLZ_F16 ? SLZ_EL_F16 : SLZ_EL_BF16, PIECES = i4_pieces<TYPE>, AHEAD = 4;
    constexpr uint32_t THREADS = THIN_WAVES * 64, ROWS = 16 * NB;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    const uint32_t n0 = blockIdx.x * ROWS, blocks = (p.K + I4_BLOCK - 1) / I4_BLOCK, pitch = i4_pitch(p.K);
    const uint32_t begin = wave * blocks / THIN_WAVES, end = (wave + 1) * blocks / THIN_WAVES;
    i4_stream<NB> q;
    q.init(p, n0, lane);
    const uint32_t groups = (p.K + (1u << SHIFT) - 1) >> SHIFT, octets = p.M * blocks * 16u, count = ROWS * groups, pitch_s = i4_pitch_scales(groups);
    const float *scale0 = p.scale + (int64_t)n0 * p.ld_scale;
    float *scales = (float *)(lds + PIECES * p.M * pitch);
    row8<TYPE> x[THIN_SLOTS];
    float sc[THIN_SLOTS];
    const auto octet = [&](uint32_t i, uint32_t &m) {
        m = p.M == 1 ? 0u : i / max(blocks * 16u, 1u);
        return (i - m * (blocks * 16u)) * 8u;
    };
    const auto load_scale = [&](uint32_t i) {
        const uint32_t row = i / groups;
        return scale0[(size_t)min(row, p.N - 1 - n0) * p.ld_scale + i - row * groups];
    };
#pragma unroll
    for (uint32_t t = 0; t < THIN_SLOTS; t++) {
        const uint32_t i = threadIdx.x + t * THREADS;
        uint32_t m;
        const uint32_t c = octet(i, m);
        if (i < octets) x[t] = row8_load<TYPE>(p.x, (size_t)m * p.ld_x, c, p.K);
        if (i < count) sc[t] = load_scale(i);
    }
    v4i32 w[AHEAD][NB];
    if (begin < end)
#pragma unroll
        for (int d = 0; d < AHEAD; d++) q.load(min(begin + d, end - 1), w[d]);
    __builtin_amdgcn_sched_barrier(0);
    const auto put_x = [&](uint32_t i, const row8<TYPE> &v) {
        uint32_t m;
        const uint32_t c = octet(i, m);
        v4i32 o[PIECES];
        i4_octet<TYPE>(v, c, p.K, o);
#pragma unroll
        for (int k = 0; k < PIECES; k++) *(v4i32 *)(lds + (k * p.M + m) * pitch + c * 2u) = o[k];
    };
#pragma unroll
    for (uint32_t t = 0; t < THIN_SLOTS; t++) {
        const uint32_t i = threadIdx.x + t * THREADS;
        if (i < octets) put_x(i, x[t]);
        if (i < count) scales[i / groups * pitch_s + i % groups] = sc[t];
    }
    for (uint32_t i = threadIdx.x + THIN_SLOTS * THREADS; i < octets; i += THREADS) {
        uint32_t m;
        const uint32_t c = octet(i, m);
        put_x(i, row8_load<TYPE>(p.x, (size_t)m * p.ld_x, c, p.K));
    }
    for (uint32_t i = threadIdx.x + THIN_SLOTS * THREADS; i < count; i += THREADS) scales[i / groups * pitch_s + i % groups] = load_scale(i);
    if (threadIdx.x < ROWS)                            // groups past the rows' ends
        for (uint32_t c = groups; c < pitch_s; c++) scales[threadIdx.x * pitch_s + c] = 0.0f;
    __syncthreads();
    const char *from = lds + min(r, p.M - 1) * pitch + g * 16u;
    const uint32_t piece = p.M * pitch;
    v4f acc[1][NB];
#pragma unroll
    for (int j = 0; j < NB; j++) acc[0][j] = v4f{0, 0, 0, 0};
    for (uint32_t b0 = begin; b0 < end; b0 += AHEAD)
#pragma unroll
        for (int d = 0; d < AHEAD; d++) {
            const uint32_t block = b0 + d;
            if (block >= end) break;
            v4f s[NB];
#pragma unroll
            for (int j = 0; j < NB; j++) {
                const float *at = scales + (j * 16 + r) * pitch_s + (block << (7 - SHIFT));
                s[j] = SHIFT == 7 ? v4f{at[0], 0, 0, 0} : SHIFT == 6 ? v4f{at[0], at[1], 0, 0} : v4f{at[0], at[1], at[2], at[3]};
            }
            i4_block<EL, PIECES, SHIFT>(w[d], s, acc, [&](int step, int, v4i32 (&o)[PIECES]) {
#pragma unroll
                for (int k = 0; k < PIECES; k++) o[k] = *(const v4i32 *)(from + k * piece + block * 256u + step * 64u);
            });
            if (block + AHEAD < end) q.load(block + AHEAD, w[d]);
        }
    __syncthreads();
    float *sums = (float *)lds;                        // [wave][row of x][row of weights]
#pragma unroll
    for (int j = 0; j < NB; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) sums[(wave * 16u + g * 4u + e) * ROWS + j * 16 + r] = acc[0][j][e];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < p.M * ROWS; i += THREADS) {
        const uint32_t m = i / ROWS, n = n0 + i % ROWS;
        if (n >= p.N) continue;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < THIN_WAVES; k++) sum += sums[k * (16 * ROWS) + i];
        slz_put(p.y, TYPE, (size_t)m * p.ld_y + n, sum * i4_sums_by<TYPE>);
    }
}

// More rows: a workgroup has 16 MI rows of x and 32 WN of weights.  Its waves are WN by WK: in each phase WK blocks of k of x and the scales that go with them
// come to shared memory, on the way through registers while the phase before is computed, and a wave multiplies one of the blocks by its 32 rows of weights,
// whose words come AHEAD phases before.  The WK waves' sums meet in shared memory at the end.  Every phase does all loads (past the end those of the last
// phase again), so that the compiler can count what is under way.
// 64 rows by 16384 x 4096 bf16: 17.5 us, 512 by 8192 x 4096 42 (820 TFLOP/s), 512 by 8192 x 8192 75 (917).  Bound by what a compute unit loads, 44 GB/s:
// without x's loads and stores (in a copy) 13.4 and 33 us, without the products 17.0 and 33, without either 10.8 and 18; x two phases ahead instead of one was
// no faster.
template <int TYPE, int MI, int WN, int WK, int BUFFERS, int SHIFT>
__global__ void __launch_bounds__(WN *WK * 64) k_rows_i4(const i4_args p, uint32_t tiles_m, uint32_t tiles_n) {
    constexpr int EL = TYPE == SLZ_F16 ? SLZ_EL_F16 : SLZ_EL_BF16, PIECES = i4_pieces<TYPE>, XB = TYPE == SLZ_F32 ? 4 : 2, NB = 2, AHEAD = 2, THREADS = WN * WK * 64;
    constexpr uint32_t TM = MI * 16, TN = WN * NB * 16, HALF = TM * 128, PIECE = 2 * HALF, BLOCK = PIECES * PIECE, BUFFER = WK * BLOCK;
    constexpr int OCTETS = WK * TM * 16 / THREADS;
    static_assert(OCTETS * THREADS == WK * TM * 16, "");
    constexpr uint32_t SUMS = WK * TM * TN * 4, LDS = BUFFERS * BUFFER > SUMS ? BUFFERS * BUFFER : SUMS;
    constexpr uint32_t GROUPS = WK << (7 - SHIFT);     // of a phase
    constexpr int SCALES = (TN * GROUPS + THREADS - 1) / THREADS;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    __shared__ float scales[2][GROUPS][TN + 4];        // [group][row of weights]
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    const uint32_t wn = wave % WN, wk = wave / WN;
    // the tiles of x that meet one tile of weights follow each other on one XCD
    const uint32_t eights = blockIdx.x / (8u * tiles_m), in = blockIdx.x % (8u * tiles_m), left = min(8u, tiles_n - eights * 8u);
    const uint32_t n0 = (eights * 8u + in % left) * TN, m0 = in / left * TM;
    const uint32_t blocks = (p.K + I4_BLOCK - 1) / I4_BLOCK, phases = (blocks + WK - 1) / WK, groups = (p.K + (1u << SHIFT) - 1) >> SHIFT;
    const auto phase_of = [&](uint32_t number) { return min(number, phases - 1); };
    i4_stream<NB> q;
    q.init(p, n0 + wn * (NB * 16), lane);
    v4i32 w[AHEAD][NB];
    // this thread's octets of x: row (the last one again where there are fewer, for sums that no one stores) and column in the phase
    const char *x0 = p.x + (int64_t)m0 * p.ld_x * XB;
    row8<TYPE> x[OCTETS];
    constexpr int PER_BLOCK = TM * 16 > THREADS ? TM * 16 / THREADS : 1, BLOCKS = TM * 16 > THREADS ? 1 : THREADS / (TM * 16);       // of a block in a row, blocks at once
    const uint32_t row0 = threadIdx.x / 16u % TM, col0 = threadIdx.x / (TM * 16) * I4_BLOCK + threadIdx.x % 16u * 8u;
    const uint32_t to0 = threadIdx.x / (TM * 16) * BLOCK + threadIdx.x % 16u / 8u * HALF + row0 * 128u + slz_piece_k<0>(row0, threadIdx.x % 8u) * 16u;
    uint32_t at_x[PER_BLOCK];
#pragma unroll
    for (int i = 0; i < PER_BLOCK; i++) at_x[i] = min(row0 + i * (THREADS / 16), p.M - 1 - m0) * (uint32_t)p.ld_x * XB;
    const auto load_x = [&](uint32_t phase) {
#pragma unroll
        for (int i = 0; i < OCTETS; i++) {
            // where the row ends inside, its last eight; i4_octet moves them down
            const uint32_t c = min(col0 + i / PER_BLOCK * BLOCKS * I4_BLOCK + phase * (WK * I4_BLOCK), p.K - 8u) * XB;
            const v4i32_any *at = (const v4i32_any *)(x0 + (size_t)(at_x[i % PER_BLOCK] + c));
            x[i].w[0] = at[0];
            if constexpr (TYPE == SLZ_F32) x[i].w[1] = at[1];
        }
    };
    const auto store_x = [&](uint32_t phase, char *to) {
        const auto all = [&](auto inside) {
#pragma unroll
            for (int i = 0; i < OCTETS; i++) {
                v4i32 o[PIECES];
                if constexpr (decltype(inside)::value) i4_octet<TYPE>(x[i], 0, 8, o);
                else i4_octet<TYPE>(x[i], col0 + i / PER_BLOCK * BLOCKS * I4_BLOCK + phase * (WK * I4_BLOCK), p.K, o);
#pragma unroll
                for (int k = 0; k < PIECES; k++) *(v4i32 *)(to + to0 + (i / PER_BLOCK * BLOCKS * BLOCK + i % PER_BLOCK * (THREADS / 16 * 128) + k * PIECE)) = o[k];
            }
        };
        if ((phase + 1) * (WK * I4_BLOCK) <= p.K) all(std::true_type());
        else all(std::false_type());
    };
    // this thread's scales: rows of weights and groups of the phase, 0 past the rows' ends
    const float *scale0 = p.scale + (int64_t)n0 * p.ld_scale;
    float sc[SCALES];
    const auto load_scales = [&](uint32_t phase) {
#pragma unroll
        for (int t = 0; t < SCALES; t++) {
            const uint32_t i = threadIdx.x + t * THREADS;
            sc[t] = scale0[min(i / GROUPS, p.N - 1 - n0) * (uint32_t)p.ld_scale + min(phase * GROUPS + i % GROUPS, groups - 1)];
        }
    };
    const auto store_scales = [&](uint32_t phase, int buffer) {
#pragma unroll
        for (int t = 0; t < SCALES; t++) {
            const uint32_t i = threadIdx.x + t * THREADS;
            if (TN * GROUPS % THREADS == 0 || i < TN * GROUPS) scales[buffer][i % GROUPS][i / GROUPS] = phase * GROUPS + i % GROUPS < groups ? sc[t] : 0.0f;
        }
    };
    const auto load_w = [&](uint32_t phase, v4i32 (&to)[NB]) { q.load(min(phase * WK + wk, blocks - 1), to); };

    // in the order of the loop's
    load_x(phase_of(0));
    load_scales(phase_of(0));
    load_w(phase_of(0), w[0]);
    store_x(phase_of(0), lds);
    store_scales(phase_of(0), 0);
    load_x(phase_of(1));
    load_scales(phase_of(1));
    load_w(phase_of(1), w[1]);
    v4f acc[MI][NB];
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) acc[i][j] = v4f{0, 0, 0, 0};
    __syncthreads();
    for (uint32_t p0 = 0; p0 < phases; p0 += AHEAD)
#pragma unroll
        for (int d = 0; d < AHEAD; d++) {
            const uint32_t number = p0 + d;
            if (number >= phases) break;
            if (BUFFERS == 2) {
                store_x(phase_of(number + 1), lds + (1 - d) * BUFFER);
                store_scales(phase_of(number + 1), 1 - d);
                load_x(phase_of(number + 2));
                load_scales(phase_of(number + 2));
                __builtin_amdgcn_sched_barrier(0);
            }
            const char *from = lds + (BUFFERS == 2 ? d : 0) * BUFFER + wk * BLOCK + r * 128u;
            v4f s[NB];
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int e = 0; e < 1 << (7 - SHIFT); e++) s[j][e] = scales[BUFFERS == 2 ? d : 0][(wk << (7 - SHIFT)) + e][(wn * NB + j) * 16 + r];
            // a block past the end is the last one again, times zeros
            i4_block<EL, PIECES, SHIFT>(w[d], s, acc, [&](int step, int i, v4i32 (&o)[PIECES]) {
#pragma unroll
                for (int k = 0; k < PIECES; k++) o[k] = *(const v4i32 *)(from + k * PIECE + step / 2 * HALF + i * 2048 + slz_piece_k<0>(r, step % 2 * 4u + g) * 16u);
            });
            load_w(phase_of(number + AHEAD), w[d]);
            __syncthreads();
            if (BUFFERS == 1) {
                store_x(phase_of(number + 1), lds);
                store_scales(phase_of(number + 1), 0);
                load_x(phase_of(number + 2));
                load_scales(phase_of(number + 2));
                __syncthreads();
            }
        }
    float *sums = (float *)lds;                        // [wk][row of x][row of weights]
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) sums[(wk * TM + i * 16 + g * 4 + e) * TN + (wn * NB + j) * 16 + r] = acc[i][j][e];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < TM * TN; i += THREADS) {
        const uint32_t m = m0 + i / TN, n = n0 + i % TN;
        if (m >= p.M || n >= p.N) continue;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < WK; k++) sum += sums[k * (TM * TN) + i];
        slz_put(p.y, TYPE, (size_t)m * p.ld_y + n, sum * i4_sums_by<TYPE>);
    }
}

// ---- values as an operand ------------------------------------------------------------------------------------------------------------
// f16 could not hold small scales, so its values are held times VALUES_UP / unit, the power of two above the largest finite scale: magnitudes of up to
// 7 2^12 are below f16's largest, and rows whose scale is down to 2^-26 of the largest keep 11 bits.
#define VALUES_UP 4096.0f
#define VALUES_TOPS 256u             // workgroups that look for the largest scale
// 2 MiB of scales: 6 us
__global__ void __launch_bounds__(256) k_scale_tops(const float *__restrict__ scale, int64_t ld_scale, uint32_t rows, uint32_t groups, float *__restrict__ tops) {
    const size_t total = (size_t)rows * groups;
    float top = 0.0f;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        size_t at = g;
        if (ld_scale != groups) {
            uint32_t c;
            at = slz_divide(g, groups, total <= 0xffffffffu, c) * ld_scale;
            at += c;
        }
        const float a = fabsf(scale[at]);
        if (a < __builtin_inff()) top = fmaxf(top, a);
    }
    top = slz_wave_max(top);
    __shared__ float of_wave[4];
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) tops[blockIdx.x] = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
}
// 4-bit rows and how their values are held: tops of `count` workgroups, from which the first one makes the unit; nothing of them for other types
struct i4_rows { const uint8_t *q; int64_t ld_q; const float *scale; int64_t ld_scale; uint32_t group, rows, cols; };
struct i4_unit { const float *tops; uint32_t count; float *unit; };
// what values are multiplied by
template <int TYPE> __device__ __forceinline__ float values_by(const i4_unit &u) {
    if constexpr (TYPE != SLZ_F16) return 1.0f;
    __shared__ float of_wave[4];
    float top = slz_wave_max(threadIdx.x < u.count ? u.tops[threadIdx.x] : 0.0f);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
    int e = 0;
    if (top > 0.0f) frexpf(top, &e);
    const float unit = ldexpf(1.0f, e < -100 ? -100 : e > 100 ? 100 : e);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *u.unit = unit;
    return VALUES_UP / unit;
}
// a value in the operand's pieces
template <int TYPE> __device__ __forceinline__ void values_pieces(float v, float by, uint16_t (&t)[i4_pieces<TYPE>]) {
    if constexpr (TYPE == SLZ_F32) slz_split3(v, t);
    else t[0] = slz_half(v * by, TYPE);
}
// Rows as they are, padded with zeros to ld_out bytes; bound by memory: 8192 x 8192 f16 32 us (5.3 TB/s)
template <int TYPE>
__global__ void __launch_bounds__(256) k_values_operand(const i4_rows w, const i4_unit u, char *__restrict__ out, uint32_t ld_out, int64_t piece, uint32_t wide) {
    constexpr int PIECES = i4_pieces<TYPE>;
    const float by = values_by<TYPE>(u);
    const i4_walk at(wide);
    const uint32_t c = at.i * 8u, last = (w.cols - 1) / 8u;
    if (at.i * 16u >= ld_out) return;
    for (uint32_t r0 = at.row; r0 < w.rows; r0 += at.step) {
        uint32_t word[I4_DOWN];
        float sc[I4_DOWN];
#pragma unroll
        for (uint32_t d = 0; d < I4_DOWN; d++) {
            const size_t r = min(r0 + d * at.next, w.rows - 1);
            word[d] = *(const uint32_t *)(w.q + r * w.ld_q + i4_place(min(at.i, last)) * 4u);
            sc[d] = w.scale[r * w.ld_scale + min(c, w.cols - 1) / w.group];
        }
#pragma unroll
        for (uint32_t d = 0; d < I4_DOWN; d++) {
            const size_t r = r0 + d * at.next;
            if (r >= w.rows) break;
            float v[8];
            i4_numbers(word[d], 0, sc[d], v);
            i4_numbers(word[d], 1, sc[d], v + 4);
            if (c + 8u > w.cols)
#pragma unroll
                for (uint32_t e = 0; e < 8; e++) v[e] = c + e < w.cols ? v[e] : 0.0f;
            uint16_t t[8][PIECES];
#pragma unroll
            for (int e = 0; e < 8; e++) values_pieces<TYPE>(v[e], by, t[e]);
#pragma unroll
            for (int k = 0; k < PIECES; k++) {
                uint32_t o[4];
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] = t[2 * e][k] | (uint32_t)t[2 * e + 1][k] << 16;
                *(uint4 *)(out + k * piece + r * ld_out + (size_t)at.i * 16u) = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
    }
}
// The transpose: out [cols][ld_out], rows of the entries' columns, so that a product that sums over the weights' rows has them in a row too (the tiled product
// takes 105 us instead of 125 for 4096^3 then).  A workgroup has 128 rows by a block; a thread two rows' entries of a column as one word in shared memory,
// whose rows are 66 words so that a wave's words meet different banks.
// 4096 x 4096 bf16 9.7 us (4.4 TB/s).
template <int TYPE>
__global__ void __launch_bounds__(256) k_values_transposed(const i4_rows w, const i4_unit u, char *__restrict__ out, uint32_t ld_out, int64_t piece) {
    constexpr int PIECES = i4_pieces<TYPE>;
    __shared__ __attribute__((aligned(8))) uint32_t tile[I4_BLOCK][66];
    const float by = values_by<TYPE>(u);
    const uint32_t pair = threadIdx.x / 4u, j = threadIdx.x % 4u, block = blockIdx.y, k0 = block * I4_BLOCK;
    for (uint32_t r0 = blockIdx.x * 128u; r0 < ld_out / 2u; r0 += gridDim.x * 128u) {
        v4i32 word[2];
        float sc[2][4];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const size_t r = min(r0 + pair * 2u + h, w.rows - 1);
            word[h] = *(const v4i32 *)(w.q + r * w.ld_q + block * 64u + j * 16u);
#pragma unroll
            for (uint32_t s = 0; s < 4; s++) {
                const float v = w.scale[r * w.ld_scale + min(k0 + s * 32u, w.cols - 1) / w.group];
                sc[h][s] = r0 + pair * 2u + h < w.rows ? v : 0.0f;
            }
            if (r0 + pair * 2u + h >= w.rows) word[h] = v4i32{0, 0, 0, 0};
        }
#pragma unroll
        for (int k = 0; k < PIECES; k++) {
            if (r0 != blockIdx.x * 128u || k) __syncthreads();
#pragma unroll
            for (int s = 0; s < 4; s++) {
                float v[2][8];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    i4_numbers((uint32_t)word[h][s], 0, sc[h][s], v[h]);
                    i4_numbers((uint32_t)word[h][s], 1, sc[h][s], v[h] + 4);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    uint16_t a[PIECES], b[PIECES];
                    values_pieces<TYPE>(v[0][e], by, a);
                    values_pieces<TYPE>(v[1][e], by, b);
                    tile[s * 32 + j * 8 + e][pair] = a[k] | (uint32_t)b[k] << 16;
                }
            }
            __syncthreads();
            // 16 bytes of a row of the result a thread
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t c = (threadIdx.x + i * 256u) / 16u, n = threadIdx.x % 16u;
                if (k0 + c >= w.cols || r0 + n * 8u >= ld_out / 2u) continue;
                const uint2 lo = *(const uint2 *)&tile[c][n * 4u], hi = *(const uint2 *)&tile[c][n * 4u + 2u];
                *(uint4 *)(out + k * piece + (size_t)(k0 + c) * ld_out + (r0 + n * 8u) * 2u) = make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
        }
    }
}
// bytes of the values of rows x cols as an operand whose rows are `row` long, and of the unit with what it is made from
static uint32_t values_row(uint32_t cols) { return (uint32_t)(((size_t)cols * 2 + 127) / 128 * 128); }
static size_t values_bytes(int type, uint32_t rows, uint32_t cols) { return (type == SLZ_F32 ? 3 : 1) * up256((size_t)rows * values_row(cols)) + 256 + VALUES_TOPS * 4; }
// the operand: rows x cols, or transposed cols x rows
static slz_operand values_operand(const i4_rows &w, bool transposed, int type, char *ws, float **unit, hipStream_t s) {
    const uint32_t row = values_row(transposed ? w.rows : w.cols), count = transposed ? w.cols : w.rows;
    const size_t piece = up256((size_t)count * row);
    const slz_operand o{ws, (int64_t)row, type == SLZ_F32 ? (int64_t)piece : 0, type == SLZ_F32 ? 3u : 1u, type == SLZ_F16 ? SLZ_F16 : SLZ_BF16};
    *unit = nullptr;
    if (w.rows == 0 || w.cols == 0) return o;
    float *at = (float *)(ws + o.pieces * piece);
    i4_unit u{at + 64, 0, at};
    if (type == SLZ_F16) {
        const size_t scales = (size_t)w.rows * i4_groups(w.cols, w.group);
        u.count = scales < (size_t)VALUES_TOPS * 256 ? (uint32_t)((scales + 255) / 256) : VALUES_TOPS;
        hipLaunchKernelGGL(k_scale_tops, dim3(u.count), dim3(256), 0, s, w.scale, w.ld_scale, w.rows, i4_groups(w.cols, w.group), at + 64);
        *unit = at;
    }
    if (transposed) {
        const auto k = type == SLZ_F32 ? k_values_transposed<SLZ_F32> : type == SLZ_BF16 ? k_values_transposed<SLZ_BF16> : k_values_transposed<SLZ_F16>;
        const uint32_t blocks = i4_blocks(w.cols), tiles = (row / 2u + 127u) / 128u, most = 65536u / blocks ? 65536u / blocks : 1u;
        hipLaunchKernelGGL(k, dim3(tiles < most ? tiles : most, blocks), dim3(256), 0, s, w, u, ws, row, (int64_t)piece);
    } else {
        const auto k = type == SLZ_F32 ? k_values_operand<SLZ_F32> : type == SLZ_BF16 ? k_values_operand<SLZ_BF16> : k_values_operand<SLZ_F16>;
        hipLaunchKernelGGL(k, walk_grid(w.rows, row / 16u), dim3(256), 0, s, w, u, ws, row, (int64_t)piece, walk_wide(row / 16u));
    }
    return o;
}

// ---- product -------------------------------------------------------------------------------------------------------------------------
static int shape_check(const slz_i4_shape *sh) {
    if (!sh || !slz_type_ok(sh->type)) return SLZ_E_INVALID_ARG;
    if (sh->m > SLZ_CLEAR_MAX_LEN || sh->n > SLZ_CLEAR_MAX_LEN || sh->k > SLZ_CLEAR_MAX_LEN) return SLZ_E_TOO_LARGE;
    return i4_group_check(sh->group);
}
static i4_rows weights_of(const slz_i4_shape *sh, const uint8_t *q, const float *scale) { return {q, sh->ld_q, scale, sh->ld_scale, sh->group, sh->n, sh->k}; }
static uint32_t pairs_of(int type) { return type == SLZ_F32 ? 6 : 1; }

template <int TYPE, int SHIFT, int NB> static void thin_launch(const i4_args &p, hipStream_t s) {
    const size_t x = i4_thin_bytes(p.M, p.K, p.group, TYPE == SLZ_F32, NB), sums = (size_t)THIN_WAVES * 16 * NB * 16 * 4;
    hipLaunchKernelGGL((k_thin_i4<TYPE, NB, SHIFT>), dim3((p.N + 16 * NB - 1) / (16 * NB)), dim3(THIN_WAVES * 64), x > sums ? x : sums, s, p);
}
template <int TYPE, int SHIFT, int MI, int WN, int WK, int BUFFERS> static void rows_launch(const i4_args &p, hipStream_t s) {
    const uint32_t tiles_m = (p.M + MI * 16 - 1) / (MI * 16), tiles_n = (p.N + WN * 32 - 1) / (WN * 32);
    hipLaunchKernelGGL((k_rows_i4<TYPE, MI, WN, WK, BUFFERS, SHIFT>), dim3(tiles_m * tiles_n), dim3(WN * WK * 64), 0, s, p, tiles_m, tiles_n);
}
template <int TYPE, int SHIFT> static void stream_of(const i4_args &p, const i4_route &R, hipStream_t s) {
    if (R.way == i4_route::THIN) {
        // 16 rows of weights a workgroup.  With 32 there are half of them, each longer: bf16, one row by 4096, 8192, 16384 x 4096: 5.2, 6.5, 8.9
        // us and 6.6, 7.4, 9.8.  f32 has three workgroups of 16 at once on a compute unit, and more than 768 of them begin a second time: two rows by 12288,
        // 16384 x 1024: 6.5, 8.2 us and 7.2, 7.2 with 32.
        if (TYPE == SLZ_F32 && p.N > 12288) thin_launch<TYPE, SHIFT, TYPE == SLZ_F32 ? 2 : 1>(p, s);
        else thin_launch<TYPE, SHIFT, 1>(p, s);
    } else if constexpr (TYPE == SLZ_F32) rows_launch<TYPE, SHIFT, 1, 2, 4, 1>(p, s);
    else if (R.kind == 0) rows_launch<TYPE, SHIFT, 1, 1, 8, 2>(p, s);
    else if (R.kind == 1) rows_launch<TYPE, SHIFT, 1, 2, 4, 2>(p, s);
    else if (R.kind == 2) rows_launch<TYPE, SHIFT, 2, 2, 4, 2>(p, s);
    else if (R.kind == 3) rows_launch<TYPE, SHIFT, 4, 2, 4, 2>(p, s);
    else rows_launch<TYPE, SHIFT, 8, 4, 2, 2>(p, s);
}
template <int TYPE> static void stream_typed(const i4_args &p, const i4_route &R, hipStream_t s) {
    p.group == 32 ? stream_of<TYPE, 5>(p, R, s) : p.group == 64 ? stream_of<TYPE, 6>(p, R, s) : stream_of<TYPE, 7>(p, R, s);
}
static int stream_product(const slz_i4_shape *sh, const i4_route &R, const void *x, const uint8_t *q, const float *scale, void *y, hipStream_t s) {
    const i4_args p{(const char *)x, (const char *)q, scale, (char *)y, sh->ld_x, sh->ld_q, sh->ld_scale, sh->ld_y, sh->m, sh->n, sh->k, sh->group};
    if (sh->type == SLZ_F32) stream_typed<SLZ_F32>(p, R, s);
    else if (sh->type == SLZ_BF16) stream_typed<SLZ_BF16>(p, R, s);
    else stream_typed<SLZ_F16>(p, R, s);
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}

struct linear_plan { size_t x, ranges, total; i4_route R; };
static linear_plan plan_linear(const slz_i4_shape *sh, const void *x) {
    linear_plan P;
    P.R = i4_route_of(sh->m, sh->n, sh->k, sh->type == SLZ_F32, sh->group);
    P.x = values_bytes(sh->type, sh->n, sh->k);
    P.ranges = P.x + slz_operand_bytes(x, sh->type, sh->m, sh->k, sh->ld_x);
    P.total = P.R.way == i4_route::TILES && sh->m && sh->n ? P.ranges + slz_ranges_bytes(P.R.c, sh->m, sh->n) : 0;
    return P;
}
// out [M][N] = left times values laid out by values_operand, both with the sum's index in a row
static int values_product(const slz_operand &left, const slz_operand &values, uint32_t M, uint32_t N, uint32_t K, const slz_choice &c, const float *unit, void *out, int type, int64_t ld,
                          char *ranges, hipStream_t s) {
    const slz_gemm p = slz_gemm_of(left, values, M, N, K);
    const slz_times_unit f{unit, 1.0f / VALUES_UP};
    return type == SLZ_F16 ? slz_gemm_to<SLZ_EL_F16, false, false>(p, c, f, out, type, ld, ranges, s) : slz_gemm_to<SLZ_EL_BF16, false, false>(p, c, f, out, type, ld, ranges, s);
}
extern "C" int slz_linear_i4_workspace(const slz_i4_shape *sh, const void *x, size_t *bytes) {
    const int rc = shape_check(sh);
    if (rc != SLZ_OK) return rc;
    if (!bytes) return SLZ_E_INVALID_ARG;
    *bytes = plan_linear(sh, x).total;
    return SLZ_OK;
}
extern "C" int slz_linear_i4(const slz_i4_shape *sh, const void *x, const uint8_t *q, const float *scale, void *y, void *ws, size_t ws_bytes, void *stream) {
    int rc = shape_check(sh);
    if (rc == SLZ_OK) rc = slz_matrix_check(x, sh->m, sh->k, sh->ld_x, slz_type_bytes(sh->type));
    if (rc == SLZ_OK) rc = i4_check(q, sh->ld_q, scale, sh->ld_scale, sh->n, sh->k, sh->group);
    if (rc == SLZ_OK) rc = slz_matrix_check(y, sh->m, sh->n, sh->ld_y, slz_type_bytes(sh->type));
    if (rc != SLZ_OK || sh->m == 0 || sh->n == 0) return rc;
    const linear_plan P = plan_linear(sh, x);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    if (P.R.way != i4_route::TILES) return stream_product(sh, P.R, x, q, scale, y, s);
    char *at = (char *)ws;
    slz_layouts jobs = {};
    const slz_operand a = slz_operand_of(x, sh->type, sh->m, sh->k, sh->ld_x, at + P.x, jobs);
    slz_layout_run(jobs, s);
    float *unit;
    const slz_operand b = values_operand(weights_of(sh, q, scale), false, sh->type, at, &unit, s);
    rc = values_product(a, b, sh->m, sh->n, sh->k, P.R.c, unit, y, sh->type, sh->ld_y, at + P.ranges, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- gradient ------------------------------------------------------------------------------------------------------------------------
struct i4_grad_plan { size_t dy, x, values, ranges, total; slz_choice dx, dw; };
static i4_grad_plan plan_i4_grad(const slz_i4_shape *sh, const void *dy, const void *x) {
    i4_grad_plan P;
    const uint32_t pairs = pairs_of(sh->type);
    // a step with both operands' rows k takes 2.3 to 2.8 times what the choice reckons, which leaves sides as they are and makes ranges worth more: 1555 x
    // 1001 by 777 deep f32 42 us for 63, 2000 x 500 by 1000 deep 37 for 48
    P.dw = slz_choose(sh->n, sh->k, (sh->m + 63) / 64 * pairs * 5 / 2, 1, false, 16, true);
    // and one of small tiles twice as long: 777 x 1001 by 1555 deep f16 28.6 us with what lays out for 31.4, 256 x 1024 by 1024 15.9 for 17.5
    P.dx = slz_choose(sh->m, sh->k, (sh->n + 63) / 64 * pairs * 2, 1, false, 16);
    P.dy = 0;
    P.x = slz_operand_bytes(dy, sh->type, sh->m, sh->n, sh->ld_y);
    P.values = P.x + slz_operand_bytes(x, sh->type, sh->m, sh->k, sh->ld_x);
    P.ranges = P.values + values_bytes(sh->type, sh->k, sh->n);
    const size_t for_x = slz_ranges_bytes(P.dx, sh->m, sh->k), for_w = slz_ranges_bytes(P.dw, sh->n, sh->k);
    P.total = P.ranges + (for_x > for_w ? for_x : for_w);
    return P;
}
extern "C" int slz_linear_i4_grad_workspace(const slz_i4_shape *sh, const void *dy, const void *x, size_t *bytes) {
    const int rc = shape_check(sh);
    if (rc != SLZ_OK) return rc;
    if (!bytes) return SLZ_E_INVALID_ARG;
    *bytes = plan_i4_grad(sh, dy, x).total;
    return SLZ_OK;
}
extern "C" int slz_linear_i4_grad(const slz_i4_shape *sh, const void *dy, const void *x, const uint8_t *q, const float *scale, void *dx, int64_t ld_dx, void *dw, int64_t ld_dw,
                                  void *ws, size_t ws_bytes, void *stream) {
    int rc = shape_check(sh);
    if (rc != SLZ_OK) return rc;
    const uint32_t eb = slz_type_bytes(sh->type);
    rc = slz_matrix_check(dy, sh->m, sh->n, sh->ld_y, eb);
    if (rc == SLZ_OK && dx) rc = i4_check(q, sh->ld_q, scale, sh->ld_scale, sh->n, sh->k, sh->group);
    if (rc == SLZ_OK && dx) rc = slz_matrix_check(dx, sh->m, sh->k, ld_dx, eb);
    if (rc == SLZ_OK && dw) rc = slz_matrix_check(x, sh->m, sh->k, sh->ld_x, eb);
    if (rc == SLZ_OK && dw) rc = slz_matrix_check(dw, sh->n, sh->k, ld_dw, eb);
    if (rc != SLZ_OK || sh->k == 0) return rc;
    const i4_grad_plan P = plan_i4_grad(sh, dy, x);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    char *at = (char *)ws;
    slz_layouts jobs = {};
    const slz_operand d = slz_operand_of(dy, sh->type, sh->m, sh->n, sh->ld_y, at + P.dy, jobs);
    slz_operand b{};
    if (dw) b = slz_operand_of(x, sh->type, sh->m, sh->k, sh->ld_x, at + P.x, jobs);
    slz_layout_run(jobs, s);
    if (dx && sh->m) {
        float *unit;
        const slz_operand w = values_operand(weights_of(sh, q, scale), true, sh->type, at + P.values, &unit, s);
        rc = values_product(d, w, sh->m, sh->k, sh->n, P.dx, unit, dx, sh->type, ld_dx, at + P.ranges, s);
    }
    if (rc == SLZ_OK && dw && sh->n) rc = slz_float_product(d, true, b, sh->n, sh->k, sh->m, P.dw, nullptr, 1.0f, dw, sh->type, ld_dw, at + P.ranges, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
