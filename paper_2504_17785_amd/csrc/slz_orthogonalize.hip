// Updates orthogonalised by Newton-Schulz products (include/silenzio_clear.h):  X <- a X + (b A + c A A) X,  A = X X^T.
//
// The products run on f16 matrix instructions.  A step moves singular values near 1 little while it multiplies small ones by a, so what
// rounding adds to X itself grows by a^steps against it, and b A + c A A comes near -2.7 I, against which a X nearly cancels.  Hence
//   * X is held in two f16 (22 bits); a X and the diagonal's part of the product use both, the product's operand is the first;
//   * the diagonals of A and of B = b A + c A A are held in 32 bits apart, their f16 operands have zeros there:
//     A A = O O + (d_i + d_j) O_ij + d_i^2 [i = j]  with A = O + diag d,  and  X' = (a + B_ii) X + (B - diag) X.
// With the operands 8 times as precise as bf16's, and that, a result of 128 to 512 rows differs from the formula's by 4e-4 to 1.1e-3 of its norm (a model of the
// roundings on the CPU; rounding to bf16 adds 1.7e-3, all operands in bf16 1e-2 to 9e-2); with 16 rows, most singular values a hundredth of the largest, by 4e-3.  For f16 and f32 results O, B and X enter the products with both their halves (three products instead of one).
// The first X is g times a power of two; what is missing to g / |g| is a factor of the first step.
// A and A A are symmetric: tiles on and below the diagonal are computed and stored twice.
// Measured, a step: 4096 x 8192 bf16 A 155 us, B 93, X' 336 (0.82 PFLOP/s; matrix cores 39 % busy, waves wait 51 %); 6 x 500 x 1000 f16 15.3, 13.2, 25.6, where no
// other tiling is more than 6 % faster: launches of 8 or 16 steps of k, mostly fill and epilogue.
#include "slz_gemm.h"

// A and B are held times ORTH_UP: what is lost of them below 2^-31 is nothing against a I, to which they are added.  X is held times ORTH_X_UP, since its
// small entries grow by a each step: relative to a norm of 1 they are 1 / sqrt(mn), and their second halves have to stay out of f16's subnormal numbers.
// f32, 4096 x 8192, error against 64 bits: 1.1e-6 (Gaussian), 1.4e-5 (four strong directions), with 64 in place of 1024 3.1e-6 and 1.4e-4, 4096 no better;
// the same steps in 32 bits 7.1e-6 and 3.5e-5.  Entries of X up to 63 and, off the diagonal, of A and B up to 1023 stay finite.
#define ORTH_UP 64.0f
#define ORTH_X_UP 1024.0f
#define ORTH_NORM_BLOCKS 1024

struct orth_view {                   // a batch of matrices of two f16 each; rows of a multiple of 64 elements
    uint16_t *hi, *lo;               // lo may be null
    uint32_t ld;
    size_t stride;                   // elements from matrix to matrix
};
typedef _Float16 orth_h2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t orth_pack(_Float16 a, _Float16 b) { return __builtin_bit_cast(uint32_t, orth_h2{a, b}); }
// Values as they are held, ORTH_UP or ORTH_X_UP times the number: u to its two halves and back
__device__ __forceinline__ void orth_halves(float u, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)u;
    lo = (_Float16)(u - (float)hi);
}
// four in a row, at a multiple of four
__device__ __forceinline__ void orth_put4(const orth_view &v, size_t at, const float (&u)[4]) {
    _Float16 hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; i++) orth_halves(u[i], hi[i], lo[i]);
    *(uint2 *)(v.hi + at) = make_uint2(orth_pack(hi[0], hi[1]), orth_pack(hi[2], hi[3]));
    if (v.lo) *(uint2 *)(v.lo + at) = make_uint2(orth_pack(lo[0], lo[1]), orth_pack(lo[2], lo[3]));
}
__device__ __forceinline__ void orth_get4(const orth_view &v, size_t at, float (&u)[4]) {
    const uint2 h = *(const uint2 *)(v.hi + at);
    const orth_h2 h0 = __builtin_bit_cast(orth_h2, h.x), h1 = __builtin_bit_cast(orth_h2, h.y);
    u[0] = (float)h0.x; u[1] = (float)h0.y; u[2] = (float)h1.x; u[3] = (float)h1.y;
    if (v.lo) {
        const uint2 l = *(const uint2 *)(v.lo + at);
        const orth_h2 l0 = __builtin_bit_cast(orth_h2, l.x), l1 = __builtin_bit_cast(orth_h2, l.y);
        u[0] += (float)l0.x; u[1] += (float)l0.y; u[2] += (float)l1.x; u[3] += (float)l1.y;
    }
}
__device__ __forceinline__ float orth_get(const orth_view &v, size_t at) {
    const float h = slz_f16_to_f32(v.hi[at]);
    return (v.lo ? h + slz_f16_to_f32(v.lo[at]) : h) * (1.0f / ORTH_X_UP);
}

// The first X is g 2^-e; with 2^e the power of two at or below the norm (1 for a norm of 0 or none) what is missing to g / norm is a factor above 1/2, at most 1
__device__ __forceinline__ int orth_exponent(double norm) {
    int e = 1;
    if (norm > 0.0 && norm < 1e300) frexp(norm, &e);
    return e - 1;
}

// ---- norm and first X -------------------------------------------------------------------------------------------------------------------
// Sums of squares of a matrix, in ORTH_NORM_BLOCKS parts at most; eight elements of a row at a time, four such under way in a thread
template <int TYPE>
__global__ void __launch_bounds__(256)
k_orth_norm(const void *__restrict__ g, uint32_t rows, uint32_t cols, int64_t ld, int64_t stride, double *__restrict__ part) {
    const uint32_t per_row = (cols + 7u) / 8u;
    const size_t base = (size_t)blockIdx.y * stride, total = (size_t)rows * per_row, each = (total + gridDim.x - 1) / gridDim.x;
    const size_t first = blockIdx.x * each, last = first + each < total ? first + each : total;
    double sum = 0.0;
    for (size_t i0 = first + threadIdx.x; i0 < last; i0 += 256 * 4) {
        row8<TYPE> x[4];
        uint32_t c[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const size_t r = slz_divide(i0 + q * 256 < last ? i0 + q * 256 : i0, per_row, total <= 0xffffffffu, c[q]);
            c[q] *= 8u;
            x[q] = row8_load<TYPE>(g, base + r * ld, c[q], cols);
        }
#pragma unroll
        for (int q = 0; q < 4; q++) {
            if (i0 + q * 256 >= last) continue;
            float v[8];
            row8_values<TYPE>(x[q], c[q], cols, v);
#pragma unroll
            for (int k = 0; k < 8; k++) sum += (double)v[k] * (double)v[k];
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    __shared__ double waves[4];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.y * ORTH_NORM_BLOCKS + blockIdx.x] = waves[0] + waves[1] + waves[2] + waves[3];
}
// 64 x 64 elements per workgroup, through shared memory where the transpose is wanted; factor: what g / (|g| + eps) is of the X written
template <int TYPE>
__global__ void __launch_bounds__(256)
k_orth_load(const void *__restrict__ g, uint32_t rows, uint32_t cols, int64_t ld, int64_t stride, int tall, const double *__restrict__ part,
            uint32_t parts, float eps, orth_view x, float *__restrict__ factor) {
    __shared__ float tile[64][65];
    const uint32_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, t = threadIdx.x;
    const size_t base = (size_t)blockIdx.z * stride;
    float own[16];
#pragma unroll
    for (int q = 0; q < 16; q++) {
        const uint32_t i = t + q * 256, r = r0 + i / 64, c = c0 + i % 64;
        own[q] = slz_get(g, TYPE, base + (size_t)min(r, rows - 1u) * ld + min(c, cols - 1u));       // all sixteen under way
        if (r >= rows || c >= cols) own[q] = 0.0f;
    }
    double sum = 0.0;
    for (uint32_t i = t & 63u; i < parts; i += 64) sum += part[blockIdx.z * ORTH_NORM_BLOCKS + i];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    const double norm = sqrt(sum) + (double)eps;
    const int e = orth_exponent(norm);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) factor[blockIdx.z] = (float)(ldexp(1.0, e) / norm);
#pragma unroll
    for (int q = 0; q < 16; q++) tile[(t + q * 256) / 64][t % 64] = ldexpf(own[q], -e) * ORTH_X_UP;
    __syncthreads();
    const uint32_t m = tall ? cols : rows, wide = ((tall ? rows : cols) + 7u) & ~7u;
#pragma unroll
    for (uint32_t i = t; i < t + 1024; i += 256) {
        const uint32_t a = i / 16, b = i % 16 * 4, r = (tall ? c0 : r0) + a, c = (tall ? r0 : c0) + b;
        float v[4];
        for (int q = 0; q < 4; q++) v[q] = tall ? tile[b + q][a] : tile[a][b + q];
        if (r < m && c < wide) orth_put4(x, blockIdx.z * x.stride + (size_t)r * x.ld + c, v);
    }
}
__global__ void __launch_bounds__(256)
k_orth_store(orth_view x, const float *__restrict__ factor, void *__restrict__ out, int type, uint32_t rows, uint32_t cols, int64_t ld, int64_t stride, int tall) {
    const size_t total = (size_t)rows * cols;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        const size_t r = g / cols, c = g % cols;
        slz_put(out, type, blockIdx.y * stride + r * ld + c, orth_get(x, blockIdx.y * x.stride + (tall ? c * x.ld + r : r * x.ld + c)) * factor[blockIdx.y]);
    }
}

// ---- the three products of a step -----------------------------------------------------------------------------------------------------------
// A symmetric product's result: the diagonal apart, the rest to `out` with zeros on the diagonal and in the columns up to the next multiple of 8.
// A tile below the diagonal is stored a second time, transposed through shared memory, half by half.
template <class F> struct orth_symmetric_epi {
    static constexpr bool any_side = true;
    static constexpr int widest = 192;
    orth_view out;
    float *diagonal;                 // [batch][m]
    F f;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *lds) const {
        // Transposed 2-byte words of one half, or of both where the operands' buffers hold them.  The pitch keeps 16-byte alignment; without the 8 both
        // halves of a tile of 128 x 128 fill the buffers.
        constexpr uint32_t TM = WM * MI * 16, TN = WN * NI * 16, ROOM = 2 * (TM + TN) * 128, PITCH = TM + (TM == 128 ? 0 : 8), HALF = TN * PITCH;
        constexpr int AT_ONCE = 2 * HALF * 2 <= ROOM ? 2 : 1;
        static_assert(HALF * 2 <= ROOM, "fits the operands' buffers");
        const uint32_t wide = (p.M + 7u) & ~7u, m0 = at.tile_m * TM, n0 = at.tile_n * TN;
        const size_t base = at.batch * out.stride;
        uint16_t *turned = (uint16_t *)lds;
        // all that is read before anything is written: the compiler may not move one past the other
        float u[MI][NI][4];
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const uint32_t m = slz_row(at, i), n = slz_col<NI, RUN>(at, j);
                u[i][j][0] = u[i][j][1] = u[i][j][2] = u[i][j][3] = 0.0f;
                if (m < p.M && n < p.M) f(at.batch, m, n, acc[i][j], u[i][j]);
            }
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const uint32_t m = slz_row(at, i), n = slz_col<NI, RUN>(at, j);
                if (at.tile_m == at.tile_n)
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        if (m == n + c && m < p.M) {
                            diagonal[at.batch * p.M + m] = f.on_diagonal(at.batch, m, u[i][j][c]);
                            u[i][j][c] = 0.0f;
                        }
#pragma unroll
                for (int c = 0; c < 4; c++) u[i][j][c] = n + c < p.M ? u[i][j][c] : 0.0f;
                if (m < p.M && n < wide) orth_put4(out, base + (size_t)m * out.ld + n, u[i][j]);
            }
        if (at.tile_m == at.tile_n) return;
        const int halves = out.lo ? 2 : 1;
        for (int first = 0; first < halves; first += AT_ONCE) {
            const int last = min(halves, first + AT_ONCE);
            for (int half = first; half < last; half++)
#pragma unroll
                for (int i = 0; i < MI; i++)
#pragma unroll
                    for (int j = 0; j < NI; j++)
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            _Float16 hi, lo;
                            orth_halves(u[i][j][c], hi, lo);
                            turned[(half - first) * HALF + (slz_col<NI, RUN>(at, j) - n0 + c) * PITCH + slz_row(at, i) - m0] = __builtin_bit_cast(uint16_t, half ? lo : hi);
                        }
            __syncthreads();
            for (int half = first; half < last; half++) {
                uint16_t *to = (half ? out.lo : out.hi) + base;
                for (uint32_t g = threadIdx.x; g < TN * (TM / 8); g += WM * WN * 64) {
                    const uint32_t n = g / (TM / 8), m = g % (TM / 8) * 8;
                    if (n0 + n < p.M && m0 + m < wide) *(uint4 *)(to + (size_t)(n0 + n) * out.ld + m0 + m) = *(const uint4 *)(turned + (half - first) * HALF + n * PITCH + m);
                }
            }
            __syncthreads();
        }
    }
};
struct orth_gram {
    const float *factor;             // or null
    __device__ __forceinline__ void operator()(uint32_t batch, uint32_t, uint32_t, const v4f &sum, float (&u)[4]) const {
        const float f = factor ? factor[batch] : 1.0f, by = f * f * (ORTH_UP / ORTH_X_UP / ORTH_X_UP);
#pragma unroll
        for (int c = 0; c < 4; c++) u[c] = sum[c] * by;
    }
    __device__ __forceinline__ float on_diagonal(uint32_t, uint32_t, float u) const { return u * (1.0f / ORTH_UP); }
};
// The same of sums in ranges: few tiles and many columns leave most of the chip idle, so k is cut, all tiles are computed and their sums joined here.
// A thread has four columns.
__global__ void __launch_bounds__(256)
k_orth_gram_join(const float *__restrict__ ranges, uint32_t count, uint32_t batches, uint32_t M, uint32_t ld, orth_gram f, orth_view out, float *__restrict__ diagonal) {
    const uint32_t batch = blockIdx.z, m = blockIdx.y, n = (blockIdx.x * 256 + threadIdx.x) * 4, wide = (M + 7u) & ~7u;
    if (n >= wide) return;
    v4f sum = v4f{0, 0, 0, 0};
    if (n < M)
#pragma unroll 8
        for (uint32_t r = 0; r < count; r++) sum += *(const v4f *)(ranges + (((size_t)r * batches + batch) * M + m) * ld + n);
    float u[4];
    f(batch, m, n, sum, u);
#pragma unroll
    for (int c = 0; c < 4; c++) {
        if (m == n + c) diagonal[batch * M + m] = f.on_diagonal(batch, m, u[c]);
        if (m == n + c || n + c >= M) u[c] = 0.0f;
    }
    orth_put4(out, batch * out.stride + (size_t)m * out.ld + n, u);
}
// b O + c (O O + (d_m + d_n) O), and a + b d + c (O O + d^2) on the diagonal, where O is zero
struct orth_polynomial {
    orth_view o;
    const float *d;                  // of A
    uint32_t m_all;
    float a, b, c;
    __device__ __forceinline__ void operator()(uint32_t batch, uint32_t m, uint32_t n, const v4f &sum, float (&u)[4]) const {
        float x[4];
        orth_get4(o, batch * o.stride + (size_t)m * o.ld + n, x);
        const float bm = b + c * d[batch * m_all + m];
#pragma unroll
        for (int q = 0; q < 4; q++) u[q] = sum[q] * (c / ORTH_UP) + (bm + c * d[batch * m_all + min(n + q, m_all - 1)]) * x[q];
    }
    __device__ __forceinline__ float on_diagonal(uint32_t batch, uint32_t m, float u) const {
        const float dm = d[batch * m_all + m];
        return a + u * (1.0f / ORTH_UP) + dm * (b + c * dm);
    }
};
struct orth_apply_epi {
    static constexpr bool any_side = true;
    static constexpr int widest = 256;
    orth_view x, next;               // this step's X and the next one's
    const float *diagonal;           // a + B_ii
    const float *factor;             // or null
    void *out;                       // the last step's result goes here, or null
    int type, tall;
    uint32_t aligned;                // its rows begin at multiples of 16 bytes
    int64_t ld_out, stride_out;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *) const {
        const uint32_t wide = (p.N + 7u) & ~7u;
        const float f = factor ? factor[at.batch] : 1.0f;
        // a row's X is read before the row before it is written
        float old[2][NI][4], d[2];
        const auto load = [&](int i) {
            const uint32_t m = min(slz_row(at, i), p.M - 1);
            d[i & 1] = f * diagonal[at.batch * p.M + m];
#pragma unroll
            for (int j = 0; j < NI; j++) orth_get4(x, at.batch * x.stride + (size_t)m * x.ld + min(slz_col<NI, RUN>(at, j), wide - 4), old[i & 1][j]);
        };
        load(0);
#pragma unroll
        for (int i = 0; i < MI; i++) {
            if (i + 1 < MI) load(i + 1);
            const uint32_t m = slz_row(at, i);
            if (m >= p.M) continue;
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const uint32_t n = slz_col<NI, RUN>(at, j);
                if (n >= wide) continue;
                float v[4];
#pragma unroll
                for (int c = 0; c < 4; c++) v[c] = n + c < p.N ? d[i & 1] * old[i & 1][j][c] + acc[i][j][c] * (f / ORTH_UP) : 0.0f;
                if (!out) orth_put4(next, at.batch * x.stride + (size_t)m * x.ld + n, v);
                else if (n < p.N) {
#pragma unroll
                    for (int c = 0; c < 4; c++) v[c] *= 1.0f / ORTH_X_UP;
                    const int64_t first = at.batch * stride_out;
                    if (!tall) slz_put_run<4>((char *)out + (first + (int64_t)m * ld_out + n) * slz_type_bytes(type), type, v, p.N - n, aligned);
                    else
#pragma unroll
                        for (int c = 0; c < 4; c++)
                            if (n + c < p.N) slz_put(out, type, first + (int64_t)(n + c) * ld_out + m, v[c]);
                }
            }
        }
    }
};

// ---- up to 128 rows -----------------------------------------------------------------------------------------------------------------------------
// A step's three products need of X only a slice of columns, but for the sum over slices that is A.  A workgroup holds a slice in shared memory: it
// makes B = b A + c A A (every workgroup the same), applies it to its columns in place, and adds up its part of the next A.  Where one slice
// holds the matrix, all steps are one launch; otherwise a step is one, and the parts of A go through memory.  The tiled products would be three
// launches a step with little to do.
// MP: rows padded with zeros.  A wave has MP / (WAVES / 2) rows and half the columns of A and B, and takes 16 columns of X at a time.
#define SMALL_ROWS 128
#define SMALL_LDS (152u << 10)
#define SMALL_PARTS (1u << 17)
template <int MP> struct small_shape {
    static constexpr int WAVES = MP == 32 ? 4 : 8, GM = MP / (WAVES / 2) / 16, GN = MP / 2 / 16;
    static constexpr uint32_t PITCH_O = MP * 2 + 16, BYTES_O = MP * PITCH_O;
};
struct small_args {
    const void *g;
    int type, tall;
    uint32_t rows, cols;
    int64_t ld_g, stride_g;
    void *out;
    uint32_t aligned;                // out's rows begin at multiples of 16 bytes
    int64_t ld_out, stride_out;
    orth_view x;                     // between launches
    const float *sums;               // parts of A: [batch][count][lanes' order]
    uint32_t count;
    float *next_sums;                // [batch][slices][lanes' order]
    const double *part;              // sums of squares, or null: one slice, which adds them up itself
    uint32_t parts;
    float eps;
    float *factor;                   // [batch]; null after the first step
    uint32_t m, n, slice;            // columns of a slice, a multiple of 32
    uint32_t steps, last;            // of SMALL_ALL; whether a step's X is the result
    float a, b, c;
};

// f(row, column within the slice or, for tall, of g, values) for every eight elements of a slice of g, zeros past a row's end; four such under way
template <int TYPE, int THREADS, class F>
__device__ __forceinline__ void small_elements_of(const small_args &p, uint32_t batch, uint32_t c0, uint32_t width, const F &f) {
    const uint32_t in_rows = p.tall ? width : p.rows, per_row = ((p.tall ? p.cols : width) + 7u) / 8u, total = in_rows * per_row;
    const uint32_t first_row = p.tall ? c0 : 0u, first_col = p.tall ? 0u : c0;
    for (uint32_t i0 = threadIdx.x; i0 < total; i0 += THREADS * 4) {
        row8<TYPE> x[4];
        uint32_t row[4], col[4];
#pragma unroll
        for (uint32_t q = 0; q < 4; q++) {
            const uint32_t i = min(i0 + q * THREADS, total - 1);
            row[q] = i / per_row;
            col[q] = (i - row[q] * per_row) * 8u;
            x[q] = row8_load<TYPE>(p.g, (size_t)batch * p.stride_g + (size_t)(first_row + row[q]) * p.ld_g, first_col + col[q], p.cols);
        }
#pragma unroll
        for (uint32_t q = 0; q < 4; q++) {
            if (i0 + q * THREADS >= total) continue;
            float v[8];
            row8_values<TYPE>(x[q], first_col + col[q], p.cols, v);
            f(row[q], col[q], v);
        }
    }
}
template <int THREADS, class F> __device__ __forceinline__ void small_elements(const small_args &p, uint32_t batch, uint32_t c0, uint32_t width, const F &f) {
    if (p.type == SLZ_F32) small_elements_of<SLZ_F32, THREADS>(p, batch, c0, width, f);
    else if (p.type == SLZ_BF16) small_elements_of<SLZ_BF16, THREADS>(p, batch, c0, width, f);
    else small_elements_of<SLZ_F16, THREADS>(p, batch, c0, width, f);
}

// The launches: all of a matrix that is one slice; the first part of A of X from g; a step.
// All of it: 128 x 784 bf16 77 us (a step: this 11.0, the sum of A's parts 4.0), 128 x 128 38, 64 x 512 45, 32 x 8192 64; bound by the latency of products in a row.
enum { SMALL_ALL, SMALL_FIRST, SMALL_STEP };
template <int MP, int PIECES, int KIND>
__global__ void __launch_bounds__(small_shape<MP>::WAVES * 64) k_orth_small(const small_args p) {
    using S = small_shape<MP>;
    constexpr int THREADS = S::WAVES * 64, GM = S::GM, GN = S::GN, RT = MP / 16;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float diagonal[MP], scale[MP];
    __shared__ double wave_sums[S::WAVES];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    const uint32_t batch = blockIdx.y, c0 = blockIdx.x * p.slice, width = min(p.slice, p.n - c0), padded = (width + 31u) & ~31u;
    const uint32_t pitch = p.slice * 2u + 16u, bytes_x = MP * pitch;
    char *o_at[2] = {lds, lds + S::BYTES_O}, *x_at[2] = {lds + PIECES * S::BYTES_O, lds + PIECES * S::BYTES_O + bytes_x};
    const uint32_t m_wave = (wave >> 1) * (GM * 16), n_wave = (wave & 1u) * (GN * 16);

    // the slice: zeros in rows past m and columns past n
    if (p.m < MP || width < p.slice)
        for (uint32_t i = threadIdx.x * 16u; i < 2u * bytes_x; i += THREADS * 16u) *(uint4 *)(x_at[0] + i) = make_uint4(0, 0, 0, 0);
    const uint32_t order = (wave * GM * GN * 64u + lane) * 4u;                      // a wave's sums lie together, 16 bytes a lane
    constexpr uint32_t SQUARE = MP * MP;
    v4f acc[GM][GN];
    if constexpr (KIND == SMALL_STEP) {
        // this step's A: the parts in their order
        const float *from = p.sums + (size_t)batch * p.count * SQUARE + order;
#pragma unroll
        for (int i = 0; i < GM; i++)
#pragma unroll
            for (int j = 0; j < GN; j++) acc[i][j] = *(const v4f *)(from + (i * GN + j) * 256);
#pragma unroll 4
        for (uint32_t q = 1; q < p.count; q++)
#pragma unroll
            for (int i = 0; i < GM; i++)
#pragma unroll
                for (int j = 0; j < GN; j++) acc[i][j] += *(const v4f *)(from + (size_t)q * SQUARE + (i * GN + j) * 256);
    }
    float factor = 1.0f;
    if constexpr (KIND != SMALL_STEP) {
        double sum = 0.0;
        if constexpr (KIND == SMALL_FIRST)
            for (uint32_t i = threadIdx.x; i < p.parts; i += THREADS) sum += p.part[batch * ORTH_NORM_BLOCKS + i];
        else small_elements<THREADS>(p, batch, c0, width, [&](uint32_t, uint32_t, const float (&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; i++) sum += (double)v[i] * (double)v[i];
        });
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
        if (lane == 0) wave_sums[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < S::WAVES; w++) sum += wave_sums[w];
        const double norm = sqrt(sum) + (double)p.eps;
        const int e = orth_exponent(norm);
        factor = (float)(ldexp(1.0, e) / norm);
        if (KIND == SMALL_FIRST && blockIdx.x == 0 && threadIdx.x == 0) p.factor[batch] = factor;
        small_elements<THREADS>(p, batch, c0, width, [&](uint32_t row, uint32_t col, const float (&v)[8]) {
            _Float16 hi[8], lo[8];
#pragma unroll
            for (int i = 0; i < 8; i++) orth_halves(ldexpf(v[i], -e) * ORTH_X_UP, hi[i], lo[i]);
            if (!p.tall) {
                const uint32_t to = row * pitch + col * 2u;
                *(uint4 *)(x_at[0] + to) = make_uint4(orth_pack(hi[0], hi[1]), orth_pack(hi[2], hi[3]), orth_pack(hi[4], hi[5]), orth_pack(hi[6], hi[7]));
                *(uint4 *)(x_at[1] + to) = make_uint4(orth_pack(lo[0], lo[1]), orth_pack(lo[2], lo[3]), orth_pack(lo[4], lo[5]), orth_pack(lo[6], lo[7]));
            } else
#pragma unroll
                for (uint32_t i = 0; i < 8; i++)
                    if (col + i < p.cols) {
                        *(_Float16 *)(x_at[0] + (col + i) * pitch + row * 2u) = hi[i];
                        *(_Float16 *)(x_at[1] + (col + i) * pitch + row * 2u) = lo[i];
                    }
        });
    } else {
        __syncthreads();
        const size_t base = batch * p.x.stride + c0;
        const uint32_t chunks = (width + 7u) / 8u;
        for (uint32_t i0 = threadIdx.x; i0 < p.m * chunks; i0 += THREADS * 4) {
            v4i32 hi[4], lo[4];
            uint32_t to[4];
#pragma unroll
            for (uint32_t q = 0; q < 4; q++) {
                const uint32_t i = min(i0 + q * THREADS, p.m * chunks - 1), row = i / chunks, col = (i - row * chunks) * 8u;
                hi[q] = *(const v4i32 *)(p.x.hi + base + (size_t)row * p.x.ld + col);
                lo[q] = *(const v4i32 *)(p.x.lo + base + (size_t)row * p.x.ld + col);
                to[q] = row * pitch + col * 2u;
            }
#pragma unroll
            for (uint32_t q = 0; q < 4; q++) {
                *(v4i32 *)(x_at[0] + to[q]) = hi[q];
                *(v4i32 *)(x_at[1] + to[q]) = lo[q];
            }
        }
        if (p.factor) factor = p.factor[batch];
    }
    __syncthreads();

    // sums of products of rows: of X over the slice's columns, of O over all of its own
    const auto rows_product = [&](char *const(&from)[2], uint32_t row_pitch, uint32_t depth) {
#pragma unroll
        for (int i = 0; i < GM; i++)
#pragma unroll
            for (int j = 0; j < GN; j++) acc[i][j] = v4f{0, 0, 0, 0};
#pragma unroll 1
        for (int pair = PIECES == 2 ? 0 : 2; pair < 3; pair++) {
            const char *pa = from[pair == 0 ? 1 : 0], *pb = from[pair == 1 ? 1 : 0];
            for (uint32_t k = 0; k < depth; k += 32) {
                v4i32 fa[GM], fb[GN];
#pragma unroll
                for (int i = 0; i < GM; i++) fa[i] = *(const v4i32 *)(pa + (m_wave + i * 16 + r) * row_pitch + k * 2u + g * 16u);
#pragma unroll
                for (int j = 0; j < GN; j++) fb[j] = *(const v4i32 *)(pb + (n_wave + j * 16 + r) * row_pitch + k * 2u + g * 16u);
#pragma unroll
                for (int i = 0; i < GM; i++)
#pragma unroll
                    for (int j = 0; j < GN; j++) acc[i][j] = slz_mma<SLZ_EL_F16>(fb[j], fa[i], acc[i][j]);
            }
        }
    };
    // the wave's part of O or of B - diagonal, from values u; their diagonal has been taken out
    const auto put_square = [&](const float (&u)[GM][GN][4]) {
#pragma unroll
        for (int i = 0; i < GM; i++)
#pragma unroll
            for (int j = 0; j < GN; j++) {
                const uint32_t at = (m_wave + i * 16 + r) * S::PITCH_O + (n_wave + j * 16 + g * 4) * 2u;
                _Float16 hi[4], lo[4];
#pragma unroll
                for (int c = 0; c < 4; c++) orth_halves(u[i][j][c], hi[c], lo[c]);
                *(uint2 *)(o_at[0] + at) = make_uint2(orth_pack(hi[0], hi[1]), orth_pack(hi[2], hi[3]));
                if (PIECES == 2) *(uint2 *)(o_at[1] + at) = make_uint2(orth_pack(lo[0], lo[1]), orth_pack(lo[2], lo[3]));
            }
    };
    // f(row, value) for the wave's entries on the diagonal, which become zero
    const auto take_diagonal = [&](float (&u)[GM][GN][4], const auto &f) {
#pragma unroll
        for (int i = 0; i < GM; i++)
#pragma unroll
            for (int j = 0; j < GN; j++)
                if (m_wave + i * 16 == n_wave + j * 16)
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        if (r == g * 4 + c) {
                            f(m_wave + i * 16 + r, u[i][j][c]);
                            u[i][j][c] = 0.0f;
                        }
    };
    if constexpr (KIND != SMALL_STEP) rows_product(x_at, pitch, padded);
    const uint32_t steps = KIND == SMALL_ALL ? p.steps : KIND == SMALL_FIRST ? 0u : 1u;
    for (uint32_t step = 0; step < steps; step++) {
        float u[GM][GN][4];
        const float by = factor * factor * (ORTH_UP / ORTH_X_UP / ORTH_X_UP);
#pragma unroll
        for (int i = 0; i < GM; i++)
#pragma unroll
            for (int j = 0; j < GN; j++)
#pragma unroll
                for (int c = 0; c < 4; c++) u[i][j][c] = acc[i][j][c] * by;
        take_diagonal(u, [&](uint32_t m, float x) { diagonal[m] = x * (1.0f / ORTH_UP); });
        put_square(u);
        __syncthreads();
        rows_product(o_at, S::PITCH_O, MP);
        // b O + c (O O + (d_m + d_n) O) with O as its operand holds it, and a + b d + c (O O + d^2) on the diagonal
        float by_n[GN][4];
#pragma unroll
        for (int j = 0; j < GN; j++)
#pragma unroll
            for (int c = 0; c < 4; c++) by_n[j][c] = p.c * diagonal[n_wave + j * 16 + g * 4 + c];
#pragma unroll
        for (int i = 0; i < GM; i++) {
            const float by_m = p.b + p.c * diagonal[m_wave + i * 16 + r];
#pragma unroll
            for (int j = 0; j < GN; j++)
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    _Float16 hi, lo;
                    orth_halves(u[i][j][c], hi, lo);
                    u[i][j][c] = acc[i][j][c] * (p.c / ORTH_UP) + (by_m + by_n[j][c]) * (PIECES == 2 ? (float)hi + (float)lo : (float)hi);
                }
        }
        take_diagonal(u, [&](uint32_t m, float x) { scale[m] = p.a + x * (1.0f / ORTH_UP) + diagonal[m] * (p.b + p.c * diagonal[m]); });
        __syncthreads();
        put_square(u);
        __syncthreads();
        const bool to_out = KIND == SMALL_ALL ? step + 1 == steps : p.last;
        for (uint32_t col = wave * 16u; col < padded; col += S::WAVES * 16u) {
            v4f sum[RT];
#pragma unroll
            for (int i = 0; i < RT; i++) sum[i] = v4f{0, 0, 0, 0};
#pragma unroll 1
            for (int pair = PIECES == 2 ? 0 : 2; pair < 3; pair++) {
                const char *pa = o_at[pair == 0 ? 1 : 0], *pb = x_at[pair == 1 ? 1 : 0];
#pragma unroll
                for (int k = 0; k < MP; k += 32) {
                    v4i32 fx;
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const char *q = pb + (k + g * 8 + h * 4 + (r >> 2)) * pitch + (col + (r & 3u) * 4u) * 2u;
                        const uint64_t w = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s16 *)q));
                        fx[2 * h] = (int)(uint32_t)w;
                        fx[2 * h + 1] = (int)(uint32_t)(w >> 32);
                    }
#pragma unroll
                    for (int i = 0; i < RT; i++) sum[i] = slz_mma<SLZ_EL_F16>(fx, *(const v4i32 *)(pa + (i * 16 + r) * S::PITCH_O + k * 2 + g * 16u), sum[i]);
                }
            }
            // these columns are read and written by this wave alone
#pragma unroll
            for (int i = 0; i < RT; i++) {
                const uint32_t m = i * 16 + r, n = col + g * 4u;
                const orth_view here{(uint16_t *)x_at[0], (uint16_t *)x_at[1], 0, 0};
                const size_t at = m * (pitch / 2u) + n;
                float x[4];
                orth_get4(here, at, x);
                const float d = factor * scale[m];
#pragma unroll
                for (int c = 0; c < 4; c++) x[c] = d * x[c] + sum[i][c] * (factor / ORTH_UP);
                if (!to_out) orth_put4(here, at, x);
                else if (m < p.m && n < width) {
                    const size_t first = (size_t)batch * p.stride_out;
#pragma unroll
                    for (int c = 0; c < 4; c++) x[c] *= 1.0f / ORTH_X_UP;
                    if (!p.tall)
                        slz_put_run<4>((char *)p.out + (first + (size_t)m * p.ld_out + c0 + n) * slz_type_bytes(p.type), p.type, x, width - n, p.aligned);
                    else
#pragma unroll
                        for (int c = 0; c < 4; c++)
                            if (n + c < width) slz_put(p.out, p.type, first + (size_t)(c0 + n + c) * p.ld_out + m, x[c]);
                }
            }
        }
        factor = 1.0f;
        if (to_out) return;
        __syncthreads();
        rows_product(x_at, pitch, padded);
    }
    if constexpr (KIND == SMALL_ALL) return;
    // for the next launch
    float *to = p.next_sums + ((size_t)batch * gridDim.x + blockIdx.x) * SQUARE + order;
#pragma unroll
    for (int i = 0; i < GM; i++)
#pragma unroll
        for (int j = 0; j < GN; j++) *(v4f *)(to + (i * GN + j) * 256) = acc[i][j];
    const size_t base = batch * p.x.stride + c0;
    const uint32_t chunks = (width + 7u) / 8u;
    for (uint32_t i = threadIdx.x; i < p.m * chunks; i += THREADS) {
        const uint32_t row = i / chunks, col = (i - row * chunks) * 8u;
        *(uint4 *)(p.x.hi + base + (size_t)row * p.x.ld + col) = *(const uint4 *)(x_at[0] + row * pitch + col * 2u);
        *(uint4 *)(p.x.lo + base + (size_t)row * p.x.ld + col) = *(const uint4 *)(x_at[1] + row * pitch + col * 2u);
    }
}
// many parts of A to one
__global__ void __launch_bounds__(256) k_orth_sum(const float *__restrict__ parts, uint32_t count, uint32_t square, float *__restrict__ sum) {
    const uint32_t i = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= square) return;
    const float *from = parts + (size_t)blockIdx.y * count * square + i;
    v4f s = *(const v4f *)from;
#pragma unroll 8
    for (uint32_t q = 1; q < count; q++) s += *(const v4f *)(from + (size_t)q * square);
    *(v4f *)(sum + (size_t)blockIdx.y * square + i) = s;
}

struct orth_plan {
    uint32_t m, n, pieces;
    uint32_t ld_x, ld_a;
    size_t one_x, one_a;             // bytes of a piece of X, of A or B
    size_t x[2], a, b, da, db, factor, part, total;
    slz_choice gram, polynomial, apply;
    size_t ranges;
    uint32_t padded, slice, slices;                  // up to 128 rows: rows padded, columns of a workgroup, workgroups of a matrix
    size_t sums[2];
};
// Columns of a workgroup: as many as its shared memory holds where that is all of them, else fewer, so that more workgroups share a step out
static uint32_t small_lds(uint32_t padded, uint32_t pieces, uint32_t slice) { return pieces * padded * (padded * 2 + 16) + 2 * padded * (slice * 2 + 16); }
static void small_slices(orth_plan &P) {
    const uint32_t all = (P.n + 31) / 32 * 32;
    if (all <= 8192 && small_lds(P.padded, P.pieces, all) <= SMALL_LDS) { P.slice = all; P.slices = 1; return; }
    P.slice = 16384 / P.padded;
    P.slices = (P.n + P.slice - 1) / P.slice;
}
// Two pieces: three products one after the other in any tiling, or tiles of 64 that load both pieces at once.  These read a third less, but large
// tiles read less still: f32, 6 x 500 x 1000 277 us together and 345 in turn, 1024^2 279 and 431, 4096 x 8192 9532 and 6889
static slz_choice orth_choose(const orth_plan &P, uint32_t N, uint32_t steps, uint32_t batch, bool symmetric, uint32_t most_ranges, bool rows_k) {
    if (P.pieces == 1) return slz_choose(P.m, N, steps, batch, symmetric, most_ranges, rows_k);
    const slz_choice in_turn = slz_choose(P.m, N, steps * 3, batch, symmetric, most_ranges, rows_k);
    const slz_choice together = slz_choose(P.m, N, steps, batch, symmetric, most_ranges, rows_k, true, 2);
    return together.us < in_turn.us ? together : in_turn;
}
static orth_plan plan_orth(const slz_orth_shape *sh) {
    orth_plan P = {};
    P.m = sh->rows < sh->cols ? sh->rows : sh->cols;
    P.n = sh->rows < sh->cols ? sh->cols : sh->rows;
    P.pieces = sh->type == SLZ_BF16 ? 1 : 2;
    P.ld_x = (P.n + 63) / 64 * 64;
    P.ld_a = (P.m + 63) / 64 * 64;
    P.one_x = up256((size_t)sh->batch * P.m * P.ld_x * 2);
    P.one_a = up256((size_t)sh->batch * P.m * P.ld_a * 2);
    P.padded = P.m <= 32 ? 32 : P.m <= 64 ? 64 : P.m <= SMALL_ROWS ? 128 : 0;
    if (P.padded && sh->steps) {
        small_slices(P);
        size_t o = 0;
        if (P.slices > 1) {
            const size_t square = (size_t)P.padded * P.padded * 4;
            P.x[0] = o; o += 2 * P.one_x;
            for (int i = 0; i < 2; i++) { P.sums[i] = o; o += up256((size_t)sh->batch * P.slices * square); }
            P.factor = o; o += up256((size_t)sh->batch * 4);
            P.part = o; o += up256((size_t)sh->batch * ORTH_NORM_BLOCKS * 8);
        }
        P.total = o;
        return P;
    }
    size_t o = 0;
    for (int i = 0; i < 2; i++) { P.x[i] = o; o += 2 * P.one_x; }
    P.a = o; o += P.pieces * P.one_a;
    P.b = o; o += P.pieces * P.one_a;
    P.da = o; o += up256((size_t)sh->batch * P.m * 4);
    P.db = o; o += up256((size_t)sh->batch * P.m * 4);
    P.factor = o; o += up256((size_t)sh->batch * 4);
    P.part = o; o += up256((size_t)sh->batch * ORTH_NORM_BLOCKS * 8);
    const uint32_t steps = (P.n + 63) / 64;
    P.gram = orth_choose(P, P.m, steps, sh->batch, true, 1, false);
    const slz_choice cut = orth_choose(P, P.m, steps, sh->batch, false, 32, false);
    if (cut.us < P.gram.us && P.m <= 65535) P.gram = cut;
    P.ranges = o; o += P.gram.split > 1 ? up256((size_t)P.gram.split * sh->batch * P.m * slz_ranges_ld(P.m) * 4) : 0;
    P.total = o;
    P.polynomial = orth_choose(P, P.m, (P.m + 63) / 64, sh->batch, true, 1, false);
    P.apply = orth_choose(P, P.n, (P.m + 63) / 64, sh->batch, false, 1, true);
    return P;
}
static int orth_check(const slz_orth_shape *sh) {
    if (!sh || !slz_type_ok(sh->type) || sh->steps > 64) return SLZ_E_INVALID_ARG;
    if (sh->ld_g < (int64_t)sh->cols || sh->ld_out < (int64_t)sh->cols) return SLZ_E_INVALID_ARG;
    if (sh->batch > 65535 || sh->rows >= SLZ_CLEAR_MAX_LD || sh->cols > SLZ_CLEAR_MAX_LD) return SLZ_E_TOO_LARGE;
    return SLZ_OK;
}
extern "C" int slz_orthogonalize_workspace(const slz_orth_shape *sh, size_t *bytes) {
    const int rc = orth_check(sh);
    if (rc != SLZ_OK) return rc;
    if (!bytes) return SLZ_E_INVALID_ARG;
    *bytes = sh->batch && sh->rows && sh->cols ? plan_orth(sh).total : 0;
    return SLZ_OK;
}

static slz_gemm orth_product(const orth_view &a, const orth_view &b, uint32_t pieces, const slz_choice &c, uint32_t M, uint32_t N, uint32_t K) {
    slz_gemm p = {};
    p.a = (const char *)a.hi; p.b = (const char *)b.hi;
    p.lda = (int64_t)a.ld * 2; p.ldb = (int64_t)b.ld * 2;
    p.a_batch = (int64_t)a.stride * 2; p.b_batch = (int64_t)b.stride * 2;
    p.M = M; p.N = N; p.K = K;
    p.split = 1;
    p.pairs = pieces == 2 && c.pieces == 1 ? 3 : 1;    // in turn, the small products first
    if (pieces == 2) {
        p.a_piece[c.pieces == 2 ? 1 : 0] = (const char *)a.lo - (const char *)a.hi;
        p.b_piece[1] = (const char *)b.lo - (const char *)b.hi;
    }
    return p;
}

static uint32_t orth_aligned(const slz_orth_shape *sh, const void *out) {
    const uint32_t eb = slz_type_bytes(sh->type);
    return slz_in_place(out, 16, sh->ld_out, eb) && (sh->batch == 1 || sh->stride_out * eb % 16 == 0);
}
// sums of squares of each matrix, in the returned number of parts
static uint32_t orth_norm(const slz_orth_shape *sh, const void *g, double *part, hipStream_t s) {
    const uint64_t needed = ((uint64_t)sh->rows * sh->cols + 8191) / 8192;
    const uint32_t parts = needed < ORTH_NORM_BLOCKS ? (uint32_t)needed : ORTH_NORM_BLOCKS;
    const auto norm = sh->type == SLZ_F32 ? k_orth_norm<SLZ_F32> : sh->type == SLZ_BF16 ? k_orth_norm<SLZ_BF16> : k_orth_norm<SLZ_F16>;
    hipLaunchKernelGGL(norm, dim3(parts, sh->batch), dim3(256), 0, s, g, sh->rows, sh->cols, sh->ld_g, sh->stride_g, part);
    return parts;
}
template <int MP, int PIECES> static void small_launch_of(const small_args &p, int kind, const orth_plan &P, uint32_t batch, hipStream_t s) {
    const auto k = kind == SMALL_ALL ? k_orth_small<MP, PIECES, SMALL_ALL> : kind == SMALL_FIRST ? k_orth_small<MP, PIECES, SMALL_FIRST> : k_orth_small<MP, PIECES, SMALL_STEP>;
    hipLaunchKernelGGL(k, dim3(P.slices, batch), dim3(small_shape<MP>::WAVES * 64), small_lds(MP, P.pieces, P.slice), s, p);
}
template <int MP> static void small_launch(const small_args &p, int kind, const orth_plan &P, uint32_t batch, hipStream_t s) {
    if (P.pieces == 2) small_launch_of<MP, 2>(p, kind, P, batch, s);
    else small_launch_of<MP, 1>(p, kind, P, batch, s);
}
static int orth_small(const slz_orth_shape *sh, const orth_plan &P, const void *g, void *out, char *w, hipStream_t s) {
    small_args p = {};
    p.g = g; p.type = sh->type; p.tall = sh->rows > sh->cols;
    p.rows = sh->rows; p.cols = sh->cols; p.ld_g = sh->ld_g; p.stride_g = sh->stride_g;
    p.out = out; p.aligned = orth_aligned(sh, out); p.ld_out = sh->ld_out; p.stride_out = sh->stride_out;
    p.eps = sh->eps;
    p.m = P.m; p.n = P.n; p.slice = P.slice;
    p.a = sh->a; p.b = sh->b; p.c = sh->c;
    const auto launch = [&](int kind) {
        if (P.padded == 32) small_launch<32>(p, kind, P, sh->batch, s);
        else if (P.padded == 64) small_launch<64>(p, kind, P, sh->batch, s);
        else small_launch<128>(p, kind, P, sh->batch, s);
    };
    if (P.slices == 1) {
        p.steps = sh->steps;
        launch(SMALL_ALL);
        return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
    }
    const uint32_t square = P.padded * P.padded;
    float *sums[2] = {(float *)(w + P.sums[0]), (float *)(w + P.sums[1])};
    p.x = {(uint16_t *)(w + P.x[0]), (uint16_t *)(w + P.x[0] + P.one_x), P.ld_x, (size_t)P.m * P.ld_x};
    p.part = (double *)(w + P.part);
    p.parts = orth_norm(sh, g, (double *)(w + P.part), s);
    p.factor = (float *)(w + P.factor);
    p.next_sums = sums[0];
    launch(SMALL_FIRST);
    // parts of A that every workgroup would read in more than the time of a launch are added up by one
    const bool many = (size_t)P.slices * square * 4 > SMALL_PARTS;
    for (uint32_t i = 0; i < sh->steps; i++) {
        float *now = sums[many ? 0 : i & 1];
        p.sums = now;
        p.count = P.slices;
        p.next_sums = sums[many ? 0 : (i & 1) ^ 1];
        if (many) {
            hipLaunchKernelGGL(k_orth_sum, dim3((square / 4 + 255) / 256, sh->batch), dim3(256), 0, s, now, P.slices, square, sums[1]);
            p.sums = sums[1];
            p.count = 1;
        }
        p.factor = i == 0 ? (float *)(w + P.factor) : nullptr;
        p.last = i + 1 == sh->steps;
        launch(SMALL_STEP);
    }
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}

template <bool B_ROWS_K, class EPI> static int orth_run(const slz_gemm &p, const EPI &epi, const slz_choice &c, uint32_t batches, hipStream_t s) {
    return c.pieces == 2 ? slz_gemm_run2<SLZ_EL_F16, false, B_ROWS_K>(p, epi, batches, s) : slz_gemm_run<SLZ_EL_F16, false, B_ROWS_K>(p, epi, c.side, batches, s);
}
extern "C" int slz_orthogonalize(const slz_orth_shape *sh, const void *g, void *out, void *ws, size_t ws_bytes, void *stream) {
    const int rc0 = orth_check(sh);
    if (rc0 != SLZ_OK) return rc0;
    if (sh->batch == 0 || sh->rows == 0 || sh->cols == 0) return SLZ_OK;
    const uint32_t eb = slz_type_bytes(sh->type);
    if (!g || !out || (uintptr_t)g % eb || (uintptr_t)out % eb) return SLZ_E_INVALID_ARG;
    const orth_plan P = plan_orth(sh);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    char *w = (char *)ws;
    if (P.padded && sh->steps) return orth_small(sh, P, g, out, w, s);
    const int tall = sh->rows > sh->cols;
    const size_t xs = (size_t)P.m * P.ld_x, as = (size_t)P.m * P.ld_a;
    orth_view x[2], a, b;
    for (int i = 0; i < 2; i++) x[i] = {(uint16_t *)(w + P.x[i]), (uint16_t *)(w + P.x[i] + P.one_x), P.ld_x, xs};
    a = {(uint16_t *)(w + P.a), P.pieces == 2 ? (uint16_t *)(w + P.a + P.one_a) : nullptr, P.ld_a, as};
    b = {(uint16_t *)(w + P.b), P.pieces == 2 ? (uint16_t *)(w + P.b + P.one_a) : nullptr, P.ld_a, as};
    float *da = (float *)(w + P.da), *db = (float *)(w + P.db), *factor = (float *)(w + P.factor);
    double *part = (double *)(w + P.part);
    const uint32_t aligned = orth_aligned(sh, out);
    const uint32_t parts = orth_norm(sh, g, part, s);
    const auto load = sh->type == SLZ_F32 ? k_orth_load<SLZ_F32> : sh->type == SLZ_BF16 ? k_orth_load<SLZ_BF16> : k_orth_load<SLZ_F16>;
    hipLaunchKernelGGL(load, dim3((sh->cols + 63) / 64, (sh->rows + 63) / 64, sh->batch), dim3(256), 0, s, g, sh->rows, sh->cols, sh->ld_g,
                       sh->stride_g, tall, part, parts, sh->eps, x[0], factor);
    if (sh->steps == 0)
        hipLaunchKernelGGL(k_orth_store, dim3(1024, sh->batch), dim3(256), 0, s, x[0], factor, out, sh->type, sh->rows, sh->cols, sh->ld_out, sh->stride_out, tall);
    for (uint32_t i = 0; i < sh->steps; i++) {
        const orth_view &now = x[i & 1], &next = x[(i & 1) ^ 1];
        const float *f = i == 0 ? factor : nullptr;
        slz_gemm p = orth_product(now, now, P.pieces, P.gram, P.m, P.m, P.n);
        int rc;
        if (P.gram.split == 1) {
            p.symmetric = 1;
            rc = orth_run<false>(p, orth_symmetric_epi<orth_gram>{a, da, {f}}, P.gram, sh->batch, s);
        } else {
            const uint32_t ld = slz_ranges_ld(P.m);
            p.split = P.gram.split;
            rc = orth_run<false>(p, slz_partial_epi<float>{(float *)(w + P.ranges), ld, sh->batch, 0}, P.gram, sh->batch, s);
            hipLaunchKernelGGL(k_orth_gram_join, dim3((P.m + 1030) / 1024, P.m, sh->batch), dim3(256), 0, s, (const float *)(w + P.ranges), P.gram.split, sh->batch,
                               P.m, ld, orth_gram{f}, a, da);
        }
        if (rc != SLZ_OK) return rc;
        p = orth_product(a, a, P.pieces, P.polynomial, P.m, P.m, P.m);
        p.symmetric = 1;
        rc = orth_run<false>(p, orth_symmetric_epi<orth_polynomial>{b, db, {a, da, P.m, sh->a, sh->b, sh->c}}, P.polynomial, sh->batch, s);
        if (rc != SLZ_OK) return rc;
        p = orth_product(b, now, P.pieces, P.apply, P.m, P.n, P.m);
        const orth_apply_epi epi{now, next, db, f, i + 1 == sh->steps ? out : nullptr, sh->type, tall, aligned, sh->ld_out, sh->stride_out};
        rc = orth_run<true>(p, epi, P.apply, sh->batch, s);
        if (rc != SLZ_OK) return rc;
    }
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
