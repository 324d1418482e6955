// Updates orthogonalised by Newton-Schulz products (include/silenzio_clear.h):  X <- a X + (b A + c A A) X,  A = X X^T.
//
// The products run on f16 matrix instructions.  A step moves singular values near 1 little while it multiplies small ones by a, so what
// rounding adds to X itself grows by a^steps against it, and b A + c A A comes near -2.7 I, against which a X nearly cancels.  Hence
//   * X is held in two f16 (22 bits); a X and the diagonal's part of the product use both, the product's operand is the first;
//   * the diagonals of A and of B = b A + c A A are held in 32 bits apart, their f16 operands have zeros there:
//     A A = O O + (d_i + d_j) O_ij + d_i^2 [i = j]  with A = O + diag d,  and  X' = (a + B_ii) X + (B - diag) X.
// With the operands 8 times as precise as bf16's, and that, a result differs from the formula's by 2^-11 of its norm, a third of what rounding
// it to bf16 adds.  For f16 and f32 results O, B and X enter the products with both their halves (three products instead of one).
// The first X is g times a power of two, exact; what is missing to g / |g| is a factor of the first step.
// A and A A are symmetric: tiles on and below the diagonal are computed and stored twice.
#include "slz_gemm.h"

#define ORTH_UP 64.0f                // operands are held times this: the second halves stay out of the subnormal numbers
#define ORTH_NORM_BLOCKS 1024

struct orth_view {                   // a batch of matrices of two f16 each; rows of a multiple of 64 elements
    uint16_t *hi, *lo;               // lo may be null
    uint32_t ld;
    size_t stride;                   // elements from matrix to matrix
};
__device__ __forceinline__ uint32_t orth_pack(float a, float b) { return slz_f32_to_f16(a) | ((uint32_t)slz_f32_to_f16(b) << 16); }
// the two halves of ORTH_UP x
__device__ __forceinline__ void orth_halves(float x, float &hi, float &lo) {
    const float u = x * ORTH_UP;
    hi = (float)(_Float16)u;
    lo = u - hi;
}
// four in a row, at a multiple of four
__device__ __forceinline__ void orth_put4(const orth_view &v, size_t at, const float (&x)[4]) {
    float hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; i++) orth_halves(x[i], hi[i], lo[i]);
    *(uint2 *)(v.hi + at) = make_uint2(orth_pack(hi[0], hi[1]), orth_pack(hi[2], hi[3]));
    if (v.lo) *(uint2 *)(v.lo + at) = make_uint2(orth_pack(lo[0], lo[1]), orth_pack(lo[2], lo[3]));
}
__device__ __forceinline__ void orth_get4(const orth_view &v, size_t at, float (&x)[4]) {
    const uint2 h = *(const uint2 *)(v.hi + at);
    uint2 l = make_uint2(0, 0);
    if (v.lo) l = *(const uint2 *)(v.lo + at);
    const uint32_t hw[2] = {h.x, h.y}, lw[2] = {l.x, l.y};
#pragma unroll
    for (int i = 0; i < 4; i++)
        x[i] = (slz_f16_to_f32((uint16_t)(hw[i / 2] >> (16 * (i & 1)))) + slz_f16_to_f32((uint16_t)(lw[i / 2] >> (16 * (i & 1))))) * (1.0f / ORTH_UP);
}
__device__ __forceinline__ float orth_get(const orth_view &v, size_t at) {
    const float h = slz_f16_to_f32(v.hi[at]);
    return (v.lo ? h + slz_f16_to_f32(v.lo[at]) : h) * (1.0f / ORTH_UP);
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
__global__ void __launch_bounds__(256)
k_orth_load(const void *__restrict__ g, int type, uint32_t rows, uint32_t cols, int64_t ld, int64_t stride, int tall, const double *__restrict__ part,
            uint32_t parts, float eps, orth_view x, float *__restrict__ factor) {
    __shared__ float tile[64][65];
    const uint32_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, t = threadIdx.x;
    const size_t base = (size_t)blockIdx.z * stride;
    float own[16];
#pragma unroll
    for (int q = 0; q < 16; q++) {
        const uint32_t i = t + q * 256, r = r0 + i / 64, c = c0 + i % 64;
        own[q] = r < rows && c < cols ? slz_get(g, type, base + (size_t)r * ld + c) : 0.0f;
    }
    double sum = 0.0;
    for (uint32_t i = t & 63u; i < parts; i += 64) sum += part[blockIdx.z * ORTH_NORM_BLOCKS + i];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    const double norm = sqrt(sum) + (double)eps;
    int e = 0;
    if (norm > 0.0 && norm < 1e300) frexp(norm, &e);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) factor[blockIdx.z] = (float)(ldexp(1.0, e) / norm);
#pragma unroll
    for (int q = 0; q < 16; q++) tile[(t + q * 256) / 64][t % 64] = ldexpf(own[q], -e);
    __syncthreads();
    const uint32_t m = tall ? cols : rows, wide = ((tall ? rows : cols) + 7u) & ~7u;
    for (uint32_t i = t; i < 1024; i += 256) {
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
    orth_view out;
    float *diagonal;                 // [batch][m]
    F f;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *lds) const {
        // 2-byte words; the pitch keeps 16-byte alignment, and without the 8 the tile of 256 x 256 fills the shared memory of its operands
        constexpr uint32_t TM = WM * MI * 16, TN = WN * NI * 16, PITCH = TM + (TM < 256 ? 8 : 0);
        static_assert(TN * PITCH * 2 <= 2 * (TM + TN) * 128, "fits the operands' buffers");
        const uint32_t wide = (p.M + 7u) & ~7u, m0 = at.tile_m * TM, n0 = at.tile_n * TN;
        const size_t base = at.batch * out.stride;
        uint16_t *turned = (uint16_t *)lds;
        const int halves = out.lo && at.tile_m != at.tile_n ? 2 : 1;
        for (int half = 0; half < halves; half++) {
#pragma unroll
            for (int i = 0; i < MI; i++) {
                const uint32_t m = slz_row(at, i);
#pragma unroll
                for (int j = 0; j < NI; j++) {
                    const uint32_t n = slz_col<NI, RUN>(at, j);
                    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (m < p.M && n < p.M) f(at.batch, m, n, acc[i][j], v);
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        if (m < p.M && m == n + c) {
                            diagonal[at.batch * p.M + m] = f.finish(v[c]);
                            v[c] = 0.0f;
                        }
                        if (n + c >= p.M) v[c] = 0.0f;
                        float hi, lo;
                        orth_halves(v[c], hi, lo);
                        turned[(n - n0 + c) * PITCH + m - m0] = slz_f32_to_f16(half ? lo : hi);
                    }
                    if (half == 0 && m < p.M && n < wide) orth_put4(out, base + (size_t)m * out.ld + n, v);
                }
            }
            if (at.tile_m == at.tile_n) return;
            __syncthreads();
            uint16_t *to = (half ? out.lo : out.hi) + base;
            for (uint32_t g = threadIdx.x; g < TN * (TM / 8); g += WM * WN * 64) {
                const uint32_t n = g / (TM / 8), m = g % (TM / 8) * 8;
                if (n0 + n < p.M && m0 + m < wide) *(uint4 *)(to + (size_t)(n0 + n) * out.ld + m0 + m) = *(const uint4 *)(turned + n * PITCH + m);
            }
            __syncthreads();
        }
    }
};
struct orth_gram {
    const float *factor;             // or null
    __device__ __forceinline__ void operator()(uint32_t batch, uint32_t, uint32_t, const v4f &sum, float (&v)[4]) const {
        const float f = factor ? factor[batch] : 1.0f, by = f * f / (ORTH_UP * ORTH_UP);
#pragma unroll
        for (int c = 0; c < 4; c++) v[c] = sum[c] * by;
    }
    __device__ __forceinline__ float finish(float v) const { return v; }
};
struct orth_polynomial {
    orth_view o;
    const float *d;                  // of A
    uint32_t m_all;
    float a, b, c;
    __device__ __forceinline__ void operator()(uint32_t batch, uint32_t m, uint32_t n, const v4f &sum, float (&v)[4]) const {
        float x[4];
        orth_get4(o, batch * o.stride + (size_t)m * o.ld + n, x);
        const float dm = d[batch * m_all + m];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const bool on = m == n + q;
            const float dn = d[batch * m_all + min(n + q, m_all - 1)];
            const float square = sum[q] * (1.0f / (ORTH_UP * ORTH_UP)) + (dm + dn) * x[q] + (on ? dm * dm : 0.0f);
            v[q] = b * (on ? dm : x[q]) + c * square;
        }
    }
    __device__ __forceinline__ float finish(float v) const { return a + v; }
};
struct orth_apply_epi {
    static constexpr bool any_side = true;
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
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
            if (m >= p.M) continue;
            const float d = diagonal[at.batch * p.M + m];
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const uint32_t n = slz_col<NI, RUN>(at, j);
                if (n >= wide) continue;
                const size_t here = at.batch * x.stride + (size_t)m * x.ld + n;
                float old[4], v[4];
                orth_get4(x, here, old);
#pragma unroll
                for (int c = 0; c < 4; c++) v[c] = n + c < p.N ? f * (d * old[c] + acc[i][j][c] * (1.0f / (ORTH_UP * ORTH_UP))) : 0.0f;
                if (!out) orth_put4(next, here, v);
                else if (n < p.N) {
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

struct orth_plan {
    uint32_t m, n, pieces;
    uint32_t ld_x, ld_a;
    size_t one_x, one_a;             // bytes of a piece of X, of A or B
    size_t x[2], a, b, da, db, factor, part, total;
    uint32_t gram, polynomial, apply;                // sides of their tiles
};
static orth_plan plan_orth(const slz_orth_shape *sh) {
    orth_plan P;
    P.m = sh->rows < sh->cols ? sh->rows : sh->cols;
    P.n = sh->rows < sh->cols ? sh->cols : sh->rows;
    P.pieces = sh->type == SLZ_BF16 ? 1 : 2;
    P.ld_x = (P.n + 63) / 64 * 64;
    P.ld_a = (P.m + 63) / 64 * 64;
    P.one_x = up256((size_t)sh->batch * P.m * P.ld_x * 2);
    P.one_a = up256((size_t)sh->batch * P.m * P.ld_a * 2);
    size_t o = 0;
    for (int i = 0; i < 2; i++) { P.x[i] = o; o += 2 * P.one_x; }
    P.a = o; o += P.pieces * P.one_a;
    P.b = o; o += P.pieces * P.one_a;
    P.da = o; o += up256((size_t)sh->batch * P.m * 4);
    P.db = o; o += up256((size_t)sh->batch * P.m * 4);
    P.factor = o; o += up256((size_t)sh->batch * 4);
    P.part = o; o += up256((size_t)sh->batch * ORTH_NORM_BLOCKS * 8);
    P.total = o;
    const uint32_t pairs = P.pieces == 2 ? 3 : 1;
    P.gram = slz_choose(P.m, P.m, (P.n + 63) / 64 * pairs, sh->batch, true, 1).side;
    P.polynomial = slz_choose(P.m, P.m, (P.m + 63) / 64 * pairs, sh->batch, true, 1).side;
    P.apply = slz_choose(P.m, P.n, (P.m + 63) / 64 * pairs, sh->batch, false, 1).side;
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

// operands of one or two pieces; the pairs whose share of the sum is 2^-11 and more, the small ones first
static slz_gemm orth_product(const orth_view &a, const orth_view &b, uint32_t pieces, uint32_t M, uint32_t N, uint32_t K) {
    slz_gemm p = {};
    p.a = (const char *)a.hi; p.b = (const char *)b.hi;
    p.lda = (int64_t)a.ld * 2; p.ldb = (int64_t)b.ld * 2;
    p.a_batch = (int64_t)a.stride * 2; p.b_batch = (int64_t)b.stride * 2;
    p.M = M; p.N = N; p.K = K;
    p.split = 1;
    p.pairs = pieces == 2 ? 3 : 1;
    if (pieces == 2) {
        p.a_piece[0] = (const char *)a.lo - (const char *)a.hi;
        p.b_piece[1] = (const char *)b.lo - (const char *)b.hi;
    }
    return p;
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
    const int tall = sh->rows > sh->cols;
    const size_t xs = (size_t)P.m * P.ld_x, as = (size_t)P.m * P.ld_a;
    orth_view x[2], a, b;
    for (int i = 0; i < 2; i++) x[i] = {(uint16_t *)(w + P.x[i]), (uint16_t *)(w + P.x[i] + P.one_x), P.ld_x, xs};
    a = {(uint16_t *)(w + P.a), P.pieces == 2 ? (uint16_t *)(w + P.a + P.one_a) : nullptr, P.ld_a, as};
    b = {(uint16_t *)(w + P.b), P.pieces == 2 ? (uint16_t *)(w + P.b + P.one_a) : nullptr, P.ld_a, as};
    float *da = (float *)(w + P.da), *db = (float *)(w + P.db), *factor = (float *)(w + P.factor);
    double *part = (double *)(w + P.part);
    const uint32_t aligned = slz_in_place(out, 16, sh->ld_out, eb) && (sh->batch == 1 || sh->stride_out * eb % 16 == 0);
    const uint64_t needed = ((uint64_t)sh->rows * sh->cols + 8191) / 8192;
    const uint32_t parts = needed < ORTH_NORM_BLOCKS ? (uint32_t)needed : ORTH_NORM_BLOCKS;
    const auto norm = sh->type == SLZ_F32 ? k_orth_norm<SLZ_F32> : sh->type == SLZ_BF16 ? k_orth_norm<SLZ_BF16> : k_orth_norm<SLZ_F16>;
    hipLaunchKernelGGL(norm, dim3(parts, sh->batch), dim3(256), 0, s, g, sh->rows, sh->cols, sh->ld_g, sh->stride_g, part);
    hipLaunchKernelGGL(k_orth_load, dim3((sh->cols + 63) / 64, (sh->rows + 63) / 64, sh->batch), dim3(256), 0, s, g, sh->type, sh->rows, sh->cols, sh->ld_g,
                       sh->stride_g, tall, part, parts, sh->eps, x[0], factor);
    if (sh->steps == 0)
        hipLaunchKernelGGL(k_orth_store, dim3(1024, sh->batch), dim3(256), 0, s, x[0], factor, out, sh->type, sh->rows, sh->cols, sh->ld_out, sh->stride_out, tall);
    for (uint32_t i = 0; i < sh->steps; i++) {
        const orth_view &now = x[i & 1], &next = x[(i & 1) ^ 1];
        const float *f = i == 0 ? factor : nullptr;
        slz_gemm p = orth_product(now, now, P.pieces, P.m, P.m, P.n);
        p.symmetric = 1;
        int rc = slz_gemm_run<SLZ_EL_F16, false, false>(p, orth_symmetric_epi<orth_gram>{a, da, {f}}, P.gram, sh->batch, s);
        if (rc != SLZ_OK) return rc;
        p = orth_product(a, a, P.pieces, P.m, P.m, P.m);
        p.symmetric = 1;
        rc = slz_gemm_run<SLZ_EL_F16, false, false>(p, orth_symmetric_epi<orth_polynomial>{b, db, {a, da, P.m, sh->a, sh->b, sh->c}}, P.polynomial, sh->batch, s);
        if (rc != SLZ_OK) return rc;
        p = orth_product(b, now, P.pieces, P.m, P.n, P.m);
        const orth_apply_epi epi{now, next, db, f, i + 1 == sh->steps ? out : nullptr, sh->type, tall, aligned, sh->ld_out, sh->stride_out};
        rc = slz_gemm_run<SLZ_EL_F16, false, true>(p, epi, P.apply, sh->batch, s);
        if (rc != SLZ_OK) return rc;
    }
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
