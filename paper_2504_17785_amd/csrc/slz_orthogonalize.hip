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
#define ORTH_NORM_BLOCKS 64

struct orth_view {                   // a batch of matrices of two f16 each
    uint16_t *hi, *lo;               // lo may be null
    uint32_t ld;
    size_t stride;                   // elements from matrix to matrix
};
__device__ __forceinline__ void orth_put(const orth_view &v, size_t at, float x) {
    const float u = x * ORTH_UP;
    const _Float16 h = (_Float16)u;
    v.hi[at] = __builtin_bit_cast(uint16_t, h);
    if (v.lo) v.lo[at] = slz_f32_to_f16(u - (float)h);
}
__device__ __forceinline__ float orth_get(const orth_view &v, size_t at) {
    const float h = slz_f16_to_f32(v.hi[at]);
    return (v.lo ? h + slz_f16_to_f32(v.lo[at]) : h) * (1.0f / ORTH_UP);
}

// ---- norm and first X -------------------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256)
k_orth_norm(const void *__restrict__ g, int type, uint32_t rows, uint32_t cols, int64_t ld, int64_t stride, double *__restrict__ part) {
    const size_t base = (size_t)blockIdx.y * stride;
    double sum = 0.0;
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        for (uint32_t c = threadIdx.x; c < cols; c += 256) {
            const double x = slz_get(g, type, base + (size_t)r * ld + c);
            sum += x * x;
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
    __shared__ double total;
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (uint32_t i = 0; i < parts; i++) s += part[blockIdx.z * ORTH_NORM_BLOCKS + i];
        total = sqrt(s) + (double)eps;
    }
    __syncthreads();
    const double norm = total;
    int e = 0;
    if (norm > 0.0 && norm < 1e300) frexp(norm, &e);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) factor[blockIdx.z] = (float)(ldexp(1.0, e) / norm);
    const uint32_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, t = threadIdx.x;
    const size_t base = (size_t)blockIdx.z * stride;
    for (uint32_t i = t; i < 4096; i += 256) {
        const uint32_t r = r0 + i / 64, c = c0 + i % 64;
        tile[i / 64][i % 64] = r < rows && c < cols ? ldexpf(slz_get(g, type, base + (size_t)r * ld + c), -e) : 0.0f;
    }
    __syncthreads();
    const uint32_t m = tall ? cols : rows, wide = ((tall ? rows : cols) + 7u) & ~7u;
    for (uint32_t i = t; i < 4096; i += 256) {
        const uint32_t a = i / 64, b = i % 64, r = (tall ? c0 : r0) + a, c = (tall ? r0 : c0) + b;
        if (r < m && c < wide) orth_put(x, blockIdx.z * x.stride + (size_t)r * x.ld + c, tall ? tile[b][a] : tile[a][b]);
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
// A symmetric product's result: `diagonal` apart, the rest to `out` with zeros on the diagonal and in the columns up to the next multiple of 8.
template <class F> struct orth_symmetric_epi {
    orth_view out;
    float *diagonal;                 // [batch][m]
    F f;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *) const {
        const uint32_t wide = (p.M + 7u) & ~7u;
        const size_t base = at.batch * out.stride;
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const uint32_t n = slz_col<NI, RUN>(at, j);
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const bool real = m < p.M && n + c < p.M;
                    float v = real ? f(at.batch, m, n + c, acc[i][j][c]) : 0.0f;
                    if (real && m == n + c) {
                        diagonal[at.batch * p.M + m] = f.finish(v);
                        v = 0.0f;
                    }
                    if (m < p.M && n + c < wide) orth_put(out, base + (size_t)m * out.ld + n + c, v);
                    if (at.tile_m != at.tile_n && n + c < p.M && m < wide) orth_put(out, base + (size_t)(n + c) * out.ld + m, v);
                }
            }
        }
    }
};
struct orth_gram {
    const float *factor;             // or null
    __device__ __forceinline__ float operator()(uint32_t batch, uint32_t, uint32_t, float sum) const {
        const float f = factor ? factor[batch] : 1.0f;
        return sum * (f * f / (ORTH_UP * ORTH_UP));
    }
    __device__ __forceinline__ float finish(float v) const { return v; }
};
struct orth_polynomial {
    orth_view o;
    const float *d;                  // of A
    uint32_t m_all;
    float a, b, c;
    __device__ __forceinline__ float operator()(uint32_t batch, uint32_t m, uint32_t n, float sum) const {
        const float x = orth_get(o, batch * o.stride + (size_t)m * o.ld + n), dm = d[batch * m_all + m], dn = d[batch * m_all + n];
        const float square = sum * (1.0f / (ORTH_UP * ORTH_UP)) + (dm + dn) * x + (m == n ? dm * dm : 0.0f);
        return b * (m == n ? dm : x) + c * square;
    }
    __device__ __forceinline__ float finish(float v) const { return a + v; }
};
struct orth_apply_epi {
    orth_view x, next;               // this step's X and the next one's
    const float *diagonal;           // a + B_ii
    const float *factor;             // or null
    void *out;                       // the last step's result goes here, or null
    int type, tall;
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
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    if (n + c >= wide) continue;
                    const size_t here = at.batch * x.stride + (size_t)m * x.ld + n + c;
                    const float v = n + c < p.N ? f * (d * orth_get(x, here) + acc[i][j][c] * (1.0f / (ORTH_UP * ORTH_UP))) : 0.0f;
                    if (!out) orth_put(next, here, v);
                    else if (n + c < p.N) slz_put(out, type, at.batch * stride_out + (tall ? (int64_t)(n + c) * ld_out + m : (int64_t)m * ld_out + n + c), v);
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
    const uint32_t parts = sh->rows < ORTH_NORM_BLOCKS ? sh->rows : ORTH_NORM_BLOCKS;
    hipLaunchKernelGGL(k_orth_norm, dim3(parts, sh->batch), dim3(256), 0, s, g, sh->type, sh->rows, sh->cols, sh->ld_g, sh->stride_g, part);
    hipLaunchKernelGGL(k_orth_load, dim3((sh->cols + 63) / 64, (sh->rows + 63) / 64, sh->batch), dim3(256), 0, s, g, sh->type, sh->rows, sh->cols, sh->ld_g,
                       sh->stride_g, tall, part, parts, sh->eps, x[0], factor);
    if (sh->steps == 0)
        hipLaunchKernelGGL(k_orth_store, dim3(1024, sh->batch), dim3(256), 0, s, x[0], factor, out, sh->type, sh->rows, sh->cols, sh->ld_out, sh->stride_out, tall);
    for (uint32_t i = 0; i < sh->steps; i++) {
        const orth_view &now = x[i & 1], &next = x[(i & 1) ^ 1];
        const float *f = i == 0 ? factor : nullptr;
        slz_gemm p = orth_product(now, now, P.pieces, P.m, P.m, P.n);
        p.symmetric = 1;
        int rc = slz_gemm_launch<slz_tiles_128, SLZ_EL_F16, false, false>(p, orth_symmetric_epi<orth_gram>{a, da, {f}}, sh->batch, s);
        if (rc != SLZ_OK) return rc;
        p = orth_product(a, a, P.pieces, P.m, P.m, P.m);
        p.symmetric = 1;
        rc = slz_gemm_launch<slz_tiles_128, SLZ_EL_F16, false, false>(p, orth_symmetric_epi<orth_polynomial>{b, db, {a, da, P.m, sh->a, sh->b, sh->c}}, sh->batch, s);
        if (rc != SLZ_OK) return rc;
        p = orth_product(b, now, P.pieces, P.m, P.n, P.m);
        const orth_apply_epi epi{now, next, db, f, i + 1 == sh->steps ? out : nullptr, sh->type, tall, sh->ld_out, sh->stride_out};
        rc = slz_gemm_launch<slz_tiles_128, SLZ_EL_F16, false, true>(p, epi, sh->batch, s);
        if (rc != SLZ_OK) return rc;
    }
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
