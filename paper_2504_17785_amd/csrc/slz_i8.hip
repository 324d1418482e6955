// Products of 8-bit integers with a scale per row (include/silenzio_clear.h): quantisation, the product, its gradient.
#include "slz_gemm.h"

// ---- quantisation ------------------------------------------------------------------------------------------------------------------
// One workgroup per row: its largest magnitude, then its entries, read again from the cache.
// A row whose largest entry is below 2^-100 is moved up by 2^100 first, so that 127 / top stays finite.
__device__ __forceinline__ float quantize_scale(float top, bool finite, float &up, float &inv) {
    up = top < 0x1p-100f ? 0x1p100f : 1.0f;
    const float t = top * up;
    inv = finite && t > 0.0f ? 127.0f / t : 0.0f;
    return finite ? t / 127.0f / up : __builtin_nanf("");
}
__device__ __forceinline__ int8_t quantize_one(float x, float up, float inv) {
    return (int8_t)(int)fminf(fmaxf(rintf(x * up * inv), -127.0f), 127.0f);
}

__global__ void __launch_bounds__(256)
k_quantize(const void *__restrict__ x, int type, uint32_t cols, int64_t ld_x, int8_t *__restrict__ q, int64_t ld_q, float *__restrict__ scale) {
    const size_t row = blockIdx.x;
    __shared__ float tops[4];
    __shared__ int bad[4];
    float top = 0.0f;
    bool odd = false;
    for (uint32_t c = threadIdx.x; c < cols; c += 256) {
        const float v = fabsf(slz_get(x, type, row * ld_x + c));
        odd |= !(v < __builtin_inff());
        top = fmaxf(top, v);
    }
    top = slz_wave_max(top);
    const bool any = __any(odd);
    if ((threadIdx.x & 63) == 0) { tops[threadIdx.x >> 6] = top; bad[threadIdx.x >> 6] = any; }
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const bool finite = !(bad[0] | bad[1] | bad[2] | bad[3]);
    float up, inv;
    const float sc = quantize_scale(top, finite, up, inv);
    if (threadIdx.x == 0) scale[row] = sc;
    for (uint32_t c = threadIdx.x; c < cols; c += 256) q[row * ld_q + c] = finite ? quantize_one(slz_get(x, type, row * ld_x + c), up, inv) : (int8_t)0;
}

extern "C" int slz_quantize_i8(const void *x, int type, uint32_t rows, uint32_t cols, int64_t ld_x, int8_t *q, int64_t ld_q, float *scale, void *stream) {
    if (!slz_type_ok(type)) return SLZ_E_INVALID_ARG;
    int rc = slz_matrix_check(x, rows, cols, ld_x, slz_type_bytes(type));
    if (rc == SLZ_OK) rc = slz_matrix_check(q, rows, cols, ld_q, 1);
    if (rc == SLZ_OK) rc = slz_matrix_check(scale, rows, 1, 1, 4);
    if (rc != SLZ_OK || rows == 0) return rc;
    hipLaunchKernelGGL(k_quantize, dim3(rows), dim3(256), 0, (hipStream_t)stream, x, type, cols, ld_x, q, ld_q, scale);
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- product ---------------------------------------------------------------------------------------------------------------------------
struct scales_of {
    const float *a, *b;
    __device__ __forceinline__ float operator()(uint32_t, uint32_t m, uint32_t n, int sum) const { return (float)sum * (a[m] * b[n]); }
};

static int i8_check(const slz_i8_shape *sh) {
    if (!sh || !slz_type_ok(sh->type)) return SLZ_E_INVALID_ARG;
    if (sh->m > SLZ_CLEAR_MAX_LEN || sh->n > SLZ_CLEAR_MAX_LEN || sh->k >= (1u << 17)) return SLZ_E_TOO_LARGE;
    return SLZ_OK;
}

static slz_choice i8_choice(const slz_i8_shape *sh) { return slz_choose(sh->m, sh->n, (sh->k + 127) / 128, 1, false, 16); }
static int i8_product(const slz_i8_shape *sh, const slz_operand &a, const float *sa, const slz_operand &b, const float *sb, void *y, char *ranges, hipStream_t s) {
    return slz_gemm_to<SLZ_EL_I8, false, false>(slz_gemm_of(a, b, sh->m, sh->n, sh->k), i8_choice(sh), scales_of{sa, sb}, y, sh->type, sh->ld_y, ranges, s);
}

extern "C" int slz_matmul_i8_workspace(const slz_i8_shape *sh, const int8_t *a, const int8_t *b, size_t *bytes) {
    const int rc = i8_check(sh);
    if (rc != SLZ_OK) return rc;
    if (!bytes) return SLZ_E_INVALID_ARG;
    *bytes = slz_operand_i8_bytes(a, sh->m, sh->k, sh->ld_a) + slz_operand_i8_bytes(b, sh->n, sh->k, sh->ld_b) + slz_ranges_bytes(i8_choice(sh), sh->m, sh->n);
    return SLZ_OK;
}

static int i8_checks(const slz_i8_shape *sh, const void *a, uint32_t a_bytes, const int8_t *b, const float *sb, const void *y) {
    int rc = i8_check(sh);
    if (rc == SLZ_OK) rc = slz_matrix_check(a, sh->m, sh->k, sh->ld_a, a_bytes);
    if (rc == SLZ_OK) rc = slz_matrix_check(b, sh->n, sh->k, sh->ld_b, 1);
    if (rc == SLZ_OK) rc = slz_matrix_check(y, sh->m, sh->n, sh->ld_y, slz_type_bytes(sh->type));
    if (rc == SLZ_OK) rc = slz_matrix_check(sb, sh->n, 1, 1, 4);
    return rc;
}

extern "C" int slz_matmul_i8(const slz_i8_shape *sh, const int8_t *a, const float *sa, const int8_t *b, const float *sb, void *y, void *ws,
                             size_t ws_bytes, void *stream) {
    int rc = i8_checks(sh, a, 1, b, sb, y);
    if (rc == SLZ_OK) rc = slz_matrix_check(sa, sh->m, 1, 1, 4);
    if (rc != SLZ_OK || sh->m == 0 || sh->n == 0) return rc;
    const size_t for_a = slz_operand_i8_bytes(a, sh->m, sh->k, sh->ld_a), for_b = slz_operand_i8_bytes(b, sh->n, sh->k, sh->ld_b);
    if (!slz_ws_ok(ws, ws_bytes, for_a + for_b + slz_ranges_bytes(i8_choice(sh), sh->m, sh->n))) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    const slz_operand oa = slz_operand_i8_of(a, sh->m, sh->k, sh->ld_a, (char *)ws, s);
    const slz_operand ob = slz_operand_i8_of(b, sh->n, sh->k, sh->ld_b, (char *)ws + for_a, s);
    rc = i8_product(sh, oa, sa, ob, sb, y, (char *)ws + for_a + for_b, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- a layer: quantised rows of x times the weights -----------------------------------------------------------------------------------
struct linear_plan { size_t q, scale, b, ranges, total; int64_t ld_q; };
static linear_plan plan_linear(const slz_i8_shape *sh, const int8_t *b) {
    linear_plan P;
    P.ld_q = ((int64_t)sh->k + 127) / 128 * 128;
    P.q = 0;
    P.scale = up256((size_t)sh->m * P.ld_q);
    P.b = P.scale + up256((size_t)sh->m * 4);
    P.ranges = P.b + slz_operand_i8_bytes(b, sh->n, sh->k, sh->ld_b);
    P.total = P.ranges + slz_ranges_bytes(i8_choice(sh), sh->m, sh->n);
    return P;
}
extern "C" int slz_linear_i8_workspace(const slz_i8_shape *sh, const void *x, const int8_t *b, size_t *bytes) {
    const int rc = i8_check(sh);
    if (rc != SLZ_OK) return rc;
    (void)x;
    if (!bytes) return SLZ_E_INVALID_ARG;
    *bytes = plan_linear(sh, b).total;
    return SLZ_OK;
}
extern "C" int slz_linear_i8(const slz_i8_shape *sh, const void *x, const int8_t *b, const float *sb, void *y, void *ws, size_t ws_bytes, void *stream) {
    int rc = sh && slz_type_ok(sh->type) ? i8_checks(sh, x, slz_type_bytes(sh->type), b, sb, y) : SLZ_E_INVALID_ARG;
    if (rc != SLZ_OK || sh->m == 0 || sh->n == 0) return rc;
    const linear_plan P = plan_linear(sh, b);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    int8_t *q = (int8_t *)ws + P.q;
    float *sa = (float *)((char *)ws + P.scale);
    // a row's last 16 entries may end with whatever was there: b's are zero in those places
    rc = slz_quantize_i8(x, sh->type, sh->m, sh->k, sh->ld_a, q, P.ld_q, sa, stream);
    if (rc != SLZ_OK) return rc;
    const slz_operand oa{(const char *)q, P.ld_q, 0, 1, 3};
    const slz_operand ob = slz_operand_i8_of(b, sh->n, sh->k, sh->ld_b, (char *)ws + P.b, s);
    return i8_product(sh, oa, sa, ob, sb, y, (char *)ws + P.ranges, s);
}

// ---- gradient ------------------------------------------------------------------------------------------------------------------------------
// dy times the values scale_r q_rc: these are laid out as an operand once (bf16, or three bf16 for f32), then two ordinary products.  f16 could
// not hold small scales, so its values are divided by `unit`, the power of two at or above the largest scale, and the sums multiplied by it.
// eight values of a row per thread
__global__ void __launch_bounds__(256)
k_values(const int8_t *__restrict__ q, const float *__restrict__ scale, const float *__restrict__ unit, int type, uint32_t rows, uint32_t cols, int64_t ld_q,
         char *__restrict__ out, uint32_t ld_out, int64_t piece) {
    const uint32_t per_row = ld_out / 16u;
    const size_t total = (size_t)rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        const size_t r = g / per_row;
        const uint32_t c = (uint32_t)(g % per_row) * 8;
        const float sc = type == SLZ_F16 ? scale[r] / *unit : scale[r];
        uint16_t t[3][8];
        for (int i = 0; i < 8; i++) {
            const float v = c + i < cols ? (float)q[r * ld_q + c + i] * sc : 0.0f;
            if (type == SLZ_F32) {
                uint16_t u[3];
                slz_split3(v, u);
                t[0][i] = u[0]; t[1][i] = u[1]; t[2][i] = u[2];
            } else t[0][i] = slz_half(v, type);
        }
        for (int k = 0; k < (type == SLZ_F32 ? 3 : 1); k++) {
            uint32_t w[4];
            for (int i = 0; i < 4; i++) w[i] = t[k][2 * i] | ((uint32_t)t[k][2 * i + 1] << 16);
            *(uint4 *)(out + k * piece + r * ld_out + (size_t)c * 2) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

struct grad_plan { size_t dy, values[2], unit, ranges, total; uint32_t row; slz_choice da, db; };
static grad_plan plan_grad(const slz_i8_shape *sh, const void *dy) {
    grad_plan P;
    const size_t pieces = sh->type == SLZ_F32 ? 3 : 1;
    P.row = (uint32_t)(((size_t)sh->k * 2 + 127) / 128 * 128);
    P.dy = 0;
    P.values[0] = slz_operand_bytes(dy, sh->type, sh->m, sh->n, sh->ld_y);
    P.values[1] = P.values[0] + pieces * up256((size_t)sh->m * P.row);
    P.unit = P.values[1] + pieces * up256((size_t)sh->n * P.row);
    P.ranges = P.unit + 256;
    const uint32_t pairs = sh->type == SLZ_F32 ? 6 : 1;
    P.da = slz_choose(sh->m, sh->k, (sh->n + 63) / 64 * pairs, 1, false, 16);
    P.db = slz_choose(sh->n, sh->k, (sh->m + 63) / 64 * pairs, 1, false, 16);
    const size_t for_a = slz_ranges_bytes(P.da, sh->m, sh->k), for_b = slz_ranges_bytes(P.db, sh->n, sh->k);
    P.total = P.ranges + (for_a > for_b ? for_a : for_b);
    return P;
}
extern "C" int slz_matmul_i8_grad_workspace(const slz_i8_shape *sh, const void *dy, size_t *bytes) {
    const int rc = i8_check(sh);
    if (rc != SLZ_OK) return rc;
    if (!bytes) return SLZ_E_INVALID_ARG;
    *bytes = plan_grad(sh, dy).total;
    return SLZ_OK;
}

// out [M][k] = left times the values of q [rows][k]; left's rows are the sum's index where left_rows_k
static int grad_product(const slz_i8_shape *sh, const slz_operand &left, bool left_rows_k, uint32_t M, const int8_t *q, int64_t ld_q, const float *scale,
                        uint32_t rows, void *out, int64_t ld_out, char *values, float *unit, char *ranges, const grad_plan &P, hipStream_t s) {
    const int type = sh->type;
    const slz_operand right{values, (int64_t)P.row, (int64_t)up256((size_t)rows * P.row), left.pieces, left.element};
    if (type == SLZ_F16) slz_unit_of(scale, rows, unit, s);
    if (rows)
        hipLaunchKernelGGL(k_values, ew_grid((size_t)rows * P.row / 16), dim3(256), 0, s, q, scale, unit, type, rows, sh->k, ld_q, values, P.row, right.piece);
    const slz_gemm p = slz_gemm_of(left, right, M, sh->k, rows);
    const slz_times_unit f{type == SLZ_F16 ? unit : nullptr, 1.0f};
    if (type == SLZ_F16)
        return left_rows_k ? slz_gemm_to<SLZ_EL_F16, true, true>(p, P.db, f, out, type, ld_out, ranges, s)
                           : slz_gemm_to<SLZ_EL_F16, false, true>(p, P.da, f, out, type, ld_out, ranges, s);
    return left_rows_k ? slz_gemm_to<SLZ_EL_BF16, true, true>(p, P.db, f, out, type, ld_out, ranges, s)
                       : slz_gemm_to<SLZ_EL_BF16, false, true>(p, P.da, f, out, type, ld_out, ranges, s);
}

extern "C" int slz_matmul_i8_grad(const slz_i8_shape *sh, const void *dy, const int8_t *a, const float *sa, const int8_t *b, const float *sb, void *da,
                                  int64_t ld_da, void *db, int64_t ld_db, void *ws, size_t ws_bytes, void *stream) {
    int rc = sh && slz_type_ok(sh->type) ? i8_checks(sh, a, 1, b, sb, dy) : SLZ_E_INVALID_ARG;
    if (rc == SLZ_OK) rc = slz_matrix_check(sa, sh->m, 1, 1, 4);
    if (rc == SLZ_OK && da) rc = slz_matrix_check(da, sh->m, sh->k, ld_da, slz_type_bytes(sh->type));
    if (rc == SLZ_OK && db) rc = slz_matrix_check(db, sh->n, sh->k, ld_db, slz_type_bytes(sh->type));
    if (rc != SLZ_OK || sh->k == 0) return rc;
    const grad_plan P = plan_grad(sh, dy);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    char *w = (char *)ws;
    const slz_operand d = slz_operand_of(dy, sh->type, sh->m, sh->n, sh->ld_y, w + P.dy, s);
    if (da && sh->m) rc = grad_product(sh, d, false, sh->m, b, sh->ld_b, sb, sh->n, da, ld_da, w + P.values[1], (float *)(w + P.unit), w + P.ranges, P, s);
    if (rc == SLZ_OK && db && sh->n) rc = grad_product(sh, d, true, sh->n, a, sh->ld_a, sa, sh->m, db, ld_db, w + P.values[0], (float *)(w + P.unit) + 1, w + P.ranges, P, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
