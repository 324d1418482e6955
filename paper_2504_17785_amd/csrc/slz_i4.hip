// Layers whose weights have 4 bits (include/silenzio_clear.h): quantisation by groups, the values, the product and its gradient.
//
// A word of a 4-bit row has eight consecutive entries, which is what a lane feeds to a matrix instruction, and a block of 128 entries lies so that the
// four words that a lane needs for the block's four instructions are 16 bytes in a row.
#include "slz_gemm.h"

#define I4_BLOCK 128u                // entries of a block, 64 bytes
static inline uint32_t i4_blocks(uint32_t cols) { return (cols + I4_BLOCK - 1) / I4_BLOCK; }
static inline uint32_t i4_groups(uint32_t cols, uint32_t group) { return (cols + group - 1) / group; }

// entries e of a word, in the order of k: a sign and a magnitude
__device__ __forceinline__ float i4_entry(uint32_t word, int e) {
    const uint32_t code = word >> (8 * (e & 3) + 4 * (e >> 2));
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, (float)(code & 7u)) | (code & 8u) << 28);
}
// place of the word with the entries 8 i to 8 i + 7 of a row
__device__ __forceinline__ uint32_t i4_place(uint32_t i) { return (i & ~15u) + (i & 3u) * 4u + (i >> 2 & 3u); }

// ---- quantisation ------------------------------------------------------------------------------------------------------------------
// The whole number next to 7 a / top for 0 <= a <= top, ties to even.  A quotient in 32 bits decides wrongly where it is next to a half, and in 16-bit
// types exact halves are common; so it is compared exactly, 14 a against (2 q - 1) top and (2 q + 1) top: those have 11 + 4 bits for 16-bit types, and
// 24 + 4 bits for f32, compared in 64.
template <int TYPE> __device__ __forceinline__ uint32_t i4_nearest(float a, float top, float inv) {
    using wide = typename std::conditional<TYPE == SLZ_F32, double, float>::type;
    const float q = fminf(rintf(a * inv), 7.0f);
    const uint32_t n = (uint32_t)q;
    const wide at = (wide)a * 14, half = top;
    wide off;                                          // exact: 14 a and 2 q top are within a factor of 64 of each other where q > 0
    if constexpr (TYPE == SLZ_F32) off = __builtin_fma(half, (double)(-2.0f * q), at);
    else off = __builtin_fmaf(half, -2.0f * q, at);
    const bool odd = n & 1u;
    const bool up = off > half || (off == half && odd), down = -off > half || (-off == half && odd);
    return n + (up ? 1u : 0u) - (down ? 1u : 0u);
}
// A thread makes a word, a group is 4, 8 or 16 lanes.  Bound by memory.
template <int TYPE>
__global__ void __launch_bounds__(256)
k_quantize_i4(const void *__restrict__ w, uint32_t rows, uint32_t cols, int64_t ld_w, uint32_t group, char *__restrict__ q, int64_t ld_q, float *__restrict__ scale,
              int64_t ld_scale) {
    const uint32_t per_row = (cols + I4_BLOCK - 1) / I4_BLOCK * 16u;
    const size_t total = (size_t)rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {             // a block's 16 lanes together
        uint32_t i;
        const size_t r = slz_divide(g, per_row, total <= 0xffffffffu, i);
        const uint32_t c = i * 8u;
        float v[8], top = 0.0f;
        row8_values<TYPE>(row8_load<TYPE>(w, r * ld_w, c, cols), c, cols, v);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float a = fabsf(v[e]);
            top = a < __builtin_inff() ? fmaxf(top, a) : __builtin_inff();
        }
        top = slz_dpp_max<0x4e>(slz_dpp_max<0xb1>(top));
        if (group > 32) top = slz_dpp_max<0x141>(top);
        if (group > 64) top = slz_dpp_max<0x140>(top);
        const bool finite = top < __builtin_inff();
        // held where neither 14 a nor 1 / top leaves 32 bits
        const float by = top < 0x1p-100f ? 0x1p100f : top > 0x1p100f ? 0x1p-100f : 1.0f, t = top * by, inv = t > 0.0f ? 7.0f / t : 0.0f;
        uint32_t word = 0;
        if (finite)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const uint32_t n = t > 0.0f ? i4_nearest<TYPE>(fabsf(v[e]) * by, t, inv) : 0u;
                word |= (n | (v[e] < 0.0f && n ? 8u : 0u)) << (8 * (e & 3) + 4 * (e >> 2));
            }
        *(uint32_t *)(q + r * ld_q + i4_place(i) * 4u) = word;
        if ((c & (group - 1u)) == 0 && c < cols) scale[r * ld_scale + c / group] = finite ? top / 7.0f : __builtin_nanf("");
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
    hipLaunchKernelGGL(k, ew_grid((size_t)rows * i4_blocks(cols) * 16u), dim3(256), 0, (hipStream_t)stream, w, rows, cols, ld_w, group, (char *)q, ld_q, scale, ld_scale);
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- values ------------------------------------------------------------------------------------------------------------------------
// Eight values of a row, zeros past its end
__device__ __forceinline__ void i4_values(const char *q, const float *scale, size_t r, uint32_t i, uint32_t cols, int64_t ld_q, int64_t ld_scale, uint32_t group,
                                          float (&v)[8]) {
    const uint32_t c = i * 8u;
    const uint32_t word = *(const uint32_t *)(q + r * ld_q + i4_place(i) * 4u);
    const float sc = scale[r * ld_scale + c / group];
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = c + e < cols ? i4_entry(word, e) * sc : 0.0f;
}
// Bound by memory.
__global__ void __launch_bounds__(256)
k_values_i4(const char *__restrict__ q, int64_t ld_q, const float *__restrict__ scale, int64_t ld_scale, uint32_t group, uint32_t rows, uint32_t cols, char *__restrict__ out,
            int type, int64_t ld_out, uint32_t aligned) {
    const uint32_t per_row = (cols + 7u) / 8u;
    const size_t total = (size_t)rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        uint32_t i;
        const size_t r = slz_divide(g, per_row, total <= 0xffffffffu, i);
        float v[8];
        i4_values(q, scale, r, i, cols, ld_q, ld_scale, group, v);
        slz_put_run<8>(out + (r * ld_out + i * 8u) * slz_type_bytes(type), type, v, cols - i * 8u, aligned);
    }
}

extern "C" int slz_values_i4(const uint8_t *q, int64_t ld_q, const float *scale, int64_t ld_scale, uint32_t group, uint32_t rows, uint32_t cols, void *out, int type,
                             int64_t ld_out, void *stream) {
    if (!slz_type_ok(type)) return SLZ_E_INVALID_ARG;
    int rc = i4_check(q, ld_q, scale, ld_scale, rows, cols, group);
    if (rc == SLZ_OK) rc = slz_matrix_check(out, rows, cols, ld_out, slz_type_bytes(type));
    if (rc != SLZ_OK || rows == 0 || cols == 0) return rc;
    hipLaunchKernelGGL(k_values_i4, ew_grid((size_t)rows * ((cols + 7u) / 8u)), dim3(256), 0, (hipStream_t)stream, (const char *)q, ld_q, scale, ld_scale, group, rows, cols,
                       (char *)out, type, ld_out, slz_in_place(out, 16, ld_out, slz_type_bytes(type)) ? 1u : 0u);
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- values as an operand ------------------------------------------------------------------------------------------------------------
// f16 could not hold small scales, so its values are held times VALUES_UP / unit, the power of two above the largest finite scale: magnitudes of up to
// 7 2^12 are below f16's largest, and rows whose scale is down to 2^-26 of the largest keep 11 bits.
#define VALUES_UP 4096.0f
#define VALUES_TOPS 256u             // workgroups that look for the largest scale
__global__ void __launch_bounds__(256) k_scale_tops(const float *__restrict__ scale, int64_t ld_scale, uint32_t rows, uint32_t groups, float *__restrict__ tops) {
    const size_t total = (size_t)rows * groups;
    float top = 0.0f;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        uint32_t c;
        const size_t r = slz_divide(g, groups, total <= 0xffffffffu, c);
        const float a = fabsf(scale[r * ld_scale + c]);
        if (a < __builtin_inff()) top = fmaxf(top, a);
    }
    top = slz_wave_max(top);
    __shared__ float of_wave[4];
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) tops[blockIdx.x] = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
}
// tops: of `count` workgroups, or null where values are held as they are; the first workgroup writes the unit
template <int TYPE>
__global__ void __launch_bounds__(256)
k_values_operand(const char *__restrict__ q, int64_t ld_q, const float *__restrict__ scale, int64_t ld_scale, uint32_t group, uint32_t rows, uint32_t cols,
                 const float *__restrict__ tops, uint32_t count, float *__restrict__ unit, char *__restrict__ out, uint32_t ld_out, int64_t piece) {
    constexpr int PIECES = TYPE == SLZ_F32 ? 3 : 1;
    float by = 1.0f;
    if constexpr (TYPE == SLZ_F16) {
        __shared__ float of_wave[4];
        float top = slz_wave_max(threadIdx.x < count ? tops[threadIdx.x] : 0.0f);
        if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
        int e = 0;
        if (top > 0.0f) frexpf(top, &e);
        const float u = ldexpf(1.0f, e < -100 ? -100 : e > 100 ? 100 : e);
        if (blockIdx.x == 0 && threadIdx.x == 0) *unit = u;
        by = VALUES_UP / u;
    }
    const uint32_t per_row = ld_out / 16u;
    const size_t total = (size_t)rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        uint32_t i;
        const size_t r = slz_divide(g, per_row, total <= 0xffffffffu, i);
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (i * 8u < cols) i4_values(q, scale, r, i, cols, ld_q, ld_scale, group, v);
        uint16_t t[PIECES][8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            if constexpr (TYPE == SLZ_F32) {
                uint16_t u[3];
                slz_split3(v[e], u);
                for (int k = 0; k < 3; k++) t[k][e] = u[k];
            } else t[0][e] = slz_half(v[e] * by, TYPE);
        }
#pragma unroll
        for (int k = 0; k < PIECES; k++) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = t[k][2 * e] | ((uint32_t)t[k][2 * e + 1] << 16);
            *(uint4 *)(out + k * piece + r * ld_out + (size_t)i * 16u) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}
// bytes of the values of `rows` x `cols` as an operand, and of the unit with what it is made from
static uint32_t values_row(uint32_t cols) { return (uint32_t)(((size_t)cols * 2 + 127) / 128 * 128); }
static size_t values_bytes(int type, uint32_t rows, uint32_t cols) { return (type == SLZ_F32 ? 3 : 1) * up256((size_t)rows * values_row(cols)) + 256 + VALUES_TOPS * 4; }
struct i4_rows { const uint8_t *q; int64_t ld_q; const float *scale; int64_t ld_scale; uint32_t group, rows, cols; };
static slz_operand values_operand(const i4_rows &w, int type, char *ws, float **unit, hipStream_t s) {
    const uint32_t row = values_row(w.cols);
    const size_t piece = up256((size_t)w.rows * row);
    const slz_operand o{ws, (int64_t)row, type == SLZ_F32 ? (int64_t)piece : 0, type == SLZ_F32 ? 3u : 1u, type == SLZ_F16 ? SLZ_F16 : SLZ_BF16};
    *unit = nullptr;
    if (w.rows == 0 || w.cols == 0) return o;
    float *at = (float *)(ws + o.pieces * piece), *tops = at + 64;
    uint32_t count = 0;
    if (type == SLZ_F16) {
        const size_t scales = (size_t)w.rows * i4_groups(w.cols, w.group);
        count = scales < (size_t)VALUES_TOPS * 256 ? (uint32_t)((scales + 255) / 256) : VALUES_TOPS;
        hipLaunchKernelGGL(k_scale_tops, dim3(count), dim3(256), 0, s, w.scale, w.ld_scale, w.rows, i4_groups(w.cols, w.group), tops);
        *unit = at;
    }
    const auto k = type == SLZ_F32 ? k_values_operand<SLZ_F32> : type == SLZ_BF16 ? k_values_operand<SLZ_BF16> : k_values_operand<SLZ_F16>;
    hipLaunchKernelGGL(k, ew_grid((size_t)w.rows * (row / 16u)), dim3(256), 0, s, (const char *)w.q, w.ld_q, w.scale, w.ld_scale, w.group, w.rows, w.cols, tops, count, at, ws, row,
                       (int64_t)piece);
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

struct linear_plan { size_t x, ranges, total; slz_choice c; };
static linear_plan plan_linear(const slz_i4_shape *sh, const void *x) {
    linear_plan P;
    P.c = slz_choose(sh->m, sh->n, (sh->k + 63) / 64 * pairs_of(sh->type), 1, false, 16);
    P.x = values_bytes(sh->type, sh->n, sh->k);
    P.ranges = P.x + slz_operand_bytes(x, sh->type, sh->m, sh->k, sh->ld_x);
    P.total = P.ranges + slz_ranges_bytes(P.c, sh->m, sh->n);
    return P;
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
    char *at = (char *)ws;
    slz_layouts jobs = {};
    const slz_operand a = slz_operand_of(x, sh->type, sh->m, sh->k, sh->ld_x, at + P.x, jobs);
    slz_layout_run(jobs, s);
    float *unit;
    const slz_operand b = values_operand(weights_of(sh, q, scale), sh->type, at, &unit, s);
    const slz_gemm p = slz_gemm_of(a, b, sh->m, sh->n, sh->k);
    const slz_times_unit f{unit, 1.0f / VALUES_UP};
    rc = sh->type == SLZ_F16 ? slz_gemm_to<SLZ_EL_F16, false, false>(p, P.c, f, y, sh->type, sh->ld_y, at + P.ranges, s)
                             : slz_gemm_to<SLZ_EL_BF16, false, false>(p, P.c, f, y, sh->type, sh->ld_y, at + P.ranges, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

// ---- gradient ------------------------------------------------------------------------------------------------------------------------
struct i4_grad_plan { size_t dy, x, values, ranges, total; slz_choice dx, dw; };
static i4_grad_plan plan_i4_grad(const slz_i4_shape *sh, const void *dy, const void *x) {
    i4_grad_plan P;
    const uint32_t pairs = pairs_of(sh->type);
    P.dx = slz_choose(sh->m, sh->k, (sh->n + 63) / 64 * pairs, 1, false, 16, true);
    P.dw = slz_choose(sh->n, sh->k, (sh->m + 63) / 64 * pairs, 1, false, 16, true);
    P.dy = 0;
    P.x = slz_operand_bytes(dy, sh->type, sh->m, sh->n, sh->ld_y);
    P.values = P.x + slz_operand_bytes(x, sh->type, sh->m, sh->k, sh->ld_x);
    P.ranges = P.values + values_bytes(sh->type, sh->n, sh->k);
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
        const slz_operand w = values_operand(weights_of(sh, q, scale), sh->type, at + P.values, &unit, s);
        rc = slz_float_product(d, false, w, sh->m, sh->k, sh->n, P.dx, unit, 1.0f / VALUES_UP, dx, sh->type, ld_dx, at + P.ranges, s);
    }
    if (rc == SLZ_OK && dw && sh->n) rc = slz_float_product(d, true, b, sh->n, sh->k, sh->m, P.dw, nullptr, 1.0f, dw, sh->type, ld_dw, at + P.ranges, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
