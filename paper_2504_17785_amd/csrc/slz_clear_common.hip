// Operands of the matrix product: laid out in 16-byte aligned rows where a caller's matrix cannot be read as it is, and numbers of 32 bits as
// three of bf16.
#include "slz_clear.h"

// rows x cols elements of SRC bytes, rows padded with zeros to ld_out bytes; one thread per 16 bytes of the result
template <int SRC>
__global__ void __launch_bounds__(256) k_align(const char *__restrict__ x, char *__restrict__ out, uint32_t rows, uint32_t cols, int64_t ld, uint32_t ld_out) {
    constexpr int C = 16 / SRC;
    const uint32_t per_row = ld_out / 16u;
    const size_t total = (size_t)rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        const size_t r = g / per_row;
        const uint32_t c = (uint32_t)(g % per_row) * C;
        union { uint8_t b[16]; uint16_t h[8]; uint4 v; } u;
        u.v = make_uint4(0, 0, 0, 0);
        for (int i = 0; i < C; i++)
            if (c + i < cols) {
                if (SRC == 1) u.b[i] = ((const uint8_t *)x)[r * ld + c + i];
                else u.h[i % 8] = ((const uint16_t *)x)[r * ld + c + i];
            }
        *(uint4 *)(out + r * ld_out + (size_t)c * SRC) = u.v;
    }
}
__global__ void __launch_bounds__(256) k_split3(const float *__restrict__ x, char *__restrict__ out, uint32_t rows, uint32_t cols, int64_t ld, uint32_t ld_out, int64_t piece) {
    const uint32_t per_row = ld_out / 16u;
    const size_t total = (size_t)rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        const size_t r = g / per_row;
        const uint32_t c = (uint32_t)(g % per_row) * 8;
        uint16_t q[3][8];
        for (int i = 0; i < 8; i++) {
            uint16_t t[3] = {0, 0, 0};
            if (c + i < cols) slz_split3(x[r * ld + c + i], t);
            for (int k = 0; k < 3; k++) q[k][i] = t[k];
        }
        for (int k = 0; k < 3; k++) {
            uint32_t w[4];
            for (int i = 0; i < 4; i++) w[i] = q[k][2 * i] | ((uint32_t)q[k][2 * i + 1] << 16);
            *(uint4 *)(out + k * piece + r * ld_out + (size_t)c * 2) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

static size_t row_bytes(uint32_t cols, uint32_t bytes) { return ((size_t)cols * bytes + 127) / 128 * 128; }

size_t slz_operand_bytes(const void *p, int type, uint32_t rows, uint32_t cols, int64_t ld) {
    if (type == SLZ_F32) return 3 * up256(rows * row_bytes(cols, 2));
    return slz_in_place(p, cols, ld, 2) ? 0 : up256(rows * row_bytes(cols, 2));
}
slz_operand slz_operand_of(const void *p, int type, uint32_t rows, uint32_t cols, int64_t ld, char *ws, hipStream_t s) {
    const int64_t row = row_bytes(cols, 2);
    if (type == SLZ_F32) {
        const slz_operand o{ws, row, (int64_t)up256(rows * row), 3, SLZ_BF16};
        if (rows && cols)
            hipLaunchKernelGGL(k_split3, ew_grid((size_t)rows * row / 16), dim3(256), 0, s, (const float *)p, ws, rows, cols, ld, (uint32_t)row, o.piece);
        return o;
    }
    if (slz_in_place(p, cols, ld, 2)) return {(const char *)p, ld * 2, 0, 1, type};
    if (rows && cols)
        hipLaunchKernelGGL(k_align<2>, ew_grid((size_t)rows * row / 16), dim3(256), 0, s, (const char *)p, ws, rows, cols, ld, (uint32_t)row);
    return {ws, row, 0, 1, type};
}
size_t slz_operand_i8_bytes(const int8_t *p, uint32_t rows, uint32_t cols, int64_t ld) {
    return slz_in_place(p, cols, ld, 1) ? 0 : up256(rows * row_bytes(cols, 1));
}
slz_operand slz_operand_i8_of(const int8_t *p, uint32_t rows, uint32_t cols, int64_t ld, char *ws, hipStream_t s) {
    if (slz_in_place(p, cols, ld, 1)) return {(const char *)p, ld, 0, 1, 3};
    const int64_t row = row_bytes(cols, 1);
    if (rows && cols)
        hipLaunchKernelGGL(k_align<1>, ew_grid((size_t)rows * row / 16), dim3(256), 0, s, (const char *)p, ws, rows, cols, ld, (uint32_t)row);
    return {ws, row, 0, 1, 3};
}

// One workgroup: the power of two at or above the largest of the magnitudes (1 where there is none that is finite)
__global__ void __launch_bounds__(256) k_scale_unit(const float *__restrict__ scale, uint32_t count, float *__restrict__ unit) {
    float top = 0.0f;
    for (uint32_t i = threadIdx.x; i < count; i += 256) top = fmaxf(top, fabsf(scale[i]));
    top = slz_wave_max(top);
    __shared__ float tops[4];
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        int e = 0;
        if (top > 0.0f && top < __builtin_inff()) frexpf(top, &e);
        *unit = ldexpf(1.0f, e < -120 ? -120 : e > 120 ? 120 : e);
    }
}

void slz_unit_of(const float *values, uint32_t count, float *unit, hipStream_t s) {
    hipLaunchKernelGGL(k_scale_unit, dim3(1), dim3(256), 0, s, values, count, unit);
}
