// Operands of the matrix product: laid out in 16-byte aligned rows where a caller's matrix cannot be read as it is, and numbers of 32 bits as
// three of bf16.
#include "slz_clear.h"

// A thread makes 16 bytes of each piece of a job's result; jobs by grid y.
template <int SRC> __device__ __forceinline__ void align_16(const slz_layout &j, size_t r, uint32_t c, char *to) {
    constexpr uint32_t C = 16 / SRC;
    const char *from = j.x + ((int64_t)r * j.ld + c) * SRC;
    if (c + C <= j.cols) {
        *(v4i32 *)to = *(const v4i32_any *)from;
        return;
    }
    union { uint8_t b[16]; uint16_t h[8]; v4i32 v; } u;
    u.v = v4i32{0, 0, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < C; i++)
        if (c + i < j.cols) {
            if (SRC == 1) u.b[i] = ((const uint8_t *)from)[i];
            else u.h[i % 8] = ((const uint16_t *)from)[i];
        }
    *(v4i32 *)to = u.v;
}
// 777 x 1555 and 1001 x 1555 bytes (odd rows) in one launch: 5.3 us; in place where rows begin on 16 bytes
__global__ void __launch_bounds__(256) k_layout(const slz_layouts jobs) {
    const slz_layout j = jobs.job[blockIdx.y];
    const uint32_t per_row = j.ld_out / 16u;
    const size_t total = (size_t)j.rows * per_row;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        uint32_t at;
        const size_t r = slz_divide(g, per_row, total <= 0xffffffffu, at);
        at *= 16u;
        char *to = j.out + r * j.ld_out + at;
        if (j.bytes == 1) align_16<1>(j, r, at, to);
        else if (j.bytes == 2) align_16<2>(j, r, at / 2, to);
        else {
            uint32_t w[3][4];
            uint16_t t[2][3];
            float v[8];
            row8_values<SLZ_F32>(row8_load<SLZ_F32>(j.x, r * j.ld, at / 2, j.cols), at / 2, j.cols, v);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                slz_split3(v[i], t[i & 1]);
                if (i & 1)
                    for (int k = 0; k < 3; k++) w[k][i / 2] = t[0][k] | ((uint32_t)t[1][k] << 16);
            }
            for (int k = 0; k < 3; k++) *(uint4 *)(to + k * j.piece) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
        }
    }
}
void slz_layout_run(const slz_layouts &jobs, hipStream_t s) {
    size_t most = 0;
    for (uint32_t i = 0; i < jobs.count; i++) {
        const size_t n = (size_t)jobs.job[i].rows * (jobs.job[i].ld_out / 16u);
        most = n > most ? n : most;
    }
    if (most) hipLaunchKernelGGL(k_layout, dim3(ew_grid(most).x, jobs.count), dim3(256), 0, s, jobs);
}

static size_t row_bytes(uint32_t cols, uint32_t bytes) { return ((size_t)cols * bytes + 127) / 128 * 128; }
static void add(slz_layouts &jobs, const void *p, uint32_t rows, uint32_t cols, int64_t ld, uint32_t bytes, const slz_operand &o, char *ws) {
    if (rows && cols) jobs.job[jobs.count++] = {(const char *)p, ws, ld, o.piece, rows, cols, (uint32_t)o.ld, bytes};
}

size_t slz_operand_bytes(const void *p, int type, uint32_t rows, uint32_t cols, int64_t ld) {
    if (type == SLZ_F32) return 3 * up256(rows * row_bytes(cols, 2));
    return slz_in_place(p, cols, ld, 2) ? 0 : up256(rows * row_bytes(cols, 2));
}
slz_operand slz_operand_of(const void *p, int type, uint32_t rows, uint32_t cols, int64_t ld, char *ws, slz_layouts &jobs) {
    const int64_t row = row_bytes(cols, 2);
    if (type != SLZ_F32 && slz_in_place(p, cols, ld, 2)) return {(const char *)p, ld * 2, 0, 1, type};
    const slz_operand o = type == SLZ_F32 ? slz_operand{ws, row, (int64_t)up256(rows * row), 3, SLZ_BF16} : slz_operand{ws, row, 0, 1, type};
    add(jobs, p, rows, cols, ld, slz_type_bytes(type), o, ws);
    return o;
}
size_t slz_operand_i8_bytes(const int8_t *p, uint32_t rows, uint32_t cols, int64_t ld) {
    return slz_in_place(p, cols, ld, 1) ? 0 : up256(rows * row_bytes(cols, 1));
}
slz_operand slz_operand_i8_of(const int8_t *p, uint32_t rows, uint32_t cols, int64_t ld, char *ws, slz_layouts &jobs) {
    if (slz_in_place(p, cols, ld, 1)) return {(const char *)p, ld, 0, 1, 3};
    const slz_operand o{ws, (int64_t)row_bytes(cols, 1), 0, 1, 3};
    add(jobs, p, rows, cols, ld, 1, o, ws);
    return o;
}

// One workgroup
__global__ void __launch_bounds__(256)
k_scale_unit(const float *__restrict__ scale, uint32_t count, float *__restrict__ unit, const int64_t *__restrict__ labels, int64_t ignore, uint32_t classes) {
    float top = 0.0f;
    for (uint32_t i = threadIdx.x; i < count; i += 256) {
        const float a = fabsf(scale[i]);
        if (labels) {
            const int64_t label = labels[i];
            if (label == ignore || (uint64_t)label >= classes) continue;
        }
        if (a < __builtin_inff()) top = fmaxf(top, a);
    }
    top = slz_wave_max(top);
    __shared__ float tops[4];
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        int e = 0;
        if (top > 0.0f) frexpf(top, &e);
        if (labels && top > 0.0f) *unit = fminf(fmaxf(top, 0x1p-100f), 0x1p100f);
        else *unit = ldexpf(1.0f, e < -100 ? -100 : e > 100 ? 100 : e);
    }
}

void slz_unit_of(const float *values, uint32_t count, float *unit, hipStream_t s, const int64_t *labels, int64_t ignore, uint32_t classes) {
    hipLaunchKernelGGL(k_scale_unit, dim3(1), dim3(256), 0, s, values, count, unit, labels, ignore, classes);
}
