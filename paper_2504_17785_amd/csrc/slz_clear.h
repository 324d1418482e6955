// Declarations shared by the sources of include/silenzio_clear.h: element types, argument checks, operands of the matrix product.
#pragma once
#include "slz_internal.h"
#include "slz_gadget_util.h"
#include "../../include/silenzio_clear.h"

__host__ __device__ static inline uint32_t slz_type_bytes(int type) { return type == SLZ_F32 ? 4 : 2; }
static inline bool slz_type_ok(int type) { return type == SLZ_F32 || type == SLZ_BF16 || type == SLZ_F16; }

// longest row distance in elements: 256 rows stay below 2^31 bytes, the reach of a buffer descriptor's offsets
#define SLZ_CLEAR_MAX_LD ((int64_t)1 << 22)
#define SLZ_CLEAR_MAX_LEN 0x7fffffffu

// SLZ_OK, or what is wrong with a matrix of rows x cols elements
static inline int slz_matrix_check(const void *p, uint32_t rows, uint32_t cols, int64_t ld, uint32_t bytes) {
    if (rows > SLZ_CLEAR_MAX_LEN || cols > SLZ_CLEAR_MAX_LEN) return SLZ_E_TOO_LARGE;
    if (ld < (int64_t)cols) return SLZ_E_INVALID_ARG;
    if (rows == 0 || cols == 0) return SLZ_OK;
    if (!p || ((uintptr_t)p % bytes)) return SLZ_E_INVALID_ARG;
    return ld > SLZ_CLEAR_MAX_LD ? SLZ_E_TOO_LARGE : SLZ_OK;
}
static inline bool slz_in_place(const void *p, uint32_t cols, int64_t ld, uint32_t bytes) {
    return !(((uintptr_t)p | ((uint64_t)cols * bytes) | ((uint64_t)ld * bytes)) & 15u);
}

// threads of a launch along x stay below 2^32
static inline uint32_t slz_most_blocks(uint32_t threads) { return 0xffffffffu / threads; }

static inline bool slz_ws_ok(const void *ws, size_t have, size_t need) { return need == 0 || (ws && have >= need && !((uintptr_t)ws & 255u)); }

#ifdef __HIPCC__
__device__ __forceinline__ float slz_bf16_to_f32(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
__device__ __forceinline__ uint16_t slz_f32_to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ float slz_f16_to_f32(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
__device__ __forceinline__ uint16_t slz_f32_to_f16(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

__device__ __forceinline__ float slz_get(const void *p, int type, size_t i) {
    if (type == SLZ_F32) return ((const float *)p)[i];
    const uint16_t b = ((const uint16_t *)p)[i];
    return type == SLZ_BF16 ? slz_bf16_to_f32(b) : slz_f16_to_f32(b);
}
__device__ __forceinline__ uint16_t slz_half(float x, int type) { return type == SLZ_BF16 ? slz_f32_to_bf16(x) : slz_f32_to_f16(x); }
__device__ __forceinline__ void slz_put(void *p, int type, size_t i, float x) {
    if (type == SLZ_F32) ((float *)p)[i] = x;
    else ((uint16_t *)p)[i] = slz_half(x, type);
}
// A 32-bit number as three bf16 whose sum it is: its leading 8 bits, the next 8, the last 8 (cut off, so none of them overflows).
// An infinity or NaN is all in the first.
__device__ __forceinline__ void slz_split3(float x, uint16_t (&q)[3]) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    if ((u & 0x7f800000u) == 0x7f800000u) {
        q[0] = (uint16_t)(u >> 16) | ((u & 0x7fffffu) ? 0x40u : 0u);
        q[1] = q[2] = 0;
        return;
    }
    const float h = __builtin_bit_cast(float, u & 0xffff0000u), r = x - h;
    const float l = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, r) & 0xffff0000u);
    q[0] = (uint16_t)(u >> 16);
    q[1] = (uint16_t)(__builtin_bit_cast(uint32_t, l) >> 16);
    q[2] = (uint16_t)(__builtin_bit_cast(uint32_t, r - l) >> 16);
}
typedef int v4i32 __attribute__((ext_vector_type(4)));
// Eight elements of a row of `cols` at c (a multiple of 8), zeros past its end; the row may begin at any address.  Where the row ends inside,
// its last eight are read and moved down.  In two parts, so that several loads are under way before the first is looked at.
typedef v4i32 v4i32_any __attribute__((aligned(1)));
template <int TYPE> struct row8 { v4i32 w[TYPE == SLZ_F32 ? 2 : 1]; };
template <int TYPE> __device__ __forceinline__ row8<TYPE> row8_load(const void *x, size_t row, uint32_t c, uint32_t cols) {
    row8<TYPE> q;
    if (cols < 8u) {                                   // all of it, in the first threads
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = c + i < cols ? slz_get(x, TYPE, row + c + i) : 0.0f;
        if constexpr (TYPE == SLZ_F32) {
            q.w[0] = v4i32{__float_as_int(v[0]), __float_as_int(v[1]), __float_as_int(v[2]), __float_as_int(v[3])};
            q.w[1] = v4i32{__float_as_int(v[4]), __float_as_int(v[5]), __float_as_int(v[6]), __float_as_int(v[7])};
        } else {
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; i++) h[i] = slz_half(v[2 * i], TYPE) | ((uint32_t)slz_half(v[2 * i + 1], TYPE) << 16);
            q.w[0] = v4i32{(int)h[0], (int)h[1], (int)h[2], (int)h[3]};
        }
        return q;
    }
    const uint32_t from = min(c, cols - 8u);
    const v4i32_any *p = (const v4i32_any *)((const char *)x + (row + from) * slz_type_bytes(TYPE));
    q.w[0] = p[0];
    if constexpr (TYPE == SLZ_F32) q.w[1] = p[1];
    return q;
}
template <int TYPE> __device__ __forceinline__ void row8_values(const row8<TYPE> &q, uint32_t c, uint32_t cols, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if constexpr (TYPE == SLZ_F32) v[i] = __int_as_float(q.w[i / 4][i % 4]);
        else {
            const uint16_t h = (uint16_t)((uint32_t)q.w[0][i / 2] >> (16 * (i & 1)));
            v[i] = TYPE == SLZ_BF16 ? slz_bf16_to_f32(h) : slz_f16_to_f32(h);
        }
    }
    if (c + 8u <= cols) return;
    const uint32_t gone = c >= cols ? 8u : cols < 8u ? 0u : c + 8u - cols;
#pragma unroll
    for (uint32_t b = 1; b < 16; b <<= 1)
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) v[i] = gone & b ? (i + b < 8 ? v[(i + b) % 8] : 0.0f) : v[i];
}
// C consecutive values v of one row at p[0 .. C), of which `valid` exist; aligned: p is a multiple of C elements
template <int C> __device__ __forceinline__ void slz_put_run(void *p, int type, const float (&v)[C], uint32_t valid, bool aligned) {
    static_assert(C % 4 == 0, "");
    if (valid >= C && aligned) {
        if (type == SLZ_F32) {
#pragma unroll
            for (int i = 0; i < C; i += 4) *(float4 *)((float *)p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
            uint32_t w[C / 2];
#pragma unroll
            for (int i = 0; i < C / 2; i++) w[i] = slz_half(v[2 * i], type) | ((uint32_t)slz_half(v[2 * i + 1], type) << 16);
            if constexpr (C % 8 == 0) {
#pragma unroll
                for (int i = 0; i < C / 2; i += 4) *(uint4 *)((uint32_t *)p + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < C / 2; i += 2) *(uint2 *)((uint32_t *)p + i) = make_uint2(w[i], w[i + 1]);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < C; i++)
        if ((uint32_t)i < valid) slz_put(p, type, i, v[i]);
}
// i / by and the rest; in 32 bits where that holds i
__device__ __forceinline__ size_t slz_divide(size_t i, uint32_t by, bool narrow, uint32_t &rest) {
    if (narrow) {
        const uint32_t q = (uint32_t)i / by;
        rest = (uint32_t)i - q * by;
        return q;
    }
    const size_t q = i / by;
    rest = (uint32_t)(i - q * by);
    return q;
}
// maximum over a wave, in every lane: over 16 lanes by lane permutations within the row, then over the four rows
template <int CONTROL> __device__ __forceinline__ float slz_dpp_max(float x) {
    return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float slz_wave_max(float x) {
    x = slz_dpp_max<0xb1>(x);                          // lanes 1 apart, 2 apart, mirrored in 8, mirrored in 16
    x = slz_dpp_max<0x4e>(x);
    x = slz_dpp_max<0x141>(x);
    x = slz_dpp_max<0x140>(x);
    const int v = __builtin_bit_cast(int, x);
    const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 0)), b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 16));
    const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 32)), d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 48));
    return fmaxf(fmaxf(a, b), fmaxf(c, d));
}
template <int CONTROL> __device__ __forceinline__ float slz_dpp_add(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}
// sum over a wave, the same bits in every lane
__device__ __forceinline__ float slz_wave_sum(float x) {
    x = slz_dpp_add<0xb1>(x);
    x = slz_dpp_add<0x4e>(x);
    x = slz_dpp_add<0x141>(x);
    x = slz_dpp_add<0x140>(x);
    const int v = __builtin_bit_cast(int, x);
    const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 0)), b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 16));
    const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 32)), d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 48));
    return (a + b) + (c + d);
}
#endif

// ---- operands of the matrix product (slz_clear_common.hip) ---------------------------------------------------------------------
// A matrix as the product takes it: 16-byte aligned rows of bf16, f16 or int8, one or three pieces `piece` bytes apart
struct slz_operand {
    const char *p;
    int64_t ld, piece;               // bytes
    uint32_t pieces;
    int element;                     // SLZ_BF16, SLZ_F16, or 3 for int8
};
// what is to be laid out before a product: matrices of elements of 1, 2 or 4 bytes (these into three bf16), in one launch
struct slz_layout { const char *x; char *out; int64_t ld, piece; uint32_t rows, cols, ld_out, bytes; };
struct slz_layouts { slz_layout job[2]; uint32_t count; };
void slz_layout_run(const slz_layouts &jobs, hipStream_t s);
// bytes of workspace for laying out rows x cols of `type` (0 when it can be read in place)
size_t slz_operand_bytes(const void *p, int type, uint32_t rows, uint32_t cols, int64_t ld);
// and the operand; ws: that many bytes, which the job that is added fills
slz_operand slz_operand_of(const void *p, int type, uint32_t rows, uint32_t cols, int64_t ld, char *ws, slz_layouts &jobs);
size_t slz_operand_i8_bytes(const int8_t *p, uint32_t rows, uint32_t cols, int64_t ld);
slz_operand slz_operand_i8_of(const int8_t *p, uint32_t rows, uint32_t cols, int64_t ld, char *ws, slz_layouts &jobs);
// What a type of few bits could not hold is divided by *unit, from 2^-100 to 2^100 (1 where there is nothing above 0).  Without labels the power of two above
// the largest finite magnitude of `count` values; with labels this magnitude itself, of the values whose label lies in [0, classes) and is not `ignore`.
void slz_unit_of(const float *values, uint32_t count, float *unit, hipStream_t s, const int64_t *labels = nullptr, int64_t ignore = 0, uint32_t classes = 0);
