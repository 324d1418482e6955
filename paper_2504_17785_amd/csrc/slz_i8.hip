// Products of 8-bit integers with a scale per row (include/silenzio_clear.h): quantisation, the product, its gradient.
#include "slz_gemm.h"

// ---- quantisation ------------------------------------------------------------------------------------------------------------------
// A row whose largest entry is below 2^-100 is moved up by 2^100 first, so that 1 / top stays finite.
__device__ __forceinline__ float quantize_scale(float top, bool finite, float &up, float &inv) {
    up = top < 0x1p-100f ? 0x1p100f : 1.0f;
    const float t = top * up;
    inv = finite && t > 0.0f ? 1.0f / t * 127.0f : 0.0f;
    return finite ? t / 127.0f / up : __builtin_nanf("");
}
__device__ __forceinline__ int8_t quantize_one(float x, float up, float inv) {
    return (int8_t)(int)fminf(fmaxf(rintf(x * up * inv), -127.0f), 127.0f);
}

__device__ __forceinline__ float top_of(const float (&v)[8]) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float a = fabsf(v[i]);
        top = a < __builtin_inff() ? fmaxf(top, a) : __builtin_inff();             // NaN too; stays
    }
    return top;
}
__device__ __forceinline__ uint2 quantize8(const float (&v)[8], bool finite, float up, float inv) {
    uint32_t w[2] = {0, 0};
    if (finite)
#pragma unroll
        for (int i = 0; i < 8; i++) w[i / 4] |= (uint32_t)(uint8_t)quantize_one(v[i], up, inv) << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
// One workgroup per row; bound by its latency for few rows (2.5 us) and by memory for many (4096 x 4096 bf16: 12.4 us, 4.1 TB/s).  A row of up to 16
// entries a thread stays in registers, of a longer one the rest is read again from the cache.
#define QUANTIZE_KEPT 2
template <int TYPE>
__global__ void __launch_bounds__(256)
k_quantize(const void *__restrict__ x, uint32_t cols, int64_t ld_x, int8_t *__restrict__ q, int64_t ld_q, uint32_t words, float *__restrict__ scale) {
    const size_t row = blockIdx.x, at = row * ld_x;
    __shared__ float tops[4];
    float kept[QUANTIZE_KEPT][8], top = 0.0f;
    row8<TYPE> first[QUANTIZE_KEPT];
#pragma unroll
    for (int k = 0; k < QUANTIZE_KEPT; k++) first[k] = row8_load<TYPE>(x, at, (threadIdx.x + k * 256) * 8, cols);
#pragma unroll
    for (int k = 0; k < QUANTIZE_KEPT; k++) {
        row8_values<TYPE>(first[k], (threadIdx.x + k * 256) * 8, cols, kept[k]);
        top = fmaxf(top, top_of(kept[k]));
    }
    for (uint32_t c = (threadIdx.x + QUANTIZE_KEPT * 256) * 8; c < cols; c += 2048) {
        float v[8];
        row8_values<TYPE>(row8_load<TYPE>(x, at, c, cols), c, cols, v);
        top = fmaxf(top, top_of(v));
    }
    top = slz_wave_max(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const bool finite = top < __builtin_inff();
    float up, inv;
    const float sc = quantize_scale(top, finite, up, inv);
    if (threadIdx.x == 0) scale[row] = sc;
    int8_t *out = q + row * ld_q;
    for (uint32_t k = 0, c = threadIdx.x * 8; c < cols; k++, c += 2048) {
        float v[8];
        if (k < QUANTIZE_KEPT)
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = k == 0 ? kept[0][i] : kept[1][i];
        else row8_values<TYPE>(row8_load<TYPE>(x, at, c, cols), c, cols, v);
        const uint2 w = quantize8(v, finite, up, inv);
        if (words && c + 8 <= cols) *(uint2 *)(out + c) = w;
        else
            for (uint32_t i = 0; i < 8 && c + i < cols; i++) out[c + i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}
static int quantize_rows(const void *x, int type, uint32_t rows, uint32_t cols, int64_t ld_x, int8_t *q, int64_t ld_q, float *scale, hipStream_t s) {
    const uint32_t words = !(((uintptr_t)q | (uint64_t)ld_q) & 7u);               // rows of q begin at multiples of eight
    const auto k = type == SLZ_F32 ? k_quantize<SLZ_F32> : type == SLZ_BF16 ? k_quantize<SLZ_BF16> : k_quantize<SLZ_F16>;
    for (uint32_t first = 0, most = slz_most_blocks(256); first < rows; first += most) {
        const void *from = (const char *)x + (int64_t)first * ld_x * slz_type_bytes(type);
        hipLaunchKernelGGL(k, dim3(rows - first < most ? rows - first : most), dim3(256), 0, s, from, cols, ld_x, q + (int64_t)first * ld_q, ld_q, words, scale + first);
    }
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}

extern "C" int slz_quantize_i8(const void *x, int type, uint32_t rows, uint32_t cols, int64_t ld_x, int8_t *q, int64_t ld_q, float *scale, void *stream) {
    if (!slz_type_ok(type)) return SLZ_E_INVALID_ARG;
    int rc = slz_matrix_check(x, rows, cols, ld_x, slz_type_bytes(type));
    if (rc == SLZ_OK) rc = slz_matrix_check(q, rows, cols, ld_q, 1);
    if (rc == SLZ_OK) rc = slz_matrix_check(scale, rows, 1, 1, 4);
    if (rc != SLZ_OK || rows == 0) return rc;
    return quantize_rows(x, type, rows, cols, ld_x, q, ld_q, scale, (hipStream_t)stream);
}

// ---- few rows ------------------------------------------------------------------------------------------------------------------------
// Up to 32 rows of a: every byte of b is used for at most 32 products, so b is streamed once from memory straight into the matrix
// instructions' registers, and what bounds it is how much of b is under way.  A workgroup of eight waves has 16 NB rows of b, each wave an
// eighth of k with its first loads issued before anything else; a (quantised here, if it is x) lies in shared memory; the
// eight waves' sums meet there.  Rows of b may begin at any address.
// One row by 8192 x 4096: 8.8 us (3.8 TB/s, launch included), with x quantised in the same launch 10.3; the tiled product 20.
#define THIN_WAVES 8
#define THIN_AHEAD 8                 // loads of 1 KiB under way in each wave
#define THIN_WIDE 8192               // rows of b from which a wave takes 32 of them instead of 16: 32768 x 2048 13.6 us, with 16 20.7; 8192 x 4096 8.8 both
#define THIN_LDS (144u << 10)
#define THIN_MAX_ROWS 32u
#define THIN_SLOTS 8                 // parts of 512 elements of x that a wave quantises

// 16 bytes at k (a multiple of 16) of a row of `count` bytes, zeros past its end.  Where the row ends inside, its last 16 are read and moved down.
__device__ __forceinline__ v4i32 thin_load(const int8_t *row, uint32_t k, uint32_t count) {
    union { int8_t b[16]; uint64_t d[2]; v4i32 v; } u;
    u.v = v4i32{0, 0, 0, 0};
    if (k >= count) return u.v;
    if (count < 16u) {
#pragma unroll
        for (uint32_t i = 0; i < 15u; i++)
            if (i < count) u.b[i] = row[i];
        return u.v;
    }
    const uint32_t from = min(k, count - 16u), bits = (k - from) * 8u;
    u.v = *(const v4i32_any *)(row + from);
    if (bits >= 64u) {
        u.d[0] = u.d[1] >> (bits - 64u);
        u.d[1] = 0;
    } else if (bits) {
        u.d[0] = (u.d[0] >> bits) | (u.d[1] << (64u - bits));
        u.d[1] >>= bits;
    }
    return u.v;
}

typedef v4i32 v4i32_4 __attribute__((aligned(4)));

struct thin_args {
    const void *a;                   // int8, or x where it is quantised here
    const float *sa;                 // scales of a, or null
    int type;                        // of y and x
    int64_t ld_a;
    const int8_t *b;
    const float *sb;
    int64_t ld_b;
    void *y;
    int64_t ld_y;
    uint32_t M, N, K, pitch;         // pitch: bytes of a row of a in shared memory
};

// XTYPE: x's type where a is x and quantised here, or -1 where a is int8
template <int MI, int NB, int XTYPE>
__global__ void __launch_bounds__(THIN_WAVES * 64) k_thin_i8(const thin_args p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float tops[THIN_WAVES][THIN_SLOTS], scales[THIN_MAX_ROWS];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    const uint32_t n0 = blockIdx.x * (16 * NB), steps = (p.K + 63u) / 64u;
    const uint32_t begin = wave * steps / THIN_WAVES, end = (wave + 1) * steps / THIN_WAVES;
    const uint32_t whole = min(end, p.K / 64u);        // steps that end inside the rows; at most one is left, in the last wave
    constexpr int DEPTH = THIN_AHEAD / NB;
    // x: several waves share a row where there are fewer rows than waves; each wave's 512-element parts of its rows are its slots
    constexpr int SLOTS = XTYPE >= 0 ? THIN_SLOTS : 1;
    const uint32_t per_row = p.M >= THIN_WAVES ? 1u : p.M > 2 ? 2u : p.M == 2 ? 4u : 8u, parts = (p.K + per_row * 512u - 1) / (per_row * 512u);
    const uint32_t used = (p.M * per_row + THIN_WAVES - 1) / THIN_WAVES * parts;
    row8<XTYPE < 0 ? SLZ_F32 : XTYPE> x[SLOTS];
    uint32_t slot_row[SLOTS], slot_part[SLOTS], slot_first[SLOTS];                  // the slot's row, its part of it, the slot of the row's first part
    {
        uint32_t m = wave / per_row, part = 0, first = 0;
#pragma unroll
        for (uint32_t i = 0; i < SLOTS; i++) {
            slot_row[i] = m; slot_part[i] = part; slot_first[i] = first;
            if (++part == parts) { part = 0; m += THIN_WAVES / per_row; first = i + 1; }
        }
    }
    const auto slot_col = [&](int i) { return ((slot_part[i] * per_row + wave % per_row) * 64u + lane) * 8u; };
    if constexpr (XTYPE >= 0)
#pragma unroll
        for (int i = 0; i < SLOTS; i++)
            if (i < used) x[i] = row8_load<XTYPE>(p.a, (size_t)min(slot_row[i], p.M - 1) * p.ld_a, slot_col(i), p.K);
    // rows that do not begin at a multiple of 4 bytes: 16 bytes at any address take the memory path several times as long as 16 at a multiple of
    // 4, so these and the 4 behind them are read and shifted (those 4 hold bytes of the row, or are not looked at)
    const bool odd = (((uintptr_t)p.b | (uint64_t)p.ld_b) & 3u) != 0;
    const char *row[NB];
    uint32_t shift[NB];
#pragma unroll
    for (int j = 0; j < NB; j++) {
        const char *at = (const char *)p.b + (int64_t)min(n0 + j * 16 + r, p.N - 1) * p.ld_b + g * 16u;
        shift[j] = (uint32_t)(uintptr_t)at & 3u;
        row[j] = at - shift[j];
    }
    const auto b_load = [&](int j, uint32_t step, v4i32 &v, uint32_t &next) {
        const char *at = row[j] + step * 64u;
        v = *(const v4i32_4 *)at;
        if (odd) next = *(const uint32_t *)(at + (shift[j] ? 16 : 12));
    };
    const auto b_value = [&](int j, const v4i32 &v, uint32_t next) {
        if (!odd) return v;
        v4i32 o;
#pragma unroll
        for (int i = 0; i < 4; i++) o[i] = (int)__builtin_amdgcn_alignbyte(i < 3 ? (uint32_t)v[(i + 1) % 4] : next, (uint32_t)v[i], shift[j]);
        return o;
    };
    v4i32 ahead[DEPTH][NB];
    uint32_t behind[DEPTH][NB] = {};
    if (begin < whole)
#pragma unroll
        for (int d = 0; d < DEPTH; d++)
#pragma unroll
            for (int j = 0; j < NB; j++) b_load(j, min(begin + d, whole - 1), ahead[d][j], behind[d][j]);
    __builtin_amdgcn_sched_barrier(0);

    // a's rows to shared memory, zeros behind them up to a whole step
    if constexpr (XTYPE >= 0) {
#pragma unroll
        for (int i = 0; i < SLOTS; i++) {
            if (i >= used) continue;
            float v[8];
            row8_values<XTYPE>(x[i], slot_col(i), p.K, v);
            const float top = slz_wave_max(top_of(v));
            if (lane == 0) tops[wave][i] = top;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SLOTS; i++) {
            const uint32_t m = slot_row[i], c = slot_col(i);
            if (i >= used || m >= p.M) continue;
            float top = 0.0f, up, inv;
            // per_row waves have parts of it, each in `parts` slots: at most 64 values, one a lane
            const uint32_t k = lane % THIN_SLOTS, w = lane / THIN_SLOTS;
            if (k < parts && w < per_row) top = tops[wave / per_row * per_row + w][slot_first[i] + k];
            top = slz_wave_max(top);
            const bool finite = top < __builtin_inff();
            const float scale = quantize_scale(top, finite, up, inv);
            if (c == 0) scales[m] = scale;
            float v[8];
            row8_values<XTYPE>(x[i], c, p.K, v);
            if (c < steps * 64u) *(uint2 *)(lds + (size_t)m * p.pitch + c) = quantize8(v, finite, up, inv);
        }
    } else {
        for (uint32_t i = threadIdx.x; i < p.M * steps * 4u; i += THIN_WAVES * 64) {
            const uint32_t m = i / (steps * 4u), c = i % (steps * 4u) * 16u;
            *(v4i32 *)(lds + (size_t)m * p.pitch + c) = thin_load((const int8_t *)p.a + (int64_t)m * p.ld_a, c, p.K);
        }
        if (threadIdx.x < p.M) scales[threadIdx.x] = p.sa[threadIdx.x];
    }
    __syncthreads();

    v4i32 acc[MI][NB];
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) acc[i][j] = v4i32{0, 0, 0, 0};
    const auto a_at = [&](int i, uint32_t step) {
        return i * 16 + r < p.M ? *(const v4i32 *)(lds + (size_t)(i * 16 + r) * p.pitch + step * 64u + g * 16u) : v4i32{0, 0, 0, 0};
    };
    for (uint32_t s0 = begin; s0 < whole; s0 += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; d++) {
            const uint32_t s = s0 + d;
            if (s >= whole) break;
            v4i32 fa[MI];
#pragma unroll
            for (int i = 0; i < MI; i++) fa[i] = a_at(i, s);
#pragma unroll
            for (int j = 0; j < NB; j++) {
#pragma unroll
                for (int i = 0; i < MI; i++) acc[i][j] = slz_mma<SLZ_EL_I8>(b_value(j, ahead[d][j], behind[d][j]), fa[i], acc[i][j]);
                if (s + DEPTH < whole) b_load(j, s + DEPTH, ahead[d][j], behind[d][j]);
            }
        }
    if (whole < end)
#pragma unroll
        for (int j = 0; j < NB; j++) {
            const v4i32 last = thin_load((const int8_t *)row[j] + shift[j] - g * 16u, whole * 64u + g * 16u, p.K);
#pragma unroll
            for (int i = 0; i < MI; i++) acc[i][j] = slz_mma<SLZ_EL_I8>(last, a_at(i, whole), acc[i][j]);
        }
    __syncthreads();
    int *sums = (int *)lds;                            // [wave][row of a][row of b]
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) *(v4i32 *)(sums + ((wave * MI + i) * 16 + r) * (NB * 16) + j * 16 + g * 4) = acc[i][j];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < MI * 16 * NB * 16; i += THIN_WAVES * 64) {
        const uint32_t m = i / (NB * 16), n = n0 + i % (NB * 16);
        if (m >= p.M || n >= p.N) continue;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < THIN_WAVES; w++) sum += sums[w * (MI * 16 * NB * 16) + i];
        slz_put(p.y, p.type, (size_t)m * p.ld_y + n, (float)sum * (scales[m] * p.sb[n]));
    }
}

// Where it is taken: few rows that fit the shared memory.  Beyond 16 rows the tiled product is as fast where b is large and lies on 16 bytes (32 rows
// by 8192 x 4096: 16 us here, 12 there), and slower where b is small or would have to be laid out (1000 x 2049: 8 here, 19 there).
static uint32_t thin_pitch(uint32_t k) { return (k + 63u) / 64u * 64u + 16u; }
static bool thin_takes(const slz_i8_shape *sh, const int8_t *b) {
    if (sh->m > THIN_MAX_ROWS || sh->k == 0 || (size_t)sh->m * thin_pitch(sh->k) > THIN_LDS) return false;
    return sh->m <= 16 || sh->n <= 4096 || !slz_in_place(b, sh->k, sh->ld_b, 1);
}
// x is quantised by every workgroup as long as that is little work for all of them and its registers hold it: it saves a launch (3.5 us of the host,
// 2.5 of the card) and costs each round of workgroups 1.5 us for a row of 4096 entries, 6 for four
static bool thin_quantizes(uint32_t m, uint32_t n, uint32_t k) {
    if ((size_t)m * k > (n <= 2048 ? 32768 : 8192)) return false;
    const uint32_t per_row = m >= THIN_WAVES ? 1u : m > 2 ? 2u : m == 2 ? 4u : 8u, rows = (m * per_row + THIN_WAVES - 1) / THIN_WAVES;
    return rows * ((k + per_row * 512u - 1) / (per_row * 512u)) <= THIN_SLOTS;
}

template <int MI, int NB> static void thin_launch(const thin_args &p, int x_type, size_t bytes, hipStream_t s) {
    const auto k = x_type < 0 ? k_thin_i8<MI, NB, -1> : x_type == SLZ_F32 ? k_thin_i8<MI, NB, SLZ_F32> : x_type == SLZ_BF16 ? k_thin_i8<MI, NB, SLZ_BF16> : k_thin_i8<MI, NB, SLZ_F16>;
    hipLaunchKernelGGL(k, dim3((p.N + 16 * NB - 1) / (16 * NB)), dim3(THIN_WAVES * 64), bytes, s, p);
}
// x_type: of a where it is x, or -1
static int thin_product(const thin_args &p, int x_type, hipStream_t s) {
    const uint32_t mi = p.M > 16 ? 2 : 1, nb = p.N >= THIN_WIDE ? 2 : 1;
    const size_t a = (size_t)p.M * p.pitch, sums = (size_t)THIN_WAVES * mi * nb * 1024, bytes = a > sums ? a : sums;
    if (mi == 1) nb == 1 ? thin_launch<1, 1>(p, x_type, bytes, s) : thin_launch<1, 2>(p, x_type, bytes, s);
    else nb == 1 ? thin_launch<2, 1>(p, x_type, bytes, s) : thin_launch<2, 2>(p, x_type, bytes, s);
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
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
    *bytes = thin_takes(sh, b) ? 0 : slz_operand_i8_bytes(a, sh->m, sh->k, sh->ld_a) + slz_operand_i8_bytes(b, sh->n, sh->k, sh->ld_b) + slz_ranges_bytes(i8_choice(sh), sh->m, sh->n);
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
    if (thin_takes(sh, b))
        return thin_product({a, sa, sh->type, sh->ld_a, b, sb, sh->ld_b, y, sh->ld_y, sh->m, sh->n, sh->k, thin_pitch(sh->k)}, -1, (hipStream_t)stream);
    const size_t for_a = slz_operand_i8_bytes(a, sh->m, sh->k, sh->ld_a), for_b = slz_operand_i8_bytes(b, sh->n, sh->k, sh->ld_b);
    if (!slz_ws_ok(ws, ws_bytes, for_a + for_b + slz_ranges_bytes(i8_choice(sh), sh->m, sh->n))) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    slz_layouts jobs = {};
    const slz_operand oa = slz_operand_i8_of(a, sh->m, sh->k, sh->ld_a, (char *)ws, jobs);
    const slz_operand ob = slz_operand_i8_of(b, sh->n, sh->k, sh->ld_b, (char *)ws + for_a, jobs);
    slz_layout_run(jobs, s);
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
    if (thin_takes(sh, b)) P.total = thin_quantizes(sh->m, sh->n, sh->k) ? 0 : P.b;
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
    const bool thin = thin_takes(sh, b);
    const uint32_t pitch = thin_pitch(sh->k);
    if (thin && thin_quantizes(sh->m, sh->n, sh->k))
        return thin_product({x, nullptr, sh->type, sh->ld_a, b, sb, sh->ld_b, y, sh->ld_y, sh->m, sh->n, sh->k, pitch}, sh->type, s);
    int8_t *q = (int8_t *)ws + P.q;
    float *sa = (float *)((char *)ws + P.scale);
    // a row's last 16 entries may end with whatever was there: b's are zero in those places
    rc = quantize_rows(x, sh->type, sh->m, sh->k, sh->ld_a, q, P.ld_q, sa, s);
    if (rc != SLZ_OK) return rc;
    if (thin) return thin_product({q, sa, sh->type, P.ld_q, b, sb, sh->ld_b, y, sh->ld_y, sh->m, sh->n, sh->k, pitch}, -1, s);
    const slz_operand oa{(const char *)q, P.ld_q, 0, 1, 3};
    slz_layouts jobs = {};
    const slz_operand ob = slz_operand_i8_of(b, sh->n, sh->k, sh->ld_b, (char *)ws + P.b, jobs);
    slz_layout_run(jobs, s);
    return i8_product(sh, oa, sa, ob, sb, y, (char *)ws + P.ranges, s);
}

int slz_float_product(const slz_operand &left, bool left_rows_k, const slz_operand &right, uint32_t M, uint32_t N, uint32_t K, const slz_choice &c, const float *unit, float by,
                      void *out, int type, int64_t ld_out, char *ranges, hipStream_t s) {
    const slz_gemm p = slz_gemm_of(left, right, M, N, K);
    const slz_times_unit f{unit, by};
    if (type == SLZ_F16)
        return left_rows_k ? slz_gemm_to<SLZ_EL_F16, true, true>(p, c, f, out, type, ld_out, ranges, s) : slz_gemm_to<SLZ_EL_F16, false, true>(p, c, f, out, type, ld_out, ranges, s);
    return left_rows_k ? slz_gemm_to<SLZ_EL_BF16, true, true>(p, c, f, out, type, ld_out, ranges, s) : slz_gemm_to<SLZ_EL_BF16, false, true>(p, c, f, out, type, ld_out, ranges, s);
}

// ---- gradient ------------------------------------------------------------------------------------------------------------------------------
// dy times the values scale_r q_rc: these are laid out as an operand once (bf16, or three bf16 for f32), then two ordinary products.  The scale belongs to the
// index that is summed over, so it has to be in one of the operands, and rounding it there takes bf16 results from 1.7e-3 off (their own rounding) to 2.4e-3 and
// f16 ones from 2.1e-4 to 2.9e-4; two pieces instead of one would double the product.  f16 could
// not hold small scales, so its values are held times VALUES_F16_UP / `unit`, the power of two above the largest scale, and the sums multiplied by the inverse:
// magnitudes of up to 128 2^8 are below f16's largest, and rows whose scale is down to 2^-22 of the largest keep 11 bits.
#define VALUES_F16_UP 256.0f
// One row (no scale given): the integers themselves, which every type holds exactly, and the sums are multiplied by its scale.  Rounded with the scale in them the
// entries of one row can all be off the same way, by up to half as much again as the result's own rounding; over many rows that evens out.
typedef uint64_t u64_any __attribute__((aligned(1)));
// eight values of a row per thread; bound by memory: 4096 x 4096 to bf16 10.5 us (48 MiB, 4.8 TB/s)
template <int TYPE>
__global__ void __launch_bounds__(256)
k_values(const int8_t *__restrict__ q, const float *__restrict__ scale, const float *__restrict__ unit, uint32_t rows, uint32_t cols, int64_t ld_q,
         char *__restrict__ out, uint32_t ld_out, int64_t piece) {
    const uint32_t per_row = ld_out / 16u;
    const size_t total = (size_t)rows * per_row;
    constexpr int PIECES = TYPE == SLZ_F32 ? 3 : 1;
    for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < total; g += (size_t)gridDim.x * 256) {
        uint32_t c;
        const size_t r = slz_divide(g, per_row, total <= 0xffffffffu, c);
        c *= 8;
        const float sc = !scale ? 1.0f : TYPE == SLZ_F16 ? scale[r] / *unit * VALUES_F16_UP : scale[r];
        uint64_t bytes = 0;
        if (c + 8u <= cols) bytes = *(const u64_any *)(q + r * ld_q + c);
        else
            for (uint32_t i = 0; i < 8 && c + i < cols; i++) bytes |= (uint64_t)(uint8_t)q[r * ld_q + c + i] << (8 * i);
        uint16_t t[PIECES][8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float v = (float)(int8_t)(bytes >> (8 * i)) * sc;
            if constexpr (TYPE == SLZ_F32) {
                uint16_t u[3];
                slz_split3(v, u);
                for (int k = 0; k < 3; k++) t[k][i] = u[k];
            } else t[0][i] = slz_half(v, TYPE);
        }
#pragma unroll
        for (int k = 0; k < PIECES; k++) {
            uint32_t w[4];
#pragma unroll
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
    P.da = slz_choose(sh->m, sh->k, (sh->n + 63) / 64 * pairs, 1, false, 16, true);
    P.db = slz_choose(sh->n, sh->k, (sh->m + 63) / 64 * pairs, 1, false, 16, true);
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
    const bool one = rows == 1, with_unit = type == SLZ_F16 && !one;
    if (with_unit) slz_unit_of(scale, rows, unit, s);
    if (rows) {
        const auto k = type == SLZ_F32 ? k_values<SLZ_F32> : type == SLZ_BF16 ? k_values<SLZ_BF16> : k_values<SLZ_F16>;
        hipLaunchKernelGGL(k, ew_grid((size_t)rows * P.row / 16), dim3(256), 0, s, q, one ? nullptr : scale, unit, rows, sh->k, ld_q, values, P.row, right.piece);
    }
    return slz_float_product(left, left_rows_k, right, M, sh->k, rows, left_rows_k ? P.db : P.da, one ? scale : with_unit ? unit : nullptr, one ? 1.0f : 1.0f / VALUES_F16_UP, out,
                             type, ld_out, ranges, s);
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
    slz_layouts jobs = {};
    const slz_operand d = slz_operand_of(dy, sh->type, sh->m, sh->n, sh->ld_y, w + P.dy, jobs);
    slz_layout_run(jobs, s);
    if (da && sh->m) rc = grad_product(sh, d, false, sh->m, b, sh->ld_b, sb, sh->n, da, ld_da, w + P.values[1], (float *)(w + P.unit), w + P.ranges, P, s);
    if (rc == SLZ_OK && db && sh->n) rc = grad_product(sh, d, true, sh->n, a, sh->ld_a, sa, sh->m, db, ld_db, w + P.values[0], (float *)(w + P.unit) + 1, w + P.ranges, P, s);
    if (rc != SLZ_OK) return rc;
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
