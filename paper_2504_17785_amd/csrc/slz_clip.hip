// The norm of many gradients together, and all of them held to one (include/silenzio_clear.h).
//
// The tensors are cut into chunks of as many elements, numbered through all of them.  Workgroup b of G takes the chunks b, b + G, ..., adds up squares in 64 bits
// and leaves one sum; the second launch adds the sums in their order, so the result is the same bits whatever ran when, and multiplies.
#include "slz_clear.h"
#include "slz_clip_places.h"
#include <algorithm>
#include <stdlib.h>

#define CLIP_INLINE 64u              // tensors that a launch takes in its arguments
#define CLIP_GROUPS 2048u            // most workgroups, and sums

// a tensor as the kernels see it: `count` elements, cols is 0 where they are one run
struct clip_desc { const char *g; char *out; uint64_t count; int64_t ld_g, ld_out; uint32_t cols; int type; };
// first[i] is the number of tensor i's first chunk
struct clip_few { uint32_t first[CLIP_INLINE]; clip_desc desc[CLIP_INLINE]; };
struct clip_table { const uint32_t *first; const clip_desc *desc; };
struct clip_work { uint32_t count, chunks, chunk; };                             // tensors, chunks, elements of a chunk

__device__ __forceinline__ uint32_t clip_first(const clip_few &t, uint32_t i) { return t.first[i]; }
__device__ __forceinline__ uint32_t clip_first(const clip_table &t, uint32_t i) { return t.first[i]; }
__device__ __forceinline__ clip_desc clip_at(const clip_few &t, uint32_t i) { return t.desc[i]; }
__device__ __forceinline__ clip_desc clip_at(const clip_table &t, uint32_t i) { return t.desc[i]; }

// The tensor that has a chunk: the last one that begins at it or before.  Each lane looks at one of 64.
template <class T> __device__ __forceinline__ uint32_t clip_find(const T &t, uint32_t count, uint32_t chunk) {
    uint32_t lo = 0, span = 1;
    const uint32_t lane = threadIdx.x & 63u;
    while (span < count) span *= 64u;                  // at most 64^5 = 2^30, as count is below 2^26
    while (span > 1) {
        span /= 64u;
        const uint32_t i = lo + lane * span;
        const uint64_t in = __ballot(i < count && clip_first(t, min(i, count - 1)) <= chunk);
        lo += ((uint32_t)__popcll(in) - 1u) * span;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

template <int TYPE> struct run16 { static constexpr int E = TYPE == SLZ_F32 ? 4 : 8; v4i32 w; };
template <int TYPE> __device__ __forceinline__ float run_value(const v4i32 &w, int i) {
    if constexpr (TYPE == SLZ_F32) return __int_as_float(w[i]);
    else {
        const uint16_t h = (uint16_t)((uint32_t)w[i / 2] >> (16 * (i & 1)));
        return TYPE == SLZ_BF16 ? slz_bf16_to_f32(h) : slz_f16_to_f32(h);
    }
}
// What is done with n elements from `start` on of a tensor: whole runs of 16 bytes, several under way, and single elements, of which the places are given
template <int TYPE, class RUN, class ONE> __device__ __forceinline__ void clip_chunk(const clip_desc &d, uint64_t start, uint32_t n, const RUN &on_run, const ONE &on_one) {
    constexpr uint32_t E = run16<TYPE>::E, AHEAD = 4, B = TYPE == SLZ_F32 ? 4 : 2;
    if (d.cols == 0) {
        const char *g = d.g + start * B;
        const uint32_t runs = n / E;
        for (uint32_t r0 = threadIdx.x; r0 < runs; r0 += AHEAD * 256u) {
            v4i32 w[AHEAD];
#pragma unroll
            for (uint32_t a = 0; a < AHEAD; a++) w[a] = *(const v4i32_any *)(g + (size_t)min(r0 + a * 256u, runs - 1) * 16u);
#pragma unroll
            for (uint32_t a = 0; a < AHEAD; a++)
                if (r0 + a * 256u < runs) on_run(start + (uint64_t)(r0 + a * 256u) * E, w[a]);
        }
        const uint32_t i = runs * E + threadIdx.x;
        if (i < n) on_one(start + i, start + i);
        return;
    }
    for (uint32_t i = threadIdx.x; i < n; i += 256u) {
        uint32_t c;
        const size_t r = slz_divide(start + i, d.cols, start + i <= 0xffffffffu, c);
        const size_t from = r * d.ld_g + c;
        on_one(from, r * d.ld_out + c);
    }
}
template <class F> __device__ __forceinline__ void clip_typed(int type, const F &f) {
    if (type == SLZ_F32) f(std::integral_constant<int, SLZ_F32>());
    else if (type == SLZ_BF16) f(std::integral_constant<int, SLZ_BF16>());
    else f(std::integral_constant<int, SLZ_F16>());
}
// the sum over a workgroup, in every thread; sums: shared, four
__device__ __forceinline__ double clip_sum(double x, double *sums) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
    __syncthreads();
    return (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// Bound by memory: 1 GiB of bf16 187 us (5.7 TB/s), 16 MiB 9; a conversion and a 64-bit multiply-add an element are 28 % of the issue
template <class T> __global__ void __launch_bounds__(256) k_squares(const T table, const clip_work work, double *__restrict__ partial) {
    __shared__ double sums[4];
    double sum[4] = {0, 0, 0, 0};
    for (uint32_t c = blockIdx.x; c < work.chunks; c += gridDim.x) {
        const uint32_t i = clip_find(table, work.count, c);
        const clip_desc d = clip_at(table, i);
        const uint64_t start = (uint64_t)(c - clip_first(table, i)) * work.chunk;
        const uint32_t n = (uint32_t)min((uint64_t)work.chunk, d.count - start);
        clip_typed(d.type, [&](auto type) {
            constexpr int TYPE = decltype(type)::value;
            clip_chunk<TYPE>(d, start, n, [&](uint64_t, const v4i32 &w) {
#pragma unroll
                for (int e = 0; e < run16<TYPE>::E; e++) {
                    const double v = run_value<TYPE>(w, e);
                    sum[e & 3] = __builtin_fma(v, v, sum[e & 3]);
                }
            }, [&](uint64_t at, uint64_t) {
                const double v = slz_get(d.g, TYPE, at);
                sum[0] = __builtin_fma(v, v, sum[0]);
            });
        });
    }
    const double all = clip_sum((sum[0] + sum[1]) + (sum[2] + sum[3]), sums);
    if (threadIdx.x == 0) partial[blockIdx.x] = all;
}
// the norm from the workgroups' sums, in every thread
__device__ __forceinline__ float clip_norm(const double *partial, uint32_t count, double *sums) {
    double x = 0;
#pragma unroll
    for (uint32_t k = 0; k < CLIP_GROUPS / 256u; k++)
        if (k * 256u + threadIdx.x < count) x += partial[k * 256u + threadIdx.x];
    return (float)__builtin_sqrt(clip_sum(x, sums));
}
__global__ void __launch_bounds__(256) k_norm(const double *__restrict__ partial, uint32_t count, float *__restrict__ norm) {
    __shared__ double sums[4];
    const float n = clip_norm(partial, count, sums);
    if (threadIdx.x == 0) *norm = n;
}
// partial: null where the norm is given.  Every workgroup adds the sums itself: a launch less, and 16 KiB from the cache.  Bound by memory: 1 GiB read and
// written 397 us (5.4 TB/s).
template <class T>
__global__ void __launch_bounds__(256) k_clip(const T table, const clip_work work, const double *__restrict__ partial, uint32_t count, float max_norm, float eps, float *__restrict__ norm) {
    __shared__ double sums[4];
    float n;
    if (partial) {
        n = clip_norm(partial, count, sums);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
    } else n = *norm;
    // from the norm as it is given back, rounded to 32 bits: a caller that gives it gets the same bits
    const double limit = (double)n + (double)eps;
    const float f = limit > (double)max_norm ? (float)((double)max_norm / limit) : limit <= (double)max_norm ? 1.0f : __builtin_nanf("");
    for (uint32_t b = blockIdx.x; b < work.chunks; b += gridDim.x) {
        const uint32_t c = work.chunks - 1u - b;       // from the last one on: what was read last is still in the cache
        const uint32_t i = clip_find(table, work.count, c);
        const clip_desc d = clip_at(table, i);
        if (f == 1.0f && d.g == d.out) continue;
        const uint64_t start = (uint64_t)(c - clip_first(table, i)) * work.chunk;
        const uint32_t elements = (uint32_t)min((uint64_t)work.chunk, d.count - start);
        clip_typed(d.type, [&](auto type) {
            constexpr int TYPE = decltype(type)::value, E = run16<TYPE>::E;
            clip_chunk<TYPE>(d, start, elements, [&](uint64_t at, const v4i32 &w) {
                v4i32 o;
                if constexpr (TYPE == SLZ_F32) {
#pragma unroll
                    for (int e = 0; e < 4; e++) o[e] = __float_as_int(run_value<TYPE>(w, e) * f);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        o[e] = (int)(slz_half(run_value<TYPE>(w, 2 * e) * f, TYPE) | ((uint32_t)slz_half(run_value<TYPE>(w, 2 * e + 1) * f, TYPE) << 16));
                }
                // past the caches where the tensors are more than these hold: 1 GiB 593 us, 584 so; 256 MiB 150 and 126
                if (work.chunk >= 16384u) __builtin_nontemporal_store(f == 1.0f ? w : o, (v4i32_any *)(d.out + at * (16 / E)));
                else *(v4i32_any *)(d.out + at * (16 / E)) = f == 1.0f ? w : o;
            }, [&](uint64_t at, uint64_t to) {
                // bits in the first place: a product would change a NaN's
                if constexpr (TYPE == SLZ_F32) {
                    const uint32_t w = ((const uint32_t *)d.g)[at];
                    ((uint32_t *)d.out)[to] = f == 1.0f ? w : __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, w) * f);
                } else {
                    const uint16_t w = ((const uint16_t *)d.g)[at];
                    ((uint16_t *)d.out)[to] = f == 1.0f ? w : slz_half((TYPE == SLZ_BF16 ? slz_bf16_to_f32(w) : slz_f16_to_f32(w)) * f, TYPE);
                }
            });
        });
    }
}
// tables of many tensors come to the workspace in the arguments of a few small launches
__global__ void __launch_bounds__(64) k_clip_table(const clip_few few, uint32_t begin, uint32_t count, uint32_t *__restrict__ first, clip_desc *__restrict__ desc) {
    if (threadIdx.x < count) {
        first[begin + threadIdx.x] = few.first[threadIdx.x];
        desc[begin + threadIdx.x] = few.desc[threadIdx.x];
    }
}

// the same of tensors that are runs, from 24 bytes each: the chunks before a tensor are counted here.  1000 tensors: seven launches instead of sixteen
#define CLIP_RUNS 160u
struct clip_runs { struct { const char *g; char *out; uint64_t count_type; } run[CLIP_RUNS]; };
__global__ void __launch_bounds__(256) k_clip_runs(const clip_runs runs, uint32_t begin, uint32_t count, uint32_t before, uint32_t chunk, uint32_t *__restrict__ first, clip_desc *__restrict__ desc) {
    __shared__ uint32_t sums[4];
    const uint32_t i = threadIdx.x, lane = i & 63u;
    const auto r = runs.run[min(i, count - 1)];
    const uint64_t elements = r.count_type >> 2;
    const uint32_t mine = i < count ? (uint32_t)((elements + chunk - 1) / chunk) : 0u;
    uint32_t sum = mine;
    for (uint32_t o = 1; o < 64; o *= 2) {
        const uint32_t other = __shfl_up(sum, o);
        if (lane >= o) sum += other;
    }
    if (lane == 63) sums[i >> 6] = sum;
    __syncthreads();
    for (uint32_t w = 0; w < i >> 6; w++) before += sums[w];
    if (i >= count) return;
    first[begin + i] = before + sum - mine;
    desc[begin + i] = {r.g, r.out, elements, 0, 0, 0u, (int)(r.count_type & 3u)};
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------
static int clip_check(const slz_grad_tensor *t, uint32_t count, bool outputs) {
    if (count > 0 && !t) return SLZ_E_INVALID_ARG;
    if (count >= (1u << 26)) return SLZ_E_TOO_LARGE;
    for (uint32_t i = 0; i < count; i++) {
        if (!slz_type_ok(t[i].type)) return SLZ_E_INVALID_ARG;
        if (t[i].rows > SLZ_CLEAR_MAX_LEN || t[i].cols > SLZ_CLEAR_MAX_LEN) return SLZ_E_TOO_LARGE;
        if (t[i].ld_g < (int64_t)t[i].cols || (outputs && t[i].ld_out < (int64_t)t[i].cols)) return SLZ_E_INVALID_ARG;
        if (t[i].rows == 0 || t[i].cols == 0) continue;
        const uint32_t b = slz_type_bytes(t[i].type);
        const int64_t most = ((int64_t)1 << 50) / ((int64_t)t[i].rows * b);         // a matrix ends within 2^50 bytes, so that nothing here leaves 64 bits
        if (t[i].cols > most || (t[i].rows > 1 && (t[i].ld_g > most || (outputs && t[i].ld_out > most)))) return SLZ_E_TOO_LARGE;
        if (!t[i].g || (uintptr_t)t[i].g % b) return SLZ_E_INVALID_ARG;
        if (outputs && (!t[i].out || (uintptr_t)t[i].out % b)) return SLZ_E_INVALID_ARG;
    }
    return SLZ_OK;
}
static clip_place place_of(const slz_grad_tensor &t, bool out) {
    const uint64_t b = slz_type_bytes(t.type), ld = (uint64_t)(out ? t.ld_out : t.ld_g) * b, row = t.cols * b;
    const uintptr_t p = (uintptr_t)(out ? t.out : t.g);
    if (t.rows == 1 || ld == row) return {p, p + t.rows * row, t.rows * row, 0, out ? 1u : 0u};
    return {p, p + (t.rows - 1) * ld + row, row, ld, out ? 1u : 0u};
}
// outputs apart from each other, from other tensors' gradients and from the norm; the norm from the gradients too where it is written
static int clip_overlaps(const slz_grad_tensor *t, uint32_t count, const float *norm, bool norm_given) {
    clip_place *p = (clip_place *)malloc(sizeof(clip_place) * (2 * (size_t)count + 1));
    if (!p) return SLZ_E_NOMEM;
    size_t n = 0;
    p[n++] = {(uintptr_t)norm, (uintptr_t)norm + 4, 4, 0, norm_given ? 0u : 1u};
    int rc = SLZ_OK;
    for (uint32_t i = 0; i < count && rc == SLZ_OK; i++) {
        if (t[i].rows == 0 || t[i].cols == 0) continue;
        p[n++] = place_of(t[i], true);
        if (t[i].out == t[i].g) rc = t[i].rows > 1 && t[i].ld_out != t[i].ld_g ? SLZ_E_INVALID_ARG : SLZ_OK;
        else p[n++] = place_of(t[i], false);
    }
    std::sort(p, p + n, [](const clip_place &a, const clip_place &b) { return a.begin < b.begin; });
    for (size_t i = 0; i < n && rc == SLZ_OK; i++)
        for (size_t j = i + 1; j < n && p[j].begin < p[i].end && rc == SLZ_OK; j++)
            if ((p[i].out || p[j].out) && clip_meet(p[i], p[j])) rc = SLZ_E_INVALID_ARG;
    free(p);
    return rc;
}

struct clip_plan { clip_work work; uint32_t groups, tensors; size_t first, desc, total; };
static int clip_plan_of(const slz_grad_tensor *t, uint32_t count, clip_plan &P) {
    uint64_t elements = 0;
    P.tensors = 0;
    for (uint32_t i = 0; i < count; i++) {
        const uint64_t n = (uint64_t)t[i].rows * t[i].cols;
        if ((elements += n) > ((uint64_t)1 << 50)) return SLZ_E_TOO_LARGE;
        P.tensors += n != 0;
    }
    // small chunks fill the chip with little, large ones are found and begun less often
    uint32_t chunk = 2048;
    while (chunk < 32768u && elements / chunk > 4 * CLIP_GROUPS) chunk *= 2;
    uint64_t chunks = 0;
    for (uint32_t i = 0; i < count; i++) chunks += ((uint64_t)t[i].rows * t[i].cols + chunk - 1) / chunk;
    if (chunks > 0xffff0000u) return SLZ_E_TOO_LARGE;
    P.work = {P.tensors, (uint32_t)chunks, chunk};
    P.groups = chunks < CLIP_GROUPS ? (uint32_t)chunks : CLIP_GROUPS;
    P.first = up256(P.groups * sizeof(double));
    P.desc = P.first + (P.tensors > CLIP_INLINE ? up256((size_t)P.tensors * 4) : 0);
    P.total = P.desc + (P.tensors > CLIP_INLINE ? up256((size_t)P.tensors * sizeof(clip_desc)) : 0);
    return SLZ_OK;
}
extern "C" int slz_clip_workspace(const slz_grad_tensor *t, uint32_t count, size_t *bytes) {
    int rc = clip_check(t, count, false);
    if (rc != SLZ_OK) return rc;
    if (!bytes) return SLZ_E_INVALID_ARG;
    clip_plan P;
    rc = clip_plan_of(t, count, P);
    if (rc == SLZ_OK) *bytes = P.total;
    return rc;
}
// the kernels with their table: in their arguments, or in the workspace, filled first
template <class F> static void with_table(const slz_grad_tensor *t, uint32_t count, const clip_plan &P, bool outputs, char *ws, hipStream_t s, const F &run) {
    uint32_t at = 0, done = 0;
    uint64_t chunk = 0;
    uint32_t *first = (uint32_t *)(ws + P.first);
    clip_desc *desc = (clip_desc *)(ws + P.desc);
    const auto is_run = [&](const slz_grad_tensor &g) { return g.rows == 1 || (g.ld_g == (int64_t)g.cols && (!outputs || g.ld_out == (int64_t)g.cols)); };
    bool all = P.tensors > CLIP_INLINE;
    for (uint32_t i = 0; i < count && all; i++) all = is_run(t[i]) || t[i].rows == 0 || t[i].cols == 0;
    if (all) {
        clip_runs runs;
        for (uint32_t i = 0, before = 0; i < count; i++) {
            const uint64_t n = (uint64_t)t[i].rows * t[i].cols;
            if (n == 0) continue;
            runs.run[at] = {(const char *)t[i].g, (char *)t[i].out, n << 2 | (uint32_t)t[i].type};
            chunk += (n + P.work.chunk - 1) / P.work.chunk;
            if (++at < CLIP_RUNS && done + at < P.tensors) continue;
            hipLaunchKernelGGL(k_clip_runs, dim3(1), dim3(256), 0, s, runs, done, at, before, P.work.chunk, first, desc);
            before = (uint32_t)chunk;
            done += at;
            at = 0;
        }
        return run(clip_table{first, desc});
    }
    clip_few few;
    for (uint32_t i = 0; i < count; i++) {
        const uint64_t n = (uint64_t)t[i].rows * t[i].cols;
        if (n == 0) continue;
        const bool run_of = is_run(t[i]);
        few.first[at] = (uint32_t)chunk;
        few.desc[at] = {(const char *)t[i].g, (char *)t[i].out, n, t[i].ld_g, t[i].ld_out, run_of ? 0u : t[i].cols, t[i].type};
        chunk += (n + P.work.chunk - 1) / P.work.chunk;
        if (++at < CLIP_INLINE || P.tensors <= CLIP_INLINE) continue;
        hipLaunchKernelGGL(k_clip_table, dim3(1), dim3(64), 0, s, few, done, at, first, desc);
        done += at;
        at = 0;
    }
    if (P.tensors <= CLIP_INLINE) return run(few);
    if (at) hipLaunchKernelGGL(k_clip_table, dim3(1), dim3(64), 0, s, few, done, at, first, desc);
    run(clip_table{first, desc});
}

extern "C" int slz_grad_norm(const slz_grad_tensor *t, uint32_t count, float *norm, void *ws, size_t ws_bytes, void *stream) {
    int rc = clip_check(t, count, false);
    if (rc == SLZ_OK) rc = slz_matrix_check(norm, 1, 1, 1, 4);
    clip_plan P;
    if (rc == SLZ_OK) rc = clip_plan_of(t, count, P);
    if (rc != SLZ_OK) return rc;
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    double *partial = (double *)ws;
    if (P.tensors)
        with_table(t, count, P, false, (char *)ws, s, [&](const auto &table) {
            hipLaunchKernelGGL(k_squares<typename std::decay<decltype(table)>::type>, dim3(P.groups), dim3(256), 0, s, table, P.work, partial);
        });
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(256), 0, s, partial, P.groups, norm);
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

extern "C" int slz_clip_by_norm(const slz_grad_tensor *t, uint32_t count, float max_norm, float eps, int norm_given, float *norm, void *ws, size_t ws_bytes, void *stream) {
    if (!(max_norm >= 0.0f) || !(eps >= 0.0f)) return SLZ_E_INVALID_ARG;
    int rc = clip_check(t, count, true);
    if (rc == SLZ_OK) rc = slz_matrix_check(norm, 1, 1, 1, 4);
    if (rc == SLZ_OK) rc = clip_overlaps(t, count, norm, norm_given != 0);
    clip_plan P;
    if (rc == SLZ_OK) rc = clip_plan_of(t, count, P);
    if (rc != SLZ_OK) return rc;
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    double *partial = (double *)ws;
    if (P.tensors == 0) {
        if (!norm_given) hipLaunchKernelGGL(k_norm, dim3(1), dim3(256), 0, s, partial, 0u, norm);
    } else
        with_table(t, count, P, true, (char *)ws, s, [&](const auto &table) {
            using T = typename std::decay<decltype(table)>::type;
            if (!norm_given) hipLaunchKernelGGL(k_squares<T>, dim3(P.groups), dim3(256), 0, s, table, P.work, partial);
            hipLaunchKernelGGL(k_clip<T>, dim3(P.groups), dim3(256), 0, s, table, P.work, norm_given ? (const double *)nullptr : partial, P.groups, max_norm, eps, norm);
        });
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
