// Softmax cross entropy of a linear layer's outputs z = h w^T over a large vocabulary, and its gradient, without keeping z
// (include/silenzio_clear.h).
//
// Forward: the tiled product; from a tile's z in its registers the maximum and the sum of exp(z - maximum) of each 32 words go to memory, and
// the label's z; a second kernel joins a token's pairs.
// Gradient: in pieces of the vocabulary, z again, from it g = (exp(z - lse) - [v = label]) dloss to the workspace, then the two products
// dw = g^T h (complete for the piece's rows) and dh += g w (summed over the pieces in 32 bits).
// Bound by the matrix cores where rows are long: 4096 tokens x 4096 x 131072 bf16: forward 3.46 ms (1.27 PFLOP/s), each 16384 words' g 482 us (1.14),
// dw 538 (1.02), dh 516 (1.06).  Short rows leave the epilogues: 1003 x 768 x 50021 f16: forward 110 us (0.70), g 142 (0.54), dw 118, dh 108; tiles of 256 instead of
// the 128 taken were no faster for z (105 and, before labels and factors were read ahead, 163 to 160), and slower for dw (product alone 114, 128 with 192, 103 with 128).
#include "slz_gemm.h"

// a piece's g takes this much at most (at least 1024 words of the vocabulary)
#define CE_PIECE_BYTES ((size_t)128 << 20)
#define CE_PIECE_WORDS ((size_t)1 << 21)     // rows of g stay as short as any operand's
// bf16 and f16: g is held relative to the largest |dloss| that counts.  Losses are often weighted alike (a mean), and then the label's g, -1 + p, loses little,
// where the rounding of -dloss would be the same for all tokens: an error of all of dh and dw of up to 2^-8 (bf16) or 2^-11 (f16).
// f16: times CE_F16_UP; |g| <= |dloss|, so that the largest stay finite and those from 2^-28 of the largest keep 11 bits
#define CE_F16_UP 16384.0f

// (maximum, sum of exp(z - maximum)) of two sets of z; a set whose z are all -inf has (-inf, 0) and adds nothing
__device__ __forceinline__ float2 ce_both(float2 p, float2 q) {
    const float top = fmaxf(p.x, q.x), from = top == -__builtin_inff() ? 0.0f : top;
    return make_float2(top, p.y * __expf(p.x - from) + q.y * __expf(q.x - from));
}

// which of `count` words from `first` on the label is, or -1
__device__ __forceinline__ int ce_word(int64_t label, uint32_t first, uint32_t count) {
    const uint64_t d = (uint64_t)label - first;
    return d < count ? (int)d : -1;
}

// One pair for every 32 words, whatever the tiling: sums of eight, then of four such.  A token's loss so has the same bits alone and among others.
#define CE_BLOCK 32
struct ce_lse_epi {
    static constexpr int widest = 256;
    static constexpr bool any_side = false;            // blocks of 32 words lie within a wave's columns
    float2 *pairs;                   // [block of words][tokens]
    float *label_z;
    const int64_t *labels;
    uint32_t first_word;             // a multiple of CE_BLOCK
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *) const {
        static_assert(RUN && (NI == 2 || NI == 4), "a lane has 8 or 16 columns, four or two lanes a block");
        if (at.n0 + NI * 16u <= p.N) part<MI, NI, RUN, true>(acc, at, p);
        else part<MI, NI, RUN, false>(acc, at, p);
    }
    // WHOLE: all the wave's columns are words
    template <int MI, int NI, bool RUN, bool WHOLE, class ACC>
    __device__ __forceinline__ void part(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p) const {
        const uint32_t n0 = slz_col<NI, RUN>(at, 0);
        int words[MI];                                 // read for all rows before the first is written
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
            words[i] = m < p.M && n0 < p.N ? ce_word(labels[m], first_word + n0, min(NI * 4u, p.N - n0)) : -1;
        }
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
            float top = -__builtin_inff();
#pragma unroll
            for (int c = 0; c < NI * 4; c++) top = WHOLE || n0 + c < p.N ? fmaxf(top, acc[i][c / 4][c % 4]) : top;
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            if (NI == 2) top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float from = top == -__builtin_inff() ? 0.0f : top;
            float sums[NI / 2];
#pragma unroll
            for (int h = 0; h < NI / 2; h++) {
                sums[h] = 0.0f;
#pragma unroll
                for (int c = h * 8; c < h * 8 + 8; c++) sums[h] += WHOLE || n0 + c < p.N ? __expf(acc[i][c / 4][c % 4] - from) : 0.0f;
            }
            float sum = sums[0];
            if (NI == 4) sum += sums[NI / 2 - 1];
            sum += __shfl_xor(sum, 16, 64);
            if (NI == 2) sum += __shfl_xor(sum, 32, 64);
            if (m >= p.M || n0 >= p.N) continue;
            const int word = words[i];
            if (word >= 0) {
                float z = 0.0f;
#pragma unroll
                for (int c = 0; c < NI * 4; c++) z = word == c ? acc[i][c / 4][c % 4] : z;
                label_z[m] = z;
            }
            if (n0 % CE_BLOCK == 0) pairs[(size_t)((first_word + n0) / CE_BLOCK) * p.M + m] = make_float2(top, sum);
        }
    }
};

// 16 tokens per workgroup; each token's blocks go to 64 threads in turn, whose pairs are joined in a fixed order.  Bound by memory (4096 tokens x 4096
// blocks: 28.6 us, 4.7 TB/s), for few tokens by latency (8 x 2048: 6.7 us).  256 threads a token: 4.7 there, but 11.2 instead of 8.2 for 1003 x 1564.
__global__ void __launch_bounds__(1024)
k_ce_join(const float2 *__restrict__ pairs, const float *__restrict__ label_z, const int64_t *__restrict__ labels, float *__restrict__ loss,
          float *__restrict__ lse, uint32_t tokens, uint32_t blocks, uint32_t vocab, int64_t ignore) {
    __shared__ float2 part[64][16];
    const uint32_t r = threadIdx.x & 15u, slice = threadIdx.x >> 4, t = (blockIdx.y * gridDim.x + blockIdx.x) * 16 + r;
    float2 all = make_float2(-__builtin_inff(), 0.0f);
    if (t < tokens)
        for (uint32_t i = slice; i < blocks; i += 64 * 8) {
            float2 some[8];
#pragma unroll
            for (int q = 0; q < 8; q++) some[q] = i + q * 64 < blocks ? pairs[(size_t)(i + q * 64) * tokens + t] : make_float2(-__builtin_inff(), 0.0f);
            float top = all.x;
#pragma unroll
            for (int q = 0; q < 8; q++) top = fmaxf(top, some[q].x);
            const float from = top == -__builtin_inff() ? 0.0f : top;
            all.y *= __expf(all.x - from);
            all.x = top;
#pragma unroll
            for (int q = 0; q < 8; q++) all.y += some[q].y * __expf(some[q].x - from);
        }
    part[slice][r] = all;
    for (uint32_t half = 32; half > 0; half >>= 1) {
        __syncthreads();
        if (slice < half) part[slice][r] = ce_both(part[slice][r], part[slice + half][r]);
    }
    if (slice != 0 || t >= tokens) return;
    const float l = part[0][r].x + logf(part[0][r].y);
    const int64_t label = labels[t];
    lse[t] = l;
    loss[t] = label == ignore ? 0.0f : label < 0 || label >= (int64_t)vocab ? __builtin_nanf("") : l - label_z[t];
}

// g of a piece: [pieces][tokens][ld], columns from N to the next multiple of 8 zero
struct ce_grad_epi {
    static constexpr int widest = 256;
    static constexpr bool any_side = false;            // eight columns of a lane at a time
    char *g;
    int64_t ld, piece;               // bytes
    int type;
    const float *lse, *dloss, *unit;
    const int64_t *labels;
    int64_t ignore;
    uint32_t first_word, vocab;
    template <int MI, int NI, bool RUN, int WM, int WN, class ACC>
    __device__ __forceinline__ void run(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p, float *) const {
        static_assert(RUN && NI % 2 == 0, "");
        if (at.n0 + NI * 16u <= p.N) part<MI, NI, RUN, true>(acc, at, p);
        else part<MI, NI, RUN, false>(acc, at, p);
    }
    template <int MI, int NI, bool RUN, bool WHOLE, class ACC>
    __device__ __forceinline__ void part(const ACC (&acc)[MI][NI], const slz_place &at, const slz_gemm &p) const {
        const uint32_t n0 = slz_col<NI, RUN>(at, 0), wide = (p.N + 7u) & ~7u;
        const float up = type == SLZ_F32 ? 1.0f : (type == SLZ_F16 ? CE_F16_UP : 1.0f) / *unit;
        float bys[MI], ls[MI];                         // read for all rows before the first is written
        int words[MI];                                 // -2: not counted
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = min(slz_row(at, i), p.M - 1u);
            const int64_t label = labels[m];
            const float d = dloss[m] * up;
            ls[i] = lse[m];
            bys[i] = label < 0 || label >= (int64_t)vocab ? __builtin_nanf("") : d;
            words[i] = label == ignore ? -2 : ce_word(label, first_word + n0, NI * 4);
        }
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const uint32_t m = slz_row(at, i);
            if (m >= p.M) continue;
            const bool counts = words[i] != -2;
            const float by = bys[i], l = ls[i];
            const int word = words[i];
#pragma unroll
            for (int q = 0; q < NI / 2; q++) {
                const uint32_t n = n0 + q * 8u;
                if (!WHOLE && n >= wide) continue;
                float v[8];
#pragma unroll
                for (int c = 0; c < 8; c++) {
                    const float z = acc[i][q * 2 + c / 4][c % 4], e = type == SLZ_F32 ? expf(z - l) : __expf(z - l);
                    v[c] = counts && (WHOLE || n + c < p.N) ? (e - (word == q * 8 + c ? 1.0f : 0.0f)) * by : 0.0f;
                }
                char *to = g + (int64_t)m * ld + (int64_t)n * 2;
                if (type == SLZ_F32) {
                    uint32_t w[3][4];
#pragma unroll
                    for (int c = 0; c < 8; c += 2) {
                        uint16_t x[3], y[3];
                        slz_split3(v[c], x);
                        slz_split3(v[c + 1], y);
                        for (int k = 0; k < 3; k++) w[k][c / 2] = x[k] | ((uint32_t)y[k] << 16);
                    }
                    for (int k = 0; k < 3; k++) *(uint4 *)(to + k * piece) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
                } else slz_put_run<8>(to, type, v, 8, true);
            }
        }
    }
};

// ---- few classes ---------------------------------------------------------------------------------------------------------------------------
// A classifier's head: w fits a workgroup's shared memory in 32 bits, a wave computes all of a token's z, and the whole call is one launch (the
// gradient of many tokens: two), where the tiled products would be four to eight.  Taken by the sizes of w alone, so that a token's loss does not
// depend on how many there are.  32 tokens x 128 x 10: loss 6.2 us, gradient 14.6 in its one workgroup, both less than the host's time for a call.
#define FEW_CLASSES 16
#define FEW_INNER 512                // longer rows leave too few tokens of a workgroup at a time
#define FEW_WEIGHTS (FEW_CLASSES * FEW_INNER)
#define FEW_THREADS 1024
#define FEW_TOKENS_LDS 16384         // entries of h that a workgroup holds
#define FEW_BLOCKS 256
struct few_args {
    const void *h, *w;
    int type;
    int64_t ld_h, ld_w;
    const int64_t *labels;
    int64_t ignore;
    uint32_t tokens, inner, vocab;
};
// rows of w or h to shared memory in 32 bits, a wave a row, four loads under way
template <int TYPE> __device__ __forceinline__ void few_rows_of(const void *x, int64_t ld, uint32_t rows, uint32_t inner, float *to) {
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t r = threadIdx.x >> 6; r < rows; r += FEW_THREADS / 64)
        for (uint32_t d0 = lane; d0 < inner; d0 += 256) {
            float v[4];
#pragma unroll
            for (uint32_t q = 0; q < 4; q++) v[q] = slz_get(x, TYPE, (size_t)r * ld + min(d0 + q * 64, inner - 1));
#pragma unroll
            for (uint32_t q = 0; q < 4; q++)
                if (d0 + q * 64 < inner) to[r * inner + d0 + q * 64] = v[q];
        }
}
__device__ __forceinline__ void few_rows(const void *x, int type, int64_t ld, uint32_t rows, uint32_t inner, float *to) {
    if (type == SLZ_F32) few_rows_of<SLZ_F32>(x, ld, rows, inner, to);
    else if (type == SLZ_BF16) few_rows_of<SLZ_BF16>(x, ld, rows, inner, to);
    else few_rows_of<SLZ_F16>(x, ld, rows, inner, to);
}
// Softmax of a token by a wave: lane v has z of class v (-inf behind the last), and gets the logarithm of the sum of exp.
template <int C> __device__ __forceinline__ float few_logits(const float *h, const float *w, uint32_t inner, uint32_t vocab, uint32_t lane) {
    float z[C];
#pragma unroll
    for (int v = 0; v < C; v++) z[v] = 0.0f;
    for (uint32_t d = lane; d < inner; d += 64) {
        const float x = h[d];
#pragma unroll
        for (int v = 0; v < C; v++)
            if ((uint32_t)v < vocab) z[v] = __builtin_fmaf(x, w[v * inner + d], z[v]);
    }
    float own = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < C; v++)
        if ((uint32_t)v < vocab) {
            const float sum = slz_wave_sum(z[v]);
            own = lane == (uint32_t)v ? sum : own;
        }
    return own;
}
__device__ __forceinline__ float few_lse(float own, bool real) {
    const float top = slz_wave_max(own), from = top == -__builtin_inff() ? 0.0f : top;
    return top + logf(slz_wave_sum(real ? expf(own - from) : 0.0f));
}

// `group` tokens at a time
template <int C>
__global__ void __launch_bounds__(FEW_THREADS) k_few_loss(const few_args p, uint32_t group, float *__restrict__ loss, float *__restrict__ lse) {
    extern __shared__ __attribute__((aligned(16))) float few[];
    float *w = few, *h = few + p.vocab * p.inner;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    few_rows(p.w, p.type, p.ld_w, p.vocab, p.inner, w);
    for (uint32_t first = blockIdx.x * group; first < p.tokens; first += gridDim.x * group) {
        const uint32_t count = min(group, p.tokens - first);
        const int64_t own_label = lane < count ? p.labels[first + lane] : 0;            // group is 32 at most
        few_rows((const char *)p.h + (size_t)first * p.ld_h * slz_type_bytes(p.type), p.type, p.ld_h, count, p.inner, h);
        __syncthreads();
        for (uint32_t t = wave; t < count; t += FEW_THREADS / 64) {
            const float z = few_logits<C>(h + t * p.inner, w, p.inner, p.vocab, lane), l = few_lse(z, lane < p.vocab);
            const int64_t label = __shfl(own_label, (int)t, 64);
            const bool inside = label >= 0 && label < (int64_t)p.vocab;
            const float at_label = __shfl(z, inside ? (int)label : 0, 64);
            if (lane == 0) {
                lse[first + t] = l;
                loss[first + t] = label == p.ignore ? 0.0f : inside ? l - at_label : __builtin_nanf("");
            }
        }
        __syncthreads();
    }
}

// dw: the sums of each workgroup's tokens go to `part` [workgroup][vocab][inner], or with one workgroup to dw
// OWN: entries of dw of a thread
template <int C, int OWN>
__global__ void __launch_bounds__(FEW_THREADS)
k_few_grad(const few_args p, uint32_t group, const float *__restrict__ lse, const float *__restrict__ dloss, void *__restrict__ dh, int64_t ld_dh,
           void *__restrict__ dw, int64_t ld_dw, float *__restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) float few[];
    const uint32_t weights = p.vocab * p.inner;
    float *w = few, *g = w + weights, *h = g + group * p.vocab;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    float sum[OWN];
    uint32_t own_at[OWN];                              // class and place in the row
#pragma unroll
    for (int i = 0; i < OWN; i++) {
        const uint32_t e = i * FEW_THREADS + threadIdx.x;
        sum[i] = 0.0f;
        own_at[i] = e < weights ? (e / p.inner) << 16 | e % p.inner : 0u;
    }
    few_rows(p.w, p.type, p.ld_w, p.vocab, p.inner, w);
    for (uint32_t first = blockIdx.x * group; first < p.tokens; first += gridDim.x * group) {
        const uint32_t count = min(group, p.tokens - first);
        const int64_t own_label = lane < count ? p.labels[first + lane] : 0;            // group is 32 at most
        const float own_lse = lane < count ? lse[first + lane] : 0.0f, own_dloss = lane < count ? dloss[first + lane] : 0.0f;
        few_rows((const char *)p.h + (size_t)first * p.ld_h * slz_type_bytes(p.type), p.type, p.ld_h, count, p.inner, h);
        __syncthreads();
        for (uint32_t t = wave; t < count; t += FEW_THREADS / 64) {
            const float z = few_logits<C>(h + t * p.inner, w, p.inner, p.vocab, lane), l = __shfl(own_lse, (int)t, 64);
            const int64_t label = __shfl(own_label, (int)t, 64);
            const float by = label < 0 || label >= (int64_t)p.vocab ? __builtin_nanf("") : __shfl(own_dloss, (int)t, 64);
            const float own = label == p.ignore ? 0.0f : (expf(z - l) - (label == (int64_t)lane ? 1.0f : 0.0f)) * by;
            if (lane < p.vocab) g[t * p.vocab + lane] = own;
            for (uint32_t d = lane; d < p.inner; d += 64) {
                float x = 0.0f;
#pragma unroll
                for (int v = 0; v < C; v++)
                    if ((uint32_t)v < p.vocab) x = __builtin_fmaf(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, own), v)), w[v * p.inner + d], x);
                slz_put(dh, p.type, (size_t)(first + t) * ld_dh + d, x);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < OWN; i++)
            if ((uint32_t)i * FEW_THREADS < weights) {
                const float *gi = g + (own_at[i] >> 16), *hi = h + (own_at[i] & 0xffffu);
#pragma unroll 2
                for (uint32_t t = 0; t < count; t++) sum[i] = __builtin_fmaf(gi[t * p.vocab], hi[t * p.inner], sum[i]);
            }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < OWN; i++) {
        const uint32_t e = i * FEW_THREADS + threadIdx.x;
        if (e >= weights) continue;
        if (part) part[(size_t)blockIdx.x * weights + e] = sum[i];
        else slz_put(dw, p.type, (size_t)(own_at[i] >> 16) * ld_dw + (own_at[i] & 0xffffu), sum[i]);
    }
}
__global__ void __launch_bounds__(256)
k_few_join(const float *__restrict__ part, uint32_t blocks, uint32_t vocab, uint32_t inner, void *__restrict__ dw, int type, int64_t ld_dw) {
    const uint32_t e = blockIdx.x * 256 + threadIdx.x, weights = vocab * inner;
    if (e >= weights) return;
    float sum = 0.0f;
    for (uint32_t b = 0; b < blocks; b++) sum += part[(size_t)b * weights + e];
    slz_put(dw, type, (size_t)(e / inner) * ld_dw + e % inner, sum);
}

static bool few_takes(const slz_ce_shape *sh) { return sh->vocab <= FEW_CLASSES && sh->inner <= FEW_INNER; }
// tokens a workgroup takes at a time, `most` or what its shared memory holds, and workgroups.  Loss: a token for each of its waves; gradient: two, since
// the second launch costs more
static uint32_t few_group(const slz_ce_shape *sh, uint32_t most) {
    const uint32_t fit = FEW_TOKENS_LDS / sh->inner;
    return fit < 1 ? 1 : fit > most ? most : fit;
}
static uint32_t few_blocks(const slz_ce_shape *sh, uint32_t group) {
    const uint32_t n = (sh->tokens + group - 1) / group;
    return n < 1 ? 1 : n > FEW_BLOCKS ? FEW_BLOCKS : n;
}
static size_t few_workspace(const slz_ce_shape *sh) {
    const uint32_t blocks = few_blocks(sh, few_group(sh, 32));
    return blocks == 1 ? 0 : up256((size_t)blocks * sh->vocab * sh->inner * 4);
}
static few_args few_of(const slz_ce_shape *sh, const void *h, const void *w, const int64_t *labels) {
    return {h, w, sh->type, sh->ld_h, sh->ld_w, labels, sh->ignore_index, sh->tokens, sh->inner, sh->vocab};
}
static int few_loss(const slz_ce_shape *sh, const void *h, const void *w, const int64_t *labels, float *loss, float *lse, hipStream_t s) {
    const uint32_t group = few_group(sh, 16);
    const auto k = sh->vocab <= 8 ? k_few_loss<8> : k_few_loss<16>;
    hipLaunchKernelGGL(k, dim3(few_blocks(sh, group)), dim3(FEW_THREADS), (sh->vocab + group) * sh->inner * 4, s, few_of(sh, h, w, labels), group, loss, lse);
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}
static int few_grad(const slz_ce_shape *sh, const void *h, const void *w, const int64_t *labels, const float *lse, const float *dloss, void *dh, void *dw,
                    float *part, hipStream_t s) {
    const uint32_t group = few_group(sh, 32), blocks = few_blocks(sh, group);
    const bool small = sh->vocab * sh->inner <= 2 * FEW_THREADS;
    constexpr int all = FEW_WEIGHTS / FEW_THREADS;
    const auto k = small ? k_few_grad<16, 2> : k_few_grad<16, all>;
    hipLaunchKernelGGL(k, dim3(blocks), dim3(FEW_THREADS), ((sh->vocab + group) * sh->inner + group * sh->vocab) * 4, s, few_of(sh, h, w, labels), group, lse,
                       dloss, dh, sh->ld_dh, dw, sh->ld_dw, blocks > 1 ? part : nullptr);
    if (blocks > 1)
        hipLaunchKernelGGL(k_few_join, dim3((sh->vocab * sh->inner + 255) / 256), dim3(256), 0, s, part, blocks, sh->vocab, sh->inner, dw, sh->type, sh->ld_dw);
    return hipGetLastError() == hipSuccess ? SLZ_OK : SLZ_E_HIP;
}

struct ce_plan {
    uint32_t words;                  // of a piece
    size_t h, w, pairs, label_z, g, dh, dw, unit, total;
    uint32_t g_row, dh_ld;
    uint32_t side;                   // of the tiles of z
    slz_choice dh_choice, dw_choice;
};
static ce_plan plan_ce(const slz_ce_shape *sh, const void *h, const void *w, bool grad) {
    ce_plan P = {};
    const size_t pieces = sh->type == SLZ_F32 ? 3 : 1;
    const bool w_there = slz_operand_bytes(w, sh->type, 1, sh->inner, sh->ld_w) == 0;
    // words of a piece, and of them a multiple that gives whole rounds of tiles on 256 compute units where it fits (4096 tokens: 4096; 4096 x 4096
    // x 131072 takes 15.2 ms in pieces of 8192, 16384 or 131072 words and 15.9 in five of 26368)
    size_t words = sh->vocab;
    const size_t for_g = CE_PIECE_BYTES / (2 * pieces * (sh->tokens ? sh->tokens : 1)), for_w = CE_PIECE_BYTES / (2 * pieces * sh->inner);
    if (grad && words > for_g) words = for_g;
    if (grad && words > CE_PIECE_WORDS) words = CE_PIECE_WORDS;
    if (!w_there && words > for_w) words = for_w;
    if (words < sh->vocab) {
        uint32_t unit = 65536, rows = (sh->tokens + 255) / 256;
        for (; unit > 256 && rows && rows % 2 == 0; rows /= 2) unit /= 2;
        words = words >= unit ? words / unit * unit : words >= 1024 ? words & ~(size_t)255 : 1024;
    }
    P.words = (uint32_t)(words < sh->vocab ? words : sh->vocab);
    const uint32_t pairs = sh->type == SLZ_F32 ? 6 : 1;
    P.side = slz_choose(sh->tokens, P.words, (sh->inner + 63) / 64 * pairs, 1, false, 1, false, false).side;
    size_t o = 0;
    P.h = o; o += slz_operand_bytes(h, sh->type, sh->tokens, sh->inner, sh->ld_h);
    P.w = o; o += slz_operand_bytes(w, sh->type, P.words, sh->inner, sh->ld_w);
    if (!grad) {
        P.pairs = o; o += up256(((size_t)sh->vocab + CE_BLOCK - 1) / CE_BLOCK * sh->tokens * 8);
        P.label_z = o; o += up256((size_t)sh->tokens * 4);
    } else {
        P.g_row = (uint32_t)(((size_t)P.words * 2 + 127) / 128 * 128);
        P.g = o; o += pieces * up256((size_t)sh->tokens * P.g_row);
        P.dh_ld = slz_ranges_ld(sh->inner);
        // dh: one launch over a piece, or its sums kept in ranges of the piece's words, to which each piece adds
        P.dh_choice = slz_choose(sh->tokens, sh->inner, (P.words + 63) / 64 * pairs, 1, false, 64, true);
        P.dw_choice = slz_choose(P.words, sh->inner, (sh->tokens + 63) / 64 * pairs, 1, false, 32, true);
        P.dw = o; o += slz_ranges_bytes(P.dw_choice, P.words, sh->inner);
        P.dh = o; o += P.words < sh->vocab || P.dh_choice.split > 1 ? up256((size_t)P.dh_choice.split * sh->tokens * P.dh_ld * 4) : 0;
        P.unit = o; o += 256;
    }
    P.total = o;
    return P;
}

static int ce_check(const slz_ce_shape *sh, const void *h, const void *w, const int64_t *labels) {
    if (!sh || !slz_type_ok(sh->type) || sh->inner == 0 || sh->vocab == 0) return SLZ_E_INVALID_ARG;
    const uint32_t eb = slz_type_bytes(sh->type);
    int rc = slz_matrix_check(h, sh->tokens, sh->inner, sh->ld_h, eb);
    if (rc == SLZ_OK) rc = slz_matrix_check(w, sh->vocab, sh->inner, sh->ld_w, eb);
    if (rc == SLZ_OK) rc = slz_matrix_check(labels, sh->tokens, 1, 1, 8);
    return rc;
}
static int ce_workspace(const slz_ce_shape *sh, const void *h, const void *w, bool grad, size_t *bytes) {
    if (!sh || !bytes || !slz_type_ok(sh->type) || sh->inner == 0 || sh->vocab == 0) return SLZ_E_INVALID_ARG;
    if (sh->tokens > SLZ_CLEAR_MAX_LEN || sh->vocab > SLZ_CLEAR_MAX_LEN || sh->inner > SLZ_CLEAR_MAX_LD) return SLZ_E_TOO_LARGE;
    *bytes = few_takes(sh) ? (grad ? few_workspace(sh) : 0) : plan_ce(sh, h, w, grad).total;
    return SLZ_OK;
}
extern "C" int slz_linear_ce_workspace(const slz_ce_shape *sh, const void *h, const void *w, size_t *bytes) { return ce_workspace(sh, h, w, false, bytes); }
extern "C" int slz_linear_ce_grad_workspace(const slz_ce_shape *sh, const void *h, const void *w, size_t *bytes) {
    return ce_workspace(sh, h, w, true, bytes);
}

template <class EPI> static int ce_logits(int type, const slz_gemm &p, const EPI &epi, uint32_t side, hipStream_t s) {
    return type == SLZ_F16 ? slz_gemm_run<SLZ_EL_F16, false, false>(p, epi, side, 1, s) : slz_gemm_run<SLZ_EL_BF16, false, false>(p, epi, side, 1, s);
}
static const char *rows_of(const void *w, const slz_ce_shape *sh, uint32_t first) {
    return (const char *)w + (int64_t)first * sh->ld_w * slz_type_bytes(sh->type);
}

extern "C" int slz_linear_ce(const slz_ce_shape *sh, const void *h, const void *w, const int64_t *labels, float *loss, float *lse, void *ws,
                             size_t ws_bytes, void *stream) {
    int rc = ce_check(sh, h, w, labels);
    if (rc == SLZ_OK) rc = slz_matrix_check(loss, sh->tokens, 1, 1, 4);
    if (rc == SLZ_OK) rc = slz_matrix_check(lse, sh->tokens, 1, 1, 4);
    if (rc != SLZ_OK || sh->tokens == 0) return rc;
    if (few_takes(sh)) return few_loss(sh, h, w, labels, loss, lse, (hipStream_t)stream);
    const ce_plan P = plan_ce(sh, h, w, false);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    char *base = (char *)ws;
    float2 *pairs = (float2 *)(base + P.pairs);
    float *label_z = (float *)(base + P.label_z);
    slz_layouts jobs = {};
    const slz_operand oh = slz_operand_of(h, sh->type, sh->tokens, sh->inner, sh->ld_h, base + P.h, jobs);
    for (uint32_t v = 0; v < sh->vocab; v += P.words) {
        const uint32_t words = sh->vocab - v < P.words ? sh->vocab - v : P.words;
        const slz_operand ow = slz_operand_of(rows_of(w, sh, v), sh->type, words, sh->inner, sh->ld_w, base + P.w, jobs);
        slz_layout_run(jobs, s);                       // with h before the first piece
        jobs.count = 0;
        const ce_lse_epi epi{pairs, label_z, labels, v};
        rc = ce_logits(sh->type, slz_gemm_of(oh, ow, sh->tokens, words, sh->inner), epi, P.side, s);
        if (rc != SLZ_OK) return rc;
    }
    const uint32_t joins = (sh->tokens + 15) / 16, most = slz_most_blocks(1024), along = joins < most ? joins : most;
    hipLaunchKernelGGL(k_ce_join, dim3(along, (joins + along - 1) / along), dim3(1024), 0, s, pairs, label_z, labels, loss, lse, sh->tokens, (sh->vocab + CE_BLOCK - 1) / CE_BLOCK,
                       sh->vocab, sh->ignore_index);
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}

template <int EL> static int ce_products(const slz_ce_shape *sh, const ce_plan &P, const slz_operand &g, const slz_operand &oh, const slz_operand &ow,
                                         uint32_t first, uint32_t words, void *dh, void *dw, float *dh_sum, char *dw_ranges, const slz_times_unit &f, hipStream_t s) {
    char *dw_rows = (char *)dw + (int64_t)first * sh->ld_dw * slz_type_bytes(sh->type);
    int rc = slz_gemm_to<EL, true, true>(slz_gemm_of(g, oh, words, sh->inner, sh->tokens), P.dw_choice, f, dw_rows, sh->type, sh->ld_dw, dw_ranges, s);
    if (rc != SLZ_OK) return rc;
    slz_gemm p = slz_gemm_of(g, ow, sh->tokens, sh->inner, words);
    if (P.words == sh->vocab) return slz_gemm_to<EL, false, true>(p, P.dh_choice, f, dh, sh->type, sh->ld_dh, (char *)dh_sum, s);
    p.split = P.dh_choice.split;
    return slz_gemm_run<EL, false, true>(p, slz_partial_epi<float>{dh_sum, P.dh_ld, 1, first != 0}, P.dh_choice.side, 1, s);
}

extern "C" int slz_linear_ce_grad(const slz_ce_shape *sh, const void *h, const void *w, const int64_t *labels, const float *lse, const float *dloss,
                                  void *dh, void *dw, void *ws, size_t ws_bytes, void *stream) {
    int rc = ce_check(sh, h, w, labels);
    if (rc == SLZ_OK) rc = slz_matrix_check(lse, sh->tokens, 1, 1, 4);
    if (rc == SLZ_OK) rc = slz_matrix_check(dloss, sh->tokens, 1, 1, 4);
    if (rc == SLZ_OK) rc = slz_matrix_check(dh, sh->tokens, sh->inner, sh->ld_dh, slz_type_bytes(sh->type));
    if (rc == SLZ_OK) rc = slz_matrix_check(dw, sh->vocab, sh->inner, sh->ld_dw, slz_type_bytes(sh->type));
    if (rc != SLZ_OK) return rc;
    if (few_takes(sh)) {
        if (!slz_ws_ok(ws, ws_bytes, few_workspace(sh))) return SLZ_E_INVALID_ARG;
        return few_grad(sh, h, w, labels, lse, dloss, dh, dw, (float *)ws, (hipStream_t)stream);
    }
    const ce_plan P = plan_ce(sh, h, w, true);
    if (!slz_ws_ok(ws, ws_bytes, P.total)) return SLZ_E_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    char *base = (char *)ws;
    float *dh_sum = (float *)(base + P.dh), *unit = (float *)(base + P.unit);
    if (sh->type != SLZ_F32) slz_unit_of(dloss, sh->tokens, unit, s, labels, sh->ignore_index, sh->vocab);
    const slz_times_unit f{sh->type != SLZ_F32 ? unit : nullptr, sh->type == SLZ_F16 ? 1.0f / CE_F16_UP : 1.0f};
    slz_layouts jobs = {};
    const slz_operand oh = slz_operand_of(h, sh->type, sh->tokens, sh->inner, sh->ld_h, base + P.h, jobs);
    const slz_operand g{base + P.g, (int64_t)P.g_row, (int64_t)up256((size_t)sh->tokens * P.g_row), oh.pieces, oh.element};
    for (uint32_t v = 0; v < sh->vocab; v += P.words) {
        const uint32_t words = sh->vocab - v < P.words ? sh->vocab - v : P.words;
        const slz_operand ow = slz_operand_of(rows_of(w, sh, v), sh->type, words, sh->inner, sh->ld_w, base + P.w, jobs);
        slz_layout_run(jobs, s);                       // with h before the first piece
        jobs.count = 0;
        const ce_grad_epi epi{base + P.g, g.ld, g.piece, sh->type, lse, dloss, unit, labels, sh->ignore_index, v, sh->vocab};
        rc = ce_logits(sh->type, slz_gemm_of(oh, ow, sh->tokens, words, sh->inner), epi, P.side, s);
        if (rc == SLZ_OK)
            rc = sh->type == SLZ_F16 ? ce_products<SLZ_EL_F16>(sh, P, g, oh, ow, v, words, dh, dw, dh_sum, base + P.dw, f, s)
                                     : ce_products<SLZ_EL_BF16>(sh, P, g, oh, ow, v, words, dh, dw, dh_sum, base + P.dw, f, s);
        if (rc != SLZ_OK) return rc;
    }
    if (P.words < sh->vocab && sh->tokens)
        hipLaunchKernelGGL((k_join<float, slz_times_unit>), ew_grid((size_t)sh->tokens * ((sh->inner + 3) / 4)), dim3(256), 0, s, (const float *)dh_sum, P.dh_choice.split,
                           sh->tokens, sh->inner, P.dh_ld, dh, sh->type, sh->ld_dh, f);
    SLZ_HIP(hipGetLastError());
    return SLZ_OK;
}
