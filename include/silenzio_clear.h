/* Training and running a network in the clear, next to the gadgets that do it on ciphertexts (silenzio_gadgets.h): what an
 * encrypted run is compared with.  Scales are any numbers here; the gadgets' block scaling is by powers of two.
 *   slz_quantize_i8, slz_matmul_i8, slz_linear_i8, slz_matmul_i8_grad   products of 8-bit integers with a scale per row
 *   slz_linear_ce, slz_linear_ce_grad     softmax cross entropy of a linear layer's outputs, without keeping them, and its gradient
 *   slz_orthogonalize                     updates orthogonalised by Newton-Schulz products
 *
 * Conventions as in silenzio_pbs.h: C ABI, plain device pointers, the caller owns every buffer, work is enqueued on the given
 * HIP stream of the current device and the call returns at once, return codes are the SLZ_* codes.  Nothing is allocated and
 * nothing is kept between calls; every function can be captured into a HIP graph.  The same inputs give the same bits.
 * Matrices are row-major; a leading dimension ("ld") is the distance of two rows in elements, at least the row's length, and
 * any such distance and any address that is a multiple of the element's size will do.  Operands whose address, row length and
 * row distance are all multiples of 16 bytes are read where they are, others are laid out once per call in the workspace.
 * Workspace: the _workspace function says how many bytes a call of this shape and these addresses (only their alignment is
 * looked at) needs; the buffer starts at a multiple of 256 bytes and may be null where 0 is said.  It must not be used by
 * others until the call's work on the stream is done.
 * A length of zero is no error where a result remains to be defined: outputs without elements are not touched, and a product
 * over nothing is zero.
 * SLZ_E_INVALID_ARG: a null or misaligned pointer where elements are read or written, an unknown type, a leading dimension shorter than a row,
 * a workspace that is too small.  SLZ_E_TOO_LARGE: a length of 2^31 or more, rows further than 2^22 elements apart, or
 * (slz_orthogonalize) 2^22 rows or 2^16 matrices.
 */
#ifndef SILENZIO_CLEAR_H
#define SILENZIO_CLEAR_H
#include <stddef.h>
#include <stdint.h>
#include "silenzio_pbs.h"

#ifdef __cplusplus
extern "C" {
#endif

/* types of floating inputs and outputs */
#define SLZ_F32 0
#define SLZ_BF16 1
#define SLZ_F16 2

/* ---- products of 8-bit integers ------------------------------------------------------------------------------------------ */

/* Row i of x [rows][cols] to 8 bits: top = max_k |x_ik|, scale_i = top / 127, q_ik = rint(x_ik ((1 / top) 127)) (ties to
 * even), each operation in 32-bit floating point; a row of zeros has scale 0 and zeros, a row with an infinity or NaN has scale NaN and zeros. */
int slz_quantize_i8(const void *x_dev, int type, uint32_t rows, uint32_t cols, int64_t ld_x, int8_t *q_dev, int64_t ld_q,
                    float *scale_dev, void *hip_stream);

typedef struct {
    uint32_t m, n, k;                    /* a is m x k, b is n x k, y is m x n */
    int type;                            /* of y, and of x and the gradients */
    int64_t ld_a, ld_b, ld_y;            /* ld_a is x's in slz_linear_i8 */
} slz_i8_shape;

/* y_ij = a_scale_i b_scale_j sum_k a_ik b_jk: the sum exact in 32-bit integers and then rounded to 32-bit floating point, times the
 * product of the scales, each operation in 32 bits, and one rounding to y's type.
 * Entries may be any int8.  SLZ_E_TOO_LARGE also for k >= 2^17, where the sum could leave 32 bits. */
int slz_matmul_i8_workspace(const slz_i8_shape *shape, const int8_t *a_dev, const int8_t *b_dev, size_t *bytes);
int slz_matmul_i8(const slz_i8_shape *shape, const int8_t *a_dev, const float *a_scale_dev, const int8_t *b_dev,
                  const float *b_scale_dev, void *y_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* The same with a the quantised rows of x [m][k] (slz_quantize_i8): a linear layer whose weights the program keeps in 8 bits. */
int slz_linear_i8_workspace(const slz_i8_shape *shape, const void *x_dev, const int8_t *b_dev, size_t *bytes);
int slz_linear_i8(const slz_i8_shape *shape, const void *x_dev, const int8_t *b_dev, const float *b_scale_dev, void *y_dev,
                  void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* Gradients with respect to the values A_ik = a_scale_i a_ik and B_jk = b_scale_j b_jk (the rounding of a quantisation is passed
 * straight through):  da_ik = sum_j dy_ij B_jk,  db_jk = sum_i dy_ij A_ik.  dy is [m][n] with ld_y, da [m][k], db [n][k]; either
 * of the two may be null.  For bf16 and f16 the values A and B are rounded to 8 and 11 bits for the products, which are summed
 * in 32 bits (f16: to fewer in rows whose scale is below 2^-22 of the largest finite one; a single row is not rounded); for f32 they are carried in 24 bits. */
int slz_matmul_i8_grad_workspace(const slz_i8_shape *shape, const void *dy_dev, size_t *bytes);
int slz_matmul_i8_grad(const slz_i8_shape *shape, const void *dy_dev, const int8_t *a_dev, const float *a_scale_dev,
                       const int8_t *b_dev, const float *b_scale_dev, void *da_dev, int64_t ld_da, void *db_dev, int64_t ld_db,
                       void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* ---- softmax cross entropy of a linear layer --------------------------------------------------------------------------------- */
typedef struct {
    uint32_t tokens, inner, vocab;       /* h is tokens x inner, w is vocab x inner; inner and vocab at least 1 */
    int type;                            /* of h, w, dh, dw */
    int64_t ld_h, ld_w, ld_dh, ld_dw;
    int64_t ignore_index;                /* tokens with this label do not count */
} slz_ce_shape;

/* z_tv = sum_d h_td w_vd, lse_t = log sum_v exp z_tv, loss_t = lse_t - z_t,label.  loss is 0 where the label is ignore_index and NaN
 * where another label lies outside [0, vocab).  The z are summed and kept in 32 bits, a tile of the vocabulary at a time; none
 * is written to memory.  A z of NaN or +inf makes its token's results NaN; one of -inf adds nothing (f32: an infinity in h or w
 * counts as NaN).  A token's results have the same bits whatever the other tokens are.  labels int64 [tokens], loss and lse [tokens] 32-bit floating point.
 * The workspace has 8 bytes for every token and 32 words, an eighth of the z in 16 bits. */
int slz_linear_ce_workspace(const slz_ce_shape *shape, const void *h_dev, const void *w_dev, size_t *bytes);
int slz_linear_ce(const slz_ce_shape *shape, const void *h_dev, const void *w_dev, const int64_t *labels_dev, float *loss_dev,
                  float *lse_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* With lse of slz_linear_ce and dloss [tokens] the gradient of what the losses are used for:
 *   g_tv = (exp(z_tv - lse_t) - [v = label_t]) dloss_t (0 for ignored tokens, NaN for labels out of range),  dh = g w,  dw = g^T h.
 * The z are computed again, in pieces of the vocabulary; a piece's g is held in h's type (f16, bf16: relative to
 * the largest finite |dloss| of the tokens that count; f32: in 24 bits), the sums in 32 bits.  dh [tokens][inner],
 * dw [vocab][inner].  A g of 0 times an infinity or NaN is NaN, as in the formula: a row of h that holds one reaches dw even where its token is ignored. */
int slz_linear_ce_grad_workspace(const slz_ce_shape *shape, const void *h_dev, const void *w_dev, size_t *bytes);
int slz_linear_ce_grad(const slz_ce_shape *shape, const void *h_dev, const void *w_dev, const int64_t *labels_dev,
                       const float *lse_dev, const float *dloss_dev, void *dh_dev, void *dw_dev, void *workspace_dev,
                       size_t workspace_bytes, void *hip_stream);

/* ---- orthogonalised updates ----------------------------------------------------------------------------------------------------- */
typedef struct {
    uint32_t batch, rows, cols;          /* that many matrices of one shape */
    int type;                            /* of g and out */
    int64_t ld_g, stride_g;              /* elements between rows, and between matrices, of g */
    int64_t ld_out, stride_out;
    uint32_t steps;                      /* at most 64 */
    float a, b, c;                       /* the coefficients of a step */
    float eps;
} slz_orth_shape;

/* Each matrix: X = g / (|g| + eps), |g| the root of the sum of squares, then `steps` times  A = X X^T,  X <- a X + (b A + c A A) X
 * (for more rows than columns the same of the transpose).  Products of 11-bit numbers, summed in 32 bits, the diagonals of A and
 * of b A + c A A apart from them in 32 bits; for f16 and f32 products of 22-bit numbers.  Between the steps X has 22 bits, or 2^-35 where that is more.
 * It is held in a format that reaches 63, and A and b A + c A A, off their diagonals, in one that reaches 1023: coefficients and numbers of steps that lead
 * beyond make the matrix infinite or NaN.
 * out may not overlap g. */
int slz_orthogonalize_workspace(const slz_orth_shape *shape, size_t *bytes);
int slz_orthogonalize(const slz_orth_shape *shape, const void *g_dev, void *out_dev, void *workspace_dev, size_t workspace_bytes,
                      void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SILENZIO_CLEAR_H */
