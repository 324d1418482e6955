/* Training and running a network in the clear, next to the gadgets that do it on ciphertexts (silenzio_gadgets.h): what an
 * encrypted run is compared with.  Scales are any numbers here; the gadgets' block scaling is by powers of two.
 *   slz_quantize_i8, slz_matmul_i8, slz_linear_i8, slz_matmul_i8_grad   products of 8-bit integers with a scale per row
 *   slz_linear_ce, slz_linear_ce_grad     softmax cross entropy of a linear layer's outputs, without keeping them, and its gradient
 *   slz_quantize_i4, slz_values_i4, slz_linear_i4, slz_linear_i4_grad   layers whose weights have 4 bits, with a scale per group of them
 *   slz_orthogonalize                     updates orthogonalised by Newton-Schulz products
 *   slz_grad_norm, slz_clip_by_norm       the norm that many gradients have together, and all of them held to one
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

/* ---- layers with 4-bit weights ------------------------------------------------------------------------------------------------- */
/* 4-bit rows: a row of k weights in whole blocks of 128, each of 64 bytes or 16 words of 32 bits.  Word 4 j + s of a block (j, s = 0 .. 3) has the block's
 * entries 32 s + 8 j + e, e = 0 .. 7: those with e < 4 in the low four bits of byte e, the others in the high four of byte e - 4.  Four
 * bits are a sign (the highest) and a magnitude of 0 to 7.  Entries past the row's end count for nothing, whatever they are; slz_quantize_i4 writes zeros.
 * Scales are 32-bit floating point, one for every `group` consecutive weights of a row (the last of a row may have fewer): group is 32, 64 or
 * 128.  A weight's value is scale times entry.  The rows lie on 16 bytes: the address and ld_q, in bytes, are multiples of 16 (ld_q where there are
 * several rows); a range of rows, or of columns from a multiple of 128 on, can so be given as it is.  The leading dimensions are of q in bytes and of the scales in elements. */

/* w [rows][cols] to 4 bits: for each group top = max |w|, scale = top / 7 in 32-bit floating point, entry = the whole number nearest to 7 w / top (the
 * exact quotient, ties to even); a group of zeros has scale 0 and zeros, one with an infinity or NaN scale NaN and zeros. */
int slz_quantize_i4(const void *w_dev, int type, uint32_t rows, uint32_t cols, int64_t ld_w, uint32_t group, uint8_t *q_dev, int64_t ld_q,
                    float *scale_dev, int64_t ld_scale, void *hip_stream);
/* The values of 4-bit rows, out [rows][cols] of `type`: the product in 32 bits, rounded to the type. */
int slz_values_i4(const uint8_t *q_dev, int64_t ld_q, const float *scale_dev, int64_t ld_scale, uint32_t group, uint32_t rows, uint32_t cols,
                  void *out_dev, int type, int64_t ld_out, void *hip_stream);

typedef struct {
    uint32_t m, n, k;                    /* x is m x k, the weights n x k, y is m x n */
    int type;                            /* of x, y and the gradients */
    uint32_t group;
    int64_t ld_x, ld_q, ld_scale, ld_y;  /* ld_y is dy's in slz_linear_i4_grad */
} slz_i4_shape;

/* y_ij = sum_k x_ik w_jk with the values w, summed in 32 bits and rounded to the type.  Few rows of x are multiplied by the entries as they are, and each group's sum by its
 * scale; for many (a thousand, about; from nine on where k is below 8) the values are held in the type first: rounded to 8 bits for bf16 and to 11 for f16 (to
 * fewer where the scale is below 2^-26 of the largest finite one), and carried in 24 for f32.  What of an f32 input lies below 2^-133 is lost.
 * A group's sum does not overflow before its scale brings it down.  bf16: where entries are multiplied as they are, what of a group's product lies below 2^-139 is lost.
 * An infinity or NaN in x makes its row's results infinite or NaN, a NaN scale its column's. */
int slz_linear_i4_workspace(const slz_i4_shape *shape, const void *x_dev, size_t *bytes);
int slz_linear_i4(const slz_i4_shape *shape, const void *x_dev, const uint8_t *q_dev, const float *scale_dev, void *y_dev, void *workspace_dev,
                  size_t workspace_bytes, void *hip_stream);

/* Gradients for dy [m][n] with respect to x and to the values (the rounding of a quantisation is passed straight through):
 *   dx_ik = sum_j dy_ij w_jk,  dw_jk = sum_i dy_ij x_ik.  dx is [m][k], dw [n][k]; either of the two may be null, and then x (without dw) or q and scale (without
 * dx) are not read.  For bf16 and f16 the values are rounded to 8 and 11 bits for dx (f16: to fewer where the scale is below 2^-26 of the largest
 * finite one); for f32 they are carried in 24 bits.  The workspace is that of both gradients. */
int slz_linear_i4_grad_workspace(const slz_i4_shape *shape, const void *dy_dev, const void *x_dev, size_t *bytes);
int slz_linear_i4_grad(const slz_i4_shape *shape, const void *dy_dev, const void *x_dev, const uint8_t *q_dev, const float *scale_dev, void *dx_dev,
                       int64_t ld_dx, void *dw_dev, int64_t ld_dw, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

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

/* ---- gradients clipped by their norm -------------------------------------------------------------------------------------------- */
typedef struct {
    const void *g;                       /* a gradient [rows][cols] on the device */
    void *out;                           /* [rows][cols] of the same type; the same place as g (with the same leading dimension) or one that overlaps no gradient */
    uint32_t rows, cols;
    int64_t ld_g, ld_out;                /* any distance; where it is cols the rows are one run of elements */
    int type;
} slz_grad_tensor;

/* norm = root of the sum of the squares of all elements of all `count` tensors (an array on the host), squared and summed in 64 bits and
 * rounded to 32-bit floating point.  0 without elements; out, ld_out are not looked at. */
int slz_clip_workspace(const slz_grad_tensor *tensors, uint32_t count, size_t *bytes);
int slz_grad_norm(const slz_grad_tensor *tensors, uint32_t count, float *norm_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream);
/* out = g f in 32 bits, rounded to the type, with f = 1 where norm + eps <= max_norm, else max_norm / (norm + eps) (in 64 bits, rounded to 32), and NaN where
 * norm is NaN.  The norm is computed as by slz_grad_norm and left in norm_dev, or, with norm_given, taken from there (the norm of more gradients than these).
 * Where f is 1 the elements keep their bits. SLZ_E_INVALID_ARG also where max_norm or eps is negative or NaN, and where an output overlaps another one,
 * another gradient or norm_dev, or norm_dev, where it is written, a gradient. */
int slz_clip_by_norm(const slz_grad_tensor *tensors, uint32_t count, float max_norm, float eps, int norm_given, float *norm_dev, void *workspace_dev,
                     size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SILENZIO_CLEAR_H */
