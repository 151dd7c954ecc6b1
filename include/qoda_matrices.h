/*
 * qoda_matrices.h -- C ABI of what is done with a model's matrices in a round, on MI355X (gfx950): rounding to four bits with a shared
 * scale for every 32 entries (microscaled floating point), products between such matrices with the epilogues of qoda_operators.h and
 * both gradients, and the orthogonalisation of an update by Newton-Schulz products.  Exported by libqoda beside the calls of qoda.h
 * and qoda_operators.h; the conventions of qoda_operators.h hold (no context, nothing allocated, only kernels enqueued, errors by code and
 * qoda_operator_error(), sizes of zero, strides, any number of host threads, capture into graphs).
 *
 * Microscaled matrices.  A row's entries in blocks of 32 (the last may be shorter) have a scale 2^e in common, and an entry is a sign and one of
 * the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 to 7, the sign in bit 3) times it.  With m the block's largest magnitude and v = |x| / 2^e:
 *   to nearest       e = floor(log2 m) - 2; v goes to the nearer magnitude, halves to the even code, above 6 to 6.
 *   stochastically   e is the least with m <= 6 2^e, so that nothing is cut off; v between neighbours q and q + d goes to q + d where lot + 1/2 <=
 *                    65536 (v - q) / d, otherwise to q: the mean over the lots is v, to 2^-17 d.  Lots are dropout's (qoda_operators.h) with the
 *                    key seed xor QODA_MX_KEY and (r, c) the entry's place in the microscaled matrix.
 * e is at least -127, which is also that of a block of zeros.  A block with an infinity or a NaN is NaN throughout.
 * In memory: `codes` has rows of qoda_mx_code_bytes(1, cols) bytes, 16 a block, the entry of even place in a byte's low half, and every row
 * filled up to a multiple of eight blocks with zeros.  `scales` has bytes e + 127 (255: NaN) in the order in which the matrix
 * instruction's lanes take them, [blocks / 4][rows / 64][4][4][4][2][2], the rows filled up to a multiple of 64: block 4 b + g of row
 * 64 r + 32 f + 8 q + 4 h + j has place (b, r, g, q, j, f, h).  Both are aligned to 16 bytes.  Bytes that fill up are written as 0, and products count on that.
 */
#ifndef QODA_MATRICES_H_
#define QODA_MATRICES_H_

#include "qoda_operators.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QODA_MX_KEY 0x6D78666F75726269ull
#define QODA_MX_MAX_SUM 0x1000000 /* entries that a product between microscaled matrices may sum over */
#define QODA_MAX_STEPS 1000       /* of an orthogonalisation */

typedef struct {
  void *codes, *scales;
} qoda_mx;

/* Bytes of a microscaled matrix of rows x cols; QODA_EINVAL for sizes outside [0, QODA_MAX_SIDE]. */
int64_t qoda_mx_code_bytes(int64_t rows, int64_t cols);
int64_t qoda_mx_scale_bytes(int64_t rows, int64_t cols);

/* q = x [rows][cols] rounded or, transposed != 0, x^T: q then has cols rows and blocks along x's rows. */
typedef struct {
  int32_t dtype, transposed, stochastic;
  int64_t rows, cols;
  qoda_matrix x;
  qoda_mx q;
  uint64_t seed, offset;
} qoda_mx_quantize_args;
int qoda_mx_quantize(const qoda_mx_quantize_args *a, void *stream);

/* y [rows][cols] = what q stands for; exact in both types, but that a stochastic rounding of an entry above 3 2^126 may go to 2^128, which both have as infinity. */
typedef struct {
  int32_t dtype;
  int64_t rows, cols;
  qoda_mx q;
  qoda_matrix y;
} qoda_mx_values_args;
int qoda_mx_values(const qoda_mx_values_args *a, void *stream);

/* The products of qoda_operators.h with microscaled operands, whose blocks lie along the sum: entries, epilogues and workspaces as there.
 * qoda_mx_linear: w [out][in]; x [rows][in], microscaled (xq) or, where x.data is not NULL, of dtype: it is then rounded to nearest in the call.
 *   residual, y, pre of dtype.
 * qoda_mx_linear_input_grad: wt [in][out] is the weight's transpose; dz [rows][out] like x above.
 * qoda_mx_linear_weight_grad: dzt [out][rows] and xt [in][rows]; dw fp32 [out][in], dbias fp32 [out] or NULL: the sums of dzt's rows. */
typedef struct {
  int32_t dtype, activation;
  int64_t rows, in, out;
  qoda_matrix x;
  qoda_mx xq, w;
  qoda_matrix residual, y, pre;
  const float *bias;
  double p;
  uint64_t seed, offset;
} qoda_mx_linear_args;

typedef struct {
  int32_t dtype, activation;
  int64_t rows, in, out;
  qoda_matrix dz;
  qoda_mx dzq, wt;
  qoda_matrix pre, residual, dx;
  double p;
  uint64_t seed, offset;
} qoda_mx_linear_input_grad_args;

typedef struct {
  int32_t accumulate;
  int64_t rows, in, out;
  qoda_mx dzt, xt;
  qoda_matrix dw;
  float *dbias;
} qoda_mx_linear_weight_grad_args;

int64_t qoda_mx_linear_workspace_bytes(const qoda_mx_linear_args *a);
int64_t qoda_mx_linear_input_grad_workspace_bytes(const qoda_mx_linear_input_grad_args *a);
int64_t qoda_mx_linear_weight_grad_workspace_bytes(const qoda_mx_linear_weight_grad_args *a);
int qoda_mx_linear(const qoda_mx_linear_args *a, void *workspace, size_t workspace_bytes, void *stream);
int qoda_mx_linear_input_grad(const qoda_mx_linear_input_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);
int qoda_mx_linear_weight_grad(const qoda_mx_linear_weight_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* x = the orthogonalised g, matrix by matrix of a batch: entry (n, i, j) is data[n * matrix + i * row + j].
 *   X_0 = g / (|g| + eps), |g| the root of the sum of squares;  A = X X^T,  X <- a X + (b A + c A A) X, steps times;
 * where g has more rows than columns X^T takes X's place, with the same result.  steps is at most QODA_MAX_STEPS, a, b, c are finite, and the singular values stay
 * below 2^40 for every g (a bound from a, b and c; otherwise QODA_EINVAL).  The smaller side is at most 2^17, the larger at most 2^22.  x may be g itself, with the
 * same strides; where one lies in the other's entries otherwise, QODA_EINVAL.  A matrix with an infinity or a NaN becomes NaN throughout, if steps > 0.
 * Accurate as fp32 products are: what the matrix cores take are pairs of fp16 numbers, 22 bits of a number or 2^-41 of a bound on it.  The bound is that of the
 * polynomial where it stays near |a| a step, as for those that bring singular values towards 1; digits are then lost where |g| is less than 2^-8 eps.  For others (a
 * small or 0, or large singular values that grow faster than small ones) it is that of the norms that X and A have in each step, which takes longer. */
typedef struct {
  void *data;
  int64_t matrix, row; /* entries from one matrix, and from one row, to the next */
} qoda_matrices;

typedef struct {
  int32_t dtype, steps;
  int64_t matrices, rows, cols;
  qoda_matrices g, x;
  double a, b, c, eps;
} qoda_orthogonalize_args;

int64_t qoda_orthogonalize_workspace_bytes(const qoda_orthogonalize_args *a);
int qoda_orthogonalize(const qoda_orthogonalize_args *a, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QODA_MATRICES_H_ */
