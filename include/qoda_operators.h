/*
 * qoda_operators.h -- C ABI of the operators that make a node's dual vector on MI355X (gfx950): the matrix product with bias,
 * activation, dropout and residual in its epilogue, dropout from a counter-based generator, group normalisation with an
 * activation (channels last), and the gradient of each.  Weight gradients are fp32 and are written where qoda_quantize reads
 * them: into the caller's gradient vector.  Exported by libqoda beside the calls of qoda.h.
 *
 * Conventions
 *   - No context: a call works on the device that is current and enqueues on `stream` (a hipStream_t as void*, NULL = the
 *     default stream) kernels only; it allocates nothing, waits for nothing and may be captured into a graph.  Scratch memory
 *     is the caller's: *_workspace_bytes() says how much a call with these arguments, addresses among them, needs (0 for many), on the
 *     call's stream until the call's work is done, aligned to 16 bytes.  Calls may be made from any number of host threads.
 *   - Every call returns QODA_OK (0) or a negative error code, and then qoda_operator_error() describes it (the calling
 *     thread's last error).  Arguments are checked before anything is launched; nothing throws across this boundary.
 *   - A matrix is row-major: `data` points at entry (0, 0) in device memory, entries of a row are adjacent, rows are `stride`
 *     entries apart (stride >= columns where there is more than one row).  Any alignment that the type itself has will do;
 *     rows that start at multiples of 16 bytes are fastest.  Offsets are 64-bit throughout; rows, columns, samples, positions and
 *     channels number at most QODA_MAX_SIDE each, and samples times groups are fewer than 2^31.
 *   - Outputs may be no input's memory, except where a call says so.  A size of zero is no error: an empty output is left alone, and
 *     a sum over nothing is 0.
 *   - Entries are fp32 (QODA_F32) or bfloat16 (QODA_BF16); biases, scales, statistics and gradients of parameters are fp32.
 *     Sums run in fp32 (matrix products, statistics) and an entry is rounded once, to nearest even, where it is stored.
 *     Infinities and NaN go through the formulas as IEEE arithmetic has it.
 *
 * Dropout.  Entry (r, c) of a matrix is kept where its lot is at least T = floor(p * 65536 + 1/2), and is then multiplied by
 * 65536 / (65536 - T), so that the mean is exact for the probability in use; otherwise it is 0, whatever it was.  Lots are 16-bit
 * pieces of Philox4x32-10 with the counter (c >> 3, r, offset low, offset high) and the key seed xor QODA_DROPOUT_KEY (the
 * quantizer draws from the same generator; the constant keeps the two apart for one seed): lot c & 7 is the low half of word
 * c & 3, or its high half if c & 4.  A gradient call with the same p, seed and offset has the same mask; no mask is stored.
 * Another call that is to have another mask gets another offset.  p = 0: nothing is dropped; p = 1: everything is.
 */
#ifndef QODA_OPERATORS_H_
#define QODA_OPERATORS_H_

#include <stddef.h>
#include <stdint.h>

#include "qoda.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QODA_MAX_SIDE 0x7fff0000

#define QODA_F32 0
#define QODA_BF16 1

#define QODA_ACT_NONE 0
#define QODA_ACT_RELU 1       /* max(z, 0); slope 0 at 0 */
#define QODA_ACT_LEAKY_RELU 2 /* z where z > 0, else 0.2 z */
#define QODA_ACT_GELU 3       /* z Phi(z), Phi the normal distribution function */
#define QODA_ACT_SILU 4       /* z / (1 + exp(-z)) */

#define QODA_DROPOUT_KEY 0x64726F706F757473ull

typedef struct {
  void *data;     /* device memory; NULL where the matrix is optional and absent */
  int64_t stride; /* entries from one row to the next */
} qoda_matrix;

/* y = residual + drop(act(x w^T + bias)).
 *   x [rows][in], w [out][in], bias fp32 [out] or NULL, residual [rows][out] or absent, y [rows][out];
 *   pre [rows][out] or absent: receives x w^T + bias, which the gradient of an activation needs.
 * residual may be y's memory. */
typedef struct {
  int32_t dtype, activation;
  int64_t rows, in, out;
  qoda_matrix x, w, residual, y, pre;
  const float *bias;
  double p;
  uint64_t seed, offset;
} qoda_linear_args;

/* dx = residual + drop((dz w) * act'(pre)): the gradient of linear's x and, with pre, on through the activation and the
 * dropout of the layer before, whose pre it is and whose p, seed and offset these are.
 *   dz [rows][out], w [out][in], pre [rows][in] or absent (then activation is QODA_ACT_NONE), residual [rows][in] or absent, dx [rows][in].
 * residual may be dx's memory. */
typedef struct {
  int32_t dtype, activation;
  int64_t rows, in, out;
  qoda_matrix dz, w, pre, residual, dx;
  double p;
  uint64_t seed, offset;
} qoda_linear_input_grad_args;

/* dw = dz^T x and dbias = the sum of dz's rows, fp32; accumulate != 0: added to what is there.
 *   dz [rows][out], x [rows][in], dw fp32 [out][in], dbias fp32 [out] or NULL. */
typedef struct {
  int32_t dtype, accumulate;
  int64_t rows, in, out;
  qoda_matrix dz, x, dw;
  float *dbias;
} qoda_linear_weight_grad_args;

int64_t qoda_linear_workspace_bytes(const qoda_linear_args *a);
int64_t qoda_linear_input_grad_workspace_bytes(const qoda_linear_input_grad_args *a);
int64_t qoda_linear_weight_grad_workspace_bytes(const qoda_linear_weight_grad_args *a);
int qoda_linear(const qoda_linear_args *a, void *workspace, size_t workspace_bytes, void *stream);
int qoda_linear_input_grad(const qoda_linear_input_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);
int qoda_linear_weight_grad(const qoda_linear_weight_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* qoda_dropout: y = residual + drop(act(x)); extra is the residual or absent, and both x and extra may be y's memory.
 * qoda_dropout_grad: y = drop(x * act'(extra)); x is the gradient of drop(act(z)), extra is z (absent with QODA_ACT_NONE), and
 * both may be y's memory.  All matrices are [rows][cols]. */
typedef struct {
  int32_t dtype, activation;
  int64_t rows, cols;
  qoda_matrix x, extra, y;
  double p;
  uint64_t seed, offset;
} qoda_dropout_args;

int qoda_dropout(const qoda_dropout_args *a, void *stream);
int qoda_dropout_grad(const qoda_dropout_args *a, void *stream);

/* Values of samples, positions and channels, channels adjacent: entry (n, s, c) is data[n * sample + s * position + c]. */
typedef struct {
  void *data;
  int64_t sample, position;
} qoda_channels_last;

/* Group normalisation: groups divides channels, group g of a sample is its channels g C/G .. (g+1) C/G - 1 at all positions;
 *   mean, rstd fp32 [samples][groups]: mean, and 1 / sqrt(variance + eps) with the variance of the population;
 *   y = act((x - mean) * rstd * weight + bias), weight and bias fp32 [channels], NULL: 1 and 0.
 * Without positions or channels there is nothing to write, and mean and rstd are left alone.
 * One position and one group make it a layer normalisation of rows. */
typedef struct {
  int32_t dtype, activation;
  int64_t samples, positions, channels, groups;
  qoda_channels_last x, y;
  const float *weight, *bias;
  float *mean, *rstd;
  double eps;
} qoda_group_norm_args;

/* dx = residual + the gradient of x; dweight, dbias fp32 [channels] (each may be NULL), accumulate != 0: added to what is there.
 * x, weight, bias, mean and rstd as in the forward call; dy is the gradient of y.  residual may be dx's memory. */
typedef struct {
  int32_t dtype, activation;
  int64_t samples, positions, channels, groups;
  qoda_channels_last dy, x, residual, dx;
  const float *weight, *bias, *mean, *rstd;
  float *dweight, *dbias;
  int32_t accumulate;
} qoda_group_norm_grad_args;

int64_t qoda_group_norm_workspace_bytes(const qoda_group_norm_args *a);
int64_t qoda_group_norm_grad_workspace_bytes(const qoda_group_norm_grad_args *a);
int qoda_group_norm(const qoda_group_norm_args *a, void *workspace, size_t workspace_bytes, void *stream);
int qoda_group_norm_grad(const qoda_group_norm_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* What the calling thread's last failing call of this header found wrong ("" before the first). */
const char *qoda_operator_error(void);

#ifdef __cplusplus
}
#endif

#endif /* QODA_OPERATORS_H_ */
