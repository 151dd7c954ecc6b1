// What the host side of the operators of include/qoda_matrices.h hands to their kernels.
#pragma once

#include "qoda_operators.h"

namespace qoda {

typedef unsigned char u8;

// A microscaled matrix: rows of 128 bytes a step of 256 entries, and scales of 256 bytes for 64 rows and four blocks.
constexpr int kMxStep = 256;
inline long long mx_steps(long long cols) { return (cols + kMxStep - 1) / kMxStep; }
inline long long mx_groups(long long rows) { return (rows + 63) / 64; }

struct MxRounding {   // x is read, q written; values: the other way round
  int type, transposed, stochastic;
  long long rows, cols;       // of x
  void *x;
  long long ldx;
  u8 *codes, *scales;
  unsigned int k0, k1, o0, o1;   // the lots' key and the upper half of their counter
  long long first;               // of in_launches()
};

// p: sizes, outputs and epilogue as in a product of entries; its operands are these.
struct MxProduct {
  Product p;
  const u8 *a, *a_scales, *b, *b_scales;   // a: null where the rows are plain (x)
  const void *x;
  long long ldx;
  int steps;                               // of 256 entries along the sum
  float *row_sums;                         // of a, or null
  long long first;
};

// Matrices g [rows][cols]; X [m][n] is g or its transpose, m <= n, both sides filled up to multiples of 32.  by_norm: how far X's numbers are from the bound on them is not known
// before the call.
struct Orthogonal {
  int type, steps, transposed, parts, by_norm;
  long long matrices, rows, cols, m, n;
  const void *g;
  void *x;
  long long g_matrix, g_row, x_matrix, x_row;
  double a, b, c, eps;
  double *squares;   // [matrices][parts]
  void *xs, *xt;     // X and its transpose in pairs of fp16
  float scale;
  float *scales;     // by_norm: [matrices][4], two factors of B and two of X
  long long first;
};

// What the sums of a step's three products, and what is added to the second and third, are multiplied with.
struct StepFactors {
  float a, b, b_extra, x, x_extra;
};
constexpr int kMostSmallSteps = 16;
struct SmallOrthogonal {
  Orthogonal o;
  StepFactors f[kMostSmallSteps];
  long long first;
};

// out = a b^T factor + e extra + e2 extra2 of matrices of pairs, a [m][k], b [n][k], e, e2 (each may be null) and out [m][n], out_t [n][m] the transpose of out; x: where the result goes
// instead, in the caller's type.  symmetric: m = n and out = out_t, of which the tiles above the diagonal are computed.
struct PairProduct {
  int symmetric, type, x_transposed;
  long long matrices, m, n, k;
  const void *a, *b, *e, *e2;
  void *out, *out_t, *x;
  long long x_matrix, x_row, x_rows, x_cols;
  float factor, extra, extra2;
  const float *scales;   // null, or of a product with partial sums: of every fourth matrix's place on, further factors of the sums and of e
  float *partial;        // of split sums: [splits][matrices][m][n]
  long long first;
};

bool orthogonal_bounded(double a, double b, double c, int steps);
bool orthogonal_by_norm(double a, double b, double c, int steps);
void orthogonal_sides(Orthogonal *o);
size_t orthogonal_scratch(const Orthogonal &o);
hipError_t launch_orthogonalize(const Orthogonal &o, void *workspace, hipStream_t s);

hipError_t launch_mx_quantize(const MxRounding &q, hipStream_t s);
hipError_t launch_mx_values(const MxRounding &q, hipStream_t s);
bool mx_takes_plain_rows(const Product &p);   // whether the product rounds plain rows itself
size_t mx_product_scratch(const MxProduct &p);
hipError_t launch_mx_product(const MxProduct &p, hipStream_t s);

}  // namespace qoda
