// What the host side of the operators of include/qoda_operators.h hands to their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qoda {

enum EntryType { kF32 = 0, kBf16 = 1 };
enum Activation { kActNone = 0, kActRelu = 1, kActLeakyRelu = 2, kActGelu = 3, kActSilu = 4 };
constexpr int kNumActivations = 5;

// Dropout of a call: entries whose lot is below the threshold are dropped, the others multiplied by the scale.  limit: 2^16 threshold - 1,
// modulo 2^32 (of no use with threshold 0, which drops nothing).
struct Drop {
  unsigned int threshold, limit;
  float scale;
  unsigned int k0, k1, o0, o1;   // the generator's key and the upper half of its counter
};

// c[i][j] = sum over l of a(i, l) b(j, l), and what becomes of it.  form: which side's entries are adjacent along l.
enum ProductForm {
  kProductRows = 0,      // a[i][l], b[j][l]   x w^T
  kProductMixed = 1,     // a[i][l], b[l][j]   dz w
  kProductColumns = 2    // a[l][i], b[l][j]   dz^T x
};
struct Product {
  int form, type;
  int m, n, k;
  const void *a, *b;
  long long lda, ldb;
  // kProductRows: out = extra + drop(act(c + bias)), and pre receives c + bias; kProductMixed: out = extra + drop(c * act'(pre));
  // kProductColumns: out = c, or out + c, in fp32, and sums receives the sums of a's columns, or is added to
  void *out, *pre;
  const void *extra;
  long long ldo, ldp, lde;
  const float *bias;
  float *sums;
  int activation, accumulate;
  Drop drop;
  float *partial;   // products split over l: [splits][m][n]
  long long first;  // of in_launches()
};

struct Entries {   // y = extra + drop(act(x)), or gradient: y = drop(x * act'(extra))
  int type, activation, gradient;
  long long rows, cols;
  const void *x, *extra;
  void *y;
  long long ldx, lde, ldy;
  Drop drop;
  long long first;
};

struct GroupNorm {
  int type, activation, accumulate;
  long long samples, positions, channels, groups;
  const void *x, *dy, *extra;   // extra: the residual of the gradient
  void *out;                    // y or dx
  long long x_sample, x_pos, dy_sample, dy_pos, extra_sample, extra_pos, out_sample, out_pos;
  const float *weight, *bias;
  float *mean, *rstd;
  float *dweight, *dbias;
  float eps;
  float *scratch;
  long long first;
};

// HIP launches fewer than 2^32 work-items along a dimension of the grid.  Calls launch(args, grid.x) for `workgroups` of `threads` each, in as many
// launches as that takes; a kernel's workgroup is number args.first + blockIdx.x.
template <class Args, class F>
void in_launches(const Args &args, long long workgroups, int threads, F &&launch) {
  const long long most = ((1ll << 32) - 1) / threads;
  Args a = args;
  for (a.first = 0; a.first < workgroups; a.first += most) launch(a, (unsigned)(workgroups - a.first < most ? workgroups - a.first : most));
}

size_t product_scratch(const Product &p);        // bytes of p.partial
hipError_t launch_product(const Product &p, hipStream_t s);
hipError_t launch_entries(const Entries &e, hipStream_t s);
size_t group_norm_scratch(const GroupNorm &g, bool gradient);
hipError_t launch_group_norm(const GroupNorm &g, hipStream_t s);
hipError_t launch_group_norm_grad(const GroupNorm &g, hipStream_t s);

}  // namespace qoda
