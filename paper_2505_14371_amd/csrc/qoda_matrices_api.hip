// Host side of the operators declared in include/qoda_matrices.h: checks of arguments, and the kernels' arguments from the caller's.

#include "../../include/qoda_matrices.h"
#include "qoda_matrices.h"
#include "qoda_operators_checks.h"

#include <cstdlib>

using namespace qoda;

namespace {

size_t code_bytes(int64_t rows, int64_t cols) { return (size_t)rows * (size_t)mx_steps(cols) * 128; }
size_t scale_bytes(int64_t rows, int64_t cols) { return (size_t)mx_groups(rows) * (size_t)mx_steps(cols) * 512; }

int check_mx(const char *call, const char *name, const qoda_mx &q, int64_t rows, int64_t cols) {
  if (rows == 0 || cols == 0) return QODA_OK;
  if (!q.codes || !q.scales) return fail(QODA_EINVAL, "%s: %s is null", call, name);
  if (!aligned(q.codes, 16) || !aligned(q.scales, 16)) return fail(QODA_EINVAL, "%s: codes or scales of %s are not aligned to 16 bytes", call, name);
  return QODA_OK;
}

int check_sum(const char *call, int64_t k) {
  if (k > QODA_MX_MAX_SUM) return fail(QODA_EINVAL, "%s: sums over %lld entries; %d at most", call, (long long)k, QODA_MX_MAX_SUM);
  return QODA_OK;
}

int check_type(const char *call, int32_t dtype) { return check_common(call, dtype, kActNone); }

int rounding_of(const qoda_mx_quantize_args *a, MxRounding *q) {
  const char *call = "qoda_mx_quantize";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_type(call, a->dtype));
  TRY(check_sides(call, a->rows, a->cols, 0));
  TRY(check_matrix(call, "x", a->x, a->rows, a->cols, entry_bytes(a->dtype), false));
  TRY(check_mx(call, "q", a->q, a->rows, a->cols));
  const uint64_t key = a->seed ^ QODA_MX_KEY;
  *q = {};
  q->type = a->dtype, q->transposed = a->transposed != 0, q->stochastic = a->stochastic != 0;
  q->rows = a->rows, q->cols = a->cols;
  q->x = a->x.data, q->ldx = stride_of(a->x, a->rows, a->cols);
  q->codes = static_cast<u8 *>(a->q.codes), q->scales = static_cast<u8 *>(a->q.scales);
  q->k0 = (unsigned)key, q->k1 = (unsigned)(key >> 32), q->o0 = (unsigned)a->offset, q->o1 = (unsigned)(a->offset >> 32);
  return QODA_OK;
}

void operands(MxProduct *m, const qoda_mx &a, const qoda_mx &b, int64_t k) {
  m->a = static_cast<const u8 *>(a.codes), m->a_scales = static_cast<const u8 *>(a.scales);
  m->b = static_cast<const u8 *>(b.codes), m->b_scales = static_cast<const u8 *>(b.scales);
  m->steps = (int)mx_steps(k);
  m->p.k = (int)k;
}

int linear_of(const qoda_mx_linear_args *a, MxProduct *m) {
  const char *call = "qoda_mx_linear";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_sides(call, a->rows, a->in, a->out));
  TRY(check_sum(call, a->in));
  *m = {};
  Product *p = &m->p;
  TRY(make_drop(call, a->p, a->seed, a->offset, &p->drop));
  const size_t e = entry_bytes(a->dtype);
  if (a->out > 0) {
    if (a->x.data) TRY(check_matrix(call, "x", a->x, a->rows, a->in, e, false));
    else TRY(check_mx(call, "x", a->xq, a->rows, a->in));
  }
  if (a->rows > 0) TRY(check_mx(call, "w", a->w, a->out, a->in));
  TRY(check_matrix(call, "residual", a->residual, a->rows, a->out, e, true));
  TRY(check_matrix(call, "y", a->y, a->rows, a->out, e, false));
  TRY(check_matrix(call, "pre", a->pre, a->rows, a->out, e, true));
  if (!aligned(a->bias, 4)) return fail(QODA_EINVAL, "%s: bias is not aligned to its entries", call);
  p->form = kProductRows, p->type = a->dtype;
  p->m = (int)a->rows, p->n = (int)a->out;
  p->out = a->y.data, p->ldo = stride_of(a->y, a->rows, a->out);
  p->pre = a->pre.data, p->ldp = stride_of(a->pre, a->rows, a->out);
  p->extra = a->residual.data, p->lde = stride_of(a->residual, a->rows, a->out);
  p->bias = a->bias, p->activation = a->activation;
  operands(m, a->xq, a->w, a->in);
  m->x = a->x.data, m->ldx = stride_of(a->x, a->rows, a->in);
  return QODA_OK;
}

int input_grad_of(const qoda_mx_linear_input_grad_args *a, MxProduct *m) {
  const char *call = "qoda_mx_linear_input_grad";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_sides(call, a->rows, a->in, a->out));
  TRY(check_sum(call, a->out));
  *m = {};
  Product *p = &m->p;
  TRY(make_drop(call, a->p, a->seed, a->offset, &p->drop));
  const size_t e = entry_bytes(a->dtype);
  if (a->in > 0) {
    if (a->dz.data) TRY(check_matrix(call, "dz", a->dz, a->rows, a->out, e, false));
    else TRY(check_mx(call, "dz", a->dzq, a->rows, a->out));
  }
  if (a->rows > 0) TRY(check_mx(call, "wt", a->wt, a->in, a->out));
  TRY(check_matrix(call, "pre", a->pre, a->rows, a->in, e, a->activation == kActNone));
  TRY(check_matrix(call, "residual", a->residual, a->rows, a->in, e, true));
  TRY(check_matrix(call, "dx", a->dx, a->rows, a->in, e, false));
  p->form = kProductMixed, p->type = a->dtype;
  p->m = (int)a->rows, p->n = (int)a->in;
  p->out = a->dx.data, p->ldo = stride_of(a->dx, a->rows, a->in);
  p->pre = a->activation == kActNone ? nullptr : a->pre.data, p->ldp = stride_of(a->pre, a->rows, a->in);
  p->extra = a->residual.data, p->lde = stride_of(a->residual, a->rows, a->in);
  p->activation = a->activation;
  operands(m, a->dzq, a->wt, a->out);
  m->x = a->dz.data, m->ldx = stride_of(a->dz, a->rows, a->out);
  return QODA_OK;
}

int weight_grad_of(const qoda_mx_linear_weight_grad_args *a, MxProduct *m) {
  const char *call = "qoda_mx_linear_weight_grad";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_sides(call, a->rows, a->in, a->out));
  TRY(check_sum(call, a->rows));
  *m = {};
  Product *p = &m->p;
  TRY(check_mx(call, "dzt", a->dzt, a->out, a->rows));
  if (a->out > 0) TRY(check_mx(call, "xt", a->xt, a->in, a->rows));
  TRY(check_matrix(call, "dw", a->dw, a->out, a->in, 4, false));
  if (!aligned(a->dbias, 4)) return fail(QODA_EINVAL, "%s: dbias is not aligned to its entries", call);
  p->form = kProductColumns, p->type = kF32;
  p->m = (int)a->out, p->n = (int)a->in;
  p->out = a->dw.data, p->ldo = stride_of(a->dw, a->out, a->in);
  p->accumulate = a->accumulate != 0;
  operands(m, a->dzt, a->xt, a->rows);
  m->x = nullptr;
  m->row_sums = a->dbias;
  return QODA_OK;
}

// The rows that the product does not round itself are rounded into the workspace, before the split sums.
size_t rounded_bytes(const MxProduct &m) {
  if (!m.x || m.p.m == 0 || m.p.n == 0 || m.p.k == 0 || mx_takes_plain_rows(m.p)) return 0;
  return code_bytes(m.p.m, m.p.k) + scale_bytes(m.p.m, m.p.k);
}

template <class Args>
int64_t scratch_of(const Args *a, int (*make)(const Args *, MxProduct *)) {
  MxProduct m;
  const int rc = make(a, &m);
  return rc != QODA_OK ? rc : (int64_t)(rounded_bytes(m) + mx_product_scratch(m));
}

int run(const char *call, MxProduct *m, void *workspace, size_t bytes, void *stream) {
  if (m->p.m == 0 || (m->p.n == 0 && !m->row_sums)) return QODA_OK;
  const size_t rounded = rounded_bytes(*m);
  TRY(check_workspace(call, workspace, bytes, rounded + mx_product_scratch(*m)));
  u8 *w = static_cast<u8 *>(workspace);
  if (m->x && m->p.k > 0 && mx_takes_plain_rows(m->p)) {
    m->a = nullptr;
  } else if (m->x) {
    MxRounding q = {};
    q.type = m->p.type, q.rows = m->p.m, q.cols = m->p.k;
    q.x = const_cast<void *>(m->x), q.ldx = m->ldx;
    q.codes = w, q.scales = w + code_bytes(m->p.m, m->p.k);
    m->a = q.codes, m->a_scales = q.scales;
    if (m->p.k > 0) TRY(done(call, launch_mx_quantize(q, static_cast<hipStream_t>(stream))));
  }
  m->p.partial = reinterpret_cast<float *>(w + rounded);
  return done(call, launch_mx_product(*m, static_cast<hipStream_t>(stream)));
}

constexpr int64_t kMostLeast = 1 << 17, kMostSideOfUpdate = 1 << 22;   // 32-bit offsets inside a tile, and numbers of tiles

int check_matrices(const char *call, const char *name, const qoda_matrices &v, int64_t n, int64_t rows, int64_t cols, size_t bytes, long long *row, long long *matrix) {
  *row = rows > 1 ? v.row : cols;   // a stride that no entry is reached by is not looked at
  *matrix = n > 1 ? v.matrix : 0;
  if (!v.data) return fail(QODA_EINVAL, "%s: %s is null", call, name);
  if (!aligned(v.data, bytes)) return fail(QODA_EINVAL, "%s: %s is not aligned to its entries", call, name);
  if (*row < cols || *row >= kMostStride || (n > 1 && (*matrix < (__int128)(rows - 1) * *row + cols || *matrix >= kMostStride * 1024)))
    return fail(QODA_EINVAL, "%s: the strides of %s do not fit matrices of %lld rows and %lld columns", call, name, (long long)rows, (long long)cols);
  return QODA_OK;
}

// Whether x is neither g itself nor apart from it: an entry of the one lies where another one of the other does.  Rows of one set are apart and in the order of their addresses.
bool overlapping(const Orthogonal &o, size_t bytes) {
  if (o.g == o.x && o.g_row == o.x_row && o.g_matrix == o.x_matrix) return false;
  const long long off = ((intptr_t)o.x - (intptr_t)o.g) / (long long)bytes;   // of x's first entry from g's
  const auto last = [&](long long matrix, long long row) { return (__int128)(o.matrices - 1) * matrix + (o.rows - 1) * row + o.cols; };
  if (off >= last(o.g_matrix, o.g_row) || -off >= last(o.x_matrix, o.x_row)) return false;
  if (o.g_row == o.x_row && o.g_matrix == o.x_matrix) {   // the distances of matrices and of rows that come near `off`
    const auto below = [](long long v, long long by) { return v >= 0 ? v / by : -((by - 1 - v) / by); };
    const long long n0 = o.g_matrix ? below(off, o.g_matrix) : 0;
    for (long long n = n0; n <= n0 + (o.g_matrix ? 1 : 0); ++n) {
      const long long rest = off - n * o.g_matrix, i0 = below(rest, o.g_row);
      for (long long i = i0; i <= i0 + 1; ++i)
        if (n > -o.matrices && n < o.matrices && i > -o.rows && i < o.rows && std::llabs(rest - i * o.g_row) < o.cols) return true;
    }
    return false;
  }
  const long long rows = o.matrices * o.rows;
  for (long long g = 0, x = 0; g < rows && x < rows;) {
    const long long at = g / o.rows * o.g_matrix + g % o.rows * o.g_row, to = off + x / o.rows * o.x_matrix + x % o.rows * o.x_row;
    if (at < to + o.cols && to < at + o.cols) return true;
    at < to ? ++g : ++x;
  }
  return false;
}

int orthogonal_of(const qoda_orthogonalize_args *a, Orthogonal *o) {
  const char *call = "qoda_orthogonalize";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_type(call, a->dtype));
  TRY(check_sides(call, a->matrices, a->rows, a->cols));
  if (a->steps < 0 || a->steps > QODA_MAX_STEPS) return fail(QODA_EINVAL, "%s: %d steps, which are not in [0, %d]", call, a->steps, QODA_MAX_STEPS);
  if (!(a->eps >= 0.0) || !std::isfinite(a->eps)) return fail(QODA_EINVAL, "%s: eps = %g", call, a->eps);
  if (!std::isfinite(a->a) || !std::isfinite(a->b) || !std::isfinite(a->c) || !orthogonal_bounded(a->a, a->b, a->c, a->steps))
    return fail(QODA_EINVAL, "%s: %d steps with the coefficients %g, %g, %g may leave 2^40", call, a->steps, a->a, a->b, a->c);
  *o = {};
  o->type = a->dtype, o->steps = a->steps;
  o->matrices = a->matrices, o->rows = a->rows, o->cols = a->cols;
  if (a->matrices == 0 || a->rows == 0 || a->cols == 0) return QODA_OK;
  const int64_t least = a->rows < a->cols ? a->rows : a->cols, most = a->rows < a->cols ? a->cols : a->rows;
  if (least > kMostLeast || most > kMostSideOfUpdate)
    return fail(QODA_EINVAL, "%s: sides of %lld and %lld; %lld and %lld at most", call, (long long)least, (long long)most, (long long)kMostLeast, (long long)kMostSideOfUpdate);
  const size_t e = entry_bytes(a->dtype);
  TRY(check_matrices(call, "g", a->g, a->matrices, a->rows, a->cols, e, &o->g_row, &o->g_matrix));
  TRY(check_matrices(call, "x", a->x, a->matrices, a->rows, a->cols, e, &o->x_row, &o->x_matrix));
  o->g = a->g.data, o->x = a->x.data;
  if (overlapping(*o, e)) return fail(QODA_EINVAL, "%s: x is neither g nor apart from it", call);
  o->a = a->a, o->b = a->b, o->c = a->c, o->eps = a->eps;
  o->by_norm = orthogonal_by_norm(a->a, a->b, a->c, a->steps);
  orthogonal_sides(o);
  return QODA_OK;
}

bool nothing(const Orthogonal &o) { return o.matrices == 0 || o.rows == 0 || o.cols == 0; }

}  // namespace

extern "C" {

int64_t qoda_mx_code_bytes(int64_t rows, int64_t cols) {
  const int rc = check_sides("qoda_mx_code_bytes", rows, cols, 0);
  return rc != QODA_OK ? rc : (int64_t)code_bytes(rows, cols);
}

int64_t qoda_mx_scale_bytes(int64_t rows, int64_t cols) {
  const int rc = check_sides("qoda_mx_scale_bytes", rows, cols, 0);
  return rc != QODA_OK ? rc : (int64_t)scale_bytes(rows, cols);
}

int qoda_mx_quantize(const qoda_mx_quantize_args *a, void *stream) {
  MxRounding q;
  TRY(rounding_of(a, &q));
  if (q.rows == 0 || q.cols == 0) return QODA_OK;
  return done("qoda_mx_quantize", launch_mx_quantize(q, static_cast<hipStream_t>(stream)));
}

int qoda_mx_values(const qoda_mx_values_args *a, void *stream) {
  const char *call = "qoda_mx_values";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_type(call, a->dtype));
  TRY(check_sides(call, a->rows, a->cols, 0));
  TRY(check_mx(call, "q", a->q, a->rows, a->cols));
  TRY(check_matrix(call, "y", a->y, a->rows, a->cols, entry_bytes(a->dtype), false));
  if (a->rows == 0 || a->cols == 0) return QODA_OK;
  MxRounding q = {};
  q.type = a->dtype, q.rows = a->rows, q.cols = a->cols;
  q.x = a->y.data, q.ldx = stride_of(a->y, a->rows, a->cols);
  q.codes = static_cast<u8 *>(a->q.codes), q.scales = static_cast<u8 *>(a->q.scales);
  return done(call, launch_mx_values(q, static_cast<hipStream_t>(stream)));
}

int64_t qoda_mx_linear_workspace_bytes(const qoda_mx_linear_args *a) { return scratch_of(a, linear_of); }
int64_t qoda_mx_linear_input_grad_workspace_bytes(const qoda_mx_linear_input_grad_args *a) { return scratch_of(a, input_grad_of); }
int64_t qoda_mx_linear_weight_grad_workspace_bytes(const qoda_mx_linear_weight_grad_args *a) { return scratch_of(a, weight_grad_of); }

int qoda_mx_linear(const qoda_mx_linear_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  MxProduct m;
  TRY(linear_of(a, &m));
  return run("qoda_mx_linear", &m, workspace, workspace_bytes, stream);
}

int qoda_mx_linear_input_grad(const qoda_mx_linear_input_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  MxProduct m;
  TRY(input_grad_of(a, &m));
  return run("qoda_mx_linear_input_grad", &m, workspace, workspace_bytes, stream);
}

int qoda_mx_linear_weight_grad(const qoda_mx_linear_weight_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  MxProduct m;
  TRY(weight_grad_of(a, &m));
  return run("qoda_mx_linear_weight_grad", &m, workspace, workspace_bytes, stream);
}

int64_t qoda_orthogonalize_workspace_bytes(const qoda_orthogonalize_args *a) {
  Orthogonal o;
  const int rc = orthogonal_of(a, &o);
  return rc != QODA_OK ? rc : nothing(o) ? 0 : (int64_t)orthogonal_scratch(o);
}

int qoda_orthogonalize(const qoda_orthogonalize_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  Orthogonal o;
  TRY(orthogonal_of(a, &o));
  if (nothing(o)) return QODA_OK;
  TRY(check_workspace("qoda_orthogonalize", workspace, workspace_bytes, orthogonal_scratch(o)));
  return done("qoda_orthogonalize", launch_orthogonalize(o, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
