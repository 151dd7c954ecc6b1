// Host side of the operators declared in include/qoda_operators.h: checks of arguments, and the kernels' arguments from the caller's.

#include <hip/hip_runtime.h>

#include "qoda_operators_checks.h"

using namespace qoda;

namespace {

int linear_product(const qoda_linear_args *a, Product *p) {
  const char *call = "qoda_linear";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_sides(call, a->rows, a->in, a->out));
  *p = {};
  TRY(make_drop(call, a->p, a->seed, a->offset, &p->drop));
  const size_t e = entry_bytes(a->dtype);
  TRY(check_matrix(call, "x", a->x, a->rows, a->in, e, a->out == 0));
  TRY(check_matrix(call, "w", a->w, a->out, a->in, e, a->rows == 0));
  TRY(check_matrix(call, "residual", a->residual, a->rows, a->out, e, true));
  TRY(check_matrix(call, "y", a->y, a->rows, a->out, e, false));
  TRY(check_matrix(call, "pre", a->pre, a->rows, a->out, e, true));
  if (!aligned(a->bias, 4)) return fail(QODA_EINVAL, "%s: bias is not aligned to its entries", call);
  p->form = kProductRows;
  p->type = a->dtype;
  p->m = (int)a->rows, p->n = (int)a->out, p->k = (int)a->in;
  p->a = a->x.data, p->lda = stride_of(a->x, a->rows, a->in);
  p->b = a->w.data, p->ldb = stride_of(a->w, a->out, a->in);
  p->out = a->y.data, p->ldo = stride_of(a->y, a->rows, a->out);
  p->pre = a->pre.data, p->ldp = stride_of(a->pre, a->rows, a->out);
  p->extra = a->residual.data, p->lde = stride_of(a->residual, a->rows, a->out);
  p->bias = a->bias;
  p->activation = a->activation;
  return QODA_OK;
}

int input_grad_product(const qoda_linear_input_grad_args *a, Product *p) {
  const char *call = "qoda_linear_input_grad";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_sides(call, a->rows, a->in, a->out));
  *p = {};
  TRY(make_drop(call, a->p, a->seed, a->offset, &p->drop));
  const size_t e = entry_bytes(a->dtype);
  TRY(check_matrix(call, "dz", a->dz, a->rows, a->out, e, a->in == 0));
  TRY(check_matrix(call, "w", a->w, a->out, a->in, e, a->rows == 0));
  TRY(check_matrix(call, "pre", a->pre, a->rows, a->in, e, a->activation == kActNone));
  TRY(check_matrix(call, "residual", a->residual, a->rows, a->in, e, true));
  TRY(check_matrix(call, "dx", a->dx, a->rows, a->in, e, false));
  p->form = kProductMixed;
  p->type = a->dtype;
  p->m = (int)a->rows, p->n = (int)a->in, p->k = (int)a->out;
  p->a = a->dz.data, p->lda = stride_of(a->dz, a->rows, a->out);
  p->b = a->w.data, p->ldb = stride_of(a->w, a->out, a->in);
  p->out = a->dx.data, p->ldo = stride_of(a->dx, a->rows, a->in);
  p->pre = a->activation == kActNone ? nullptr : a->pre.data, p->ldp = stride_of(a->pre, a->rows, a->in);
  p->extra = a->residual.data, p->lde = stride_of(a->residual, a->rows, a->in);
  p->activation = a->activation;
  return QODA_OK;
}

int weight_grad_product(const qoda_linear_weight_grad_args *a, Product *p) {
  const char *call = "qoda_linear_weight_grad";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, kActNone));
  TRY(check_sides(call, a->rows, a->in, a->out));
  *p = {};
  const size_t e = entry_bytes(a->dtype);
  TRY(check_matrix(call, "dz", a->dz, a->rows, a->out, e, false));
  TRY(check_matrix(call, "x", a->x, a->rows, a->in, e, a->out == 0));
  TRY(check_matrix(call, "dw", a->dw, a->out, a->in, 4, false));
  if (!aligned(a->dbias, 4)) return fail(QODA_EINVAL, "%s: dbias is not aligned to its entries", call);
  p->form = kProductColumns;
  p->type = a->dtype;
  p->m = (int)a->out, p->n = (int)a->in, p->k = (int)a->rows;
  p->a = a->dz.data, p->lda = stride_of(a->dz, a->rows, a->out);
  p->b = a->x.data, p->ldb = stride_of(a->x, a->rows, a->in);
  p->out = a->dw.data, p->ldo = stride_of(a->dw, a->out, a->in);
  p->sums = a->dbias;
  p->accumulate = a->accumulate != 0;
  return QODA_OK;
}

int run_product(const char *call, Product *p, void *workspace, size_t bytes, void *stream) {
  if (p->m == 0 || (p->n == 0 && !p->sums)) return QODA_OK;
  TRY(check_workspace(call, workspace, bytes, product_scratch(*p)));
  p->partial = static_cast<float *>(workspace);
  return done(call, launch_product(*p, static_cast<hipStream_t>(stream)));
}

template <class Args>
int64_t scratch_of(const Args *a, int (*make)(const Args *, Product *)) {
  Product p;
  const int rc = make(a, &p);
  return rc != QODA_OK ? rc : (int64_t)product_scratch(p);
}

int run_entries(const char *call, const qoda_dropout_args *a, bool gradient, void *stream) {
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_sides(call, a->rows, a->cols, 0));
  Entries e = {};
  TRY(make_drop(call, a->p, a->seed, a->offset, &e.drop));
  const size_t b = entry_bytes(a->dtype);
  TRY(check_matrix(call, "x", a->x, a->rows, a->cols, b, false));
  TRY(check_matrix(call, gradient ? "extra (the activation's input)" : "extra (the residual)", a->extra, a->rows, a->cols, b,
                   !gradient || a->activation == kActNone));
  TRY(check_matrix(call, "y", a->y, a->rows, a->cols, b, false));
  if (a->rows == 0 || a->cols == 0) return QODA_OK;
  e.type = a->dtype, e.activation = a->activation, e.gradient = gradient;
  e.rows = a->rows, e.cols = a->cols;
  e.x = a->x.data, e.ldx = stride_of(a->x, a->rows, a->cols);
  e.extra = gradient && a->activation == kActNone ? nullptr : a->extra.data, e.lde = stride_of(a->extra, a->rows, a->cols);
  e.y = a->y.data, e.ldy = stride_of(a->y, a->rows, a->cols);
  return done(call, launch_entries(e, static_cast<hipStream_t>(stream)));
}

struct Values { long long sample, position; };

int check_values(const char *call, const char *name, const qoda_channels_last &v, int64_t samples, int64_t positions, int64_t channels,
                 size_t bytes, bool optional, Values *out) {
  // a stride that no entry is reached by is not looked at
  out->position = positions > 1 ? v.position : channels;
  out->sample = samples > 1 ? v.sample : 0;
  if (samples == 0 || positions == 0 || channels == 0) return QODA_OK;
  if (!v.data) return optional ? QODA_OK : fail(QODA_EINVAL, "%s: %s is null", call, name);
  if (!aligned(v.data, bytes)) return fail(QODA_EINVAL, "%s: %s is not aligned to its entries", call, name);
  // positions apart by at least the channels, samples by at least what the positions span: no two entries share an address
  if (out->position < channels || out->position >= kMostStride ||
      (samples > 1 && (out->sample < (__int128)(positions - 1) * out->position + channels || out->sample >= kMostStride * 1024)))
    return fail(QODA_EINVAL, "%s: the strides of %s do not fit its %lld channels and %lld positions", call, name, (long long)channels, (long long)positions);
  return QODA_OK;
}

int check_groups(const char *call, int64_t samples, int64_t positions, int64_t channels, int64_t groups) {
  TRY(check_sides(call, samples, positions, channels));
  if (groups < 1 || channels % groups != 0 || groups > kMostSide)
    return fail(QODA_EINVAL, "%s: %lld groups do not divide %lld channels", call, (long long)groups, (long long)channels);
  if (samples * groups >= (int64_t)1 << 31) return fail(QODA_EINVAL, "%s: %lld samples of %lld groups are 2^31 statistics or more", call, (long long)samples, (long long)groups);
  return QODA_OK;
}

int check_vectors(const char *call, std::initializer_list<const void *> vs) {
  for (const void *v : vs)
    if (!aligned(v, 4)) return fail(QODA_EINVAL, "%s: a vector of fp32 is not aligned to its entries", call);
  return QODA_OK;
}

int norm_of(const qoda_group_norm_args *a, GroupNorm *g) {
  const char *call = "qoda_group_norm";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_groups(call, a->samples, a->positions, a->channels, a->groups));
  if (!(a->eps >= 0.0) || !std::isfinite(a->eps)) return fail(QODA_EINVAL, "%s: eps = %g", call, a->eps);
  const size_t b = entry_bytes(a->dtype);
  Values x, y;
  TRY(check_values(call, "x", a->x, a->samples, a->positions, a->channels, b, false, &x));
  TRY(check_values(call, "y", a->y, a->samples, a->positions, a->channels, b, false, &y));
  if (a->samples && a->positions && a->channels && (!a->mean || !a->rstd)) return fail(QODA_EINVAL, "%s: mean or rstd is null", call);
  TRY(check_vectors(call, {a->weight, a->bias, a->mean, a->rstd}));
  *g = {};
  g->type = a->dtype, g->activation = a->activation;
  g->samples = a->samples, g->positions = a->positions, g->channels = a->channels, g->groups = a->groups;
  g->x = a->x.data, g->x_sample = x.sample, g->x_pos = x.position;
  g->out = a->y.data, g->out_sample = y.sample, g->out_pos = y.position;
  g->weight = a->weight, g->bias = a->bias, g->mean = a->mean, g->rstd = a->rstd;
  g->eps = (float)a->eps;
  return QODA_OK;
}

int norm_grad_of(const qoda_group_norm_grad_args *a, GroupNorm *g) {
  const char *call = "qoda_group_norm_grad";
  if (!a) return fail(QODA_EINVAL, "%s: null arguments", call);
  TRY(check_common(call, a->dtype, a->activation));
  TRY(check_groups(call, a->samples, a->positions, a->channels, a->groups));
  const size_t b = entry_bytes(a->dtype);
  Values dy, x, r, dx;
  TRY(check_values(call, "dy", a->dy, a->samples, a->positions, a->channels, b, false, &dy));
  TRY(check_values(call, "x", a->x, a->samples, a->positions, a->channels, b, false, &x));
  TRY(check_values(call, "residual", a->residual, a->samples, a->positions, a->channels, b, true, &r));
  TRY(check_values(call, "dx", a->dx, a->samples, a->positions, a->channels, b, false, &dx));
  if (a->samples && a->positions && a->channels && (!a->mean || !a->rstd)) return fail(QODA_EINVAL, "%s: mean or rstd is null", call);
  TRY(check_vectors(call, {a->weight, a->bias, a->mean, a->rstd, a->dweight, a->dbias}));
  *g = {};
  g->type = a->dtype, g->activation = a->activation, g->accumulate = a->accumulate != 0;
  g->samples = a->samples, g->positions = a->positions, g->channels = a->channels, g->groups = a->groups;
  g->dy = a->dy.data, g->dy_sample = dy.sample, g->dy_pos = dy.position;
  g->x = a->x.data, g->x_sample = x.sample, g->x_pos = x.position;
  g->extra = a->residual.data, g->extra_sample = r.sample, g->extra_pos = r.position;
  g->out = a->dx.data, g->out_sample = dx.sample, g->out_pos = dx.position;
  g->weight = a->weight, g->bias = a->bias;
  g->mean = const_cast<float *>(a->mean), g->rstd = const_cast<float *>(a->rstd);
  g->dweight = a->dweight, g->dbias = a->dbias;
  return QODA_OK;
}

}  // namespace

extern "C" {

int64_t qoda_linear_workspace_bytes(const qoda_linear_args *a) { return scratch_of(a, linear_product); }
int64_t qoda_linear_input_grad_workspace_bytes(const qoda_linear_input_grad_args *a) { return scratch_of(a, input_grad_product); }
int64_t qoda_linear_weight_grad_workspace_bytes(const qoda_linear_weight_grad_args *a) { return scratch_of(a, weight_grad_product); }

int qoda_linear(const qoda_linear_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  Product p;
  TRY(linear_product(a, &p));
  return run_product("qoda_linear", &p, workspace, workspace_bytes, stream);
}

int qoda_linear_input_grad(const qoda_linear_input_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  Product p;
  TRY(input_grad_product(a, &p));
  return run_product("qoda_linear_input_grad", &p, workspace, workspace_bytes, stream);
}

int qoda_linear_weight_grad(const qoda_linear_weight_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  Product p;
  TRY(weight_grad_product(a, &p));
  return run_product("qoda_linear_weight_grad", &p, workspace, workspace_bytes, stream);
}

int qoda_dropout(const qoda_dropout_args *a, void *stream) { return run_entries("qoda_dropout", a, false, stream); }
int qoda_dropout_grad(const qoda_dropout_args *a, void *stream) { return run_entries("qoda_dropout_grad", a, true, stream); }

int64_t qoda_group_norm_workspace_bytes(const qoda_group_norm_args *a) {
  GroupNorm g;
  const int rc = norm_of(a, &g);
  return rc != QODA_OK ? rc : (int64_t)group_norm_scratch(g, false);
}

int64_t qoda_group_norm_grad_workspace_bytes(const qoda_group_norm_grad_args *a) {
  GroupNorm g;
  const int rc = norm_grad_of(a, &g);
  return rc != QODA_OK ? rc : (int64_t)group_norm_scratch(g, true);
}

int qoda_group_norm(const qoda_group_norm_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  GroupNorm g;
  TRY(norm_of(a, &g));
  if (g.samples == 0 || g.positions == 0 || g.channels == 0) return QODA_OK;
  TRY(check_workspace("qoda_group_norm", workspace, workspace_bytes, group_norm_scratch(g, false)));
  g.scratch = static_cast<float *>(workspace);
  return done("qoda_group_norm", launch_group_norm(g, static_cast<hipStream_t>(stream)));
}

int qoda_group_norm_grad(const qoda_group_norm_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  GroupNorm g;
  TRY(norm_grad_of(a, &g));
  if (g.channels == 0) return QODA_OK;
  if ((g.samples == 0 || g.positions == 0) && (g.accumulate || (!g.dweight && !g.dbias))) return QODA_OK;
  TRY(check_workspace("qoda_group_norm_grad", workspace, workspace_bytes, group_norm_scratch(g, true)));
  g.scratch = static_cast<float *>(workspace);
  return done("qoda_group_norm_grad", launch_group_norm_grad(g, static_cast<hipStream_t>(stream)));
}

const char *qoda_operator_error(void) { return operator_error; }

}  // extern "C"
