// C ABI of the operators of a language model's blocks (declared in include/abs.h): argument checks and launches.
#include <cmath>
#include <cstring>

#include "../../include/abs.h"
#include "api_status.h"
#include "operand_checks.h"
#include "ops.h"

using namespace absk;

namespace {

// ---- token embedding -------------------------------------------------------------------------------------------------

abs_status check_embedding(const abs_embedding_shape *s, bool backward) {
  if (!s) return set_error(ABS_EINVAL, "shape is NULL");
  if (s->M < 1 || s->b < 1 || s->T < 1 || s->V < 1 || s->D < 1) return set_error(ABS_EINVAL, "M, b, T, V and D must be at least 1");
  if (s->token_type != ABS_TYPE_I32 && s->token_type != ABS_TYPE_I64) return set_error(ABS_EINVAL, "token_type must be ABS_TYPE_I32 or ABS_TYPE_I64");
  if (!known_type(s->type) || (!backward && !known_type(s->table_type))) return set_error(ABS_EINVAL, "unknown type");
  const int64_t rows = (int64_t)s->b * s->T;
  // (a grid counts its threads in 32 bits, and up to 128 of them look at a sample)
  if (s->M > 1 << 20 || (int64_t)s->M * s->b > 1 << 25 || rows > 0x7fffffff / s->M || s->V > 1 << 30 || (int64_t)s->M * s->V > ((int64_t)1 << 46) / s->D)
    return set_error(ABS_EUNSUPPORTED, "more than 2^20 replicas, 2^25 samples, 2^31 - 1 tokens, 2^30 words or 2^46 values of tables");
  if (!strides_ok(s->M, s->stride_y, rows, s->ldy, s->D)) return set_error(ABS_EINVAL, "strides: ld >= D, and rows must not overlap");
  return ABS_OK;
}
EmbeddingP embedding_args(const abs_embedding_shape *s) {
  EmbeddingP p;
  std::memset(&p, 0, sizeof(p));
  p.M = s->M; p.b = s->b; p.T = s->T; p.V = s->V; p.D = s->D;
  p.wide = s->token_type == ABS_TYPE_I64; p.type = s->type; p.ttype = s->table_type; p.ldy = s->ldy; p.sy = s->stride_y;
  return p;
}
int token_bytes(const abs_embedding_shape *s) { return s->token_type == ABS_TYPE_I64 ? 8 : 4; }

// ---- root-mean-square norm -------------------------------------------------------------------------------------------

abs_status check_rms(const abs_rms_norm_shape *s, bool add) {
  if (!s) return set_error(ABS_EINVAL, "shape is NULL");
  if (s->M < 1 || s->b < 1 || s->T < 1 || s->D < 1) return set_error(ABS_EINVAL, "M, b, T and D must be at least 1");
  if (!known_type(s->type)) return set_error(ABS_EINVAL, "unknown type");
  if (s->param_type != s->type && s->param_type != ABS_TYPE_F32) return set_error(ABS_EINVAL, "param_type must be ABS_TYPE_F32 or type");
  const int64_t rows = (int64_t)s->b * s->T;
  // (a grid counts its threads in 32 bits, and 512 of them add the partial gradients of 64 gains)
  if (s->M > 1 << 20 || (int64_t)s->M * s->D > 1 << 27 || rows > 0x7fffffff / s->M)
    return set_error(ABS_EUNSUPPORTED, "more than 2^20 replicas, 2^27 gains or 2^31 - 1 rows");
  if (!strides_ok(s->M, s->stride_x, rows, s->ldx, s->D) || !strides_ok(s->M, s->stride_y, rows, s->ldy, s->D) ||
      (add && (!strides_ok(s->M, s->stride_r, rows, s->ldr, s->D) || !strides_ok(s->M, s->stride_h, rows, s->ldh, s->D))))
    return set_error(ABS_EINVAL, "strides: ld >= D, and rows must not overlap");
  return ABS_OK;
}
RmsNormP rms_args(const abs_rms_norm_shape *s) {
  RmsNormP p;
  std::memset(&p, 0, sizeof(p));
  p.M = s->M; p.b = s->b; p.T = s->T; p.D = s->D; p.type = s->type; p.ptype = s->param_type;
  p.ldx = s->ldx; p.sx = s->stride_x; p.ldr = s->ldr; p.sr = s->stride_r; p.ldh = s->ldh; p.sh = s->stride_h; p.ldy = s->ldy; p.sy = s->stride_y;
  return p;
}

}  // namespace

extern "C" {

abs_status abs_embedding(const abs_embedding_shape *shape, const void *tokens_dev, const void *table_dev, float scale, void *y_dev, void *hip_stream) try {
  abs_status st = check_embedding(shape, false);
  if (st != ABS_OK) return st;
  if (!tokens_dev || !table_dev || !y_dev) return set_error(ABS_EINVAL, "NULL argument");
  if (!std::isfinite(scale)) return set_error(ABS_EINVAL, "scale must be finite");
  const int e = type_bytes(shape->type), te = type_bytes(shape->table_type), ke = token_bytes(shape);
  if (!aligned_to(tokens_dev, ke) || !aligned_to(table_dev, te) || !aligned_to(y_dev, e)) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const int64_t rows = (int64_t)shape->b * shape->T;
  const Block in[] = {piece(tokens_dev, shape->M * rows, ke), piece(table_dev, (int64_t)shape->M * shape->V * shape->D, te)};
  const Block out[] = {{y_dev, shape->M, shape->stride_y, rows, shape->ldy, shape->D, e}};
  if (outputs_overlap(out, in)) return set_error(ABS_EINVAL, "y_dev must not overlap an input");
  EmbeddingP p = embedding_args(shape);
  p.tokens = tokens_dev; p.table = table_dev; p.scale = scale; p.y = y_dev;
  return hip_status(launch_embedding(p, static_cast<hipStream_t>(hip_stream)), "abs_embedding");
} catch (...) { return exception_status(); }

abs_status abs_embedding_backward_workspace_bytes(const abs_embedding_shape *shape, int want_n, int want_q, size_t *bytes) try {
  if (!bytes) return set_error(ABS_EINVAL, "bytes is NULL");
  abs_status st = check_embedding(shape, true);
  if (st != ABS_OK) return st;
  *bytes = embedding_backward_bytes(embedding_args(shape), want_n != 0, want_q != 0);
  return ABS_OK;
} catch (...) { return exception_status(); }

abs_status abs_embedding_backward(const abs_embedding_shape *shape, const void *dy_dev, const void *tokens_dev, float scale, float *dtable_dev,
                                  float *n_dev, float *q_dev, void *workspace, size_t workspace_bytes, void *hip_stream) try {
  abs_status st = check_embedding(shape, true);
  if (st != ABS_OK) return st;
  if (!dy_dev || !tokens_dev || !dtable_dev) return set_error(ABS_EINVAL, "NULL argument");
  if (!std::isfinite(scale)) return set_error(ABS_EINVAL, "scale must be finite");
  if (!workspace || !aligned_to(workspace, 256)) return set_error(ABS_EINVAL, "workspace must be a 256-byte aligned device pointer");
  EmbeddingP p = embedding_args(shape);
  const size_t need = embedding_backward_bytes(p, n_dev != nullptr, q_dev != nullptr);
  if (workspace_bytes < need) return set_error(ABS_ENOMEM, "workspace too small (see abs_embedding_backward_workspace_bytes)");
  const int e = type_bytes(shape->type), ke = token_bytes(shape);
  if (!aligned_to(tokens_dev, ke) || !aligned_to(dy_dev, e) || !aligned_to(dtable_dev, 4) || !aligned_to(n_dev, 4) || !aligned_to(q_dev, 4))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const int64_t rows = (int64_t)shape->b * shape->T, samples = (int64_t)shape->M * shape->b;
  const Block in[] = {{dy_dev, shape->M, shape->stride_y, rows, shape->ldy, shape->D, e}, piece(tokens_dev, shape->M * rows, ke)};
  const Block out[] = {piece(dtable_dev, (int64_t)shape->M * shape->V * shape->D, 4), piece(n_dev, samples, 4), piece(q_dev, samples, 4),
                       piece(workspace, (int64_t)need, 1)};
  if (outputs_overlap(out, in)) return set_error(ABS_EINVAL, "outputs and the workspace must not overlap an input or each other");
  p.dy = dy_dev; p.tokens = tokens_dev; p.scale = scale; p.dtable = dtable_dev; p.n = n_dev; p.q = q_dev;
  return hip_status(launch_embedding_backward(p, workspace, static_cast<hipStream_t>(hip_stream)), "abs_embedding_backward");
} catch (...) { return exception_status(); }

abs_status abs_rms_norm(const abs_rms_norm_shape *shape, const void *x_dev, const void *residual_dev, const void *w_dev, float eps, void *h_dev,
                        void *y_dev, float *scale_dev, float *rstd_dev, void *hip_stream) try {
  abs_status st = check_rms(shape, residual_dev != nullptr);
  if (st != ABS_OK) return st;
  if (!x_dev || !w_dev || !y_dev) return set_error(ABS_EINVAL, "NULL argument");
  if ((residual_dev != nullptr) != (h_dev != nullptr)) return set_error(ABS_EINVAL, "h_dev is given where residual_dev is, and nowhere else");
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(ABS_EINVAL, "eps must be finite and not negative");
  const int e = type_bytes(shape->type), pe = type_bytes(shape->param_type), ye = scale_dev ? 1 : e;
  if (!aligned_to(x_dev, e) || !aligned_to(residual_dev, e) || !aligned_to(h_dev, e) || !aligned_to(y_dev, ye) || !aligned_to(w_dev, pe) ||
      !aligned_to(scale_dev, 4) || !aligned_to(rstd_dev, 4))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const int64_t rows = (int64_t)shape->b * shape->T, all = shape->M * rows;
  const Block x = {x_dev, shape->M, shape->stride_x, rows, shape->ldx, shape->D, e}, r = {residual_dev, shape->M, shape->stride_r, rows, shape->ldr, shape->D, e},
              h = {h_dev, shape->M, shape->stride_h, rows, shape->ldh, shape->D, e}, y = {y_dev, shape->M, shape->stride_y, rows, shape->ldy, shape->D, ye};
  // a result may take the place of an operand that it is made of, of the same strides
  auto in_place = [&](const Block &o, const Block &i) { return o.p == i.p && o.bytes == i.bytes && o.stride == i.stride && o.ld == i.ld; };
  for (const Block *o : {&h, &y})
    for (const Block *i : {&x, &r})
      if (o->p && i->p && !in_place(*o, *i) && overlap(*o, *i)) return set_error(ABS_EINVAL, "h_dev and y_dev must be x_dev or residual_dev or not overlap them");
  const Block out[] = {y, h, piece(scale_dev, all, 4), piece(rstd_dev, all, 4)}, small[] = {out[2], out[3]};
  const Block params[] = {piece(w_dev, (int64_t)shape->M * shape->D, pe)}, big[] = {x, r};
  if (outputs_overlap(out, params) || outputs_overlap(small, big))
    return set_error(ABS_EINVAL, "outputs must not overlap the gains, each other, or (scale_dev, rstd_dev) an input");
  RmsNormP p = rms_args(shape);
  p.x = x_dev; p.res = residual_dev; p.w = w_dev; p.eps = eps; p.h = h_dev; p.y = y_dev; p.scale = scale_dev; p.rstd = rstd_dev;
  return hip_status(launch_rms_norm(p, static_cast<hipStream_t>(hip_stream)), "abs_rms_norm");
} catch (...) { return exception_status(); }

abs_status abs_rms_norm_backward_workspace_bytes(const abs_rms_norm_shape *shape, int want_n, int want_q, size_t *bytes) try {
  if (!bytes) return set_error(ABS_EINVAL, "bytes is NULL");
  abs_status st = check_rms(shape, false);
  if (st != ABS_OK) return st;
  *bytes = rms_norm_backward_bytes(rms_args(shape), want_n != 0, want_q != 0);
  return ABS_OK;
} catch (...) { return exception_status(); }

abs_status abs_rms_norm_backward(const abs_rms_norm_shape *shape, const void *dy_dev, const void *h_dev, const void *dh_dev, const void *w_dev,
                                 const float *rstd_dev, void *dx_dev, float *dw_dev, float *n_dev, float *q_dev, void *workspace,
                                 size_t workspace_bytes, void *hip_stream) try {
  abs_status st = check_rms(shape, false);
  if (st != ABS_OK) return st;
  if (!dy_dev || !h_dev || !w_dev || !rstd_dev || !dx_dev || !dw_dev) return set_error(ABS_EINVAL, "NULL argument");
  const int64_t rows = (int64_t)shape->b * shape->T, all = shape->M * rows, samples = (int64_t)shape->M * shape->b, gains = (int64_t)shape->M * shape->D;
  if (!strides_ok(shape->M, shape->stride_h, rows, shape->ldh, shape->D) || (dh_dev && !strides_ok(shape->M, shape->stride_r, rows, shape->ldr, shape->D)))
    return set_error(ABS_EINVAL, "strides: ld >= D, and rows must not overlap");
  if (!workspace || !aligned_to(workspace, 256)) return set_error(ABS_EINVAL, "workspace must be a 256-byte aligned device pointer");
  RmsNormP p = rms_args(shape);
  const size_t need = rms_norm_backward_bytes(p, n_dev != nullptr, q_dev != nullptr);
  if (workspace_bytes < need) return set_error(ABS_ENOMEM, "workspace too small (see abs_rms_norm_backward_workspace_bytes)");
  const int e = type_bytes(shape->type), pe = type_bytes(shape->param_type);
  if (!aligned_to(dy_dev, e) || !aligned_to(h_dev, e) || !aligned_to(dh_dev, e) || !aligned_to(dx_dev, e) || !aligned_to(w_dev, pe))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  for (const void *f : {(const void *)rstd_dev, (const void *)dw_dev, (const void *)n_dev, (const void *)q_dev})
    if (!aligned_to(f, 4)) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const Block in[] = {{h_dev, shape->M, shape->stride_x, rows, shape->ldx, shape->D, e}, {dy_dev, shape->M, shape->stride_y, rows, shape->ldy, shape->D, e},
                      {dh_dev, shape->M, shape->stride_r, rows, shape->ldr, shape->D, e}, piece(w_dev, gains, pe), piece(rstd_dev, all, 4)};
  const Block out[] = {{dx_dev, shape->M, shape->stride_h, rows, shape->ldh, shape->D, e}, piece(dw_dev, gains, 4), piece(n_dev, samples, 4),
                       piece(q_dev, samples, 4), piece(workspace, (int64_t)need, 1)};
  if (outputs_overlap(out, in)) return set_error(ABS_EINVAL, "outputs and the workspace must not overlap an input or each other");
  p.x = h_dev; p.res = dh_dev; p.w = w_dev; p.rstd = const_cast<float *>(rstd_dev); p.dy = dy_dev; p.dx = dx_dev; p.dw = dw_dev; p.n = n_dev; p.q = q_dev;
  return hip_status(launch_rms_norm_backward(p, workspace, static_cast<hipStream_t>(hip_stream)), "abs_rms_norm_backward");
} catch (...) { return exception_status(); }

}  // extern "C"
