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

// ---- causal attention ------------------------------------------------------------------------------------------------

// Heads of rows of D values: blocks of [heads][rows][D], head after head or (as projections leave them) interleaved by rows
Block heads_of(const void *t, const abs_attention_shape *s, int heads, int64_t ld, int64_t head) {
  return {t, heads, head, s->rows, ld, s->D, type_bytes(s->type)};
}
AttentionP attention_args(const abs_attention_shape *s) {
  AttentionP p;
  std::memset(&p, 0, sizeof(p));
  p.type = s->type; p.Hq = s->Hq; p.Hkv = s->Hkv; p.D = s->D; p.seqs = s->seqs; p.T = s->T; p.rows = s->rows;
  p.wide = s->offsets_type == ABS_TYPE_I64;
  p.ldq = s->ldq; p.hq = s->head_q; p.ldk = s->ldk; p.hk = s->head_k; p.ldv = s->ldv; p.hv = s->head_v; p.ldo = s->ldo; p.ho = s->head_o;
  p.lddo = s->lddo; p.hdo = s->head_do; p.lddq = s->lddq; p.hdq = s->head_dq; p.lddk = s->lddk; p.hdk = s->head_dk; p.lddv = s->lddv; p.hdv = s->head_dv;
  return p;
}
int64_t shape_tiles(const abs_attention_shape *s) {
  AttentionP p = attention_args(s);
  p.offsets = s->offsets_type ? s : nullptr;             // (asked whether there are any)
  return attention_tiles(p);
}
struct AttentionPieces { size_t list, inner, most, total; };
AttentionPieces attention_pieces(const abs_attention_shape *s, bool backward) {
  AttentionPieces q;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t r = at; at = (at + bytes + 255) / 256 * 256; return r; };
  q.list = take(s->offsets_type && s->seqs > 64 ? ((size_t)shape_tiles(s) + 1) * 8 : 0);
  q.inner = take(backward ? (size_t)s->Hq * s->rows * 4 : 0);
  q.most = take(backward && s->type == ABS_TYPE_F16 ? (size_t)shape_tiles(s) * (s->Hq + s->Hkv) * 4 : 0);
  q.total = at;
  return q;
}
abs_status check_attention(const abs_attention_shape *s, bool backward) {
  if (!s) return set_error(ABS_EINVAL, "shape is NULL");
  if (!known_type(s->type)) return set_error(ABS_EINVAL, "unknown type");
  if (s->offsets_type && s->offsets_type != ABS_TYPE_I32 && s->offsets_type != ABS_TYPE_I64)
    return set_error(ABS_EINVAL, "offsets_type must be ABS_TYPE_I32, ABS_TYPE_I64, or 0 for sequences of T rows");
  if (s->seqs < 1 || s->rows < 1 || s->Hq < 1 || s->Hkv < 1 || s->D < 1) return set_error(ABS_EINVAL, "seqs, rows, Hq, Hkv and D must be at least 1");
  if (s->Hq % s->Hkv) return set_error(ABS_EINVAL, "Hq must be a multiple of Hkv");
  if (!s->offsets_type && (s->T < 1 || (int64_t)s->seqs * s->T != s->rows)) return set_error(ABS_EINVAL, "without offsets rows must be seqs times T");
  if (s->D > ATTENTION_MAX_D) return set_error(ABS_EUNSUPPORTED, "heads of more than 128 values");
  if (s->rows > 0x7fffffff) return set_error(ABS_EUNSUPPORTED, "more than 2^31 - 1 rows");
  if (shape_tiles(s) > 0x7f0000 / s->Hq) return set_error(ABS_EUNSUPPORTED, "more heads of 128-row tiles than a grid counts");
  const int heads[8] = {s->Hq, s->Hkv, s->Hkv, s->Hq, s->Hq, s->Hq, s->Hkv, s->Hkv};
  const int64_t ld[8] = {s->ldq, s->ldk, s->ldv, s->ldo, s->lddo, s->lddq, s->lddk, s->lddv};
  const int64_t head[8] = {s->head_q, s->head_k, s->head_v, s->head_o, s->head_do, s->head_dq, s->head_dk, s->head_dv};
  for (int i = 0; i < (backward ? 8 : 4); ++i)
    if (!strides_ok(heads[i], head[i], s->rows, ld[i], s->D)) return set_error(ABS_EINVAL, "strides: ld >= D, and rows and heads must not overlap");
  return ABS_OK;
}
abs_status check_attention_call(const abs_attention_shape *s, const void *offsets, float scale, const void *workspace, size_t have, size_t need) {
  if ((offsets != nullptr) != (s->offsets_type != 0)) return set_error(ABS_EINVAL, "offsets_dev is given where there is an offsets_type, and nowhere else");
  if (!aligned_to(offsets, s->offsets_type == ABS_TYPE_I64 ? 8 : 4)) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  if (!(scale > 0.0f) || !std::isfinite(scale)) return set_error(ABS_EINVAL, "scale must be positive and finite");
  if (need && (!workspace || !aligned_to(workspace, 256))) return set_error(ABS_EINVAL, "workspace must be a 256-byte aligned device pointer");
  if (have < need) return set_error(ABS_ENOMEM, "workspace too small (see abs_causal_attention_workspace_bytes)");
  return ABS_OK;
}
Block offsets_of(const abs_attention_shape *s, const void *offsets) { return piece(offsets, (int64_t)s->seqs + 1, s->offsets_type == ABS_TYPE_I64 ? 8 : 4); }

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

abs_status abs_causal_attention_workspace_bytes(const abs_attention_shape *shape, int backward, size_t *bytes) try {
  if (!bytes) return set_error(ABS_EINVAL, "bytes is NULL");
  abs_status st = check_attention(shape, backward != 0);
  if (st != ABS_OK) return st;
  *bytes = attention_pieces(shape, backward != 0).total;
  return ABS_OK;
} catch (...) { return exception_status(); }

abs_status abs_causal_attention(const abs_attention_shape *shape, const void *q_dev, const void *k_dev, const void *v_dev, const void *offsets_dev,
                                float scale, void *o_dev, float *lse_dev, int zero_rest, void *workspace, size_t workspace_bytes, void *hip_stream) try {
  abs_status st = check_attention(shape, false);
  if (st != ABS_OK) return st;
  if (!q_dev || !k_dev || !v_dev || !o_dev) return set_error(ABS_EINVAL, "NULL argument");
  const AttentionPieces at = attention_pieces(shape, false);
  st = check_attention_call(shape, offsets_dev, scale, workspace, workspace_bytes, at.total);
  if (st != ABS_OK) return st;
  const int e = type_bytes(shape->type);
  if (!aligned_to(q_dev, e) || !aligned_to(k_dev, e) || !aligned_to(v_dev, e) || !aligned_to(o_dev, e) || !aligned_to(lse_dev, 4))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const Block in[] = {heads_of(q_dev, shape, shape->Hq, shape->ldq, shape->head_q), heads_of(k_dev, shape, shape->Hkv, shape->ldk, shape->head_k),
                      heads_of(v_dev, shape, shape->Hkv, shape->ldv, shape->head_v), offsets_of(shape, offsets_dev)};
  const Block out[] = {heads_of(o_dev, shape, shape->Hq, shape->ldo, shape->head_o), piece(lse_dev, shape->Hq * shape->rows, 4),
                       piece(at.total ? workspace : nullptr, (int64_t)at.total, 1)};
  if (outputs_overlap(out, in)) return set_error(ABS_EINVAL, "outputs and the workspace must not overlap an input or each other");
  AttentionP p = attention_args(shape);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  p.q = q_dev; p.k = k_dev; p.v = v_dev; p.offsets = offsets_dev; p.scale = scale; p.o = o_dev; p.lse = lse_dev; p.zero_rest = zero_rest != 0;
  p.list = reinterpret_cast<const int2 *>(ws + at.list);
  return hip_status(launch_attention(p, static_cast<hipStream_t>(hip_stream)), "abs_causal_attention");
} catch (...) { return exception_status(); }

abs_status abs_causal_attention_backward(const abs_attention_shape *shape, const void *do_dev, const void *q_dev, const void *k_dev, const void *v_dev,
                                         const void *o_dev, const float *lse_dev, const void *offsets_dev, float scale, void *dq_dev, void *dk_dev,
                                         void *dv_dev, int zero_rest, void *workspace, size_t workspace_bytes, void *hip_stream) try {
  abs_status st = check_attention(shape, true);
  if (st != ABS_OK) return st;
  if (!do_dev || !q_dev || !k_dev || !v_dev || !o_dev || !lse_dev || !dq_dev || !dk_dev || !dv_dev) return set_error(ABS_EINVAL, "NULL argument");
  const AttentionPieces at = attention_pieces(shape, true);
  st = check_attention_call(shape, offsets_dev, scale, workspace, workspace_bytes, at.total);
  if (st != ABS_OK) return st;
  const int e = type_bytes(shape->type);
  for (const void *t : {do_dev, q_dev, k_dev, v_dev, o_dev, (const void *)dq_dev, (const void *)dk_dev, (const void *)dv_dev})
    if (!aligned_to(t, e)) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  if (!aligned_to(lse_dev, 4)) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const Block in[] = {heads_of(do_dev, shape, shape->Hq, shape->lddo, shape->head_do), heads_of(q_dev, shape, shape->Hq, shape->ldq, shape->head_q),
                      heads_of(k_dev, shape, shape->Hkv, shape->ldk, shape->head_k), heads_of(v_dev, shape, shape->Hkv, shape->ldv, shape->head_v),
                      heads_of(o_dev, shape, shape->Hq, shape->ldo, shape->head_o), piece(lse_dev, shape->Hq * shape->rows, 4), offsets_of(shape, offsets_dev)};
  const Block out[] = {heads_of(dq_dev, shape, shape->Hq, shape->lddq, shape->head_dq), heads_of(dk_dev, shape, shape->Hkv, shape->lddk, shape->head_dk),
                       heads_of(dv_dev, shape, shape->Hkv, shape->lddv, shape->head_dv), piece(workspace, (int64_t)at.total, 1)};
  if (outputs_overlap(out, in)) return set_error(ABS_EINVAL, "outputs and the workspace must not overlap an input or each other");
  AttentionP p = attention_args(shape);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  p.dout = do_dev; p.q = q_dev; p.k = k_dev; p.v = v_dev; p.o = const_cast<void *>(o_dev); p.lse = const_cast<float *>(lse_dev);
  p.offsets = offsets_dev; p.scale = scale; p.dq = dq_dev; p.dk = dk_dev; p.dv = dv_dev; p.zero_rest = zero_rest != 0;
  p.list = reinterpret_cast<const int2 *>(ws + at.list);
  p.inner = reinterpret_cast<float *>(ws + at.inner);
  p.most = reinterpret_cast<float *>(ws + at.most);
  return hip_status(launch_attention_backward(p, static_cast<hipStream_t>(hip_stream)), "abs_causal_attention_backward");
} catch (...) { return exception_status(); }

}  // extern "C"
