// C ABI of the operators beside the replicas' step (declared in include/abs.h): argument checks and launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <numeric>

#include "../../include/abs.h"
#include "api_status.h"
#include "ops.h"

using namespace absk;

namespace {

bool known_type(int t) { return t >= ABS_TYPE_F32 && t <= ABS_TYPE_F16; }
bool aligned_to(const void *p, int bytes) { return !(reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)); }

// A [n][rows][cols] block in memory, `bytes` to a value.  Looked at as a whole (level 0), as what repeats in its longer step (1), or as rows (2)
struct Block {
  const void *p;
  int64_t n, stride, rows, ld, cols;
  int bytes;
  uintptr_t at() const { return reinterpret_cast<uintptr_t>(p); }
  int64_t over(int64_t count, int64_t step) const { return count > 1 ? step : 0; }
  int64_t longer() const { return std::max(over(n, stride), over(rows, ld)) * bytes; }
  // bytes of a piece, from its first value to behind its last, and what the distances between pieces are multiples of (0: one piece)
  uintptr_t length(int level) const {
    const int64_t matrices = over(n, stride) * (n - 1), lines = over(rows, ld) * (rows - 1);
    const bool by_matrix = over(n, stride) >= over(rows, ld);
    return (uintptr_t)(((level == 0 ? matrices + lines : level == 1 ? (by_matrix ? lines : matrices) : 0) + cols) * bytes);
  }
  uintptr_t pitch(int level) const {
    return (uintptr_t)(level == 0 ? 0 : level == 1 ? longer() : std::gcd(over(n, stride), over(rows, ld)) * bytes);
  }
};
Block piece(const void *p, int64_t values, int bytes) { return {p, 1, 0, 1, 0, values, bytes}; }
// Apart: one ends before the other begins, or all pieces of both begin at two places, with room for each, of spaces of one pitch
bool overlap(const Block &a, const Block &b) {
  const uintptr_t p = a.at(), q = b.at();
  if (p + a.length(0) <= q || q + b.length(0) <= p) return false;
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 3; ++j) {
      const uintptr_t space = std::gcd(a.pitch(i), b.pitch(j));
      if (!space) continue;
      const uintptr_t d = q >= p ? (q - p) % space : (space - (p - q) % space) % space;
      if (d >= a.length(i) && d + b.length(j) <= space) return false;
    }
  return true;
}
// Any of the outputs over an input or another output (absent ones: null)
template <size_t NO, size_t NI> bool outputs_overlap(const Block (&out)[NO], const Block (&in)[NI]) {
  for (size_t i = 0; i < NO; ++i) {
    if (!out[i].p) continue;
    for (const Block &x : in)
      if (x.p && overlap(out[i], x)) return true;
    for (size_t j = 0; j < i; ++j)
      if (out[j].p && overlap(out[i], out[j])) return true;
  }
  return false;
}
// rows that do not overlap, matrix after matrix or interleaved; offsets that 64 bits hold
bool strides_ok(int64_t n, int64_t stride, int64_t rows, int64_t ld, int64_t cols) {
  const int64_t big = (int64_t)1 << 46;
  if (ld < cols || ld >= big / rows || stride < 0 || stride >= big / n) return false;
  return n == 1 || stride >= (rows - 1) * ld + cols || (stride >= cols && ld >= (n - 1) * stride + cols);
}
abs_status hip_status(hipError_t e, const char *what) {
  return e == hipSuccess ? ABS_OK : set_error(ABS_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

abs_status check_matrices(int batch, int rows, int cols, int prec) {
  if (batch < 1 || rows < 1 || cols < 1) return set_error(ABS_EINVAL, "batch, rows and cols must be at least 1");
  if (prec != ABS_PREC_F32 && prec != ABS_PREC_BF16) return set_error(ABS_EINVAL, "unknown precision");
  if (((int64_t)rows + 31) * ((int64_t)cols + 31) >= (1LL << 29)) return set_error(ABS_EUNSUPPORTED, "a matrix must hold fewer than 2^29 values");
  return ABS_OK;
}
abs_status check_orth(int batch, int rows, int cols, int steps, const float *coef, float eps, int prec, const void *workspace,
                      size_t workspace_bytes, OrthPlan &pl) {
  abs_status st = check_matrices(batch, rows, cols, prec);
  if (st != ABS_OK) return st;
  if (steps < 1 || steps > ORTH_MAX_STEPS) return set_error(ABS_EINVAL, "steps must be in [1, 32]");
  if (!(eps > 0.0f) || !std::isfinite(eps)) return set_error(ABS_EINVAL, "eps must be positive and finite");
  if (const char *why = orth_plan(batch, rows, cols, prec == ABS_PREC_F32, steps, coef, pl)) return set_error(ABS_EINVAL, why);
  if (!workspace || !aligned_to(workspace, 256)) return set_error(ABS_EINVAL, "workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < pl.total) return set_error(ABS_ENOMEM, "workspace too small (see abs_orthogonalize_workspace_bytes)");
  return ABS_OK;
}

abs_status check_shape(const abs_layer_norm_shape *s, bool backward) {
  if (!s) return set_error(ABS_EINVAL, "shape is NULL");
  if (s->M < 1 || s->b < 1 || s->T < 1 || s->D < 1) return set_error(ABS_EINVAL, "M, b, T and D must be at least 1");
  if (!known_type(s->type)) return set_error(ABS_EINVAL, "unknown type");
  if (s->param_type != s->type && s->param_type != ABS_TYPE_F32) return set_error(ABS_EINVAL, "param_type must be ABS_TYPE_F32 or type");
  const int64_t rows = (int64_t)s->b * s->T;
  // (a grid counts its threads in 32 bits, and 512 of them add the partial gradients of 64 gains or biases)
  if (s->M > 1 << 20 || (int64_t)s->M * s->D > 1 << 27 || rows > 0x7fffffff / s->M)
    return set_error(ABS_EUNSUPPORTED, "more than 2^20 replicas, 2^27 gains or 2^31 - 1 rows");
  if (!strides_ok(s->M, s->stride_x, rows, s->ldx, s->D) || !strides_ok(s->M, s->stride_y, rows, s->ldy, s->D) ||
      (backward && !strides_ok(s->M, s->stride_dx, rows, s->lddx, s->D)))
    return set_error(ABS_EINVAL, "strides: ld >= D, and rows must not overlap");
  return ABS_OK;
}
LayerNormP layer_norm_args(const abs_layer_norm_shape *s) {
  LayerNormP p;
  std::memset(&p, 0, sizeof(p));
  p.M = s->M; p.b = s->b; p.T = s->T; p.D = s->D; p.type = s->type; p.ptype = s->param_type;
  p.ldx = s->ldx; p.sx = s->stride_x; p.ldy = s->ldy; p.sy = s->stride_y; p.lddx = s->lddx; p.sdx = s->stride_dx;
  return p;
}

}  // namespace

extern "C" {

abs_status abs_orthogonalize_workspace_bytes(int batch, int rows, int cols, int prec, size_t *bytes) try {
  if (!bytes) return set_error(ABS_EINVAL, "bytes is NULL");
  abs_status st = check_matrices(batch, rows, cols, prec);
  if (st != ABS_OK) return st;
  OrthPlan pl;
  (void)orth_plan(batch, rows, cols, prec == ABS_PREC_F32, 1, nullptr, pl);
  *bytes = pl.total;
  return ABS_OK;
} catch (...) { return exception_status(); }

abs_status abs_orthogonalize(const void *g_dev, int g_type, int64_t ldg, int64_t stride_g, void *o_dev, int o_type, int64_t ldo,
                             int64_t stride_o, int batch, int rows, int cols, int steps, const float *coef, float eps, int prec,
                             void *workspace, size_t workspace_bytes, void *hip_stream) try {
  if (!g_dev || !o_dev) return set_error(ABS_EINVAL, "NULL argument");
  if (!known_type(g_type) || !known_type(o_type)) return set_error(ABS_EINVAL, "unknown type");
  OrthPlan pl;
  abs_status st = check_orth(batch, rows, cols, steps, coef, eps, prec, workspace, workspace_bytes, pl);
  if (st != ABS_OK) return st;
  if (!strides_ok(batch, stride_g, rows, ldg, cols) || !strides_ok(batch, stride_o, rows, ldo, cols) || ldg > 0x7fffffff || ldo > 0x7fffffff)
    return set_error(ABS_EINVAL, "strides: ld >= cols, and rows must not overlap");
  if (!aligned_to(g_dev, type_bytes(g_type)) || !aligned_to(o_dev, type_bytes(o_type))) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const bool same = g_dev == o_dev && g_type == o_type && ldg == ldo && stride_g == stride_o;
  const Block g = {g_dev, batch, stride_g, rows, ldg, cols, type_bytes(g_type)}, o = {o_dev, batch, stride_o, rows, ldo, cols, type_bytes(o_type)};
  const Block ws = piece(workspace, (int64_t)pl.total, 1);
  if ((!same && overlap(g, o)) || overlap(ws, g) || overlap(ws, o))
    return set_error(ABS_EINVAL, "o_dev must be g_dev or not overlap it, and the workspace neither");
  const OrthIn in = {g_dev, g_type, stride_g, (int)ldg, nullptr, 0, 0.0f, 0};
  OrthOut out;
  std::memset(&out, 0, sizeof(out));
  out.o = o_dev; out.type = o_type; out.so = stride_o; out.ldo = (int)ldo;
  return hip_status(launch_orthogonalize(pl, in, out, eps, workspace, static_cast<hipStream_t>(hip_stream)), "abs_orthogonalize");
} catch (...) { return exception_status(); }

abs_status abs_muon_step(void *x_dev, int x_type, const void *g_dev, int g_type, float *v_dev, int batch, int rows, int cols, float lr,
                         float momentum, int nesterov, float weight_decay, float scale, int steps, const float *coef, float eps, int prec,
                         void *workspace, size_t workspace_bytes, void *hip_stream) try {
  if (!x_dev || !g_dev || !v_dev) return set_error(ABS_EINVAL, "NULL argument");
  if (!known_type(x_type) || !known_type(g_type)) return set_error(ABS_EINVAL, "unknown type");
  if (!std::isfinite(lr) || !std::isfinite(momentum) || !std::isfinite(weight_decay) || !std::isfinite(scale))
    return set_error(ABS_EINVAL, "lr, momentum, weight_decay and scale must be finite");
  OrthPlan pl;
  abs_status st = check_orth(batch, rows, cols, steps, coef, eps, prec, workspace, workspace_bytes, pl);
  if (st != ABS_OK) return st;
  if (!aligned_to(x_dev, type_bytes(x_type)) || !aligned_to(g_dev, type_bytes(g_type)) || !aligned_to(v_dev, 4))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const int64_t n = (int64_t)rows * cols;
  const Block used[4] = {piece(x_dev, batch * n, type_bytes(x_type)), piece(g_dev, batch * n, type_bytes(g_type)), piece(v_dev, batch * n, 4),
                         piece(workspace, (int64_t)pl.total, 1)};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(used[i], used[j])) return set_error(ABS_EINVAL, "x, g, v and the workspace must not overlap");
  const OrthIn in = {g_dev, g_type, n, cols, v_dev, n, momentum, nesterov != 0};
  OrthOut out;
  std::memset(&out, 0, sizeof(out));
  out.o = x_dev; out.type = x_type; out.so = n; out.ldo = cols;
  out.update = 1; out.lr = lr; out.scale = scale; out.wd = weight_decay;
  return hip_status(launch_orthogonalize(pl, in, out, eps, workspace, static_cast<hipStream_t>(hip_stream)), "abs_muon_step");
} catch (...) { return exception_status(); }

abs_status abs_layer_norm(const abs_layer_norm_shape *shape, const void *x_dev, const void *gamma_dev, const void *beta_dev, float eps,
                          void *y_dev, float *mean_dev, float *rstd_dev, void *hip_stream) try {
  abs_status st = check_shape(shape, false);
  if (st != ABS_OK) return st;
  if (!x_dev || !gamma_dev || !y_dev) return set_error(ABS_EINVAL, "NULL argument");
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(ABS_EINVAL, "eps must be finite and not negative");
  const int e = type_bytes(shape->type), pe = type_bytes(shape->param_type);
  if (!aligned_to(x_dev, e) || !aligned_to(y_dev, e) || !aligned_to(gamma_dev, pe) || !aligned_to(beta_dev, pe) || !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const int64_t rows = (int64_t)shape->b * shape->T;
  const bool same = x_dev == y_dev && shape->ldx == shape->ldy && shape->stride_x == shape->stride_y;
  const Block x = {x_dev, shape->M, shape->stride_x, rows, shape->ldx, shape->D, e}, y = {y_dev, shape->M, shape->stride_y, rows, shape->ldy, shape->D, e};
  if (!same && overlap(x, y)) return set_error(ABS_EINVAL, "y_dev must be x_dev or not overlap it");
  const int64_t all = shape->M * rows, gains = (int64_t)shape->M * shape->D;
  const Block out[] = {y, piece(mean_dev, all, 4), piece(rstd_dev, all, 4)}, params[] = {piece(gamma_dev, gains, pe), piece(beta_dev, gains, pe)};
  if (outputs_overlap(out, params) || outputs_overlap({out[1], out[2]}, {x}))
    return set_error(ABS_EINVAL, "y_dev, mean_dev and rstd_dev must not overlap an input or each other");
  LayerNormP p = layer_norm_args(shape);
  p.x = x_dev; p.gamma = gamma_dev; p.beta = beta_dev; p.eps = eps; p.y = y_dev; p.mean = mean_dev; p.rstd = rstd_dev;
  return hip_status(launch_layer_norm(p, static_cast<hipStream_t>(hip_stream)), "abs_layer_norm");
} catch (...) { return exception_status(); }

abs_status abs_layer_norm_backward_workspace_bytes(const abs_layer_norm_shape *shape, int want_n, int want_q, size_t *bytes) try {
  if (!bytes) return set_error(ABS_EINVAL, "bytes is NULL");
  abs_status st = check_shape(shape, true);
  if (st != ABS_OK) return st;
  *bytes = layer_norm_backward_bytes(layer_norm_args(shape), want_n != 0, want_q != 0);
  return ABS_OK;
} catch (...) { return exception_status(); }

abs_status abs_layer_norm_backward(const abs_layer_norm_shape *shape, const void *dy_dev, const void *x_dev, const void *gamma_dev,
                                   const float *mean_dev, const float *rstd_dev, void *dx_dev, float *dgamma_dev, float *dbeta_dev,
                                   float *n_dev, float *q_dev, void *workspace, size_t workspace_bytes, void *hip_stream) try {
  abs_status st = check_shape(shape, true);
  if (st != ABS_OK) return st;
  if (!dy_dev || !x_dev || !gamma_dev || !mean_dev || !rstd_dev || !dx_dev || !dgamma_dev) return set_error(ABS_EINVAL, "NULL argument");
  if (!workspace || !aligned_to(workspace, 256)) return set_error(ABS_EINVAL, "workspace must be a 256-byte aligned device pointer");
  LayerNormP p = layer_norm_args(shape);
  const size_t need = layer_norm_backward_bytes(p, n_dev != nullptr, q_dev != nullptr);
  if (workspace_bytes < need) return set_error(ABS_ENOMEM, "workspace too small (see abs_layer_norm_backward_workspace_bytes)");
  const int e = type_bytes(shape->type);
  if (!aligned_to(dy_dev, e) || !aligned_to(x_dev, e) || !aligned_to(dx_dev, e) || !aligned_to(gamma_dev, type_bytes(shape->param_type)))
    return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  for (const void *f : {(const void *)mean_dev, (const void *)rstd_dev, (const void *)dgamma_dev, (const void *)dbeta_dev, (const void *)n_dev, (const void *)q_dev})
    if (!aligned_to(f, 4)) return set_error(ABS_EINVAL, "pointers must be aligned to their type");
  const int64_t rows = (int64_t)shape->b * shape->T;
  const int64_t all = shape->M * rows, gains = (int64_t)shape->M * shape->D, samples = (int64_t)shape->M * shape->b;
  const Block in[] = {{x_dev, shape->M, shape->stride_x, rows, shape->ldx, shape->D, e}, {dy_dev, shape->M, shape->stride_y, rows, shape->ldy, shape->D, e},
                      piece(gamma_dev, gains, type_bytes(shape->param_type)), piece(mean_dev, all, 4), piece(rstd_dev, all, 4)};
  const Block out[] = {{dx_dev, shape->M, shape->stride_dx, rows, shape->lddx, shape->D, e}, piece(dgamma_dev, gains, 4), piece(dbeta_dev, gains, 4),
                       piece(n_dev, samples, 4), piece(q_dev, samples, 4), piece(workspace, (int64_t)need, 1)};
  if (outputs_overlap(out, in)) return set_error(ABS_EINVAL, "outputs and the workspace must not overlap an input or each other");
  p.x = x_dev; p.gamma = gamma_dev; p.mean = const_cast<float *>(mean_dev); p.rstd = const_cast<float *>(rstd_dev);
  p.dy = dy_dev; p.dx = dx_dev; p.dgamma = dgamma_dev; p.dbeta = dbeta_dev; p.n = n_dev; p.q = q_dev;
  return hip_status(launch_layer_norm_backward(p, workspace, static_cast<hipStream_t>(hip_stream)), "abs_layer_norm_backward");
} catch (...) { return exception_status(); }

}  // extern "C"
