// Internal declarations of the operators that stand beside the replicas' step: the orthogonalised update (orthogonalize.hip)
// and layer norm (layer_norm.hip).  Host launchers only; kernels stay private to their file.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include <atomic>
#include "abs_internal.h"

namespace absk {

enum { TYPE_F32 = 0, TYPE_BF16 = 1, TYPE_F16 = 2 };
// Lets a kernel take more than 64 KB of LDS on the current device (`done`: the kernel's own, a bit per device)
inline hipError_t allow_lds(const void *kernel, size_t bytes, std::atomic<uint64_t> &done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}
inline int type_bytes(int t) { return t == TYPE_F32 ? 4 : 2; }

// ---- orthogonalisation ---------------------------------------------------------------------------------------------

constexpr int ORTH_MAX_STEPS = 32;
constexpr int ORTH_PARTS = 256;          // most partial sums of a matrix's norm

// Factors of one step between the powers of two that the operands are stored with: A = gram X X^T, B = poly_a A + poly_aa A A,
// X' = apply_x X + apply_bx B X
struct OrthScale { float gram, poly_a, poly_aa, apply_x, apply_bx; };

struct OrthPlan {
  int batch, rows, cols, steps, split;   // split: operands as sums of two fp16 values (fp32-class products)
  int wide;                              // rows <= cols: the products A = X X^T, else A = X^T X
  int rp, cp, mp;                        // rows, columns and the smaller side rounded up to 8 (32 with split)
  int nparts;                            // partial sums of a matrix's norm
  float a[ORTH_MAX_STEPS], b[ORTH_MAX_STEPS], c[ORTH_MAX_STEPS];
  int ex[ORTH_MAX_STEPS + 1], ea[ORTH_MAX_STEPS], eb[ORTH_MAX_STEPS];   // powers of two that X, A and B are stored with
  size_t o_part, o_x[2], o_xl, o_a, o_b, o_diag, total;          // pieces of the workspace
  OrthScale scale(int k) const;
};

// What is orthogonalised: G, or with a momentum buffer (fp32) v <- momentum v + G and u = nesterov ? G + momentum v : v.
struct OrthIn {
  const void *g; int type; long long sg; int ldg;
  float *v; long long sv; float momentum; int nesterov;      // v: rows of cols values
};
// Where the result goes: O, or with `update` the step  x <- (1 - lr wd) x - lr scale O  on x (and its bf16 copy).
struct OrthOut {
  void *o; int type; long long so; int ldo;
  int update; float lr, scale, wd;
  const float *scal;                     // optional (device): lr is read from scal[0], for launches that are replayed
  bf16_t *shadow; long long sshadow;     // rows of ldo values
};

// nullptr, or why these coefficients (3 per step; null: the quintic's) cannot be taken
const char *orth_plan(int batch, int rows, int cols, int split, int steps, const float *coef, OrthPlan &pl);
hipError_t launch_orthogonalize(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, void *workspace, hipStream_t s);

// the rule for a product's tiles (tests ask it too, to reach every kind)
int orth_product_shape(int Md, int Nd, int K, int batch, int sym);

// orthogonalize_small.hip: a work-group's LDS holds the matrix
bool orth_small_fits(int batch, int rows, int cols);
hipError_t launch_orth_small(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, hipStream_t s);
// or not, but the smaller side is short: the norm's partial sums are there already
bool orth_slices_fit(int batch, int rows, int cols);
size_t orth_slices_bytes(const OrthPlan &pl, size_t &o_x, size_t &o_a, size_t &o_part);
hipError_t launch_orth_slices(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, const double *norm, unsigned char *ws, hipStream_t s);

// ---- layer norm ----------------------------------------------------------------------------------------------------

// M replicas with gains and biases of their own [M x D]; each has b samples of T rows of D values.
struct LayerNormP {
  int M, b, T, D, type, ptype;
  long long ldx, sx, ldy, sy, lddx, sdx;   // x; y or dy; dx: values from row to row and from replica to replica
  const void *x, *gamma, *beta;            // beta may be null
  float eps;
  void *y; float *mean, *rstd;             // forward: outputs (mean and rstd may be null); backward: inputs
  const void *dy;
  void *dx; float *dgamma, *dbeta;         // dbeta, n, q may be null
  float *n, *q;
};
size_t layer_norm_backward_bytes(const LayerNormP &p, bool want_n, bool want_q);
hipError_t launch_layer_norm(const LayerNormP &p, hipStream_t s);
hipError_t launch_layer_norm_backward(const LayerNormP &p, void *workspace, hipStream_t s);

// ---- root-mean-square norm -------------------------------------------------------------------------------------------

constexpr int RMS_MAX_D = 8192;          // longest row that a block's registers hold
constexpr int RMS_BLOCKS = 512;          // of the backward pass, as layer norm's
// lanes and vectors to a row: 16 x 1, 64 x 1, 64 x 2, 256 x 1, 256 x 2, 512 x 2
inline int rms_shape(int D) { return D <= 128 ? 0 : D <= 512 ? 1 : D <= 1024 ? 2 : D <= 2048 ? 3 : D <= 4096 ? 4 : 5; }

// M replicas with gains of their own [M x D]; each has b samples of T rows of D values.  Strides: values from row to row and from replica
// to replica.
struct RmsNormP {
  int M, b, T, D, type, ptype;
  long long ldx, sx, ldr, sr, ldh, sh, ldy, sy;
  const void *x, *res, *w;                 // forward: x (ldx), residual (ldr, may be null); backward: h (ldx), dh (ldr, may be null)
  float eps;
  void *h, *y; float *scale;               // forward: h (ldh; with a residual), y (ldy; e4m3 if there is a scale)
  float *rstd;                             // forward: output (may be null); backward: input
  const void *dy; void *dx;                // backward: dy (ldy), dx (ldh)
  float *dw, *n, *q;                       // n, q may be null
};
size_t rms_norm_backward_bytes(const RmsNormP &p, bool want_n, bool want_q);
hipError_t launch_rms_norm(const RmsNormP &p, hipStream_t s);
hipError_t launch_rms_norm_backward(const RmsNormP &p, void *workspace, hipStream_t s);

// ---- token embedding -------------------------------------------------------------------------------------------------

// M replicas with tables of their own [M][V][D]; each has b samples of T tokens.
struct EmbeddingP {
  int M, b, T, V, D;
  int wide;                                // tokens of 64 bits, not 32
  int type, ttype;                         // of y or dy; of the table (forward)
  long long ldy, sy;                       // y or dy: values from row to row and from replica to replica
  const void *tokens, *table; float scale;
  void *y; const void *dy;
  float *dtable, *n, *q;                   // n, q may be null
};
size_t embedding_backward_bytes(const EmbeddingP &p, bool want_n, bool want_q);
hipError_t launch_embedding(const EmbeddingP &p, hipStream_t s);
hipError_t launch_embedding_backward(const EmbeddingP &p, void *workspace, hipStream_t s);

// ---- causal attention ------------------------------------------------------------------------------------------------

constexpr int ATTENTION_ROWS = 128;      // queries or keys of a block
constexpr int ATTENTION_MAX_D = 128;

// `seqs` sequences among `rows` rows: between offsets[s] and offsets[s + 1], or without offsets of T rows each.  Strides: values from row to row
// (ld) and from head to head (h).
struct AttentionP {
  int type, Hq, Hkv, D, seqs, T;
  int wide;                                // offsets of 64 bits, not 32
  int zero_rest;                           // zeros in rows of no sequence (else they stay as they are)
  long long rows;
  const void *offsets;
  const int2 *list;                        // workspace, with more than 64 sequences: number of tiles; sequence and level of each
  long long ldq, hq, ldk, hk, ldv, hv, ldo, ho;
  const void *q, *k, *v;
  float scale;
  void *o; float *lse;                     // lse [Hq][rows]: forward an output (may be null), backward an input
  // backward
  long long lddo, hdo, lddq, hdq, lddk, hdk, lddv, hdv;
  const void *dout;
  void *dq, *dk, *dv;
  float *inner;                            // workspace [Hq][rows]: do_i . o_i
  float *most;                             // workspace (fp16) [Hq + Hkv][tiles]: largest squared lengths of do_i, and of v_j, of each tile's rows
};
// Tiles of all sequences: what they are, or with offsets the most that they can be
__host__ __device__ inline long long attention_tiles(const AttentionP &p) {
  if (!p.offsets) return p.seqs * ((p.T + (ATTENTION_ROWS - 1LL)) / ATTENTION_ROWS);
  return p.rows / ATTENTION_ROWS + p.seqs;
}
hipError_t launch_attention_tiles(const AttentionP &p, hipStream_t s);
hipError_t launch_attention(const AttentionP &p, hipStream_t s);
hipError_t launch_attention_backward(const AttentionP &p, hipStream_t s);

}  // namespace absk
