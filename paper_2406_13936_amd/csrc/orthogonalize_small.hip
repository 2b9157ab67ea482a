// Orthogonalisation of matrices that a work-group's LDS holds (the formulas and number formats of orthogonalize.hip, operands as
// hi + lo): one launch, one work-group of eight wavefronts to a matrix, which takes the momentum's step, the norm, all
// Newton-Schulz steps and the update.  Such matrices are latency: launch by launch every product is a handful of k-tiles
// behind 8 us (4 of 64 x 96: 132 us for 17 launches, here 33).
//
// LDS: X [mp][np + 8] and A [mp][mp + 8] as two fp16 values each, m = the smaller side, sides rounded up to 32 with zeros
// (rows 16 bytes off a multiple of 64 bytes: the 16 rows of a fragment read meet different banks).
//   A = X X^T      both operands are rows of X
//   B = b A + c A A   both are rows of A; B takes A's place once every wavefront has its tiles
//   X' = a X + B X    rows of B, and columns of X by transposing reads.  A block of 16 columns of X' needs these columns of X
//                  only, so one wavefront reads and replaces them without waiting for the others
#include <algorithm>
#include <cstring>
#include <mutex>
#include "device_utils.h"
#include "mfma_tile.h"
#include "ops.h"
#include "orth_parts.h"
#include "typed_mem.h"

namespace absk {
namespace {

constexpr int SM_WAVES = 8, SM_THREADS = SM_WAVES * 64;
constexpr int SM_MAX_M = 128, SM_TILES = SM_MAX_M / 16;
constexpr size_t SM_RED = SM_WAVES * 256 * sizeof(float);          // partial tiles of reductions shared by wavefronts

int up(int v, int a) { return (v + a - 1) / a * a; }
size_t small_lds(int rows, int cols) {
  const size_t m = up(std::min(rows, cols), 32), n = up(std::max(rows, cols), 32);
  return (m * (n + 8) + m * (m + 8)) * 4 + SM_RED;
}

struct OrthSmallP {
  OrthIn in; OrthOut out;
  int rows, cols, vec, wide, steps;
  float eps, first;                      // first: the power of two that X_0 is stored with
  OrthScale sc[ORTH_MAX_STEPS];
};

__device__ __forceinline__ f32x4 mfma16(f16x8 p, f16x8 q, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, c, 0, 0, 0); }
__device__ __forceinline__ f16x8 rows8(const uint16_t *q) { return *reinterpret_cast<const f16x8 *>(q); }
// eight k of a column of a row-major matrix: lanes of a group of 16 address (k = lane / 4, columns 4 (lane % 4) ..) and receive
// four k of column lane % 16
__device__ __forceinline__ f16x8 cols8(const uint16_t *q, int ld) {
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q + 4 * ld));
  return __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// four values as hi + lo at q, r
__device__ __forceinline__ void put4(uint16_t *hi, uint16_t *lo, const float (&v)[4]) {
  uint32_t h[2], l[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint16_t a = f16_bits(v[2 * e]), b = f16_bits(v[2 * e + 1]);
    h[e] = (uint32_t)a | ((uint32_t)b << 16);
    l[e] = (uint32_t)f16_bits(v[2 * e] - f16_val(a)) | ((uint32_t)f16_bits(v[2 * e + 1] - f16_val(b)) << 16);
  }
  *reinterpret_cast<uint2 *>(hi) = make_uint2(h[0], h[1]);
  *reinterpret_cast<uint2 *>(lo) = make_uint2(l[0], l[1]);
}
__device__ __forceinline__ void get4(const uint16_t *hi, const uint16_t *lo, float (&v)[4]) {
  const uint2 h = *reinterpret_cast<const uint2 *>(hi), l = *reinterpret_cast<const uint2 *>(lo);
  v[0] = f16_val(h.x & 0xffffu) + f16_val(l.x & 0xffffu); v[1] = f16_val(h.x >> 16) + f16_val(l.x >> 16);
  v[2] = f16_val(h.y & 0xffffu) + f16_val(l.y & 0xffffu); v[3] = f16_val(h.y >> 16) + f16_val(l.y >> 16);
}

// C = alpha C_old + beta R R^T for the nt x nt tiles of 16 x 16, R = rh + rl with K values (a multiple of 32) to a row.
// A wavefront has tiles of one row of tiles (the fragments of that row are read once), or, where there are fewer tiles than
// wavefronts, a share of a tile's reduction; shares are added in order.  C may be R: it is written behind a barrier.
__device__ __forceinline__ void gram(const uint16_t *rh, const uint16_t *rl, int ldr, int K, uint16_t *ch, uint16_t *cl, int ldc, int nt,
                                     float alpha, float beta, float *red) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g16 = lane >> 4;
  const int per = nt >= 4 ? SM_WAVES / nt : 1;             // wavefronts to a row of tiles
  const int shares = nt == 1 ? 8 : nt == 2 ? 2 : 1;        // of a reduction
  f32x4 acc[SM_TILES];
  int ti, t0, dt, k0 = 0, k1 = K;
  if (shares > 1) {
    const int tile = wave / shares, s = wave - tile * shares, kc = (K / 32 + shares - 1) / shares * 32;
    ti = tile / nt; t0 = tile - ti * nt; dt = SM_TILES;
    k0 = min(K, s * kc); k1 = min(K, k0 + kc);
  } else if (nt == 3) {                                    // nine tiles: row by row, one wavefront to each
    ti = wave; t0 = 0; dt = 1;
  } else {
    ti = wave / per; t0 = wave - ti * per; dt = per;
  }
  const bool on = ti < nt;
#pragma unroll
  for (int j = 0; j < SM_TILES; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (on) {
    const int own = (ti * 16 + i16) * ldr + g16 * 8;
    for (int k = k0; k < k1; k += 32) {
      const f16x8 qh = rows8(rh + own + k), ql = rows8(rl + own + k);
#pragma unroll
      for (int j = 0; j < SM_TILES; ++j) {
        const int tj = t0 + j * dt;
        if (tj >= nt) break;
        const int o = (tj * 16 + i16) * ldr + g16 * 8 + k;
        const f16x8 ph = rows8(rh + o), pl = rows8(rl + o);
        acc[j] = mfma16(ph, ql, acc[j]);
        acc[j] = mfma16(pl, qh, acc[j]);
        acc[j] = mfma16(ph, qh, acc[j]);
      }
    }
  }
  if (shares > 1) {
    *reinterpret_cast<f32x4 *>(red + (wave * 64 + lane) * 4) = acc[0];
    __syncthreads();
    if (wave % shares == 0)
      for (int s = 1; s < shares; ++s) acc[0] += *reinterpret_cast<const f32x4 *>(red + ((wave + s) * 64 + lane) * 4);
  }
  // (a lane has four consecutive columns of one row)
  const bool writes = on && (shares == 1 || wave % shares == 0);
  if (writes && alpha != 0.0f) {
#pragma unroll
    for (int j = 0; j < SM_TILES; ++j) {
      const int tj = t0 + j * dt;
      if (tj >= nt) break;
      const int o = (ti * 16 + i16) * ldc + tj * 16 + g16 * 4;
      float c[4];
      get4(ch + o, cl + o, c);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(alpha, c[e], beta * acc[j][e]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < SM_TILES; ++j) acc[j] *= beta;
  }
  __syncthreads();                                         // every read of R is done
  if (writes) {
#pragma unroll
    for (int j = 0; j < SM_TILES; ++j) {
      const int tj = t0 + j * dt;
      if (tj >= nt) break;
      const int o = (ti * 16 + i16) * ldc + tj * 16 + g16 * 4;
      const float v[4] = {acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
      put4(ch + o, cl + o, v);
    }
  }
  __syncthreads();
}

__global__ void __launch_bounds__(SM_THREADS) orth_small_kernel(const OrthSmallP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  __shared__ double sm[SM_WAVES];
  __shared__ double norm2;
  const int z = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g16 = lane >> 4;
  const int m = min(p.rows, p.cols), n = max(p.rows, p.cols);
  const int mp = (m + 31) & ~31, np = (n + 31) & ~31, ldx = np + 8, lda = mp + 8;
  uint16_t *xh = reinterpret_cast<uint16_t *>(smem_raw), *xl = xh + mp * ldx, *ah = xl + mp * ldx, *al = ah + mp * lda;
  float *red = reinterpret_cast<float *>(al + mp * lda);

  // zeros where the sides are rounded up; the norm, and the momentum's step
  for (int i = tid; i < (mp * ldx + mp * lda) / 4; i += SM_THREADS) reinterpret_cast<uint4 *>(xh)[i] = make_uint4(0, 0, 0, 0);
  const int cc = (p.cols + 7) >> 3, chunks = p.rows * cc;
  double sum = 0.0;
  for (int i = tid; i < chunks; i += SM_THREADS) {
    const int r = i / cc, c = (i - r * cc) * 8;
    float u[8];
    load_u8<true>(p.in, p.rows, p.cols, p.vec, z, r, c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)u[e], (double)u[e], sum);
  }
  sum = block_sum<SM_WAVES>(sum, sm);
  if (tid == 0) norm2 = sum;
  __syncthreads();
  const double scale = (double)p.first / (sqrt(norm2) + (double)p.eps);
  for (int i = tid; i < chunks; i += SM_THREADS) {         // (a thread meets the values of v that it has written)
    const int r = i / cc, c = (i - r * cc) * 8;
    float u[8];
    load_u8<false>(p.in, p.rows, p.cols, p.vec, z, r, c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (c + e >= p.cols) break;
      const float v = (float)((double)u[e] * scale);
      const uint16_t h = f16_bits(v);
      const int o = p.wide ? r * ldx + c + e : (c + e) * ldx + r;
      xh[o] = h;
      xl[o] = f16_bits(v - f16_val(h));
    }
  }
  __syncthreads();

  const int nt = (m + 15) >> 4, nb = (n + 15) >> 4;
  // wavefronts to a block of 16 columns, each with some of its tiles: one where there are enough blocks
  const int share = nb <= 1 ? 8 : nb <= 2 ? 4 : nb <= 4 ? 2 : 1, tiles = (nt + share - 1) / share;
  float lr = p.out.lr;
  if (p.out.scal) lr = p.out.scal[0];
  const float decay = 1.0f - lr * p.out.wd, gain = lr * p.out.scale;
  for (int k = 0; k < p.steps; ++k) {
    const OrthScale s = p.sc[k];
    gram(xh, xl, ldx, np, ah, al, lda, nt, 0.0f, s.gram, red);
    gram(ah, al, lda, mp, ah, al, lda, nt, s.poly_a, s.poly_aa, red);
    const bool last = k + 1 == p.steps;
    for (int cb0 = 0; cb0 < nb; cb0 += SM_WAVES / share) {
      const int cb = cb0 + wave / share, t0 = wave % share * tiles, t1 = min(nt, t0 + tiles);
      f32x4 acc[SM_TILES];
#pragma unroll
      for (int j = 0; j < SM_TILES; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (cb < nb) {
        const int xo = (g16 * 8 + (i16 >> 2)) * ldx + cb * 16 + 4 * (i16 & 3);
        for (int kk = 0; kk < mp; kk += 32) {
          const f16x8 ph = cols8(xh + xo + kk * ldx, ldx), pl = cols8(xl + xo + kk * ldx, ldx);
#pragma unroll
          for (int j = 0; j < SM_TILES; ++j) {
            if (t0 + j >= t1) break;
            const int o = ((t0 + j) * 16 + i16) * lda + g16 * 8 + kk;
            const f16x8 qh = rows8(ah + o), ql = rows8(al + o);
            acc[j] = mfma16(ph, ql, acc[j]);
            acc[j] = mfma16(pl, qh, acc[j]);
            acc[j] = mfma16(ph, qh, acc[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < SM_TILES; ++j) {
          if (t0 + j >= t1) break;
          const int o = ((t0 + j) * 16 + i16) * ldx + cb * 16 + g16 * 4;
          float x[4];
          get4(xh + o, xl + o, x);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(s.apply_x, x[e], s.apply_bx * acc[j][e]);
        }
      }
      if (share > 1) __syncthreads();                      // others read these columns too (then there is one round)
      if (cb >= nb) continue;
#pragma unroll
      for (int j = 0; j < SM_TILES; ++j) {
        if (t0 + j >= t1) break;
        const int i = (t0 + j) * 16 + i16, c = cb * 16 + g16 * 4;          // X'[i][c ..]
        float v[4] = {acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
        if (!last) { put4(xh + i * ldx + c, xl + i * ldx + c, v); continue; }
        if (i >= m) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (c + e >= n) continue;
          const int r = p.wide ? i : c + e, q = p.wide ? c + e : i;
          const long long at = z * p.out.so + (long long)r * p.out.ldo + q;
          const float x = p.out.update ? fmaf(decay, load_as_f32(p.out.o, p.out.type, at), -gain * v[e]) : v[e];
          store_from_f32(p.out.o, p.out.type, at, x);
          if (p.out.shadow) p.out.shadow[z * p.out.sshadow + (long long)r * p.out.ldo + q] = f2bf(x);
        }
      }
    }
    __syncthreads();
  }
}

}  // namespace

bool orth_small_fits(int rows, int cols) { return std::min(rows, cols) <= SM_MAX_M && std::max(rows, cols) <= 8192 && small_lds(rows, cols) <= 160 * 1024 - 256; }

hipError_t launch_orth_small(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, hipStream_t s) {
  OrthSmallP p;
  std::memset(&p, 0, sizeof(p));
  p.in = in; p.out = out; p.rows = pl.rows; p.cols = pl.cols; p.wide = pl.wide; p.steps = pl.steps; p.eps = eps;
  p.vec = rows_of_vectors(in.g, in.type, in.sg, in.ldg, pl.cols) && (!in.v || rows_of_vectors(in.v, TYPE_F32, in.sv, pl.cols, pl.cols));
  p.first = (float)(1u << pl.ex[0]);
  for (int k = 0; k < pl.steps; ++k) p.sc[k] = pl.scale(k);
  static std::once_flag once;
  static hipError_t err = hipSuccess;
  std::call_once(once, [&] { err = hipFuncSetAttribute(reinterpret_cast<const void *>(orth_small_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024 - 256); });
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(orth_small_kernel, dim3(pl.batch), dim3(SM_THREADS), small_lds(pl.rows, pl.cols), s, p);
  return hipGetLastError();
}

}  // namespace absk
