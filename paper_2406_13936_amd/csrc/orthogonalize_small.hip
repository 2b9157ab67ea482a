// Orthogonalisation of matrices that a work-group's LDS holds (the formulas and number formats of orthogonalize.hip, operands as
// hi + lo): one launch, one work-group of eight wavefronts to a matrix, which takes the momentum's step, the norm, all
// Newton-Schulz steps and the update.  Such matrices are latency: launch by launch every product is a handful of k-tiles
// behind a launch's 3 to 8 us.  5 steps, replayed from a graph, this kernel against the launches of orthogonalize.hip: 4 of 64 x 96
// 25 us against 61, 4 of 16 x 1000 37 / 93, 4 of 128 x 128 70 / 75, 512 of 64 x 512 169 / 384, 512 of
// 128 x 128 151 / 281, 2048 of 16 x 16 46 / 293; so every matrix that fits is taken here, or by the slices below.  What bounds it is the chain of LDS reads,
// dependent MFMAs and barriers of one work-group (3.3 us a step of 64 x 96, 1.3 of 16 x 16, 10 of 128 x 128); the number of
// tiles is a template's, so that their loops are straight code (4 of 64 x 96 with run-time loops: 35 us).
//
// LDS: X [mp][np + 8] and A [mp][mp + 8] as two fp16 values each, m = the smaller side, sides rounded up to 32 with zeros
// (rows 16 bytes off a multiple of 64 bytes: the 16 rows of a fragment read meet different banks).
//   A = X X^T      both operands are rows of X
//   B = b A + c A A   both are rows of A; B takes A's place once every wavefront has its tiles
//   X' = a X + B X    rows of B, and columns of X by transposing reads.  A block of 16 columns of X' needs these columns of X
//                  only, so one wavefront reads and replaces them without waiting for the others
#include <algorithm>
#include <cstring>
#include "device_utils.h"
#include "mfma_tile.h"
#include "ops.h"
#include "orth_parts.h"
#include "typed_mem.h"

namespace absk {
namespace {

constexpr int SM_WAVES = 8, SM_THREADS = SM_WAVES * 64;
constexpr int SM_MAX_M = 128;
constexpr size_t SM_LDS = 160 * 1024 - 1024;               // (what a work-group has less the kernel's own few arrays)
constexpr size_t SM_RED = SM_WAVES * 256 * sizeof(float);          // partial tiles of reductions shared by wavefronts

int up(int v, int a) { return (v + a - 1) / a * a; }
// tiles of 16 that hold the smaller side, as there are kernels for
int small_tiles(int rows, int cols) {
  const int t = (std::min(rows, cols) + 15) / 16;
  return t <= 2 ? t : t <= 4 ? 4 : t <= 6 ? 6 : 8;
}
size_t small_lds(int rows, int cols) {
  const size_t m = std::max(32, 16 * small_tiles(rows, cols)), n = up(std::max(rows, cols), 32);
  return (m * (n + 8) + m * (m + 8)) * 4 + SM_RED;
}

struct OrthSmallP {
  OrthIn in; OrthOut out;
  int rows, cols, wide, steps;
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

// hi + lo of both operands, the small products first
__device__ __forceinline__ f32x4 mfma_split(f16x8 ph, f16x8 pl, f16x8 qh, f16x8 ql, f32x4 c) { return mfma16(ph, qh, mfma16(pl, qh, mfma16(ph, ql, c))); }

// C = alpha C_old + beta R R^T for the NT x NT tiles of 16 x 16, R = rh + rl with K values (a multiple of 32) to a row.  SELF: C is R, and
// its old value counts.  PART: C is fp32 in memory, 16 NT values to a row.  A wavefront has tiles of one row of tiles (the fragments of that row are read once), or, where there are
// fewer tiles than wavefronts, a share of a tile's reduction; shares are added in order.
enum { GRAM_NEW = 0, GRAM_SELF = 1, GRAM_PART = 2 };
template <int NT, int KIND>
__device__ __forceinline__ void gram(const uint16_t *rh, const uint16_t *rl, int ldr, int K, uint16_t *ch, uint16_t *cl, int ldc,
                                     float alpha, float beta, float *red, float *part = nullptr) {
  constexpr bool SELF = KIND == GRAM_SELF;
  constexpr int SHARES = NT == 1 ? 8 : NT == 2 ? 2 : 1;    // of a reduction
  constexpr int PER = NT == 4 ? 2 : 1;                     // wavefronts to a row of tiles
  constexpr int TILES = SHARES > 1 ? 1 : NT / PER;         // of a wavefront, PER apart
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g16 = lane >> 4;
  const int tile = wave / SHARES, s = wave % SHARES;
  const int ti = SHARES > 1 ? tile / NT : wave / PER, t0 = SHARES > 1 ? tile % NT : wave % PER;
  const bool on = ti < NT;
  f32x4 acc[TILES];
#pragma unroll
  for (int j = 0; j < TILES; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (on) {
    const int kc = SHARES > 1 ? (K / 32 + SHARES - 1) / SHARES * 32 : K, k0 = SHARES > 1 ? s * kc : 0, k1 = min(K, k0 + kc);
    const int own = (ti * 16 + i16) * ldr + g16 * 8, other = (t0 * 16 + i16) * ldr + g16 * 8;
    for (int k = k0; k < k1; k += 32) {
      const f16x8 qh = rows8(rh + own + k), ql = rows8(rl + own + k);
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const int o = other + j * PER * 16 * ldr + k;
        acc[j] = mfma_split(rows8(rh + o), rows8(rl + o), qh, ql, acc[j]);
      }
    }
  }
  if (SHARES > 1) {
    *reinterpret_cast<f32x4 *>(red + (wave * 64 + lane) * 4) = acc[0];
    __syncthreads();
    if (s == 0) {
#pragma unroll
      for (int h = 1; h < SHARES; ++h) acc[0] += *reinterpret_cast<const f32x4 *>(red + ((wave + h) * 64 + lane) * 4);
    }
  }
  const bool writes = on && s == 0;
  const int at = (ti * 16 + i16) * ldc + t0 * 16 + g16 * 4;          // (a lane has four consecutive columns of one row)
#pragma unroll
  for (int j = 0; j < TILES; ++j) {
    acc[j] *= beta;
    if (SELF && writes) {
      float c[4];
      get4(ch + at + j * PER * 16, cl + at + j * PER * 16, c);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(alpha, c[e], acc[j][e]);
    }
  }
  if (SELF) __syncthreads();                               // every read of R is done
  if (writes) {
#pragma unroll
    for (int j = 0; j < TILES; ++j) {
      if (KIND == GRAM_PART) {
        *reinterpret_cast<f32x4 *>(part + (ti * 16 + i16) * (NT * 16) + (t0 + j * PER) * 16 + g16 * 4) = acc[j];
        continue;
      }
      const float v[4] = {acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
      put4(ch + at + j * PER * 16, cl + at + j * PER * 16, v);
    }
  }
  __syncthreads();
}

// X' = ax X + bx B X, or the result of the last step, for n columns that are columns n0 .. of the matrix.  SHARE wavefronts to a block of
// 16 columns, each with some of its tiles.
template <int NT, int SHARE>
__device__ __forceinline__ void apply(const OrthSmallP &p, int z, uint16_t *xh, uint16_t *xl, int ldx, const uint16_t *bh, const uint16_t *bl,
                                      int ldb, int m, int n, int n0, int mp, float ax, float bx, bool last) {
  constexpr int TILES = (NT + SHARE - 1) / SHARE;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g16 = lane >> 4, nb = (n + 15) >> 4, t0 = wave % SHARE * TILES;
  for (int cb = wave / SHARE; SHARE > 1 || cb < nb; cb += SM_WAVES / SHARE) {
    f32x4 acc[TILES];
#pragma unroll
    for (int j = 0; j < TILES; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const bool on = (SHARE == 1 || cb < nb) && t0 < NT;
    const int xt = (t0 * 16 + i16) * ldx + cb * 16 + g16 * 4;        // X[i][c ..], i = 16 (t0 + j) + i16
    if (on) {
      const int xo = (g16 * 8 + (i16 >> 2)) * ldx + cb * 16 + 4 * (i16 & 3), bo = (t0 * 16 + i16) * ldb + g16 * 8;
      for (int k = 0; k < mp; k += 32) {
        const f16x8 ph = cols8(xh + xo + k * ldx, ldx), pl = cols8(xl + xo + k * ldx, ldx);
#pragma unroll
        for (int j = 0; j < TILES; ++j) {
          const int o = bo + j * 16 * ldb + k;
          acc[j] = mfma_split(ph, pl, rows8(bh + o), rows8(bl + o), acc[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        float x[4];
        get4(xh + xt + j * 16 * ldx, xl + xt + j * 16 * ldx, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(ax, x[e], bx * acc[j][e]);
      }
    }
    if (SHARE > 1) __syncthreads();                        // others read these columns too
    if (on && !last) {
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const float v[4] = {acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
        put4(xh + xt + j * 16 * ldx, xl + xt + j * 16 * ldx, v);
      }
    } else if (on) {
      const float lr = p.out.scal ? p.out.scal[0] : p.out.lr, decay = 1.0f - lr * p.out.wd, gain = lr * p.out.scale;
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const int i = (t0 + j) * 16 + i16, c = cb * 16 + g16 * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (i >= m || c + e >= n) continue;
          const int r = p.wide ? i : n0 + c + e, q = p.wide ? n0 + c + e : i;
          const long long at = z * p.out.so + (long long)r * p.out.ldo + q;
          const float v = p.out.update ? fmaf(decay, load_as_f32(p.out.o, p.out.type, at), -gain * acc[j][e]) : acc[j][e];
          store_from_f32(p.out.o, p.out.type, at, v);
          if (p.out.shadow) p.out.shadow[z * p.out.sshadow + (long long)r * p.out.ldo + q] = f2bf(v);
        }
      }
    }
    if (SHARE > 1) break;                                  // (there are no more columns than one round takes)
  }
  __syncthreads();
}

// NT: tiles of 16 that hold the smaller side (LDS has at least 32 rows, the k of one MFMA)
template <int NT>
__global__ void __launch_bounds__(SM_THREADS) orth_small_kernel(const OrthSmallP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  __shared__ double sm[SM_WAVES];
  __shared__ double norm2;
  __shared__ OrthScale sc[ORTH_MAX_STEPS];
  constexpr int mp = NT == 1 ? 32 : NT * 16, lda = mp + 8, HELD = 4;
  const int z = blockIdx.x, tid = threadIdx.x;
  const int m = min(p.rows, p.cols), n = max(p.rows, p.cols);
  const int np = (n + 31) & ~31, ldx = np + 8;
  uint16_t *xh = reinterpret_cast<uint16_t *>(smem_raw), *xl = xh + mp * ldx, *ah = xl + mp * ldx, *al = ah + mp * lda;
  float *red = reinterpret_cast<float *>(al + mp * lda);

  // the norm, and the momentum's step; up to HELD chunks of eight values to a thread stay in registers for what follows
  const int cc = (p.cols + 7) >> 3, chunks = p.rows * cc;
  float held[HELD][8];
  double sum = 0.0;
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    const int i = tid + h * SM_THREADS;
#pragma unroll
    for (int e = 0; e < 8; ++e) held[h][e] = 0.0f;
    if (i < chunks) load_u8<true>(p.in, p.rows, p.cols, z, i / cc, i % cc * 8, held[h]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)held[h][e], (double)held[h][e], sum);
  }
  for (int i = tid + HELD * SM_THREADS; i < chunks; i += SM_THREADS) {
    float u[8];
    load_u8<true>(p.in, p.rows, p.cols, z, i / cc, i % cc * 8, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)u[e], (double)u[e], sum);
  }
  // zeros where the sides are rounded up, and the steps' factors where they are at hand
  for (int i = tid; i < (mp * ldx + mp * lda) / 4; i += SM_THREADS) reinterpret_cast<uint4 *>(xh)[i] = make_uint4(0, 0, 0, 0);
  if (tid == 0)
    for (int k = 0; k < p.steps; ++k) sc[k] = p.sc[k];
  sum = block_sum<SM_WAVES>(sum, sm);
  if (tid == 0) norm2 = sum;
  __syncthreads();
  const double scale = (double)p.first / (sqrt(norm2) + (double)p.eps);
  auto put = [&](int i, const float (&u)[8]) {
    const int r = i / cc, c = (i - r * cc) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (c + e >= p.cols) break;
      const float v = (float)((double)u[e] * scale);
      const uint16_t h = f16_bits(v);
      const int o = p.wide ? r * ldx + c + e : (c + e) * ldx + r;
      xh[o] = h;
      xl[o] = f16_bits(v - f16_val(h));
    }
  };
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (tid + h * SM_THREADS < chunks) put(tid + h * SM_THREADS, held[h]);
  for (int i = tid + HELD * SM_THREADS; i < chunks; i += SM_THREADS) {       // (a thread meets the values of v that it has written)
    float u[8];
    load_u8<false>(p.in, p.rows, p.cols, z, i / cc, i % cc * 8, u);
    put(i, u);
  }
  __syncthreads();

  for (int k = 0; k < p.steps; ++k) {
    const OrthScale s = sc[k];
    const bool last = k + 1 == p.steps;
    gram<NT, GRAM_NEW>(xh, xl, ldx, np, ah, al, lda, 0.0f, s.gram, red);
    gram<NT, GRAM_SELF>(ah, al, lda, mp, ah, al, lda, s.poly_a, s.poly_aa, red);
    // two wavefronts to a block of 16 columns where there are no more than four of these
    constexpr bool TWO = NT == 2 || NT == 4;
    if (TWO && n <= 64) apply<NT, TWO ? 2 : 1>(p, z, xh, xl, ldx, ah, al, lda, m, n, 0, mp, s.apply_x, s.apply_bx, last);
    else apply<NT, 1>(p, z, xh, xl, ldx, ah, al, lda, m, n, 0, mp, s.apply_x, s.apply_bx, last);
  }
}

// The same from matrix z0 on
OrthSmallP from_matrix(const OrthSmallP &p, int z0) {
  OrthSmallP q = p;
  q.in.g = static_cast<const unsigned char *>(p.in.g) + z0 * p.in.sg * type_bytes(p.in.type);
  if (p.in.v) q.in.v = p.in.v + z0 * p.in.sv;
  q.out.o = static_cast<unsigned char *>(p.out.o) + z0 * p.out.so * type_bytes(p.out.type);
  if (p.out.shadow) q.out.shadow = p.out.shadow + z0 * p.out.sshadow;
  return q;
}

template <int NT> hipError_t launch_nt(const OrthSmallP &p, int batch, size_t lds, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  hipError_t err = allow_lds(reinterpret_cast<const void *>(orth_small_kernel<NT>), SM_LDS, done);
  constexpr int MOST = 1 << 22;                            // matrices of a launch: a grid counts its threads in 32 bits
  for (int z0 = 0; z0 < batch && err == hipSuccess; z0 += std::min(MOST, batch - z0)) {
    hipLaunchKernelGGL(orth_small_kernel<NT>, dim3(std::min(MOST, batch - z0)), dim3(SM_THREADS), lds, s, from_matrix(p, z0));
    err = hipGetLastError();
  }
  return err;
}

// ---- few rows, many columns ----------------------------------------------------------------------------------------
//
// A smaller side of up to 128 beside one that LDS does not hold: slices of SLICE columns (of the longer side), a work-group to each.  A
// step needs A of all slices and leaves every slice to itself otherwise, so it is two launches: one adds the slices' shares of A,
// in order; the other forms B (every work-group for itself: its A is in LDS, and 64 MFMAs of a wavefront are shorter than a launch),
// replaces its columns of X and leaves their share of the next A.  5 steps, replayed from a graph, against the tiles of
// orthogonalize.hip: 10 of 36 x 2972 80 us against 207, 1 of 25 x 2365 46 / 143, 3 of 2858 x 50 68 / 169, 2 of 16 x 100000 144 / 3627.
// Bound by its launches (4 to 5 us each); 512 of 32 x 2048 (453 / 860) by reading and writing X once a step.
constexpr int SLICE = 128, SLICE_LD = SLICE + 8;

struct OrthSliceP {
  OrthSmallP q;
  int slices, nparts, k;                                   // k: the step; -1: X_0 and its share of A
  const double *norm;                                      // [batch][nparts]
  uint16_t *x, *a;                                         // [batch][slices][2][mp][SLICE_LD], [batch][2][mp][mp + 8], as in LDS
  float *part;                                             // [batch][slices][16 NT][16 NT]
};

template <int NT>
__global__ void __launch_bounds__(SM_THREADS) orth_slice_kernel(const OrthSliceP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  __shared__ double sm[SM_WAVES];
  __shared__ double norm2;
  constexpr int mp = NT == 1 ? 32 : NT * 16, lda = mp + 8, ldx = SLICE_LD, XB = mp * ldx / 4, AB = mp * lda / 4;      // 16-byte pieces of both parts
  const int z = blockIdx.x / p.slices, j = blockIdx.x - z * p.slices, tid = threadIdx.x;
  const int m = min(p.q.rows, p.q.cols), n0 = j * SLICE, n = min(SLICE, max(p.q.rows, p.q.cols) - n0);
  uint16_t *xh = reinterpret_cast<uint16_t *>(smem_raw), *xl = xh + mp * ldx, *ah = xl + mp * ldx, *al = ah + mp * lda;
  float *red = reinterpret_cast<float *>(al + mp * lda);
  uint4 *xs = reinterpret_cast<uint4 *>(xh), *xg = reinterpret_cast<uint4 *>(p.x) + (long long)blockIdx.x * XB;
  const bool last = p.k + 1 == p.q.steps;
  if (p.k < 0) {
    for (int i = tid; i < XB; i += SM_THREADS) xs[i] = make_uint4(0, 0, 0, 0);
    const double sum = block_sum<SM_WAVES>(tid < p.nparts ? p.norm[(long long)z * p.nparts + tid] : 0.0, sm);
    if (tid == 0) norm2 = sum;
    __syncthreads();
    const double scale = (double)p.q.first / (sqrt(norm2) + (double)p.q.eps);
    const int r0 = p.q.wide ? 0 : n0, c0 = p.q.wide ? n0 : 0;
    const int cc = p.q.wide ? SLICE / 8 : (p.q.cols + 7) >> 3, chunks = (p.q.wide ? p.q.rows : n) * cc;
    for (int i = tid; i < chunks; i += SM_THREADS) {
      const int r = i / cc, c = (i - r * cc) * 8;
      float u[8];
      load_u8<false>(p.q.in, p.q.rows, p.q.cols, z, r0 + r, c0 + c, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c0 + c + e >= p.q.cols) break;
        const float v = (float)((double)u[e] * scale);
        const uint16_t h = f16_bits(v);
        const int o = p.q.wide ? r * ldx + c + e : (c + e) * ldx + r;
        xh[o] = h;
        xl[o] = f16_bits(v - f16_val(h));
      }
    }
  } else {
    uint4 *as = reinterpret_cast<uint4 *>(ah);
    const uint4 *ag = reinterpret_cast<const uint4 *>(p.a) + (long long)z * AB;
#pragma unroll 4
    for (int i = tid; i < AB; i += SM_THREADS) as[i] = ag[i];
#pragma unroll 4
    for (int i = tid; i < XB; i += SM_THREADS) xs[i] = xg[i];
    __syncthreads();
    const OrthScale s = p.q.sc[p.k];
    gram<NT, GRAM_SELF>(ah, al, lda, mp, ah, al, lda, s.poly_a, s.poly_aa, red);
    apply<NT, 1>(p.q, z, xh, xl, ldx, ah, al, lda, m, n, n0, mp, s.apply_x, s.apply_bx, last);
    if (last) return;
  }
  __syncthreads();
  for (int i = tid; i < XB; i += SM_THREADS) xg[i] = xs[i];
  gram<NT, GRAM_PART>(xh, xl, ldx, SLICE, nullptr, nullptr, 0, 0.0f, 1.0f, red, p.part + (long long)blockIdx.x * (NT * NT * 256));
}

// A = gram times the slices' shares, added in order (by four wavefronts a quarter each), as hi + lo where LDS will have it
template <int NT>
__global__ void __launch_bounds__(256) orth_slice_sum_kernel(const OrthSliceP p) {
  constexpr int mp = NT == 1 ? 32 : NT * 16, lda = mp + 8, side = NT * 16;
  __shared__ f32x4 sm[4][64];
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, z = blockIdx.x / (mp * mp / 256);
  const int at = (blockIdx.x - z * (mp * mp / 256)) * 256 + lane * 4, r = at / mp, c = at % mp;
  const bool in = r < side && c < side;
  const int per = (p.slices + 3) / 4, j1 = min(p.slices, (q + 1) * per);
  f32x4 v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (in) {
    const float *part = p.part + (long long)z * p.slices * side * side + r * side + c;
#pragma unroll 8
    for (int j = q * per; j < j1; ++j) v += *reinterpret_cast<const f32x4 *>(part + (long long)j * side * side);
  }
  sm[q][lane] = v;
  __syncthreads();
  if (q) return;
  v = ((sm[0][lane] + sm[1][lane]) + sm[2][lane]) + sm[3][lane];
  v *= p.q.sc[p.k].gram;
  const float f[4] = {v[0], v[1], v[2], v[3]};
  uint16_t *a = p.a + (long long)z * 2 * mp * lda + r * lda + c;
  put4(a, a + mp * lda, f);
}

template <int NT> hipError_t launch_slices(const OrthSliceP &p, int batch, hipStream_t s) {
  constexpr int mp = NT == 1 ? 32 : NT * 16;
  constexpr size_t lds = (size_t)mp * (SLICE_LD + mp + 8) * 4 + SM_RED;
  static_assert(lds <= SM_LDS, "LDS budget");
  static std::atomic<uint64_t> done{0};
  hipError_t err = allow_lds(reinterpret_cast<const void *>(orth_slice_kernel<NT>), lds, done);
  const int most = std::max(1, (1 << 22) / std::max(p.slices, mp * mp / 256));      // matrices of a launch: a grid counts its threads in 32 bits
  for (int z0 = 0; z0 < batch && err == hipSuccess; z0 += std::min(most, batch - z0)) {
    const int nz = std::min(most, batch - z0);
    OrthSliceP b = p;
    b.q = from_matrix(p.q, z0);
    b.norm += (long long)z0 * p.nparts;
    b.x += (long long)z0 * p.slices * 2 * mp * SLICE_LD; b.a += (long long)z0 * 2 * mp * (mp + 8); b.part += (long long)z0 * p.slices * NT * NT * 256;
    for (b.k = -1; b.k < p.q.steps; ++b.k) {
      if (b.k >= 0) hipLaunchKernelGGL(orth_slice_sum_kernel<NT>, dim3(nz * (mp * mp / 256)), dim3(256), 0, s, b);
      hipLaunchKernelGGL(orth_slice_kernel<NT>, dim3(nz * p.slices), dim3(SM_THREADS), lds, s, b);
    }
    err = hipGetLastError();
  }
  return err;
}

}  // namespace

// ... and which slices that are few do not take in less time.  us, one launch against slices: 4 of 32 x 768 53 / 42, of 64 x 256 44 / 54, of
// 64 x 512 75 / 55, of 96 x 224 73 / 78, of 96 x 280 91 / 78; 30 of 32 x 1000 68 / 47, 80 of 64 x 384 63 / 79.
bool orth_small_fits(int batch, int rows, int cols) {
  const int m = std::min(rows, cols), n = std::max(rows, cols);
  if (m > SM_MAX_M || n > 8192 || small_lds(rows, cols) > SM_LDS) return false;
  return m <= 16 || m > 96 || m * n <= 22000 || (long long)batch * ((n + SLICE - 1) / SLICE) > (m <= 32 ? 256 : 128);
}

// Always up to 64; from 65 on (whose LDS leaves a CU one work-group) while all slices are resident at once, and beyond 96, where B takes
// a work-group longest, only of longer rows.  us, this against tiles: 64 of 64 x 640 98 / 125, 1024 of 64 x 1024 1222 / 1499; 64 of 96 x 512
// 121 / 129, of 96 x 1024 202 / 172; 1 of 128 x 512 101 / 88, 1 of 128 x 1024 103 / 108, 16 of 128 x 2048 152 / 190, 32 270 / 229.
bool orth_slices_fit(int batch, int rows, int cols) {
  const int m = std::min(rows, cols), n = std::max(rows, cols);
  return m <= 64 || (m <= SM_MAX_M && (long long)batch * ((n + SLICE - 1) / SLICE) <= 256 && (m <= 96 || n >= 1024));
}

size_t orth_slices_bytes(const OrthPlan &pl, size_t &o_x, size_t &o_a, size_t &o_part) {
  const size_t nt = small_tiles(pl.rows, pl.cols), mp = std::max<size_t>(32, 16 * nt), slices = (std::max(pl.rows, pl.cols) + SLICE - 1) / SLICE;
  auto up256 = [](size_t b) { return (b + 255) / 256 * 256; };
  o_x = 0;
  o_a = up256(pl.batch * slices * 2 * mp * SLICE_LD * 2);
  o_part = o_a + up256(pl.batch * 2 * mp * (mp + 8) * 2);
  return o_part + up256(pl.batch * slices * nt * nt * 256 * 4);
}

static OrthSmallP small_args(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps) {
  OrthSmallP p;
  std::memset(&p, 0, sizeof(p));
  p.in = in; p.out = out; p.rows = pl.rows; p.cols = pl.cols; p.wide = pl.wide; p.steps = pl.steps; p.eps = eps;
  p.first = (float)(1u << pl.ex[0]);
  for (int k = 0; k < pl.steps; ++k) p.sc[k] = pl.scale(k);
  return p;
}

hipError_t launch_orth_small(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, hipStream_t s) {
  const OrthSmallP p = small_args(pl, in, out, eps);
  const size_t lds = small_lds(pl.rows, pl.cols);
  switch (small_tiles(pl.rows, pl.cols)) {
    case 1: return launch_nt<1>(p, pl.batch, lds, s);
    case 2: return launch_nt<2>(p, pl.batch, lds, s);
    case 4: return launch_nt<4>(p, pl.batch, lds, s);
    case 6: return launch_nt<6>(p, pl.batch, lds, s);
    default: return launch_nt<8>(p, pl.batch, lds, s);
  }
}

hipError_t launch_orth_slices(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, const double *norm, unsigned char *ws, hipStream_t s) {
  size_t o_x, o_a, o_part;
  (void)orth_slices_bytes(pl, o_x, o_a, o_part);
  OrthSliceP p;
  std::memset(&p, 0, sizeof(p));
  p.q = small_args(pl, in, out, eps);
  p.slices = (std::max(pl.rows, pl.cols) + SLICE - 1) / SLICE; p.nparts = pl.nparts; p.norm = norm;
  p.x = reinterpret_cast<uint16_t *>(ws + o_x); p.a = reinterpret_cast<uint16_t *>(ws + o_a); p.part = reinterpret_cast<float *>(ws + o_part);
  switch (small_tiles(pl.rows, pl.cols)) {
    case 1: return launch_slices<1>(p, pl.batch, s);
    case 2: return launch_slices<2>(p, pl.batch, s);
    case 4: return launch_slices<4>(p, pl.batch, s);
    case 6: return launch_slices<6>(p, pl.batch, s);
    default: return launch_slices<8>(p, pl.batch, s);
  }
}

}  // namespace absk
