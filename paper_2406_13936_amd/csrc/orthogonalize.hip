// Orthogonalisation of matrices by Newton-Schulz products, and the update that is taken with the result.
//
//   X_0 = G / (||G||_F + eps),    A = X X^T,   B = b A + c A^2,   X <- a X + B X      (rows <= cols)
//                                 A = X^T X,                      X <- a X + X B      (rows >  cols)
//
// X keeps its singular vectors and its singular values s go through p(s) = a s + b s^3 + c s^5 in every step; after five
// steps of the usual quintic they lie around 1.  The smaller side m is the side of A and B.
//
// Numbers.  X is held as the sum of two fp16 values (22 bits and a sign, as exact as fp32 in these sums); the products take
// the first of them (16-bit mode) or, with `split`, all of (hi + lo)(hi + lo) but lo lo, which is what fp32 products give.
// fp16 and not bf16, because every entry of X, A and B is bounded by a spectral norm that the host knows beforehand
// (s <= 1 before the first step and max |p| on that interval after it): each is stored times a power of two that puts
// this bound just under fp16's largest value, so three more bits of mantissa come free.  B's diagonal, where its largest
// entries lie (near -2.7 once A is near 1), stays in fp32 and is applied where X' is finished.  Relative error of the result
// for 64 x 64 to 1536 x 1536 matrices of full rank, rank 64 and of a spectrum falling over five decades: 0.5 to 1.6e-3 (with the
// diagonal rounded too 0.5 to 2.1e-3, bf16 operands 5e-3 to 1.5e-2), with `split` the same as fp32 products (1.2e-6 to 1.2e-5).  Why X cannot be rounded to 16 bits: a step
// multiplies a singular value near 0 by a = 3.4, five of them by 485, and with it the rounding noise that lies along
// those directions (rank 64 in 256 x 512: 1.8e-2 with fp16, 0.15 with bf16).  B X makes no such noise from a rounded X,
// since B's range is that of X.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include "device_utils.h"
#include "mfma_tile.h"
#include "ops.h"
#include "orth_parts.h"
#include "typed_mem.h"

namespace absk {

namespace {

// ---- norm and first X ----------------------------------------------------------------------------------------------

struct OrthPrepP {
  OrthIn in;
  int rows, cols, rp, cp, nparts, vec, ex;   // vec: all rows start on 16 bytes, cols is a multiple of 8
  double *part; uint16_t *xh, *xl;
  float eps;
};

// Sum of squares of a matrix in fp64 (entries of any size fp32 has), one partial per block; with a momentum buffer this is
// where it advances.  One pass over G (and v): bound by memory.
__global__ void __launch_bounds__(256) orth_norm_kernel(const OrthPrepP p) {
  __shared__ double sm[4];
  const int z = blockIdx.y, cc = (p.cols + 7) >> 3, n = p.rows * cc;
  double sum = 0.0;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const int r = i / cc, c = (i - r * cc) * 8;
    float u[8];
    load_u8<true>(p.in, p.rows, p.cols, p.vec, z, r, c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)u[e], (double)u[e], sum);
  }
  const double t = block_sum<4>(sum, sm);
  if (threadIdx.x == 0) p.part[(long long)z * p.nparts + blockIdx.x] = t;
}

// X_0 2^ex as two fp16 values, zeros in the rows and columns that round the sides up to 8
__global__ void __launch_bounds__(256) orth_prep_kernel(const OrthPrepP p) {
  __shared__ double sm[4];
  __shared__ double scale;
  const int z = blockIdx.y;
  const double t = block_sum<4>((int)threadIdx.x < p.nparts ? p.part[(long long)z * p.nparts + threadIdx.x] : 0.0, sm);
  if (threadIdx.x == 0) scale = ldexp(1.0 / (sqrt(t) + (double)p.eps), p.ex);
  __syncthreads();
  const double sc = scale;
  const long long x0 = (long long)z * p.rp * p.cp;
  const int cc = p.cp >> 3, n = p.rp * cc;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const int r = i / cc, c = (i - r * cc) * 8;
    float u[8];
    load_u8<false>(p.in, p.rows, p.cols, p.vec, z, r, c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = (float)((double)u[e] * sc);
    uint4 h, l;
    split8(u, h, l);
    const long long at = x0 + (long long)r * p.cp + c;
    *reinterpret_cast<uint4 *>(p.xh + at) = h;
    *reinterpret_cast<uint4 *>(p.xl + at) = l;
  }
}

// ---- the products --------------------------------------------------------------------------------------------------

// C[z][m][n] = alpha E[z][m][n] + beta sum_k A[z][m][k] B[z][n][k]   as one or two fp16 values, or the result of the last step
struct OrthGemmP {
  const uint16_t *A, *Al, *B, *Bl;       // (Al, Bl: with split)
  long long sA, sB; int lda, ldb, Md, Nd, Kd, batch;
  const uint16_t *E, *El; long long sE; int lde;
  uint16_t *C, *Cl; long long sC; int ldc;
  float alpha, beta;
  int sym;                               // C is symmetric: tiles below the diagonal are written from those above it
  float *diag; int diag_of;              // [z][mp] fp32 diagonal: DIAG_OUT: C's, which is stored as zeros there; DIAG_ROWS, DIAG_COLS:
                                         //   beta diag[m] (or [n]) times E's first part is added
  OrthOut out; int rows, cols, vec;      // the last step (C null)
};

// Tiles BM x BN x BK with WM x WN wavefronts, NS stages of direct global -> LDS loads; operands k-contiguous or row-contiguous as
// in gemm_bf16.hip.  PP: its pipelined loop of 256 x 256 tiles (eight 16 KB units of LDS, each refilled seven phases before it is
// read, four wavefronts half a phase behind the others; the reasons stand there).  SPLIT: the reduction runs three times over
// k, with (hi, lo), (lo, hi) and (hi, hi) as operands.
enum { DIAG_NONE = 0, DIAG_OUT, DIAG_ROWS, DIAG_COLS };
enum { KIND_SYM = 0, KIND_APPLY = 1, KIND_LAST = 2 };   // A and B; X'; X' of the last step
constexpr int BAND = 8;                  // columns of 256-wide tiles that stand side by side (gemm_bf16.hip)

template <int BM, int BN, int BK, int WM, int WN, int NS, bool PP, bool AT, bool BT, bool SPLIT, int KIND>
__global__ void __launch_bounds__(WM * WN * 64) orth_gemm_kernel(const OrthGemmP p, const int tilesM, const int tilesN, const int nblk, const int chunk) {
  constexpr int NW = WM * WN;
  constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 32, NI = TN / 32;
  constexpr int STAGE = (BM + BN) * BK, NPART = BK / 16;
  static_assert(!PP || (BM == 256 && BN == 256 && BK == 64 && WM == 2 && WN == 4), "the pipelined loop");
  typedef Operand<BM, BK, AT, NW> OpA;
  typedef Operand<BN, BK, BT, NW> OpB;
  constexpr int NL = OpA::NI + OpB::NI;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  bf16_t *smem = reinterpret_cast<bf16_t *>(smem_raw);

  const int lb = (blockIdx.x & 7) * chunk + (blockIdx.x >> 3);      // an XCD works on a contiguous range of tiles
  if ((int)(blockIdx.x >> 3) >= chunk || lb >= nblk) return;
  int z, tm, tn;
  if (p.sym) {                                    // tiles (tm, tn >= tm) row by row
    const int T = tilesN, per = T * (T + 1) / 2;
    z = lb / per;
    const int t = lb - z * per;
    tm = (int)((2 * T + 1 - sqrtf((float)((2 * T + 1) * (2 * T + 1) - 8 * t))) * 0.5f);
    tm = max(0, min(tm, T - 1));
    while (tm > 0 && t < tm * T - tm * (tm - 1) / 2) --tm;          // (first tile of row tm: sum of T - r over r < tm)
    while (t >= (tm + 1) * T - (tm + 1) * tm / 2) ++tm;
    tn = tm + t - (tm * T - tm * (tm - 1) / 2);
  } else {
    const int per = tilesM * tilesN;
    z = lb / per;
    const int t = lb - z * per;
    if (BM == 256 && tilesN > BAND) {             // bands of columns, row by row inside a band
      const int nb = (tilesN + BAND - 1) / BAND, bw = (tilesN + nb - 1) / nb, b = t / (bw * tilesM);
      const int w = min(bw, tilesN - b * bw), r = t - b * bw * tilesM;
      tm = r / w; tn = b * bw + r - tm * w;
    } else {
      tm = t / tilesN; tn = t - tm * tilesN;
    }
  }
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  const int abytes = (int)((long long)(AT ? p.Kd : p.Md) * p.lda * 2), bbytes = (int)((long long)(BT ? p.Kd : p.Nd) * p.ldb * 2);
  auto rsrc = [](const uint16_t *q, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(q), 0, bytes, 0x00020000); };
  const __amdgpu_buffer_rsrc_t rah = rsrc(p.A + z * p.sA, abytes), rbh = rsrc(p.B + z * p.sB, bbytes);
  const __amdgpu_buffer_rsrc_t ral = rsrc(SPLIT ? p.Al + z * p.sA : p.A, abytes), rbl = rsrc(SPLIT ? p.Bl + z * p.sB : p.B, bbytes);

  f32x16 acc[PP ? 1 : MI][PP ? 1 : NI];
  f32x4 acc16[PP ? TM / 16 : 1][PP ? TN / 16 : 1];
  if constexpr (PP) {
#pragma unroll
    for (int i = 0; i < TM / 16; ++i)
#pragma unroll
      for (int j = 0; j < TN / 16; ++j) acc16[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  } else {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  }

  const int KT1 = (p.Kd + BK - 1) / BK, KT = SPLIT ? 3 * KT1 : KT1;
  if constexpr (PP) {
    typedef Operand<128, 64, AT, NW, 32> UA;                 // A unit h: rows 128 h .. 128 h + 127 of the tile, 64 k
    typedef Operand<BT ? 256 : 128, BT ? 32 : 64, BT, NW, 32> UB;   // B unit c: k 32 c .. (BT), or columns 64 j + 32 c ..
    constexpr int UNIT = 8192;                               // elements of a unit (16 KB)
    UA ua[2];
    UB ub[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ua[h].init(wave, lane, m0 + h * 128, p.Md, p.lda);
      if constexpr (BT) ub[h].init(wave, lane, n0, p.Nd, p.ldb);
      else ub[h].template init<true>(wave, lane, n0 + h * 32, p.Nd, p.ldb);
    }
    // (k-tiles beyond the last bring zeros)
    auto load_a = [&](int kt, int slot, int h) {
      const int seg = SPLIT ? (kt >= KT1) + (kt >= 2 * KT1) : 2, k = SPLIT ? kt - seg * KT1 : kt;
      ua[h].load_all(SPLIT && seg == 1 ? ral : rah, smem + (slot * 2 + h) * UNIT, wave, k * 64, 0, p.Kd, p.lda);
    };
    auto load_b = [&](int kt, int slot, int c) {
      const int seg = SPLIT ? (kt >= KT1) + (kt >= 2 * KT1) : 2, k = SPLIT ? kt - seg * KT1 : kt;
      ub[c].load_all(SPLIT && seg == 0 ? rbl : rbh, smem + (4 + slot * 2 + c) * UNIT, wave, k * 64 + (BT ? c * 32 : 0), 0, p.Kd, p.ldb);
    };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const int i16 = lane & 15, g16 = lane >> 4;
    const int kq = g16 * 8 + (i16 >> 2);                     // transpose reads: k within the 32-wide step
    uint32_t aaddr[AT ? 4 : 2], baddr[BT ? 4 : 2];           // (transpose reads: by row tile; else by k-step)
    if constexpr (AT) {
#pragma unroll
      for (int ii = 0; ii < 4; ++ii) {
        const int rr = wm * 64 + ii * 16 + 4 * (i16 & 3);
        aaddr[ii] = lds0 + 2u * (uint32_t)(kq * 128 + ((rr >> 3) ^ tr_swizzle<32>(kq)) * 8 + (rr & 7));
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        aaddr[kk] = lds0 + (uint32_t)((wm * 64 + i16) * 128 + (((kk * 4 + g16) ^ (i16 >> 1)) << 4));
    }
    if constexpr (BT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int rr = wn * 64 + j * 16 + 4 * (i16 & 3);
        baddr[j] = lds0 + 65536u + 2u * (uint32_t)(kq * 256 + ((rr >> 3) ^ tr_swizzle<32>(kq)) * 8 + (rr & 7));
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        baddr[kk] = lds0 + 65536u + (uint32_t)((wn * 32 + i16) * 128 + (((kk * 4 + g16) ^ (i16 >> 1)) << 4));
    }
    bf16x8 fa[4][2], fb[2][4];                               // fa[row tile][k-step]; fb[unit][BT: column tile, else 2 column tile + k-step]
    auto read_a = [&](auto SLOT, auto H) {
      constexpr int U = (decltype(SLOT)::value * 2 + decltype(H)::value) * UNIT * 2;
      static_for<8>([&](auto I) {
        constexpr int kk = decltype(I)::value >> 2, ii = decltype(I)::value & 3;
        if constexpr (AT) fa[ii][kk] = lds_read_cols<U + kk * 8192, 1024>(aaddr[ii]);
        else fa[ii][kk] = lds_read_rows<U + ii * 2048>(aaddr[kk]);
      });
    };
    auto read_b = [&](auto SLOT, auto C) {
      constexpr int c = decltype(C)::value, U = (decltype(SLOT)::value * 2 + c) * UNIT * 2;
      static_for<4>([&](auto I) {
        constexpr int q = decltype(I)::value;
        if constexpr (BT) fb[c][q] = lds_read_cols<U, 2048>(baddr[q]);
        else fb[c][q] = lds_read_rows<U + (q >> 1) * 2048>(baddr[q & 1]);
      });
    };
    auto close_reads = [&]() {                               // this wave's fragment reads are done
      __builtin_amdgcn_s_waitcnt(0xC07F);
#pragma unroll
      for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(fa[q][0]), "+v"(fa[q][1]), "+v"(fb[0][q]), "+v"(fb[1][q]));
    };
    auto mfma = [](bf16x8 x, bf16x8 y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0); };
    auto phase = [&](auto SLOT, auto F, int kt) {
      constexpr int f = decltype(F)::value, h = f >> 1, c = f & 1;
      if constexpr (f == 0) { read_a(SLOT, Const<0>{}); load_b(kt + 2, SLOT.value, 0); }
      if constexpr (f == 1) { read_b(SLOT, Const<1>{}); load_a(kt + 2, SLOT.value, 0); }
      if constexpr (f == 2) { read_a(SLOT, Const<1>{}); load_b(kt + 2, SLOT.value, 1); }
      if constexpr (f == 3) { read_b(Const<1 - decltype(SLOT)::value>{}, Const<0>{}); load_a(kt + 2, SLOT.value, 1); }
      wait_vmcnt<12>();                                      // the unit read next phase has landed; six more stay in flight
      close_reads();
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      static_for<16>([&](auto I) {                           // (operands swapped: a lane owns one row of C)
        constexpr int q = decltype(I)::value;
        if constexpr (BT) {
          constexpr int ii = q >> 2, j = q & 3;
          acc16[4 * h + ii][j] = mfma(fb[c][j], fa[ii][c], acc16[4 * h + ii][j]);
        } else {
          constexpr int kk = q >> 3, ii = (q >> 1) & 3, j = q & 1;
          acc16[4 * h + ii][2 * c + j] = mfma(fb[c][2 * j + kk], fa[ii][kk], acc16[4 * h + ii][2 * c + j]);
        }
      });
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
    };
    auto ktile = [&](auto SLOT, int kt) { static_for<4>([&](auto F) { phase(SLOT, F, kt); }); };
#pragma unroll
    for (int s = 0; s < 2; ++s) { load_b(s, s, 0); load_a(s, s, 0); load_b(s, s, 1); load_a(s, s, 1); }
    wait_vmcnt<12>();
    __builtin_amdgcn_s_barrier();
    read_b(Const<0>{}, Const<0>{});
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    if (wm == 1) __builtin_amdgcn_s_barrier();               // these four waves run half a phase behind
    for (int kt = 0; kt < KT; kt += 2) {
      ktile(Const<0>{}, kt);
      if (kt + 1 < KT) ktile(Const<1>{}, kt + 1);
    }
    if (wm == 0) __builtin_amdgcn_s_barrier();
    wait_vmcnt<0>();                                         // (zeros beyond K still on their way to LDS)
  } else {
  OpA oa;
  OpB ob;
  oa.init(wave, lane, m0, p.Md, p.lda);
  ob.init(wave, lane, n0, p.Nd, p.ldb);
  auto issue = [&](int kt, int buf, int part) {
    bf16_t *sa = smem + buf * STAGE, *sb = sa + BM * BK;
    const int seg = SPLIT ? (kt >= KT1) + (kt >= 2 * KT1) : 2;
    const int k = SPLIT ? kt - seg * KT1 : kt;
    const bool full = (k + 1) * BK <= p.Kd;
#pragma unroll
    for (int l = 0; l < NL; ++l) {
      if (l % NPART != part) continue;
      if (l < OpA::NI) oa.load(l, SPLIT && seg == 1 ? ral : rah, sa, wave, k, p.Kd, p.lda, full);
      else ob.load(l - OpA::NI, SPLIT && seg == 0 ? rbl : rbh, sb, wave, k, p.Kd, p.ldb, full);
    }
  };
  Frag<BM, BK, AT> fa[MI];
  Frag<BN, BK, BT> fb[NI];
#pragma unroll
  for (int i = 0; i < MI; ++i) fa[i].init(wm * TM + i * 32, lane);
#pragma unroll
  for (int j = 0; j < NI; ++j) fb[j].init(wn * TN + j * 32, lane);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < KT) {
#pragma unroll
      for (int q = 0; q < NPART; ++q) issue(s, s, q);
    }
  for (int kt = 0; kt < KT; ++kt) {
    if (kt + NS - 1 <= KT) wait_vmcnt<(NS - 2) * NL>(); else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();                 // all waves' loads of kt visible; everyone is done with kt-1
    const bool more = kt + NS - 1 < KT;
    const bf16_t *S = smem + (kt % NS) * STAGE;
    bf16x8 af[2][MI], bfr[2][NI];
    auto read = [&](int to, int kk) {             // (transpose reads first: the compiler does not count them)
      if (BT && !AT) {
#pragma unroll
        for (int j = 0; j < NI; ++j) bfr[to][j] = fb[j].read(S + BM * BK, kk);
      }
#pragma unroll
      for (int i = 0; i < MI; ++i) af[to][i] = fa[i].read(S, kk);
      if (!(BT && !AT)) {
#pragma unroll
        for (int j = 0; j < NI; ++j) bfr[to][j] = fb[j].read(S + BM * BK, kk);
      }
    };
    read(0, 0);
#pragma unroll
    for (int kk = 0; kk < NPART; ++kk) {
      const int cur = kk & 1, nxt = cur ^ 1;
      if (kk + 1 < NPART) read(nxt, kk + 1);
      if (more) issue(kt + NS - 1, (kt + NS - 1) % NS, kk);
      if (AT || BT) {
        constexpr int RD = (AT ? 2 : 1) * MI + (BT ? 2 : 1) * NI;
        if (kk + 1 < NPART) wait_frags<RD>(af[cur], bfr[cur]); else wait_frags<0>(af[cur], bfr[cur]);
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)              // operands swapped: a lane owns one row m of C and groups of four columns
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, bfr[cur][j]), __builtin_bit_cast(f16x8, af[cur][i]), acc[i][j], 0, 0, 0);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  }
  __syncthreads();                                // the stages are dead

  // ---- epilogue: slices of 32 rows x TN columns of a wavefront, one after the other, through its own fp32 piece of LDS, so that
  // global accesses are whole 16-byte vectors; the mirror image of a symmetric tile is read from there by columns.  The loads of
  // E for the next slice are in flight while a slice is finished (one work-group to a CU: nobody else would cover them).
  constexpr int SLD = TN + 4, CPR = TN / 8, SIT = 32 * CPR / 64;
  float *stg = reinterpret_cast<float *>(smem_raw) + wave * (32 * SLD);
  auto slice_row = [&](int i) -> int { return PP ? (i >> 1) * 128 + wm * 64 + (i & 1) * 32 : wm * TM + i * 32; };
  uint4 eh[2][SIT], el[2][SIT];
  const bool two = KIND != KIND_SYM || SPLIT;     // E is hi + lo
  auto load_e = [&](int i, uint4 (&h)[SIT], uint4 (&l)[SIT]) {
#pragma unroll
    for (int it = 0; it < SIT; ++it) {
      const int q = it * 64 + lane, r = q / CPR, cc = (q % CPR) * 8;
      const int m = m0 + slice_row(i) + r, n = n0 + wn * TN + cc;
      h[it] = l[it] = make_uint4(0, 0, 0, 0);
      if (m < p.Md && n < p.Nd) {                 // (Nd is a multiple of 8)
        const long long at = z * p.sE + (long long)m * p.lde + n;
        h[it] = *reinterpret_cast<const uint4 *>(p.E + at);
        if (two) l[it] = *reinterpret_cast<const uint4 *>(p.El + at);
      }
    }
  };
  const bool has_e = KIND != KIND_SYM || p.E;
  const bool mirror = KIND == KIND_SYM && tm != tn;
  float decay = 1.0f, gain = -1.0f;
  if (KIND == KIND_LAST && p.out.update) {
    const float lr = p.out.scal ? p.out.scal[0] : p.out.lr;
    decay = 1.0f - lr * p.out.wd;
    gain = lr * p.out.scale;
  }
  if (has_e) load_e(0, eh[0], el[0]);
  static_for<MI>([&](auto SLICE) {
    constexpr int i = decltype(SLICE)::value;
    if constexpr (PP) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < TN / 16; ++c)
          *reinterpret_cast<f32x4 *>(stg + (h * 16 + (lane & 15)) * SLD + c * 16 + (lane >> 4) * 4) = acc16[2 * i + h][c];
    } else {
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<float4 *>(stg + (lane & 31) * SLD + j * 32 + c * 8 + (lane >> 5) * 4) =
              make_float4(acc[i][j][4 * c], acc[i][j][4 * c + 1], acc[i][j][4 * c + 2], acc[i][j][4 * c + 3]);
    }
    if (has_e && i + 1 < MI) load_e(i + 1, eh[(i + 1) & 1], el[(i + 1) & 1]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < SIT; ++it) {
      const int q = it * 64 + lane, r = q / CPR, cc = (q % CPR) * 8;
      const int m = m0 + slice_row(i) + r, n = n0 + wn * TN + cc;
      if (m >= p.Md || n >= p.Nd) continue;
      float v[8];
      {
        const float4 x = *reinterpret_cast<const float4 *>(stg + r * SLD + cc), y = *reinterpret_cast<const float4 *>(stg + r * SLD + cc + 4);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
      }
      if (has_e) {
        float h[8];
        unpack8(eh[i & 1][it], TYPE_F16, h);
        if (!SPLIT && KIND != KIND_SYM) {         // B's diagonal
          if (p.diag_of == DIAG_ROWS) {
            const float d = p.diag[(long long)z * p.Md + m];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(d, h[e], v[e]);
          } else {
            float d[8];
            load8(p.diag, TYPE_F32, (long long)z * p.Nd + n, d);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(d[e], h[e], v[e]);
          }
        }
        if (two) {
          float l[8];
          unpack8(el[i & 1][it], TYPE_F16, l);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] += l[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(p.alpha, h[e], p.beta * v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= p.beta;
      }
      if constexpr (KIND != KIND_LAST) {
        if (KIND == KIND_SYM && p.diag_of == DIAG_OUT) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (n + e == m) { p.diag[(long long)z * p.Md + m] = v[e]; v[e] = 0.0f; }
        }
        const long long at = z * p.sC + (long long)m * p.ldc + n;
        uint4 h, l;
        split8(v, h, l);
        *reinterpret_cast<uint4 *>(p.C + at) = h;
        if (two) *reinterpret_cast<uint4 *>(p.Cl + at) = l;
        if (mirror) {
          *reinterpret_cast<float4 *>(stg + r * SLD + cc) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4 *>(stg + r * SLD + cc + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
      } else {
        if (m >= p.rows) continue;
        const long long at = z * p.out.so + (long long)m * p.out.ldo + n, sat = z * p.out.sshadow + (long long)m * p.out.ldo + n;
        if (p.vec) {                              // (cols is a multiple of 8)
          if (p.out.update) {
            float x[8];
            load8(p.out.o, p.out.type, at, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(decay, x[e], -gain * v[e]);
          }
          store8(p.out.o, p.out.type, at, v);
          if (p.out.shadow) store8(p.out.shadow, TYPE_BF16, sat, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) stg[r * SLD + cc + e] = v[e];
#pragma unroll 1
          for (int e = 0; e < 8 && n + e < p.cols; ++e) {
            float x = stg[r * SLD + cc + e];
            if (p.out.update) x = fmaf(decay, load_as_f32(p.out.o, p.out.type, at + e), -gain * x);
            store_from_f32(p.out.o, p.out.type, at + e, x);
            if (p.out.shadow) p.out.shadow[sat + e] = f2bf(x);
          }
        }
      }
    }
    if (mirror) {
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int it = 0; it < TN * 4 / 64; ++it) {
        const int q = it * 64 + lane, c = q >> 2, r0 = (q & 3) * 8;
        const int m = m0 + slice_row(i) + r0, n = n0 + wn * TN + c;       // C[n][m ..]
        if (m >= p.Md || n >= p.Nd) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = stg[(r0 + e) * SLD + c];
        uint4 h, l;
        split8(v, h, l);
        const long long at = z * p.sC + (long long)n * p.ldc + m;
        *reinterpret_cast<uint4 *>(p.C + at) = h;
        if (SPLIT) *reinterpret_cast<uint4 *>(p.Cl + at) = l;
      }
    }
    __builtin_amdgcn_wave_barrier();
  });
}

template <int BM, int BN, int BK, int WM, int WN, int NS, bool PP, bool AT, bool BT, bool SPLIT, int KIND>
hipError_t launch_cfg(const OrthGemmP &p, hipStream_t s) {
  constexpr size_t tiles = (size_t)NS * (BM + BN) * BK * 2, epi = (size_t)WM * WN * 32 * (BN / WN + 4) * 4;
  constexpr size_t lds = tiles > epi ? tiles : epi;
  static_assert(lds <= 160 * 1024, "LDS budget");
  auto kern = orth_gemm_kernel<BM, BN, BK, WM, WN, NS, PP, AT, BT, SPLIT, KIND>;
  const int tm = (p.Md + BM - 1) / BM, tn = (p.Nd + BN - 1) / BN;
  if ((KIND == KIND_SYM) != (p.sym != 0) || (p.sym && (BM != BN || p.Md != p.Nd))) return hipErrorInvalidValue;
  const long long nblk = (p.sym ? (long long)tn * (tn + 1) / 2 : (long long)tm * tn) * p.batch;
  if (nblk > 0x3fffffff) return hipErrorInvalidValue;
  if (lds > 64 * 1024) {
    static std::once_flag once;
    static hipError_t err = hipSuccess;
    std::call_once(once, [&] { err = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds); });
    if (err != hipSuccess) return err;
  }
  const int chunk = (int)((nblk + 7) / 8);
  hipLaunchKernelGGL(kern, dim3(chunk * 8), dim3(WM * WN * 64), lds, s, p, tm, tn, (int)nblk, chunk);
  return hipGetLastError();
}

long long tile_count(const OrthGemmP &p, int e) {
  const long long tm = (p.Md + e - 1) / e, tn = (p.Nd + e - 1) / e;
  return (p.sym ? tn * (tn + 1) / 2 : tm * tn) * p.batch;
}

// Time of `blocks` 128 x 128 tiles per k-tile: full rounds of two work-groups to a CU and the last one (as in gemm_bf16.hip)
double rounds_128(long long blocks) {
  const long long full = blocks / 512, rem = blocks - full * 512;
  const double last = rem > 256 ? 1.42 : rem == 0 ? 0.0 : full == 0 ? 1.13 : 1.13 + 0.29 * (double)rem / 256;
  return 1.42 * (double)full + last;
}

template <bool AT, bool BT, bool SPLIT, int KIND>
hipError_t launch_shape(const OrthGemmP &p, hipStream_t s) {
  const long long t256 = tile_count(p, 256), t128 = tile_count(p, 128);
  if (p.Md > 128 && p.Nd > 128 && p.Kd * (SPLIT ? 3 : 1) >= 512 && 1.5 * (double)((t256 + 255) / 256) <= rounds_128(t128))
    return launch_cfg<256, 256, 64, 2, 4, 2, true, AT, BT, SPLIT, KIND>(p, s);
  if (t128 <= 256) return launch_cfg<128, 128, 64, 2, 2, 4, false, AT, BT, SPLIT, KIND>(p, s);
  return launch_cfg<128, 128, 64, 2, 2, 2, false, AT, BT, SPLIT, KIND>(p, s);
}

template <bool AT, bool BT, int KIND>
hipError_t launch_product(const OrthGemmP &p, hipStream_t s) {
  // operand checks the kernel relies on: 16-byte aligned rows of whole chunks, operands below 2 GiB per matrix
  if (((p.lda | p.ldb | p.Md | p.Nd | p.Kd) & 7) || ((p.sA | p.sB) & 7)) return hipErrorInvalidValue;
  if ((long long)(AT ? p.Kd : p.Md) * p.lda * 2 >= (1LL << 31) || (long long)(BT ? p.Kd : p.Nd) * p.ldb * 2 >= (1LL << 31)) return hipErrorInvalidValue;
  return p.Al ? launch_shape<AT, BT, true, KIND>(p, s) : launch_shape<AT, BT, false, KIND>(p, s);
}

// Few rows average little of what 16-bit operands round away (relative error up to 1.6e-2 for 2 x 2, 4.4e-3 for 8 x 8, 3.2e-3 for 17 x 33)
constexpr int SPLIT_ALWAYS = 128;

// power of two that leaves a bound just under fp16's largest value
int exponent_for(double bound) { return 15 - (int)std::ceil(std::log2(bound)); }

}  // namespace

OrthScale OrthPlan::scale(int k) const {
  const int to = k + 1 == steps ? 0 : ex[k + 1];           // (the result itself is not scaled)
  return {std::ldexp(1.0f, ea[k] - 2 * ex[k]), std::ldexp(b[k], eb[k] - ea[k]), std::ldexp(c[k], eb[k] - 2 * ea[k]),
          std::ldexp(a[k], to - ex[k]), std::ldexp(1.0f, to - eb[k] - ex[k])};
}

const char *orth_plan(int batch, int rows, int cols, int split, int steps, const float *coef, OrthPlan &pl) {
  std::memset(&pl, 0, sizeof(pl));
  pl.batch = batch; pl.rows = rows; pl.cols = cols; pl.steps = steps;
  pl.wide = rows <= cols;
  auto up8 = [](int v) { return (v + 7) / 8 * 8; };
  pl.rp = up8(rows); pl.cp = up8(cols); pl.mp = std::min(pl.rp, pl.cp);
  pl.split = split || pl.mp <= SPLIT_ALWAYS;
  // Bounds of the singular values: 1 at first, then max |p| over [0, bound], with 2^-6 more for what rounding adds.
  double s = 1.0;
  pl.ex[0] = exponent_for(s);
  for (int k = 0; k < steps; ++k) {
    const double a = coef ? coef[3 * k] : 3.4445, b = coef ? coef[3 * k + 1] : -4.7750, c = coef ? coef[3 * k + 2] : 2.0315;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return "coefficients must be finite";
    pl.a[k] = (float)a; pl.b[k] = (float)b; pl.c[k] = (float)c;
    // extrema of p on [0, s]: the ends and where a + 3 b t + 5 c t^2 = 0, t = sigma^2; of b t + c t^2: the end and -b / 2c
    const double S = s * s;
    auto poly = [&](double t) { return std::fabs(std::sqrt(t) * (a + t * (b + t * c))); };
    double top = poly(S);
    if (c != 0.0) {
      const double d = 9.0 * b * b - 20.0 * a * c;
      if (d >= 0.0)
        for (double q : {(-3.0 * b + std::sqrt(d)) / (10.0 * c), (-3.0 * b - std::sqrt(d)) / (10.0 * c)})
          if (q > 0.0 && q < S) top = std::max(top, poly(q));
    } else if (b != 0.0) {
      const double q = -a / (3.0 * b);
      if (q > 0.0 && q < S) top = std::max(top, poly(q));
    }
    double inner = std::fabs(b * S + c * S * S);
    if (c != 0.0) {
      const double q = -b / (2.0 * c);
      if (q > 0.0 && q < S) inner = std::max(inner, std::fabs(q * (b + q * c)));
    }
    s = top * (1.0 + 1.0 / 64);
    if (s > 256.0 || s < 1.0 / 256 || inner > 4096.0) return "the coefficients let singular values grow beyond 256 or vanish";
    pl.ea[k] = exponent_for(S * (1.0 + 1.0 / 32));
    pl.eb[k] = exponent_for(std::max(inner, 1.0 / 256) * (1.0 + 1.0 / 32));
    pl.ex[k + 1] = exponent_for(s);
  }
  if (orth_small_fits(rows, cols)) { pl.total = 256; return nullptr; }     // (all of it is in LDS)
  // about 16 chunks of 8 values to a thread of the norm's pass, as long as a matrix has them
  pl.nparts = (int)std::min<long long>(ORTH_PARTS, ((long long)rows * cols + 256 * 128 - 1) / (256 * 128));
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o = (o + bytes + 255) / 256 * 256; return r; };
  const size_t xb = (size_t)batch * pl.rp * pl.cp * 2, ab = (size_t)batch * pl.mp * pl.mp * 2;
  pl.o_part = take((size_t)batch * pl.nparts * 8);
  for (int i = 0; i < 2; ++i) pl.o_x[i] = take(xb);
  pl.o_xl[0] = take(xb);
  pl.o_xl[1] = pl.split ? take(xb) : pl.o_xl[0];     // (16-bit mode: no product reads it, each entry is replaced where it was read)
  pl.o_a = take(ab); pl.o_b = take(ab);
  pl.o_diag = pl.split ? 0 : take((size_t)batch * pl.mp * 4);
  pl.o_al = pl.split ? take(ab) : 0; pl.o_bl = pl.split ? take(ab) : 0;
  pl.total = o;
  return nullptr;
}

hipError_t launch_orthogonalize(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, void *workspace, hipStream_t s) {
  if (orth_small_fits(pl.rows, pl.cols)) return launch_orth_small(pl, in, out, eps, s);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  auto at = [&](size_t off) { return reinterpret_cast<uint16_t *>(ws + off); };
  const long long sx = (long long)pl.rp * pl.cp, sa = (long long)pl.mp * pl.mp;
  OrthPrepP q;
  std::memset(&q, 0, sizeof(q));
  q.in = in; q.rows = pl.rows; q.cols = pl.cols; q.rp = pl.rp; q.cp = pl.cp; q.nparts = pl.nparts; q.ex = pl.ex[0]; q.eps = eps;
  q.vec = rows_of_vectors(in.g, in.type, in.sg, in.ldg, pl.cols) && (!in.v || rows_of_vectors(in.v, TYPE_F32, in.sv, pl.cols, pl.cols));
  q.part = reinterpret_cast<double *>(ws + pl.o_part); q.xh = at(pl.o_x[0]); q.xl = at(pl.o_xl[0]);
  for (int z0 = 0; z0 < pl.batch; z0 += 32768) {  // (grids have 65535 places along y)
    OrthPrepP b = q;
    const int nz = std::min(32768, pl.batch - z0);
    b.in.g = static_cast<const unsigned char *>(in.g) + z0 * in.sg * type_bytes(in.type);
    if (in.v) b.in.v = in.v + z0 * in.sv;
    b.part += (long long)z0 * pl.nparts; b.xh += z0 * sx; b.xl += z0 * sx;
    hipLaunchKernelGGL(orth_norm_kernel, dim3(pl.nparts, nz), dim3(256), 0, s, b);
    hipLaunchKernelGGL(orth_prep_kernel, dim3((pl.rp * (pl.cp / 8) + 1023) / 1024, nz), dim3(256), 0, s, b);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  for (int k = 0; k < pl.steps; ++k) {
    const uint16_t *x = at(pl.o_x[k & 1]), *xl = at(pl.o_xl[k & 1]);
    OrthGemmP p;
    hipError_t e;
    // A 2^ea
    std::memset(&p, 0, sizeof(p));
    p.batch = pl.batch; p.sym = 1;
    p.A = p.B = x; p.sA = p.sB = sx; p.lda = p.ldb = pl.cp; p.Md = p.Nd = pl.mp; p.Kd = pl.wide ? pl.cp : pl.rp;
    if (pl.split) p.Al = p.Bl = xl;
    p.C = at(pl.o_a); p.Cl = pl.split ? at(pl.o_al) : nullptr; p.sC = sa; p.ldc = pl.mp;
    p.beta = pl.scale(k).gram;
    e = pl.wide ? launch_product<false, false, KIND_SYM>(p, s) : launch_product<true, true, KIND_SYM>(p, s);
    if (e != hipSuccess) return e;
    // B 2^eb = (b A + c A A) 2^eb
    std::memset(&p, 0, sizeof(p));
    p.batch = pl.batch; p.sym = 1;
    p.A = p.B = p.E = at(pl.o_a); p.sA = p.sB = p.sE = sa; p.lda = p.ldb = p.lde = pl.mp; p.Md = p.Nd = p.Kd = pl.mp;
    if (pl.split) p.Al = p.Bl = p.El = at(pl.o_al);
    p.C = at(pl.o_b); p.Cl = pl.split ? at(pl.o_bl) : nullptr; p.sC = sa; p.ldc = pl.mp;
    p.alpha = pl.scale(k).poly_a; p.beta = pl.scale(k).poly_aa;
    float *diag = reinterpret_cast<float *>(ws + pl.o_diag);
    if (!pl.split) { p.diag = diag; p.diag_of = DIAG_OUT; }
    e = launch_product<false, false, KIND_SYM>(p, s);
    if (e != hipSuccess) return e;
    // X' = a X + B X, or a X + X B
    std::memset(&p, 0, sizeof(p));
    p.batch = pl.batch;
    const bool last = k + 1 == pl.steps;
    p.Md = pl.rp; p.Nd = pl.cp; p.Kd = pl.mp;
    p.E = x; p.El = xl; p.sE = sx; p.lde = pl.cp;
    if (!pl.split) { p.diag = diag; p.diag_of = pl.wide ? DIAG_ROWS : DIAG_COLS; }
    p.alpha = pl.scale(k).apply_x; p.beta = pl.scale(k).apply_bx;
    if (last) {
      p.out = out; p.rows = pl.rows; p.cols = pl.cols;
      p.vec = rows_of_vectors(out.o, out.type, out.so, out.ldo, pl.cols) &&
              (!out.shadow || rows_of_vectors(out.shadow, TYPE_BF16, out.sshadow, out.ldo, pl.cols));
    } else {
      p.C = at(pl.o_x[~k & 1]); p.Cl = at(pl.o_xl[~k & 1]); p.sC = sx; p.ldc = pl.cp;
    }
    if (pl.wide) {
      p.A = at(pl.o_b); p.sA = sa; p.lda = pl.mp; p.B = x; p.sB = sx; p.ldb = pl.cp;
      if (pl.split) { p.Al = at(pl.o_bl); p.Bl = xl; }
      e = last ? launch_product<false, true, KIND_LAST>(p, s) : launch_product<false, true, KIND_APPLY>(p, s);
    } else {
      p.A = x; p.sA = sx; p.lda = pl.cp; p.B = at(pl.o_b); p.sB = sa; p.ldb = pl.mp;
      if (pl.split) { p.Al = xl; p.Bl = at(pl.o_bl); }
      e = last ? launch_product<false, false, KIND_LAST>(p, s) : launch_product<false, false, KIND_APPLY>(p, s);
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace absk
