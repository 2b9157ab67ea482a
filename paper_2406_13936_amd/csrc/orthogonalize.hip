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
//
// Memory.  16-bit mode: the two parts of X are two arrays.  With `split` a row holds 32 first parts, then the 32 second parts that
// belong to them, and so on, for X, A and B alike: one stage of operands brings both parts of 32 k and three MFMAs take them
// (hi lo, lo hi, hi hi).  A CU is fed about 43 bytes a ns, which bounds all tiles here; three passes over separate arrays
// would bring each part one and a half times.
#include <algorithm>
#include <cmath>
#include <cstring>
#include "device_utils.h"
#include "mfma_tile.h"
#include "ops.h"
#include "orth_parts.h"
#include "typed_mem.h"

namespace absk {

namespace {

// place of column c's first part in a row of pairs of 32; its second part follows 32 places on
__device__ __forceinline__ int paired(int c) { return 2 * (c & ~31) + (c & 31); }

// ---- norm and first X ----------------------------------------------------------------------------------------------

struct OrthPrepP {
  OrthIn in;
  int rows, cols, rp, cp, nparts, ex;
  double *part; uint16_t *xh, *xl;       // (split: xl null, both parts in xh)
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
    load_u8<true>(p.in, p.rows, p.cols, z, r, c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)u[e], (double)u[e], sum);
  }
  const double t = block_sum<4>(sum, sm);
  if (threadIdx.x == 0) p.part[(long long)z * p.nparts + blockIdx.x] = t;
}

// X_0 2^ex as two fp16 values, zeros in the rows and columns that round the sides up to 8.  (Loads of all of a thread's chunks before the
// scale is known: 18 -> 30 us for 4096 x 4096.)
__global__ void __launch_bounds__(256) orth_prep_kernel(const OrthPrepP p) {
  __shared__ double sm[4];
  __shared__ double scale;
  const int z = blockIdx.y;
  const double t = block_sum<4>((int)threadIdx.x < p.nparts ? p.part[(long long)z * p.nparts + threadIdx.x] : 0.0, sm);
  if (threadIdx.x == 0) scale = ldexp(1.0 / (sqrt(t) + (double)p.eps), p.ex);
  __syncthreads();
  const double sc = scale;
  const long long x0 = (long long)z * p.rp * p.cp * (p.xl ? 1 : 2);
  const int cc = p.cp >> 3, n = p.rp * cc;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const int r = i / cc, c = (i - r * cc) * 8;
    float u[8];
    load_u8<false>(p.in, p.rows, p.cols, z, r, c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = (float)((double)u[e] * sc);
    uint4 h, l;
    split8(u, h, l);
    const long long at = x0 + (p.xl ? (long long)r * p.cp + c : (long long)r * 2 * p.cp + paired(c));
    *reinterpret_cast<uint4 *>(p.xh + at) = h;
    *reinterpret_cast<uint4 *>(p.xl ? p.xl + at : p.xh + at + 32) = l;
  }
}

// ---- the products --------------------------------------------------------------------------------------------------

// C[z][m][n] = alpha E[z][m][n] + beta sum_k A[z][m][k] B[z][n][k]   as one or two fp16 values, or the result of the last step
struct OrthGemmP {
  const uint16_t *A, *B;
  long long sA, sB; int lda, ldb, Md, Nd, Kd, batch;
  const uint16_t *E, *El; long long sE; int lde;
  uint16_t *C, *Cl; long long sC; int ldc;       // (split: pairs of 32, El and Cl null; strides and ld count places of memory)
  float alpha, beta;
  int sym;                               // C is symmetric: tiles below the diagonal are written from those above it
  float *diag; int diag_of;              // [z][mp] fp32 diagonal: DIAG_OUT: C's, which is stored as zeros there; DIAG_ROWS, DIAG_COLS:
                                         //   beta diag[m] (or [n]) times E's first part is added
  OrthOut out; int rows, cols;           // the last step (C null)
};

// Tiles BM x BN x BK with WM x WN wavefronts, NS stages of direct global -> LDS loads; operands k-contiguous or row-contiguous as
// in gemm_bf16.hip.  PP: its pipelined loop of 256 x 256 tiles (eight 16 KB units of LDS, each refilled seven phases before it is
// read, four wavefronts half a phase behind the others; the reasons stand there).  SPLIT: BK places of memory are BK / 2 k.  WK: that many groups of WM x WN wavefronts share a tile, each with its part of
// every k-tile; their accumulators are added in order on the way to the epilogue.
enum { DIAG_NONE = 0, DIAG_OUT, DIAG_ROWS, DIAG_COLS };
enum { KIND_SYM = 0, KIND_APPLY = 1, KIND_LAST = 2 };   // A and B; X'; X' of the last step
constexpr int BAND = 8;                  // columns of 256-wide tiles that stand side by side (gemm_bf16.hip)

template <int BM, int BN, int BK, int WM, int WN, int WK, int NS, bool PP, bool AT, bool BT, bool SPLIT, int KIND>
__global__ void __launch_bounds__(WM * WN * WK * 64) orth_gemm_kernel(const OrthGemmP p, const int tilesM, const int tilesN, const int nblk, const int chunk) {
  constexpr int NG = WM * WN, NW = NG * WK;       // wavefronts of a group, and of the work-group
  constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 32, NI = TN / 32;
  constexpr int STAGE = (BM + BN) * BK, NPART = BK / 16 / WK;       // MFMA groups of a wavefront per k-tile
  static_assert(!PP || (WK == 1 && BM == 256 && BN == 256 && BK == 64 && WM == 2 && WN == 4), "the pipelined loop");
  // a row-contiguous operand of pairs has twice the columns and half the k
  constexpr int FA = SPLIT && AT ? 2 : 1, FB = SPLIT && BT ? 2 : 1;
  typedef Operand<BM * FA, BK / FA, AT, NW> OpA;
  typedef Operand<BN * FB, BK / FB, BT, NW> OpB;
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
  const int kg = wave / NG, wm = wave % NG / WN, wn = wave % WN;

  const int abytes = (int)((long long)(AT ? p.Kd : p.Md) * p.lda * 2), bbytes = (int)((long long)(BT ? p.Kd : p.Nd) * p.ldb * 2);
  const int KA = p.Kd * (SPLIT && !AT ? 2 : 1), KB = p.Kd * (SPLIT && !BT ? 2 : 1);       // extents of the reduction in memory
  auto rsrc = [](const uint16_t *q, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(q), 0, bytes, 0x00020000); };
  const __amdgpu_buffer_rsrc_t ra = rsrc(p.A + z * p.sA, abytes), rb = rsrc(p.B + z * p.sB, bbytes);

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

  const int KT = (p.Kd * (SPLIT ? 2 : 1) + BK - 1) / BK;
  if constexpr (PP) {
    typedef Operand<128 * FA, 64 / FA, AT, NW, 32> UA;       // A unit h: rows 128 h .. 128 h + 127 of the tile
    // B unit c: columns 64 j + 32 c ..; of a row-contiguous operand without pairs k 32 c .. of all columns
    typedef Operand<BT ? 256 : 128, BT ? 32 : 64, BT, NW, 32> UB;
    constexpr int UNIT = 8192;                               // elements of a unit (16 KB)
    UA ua[2];
    UB ub[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ua[h].init(wave, lane, (m0 + h * 128) * FA, p.Md * FA, p.lda);
      if constexpr (BT && SPLIT) ub[h].init_cols(wave, lane, 2 * p.Nd, p.ldb, [&](int ch) -> int { return 2 * n0 + (ch >> 3) * 128 + h * 64 + (ch & 7) * 8; });
      else if constexpr (BT) ub[h].init(wave, lane, n0, p.Nd, p.ldb);
      else ub[h].template init<true>(wave, lane, n0 + h * 32, p.Nd, p.ldb);
    }
    // (k-tiles beyond the last bring zeros)
    auto load_a = [&](int kt, int slot, int h) { ua[h].load_all(ra, smem + (slot * 2 + h) * UNIT, wave, kt * (64 / FA), 0, KA, p.lda); };
    auto load_b = [&](int kt, int slot, int c) { ub[c].load_all(rb, smem + (4 + slot * 2 + c) * UNIT, wave, kt * (64 / FB) + (BT && !SPLIT ? c * 32 : 0), 0, KB, p.ldb); };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const int i16 = lane & 15, g16 = lane >> 4;
    const int kq = g16 * 8 + (i16 >> 2);                     // transpose reads: k within the 32-wide step
    uint32_t aaddr[AT ? 4 * FA : 2], baddr[BT ? 4 : 2];      // (transpose reads: by row tile and part; else by k-step or part)
    if constexpr (AT) {
#pragma unroll
      for (int q = 0; q < 4 * FA; ++q) {
        const int ii = q / FA, rr = (SPLIT ? paired(wm * 64 + ii * 16) + 32 * (q & 1) : wm * 64 + ii * 16) + 4 * (i16 & 3);
        aaddr[q] = lds0 + 2u * (uint32_t)(kq * (128 * FA) + ((rr >> 3) ^ tr_swizzle<32>(kq)) * 8 + (rr & 7));
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        aaddr[kk] = lds0 + (uint32_t)((wm * 64 + i16) * 128 + (((kk * 4 + g16) ^ (i16 >> 1)) << 4));
    }
    if constexpr (BT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int rr = wn * 64 + (SPLIT ? (j >> 1) * 16 + (j & 1) * 32 : j * 16) + 4 * (i16 & 3);
        baddr[j] = lds0 + 65536u + 2u * (uint32_t)(kq * 256 + ((rr >> 3) ^ tr_swizzle<32>(kq)) * 8 + (rr & 7));
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        baddr[kk] = lds0 + 65536u + (uint32_t)((wn * 32 + i16) * 128 + (((kk * 4 + g16) ^ (i16 >> 1)) << 4));
    }
    // fa[row tile][k-step, or part]; fb[unit][2 column tile + k-step or part; row-contiguous without pairs: column tile]
    bf16x8 fa[4][2], fb[2][4];
    auto read_a = [&](auto SLOT, auto H) {
      constexpr int U = (decltype(SLOT)::value * 2 + decltype(H)::value) * UNIT * 2;
      static_for<8>([&](auto I) {
        constexpr int kk = decltype(I)::value >> 2, ii = decltype(I)::value & 3;
        if constexpr (AT && SPLIT) fa[ii][kk] = lds_read_cols<U, 2048>(aaddr[2 * ii + kk]);
        else if constexpr (AT) fa[ii][kk] = lds_read_cols<U + kk * 8192, 1024>(aaddr[ii]);
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
      static_for<SPLIT ? 24 : 16>([&](auto I) {              // (operands swapped: a lane owns one row of C)
        constexpr int q = decltype(I)::value;
        if constexpr (SPLIT) {                               // hi lo, lo hi, hi hi
          constexpr int part = q >> 3, ii = (q >> 1) & 3, j = q & 1;
          acc16[4 * h + ii][2 * c + j] = mfma(fb[c][2 * j + (part == 0)], fa[ii][part == 1], acc16[4 * h + ii][2 * c + j]);
        } else if constexpr (BT) {
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
  oa.init(wave, lane, m0 * FA, p.Md * FA, p.lda);
  ob.init(wave, lane, n0 * FB, p.Nd * FB, p.ldb);
  constexpr int GROUPS = SPLIT ? NPART / 2 : NPART;         // MFMA groups of a wavefront per k-tile (16 k each)
  auto issue = [&](int kt, int buf, int part) {
    bf16_t *sa = smem + buf * STAGE, *sb = sa + BM * BK;
    const bool full = (kt + 1) * BK <= p.Kd * (SPLIT ? 2 : 1);
#pragma unroll
    for (int l = 0; l < NL; ++l) {
      if (l % GROUPS != part) continue;
      if (l < OpA::NI) oa.load(l, ra, sa, wave, kt, KA, p.lda, full);
      else ob.load(l - OpA::NI, rb, sb, wave, kt, KB, p.ldb, full);
    }
  };
  // fragments by row tile; with pairs of a row-contiguous operand the two parts stand 32 columns apart
  Frag<BM * FA, BK / FA, AT> fa[MI][FA];
  Frag<BN * FB, BK / FB, BT> fb[NI][FB];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int h = 0; h < FA; ++h) fa[i][h].init((wm * TM + i * 32) * FA + 32 * h, lane);
#pragma unroll
  for (int j = 0; j < NI; ++j)
#pragma unroll
    for (int h = 0; h < FB; ++h) fb[j][h].init((wn * TN + j * 32) * FB + 32 * h, lane);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < KT) {
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) issue(s, s, q);
    }
  for (int kt = 0; kt < KT; ++kt) {
    if (kt + NS - 1 <= KT) wait_vmcnt<(NS - 2) * NL>(); else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();                 // all waves' loads of kt visible; everyone is done with kt-1
    const bool more = kt + NS - 1 < KT;
    const bf16_t *S = smem + (kt % NS) * STAGE;
    constexpr int PARTS = SPLIT ? 2 : 1;
    bf16x8 af[2][MI * PARTS], bfr[2][NI * PARTS];
    auto read_rows = [&](bf16x8 (&to)[MI * PARTS], int g) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int h = 0; h < PARTS; ++h)
          to[i * PARTS + h] = fa[i][FA == 2 ? h : 0].read(S, SPLIT && !AT ? (g >> 1) * 4 + (g & 1) + 2 * h : g);
    };
    auto read_cols = [&](bf16x8 (&to)[NI * PARTS], int g) {
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int h = 0; h < PARTS; ++h)
          to[j * PARTS + h] = fb[j][FB == 2 ? h : 0].read(S + BM * BK, SPLIT && !BT ? (g >> 1) * 4 + (g & 1) + 2 * h : g);
    };
    auto read = [&](int to, int q) {              // (transpose reads first: the compiler does not count them)
      const int g = WK > 1 ? kg * GROUPS + q : q;
      if (BT && !AT) { read_cols(bfr[to], g); read_rows(af[to], g); }
      else { read_rows(af[to], g); read_cols(bfr[to], g); }
    };
    read(0, 0);
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
      const int cur = q & 1, nxt = cur ^ 1;
      if (q + 1 < GROUPS) read(nxt, q + 1);
      if (more) issue(kt + NS - 1, (kt + NS - 1) % NS, q);
      if (AT || BT) {
        constexpr int RD = ((AT ? 2 : 1) * MI + (BT ? 2 : 1) * NI) * PARTS, W = RD < 15 ? RD : 14;      // (the counter holds 15 at most)
        if (q + 1 < GROUPS) wait_frags<W>(af[cur], bfr[cur]); else wait_frags<0>(af[cur], bfr[cur]);
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      auto mfma = [](bf16x8 x, bf16x8 y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0); };
#pragma unroll
      for (int part = SPLIT ? 0 : 2; part < 3; ++part)      // hi lo, lo hi, hi hi; operands swapped: a lane owns one row m of C
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j)
            acc[i][j] = mfma(bfr[cur][j * PARTS + (SPLIT && part == 0)], af[cur][i * PARTS + (SPLIT && part == 1)], acc[i][j]);
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
  static_assert(SIT >= 1, "a slice is at least a vector to a lane");
  float *stg = reinterpret_cast<float *>(smem_raw) + wave * (32 * SLD), *sum = stg - kg * NG * (32 * SLD);     // this wavefront's, and the first group's
  auto slices_meet = [&]() {                      // what the groups of a tile have written is there
    if (WK > 1) __syncthreads(); else __builtin_amdgcn_wave_barrier();
  };
  auto slice_row = [&](int i) -> int { return PP ? (i >> 1) * 128 + wm * 64 + (i & 1) * 32 : wm * TM + i * 32; };
  uint4 eh[2][SIT], el[2][SIT];
  const bool two = KIND != KIND_SYM || SPLIT;     // E is hi + lo
  auto load_e = [&](int i, uint4 (&h)[SIT], uint4 (&l)[SIT]) {
#pragma unroll
    for (int it = 0; it < SIT; ++it) {
      if (WK > 1 && it % WK != kg) continue;
      const int q = it * 64 + lane, r = q / CPR, cc = (q % CPR) * 8;
      const int m = m0 + slice_row(i) + r, n = n0 + wn * TN + cc;
      h[it] = l[it] = make_uint4(0, 0, 0, 0);
      if (m < p.Md && n < p.Nd) {                 // (Nd is a multiple of 8)
        const long long at = z * p.sE + (long long)m * p.lde + (SPLIT ? paired(n) : n);
        h[it] = *reinterpret_cast<const uint4 *>(p.E + at);
        if (two) l[it] = *reinterpret_cast<const uint4 *>(SPLIT ? p.E + at + 32 : p.El + at);
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
    slices_meet();
#pragma unroll
    for (int it = 0; it < SIT; ++it) {
      if (WK > 1 && it % WK != kg) continue;
      const int q = it * 64 + lane, r = q / CPR, cc = (q % CPR) * 8;
      const int m = m0 + slice_row(i) + r, n = n0 + wn * TN + cc;
      if (m >= p.Md || n >= p.Nd) continue;
      float v[8];
      load8(sum, TYPE_F32, r * SLD + cc, v);
#pragma unroll
      for (int g = 1; g < WK; ++g) {
        float w[8];
        load8(sum, TYPE_F32, g * NG * (32 * SLD) + r * SLD + cc, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[e];
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
        const long long at = z * p.sC + (long long)m * p.ldc + (SPLIT ? paired(n) : n);
        uint4 h, l;
        split8(v, h, l);
        *reinterpret_cast<uint4 *>(p.C + at) = h;
        if (two) *reinterpret_cast<uint4 *>(SPLIT ? p.C + at + 32 : p.Cl + at) = l;
        if (mirror) {
          store8(sum, TYPE_F32, r * SLD + cc, v);
        }
      } else {
        if (m >= p.rows || n >= p.cols) continue;
        const long long at = z * p.out.so + (long long)m * p.out.ldo + n, sat = z * p.out.sshadow + (long long)m * p.out.ldo + n;
        if (n + 8 <= p.cols) {
          if (p.out.update) {
            float x[8];
            load8_any(p.out.o, p.out.type, at, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(decay, x[e], -gain * v[e]);
          }
          store8_any(p.out.o, p.out.type, at, v);
          if (p.out.shadow) store8_any(p.out.shadow, TYPE_BF16, sat, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[r * SLD + cc + e] = v[e];
#pragma unroll 1
          for (int e = 0; e < 8 && n + e < p.cols; ++e) {
            float x = sum[r * SLD + cc + e];
            if (p.out.update) x = fmaf(decay, load_as_f32(p.out.o, p.out.type, at + e), -gain * x);
            store_from_f32(p.out.o, p.out.type, at + e, x);
            if (p.out.shadow) p.out.shadow[sat + e] = f2bf(x);
          }
        }
      }
    }
    if (mirror) {
      slices_meet();
#pragma unroll
      for (int it = 0; it < TN * 4 / 64; ++it) {
        if (WK > 1 && it % WK != kg) continue;
        const int q = it * 64 + lane, c = q >> 2, r0 = (q & 3) * 8;
        const int m = m0 + slice_row(i) + r0, n = n0 + wn * TN + c;       // C[n][m ..]
        if (m >= p.Md || n >= p.Nd) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sum[(r0 + e) * SLD + c];
        uint4 h, l;
        split8(v, h, l);
        const long long at = z * p.sC + (long long)n * p.ldc + (SPLIT ? paired(m) : m);
        *reinterpret_cast<uint4 *>(p.C + at) = h;
        if (SPLIT) *reinterpret_cast<uint4 *>(p.C + at + 32) = l;
      }
    }
    if (i + 1 < MI) slices_meet();
  });
}

template <int BM, int BN, int BK, int WM, int WN, int WK, int NS, bool PP, bool AT, bool BT, bool SPLIT, int KIND>
hipError_t launch_cfg(const OrthGemmP &p, hipStream_t s) {
  constexpr size_t tiles = (size_t)NS * (BM + BN) * BK * 2, epi = (size_t)WM * WN * WK * 32 * (BN / WN + 4) * 4;
  constexpr size_t lds = tiles > epi ? tiles : epi;
  static_assert(lds <= 160 * 1024, "LDS budget");
  auto kern = orth_gemm_kernel<BM, BN, BK, WM, WN, WK, NS, PP, AT, BT, SPLIT, KIND>;
  const int tm = (p.Md + BM - 1) / BM, tn = (p.Nd + BN - 1) / BN;
  if ((KIND == KIND_SYM) != (p.sym != 0) || (p.sym && (BM != BN || p.Md != p.Nd))) return hipErrorInvalidValue;
  const long long nblk = (p.sym ? (long long)tn * (tn + 1) / 2 : (long long)tm * tn) * p.batch;
  if ((nblk + 7) * (WM * WN * WK * 64) > 0xffffffffLL) return hipErrorInvalidValue;      // (a grid counts its threads in 32 bits)
  if (lds > 64 * 1024) {
    static std::atomic<uint64_t> done{0};
    const hipError_t err = allow_lds(reinterpret_cast<const void *>(kern), lds, done);
    if (err != hipSuccess) return err;
  }
  const int chunk = (int)((nblk + 7) / 8);
  hipLaunchKernelGGL(kern, dim3(chunk * 8), dim3(WM * WN * WK * 64), lds, s, p, tm, tn, (int)nblk, chunk);
  return hipGetLastError();
}

// Time of `blocks` 128 x 128 tiles per k-tile: full rounds of two work-groups to a CU and the last one (as in gemm_bf16.hip)
double rounds_128(long long blocks) {
  const long long full = blocks / 512, rem = blocks - full * 512;
  const double last = rem > 256 ? 1.42 : rem == 0 ? 0.0 : full == 0 ? 1.13 : 1.13 + 0.29 * (double)rem / 256;
  return 1.42 * (double)full + last;
}

long long tile_count(int Md, int Nd, int batch, int sym, int e) {
  const long long tm = (Md + e - 1) / e, tn = (Nd + e - 1) / e;
  return (sym ? tn * (tn + 1) / 2 : tm * tn) * batch;
}

template <bool AT, bool BT, bool SPLIT, int KIND>
hipError_t launch_shape(const OrthGemmP &p, hipStream_t s) {
  switch (orth_product_shape(p.Md, p.Nd, p.Kd * (SPLIT ? 2 : 1), p.batch, p.sym)) {
    case 25612: return launch_cfg<256, 256, 64, 2, 4, 1, 2, true, AT, BT, SPLIT, KIND>(p, s);
    case 12812: return launch_cfg<128, 128, 64, 2, 2, 1, 2, false, AT, BT, SPLIT, KIND>(p, s);
    case 12822: return launch_cfg<128, 128, 128, 2, 2, 2, 2, false, AT, BT, SPLIT, KIND>(p, s);
    case 6424: return launch_cfg<64, 64, 128, 2, 2, 2, 4, false, AT, BT, SPLIT, KIND>(p, s);
    case 6422: return launch_cfg<64, 64, 128, 2, 2, 2, 2, false, AT, BT, SPLIT, KIND>(p, s);
    default: return hipErrorInvalidValue;
  }
}

template <bool AT, bool BT, int KIND>
hipError_t launch_product(const OrthGemmP &p, int split, hipStream_t s) {
  // operand checks the kernel relies on: 16-byte aligned rows of whole chunks, operands below 2 GiB per matrix
  if (((p.lda | p.ldb | p.Md | p.Nd | p.Kd) & (split ? 31 : 7)) || ((p.sA | p.sB) & 7)) return hipErrorInvalidValue;
  if ((long long)(AT ? p.Kd : p.Md) * p.lda * 2 >= (1LL << 31) || (long long)(BT ? p.Kd : p.Nd) * p.ldb * 2 >= (1LL << 31)) return hipErrorInvalidValue;
  return split ? launch_shape<AT, BT, true, KIND>(p, s) : launch_shape<AT, BT, false, KIND>(p, s);
}

// Few rows average little of what 16-bit operands round away (relative error up to 1.6e-2 for 2 x 2, 4.4e-3 for 8 x 8, 3.2e-3 for 17 x 33)
constexpr int SPLIT_ALWAYS = 128;

// power of two that leaves a bound just under fp16's largest value
int exponent_for(double bound) { return 15 - (int)std::ceil(std::log2(bound)); }

}  // namespace

// Tile, groups of wavefronts to a tile and ring of stages (tile * 100 + groups * 10 + ring) of a product whose reduction is K places of
// memory long.  us a product, 128 x 128 tiles of four wavefronts with a ring of four -> this, measured over whole calls:
//   one tile of 64 x 64 to a CU: A and B of 12 of 1001 x 333 (252 tiles) in fp32 34 -> 13 and 21 -> 11, of one 1024 x 1024 (136) 40 -> 21,
//   of one 300 x 300 (15) 18 -> 9; two groups instead of one 3 to 8 % less, four no more
//   up to one and a half: 8 of 512 x 784 (288) 21 -> 10; 2 of 4096 x 1024 (272) 100 -> 50.  Beyond, 64 x 64 tiles bring too many bytes: one
//   2048 x 2048 (528 tiles; 136 of 128 x 128) 2 longer
//   up to one tile of 128 x 128 to a CU, two groups: one 2048 x 2048 (136, 256 tiles) 5 less, 8 of 512 x 784 (224) 3 less
int orth_product_shape(int Md, int Nd, int K, int batch, int sym) {
  const long long t256 = tile_count(Md, Nd, batch, sym, 256), t128 = tile_count(Md, Nd, batch, sym, 128), t64 = tile_count(Md, Nd, batch, sym, 64);
  if (t64 <= 384) return t64 <= 256 ? 6424 : 6422;
  if (K >= 512 && 1.5 * (double)((t256 + 255) / 256) <= rounds_128(t128)) return 25612;
  return t128 <= 256 ? 12822 : 12812;
}

OrthScale OrthPlan::scale(int k) const {
  const int to = k + 1 == steps ? 0 : ex[k + 1];           // (the result itself is not scaled)
  return {std::ldexp(1.0f, ea[k] - 2 * ex[k]), std::ldexp(b[k], eb[k] - ea[k]), std::ldexp(c[k], eb[k] - 2 * ea[k]),
          std::ldexp(a[k], to - ex[k]), std::ldexp(1.0f, to - eb[k] - ex[k])};
}

const char *orth_plan(int batch, int rows, int cols, int split, int steps, const float *coef, OrthPlan &pl) {
  std::memset(&pl, 0, sizeof(pl));
  pl.batch = batch; pl.rows = rows; pl.cols = cols; pl.steps = steps;
  pl.wide = rows <= cols;
  pl.split = split || std::min(rows, cols) <= SPLIT_ALWAYS;
  const int unit = pl.split ? 32 : 8;
  pl.rp = (rows + unit - 1) / unit * unit; pl.cp = (cols + unit - 1) / unit * unit; pl.mp = std::min(pl.rp, pl.cp);
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
  if (orth_small_fits(batch, rows, cols)) { pl.total = 256; return nullptr; }     // (all of it is in LDS)
  // two chunks of 8 values to a thread of the norm's pass, until there are as many blocks as one block of the next pass adds up
  pl.nparts = (int)std::min<long long>(ORTH_PARTS, ((long long)rows * cols + 4095) / 4096);
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o = (o + bytes + 255) / 256 * 256; return r; };
  const size_t xb = (size_t)batch * pl.rp * pl.cp * (pl.split ? 4 : 2), ab = (size_t)batch * pl.mp * pl.mp * (pl.split ? 4 : 2);
  pl.o_part = take((size_t)batch * pl.nparts * 8);
  if (orth_slices_fit(batch, rows, cols)) {
    size_t x, a, part;
    pl.o_x[0] = take(orth_slices_bytes(pl, x, a, part));
    pl.total = o;
    return nullptr;
  }
  for (int i = 0; i < 2; ++i) pl.o_x[i] = take(xb);
  pl.o_xl = pl.split ? 0 : take(xb);                // (no product reads it: each entry is replaced where it was read)
  pl.o_a = take(ab); pl.o_b = take(ab);
  pl.o_diag = pl.split ? 0 : take((size_t)batch * pl.mp * 4);
  pl.total = o;
  return nullptr;
}

hipError_t launch_orthogonalize(const OrthPlan &pl, const OrthIn &in, const OrthOut &out, float eps, void *workspace, hipStream_t s) {
  if (orth_small_fits(pl.batch, pl.rows, pl.cols)) return launch_orth_small(pl, in, out, eps, s);
  const bool slices = orth_slices_fit(pl.batch, pl.rows, pl.cols);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  auto at = [&](size_t off) { return reinterpret_cast<uint16_t *>(ws + off); };
  const int f = pl.split ? 2 : 1, ldx = f * pl.cp, lda = f * pl.mp;
  const long long sx = (long long)pl.rp * ldx, sa = (long long)pl.mp * lda;
  OrthPrepP q;
  std::memset(&q, 0, sizeof(q));
  q.in = in; q.rows = pl.rows; q.cols = pl.cols; q.rp = pl.rp; q.cp = pl.cp; q.nparts = pl.nparts; q.ex = pl.ex[0]; q.eps = eps;
  q.part = reinterpret_cast<double *>(ws + pl.o_part); q.xh = at(pl.o_x[0]); q.xl = pl.split ? nullptr : at(pl.o_xl);
  for (int z0 = 0; z0 < pl.batch; z0 += 32768) {  // (grids have 65535 places along y)
    OrthPrepP b = q;
    const int nz = std::min(32768, pl.batch - z0);
    b.in.g = static_cast<const unsigned char *>(in.g) + z0 * in.sg * type_bytes(in.type);
    if (in.v) b.in.v = in.v + z0 * in.sv;
    b.part += (long long)z0 * pl.nparts; b.xh += z0 * sx;
    if (b.xl) b.xl += z0 * sx;
    hipLaunchKernelGGL(orth_norm_kernel, dim3(pl.nparts, nz), dim3(256), 0, s, b);
    if (!slices) hipLaunchKernelGGL(orth_prep_kernel, dim3((pl.rp * (pl.cp / 8) + 1023) / 1024, nz), dim3(256), 0, s, b);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (slices) return launch_orth_slices(pl, in, out, eps, q.part, ws + pl.o_x[0], s);
  for (int k = 0; k < pl.steps; ++k) {
    const uint16_t *x = at(pl.o_x[k & 1]);
    OrthGemmP p;
    hipError_t e;
    // A 2^ea
    std::memset(&p, 0, sizeof(p));
    p.batch = pl.batch; p.sym = 1;
    p.A = p.B = x; p.sA = p.sB = sx; p.lda = p.ldb = ldx; p.Md = p.Nd = pl.mp; p.Kd = pl.wide ? pl.cp : pl.rp;
    p.C = at(pl.o_a); p.sC = sa; p.ldc = lda;
    p.beta = pl.scale(k).gram;
    e = pl.wide ? launch_product<false, false, KIND_SYM>(p, pl.split, s) : launch_product<true, true, KIND_SYM>(p, pl.split, s);
    if (e != hipSuccess) return e;
    // B 2^eb = (b A + c A A) 2^eb
    std::memset(&p, 0, sizeof(p));
    p.batch = pl.batch; p.sym = 1;
    p.A = p.B = p.E = at(pl.o_a); p.sA = p.sB = p.sE = sa; p.lda = p.ldb = p.lde = lda; p.Md = p.Nd = p.Kd = pl.mp;
    p.C = at(pl.o_b); p.sC = sa; p.ldc = lda;
    p.alpha = pl.scale(k).poly_a; p.beta = pl.scale(k).poly_aa;
    float *diag = reinterpret_cast<float *>(ws + pl.o_diag);
    if (!pl.split) { p.diag = diag; p.diag_of = DIAG_OUT; }
    e = launch_product<false, false, KIND_SYM>(p, pl.split, s);
    if (e != hipSuccess) return e;
    // X' = a X + B X, or a X + X B
    std::memset(&p, 0, sizeof(p));
    p.batch = pl.batch;
    const bool last = k + 1 == pl.steps;
    p.Md = pl.rp; p.Nd = pl.cp; p.Kd = pl.mp;
    p.E = x; p.El = pl.split ? nullptr : at(pl.o_xl); p.sE = sx; p.lde = ldx;
    if (!pl.split) { p.diag = diag; p.diag_of = pl.wide ? DIAG_ROWS : DIAG_COLS; }
    p.alpha = pl.scale(k).apply_x; p.beta = pl.scale(k).apply_bx;
    if (last) {
      p.out = out; p.rows = pl.rows; p.cols = pl.cols;
    } else {
      p.C = at(pl.o_x[~k & 1]); p.Cl = pl.split ? nullptr : at(pl.o_xl); p.sC = sx; p.ldc = ldx;
    }
    if (pl.wide) {
      p.A = at(pl.o_b); p.sA = sa; p.lda = lda; p.B = x; p.sB = sx; p.ldb = ldx;
      e = last ? launch_product<false, true, KIND_LAST>(p, pl.split, s) : launch_product<false, true, KIND_APPLY>(p, pl.split, s);
    } else {
      p.A = x; p.sA = sx; p.lda = ldx; p.B = at(pl.o_b); p.sB = sa; p.ldb = lda;
      e = last ? launch_product<false, false, KIND_LAST>(p, pl.split, s) : launch_product<false, false, KIND_APPLY>(p, pl.split, s);
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace absk
