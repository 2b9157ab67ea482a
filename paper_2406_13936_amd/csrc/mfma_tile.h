// Staging of 16-bit operand tiles in LDS and the reads of their matrix-core fragments, shared by the GEMM families that
// bring operands in with direct global -> LDS loads (gemm_bf16.hip, orthogonalize.hip; the tile layouts are described at
// the head of gemm_bf16.hip).  The element type only matters to the MFMA: fragments are raw 16-bit values here.
#pragma once
#include <utility>
#include "abs_internal.h"
#include "device_utils.h"

namespace absk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

namespace {

constexpr uint32_t OOB = 0x80000000u;   // byte offset beyond any operand (operands are < 2 GiB)

// XOR on the 16-byte chunk index of k-row k in a row-contiguous tile.  A 32-lane half of a transpose read meets four values of
// k x 4 chunks (KR = 16: 32 rows) or eight values of k, 0 .. 3 and 8 .. 11 of the step, x 2 chunks (KR = 32: 16 rows); either
// way the 16 chunks spread over all 64 banks (conflicts: 1 % of a weight gradient's LDS cycles, with either).  The same for k and k + 4, the fragment's second read, and for every k-step.
template <int KR> __device__ __forceinline__ int tr_swizzle(int k) { return KR == 16 ? 4 * (k & 3) : 2 * (k & 3) + (k & 8); }

template <int N> __device__ __forceinline__ void wait_vmcnt() {
  // s_waitcnt immediate on gfx9: vmcnt[3:0] | expcnt[6:4] | lgkmcnt[11:8] | vmcnt[5:4] at [15:14]
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// ---- one operand's stage: addressing of the direct loads and of the fragment reads ---------
// ROWS = tile extent along m (or n); TRANS = memory is [k][row]; KR: k per MFMA (which k-rows a transpose read meets).
template <int ROWS, int BK, bool TRANS, int NW, int KR = 16>
struct Operand {
  static constexpr int ELEMS = ROWS * BK;                 // bf16 elements per stage
  static constexpr int NI = ELEMS / 8 / 64 / NW;          // load instructions per wave per stage
  static_assert(ELEMS % (8 * 64 * NW) == 0 && NI >= 1, "tile too small for the wave count");
  static constexpr int CPR = BK / 8;                      // k-contiguous: chunks per row
  static constexpr int SWS = CPR >= 8 ? 1 : 2;
  static constexpr int CH = ROWS / 8;                     // row-contiguous: chunks per k-row
  static_assert(!TRANS || CH >= 8, "transposed tiles need at least 64 rows");

  uint32_t voff[NI];     // per-lane byte offset of its chunk at k0 = 0 (OOB if the row is outside)
  int kofs[NI];          // k (relative to k0) of the chunk, for the ragged last k-tile

  // SPREAD (k-contiguous only): stage row u holds matrix row row0 + 64 (u / 32) + u % 32, i.e. every second group of 32
  template <bool SPREAD = false>
  __device__ __forceinline__ void init(int wave, int lane, int row0, int rows, int ld) {
    static_assert(!(SPREAD && TRANS), "row-contiguous stages keep their rows in order");
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = (wave * NI + i) * 64 + lane;          // linear 16-byte chunk index in the stage
      if (!TRANS) {
        const int row = c / CPR, kc = (c % CPR) ^ ((row >> SWS) & (CPR - 1));
        const int mrow = row0 + (SPREAD ? (row >> 5) * 64 + (row & 31) : row);
        kofs[i] = kc * 8;
        voff[i] = (mrow < rows) ? (uint32_t)(mrow * ld + kc * 8) * 2u : OOB;
      } else {
        const int kq = c / CH, ch = (c % CH) ^ (tr_swizzle<KR>(kq) & (CH - 1));
        kofs[i] = kq;
        voff[i] = (row0 + ch * 8 < rows) ? (uint32_t)(kq * ld + row0 + ch * 8) * 2u : OOB;
      }
    }
  }
  // row-contiguous: chunk ch of a k-row holds the eight values from column col_of(ch) on
  template <class F>
  __device__ __forceinline__ void init_cols(int wave, int lane, int cols, int ld, F col_of) {
    static_assert(TRANS, "columns of a row-contiguous operand");
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = (wave * NI + i) * 64 + lane, kq = c / CH, col = col_of((c % CH) ^ (tr_swizzle<KR>(kq) & (CH - 1)));
      kofs[i] = kq;
      voff[i] = col < cols ? (uint32_t)(kq * ld + col) * 2u : OOB;
    }
  }
  // rows from elsewhere: matrix row r at row_of(r) of the operand (k-contiguous)
  template <class F>
  __device__ __forceinline__ void init_rows(int wave, int lane, int row0, int rows, int ld, F row_of) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int mrow = row0 + ((wave * NI + i) * 64 + lane) / CPR;
      if (mrow < rows) voff[i] = ((uint32_t)row_of(mrow) * (uint32_t)ld + (uint32_t)kofs[i]) * 2u;
    }
  }
  // byte offset added for k-tile kt (scalar)
  static __device__ __forceinline__ uint32_t soff(int kt, int ld) {
    return TRANS ? (uint32_t)kt * BK * ld * 2u : (uint32_t)kt * BK * 2u;
  }
  // i is a compile-time constant after unrolling (voff / kofs live in registers)
  __device__ __forceinline__ void load(int i, __amdgpu_buffer_rsrc_t rsrc, bf16_t *stage, int wave, int kt,
                                       int K, int ld, bool full) const {
    uint32_t v = voff[i];
    if (!full && kt * BK + kofs[i] >= K) v = OOB;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void *)(stage + (wave * NI + i) * 512), 16, v,
                                             soff(kt, ld), 0, 0);
  }
  // The whole stage from k = kbeg on, for callers that keep the number of loads in flight constant: chunks at or
  // beyond K come back as zeros, also where the stage lies wholly beyond it (then ksafe, a multiple of BK below K,
  // takes the place of kbeg in the scalar offset, which the range check subtracts from the operand's extent).
  __device__ __forceinline__ void load_all(__amdgpu_buffer_rsrc_t rsrc, bf16_t *stage, int wave, int kbeg, int ksafe, int K,
                                           int ld) const {
    const uint32_t so = (uint32_t)(kbeg < K ? kbeg : ksafe) * (TRANS ? (uint32_t)ld * 2u : 2u);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t v = kofs[i] < K - kbeg ? voff[i] : OOB;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void *)(stage + (wave * NI + i) * 512), 16, v, so, 0, 0);
    }
  }
};

// fragment of rows [r0, r0+32) for k-step kk of a stage
template <int ROWS, int BK, bool TRANS>
struct Frag {
  static constexpr int CPR = BK / 8, SWS = CPR >= 8 ? 1 : 2, CH = ROWS / 8;
  int base, swz;         // !TRANS: element offset of the row, and its swizzle
  int tbase[2];          // TRANS: element offsets for the two transpose reads at kk = 0
  __device__ __forceinline__ void init(int r0, int lane) {
    if (!TRANS) {
      const int r = r0 + (lane & 31);
      base = r * BK;
      swz = (r >> SWS) & (CPR - 1);
    } else {
      const int i16 = lane & 15, g16 = lane >> 4;
      const int rr = r0 + (g16 & 1) * 16 + 4 * (i16 & 3);     // first of this lane's 4 rows
      const int kq = (g16 >> 1) * 8 + (i16 >> 2);             // k within the 16-wide step
      const int ch = (rr >> 3) ^ (tr_swizzle<16>(kq) & (CH - 1));
      tbase[0] = kq * ROWS + ch * 8 + (rr & 7);
      tbase[1] = tbase[0] + 4 * ROWS;
    }
  }
  __device__ __forceinline__ bf16x8 read(const bf16_t *stage, int kk) const {
    if (!TRANS) {
      const int kc = kk * 2 + (threadIdx.x >> 5 & 1);
      return *reinterpret_cast<const bf16x8 *>(stage + base + ((kc ^ swz) << 3));
    } else {
      // Issued as inline assembly: through the builtin the compiler cannot tell that this read
      // does not alias the direct-to-LDS loads in flight (they fill the other stage buffer) and
      // puts s_waitcnt vmcnt(0) in front of every group of reads, which serialises the pipeline.
      // The price is that the compiler no longer counts these reads in lgkmcnt: the main loop
      // waits for them itself (wait_frags) before the MFMAs that use them.
      const uint32_t a0 = (uint32_t)(uintptr_t)(lds_void *)(stage + tbase[0] + kk * 16 * ROWS);
      const uint32_t a1 = (uint32_t)(uintptr_t)(lds_void *)(stage + tbase[1] + kk * 16 * ROWS);
      s16x4 lo, hi;
      asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(lo) : "v"(a0) : "memory");
      asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(hi) : "v"(a1) : "memory");
      const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, v);
    }
  }
};

// LDS fragment reads with the stage, row-tile and k-step as an immediate offset (inline assembly for the reason
// given in Frag::read; the caller waits for them itself)
template <int OFF> __device__ __forceinline__ bf16x8 lds_read_rows(uint32_t addr) {
  bf16x8 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
}
template <int OFF, int NEXT4> __device__ __forceinline__ bf16x8 lds_read_cols(uint32_t addr) {
  s16x4 lo, hi;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(lo) : "v"(addr), "n"(OFF) : "memory");
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(hi) : "v"(addr), "n"(OFF + NEXT4) : "memory");
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <int V> struct Const { static constexpr int value = V; };
template <int... I, class F> __device__ __forceinline__ void static_for_impl(std::integer_sequence<int, I...>, F &&f) {
  (f(Const<I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void static_for(F &&f) {
  static_for_impl(std::make_integer_sequence<int, N>{}, static_cast<F &&>(f));
}

// Wait until at most N LDS operations of this wave are outstanding, and make the fragments that
// the following MFMAs read depend on that wait (needed where fragment reads are inline assembly).
template <int N, int MI, int NI>
__device__ __forceinline__ void wait_frags(bf16x8 (&a)[MI], bf16x8 (&b)[NI]) {
  static_assert(N >= 0 && N <= 15, "lgkmcnt range");
  __builtin_amdgcn_s_waitcnt(0xC07F | (N << 8));          // vmcnt, expcnt: no wait; lgkmcnt = N
#pragma unroll
  for (int i = 0; i < MI; ++i) asm volatile("" : "+v"(a[i]));
#pragma unroll
  for (int j = 0; j < NI; ++j) asm volatile("" : "+v"(b[j]));
}

}  // namespace
}  // namespace absk
