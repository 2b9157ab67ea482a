// What the attention kernels share: sequences and their tiles, operand tiles in LDS, matrix-core fragments.
//
// Products are of 32 x 32 tiles with the reduction in steps of 16: a lane's fragment holds eight values, of row (lane & 31) of the operand and
// of the reduction's places 8 (lane >> 5) + e; results have column (lane & 31) and rows 8 (r / 4) + 4 (lane >> 5) + r % 4, r = 0 .. 15.  The order of the
// reduction is free as long as both operands have the same, so registers 8 b .. 8 b + 7 of a result are, rounded, a fragment of the next product
// whose places are rows 16 b + 8 (e / 4) + 4 (lane >> 5) + e % 4: scores never go through LDS, the other operand is read in that order instead.
// fp32 values take eight 32 x 32 x 2 products to a step, with the same fragments.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include "device_utils.h"
#include "mfma_tile.h"
#include "ops.h"
#include "row_groups.h"
#include "typed_mem.h"

namespace absk {
namespace {

// (a lambda that is called instead has what it captures, a wavefront's results, in memory)
#define INLINE __attribute__((always_inline))

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ---- types -----------------------------------------------------------------------------------------------------------

template <int TYPE> struct Frag8 { uint4 q; };                       // eight 16-bit values
template <> struct Frag8<TYPE_F32> { float v[8]; };
template <int TYPE> struct ElemOf { typedef uint16_t type; };
template <> struct ElemOf<TYPE_F32> { typedef float type; };

template <int TYPE> __device__ __forceinline__ void mma(f32x16 &c, const Frag8<TYPE> &a, const Frag8<TYPE> &b) {
  if constexpr (TYPE == TYPE_BF16) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.q), __builtin_bit_cast(bf16x8, b.q), c, 0, 0, 0);
  } else if constexpr (TYPE == TYPE_F16) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.q), __builtin_bit_cast(f16x8, b.q), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
  }
}
// registers 8 b .. 8 b + 7 of a result as a fragment
template <int TYPE> __device__ __forceinline__ Frag8<TYPE> as_frag(const f32x16 &c, int b) {
  Frag8<TYPE> f;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c[8 * b + e];
  if constexpr (TYPE == TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = v[e];
  } else {
    f.q = pack8(TYPE, v);
  }
  return f;
}
template <int TYPE> __device__ __forceinline__ void frag_values(const Frag8<TYPE> &f, float (&v)[8]) {
  if constexpr (TYPE == TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = f.v[e];
  } else {
    unpack8(f.q, TYPE, v);
  }
}
__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}
// an infinity or NaN?
__device__ __forceinline__ bool unusual(float v) { return !(fabsf(v) < __builtin_inff()); }
template <int TYPE> __device__ __forceinline__ uint32_t unusual_half(uint32_t w) {      // of a word's low 16 bits
  constexpr uint32_t E = TYPE == TYPE_BF16 ? 0x7f80u : 0x7c00u;
  return (w & E) == E;
}
// the sign bits are set where a value's exponent is all ones (one more carries into the sign's place)
template <int TYPE> __device__ __forceinline__ uint32_t unusual_signs(const uint4 q) {
  constexpr uint32_t E = TYPE == TYPE_F32 ? 0x7f800000u : TYPE == TYPE_BF16 ? 0x7f807f80u : 0x7c007c00u;
  constexpr uint32_t ONE = TYPE == TYPE_F32 ? 0x00800000u : TYPE == TYPE_BF16 ? 0x00800080u : 0x04000400u;
  return (((q.x & E) + ONE) | ((q.y & E) + ONE)) | (((q.z & E) + ONE) | ((q.w & E) + ONE));
}
template <int TYPE> __device__ __forceinline__ bool any_unusual(const Frag8<TYPE> &f) {
  if constexpr (TYPE == TYPE_F32) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) odd |= unusual(f.v[e]);
    return odd;
  } else {
    return (unusual_signs<TYPE>(f.q) & 0x80008000u) != 0;
  }
}
// zeros in the place of infinities and NaN
template <int TYPE> __device__ __forceinline__ Frag8<TYPE> usual(Frag8<TYPE> f) {
  if constexpr (TYPE == TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = unusual(f.v[e]) ? 0.0f : f.v[e];
  } else {
    uint32_t w[4] = {f.q.x, f.q.y, f.q.z, f.q.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] &= (unusual_half<TYPE>(w[e]) ? 0u : 0xffffu) | (unusual_half<TYPE>(w[e] >> 16) ? 0u : 0xffff0000u);
    f.q = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return f;
}

// ---- rows of a sequence ------------------------------------------------------------------------------------------------

// Where the next tile of a head begins: `left` rows of D values, `ld` apart (not above ROWS_LD)
constexpr long long ROWS_LD = 1 << 22;                 // a tile's offsets are below 2^31 bytes
template <int TYPE> struct Rows {
  typedef typename ElemOf<TYPE>::type E;
  const E *at;
  long long ld;
  int left, D;
  __device__ __forceinline__ Rows(const void *base, long long first, long long ld_, int left_, int D_)
      : at(static_cast<const E *>(base) + first), ld(ld_), left(left_), D(D_) {}
  __device__ __forceinline__ void skip(int rows) { at += rows * ld; left -= rows; }
  // Bytes of `rows` rows at most: the machine gives zeros beyond them (ld >= D, so no later row begins before the last one's end)
  __device__ __forceinline__ int bytes(int rows) const {
    const int n = min(left, rows);
    return n > 0 ? (int)(((n - 1) * (int)ld + D) * sizeof(E)) : 0;
  }
};

// 16 bytes of a run of `bytes` bytes, zeros beyond it: into registers, and (a wavefront's 1 KB) into LDS.  The run is the same for all lanes.
__device__ __forceinline__ uint4 run_load(const void *run, int bytes, uint32_t offset) {
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(run), 0, bytes, 0x00020000);
  return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, offset, 0, 0));
}
__device__ __forceinline__ void run_fetch(const void *run, int bytes, uint32_t offset, void *lds) {
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(run), 0, bytes, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void *)lds, 16, offset, 0, 0, 0);
}

// ---- operand tiles in LDS ----------------------------------------------------------------------------------------------

// ROWS rows of 32 ND values.  16-bit: rows of 4, 8 or 16 chunks of 16 bytes, whose places are exchanged by an XOR of the row so that neither reads
// of 16 rows' same chunk nor transposing reads of four rows' four chunks meet in a bank.  fp32: rows four words apart from a multiple of 64.
template <int TYPE, int ROWS, int ND, int THREADS = 256> struct Tile {
  typedef typename ElemOf<TYPE>::type E;
  typedef Frag8<TYPE> Frag;
  static constexpr int WIDTH = ND;
  static constexpr int CH = ND == 1 ? 4 : ND == 2 ? 8 : 16;          // chunks of a row, of which 4 ND hold values
  static constexpr int PER = TYPE == TYPE_F32 ? 4 : 8;               // values of a 16-byte vector
  static constexpr int LD = TYPE == TYPE_F32 ? ((32 * ND + 63) / 64 * 64 + 4) : CH * 8;
  static constexpr int ELEMS = ROWS * LD;
  static constexpr int VECS = ROWS * 32 * ND / PER;                  // vectors of the tile
  static constexpr int NV = (VECS + THREADS - 1) / THREADS;          // of a thread (THREADS share a tile)

  static __device__ __forceinline__ int swizzle(int row) {
    return CH == 16 ? 4 * (row & 3) | (row >> 2 & 3) : CH == 8 ? 4 * (row >> 1 & 1) | (row >> 2 & 3) : row >> 2 & 3;
  }
  static __device__ __forceinline__ int place(int row, int chunk) {  // of vector `chunk` of a row, in values
    return TYPE == TYPE_F32 ? row * LD + chunk * 4 : row * LD + (chunk ^ swizzle(row)) * 8;
  }

  // A thread's part of the tile's rows, from the next row of a sequence (Rows): zeros beyond the sequence and beyond D
  uint4 q[NV];
  template <bool VEC> __device__ __forceinline__ void load(const Rows<TYPE> &m) {
    const int bytes = m.bytes(ROWS);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = threadIdx.x % THREADS + i * THREADS, row = c / (32 * ND / PER), col = c % (32 * ND / PER) * PER;
      const bool there = col < m.D && (VECS % THREADS == 0 || row < ROWS);
      if constexpr (VEC) {
        q[i] = run_load(m.at, bytes, there ? (uint32_t)(row * (int)m.ld + col) * sizeof(E) : OOB);
      } else {
        const bool in = there && row < m.left;
        const uint4 w = load16<sizeof(E), false>(m.at, in ? row * m.ld : 0, in ? col : 0, m.D);
        q[i] = make_uint4(in ? w.x : 0u, in ? w.y : 0u, in ? w.z : 0u, in ? w.w : 0u);
      }
    }
  }
  __device__ __forceinline__ void store(E *lds) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = threadIdx.x % THREADS + i * THREADS, row = c / (32 * ND / PER), chunk = c % (32 * ND / PER);
      if (VECS % THREADS == 0 || row < ROWS) *reinterpret_cast<uint4 *>(lds + place(row, chunk)) = q[i];
    }
  }
  // The same straight into LDS, 1 KB to a wavefront's load: a lane's place is given, so it fetches the chunk that belongs there
  static constexpr bool DIRECT = TYPE != TYPE_F32 && ROWS * CH >= THREADS;
  static constexpr int ND_LOADS = DIRECT ? ROWS * CH / THREADS : 1;
  uint32_t offset[ND_LOADS];                                         // a lane's chunk of each, in bytes
  __device__ __forceinline__ void place_loads(long long ld, int D) {
#pragma unroll
    for (int i = 0; i < ND_LOADS; ++i) {
      const int c = (threadIdx.x % THREADS / 64 * ND_LOADS + i) * 64 + (threadIdx.x & 63), row = c / CH, col = ((c % CH) ^ swizzle(row)) * 8;
      offset[i] = col < D ? (uint32_t)(row * (int)ld + col) * 2u : OOB;
    }
  }
  __device__ __forceinline__ void fetch(E *lds, const Rows<TYPE> &m) const {
    const int bytes = m.bytes(ROWS);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x % THREADS / 64);
#pragma unroll
    for (int i = 0; i < ND_LOADS; ++i)
      run_fetch(m.at, bytes, offset[i], lds + (wave * ND_LOADS + i) * 512);
  }
  // Are there infinities or NaN in rows row0 .. row0 + 31?  (A wavefront looks, all lanes learn.)
  static __device__ __forceinline__ bool any(const E *lds, int row0) {
    uint32_t signs = 0;
#pragma unroll
    for (int i = 0; i < 16 * ND / PER; ++i) {
      const int c = (threadIdx.x & 63) + i * 64;
      signs |= unusual_signs<TYPE>(*reinterpret_cast<const uint4 *>(lds + place(row0 + c / (32 * ND / PER), c % (32 * ND / PER))));
    }
    return __any((signs & (TYPE == TYPE_F32 ? 0x80000000u : 0x80008000u)) != 0);
  }

  // Fragment of rows row0 .. row0 + 31 for step k of the values (16 k ..)
  static __device__ __forceinline__ Frag8<TYPE> rows(const E *lds, int row0, int k) {
    const int lane = threadIdx.x & 63, row = row0 + (lane & 31), h = lane >> 5;
    Frag8<TYPE> f;
    if constexpr (TYPE == TYPE_F32) {
      const float4 a = *reinterpret_cast<const float4 *>(lds + place(row, 4 * k + 2 * h)), b = *reinterpret_cast<const float4 *>(lds + place(row, 4 * k + 2 * h + 1));
      f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w; f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    } else {
      f.q = *reinterpret_cast<const uint4 *>(lds + place(row, 2 * k + h));
    }
    return f;
  }
  // Transposed: of values 32 d .. 32 d + 31 as rows and the tile's rows row0 + 8 (e / 4) + 4 (lane >> 5) + e % 4 as the reduction's places
  static __device__ __forceinline__ Frag8<TYPE> cols(const E *lds, int row0, int d) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    Frag8<TYPE> f;
    if constexpr (TYPE == TYPE_F32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f.v[e] = lds[(row0 + 8 * (e >> 2) + 4 * h + (e & 3)) * LD + 32 * d + (lane & 31)];
    } else {
      // a transposing read: lane i of 16 names four values of one row, and gets one value of each of four rows
      const int i16 = lane & 15, col = 32 * d + (lane >> 4 & 1) * 16 + 4 * (i16 & 3), row = row0 + 4 * h + (i16 >> 2);
      const E *a = lds + place(row, col >> 3) + (col & 7), *b = lds + place(row + 8, col >> 3) + (col & 7);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(a));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(b));
      f.q = __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    return f;
  }
  static __device__ __forceinline__ float value(const E *lds, int row, int col) {
    const E v = lds[place(row, col / PER) + col % PER];
    if constexpr (TYPE == TYPE_F32) return v;
    else return TYPE == TYPE_BF16 ? bf2f(v) : f16_val(v);
  }
};

// Every thread's part of the next tile is in LDS, and nobody reads the present one any more
template <bool DIRECT> __device__ __forceinline__ void arrived() {
  if (DIRECT) wait_vmcnt<0>();
  __syncthreads();
}

// The fragment of one row of memory for step k: the row's values 16 k + 8 (lane >> 5) + e; zeros where there is no row, and beyond D
template <int TYPE, bool VEC>
__device__ __forceinline__ Frag8<TYPE> row_frag(const void *base, long long at, bool in, int k, int D) {
  typedef typename ElemOf<TYPE>::type E;
  const int col = 16 * k + 8 * (threadIdx.x >> 5 & 1);
  Frag8<TYPE> f;
  if constexpr (TYPE == TYPE_F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool ok = in && col + 4 * h < D;
      const uint4 w = load16<4, VEC>(base, ok ? at : 0, ok ? col + 4 * h : 0, D);
      f.v[4 * h] = ok ? __uint_as_float(w.x) : 0.0f; f.v[4 * h + 1] = ok ? __uint_as_float(w.y) : 0.0f;
      f.v[4 * h + 2] = ok ? __uint_as_float(w.z) : 0.0f; f.v[4 * h + 3] = ok ? __uint_as_float(w.w) : 0.0f;
    }
  } else {
    const bool ok = in && col < D;
    const uint4 w = load16<2, VEC>(base, ok ? at : 0, ok ? col : 0, D);
    f.q = make_uint4(ok ? w.x : 0u, ok ? w.y : 0u, ok ? w.z : 0u, ok ? w.w : 0u);
  }
  return f;
}

// Reads and products in groups: left to itself the compiler puts each read in front of the product that takes it and waits for it there (gradients of
// 32768 packed rows, 16 heads of 64: 651 us, so 621; with heads of more than 64 values the forward and the pass over queries have no registers for it, the
// pass over keys, one wavefront to a SIMD there, has).  Nothing crosses the line.
__device__ __forceinline__ void group_ends() { __builtin_amdgcn_sched_barrier(0); }

template <class T> __device__ __forceinline__ void read_rows(typename T::Frag (&f)[2 * T::WIDTH], const typename T::E *lds, int row0) {
#pragma unroll
  for (int i = 0; i < 2 * T::WIDTH; ++i) f[i] = T::rows(lds, row0, i);
}
template <class T> __device__ __forceinline__ void read_cols(typename T::Frag (&f)[2][T::WIDTH], const typename T::E *lds, int row0) {
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int d = 0; d < T::WIDTH; ++d) f[b][d] = T::cols(lds, row0 + 16 * b, d);
}
// acc[d] += sum over 32 rows of (row, place) X^T Y: the two fragments of x have the rows as the reduction's places
template <bool CLEAN, int TYPE, int ND>
__device__ __forceinline__ void add_cols(f32x16 (&acc)[ND], const Frag8<TYPE> (&f)[2][ND], const Frag8<TYPE> (&x)[2]) {
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int d = 0; d < ND; ++d) mma<TYPE>(acc[d], CLEAN ? usual<TYPE>(f[b][d]) : f[b][d], x[b]);
}
// What add_cols left out with CLEAN: infinities and NaN of the tile's rows row0 .. row0 + 31, in the columns of acc (the lane's own) that the mask
// leaves to them.  They count as they are: weights are positive or make them NaN.
template <class T, class F>
__device__ __forceinline__ void add_unusual(f32x16 (&acc)[T::WIDTH], const typename T::E *lds, int row0, F &&sees) {
  const int h = threadIdx.x >> 5 & 1;
  for (int r = 0; r < 32; ++r) {
    if (!sees(r)) continue;
#pragma unroll
    for (int d = 0; d < T::WIDTH; ++d) {
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float v = T::value(lds, row0 + r, 32 * d + 8 * (k >> 2) + 4 * h + (k & 3));
        if (unusual(v)) acc[d][k] += v;
      }
      __builtin_amdgcn_sched_barrier(0);               // (no more than these in registers)
    }
  }
}

// Results to memory: the lane's row of D values from acc (its column), times `by`
template <int TYPE, int ND, bool VEC>
__device__ __forceinline__ void store_row(void *base, long long at, const f32x16 (&acc)[ND], float by, int D) {
  const int h = threadIdx.x >> 5 & 1;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = 32 * d + 8 * k + 4 * h;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[d][4 * k + e] * by;
      if (VEC) {
        if (col >= D) continue;
        if constexpr (TYPE == TYPE_F32) {
          *reinterpret_cast<float4 *>(static_cast<float *>(base) + at + col) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
          const uint32_t lo = TYPE == TYPE_BF16 ? pack2bf(v[0], v[1]) : (uint32_t)f16_bits(v[0]) | ((uint32_t)f16_bits(v[1]) << 16);
          const uint32_t hi = TYPE == TYPE_BF16 ? pack2bf(v[2], v[3]) : (uint32_t)f16_bits(v[2]) | ((uint32_t)f16_bits(v[3]) << 16);
          *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(base) + at + col) = make_uint2(lo, hi);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + e < D) store_from_f32(base, TYPE, at + col + e, v[e]);
      }
    }
}

// ---- sequences -------------------------------------------------------------------------------------------------------

struct Span { long long start; int len; };             // rows of a sequence

// The s-th sequence: between its offsets, brought into [0, rows] (a list that does not rise gives empty sequences, never rows outside)
__device__ __forceinline__ Span span_of(const AttentionP &p, int s) {
  if (!p.offsets) return {(long long)s * p.T, p.T};
  long long a, b;
  if (p.wide) { a = static_cast<const long long *>(p.offsets)[s]; b = static_cast<const long long *>(p.offsets)[s + 1]; }
  else { a = static_cast<const int *>(p.offsets)[s]; b = static_cast<const int *>(p.offsets)[s + 1]; }
  a = max(0LL, min(a, p.rows));
  b = max(a, min(b, p.rows));
  return {a, (int)(b - a)};
}

// A sequence's tile by its level, 1 .. tiles: the level-th tile of queries, the level-th of keys from the end.  Both have work for about `level` tiles.
struct Work { long long start; int len, tiles, level; };      // level 0: none

// The t-th tile of `size` rows of all sequences: the longest sequence first, so that what comes last is short, and of each the highest levels first, one
// after the other, so that blocks of one time share keys in their L2 (in the order of levels over all sequences the pass over queries of 40 sequences of
// 15 to 4211 rows took 289 us, so 245).  Every lane of a wavefront asks for the same t.  With more than 64 sequences p.list holds sequence and level of
// each (attention_tiles_kernel).
__device__ __forceinline__ Work find_tile(const AttentionP &p, int t, int size) {
  if (!p.offsets) {
    const int tiles = (p.T + size - 1) / size, s = t / tiles;
    if (s >= p.seqs) return {0, 0, 0, 0};
    return {(long long)s * p.T, p.T, tiles, tiles - (t - s * tiles)};
  }
  if (p.seqs > 64) {
    if (t >= p.list[0].x) return {0, 0, 0, 0};
    const int2 e = p.list[1 + t];
    const Span at = span_of(p, e.x);
    return {at.start, at.len, (at.len + size - 1) / size, e.y};
  }
  // lane: a sequence, its tiles, and those of longer ones (of as long ones before it)
  const int lane = threadIdx.x & 63;
  const Span mine = lane < p.seqs ? span_of(p, lane) : Span{0, 0};
  const int n = (mine.len + size - 1) / size;
  int before = 0;
  for (int s = 0; s < p.seqs; ++s) {
    const int other = __builtin_amdgcn_readlane(n, s);
    before += other > n || (other == n && s < lane) ? other : 0;
  }
  const uint64_t here = __ballot(before <= t && t < before + n);
  if (!here) return {0, 0, 0, 0};
  const int s = __ffsll((unsigned long long)here) - 1, tiles = __builtin_amdgcn_readlane(n, s);
  const Span at = span_of(p, s);
  return {at.start, at.len, tiles, tiles - (t - __builtin_amdgcn_readlane(before, s))};
}

// Heads and tiles of a block: neighbouring heads share keys and values, so they go to one XCD (blocks are dealt to the eight in turn)
__device__ __forceinline__ void head_and_tile(int block, int heads, int &head, int &tile) {
  if (heads % 8 == 0) {
    const int each = heads / 8, r = block / 8;
    head = block % 8 * each + r % each;
    tile = r / each;
  } else {
    head = block % heads;
    tile = block / heads;
  }
}

// Zeros in rows before the first and behind the last sequence: `part` of `parts` blocks
__device__ __forceinline__ void zero_rest(const AttentionP &p, void *out, int type, int heads, long long ld, long long sh, float *lse, int part, int parts) {
  const Span first = span_of(p, 0), last = span_of(p, p.seqs - 1);
  const long long head = first.start, from = last.start + last.len, n = head + max(0LL, p.rows - from), D = p.D;
  for (long long i = (long long)part * blockDim.x + threadIdx.x; i < n * heads * D; i += (long long)parts * blockDim.x) {
    const long long r = i / (heads * D), rest = i - r * heads * D, h = rest / D, row = r < head ? r : from + (r - head);
    store_from_f32(out, type, row * ld + h * sh + (rest - h * D), 0.0f);
  }
  if (lse)
    for (long long i = (long long)part * blockDim.x + threadIdx.x; i < n * heads; i += (long long)parts * blockDim.x) {
      const long long h = i / n, r = i - h * n;
      lse[h * p.rows + (r < head ? r : from + (r - head))] = 0.0f;
    }
}
constexpr int REST_BLOCKS = 64;

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

// rows that 16-byte loads may take
inline bool attention_vectors(const void *t, int type, long long head, long long ld, int D) { return ld <= ROWS_LD && rows_of_vectors(t, type, head, ld, D); }

}  // namespace
}  // namespace absk
