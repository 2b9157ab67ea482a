// Causal attention over packed sequences with grouped heads, forward.
//
//   s_ij = a q_i . k_j for j <= i of one sequence,   o_i = sum_j softmax(s_i)_j v_j,   lse_i = log sum_j exp s_ij
//
// One pass over the keys with the running maximum and sum of the softmax.  A block takes 128 queries of a head, 32 to a wavefront, and goes through
// the keys in tiles of 64 (fp32 32) that it shares, two in LDS, the next one on its way.  S^T = K Q^T, so that a query is a lane's column: its maximum needs
// one exchange between the two halves of a wavefront, its sum none until the end, and exp(S^T) is, rounded, the operand of O^T += V^T P^T without leaving
// the registers.  Tiles below the diagonal run in a loop without masks; a wavefront masks the one that its diagonal runs through.  The weights are rounded
// to the operands' type since the matrix cores take two operands of one type: with bf16 o is off by 2.0e-3 of its norm, where a result of fp32 weights,
// rounded once, is by 1.5e-3.
//
// Bound by the matrix cores together with the exponentials: one sequence of 16384, 16 heads of 128 over 4 973 to 1020 us on different cards, 1.13 to 1.08 PFLOP/s,
// where the matrix cores are busy 61 % of the time and a library's product of 16384^3 reaches 1.35, with its second operand transposed 1.60; 16 heads of
// 64, one sequence of 8192: 174 to 179 us, 0.78.  Each 1 KB fragment from LDS feeds one product (1.4 to 2.1 LDS instructions to an MFMA here and in the
// gradients).
#include <algorithm>
#include "attention_parts.h"

namespace absk {
namespace {

// Sequence and level of every tile, those of the longest sequences first, for more than 64 sequences: list[0].x of them from list[1] on.  Sequences of about
// the same number of tiles share one of 1024 places, in an order that may differ from run to run (nothing that is computed depends on it).
// Offsets that are no list may ask for far more tiles than there is room for, up to rows / 128 in every sequence: places are counted in 64 bits.
__global__ void __launch_bounds__(1024) attention_tiles_kernel(const AttentionP p, int2 *list, const int size) {
  constexpr int PLACES = 1024, ALONE = 32;
  __shared__ unsigned long long place[PLACES], sums[16];
  __shared__ int most;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  place[threadIdx.x] = 0;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  auto tiles_of = [&](int s) { return s < p.seqs ? (span_of(p, s).len + size - 1) / size : 0; };
  int n = 0;
  for (int s = threadIdx.x; s < p.seqs; s += 1024) n = max(n, tiles_of(s));
  atomicMax(&most, n);
  __syncthreads();
  const int unit = max(1, (most + PLACES - 1) / PLACES);
  for (int s = threadIdx.x; s < p.seqs; s += 1024) {
    const int mine = tiles_of(s);
    if (mine) atomicAdd(&place[PLACES - 1 - (mine - 1) / unit], (unsigned long long)mine);
  }
  __syncthreads();
  const unsigned long long count = place[threadIdx.x];
  unsigned long long upto = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += sums[w];
  place[threadIdx.x] = upto - count;
  const long long room = attention_tiles(p);           // (fits an int: a grid counts as many blocks)
  if (threadIdx.x == PLACES - 1) list[0] = make_int2((int)min((long long)upto, room), 0);
  __syncthreads();
  // a lane writes the first tiles of its sequence, a wavefront the others of each that has more
  for (int s0 = wave * 64; s0 < p.seqs; s0 += 1024) {
    const int mine = tiles_of(s0 + lane);
    const long long at = mine ? (long long)atomicAdd(&place[PLACES - 1 - (mine - 1) / unit], (unsigned long long)mine) : 0;
    const int here = (int)max(0LL, min((long long)mine, room - at));
    for (int i = 0; i < min(here, ALONE); ++i) list[1 + at + i] = make_int2(s0 + lane, mine - i);
    for (uint64_t m = __ballot(here > ALONE); m; m &= m - 1) {
      const int from = __ffsll((unsigned long long)m) - 1, all = __shfl(mine, from, 64), upto_room = __shfl(here, from, 64);
      const long long first = __shfl(at, from, 64);
      for (int i = ALONE + lane; i < upto_room; i += 64) list[1 + first + i] = make_int2(s0 + from, all - i);
    }
  }
}

// fp16 weights are held times 2^7: at most 2^8 of the reference, they stay below 65504, and those below 2^-14 of it, of which a long row has most, keep
// seven more bits.  Sums are of the same weights; lse is corrected, o divided by the sum.
template <int TYPE> constexpr float WEIGHT_SHIFT = TYPE == TYPE_F16 ? 7.0f : 0.0f;

template <int TYPE, int ND, bool VEC>
__global__ void __launch_bounds__(256, 2) attention_kernel(const AttentionP p, const int blocks) {
  constexpr int BK = TYPE == TYPE_F32 ? 32 : 64, NB = BK / 32;
  typedef Tile<TYPE, BK, ND> KV;
  typedef typename KV::E E;
  constexpr bool DIRECT = VEC && KV::DIRECT, GROUPED = TYPE != TYPE_F32 && ND <= 2;      // (wider heads have no registers for it)
  constexpr int KSTEPS = 2 * ND % 4 == 0 ? 4 : 2;      // of a group of reads
  // two buffers, by name, so that the compiler can tell what is read from what is on its way
  __shared__ __attribute__((aligned(16))) E keys_a[KV::ELEMS], values_a[KV::ELEMS], keys_b[KV::ELEMS], values_b[KV::ELEMS];
  if ((int)blockIdx.x >= blocks) return zero_rest(p, p.o, TYPE, p.Hq, p.ldo, p.ho, p.lse, blockIdx.x - blocks, REST_BLOCKS);
  int head, t;
  head_and_tile(blockIdx.x, p.Hq, head, t);
  const Work w = find_tile(p, t, ATTENTION_ROWS);
  if (!w.level) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const int q0 = (w.level - 1) * ATTENTION_ROWS, mine = q0 + wave * 32, row = mine + (lane & 31);
  const bool in = row < w.len;
  const int kvh = head / (p.Hq / p.Hkv);
  const E *q = static_cast<const E *>(p.q) + w.start * p.ldq + head * p.hq;
  Frag8<TYPE> qf[2 * ND];
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) qf[i] = row_frag<TYPE, VEC>(q, (long long)row * p.ldq, in, i, p.D);
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros16();
  float top = -__builtin_inff(), sum = 0.0f;
  const float c = p.scale * LOG2E;
  const int end = min(w.len, q0 + ATTENTION_ROWS), tiles = (end + BK - 1) / BK;
  Rows<TYPE> rk(p.k, w.start * p.ldk + kvh * p.hk, p.ldk, w.len, p.D), rv(p.v, w.start * p.ldv + kvh * p.hv, p.ldv, w.len, p.D);
  KV tk, tv;
  if constexpr (DIRECT) {
    tk.place_loads(p.ldk, p.D);
    tv.place_loads(p.ldv, p.D);
  }
  auto fetch = [&](auto buffer) INLINE {                      // the next tile
    if constexpr (DIRECT) {
      tk.fetch(decltype(buffer)::value ? keys_b : keys_a, rk);
      tv.fetch(decltype(buffer)::value ? values_b : values_a, rv);
    } else {
      tk.template load<VEC>(rk);
      tv.template load<VEC>(rv);
    }
    rk.skip(BK);
    rv.skip(BK);
  };
  auto settle = [&](auto buffer) INLINE {
    if constexpr (!DIRECT) {
      tk.store(decltype(buffer)::value ? keys_b : keys_a);
      tv.store(decltype(buffer)::value ? values_b : values_a);
    }
  };
  // MASKED: the diagonal may run through the tile
  auto step = [&](int k0, auto buffer, auto masked_tile) INLINE {
    constexpr bool MASKED = decltype(masked_tile)::value;
    const E *lk = decltype(buffer)::value ? keys_b : keys_a, *lv = decltype(buffer)::value ? values_b : values_a;
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = zeros16();
#pragma unroll
    for (int i0 = 0; i0 < 2 * ND; i0 += KSTEPS) {
      Frag8<TYPE> f[NB][KSTEPS];
#pragma unroll
      for (int i = 0; i < KSTEPS; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) f[b][i] = KV::rows(lk, 32 * b, i0 + i);
      if (GROUPED) group_ends();
#pragma unroll
      for (int i = 0; i < KSTEPS; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) mma<TYPE>(s[b], f[b][i], qf[i0 + i]);
      if (GROUPED) group_ends();
    }
    if (MASKED) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + 32 * b + 8 * (r >> 2) + 4 * h + (r & 3) > row) s[b][r] = -__builtin_inff();
    }
    float most = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) most = fmaxf(most, s[b][r]);
    most = fmaxf(most, __shfl_xor(most, 32, 64)) * c;
    // A row's reference follows its maximum only when that is 2^8 beyond it (whatever other rows' do): results are the same, what is summed
    // stays below 2^8 times the number of keys
    if (__any(most > top + 8.0f)) {
      const float next = most > top + 8.0f ? most : top, by = __builtin_amdgcn_exp2f(top - (next == -__builtin_inff() ? 0.0f : next));
      top = next;
      sum *= by;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= by;
    }
    const float ref = (top == -__builtin_inff() ? 0.0f : top) - WEIGHT_SHIFT<TYPE>;
    Frag8<TYPE> x[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -ref));
        sum += s[b][r];
      }
      x[b][0] = as_frag<TYPE>(s[b], 0);
      x[b][1] = as_frag<TYPE>(s[b], 1);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      Frag8<TYPE> vf[2][ND];
      read_cols<KV>(vf, lv, 32 * b);
      if (GROUPED) group_ends();
      add_cols<MASKED, TYPE, ND>(o, vf, x[b]);
      if (MASKED && KV::any(lv, 32 * b)) add_unusual<KV>(o, lv, 32 * b, [&](int r) { return k0 + 32 * b + r <= row; });
    }
  };
  int j = 0;
  const int whole = q0 / BK;                           // tiles below every wavefront's diagonal
  auto turn = [&](auto buffer, auto last_tiles) INLINE {
    constexpr bool LAST = decltype(last_tiles)::value;
    std::integral_constant<bool, !decltype(buffer)::value> other;
    const int k0 = j * BK;
    const bool more = !LAST || j + 1 < tiles;
    if (more) fetch(other);
    if (!LAST || (k0 <= mine + 31 && mine < w.len)) step(k0, buffer, last_tiles);
    if (more) settle(other);
    arrived<DIRECT>();
    ++j;
  };
  const std::false_type a, below;
  const std::true_type b, last;
  fetch(a);
  settle(a);
  arrived<DIRECT>();
  while (j + 2 <= whole) {
    turn(a, below);
    turn(b, below);
  }
  if (j < whole) turn(a, below);
  while (j < tiles) {
    if (j & 1) turn(b, last);
    else turn(a, last);
  }
  sum += __shfl_xor(sum, 32, 64);
  if (!in) return;
  store_row<TYPE, ND, VEC>(static_cast<E *>(p.o) + w.start * p.ldo + head * p.ho, (long long)row * p.ldo, o, 1.0f / sum, p.D);
  if (p.lse && h == 0) p.lse[head * p.rows + w.start + row] = (top - WEIGHT_SHIFT<TYPE> + __builtin_amdgcn_logf(sum)) * LN2;
}

template <int TYPE, int ND, bool VEC> hipError_t forward_launch(const AttentionP &p, hipStream_t s) {
  const long long blocks = attention_tiles(p) * p.Hq, rest = p.offsets && p.zero_rest ? REST_BLOCKS : 0;
  hipLaunchKernelGGL((attention_kernel<TYPE, ND, VEC>), dim3((unsigned)(blocks + rest)), dim3(256), 0, s, p, (int)blocks);
  return hipGetLastError();
}
template <int TYPE, bool VEC> hipError_t forward_width(const AttentionP &p, hipStream_t s) {
  switch ((p.D + 31) / 32) {
    case 1: return forward_launch<TYPE, 1, VEC>(p, s);
    case 2: return forward_launch<TYPE, 2, VEC>(p, s);
    case 3: return forward_launch<TYPE, 3, VEC>(p, s);
    default: return forward_launch<TYPE, 4, VEC>(p, s);
  }
}

}  // namespace

hipError_t launch_attention_tiles(const AttentionP &p, hipStream_t s) {
  if (!p.offsets || p.seqs <= 64) return hipSuccess;
  hipLaunchKernelGGL(attention_tiles_kernel, dim3(1), dim3(1024), 0, s, p, const_cast<int2 *>(p.list), ATTENTION_ROWS);
  return hipGetLastError();
}

hipError_t launch_attention(const AttentionP &p, hipStream_t s) {
  const hipError_t e = launch_attention_tiles(p, s);
  if (e != hipSuccess) return e;
  const bool vec = attention_vectors(p.q, p.type, p.hq, p.ldq, p.D) && attention_vectors(p.k, p.type, p.hk, p.ldk, p.D) &&
                   attention_vectors(p.v, p.type, p.hv, p.ldv, p.D) && attention_vectors(p.o, p.type, p.ho, p.ldo, p.D);
  switch (p.type) {
    case TYPE_F32: return vec ? forward_width<TYPE_F32, true>(p, s) : forward_width<TYPE_F32, false>(p, s);
    case TYPE_BF16: return vec ? forward_width<TYPE_BF16, true>(p, s) : forward_width<TYPE_BF16, false>(p, s);
    default: return vec ? forward_width<TYPE_F16, true>(p, s) : forward_width<TYPE_F16, false>(p, s);
  }
}

}  // namespace absk
