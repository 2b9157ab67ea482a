// Gradients of causal attention (attention.hip).
//
//   p_ij = exp(s_ij - lse_i),  D_i = do_i . o_i,  ds_ij = a p_ij (do_i . v_j - D_i)
//   dv_j = sum_i p_ij do_i,  dk_j = sum_i ds_ij q_i  (query heads that share the key head add up),  dq_i = sum_j ds_ij k_j
//
// Scores are formed again from q and k.  Two kernels, so that every sum has one owner and an order of its own (the same bits every time): one takes 128
// queries, 32 to a wavefront, and goes through their keys (and leaves D_i for the other); the other takes 64 keys and goes through the queries of all
// heads that share them.  Together seven products where one kernel would need five, but no sums of dq in memory by atomics.  Scores stay in registers: what
// is a result of the first products is, rounded, an operand of the second ones, whose other operand is read transposed from the tile that is in LDS anyway.
//
// Bound by the exponentials and what surrounds them beside the products, which the few wavefronts that fit overlap only in part: of five products 0.50
// PFLOP/s for 16 heads of 64 over 32768 rows in 40 sequences of 15 to 4211 (581 to 595 us: keys 345, queries 240), 0.56 for one sequence of 8192,
// 0.60 for heads of 128.  Matrix cores are busy 33 (keys) and 38 % of the time.
//
// p and ds are rounded to the operands' type since the matrix cores take two operands of one type: bf16 gradients are off by 2.4e-3 of their norm, where
// results of fp32 ones, rounded once, are by 1.7e-3; fp16 ones by 3.0e-4, where those are by 2.1e-4.
//
// fp16 operands hold p and ds in 16 bits with powers of two: p by 2^12 (else values below 2^-14, those of a row of many keys, lose bits), ds by the power that
// takes twice the largest |do_i| |v_j| of the sequence and heads in question, a bound on |ds / a|, to 2^14 at most.
#include <algorithm>
#include "attention_parts.h"

namespace absk {
namespace {

template <int TYPE> constexpr float P_SHIFT = TYPE == TYPE_F16 ? 12.0f : 0.0f;

// fp16: of every tile of 128 rows D_i of each query head, 16 lanes to a row, and the largest squared lengths of do_i and, further heads, of v_j
constexpr int INNER_ROWS = 4;                          // of a group under way
template <bool VEC>
__global__ void __launch_bounds__(256) attention_inner_kernel(const AttentionP p) {
  const int g = threadIdx.x / 16, l = threadIdx.x % 16, D = p.D, heads = p.Hq + p.Hkv, t = blockIdx.x / heads, head = blockIdx.x - t * heads;
  const Work w = find_tile(p, t, ATTENTION_ROWS);
  if (!w.level) return;
  const int r0 = (w.level - 1) * ATTENTION_ROWS, r1 = min(r0 + ATTENTION_ROWS, w.len);
  const bool of_v = head >= p.Hq;
  auto values = [&](const void *base, long long at, float (&v)[8]) INLINE {
    const uint4 q = load16<2, VEC>(base, at, l * 8, D);
    unpack8(q, TYPE_F16, v);
  };
  float longest = 0.0f;
  for (int r = r0 + g; r < r1; r += 16 * INNER_ROWS) {
    float a[INNER_ROWS][8], b[INNER_ROWS][8];
#pragma unroll
    for (int k = 0; k < INNER_ROWS; ++k) {             // (of the group's first row again where there are fewer)
      const long long row = w.start + (r + 16 * k < r1 ? r + 16 * k : r);
      if (of_v) {
        values(p.v, row * p.ldv + (head - p.Hq) * p.hv, a[k]);
      } else {
        values(p.dout, row * p.lddo + head * p.hdo, a[k]);
        values(p.o, row * p.ldo + head * p.ho, b[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < INNER_ROWS; ++k) {
      float s = 0.0f, n = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!of_v) s = fmaf(a[k][e], b[k][e], s);
        n = fmaf(a[k][e], a[k][e], n);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) { s += __shfl_xor(s, o, 16); n += __shfl_xor(n, o, 16); }
      if (!of_v && l == 0 && r + 16 * k < r1) p.inner[head * p.rows + w.start + r + 16 * k] = s;
      if (n < __builtin_inff()) longest = fmaxf(longest, n);
    }
  }
  __shared__ float sm[16];
  if (l == 0) sm[g] = longest;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 16; ++k) longest = fmaxf(longest, sm[k]);
    p.most[head * attention_tiles(p) + t] = longest;
  }
}

// The power of two that ds is held with, by the signals of `heads` heads from `head` on and the values of their keys' head in the sequence that has the t-th
// tile w: what other sequences and heads hold has no part in it
template <int TYPE> __device__ __forceinline__ float ds_factor(const AttentionP &p, const Work &w, int t, int head, int heads, int kvh) {
  if constexpr (TYPE != TYPE_F16) return 1.0f;
  const long long all = attention_tiles(p), first = t - (w.tiles - w.level);
  const int n = (int)min((long long)w.tiles, all - first);      // (offsets that are no list may name tiles that have no place)
  float a = 0.0f, b = 0.0f;
  for (int i = threadIdx.x & 63; i < n; i += 64) {
    for (int h = 0; h < heads; ++h) a = fmaxf(a, p.most[(head + h) * all + first + i]);
    b = fmaxf(b, p.most[(p.Hq + kvh) * all + first + i]);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { a = fmaxf(a, __shfl_xor(a, o, 64)); b = fmaxf(b, __shfl_xor(b, o, 64)); }
  const float bound = 2.0f * sqrtf(a) * sqrtf(b);
  if (!(bound > 0.0f)) return 1.0f;
  int e;
  (void)frexpf(bound, &e);                             // bound < 2^e
  return ldexpf(1.0f, max(-100, min(100, 14 - e)));
}

// Queries of a tile of the pass over keys
constexpr int keys_tile(int type, int nd) { return type == TYPE_F32 || nd >= 3 ? 32 : 64; }

// A block's wavefronts: two side by side, of 32 keys each, in two groups that go through the same keys' queries in turn and add up what they have at the end.
// Four side by side in one group made the longest block's work four times as long (16 heads over 4 of 64 values, 32768 rows in 40 sequences: 264 tiles of
// queries where the average of what a CU's wavefronts take is 115; one sequence of 8192, 16 heads of 128: 1752 us, so 1210), four in two groups left a CU one
// block, whose wavefronts wait for each other (the first of these 610 us, so 588).
constexpr int KEYS_WAVES = 2, KEYS_GROUPS = 2, KEYS_PARTS = ATTENTION_ROWS / (32 * KEYS_WAVES);

// dk and dv of 32 keys to a wavefront of a group
template <int TYPE, int ND, bool VEC>
__global__ void __launch_bounds__(64 * KEYS_WAVES * KEYS_GROUPS, ND >= 3 ? 1 : 2) attention_keys_kernel(const AttentionP p, const int blocks) {
  constexpr int BQ = keys_tile(TYPE, ND), GROUPS = KEYS_GROUPS, WAVES = KEYS_WAVES, THREADS = 64 * WAVES;
  typedef Tile<TYPE, BQ, ND, THREADS> T;
  typedef typename T::E E;
  constexpr bool DIRECT = VEC && T::DIRECT, GROUPED = TYPE != TYPE_F32;
  // two buffers, by name, so that the compiler can tell what is read from what is on its way
  __shared__ __attribute__((aligned(16))) E queries_a[GROUPS * T::ELEMS], signals_a[GROUPS * T::ELEMS], queries_b[GROUPS * T::ELEMS], signals_b[GROUPS * T::ELEMS];
  __shared__ __attribute__((aligned(16))) float stat_a[GROUPS][2][BQ], stat_b[GROUPS][2][BQ];      // lse (to base 2) and D of a tile's queries
  if ((int)blockIdx.x >= blocks) {
    zero_rest(p, p.dk, TYPE, p.Hkv, p.lddk, p.hdk, nullptr, blockIdx.x - blocks, REST_BLOCKS);
    return zero_rest(p, p.dv, TYPE, p.Hkv, p.lddv, p.hdv, nullptr, blockIdx.x - blocks, REST_BLOCKS);
  }
  int kvh, t;
  head_and_tile(blockIdx.x, p.Hkv, kvh, t);
  const Work w = find_tile(p, t / KEYS_PARTS, ATTENTION_ROWS);
  if (!w.level) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x % THREADS / 64, group = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS), h = lane >> 5;
  const int k0 = (w.tiles - w.level) * ATTENTION_ROWS + t % KEYS_PARTS * (32 * WAVES), mine = k0 + wave * 32, key = mine + (lane & 31), G = p.Hq / p.Hkv;
  const bool in = key < w.len;
  if (k0 >= w.len) return;
  const float f = ds_factor<TYPE>(p, w, t / KEYS_PARTS, kvh * G, G, kvh), g = f * __builtin_amdgcn_exp2f(-P_SHIFT<TYPE>);
  Frag8<TYPE> kf[2 * ND], vf[2 * ND];
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) {
    kf[i] = row_frag<TYPE, VEC>(p.k, (w.start + key) * p.ldk + kvh * p.hk, in, i, p.D);
    vf[i] = row_frag<TYPE, VEC>(p.v, (w.start + key) * p.ldv + kvh * p.hv, in, i, p.D);
  }
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dk[d] = dv[d] = zeros16();
  const float c = p.scale * LOG2E;
  // tiles of queries from the diagonal to the sequence's end, of one head after the other
  const int first = k0 / BQ, each = (w.len + BQ - 1) / BQ - first, total = each * G;
  T tq, td;
  float lse = 0.0f, inner = 0.0f;
  bool there = false;
  const int thread = threadIdx.x % THREADS;
  auto fetch = [&](auto buffer, int tile, int of) INLINE {    // of the of-th head
    const int r0 = (first + tile) * BQ, head = kvh * G + of;
    const Rows<TYPE> rq(p.q, (w.start + r0) * p.ldq + head * p.hq, p.ldq, w.len - r0, p.D);
    const Rows<TYPE> rd(p.dout, (w.start + r0) * p.lddo + head * p.hdo, p.lddo, w.len - r0, p.D);
    // (as they come: what is made of them here would be waited for here)
    const int r = r0 + thread % BQ;
    const long long at = head * p.rows + w.start + min(r, w.len - 1);
    there = r < w.len;
    lse = p.lse[at];
    inner = p.inner[at];
    if constexpr (DIRECT) {
      tq.fetch((decltype(buffer)::value ? queries_b : queries_a) + group * T::ELEMS, rq);
      td.fetch((decltype(buffer)::value ? signals_b : signals_a) + group * T::ELEMS, rd);
    } else {
      tq.template load<VEC>(rq);
      td.template load<VEC>(rd);
    }
  };
  auto settle = [&](auto buffer) INLINE {
    constexpr bool B = decltype(buffer)::value;
    if constexpr (!DIRECT) {
      tq.store((B ? queries_b : queries_a) + group * T::ELEMS);
      td.store((B ? signals_b : signals_a) + group * T::ELEMS);
    }
    if (thread < BQ) {
      (B ? stat_b : stat_a)[group][0][thread] = there ? lse * LOG2E - P_SHIFT<TYPE> : __builtin_inff();
      (B ? stat_b : stat_a)[group][1][thread] = there ? inner : 0.0f;
    }
  };
  bool odd = false;                                    // are there infinities or NaN in the wavefront's keys and values?
  // Queries q0 .. q0 + 31, block b of a tile; MASKED: perhaps the diagonal's, or the sequence's last
  auto step = [&](int q0, int b, auto buffer, auto masked_block) INLINE {
    constexpr bool MASKED = decltype(masked_block)::value, B = decltype(buffer)::value;
    const E *lq = (B ? queries_b : queries_a) + group * T::ELEMS, *ld = (B ? signals_b : signals_a) + group * T::ELEMS;
    const float(*stat)[BQ] = (B ? stat_b : stat_a)[group];
    f32x16 s = zeros16(), dp = zeros16();
    {
      Frag8<TYPE> fq[2 * ND], fd[2 * ND];
      read_rows<T>(fq, lq, 32 * b);
      read_rows<T>(fd, ld, 32 * b);
      if (GROUPED) group_ends();
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i) {
        mma<TYPE>(s, fq[i], kf[i]);
        mma<TYPE>(dp, fd[i], vf[i]);
      }
    }
    if (GROUPED) group_ends();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 l4 = *reinterpret_cast<const float4 *>(&stat[0][32 * b + 8 * k + 4 * h]);
      const float4 d4 = *reinterpret_cast<const float4 *>(&stat[1][32 * b + 8 * k + 4 * h]);
      const float l[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * k + e;
        float x = __builtin_amdgcn_exp2f(fmaf(s[r], c, -l[e])), y = TYPE == TYPE_F16 ? x * ((dp[r] - dd[e]) * g) : x * (dp[r] - dd[e]);
        if (MASKED && q0 + 8 * k + 4 * h + e < key) x = y = 0.0f;
        s[r] = x;
        dp[r] = y;
      }
    }
    if (MASKED && odd && q0 + 32 > w.len) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (q0 + 8 * (r >> 2) + 4 * h + (r & 3) >= w.len) s[r] = dp[r] = 0.0f;
    }
    const Frag8<TYPE> x[2] = {as_frag<TYPE>(s, 0), as_frag<TYPE>(s, 1)}, y[2] = {as_frag<TYPE>(dp, 0), as_frag<TYPE>(dp, 1)};
    Frag8<TYPE> cq[2][ND], cd[2][ND];
    if (GROUPED) group_ends();
    read_cols<T>(cd, ld, 32 * b);
    read_cols<T>(cq, lq, 32 * b);
    if (GROUPED) group_ends();
    add_cols<MASKED, TYPE, ND>(dv, cd, x);
    add_cols<MASKED, TYPE, ND>(dk, cq, y);
    if (MASKED && T::any(ld, 32 * b)) add_unusual<T>(dv, ld, 32 * b, [&](int r) { return q0 + r >= key; });
    if (MASKED && T::any(lq, 32 * b)) add_unusual<T>(dk, lq, 32 * b, [&](int r) { return q0 + r >= key; });
  };
  if constexpr (DIRECT) {
    tq.place_loads(p.ldq, p.D);
    td.place_loads(p.lddo, p.D);
  }
  const std::false_type a;
  const std::true_type b;
  const int rounds = (total + GROUPS - 1) / GROUPS;
  int it = 0, now = group % each, now_head = group / each;      // this group's tile: the now-th of a head, if that is one of the G
  int next = now, next_head = now_head;
  auto advance = [&](int &tile, int &of) INLINE {
    tile += GROUPS;
    while (tile >= each) { tile -= each; ++of; }
  };
  if (next_head < G) {
    fetch(a, next, next_head);
    settle(a);
  }
  // Rows beyond a sequence's end have weight 0, as their lse is infinite, but 0 times an infinite key makes NaN of it: where a wavefront has such keys or
  // values those rows are masked (in every block that ends a sequence: 300 sequences of 32768 rows 318 us, so 353)
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) odd |= any_unusual<TYPE>(kf[i]) || any_unusual<TYPE>(vf[i]);
  odd = __any(odd);
  arrived<DIRECT>();
  auto turn = [&](auto buffer) INLINE {
    std::integral_constant<bool, !decltype(buffer)::value> other;
    advance(next, next_head);
    const bool more = next_head < G;
    if (more) fetch(other, next, next_head);
    if (now_head < G && mine < w.len) {
      const int q0 = (first + now) * BQ;
      if (q0 > mine && q0 + BQ <= w.len) {
        constexpr int ONCE = BQ < 64 ? 1 : 2;
#pragma unroll 1
        for (int i = 0; i < BQ / 32; i += ONCE)
#pragma unroll
          for (int k = 0; k < ONCE; ++k) step(q0 + 32 * (i + k), i + k, buffer, std::false_type{});
      } else {
#pragma unroll 1
        for (int i = 0; i < BQ / 32; ++i)
          if (q0 + 32 * i >= mine && q0 + 32 * i < w.len) step(q0 + 32 * i, i, buffer, std::true_type{});
      }
    }
    if (more) settle(other);
    arrived<DIRECT>();
    now = next;
    now_head = next_head;
    ++it;
  };
  while (it < rounds) {
    turn(a);
    if (it < rounds) turn(b);
  }
  {                                                    // one group ends with dk, the other with dv
    constexpr int SIZE = WAVES * 64 * 16, HELD = (int)(GROUPS * T::ELEMS * sizeof(E) / (SIZE * 4));      // values of 32 columns, how many of these a tile's place holds
    static_assert(2 * HELD >= ND, "room for the exchange");
    const int at = wave * 64 * 16 + lane;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      float *const to = reinterpret_cast<float *>(group ? (d / HELD ? queries_b : queries_a) : (d / HELD ? signals_b : signals_a)) + d % HELD * SIZE;
#pragma unroll
      for (int r = 0; r < 16; ++r) to[at + r * 64] = group ? dk[d][r] : dv[d][r];
    }
    __syncthreads();
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const float *const from = reinterpret_cast<const float *>(group ? (d / HELD ? signals_b : signals_a) : (d / HELD ? queries_b : queries_a)) + d % HELD * SIZE;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (group) dv[d][r] += from[at + r * 64];
        else dk[d][r] += from[at + r * 64];
      }
    }
  }
  if (!in) return;
  if (!group) store_row<TYPE, ND, VEC>(p.dk, (w.start + key) * p.lddk + kvh * p.hdk, dk, p.scale / f, p.D);
  else store_row<TYPE, ND, VEC>(p.dv, (w.start + key) * p.lddv + kvh * p.hdv, dv, __builtin_amdgcn_exp2f(-P_SHIFT<TYPE>), p.D);
}

// dq of 128 queries of a head
template <int TYPE, int ND, bool VEC>
__global__ void __launch_bounds__(256, TYPE == TYPE_F32 && ND >= 3 ? 1 : ND <= 2 && TYPE != TYPE_F32 ? 3 : 2) attention_queries_kernel(const AttentionP p, const int blocks) {
  constexpr int BK = TYPE == TYPE_F32 ? 32 : 64;
  typedef Tile<TYPE, BK, ND> T;
  typedef typename T::E E;
  constexpr bool DIRECT = VEC && T::DIRECT, GROUPED = TYPE != TYPE_F32 && ND <= 2;      // (wider heads have no registers for it)
  __shared__ __attribute__((aligned(16))) E keys_a[T::ELEMS], values_a[T::ELEMS], keys_b[T::ELEMS], values_b[T::ELEMS];
  if ((int)blockIdx.x >= blocks) return zero_rest(p, p.dq, TYPE, p.Hq, p.lddq, p.hdq, nullptr, blockIdx.x - blocks, REST_BLOCKS);
  int head, t;
  head_and_tile(blockIdx.x, p.Hq, head, t);
  const Work w = find_tile(p, t, ATTENTION_ROWS);
  if (!w.level) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const int q0 = (w.level - 1) * ATTENTION_ROWS, mine = q0 + wave * 32, row = mine + (lane & 31);
  const bool in = row < w.len;
  const int kvh = head / (p.Hq / p.Hkv);
  const float f = ds_factor<TYPE>(p, w, t, head, 1, kvh);
  Frag8<TYPE> qf[2 * ND], of[2 * ND];
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) {
    qf[i] = row_frag<TYPE, VEC>(p.q, (w.start + row) * p.ldq + head * p.hq, in, i, p.D);
    of[i] = row_frag<TYPE, VEC>(p.dout, (w.start + row) * p.lddo + head * p.hdo, in, i, p.D);
  }
  const long long at = head * p.rows + w.start + (in ? row : 0);
  const float lse = in ? p.lse[at] * LOG2E : __builtin_inff(), c = p.scale * LOG2E;
  // D_i, for the pass over keys too, which comes behind (of fp16 operands it is there already, for the power of two)
  float inner = 0.0f;
  if constexpr (TYPE == TYPE_F16) {
    inner = in ? p.inner[at] : 0.0f;
  } else {
#pragma unroll
    for (int i = 0; i < 2 * ND; ++i) {
      float a[8], b[8];
      frag_values<TYPE>(of[i], a);
      frag_values<TYPE>(row_frag<TYPE, VEC>(p.o, (w.start + row) * p.ldo + head * p.ho, in, i, p.D), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) inner = fmaf(a[e], b[e], inner);
    }
    inner += __shfl_xor(inner, 32, 64);
    if (in && h == 0) p.inner[at] = inner;
  }
  f32x16 dq[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dq[d] = zeros16();
  const int end = min(w.len, q0 + ATTENTION_ROWS), tiles = (end + BK - 1) / BK;
  Rows<TYPE> rk(p.k, w.start * p.ldk + kvh * p.hk, p.ldk, w.len, p.D), rv(p.v, w.start * p.ldv + kvh * p.hv, p.ldv, w.len, p.D);
  T tk, tv;
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
  // Keys kb .. kb + 31, block b of a tile; MASKED: perhaps the diagonal's
  auto step = [&](int kb, int b, auto buffer, auto masked_block) INLINE {
    constexpr bool MASKED = decltype(masked_block)::value;
    const E *lk = decltype(buffer)::value ? keys_b : keys_a, *lv = decltype(buffer)::value ? values_b : values_a;
    f32x16 s = zeros16(), dp = zeros16();
    {
      Frag8<TYPE> f[2 * ND];
      read_rows<T>(f, lk, 32 * b);
      if (GROUPED) group_ends();
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i) mma<TYPE>(s, f[i], qf[i]);
      if (GROUPED) group_ends();
      read_rows<T>(f, lv, 32 * b);
      if (GROUPED) group_ends();
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i) mma<TYPE>(dp, f[i], of[i]);
    }
    if (GROUPED) group_ends();
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse));
        dp[r] = TYPE == TYPE_F16 ? x * ((dp[r] - inner) * f) : x * (dp[r] - inner);
        if (MASKED && kb + 8 * (r >> 2) + 4 * h + (r & 3) > row) dp[r] = 0.0f;
      }
    const Frag8<TYPE> y[2] = {as_frag<TYPE>(dp, 0), as_frag<TYPE>(dp, 1)};
    Frag8<TYPE> ck[2][ND];
    if (GROUPED) group_ends();
    read_cols<T>(ck, lk, 32 * b);
    if (GROUPED) group_ends();
    add_cols<MASKED, TYPE, ND>(dq, ck, y);
    if (MASKED && T::any(lk, 32 * b)) add_unusual<T>(dq, lk, 32 * b, [&](int r) { return kb + r <= row; });
  };
  int j = 0;
  const int whole = q0 / BK;                           // tiles below every wavefront's diagonal
  auto turn = [&](auto buffer, auto last_tiles) INLINE {
    constexpr bool LAST = decltype(last_tiles)::value;
    std::integral_constant<bool, !decltype(buffer)::value> other;
    const bool more = !LAST || j + 1 < tiles;
    if (more) fetch(other);
    if constexpr (!LAST) {
#pragma unroll
      for (int i = 0; i < BK / 32; ++i) step(j * BK + 32 * i, i, buffer, std::false_type{});
    } else if (mine < w.len) {
#pragma unroll 1
      for (int i = 0; i < BK / 32; ++i)
        if (j * BK + 32 * i <= mine) step(j * BK + 32 * i, i, buffer, std::true_type{});
    }
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
  if (!in) return;
  store_row<TYPE, ND, VEC>(p.dq, (w.start + row) * p.lddq + head * p.hdq, dq, p.scale / f, p.D);
}

template <int TYPE, int ND, bool VEC> hipError_t backward_launch(const AttentionP &p, hipStream_t s) {
  const long long tiles = attention_tiles(p), key_tiles = tiles * KEYS_PARTS, rest = p.offsets && p.zero_rest ? REST_BLOCKS : 0;
  if (TYPE == TYPE_F16) hipLaunchKernelGGL((attention_inner_kernel<VEC>), dim3((unsigned)(tiles * (p.Hq + p.Hkv))), dim3(256), 0, s, p);
  hipLaunchKernelGGL((attention_queries_kernel<TYPE, ND, VEC>), dim3((unsigned)(tiles * p.Hq + rest)), dim3(256), 0, s, p, (int)(tiles * p.Hq));
  hipLaunchKernelGGL((attention_keys_kernel<TYPE, ND, VEC>), dim3((unsigned)(key_tiles * p.Hkv + rest)), dim3(64 * KEYS_WAVES * KEYS_GROUPS), 0, s, p, (int)(key_tiles * p.Hkv));
  return hipGetLastError();
}
template <int TYPE, bool VEC> hipError_t backward_width(const AttentionP &p, hipStream_t s) {
  switch ((p.D + 31) / 32) {
    case 1: return backward_launch<TYPE, 1, VEC>(p, s);
    case 2: return backward_launch<TYPE, 2, VEC>(p, s);
    case 3: return backward_launch<TYPE, 3, VEC>(p, s);
    default: return backward_launch<TYPE, 4, VEC>(p, s);
  }
}

}  // namespace

hipError_t launch_attention_backward(const AttentionP &p, hipStream_t s) {
  const hipError_t e = launch_attention_tiles(p, s);
  if (e != hipSuccess) return e;
  const auto rows = [&](const void *t, long long h, long long ld) { return attention_vectors(t, p.type, h, ld, p.D); };
  const bool vec = rows(p.q, p.hq, p.ldq) && rows(p.k, p.hk, p.ldk) && rows(p.v, p.hv, p.ldv) && rows(p.o, p.ho, p.ldo) && rows(p.dout, p.hdo, p.lddo) &&
                   rows(p.dq, p.hdq, p.lddq) && rows(p.dk, p.hdk, p.lddk) && rows(p.dv, p.hdv, p.lddv);
  switch (p.type) {
    case TYPE_F32: return vec ? backward_width<TYPE_F32, true>(p, s) : backward_width<TYPE_F32, false>(p, s);
    case TYPE_BF16: return vec ? backward_width<TYPE_BF16, true>(p, s) : backward_width<TYPE_BF16, false>(p, s);
    default: return vec ? backward_width<TYPE_F16, true>(p, s) : backward_width<TYPE_F16, false>(p, s);
  }
}

}  // namespace absk
