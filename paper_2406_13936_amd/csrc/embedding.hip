// Token embedding of M replicas with tables of their own, the gradient of the tables, and the statistics that the batch tests take of it.
//
//   y_t = s table[token_t];   g_i = s sum_t dy_t e(token_t)^T of sample i (T tokens),  gbar = mean_i g_i,  n_i = ||g_i||^2,  q_i = <g_i, gbar>
//   A token outside the table is padding: zeros, no gradient.
//
// Forward is bound by memory (4 x 8192 rows of 1024 from fp32 tables of 32000 words into bf16: 27.6 us, of 20 that the bytes take).  The gradient sorts the tokens of a replica (stable, so that equal ones stay in the order of the samples) and
// sums runs of rows of dy in that order: no atomics on values, the same bits every time.  What it moves: dy once (twice with q_i, whose
// second look reads the finished gbar), the table's gradient once; zeros for words that no token names are written while the sort, which is
// all latency, is under way (the same sizes with n_i and q_i: 194 us, of them 118 the fill and the sort, 28 sums, 12 join, 24 the second look; the fill alone
// would be 85).
//   sort      stable passes of up to 11 bits of the key: counts per block, then every block adds up the counts before its own and
//             deals out its part, wavefront after wavefront; one launch for all passes where one block takes a replica's tokens
//   sums      a group of lanes takes up to 64 sorted rows: runs of one (word, sample) give n_i's shares, runs of a word gbar's row; what
//             crosses the group's ends is left as partial rows, which a second launch adds in order
//   inner     sum_t dy_t . gbar[token_t], and the shares of n_i and q_i added up in fp64
// A word's partial rows are added by one group of lanes, one after the other: of 2^18 tokens of 512 values half of which are one word it takes 478 us in all,
// where evenly spread words take 294, of 2^20 of 128 values 5.0 ms.
#include <algorithm>
#include <cstring>
#include "device_utils.h"
#include "ops.h"
#include "row_groups.h"

namespace absk {
namespace {

// a token as a row of the table; V for padding
__device__ __forceinline__ uint32_t token_at(const void *p, int wide, long long i, int V) {
  const long long t = wide ? static_cast<const long long *>(p)[i] : (long long)static_cast<const int *>(p)[i];
  return t >= 0 && t < V ? (uint32_t)t : (uint32_t)V;
}

// ---- forward -------------------------------------------------------------------------------------------------------

// (the table's rows are what should stay in the caches)
template <int TYPE> __device__ __forceinline__ void store8_once(void *p, long long at, const float (&v)[8]) {
  if constexpr (TYPE == TYPE_F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      st_once<true>(static_cast<float *>(p) + at + 4 * h, make_uint4(__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])));
  } else {
    st_once<true>(static_cast<uint16_t *>(p) + at, pack8(TYPE, v));
  }
}

// `lanes` threads to a row (a power of two), eight values each; R rows at a time, so that several rows of the table are under way
template <int TT, int TY, bool VEC, int R>
__global__ void __launch_bounds__(256) embedding_kernel(const EmbeddingP p, const int lanes, const long long all) {
  const int per = 256 / lanes, l = threadIdx.x & (lanes - 1), g = threadIdx.x / lanes, D = p.D;
  const long long n = (long long)p.b * p.T, step = (long long)gridDim.x * per;
  for (long long r0 = (long long)blockIdx.x * per + g; r0 < all; r0 += R * step) {
    uint32_t tok[R];
    long long m[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const long long r = r0 + k * step;
      m[k] = r < all ? (p.M == 1 ? 0 : r / n) : -1;
      tok[k] = r < all ? token_at(p.tokens, p.wide, r, p.V) : (uint32_t)p.V;
    }
    for (int c = l * 8; c < D; c += lanes * 8) {
      float v[R][8];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const bool in = tok[k] < (uint32_t)p.V;
        const long long at = in ? (m[k] * p.V + tok[k]) * D + c : 0;
        if (in && (VEC || c + 8 <= D)) {
          if (VEC) load8(p.table, TT, at, v[k]);
          else load8_any(p.table, TT, at, v[k]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[k][e] = in && c + e < D ? load_as_f32(p.table, TT, at + e) : 0.0f;
        }
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (m[k] < 0) continue;
        const long long at = m[k] * p.sy + (r0 + k * step - m[k] * n) * p.ldy + c;
        const bool in = tok[k] < (uint32_t)p.V;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = in ? v[k][e] * p.scale : 0.0f;
        if (VEC) store8_once<TY>(p.y, at, v[k]);
        else if (c + 8 <= D) store8_any(p.y, TY, at, v[k]);
        else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < D) store_from_f32(p.y, TY, at + e, v[k][e]);
        }
      }
    }
  }
}

template <int TT, int TY> void forward_typed(const EmbeddingP &p, hipStream_t s) {
  const long long all = (long long)p.M * p.b * p.T;
  int lanes = 8;
  while (lanes < 256 && lanes * 8 < p.D) lanes *= 2;
  const long long per = 256 / lanes, blocks = std::max(1LL, std::min((all + per - 1) / per, 4096LL));
  const bool vec = rows_of_vectors(p.table, TT, 0, p.D, p.D) && rows_of_vectors(p.y, TY, p.sy, p.ldy, p.D);
  if (vec) hipLaunchKernelGGL((embedding_kernel<TT, TY, true, 4>), dim3((unsigned)blocks), dim3(256), 0, s, p, lanes, all);
  else hipLaunchKernelGGL((embedding_kernel<TT, TY, false, 2>), dim3((unsigned)blocks), dim3(256), 0, s, p, lanes, all);
}
template <int TT> void forward_from(const EmbeddingP &p, hipStream_t s) {
  switch (p.type) {
    case TYPE_F32: return forward_typed<TT, TYPE_F32>(p, s);
    case TYPE_BF16: return forward_typed<TT, TYPE_BF16>(p, s);
    default: return forward_typed<TT, TYPE_F16>(p, s);
  }
}

// ---- the sort ------------------------------------------------------------------------------------------------------

constexpr int DIGIT_BITS = 11;           // most of a pass: the counts of four wavefronts are 32 KB of LDS
constexpr int SORT_WAVES = 4;
constexpr int SORT_BLOCKS = 64;          // to a replica at most: every block reads all blocks' counts
constexpr int SORT_ITEMS = 2048;         // of a block at least, and of a replica that one block sorts in one launch

struct SortPlan { int passes, bits, nb, items; };        // items: of a block, a multiple of 256
struct SortBuffers { uint32_t *key[2], *pos[2], *count; };      // [M][N] each, turn and turn about; counts [M][nb][2^bits]

SortPlan sort_plan(const EmbeddingP &p) {
  SortPlan s;
  const long long n = (long long)p.b * p.T;
  int bits = 1;
  while (bits < 31 && (1LL << bits) <= p.V) ++bits;      // keys up to V
  s.passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.nb = (int)std::max(1LL, std::min<long long>((n + SORT_ITEMS - 1) / SORT_ITEMS, SORT_BLOCKS));
  s.items = (int)(((n + s.nb - 1) / s.nb + 255) / 256 * 256);
  s.nb = (int)((n + s.items - 1) / s.items);
  return s;
}

__device__ __forceinline__ uint32_t sort_key(const EmbeddingP &p, const SortBuffers &t, int pass, long long base, long long i) {
  return pass == 0 ? token_at(p.tokens, p.wide, base + i, p.V) : t.key[(pass - 1) & 1][base + i];
}

// Blocks from `first` on fill the part-th of `parts` parts of the table's gradient with zeros: each launch of the sort has some to do
struct Fill { int part, parts; };
__device__ __forceinline__ void fill_zeros(float *out, long long n, int first, const Fill f) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  const long long head = min((long long)((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / 4, n), n4 = (n - head) / 4, tail = head + n4 * 4;
  const long long each = (n4 + f.parts - 1) / f.parts, i0 = f.part * each, i1 = min(i0 + each, n4);
  const long long step = (long long)(gridDim.x - first) * 256, at = (long long)(blockIdx.x - first) * 256 + threadIdx.x;
  f4 *v = reinterpret_cast<f4 *>(out + head);
  const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (long long i = i0 + at; i < i1; i += step) __builtin_nontemporal_store(zero, v + i);
  if (f.part == 0) {
    if (at < head) out[at] = 0.0f;
    if (at < n - tail) out[tail + at] = 0.0f;
  }
}

__global__ void __launch_bounds__(256) sort_count_kernel(const EmbeddingP p, const SortPlan w, const SortBuffers t, const int pass, const Fill f) {
  __shared__ uint32_t count[1 << DIGIT_BITS];
  if ((int)blockIdx.x >= p.M * w.nb) return fill_zeros(p.dtable, (long long)p.M * p.V * p.D, p.M * w.nb, f);
  const int m = blockIdx.x / w.nb, j = blockIdx.x - m * w.nb, R = 1 << w.bits;
  const long long n = (long long)p.b * p.T, base = m * n, i0 = (long long)j * w.items, i1 = min(i0 + w.items, n);
  for (int d = threadIdx.x; d < R; d += 256) count[d] = 0;
  __syncthreads();
  for (long long i = i0 + threadIdx.x; i < i1; i += 256) atomicAdd(&count[(sort_key(p, t, pass, base, i) >> (pass * w.bits)) & (R - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < R; d += 256) t.count[((long long)m * w.nb + j) * R + d] = count[d];
}

// Passes [first, last): of several only where one block has all tokens of its replica (nb == 1).
__global__ void __launch_bounds__(256) sort_deal_kernel(const EmbeddingP p, const SortPlan w, const SortBuffers t, const int first, const int last, const Fill f) {
  __shared__ uint32_t at[SORT_WAVES][1 << DIGIT_BITS];      // how many of a digit each wavefront has; then where its next one goes
  __shared__ uint32_t sums[SORT_WAVES];
  if ((int)blockIdx.x >= p.M * w.nb) return fill_zeros(p.dtable, (long long)p.M * p.V * p.D, p.M * w.nb, f);
  const int m = blockIdx.x / w.nb, j = blockIdx.x - m * w.nb, R = 1 << w.bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long n = (long long)p.b * p.T, base = m * n, i0 = (long long)j * w.items, i1 = min(i0 + w.items, n);
  const int part = w.items / SORT_WAVES;
  const long long a0 = i0 + (long long)wave * part, a1 = min(a0 + part, i1);
  for (int pass = first; pass < last; ++pass) {
    const int shift = pass * w.bits, from = (pass - 1) & 1, to = pass & 1;
    for (int d = threadIdx.x; d < R * SORT_WAVES; d += 256) at[d / R][d % R] = 0;
    __syncthreads();
    for (long long i = a0 + lane; i < a1; i += 64) atomicAdd(&at[wave][(sort_key(p, t, pass, base, i) >> shift) & (R - 1)], 1u);
    __syncthreads();
    // thread: `each` neighbouring digits; before: of all digits before them; then the blocks before this one
    const int each = (R + 255) / 256, d0 = threadIdx.x * each, d1 = min(d0 + each, R);
    uint32_t mine = 0;
    for (int d = d0; d < d1; ++d) {
      if (w.nb > 1) for (int k = 0; k < w.nb; ++k) mine += t.count[((long long)m * w.nb + k) * R + d];
      else for (int k = 0; k < SORT_WAVES; ++k) mine += at[k][d];
    }
    uint32_t before = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(before, o, 64);
      if (lane >= o) before += up;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    before -= mine;
    for (int k = 0; k < wave; ++k) before += sums[k];
    for (int d = d0; d < d1; ++d) {
      uint32_t all = 0, here = before;
      if (w.nb > 1) {
        for (int k = 0; k < w.nb; ++k) {
          const uint32_t c = t.count[((long long)m * w.nb + k) * R + d];
          all += c;
          if (k < j) here += c;
        }
      } else {
        for (int k = 0; k < SORT_WAVES; ++k) all += at[k][d];
      }
      for (int k = 0; k < SORT_WAVES; ++k) {
        const uint32_t c = at[k][d];
        at[k][d] = here;
        here += c;
      }
      before += all;
    }
    __syncthreads();
    // 64 tokens at a time, in order: those of one digit go side by side
    for (long long b0 = a0; b0 < a1; b0 += 64) {
      const long long i = b0 + lane;
      const bool in = i < a1;
      const uint32_t key = in ? sort_key(p, t, pass, base, i) : 0u, pos = !in || pass == 0 ? (uint32_t)i : t.pos[from][base + i];
      const uint32_t digit = (key >> shift) & (R - 1);
      uint64_t same = __ballot(in);
      for (int k = 0; k < w.bits; ++k) {
        const uint64_t set = __ballot((digit >> k) & 1);
        same &= (digit >> k) & 1 ? set : ~set;
      }
      const int leader = in ? __ffsll((unsigned long long)same) - 1 : lane;
      uint32_t where = 0;
      if (in && lane == leader) where = atomicAdd(&at[wave][digit], (uint32_t)__popcll(same));
      where = __shfl(where, leader, 64) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
      if (in) {
        t.key[to][base + where] = key;
        t.pos[to][base + where] = pos;
      }
    }
    __syncthreads();
  }
}

// ---- sums of runs --------------------------------------------------------------------------------------------------

struct SumPlan { int group, tile, tiles, rows, chunks, inner_rows, inner_chunks; };      // lanes; columns of a tile; sorted rows of a group
struct SumBuffers {
  const uint32_t *key, *pos;             // sorted
  float *head, *tail;                    // [M][chunks][D]: sums of a word's rows that a group's first or last row cuts off
  float *shead, *stail;                  // the same of a word's rows of one sample (n_i)
  float *share;                          // [tiles][M][N] n_i's, at the last token of each run; zeros elsewhere
  float *inner;                          // [M b][inner_chunks] q_i's
};

SumPlan sum_plan(const EmbeddingP &p) {
  SumPlan w;
  const long long n = (long long)p.b * p.T;
  w.group = p.D <= 128 ? 16 : 64;
  w.tile = w.group * 8;
  w.tiles = (p.D + w.tile - 1) / w.tile;
  w.rows = 8;
  while (w.rows < w.group && n * p.M * w.tiles / w.rows > 4096LL * 64 / w.group) w.rows *= 2;
  w.chunks = (int)((n + w.rows - 1) / w.rows);
  w.inner_rows = (int)std::max(1LL, std::min<long long>(p.T, std::max(4LL, n * p.M * w.group / (8192LL * 64))));
  w.inner_chunks = (p.T + w.inner_rows - 1) / w.inner_rows;
  return w;
}

// lane k's value in a group of G lanes; k is the same for all of them
template <int G> __device__ __forceinline__ uint32_t of_lane(uint32_t v, int k) {
  if constexpr (G == 64) return (uint32_t)__builtin_amdgcn_readlane((int)v, k);
  else return __shfl(v, k, G);
}
template <int TYPE, int G, bool VEC>
__device__ __forceinline__ void add_raw(float (&a)[8], const Raw<TYPE, 1> &r) {
  float f[8];
  raw_vals<TYPE, 1>(r, 0, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] += f[e];
}
// a lane's eight columns of an fp32 row (D of them from `out` on)
template <int TYPE, int G> __device__ __forceinline__ void store_columns(float *out, int D, int l, const float (&a)[8], float by) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = col_of<TYPE, G>(0, 4 * h, l);
    if (c + 4 <= D && !(reinterpret_cast<uintptr_t>(out + c) & 15)) {
      *reinterpret_cast<float4 *>(out + c) = make_float4(a[4 * h] * by, a[4 * h + 1] * by, a[4 * h + 2] * by, a[4 * h + 3] * by);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < D) out[c + e] = a[4 * h + e] * by;
    }
  }
}

template <int TYPE, int G, bool VEC, bool NORM>
__global__ void __launch_bounds__(256) embedding_sums_kernel(const EmbeddingP p, const SumPlan w, const SumBuffers t, const float by) {
  constexpr int GP = 256 / G, U = TYPE == TYPE_F32 ? 4 : 8;
  const int gid = G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G, l = threadIdx.x % G;
  const long long item = (long long)blockIdx.x * GP + gid;
  const long long per = (long long)w.chunks * w.tiles;
  if (item >= per * p.M) return;
  const int m = (int)(item / per), rest = (int)(item - m * per), chunk = rest / w.tiles, tile = rest - chunk * w.tiles;
  const int c0 = tile * w.tile, D = min(p.D - c0, w.tile);
  const long long n = (long long)p.b * p.T, base = m * n, i0 = (long long)chunk * w.rows;
  const int count = (int)min((long long)w.rows, n - i0);
  // lane k: word and place of the k-th row (G >= rows); what stands before and behind
  const long long mine = i0 + min(l, count - 1);
  const uint32_t key = t.key[base + mine], pos = t.pos[base + mine];
  const uint32_t sample = NORM ? pos / (uint32_t)p.T : 0u;
  const uint32_t none = 0xffffffffu;
  const uint32_t key_before = i0 > 0 ? t.key[base + i0 - 1] : none, key_behind = i0 + count < n ? t.key[base + i0 + count] : none;
  uint32_t sample_before = 0, sample_behind = 0;
  if (NORM) {
    sample_before = i0 > 0 ? t.pos[base + i0 - 1] / (uint32_t)p.T : 0u;
    sample_behind = i0 + count < n ? t.pos[base + i0 + count] / (uint32_t)p.T : 0u;
  }
  const uint32_t key0 = of_lane<G>(key, 0), sample0 = of_lane<G>(sample, 0);
  bool word_cut = key0 == key_before, run_cut = word_cut && sample0 == sample_before;      // began before this group's rows
  float word[8], run[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) word[e] = run[e] = 0.0f;
  float *head = t.head + ((long long)m * w.chunks + chunk) * p.D + c0, *tail = t.tail + ((long long)m * w.chunks + chunk) * p.D + c0;
  float *shead = nullptr, *stail = nullptr, *share = nullptr;
  if (NORM) {
    shead = t.shead + ((long long)m * w.chunks + chunk) * p.D + c0;
    stail = t.stail + ((long long)m * w.chunks + chunk) * p.D + c0;
    share = t.share + ((long long)tile * p.M + m) * n;
  }
  for (int q0 = 0; q0 < count; q0 += U) {
    Raw<TYPE, 1> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t at = of_lane<G>(pos, min(q0 + u, count - 1));
      load_raw<TYPE, G, 1, VEC>(raw[u], p.dy, m * p.sy + (long long)at * p.ldy + c0, D, l);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = q0 + u;
      if (q >= count) break;
      const uint32_t k = of_lane<G>(key, q), k1 = q + 1 < count ? of_lane<G>(key, q + 1) : key_behind;
      const uint32_t at = of_lane<G>(pos, q);
      if (k >= (uint32_t)p.V) {                   // padding, behind all words
        if (NORM && l == 0) share[at] = 0.0f;
        continue;
      }
      const bool word_ends = k1 != k;
      add_raw<TYPE, G, VEC>(NORM ? run : word, raw[u]);
      if (NORM) {
        const uint32_t s = of_lane<G>(sample, q), s1 = q + 1 < count ? of_lane<G>(sample, q + 1) : sample_behind;
        if (word_ends || s1 != s) {
          if (run_cut) {
            store_columns<TYPE, G>(shead, D, l, run, 1.0f);
          } else {
            float v = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) v = fmaf(run[e], run[e], v);      // (zeros beyond the row)
            v = lanes_sum<G>(v);
            if (l == 0) share[at] = v;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) { word[e] += run[e]; run[e] = 0.0f; }
          run_cut = false;
        } else if (l == 0) {
          share[at] = 0.0f;
        }
      }
      if (word_ends) {
        if (word_cut) store_columns<TYPE, G>(head, D, l, word, 1.0f);
        else store_columns<TYPE, G>(p.dtable + ((long long)m * p.V + k) * p.D + c0, D, l, word, by);
#pragma unroll
        for (int e = 0; e < 8; ++e) word[e] = 0.0f;
        word_cut = false;
      }
    }
  }
  // what goes on behind this group's rows
  const uint32_t kl = of_lane<G>(key, count - 1), sl = of_lane<G>(sample, count - 1);
  if (kl < (uint32_t)p.V && kl == key_behind) {
    if (NORM) {
      if (sl == sample_behind) store_columns<TYPE, G>(run_cut ? shead : stail, D, l, run, 1.0f);
#pragma unroll
      for (int e = 0; e < 8; ++e) word[e] += run[e];
    }
    store_columns<TYPE, G>(word_cut ? head : tail, D, l, word, 1.0f);
  }
}

// Words and runs that cross the ends of groups: the group where one begins adds the partial rows of those behind it.
// How many of the next groups' first rows (from row i1 on, `rows` apart) are in the run: the lanes look at one each
template <int G, class F> __device__ __forceinline__ int groups_behind(long long i1, int rows, long long n, F &&in_run) {
  const int l = threadIdx.x % G, base = threadIdx.x & 63 & ~(G - 1);
  for (int more = 0;; more += G) {
    const long long at = i1 + (long long)(more + l) * rows;
    const uint64_t in = __ballot(at < n && in_run(at)) >> base, all = G == 64 ? ~0ull : (1ull << (G & 63)) - 1;
    if ((in & all) != all) return more + __ffsll((unsigned long long)(~in & all)) - 1;
  }
}
template <int G>
__device__ __forceinline__ void add_partials(float (&a)[8], const float *tail, const float *head, int more, int stride, int D, int l) {
  if (l * 8 + 8 <= D && !((reinterpret_cast<uintptr_t>(tail) | reinterpret_cast<uintptr_t>(head) | (uintptr_t)stride * 4) & 15)) {
    load8(tail, TYPE_F32, l * 8, a);
#pragma unroll 4
    for (int k = 0; k < more; ++k) {
      float v[8];
      load8(head, TYPE_F32, (long long)k * stride + l * 8, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] += v[e];
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = l * 8 + e, at = c < D ? c : 0;
    float v = tail[at];
#pragma unroll 8
    for (int k = 0; k < more; ++k) v += head[(long long)k * stride + at];
    a[e] = c < D ? v : 0.0f;
  }
}
template <int G, bool NORM>
__global__ void __launch_bounds__(256) embedding_join_kernel(const EmbeddingP p, const SumPlan w, const SumBuffers t, const float by) {
  constexpr int GP = 256 / G;
  const int gid = G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G, l = threadIdx.x % G;
  const long long item = (long long)blockIdx.x * GP + gid, per = (long long)w.chunks * w.tiles;
  if (item >= per * p.M) return;
  const int m = (int)(item / per), rest = (int)(item - m * per), chunk = rest / w.tiles, tile = rest - chunk * w.tiles;
  const int c0 = tile * w.tile, D = min(p.D - c0, w.tile);
  const long long n = (long long)p.b * p.T, base = m * n, i0 = (long long)chunk * w.rows, i1 = i0 + w.rows;
  if (i1 >= n) return;                             // nothing behind the last group
  const uint32_t *key = t.key + base, *pos = t.pos + base;
  const uint32_t k = key[i1 - 1], T = (uint32_t)p.T, next = key[i1], before = i0 > 0 ? key[i0 - 1] : 0xffffffffu;
  const uint32_t pl = pos[i1 - 1], pn = pos[i1], pb = i0 > 0 ? pos[i0 - 1] : 0u;
  if (k >= (uint32_t)p.V || next != k) return;
  const long long slot = ((long long)m * w.chunks + chunk) * p.D + c0;
  float a[8];
  if (before != k) {                               // the word begins here
    const int more = groups_behind<G>(i1, w.rows, n, [&](long long i) { return key[i] == k; });
    add_partials<G>(a, t.tail + slot, t.head + slot + p.D, more, p.D, D, l);
    store_columns<TYPE_BF16, G>(p.dtable + ((long long)m * p.V + k) * p.D + c0, D, l, a, by);
  }
  if (NORM) {
    const uint32_t s = pl / T;
    auto in_run = [&](long long i) { return key[i] == k && pos[i] / T == s; };
    if (pn / T == s && (before != k || pb / T != s)) {
      const int more = groups_behind<G>(i1, w.rows, n, in_run);
      add_partials<G>(a, t.stail + slot, t.shead + slot + p.D, more, p.D, D, l);
      float v = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v = fmaf(a[e], a[e], v);
      v = lanes_sum<G>(v);
      // the run's last row is in the last of them, which has no more rows than the group has lanes
      const long long last = i1 + (long long)(more - 1) * w.rows;
      const int in = groups_behind<G>(last, 1, min(n, last + w.rows), in_run);
      if (l == 0) t.share[((long long)tile * p.M + m) * n + pos[last + in - 1]] = v;
    }
  }
}

// q_i's share of some of a sample's tokens: sum_t dy_t . gbar[token_t]
template <int TYPE, int G, bool VEC>
__global__ void __launch_bounds__(256) embedding_inner_kernel(const EmbeddingP p, const SumPlan w, const SumBuffers t) {
  constexpr int GP = 256 / G, U = 4;
  const int gid = G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G, l = threadIdx.x % G;
  const long long item = (long long)blockIdx.x * GP + gid;
  if (item >= (long long)p.M * p.b * w.inner_chunks) return;
  const long long i = item / w.inner_chunks, m = i / p.b, n = (long long)p.b * p.T;
  const int ch = (int)(item - i * w.inner_chunks), t0 = ch * w.inner_rows, t1 = min(t0 + w.inner_rows, p.T);
  const long long r0 = (i - m * p.b) * p.T;
  float a = 0.0f;
  for (int q = t0; q < t1; q += U) {
    uint32_t tok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) tok[u] = q + u < t1 ? token_at(p.tokens, p.wide, m * n + r0 + q + u, p.V) : (uint32_t)p.V;
    for (int c0 = 0; c0 < p.D; c0 += w.tile) {
      const int D = min(p.D - c0, w.tile);
      Raw<TYPE, 1> ry[U];
      float g[U][1][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {                // (of a padding token the first row's, not used)
        const bool in = tok[u] < (uint32_t)p.V;
        load_raw<TYPE, G, 1, VEC>(ry[u], p.dy, m * p.sy + (r0 + (in ? q + u : t0)) * p.ldy + c0, D, l);
        load_param_as<TYPE, TYPE_F32, G, 1, VEC>(g[u], p.dtable, (m * p.V + (in ? tok[u] : 0)) * p.D + c0, D, l);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (tok[u] >= (uint32_t)p.V) continue;
        float y[8];
        raw_vals<TYPE, 1>(ry[u], 0, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) a = fmaf(y[e], g[u][0][e], a);
      }
    }
  }
  a = lanes_sum<G>(a);
  if (l == 0) t.inner[item] = a;
}

// n_i = s^2 sum of the shares of its tokens, q_i = s sum of its parts: W wavefronts to a sample
template <int W> __global__ void __launch_bounds__(256) embedding_finish_kernel(const EmbeddingP p, const SumPlan w, const SumBuffers t) {
  __shared__ double sm[W];
  const long long i = W == 1 ? (long long)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (i >= (long long)p.M * p.b) return;
  const int l = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long long all = (long long)p.M * p.b * p.T, r0 = i * p.T;
  double a = 0.0, b = 0.0;
  if (p.n)
    for (int tile = 0; tile < w.tiles; ++tile)
#pragma unroll 4
      for (int k = l; k < p.T; k += W * 64) a += t.share[tile * all + r0 + k];
  if (p.q)
    for (int k = l; k < w.inner_chunks; k += W * 64) b += t.inner[i * w.inner_chunks + k];
  if constexpr (W == 1) {
    a = wave_sum(a);
    b = wave_sum(b);
  } else {
    a = block_sum<W>(a, sm);
    b = block_sum<W>(b, sm);
  }
  if (l == 0) {
    if (p.n) p.n[i] = (float)(a * p.scale * p.scale);
    if (p.q) p.q[i] = (float)(b * p.scale);
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------

struct Pieces { size_t key[2], pos[2], count, head, tail, shead, stail, share, inner, total; };
Pieces pieces(const EmbeddingP &p, const SortPlan &o, const SumPlan &w, bool want_n, bool want_q) {
  Pieces q;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t r = at; at = (at + bytes + 255) / 256 * 256; return r; };
  const size_t n = (size_t)p.M * p.b * p.T, parts = (size_t)p.M * w.chunks * p.D * 4;
  q.key[0] = take(n * 4); q.pos[0] = take(n * 4);
  q.key[1] = take(o.passes > 1 ? n * 4 : 0); q.pos[1] = take(o.passes > 1 ? n * 4 : 0);
  q.count = take(o.nb > 1 ? ((size_t)p.M * o.nb << o.bits) * 4 : 0);
  q.head = take(parts); q.tail = take(parts);
  q.shead = take(want_n ? parts : 0); q.stail = take(want_n ? parts : 0);
  q.share = take(want_n ? n * w.tiles * 4 : 0);
  q.inner = take(want_q ? (size_t)p.M * p.b * w.inner_chunks * 4 : 0);
  q.total = at;
  return q;
}

template <int TYPE, int G, bool VEC> hipError_t backward_launches(const EmbeddingP &p, const SumPlan &w, const SumBuffers &t, hipStream_t s) {
  constexpr int GP = 256 / G;
  const float by = (float)((double)p.scale / p.b);
  const long long items = (long long)p.M * w.chunks * w.tiles, blocks = (items + GP - 1) / GP;
  const long long looks = ((long long)p.M * p.b * w.inner_chunks + GP - 1) / GP;
  if (blocks > 0xffffff || (p.q && looks > 0xffffff)) return hipErrorInvalidValue;      // (a grid counts its threads in 32 bits)
  if (p.n) {
    hipLaunchKernelGGL((embedding_sums_kernel<TYPE, G, VEC, true>), dim3((unsigned)blocks), dim3(256), 0, s, p, w, t, by);
    hipLaunchKernelGGL((embedding_join_kernel<G, true>), dim3((unsigned)blocks), dim3(256), 0, s, p, w, t, by);
  } else {
    hipLaunchKernelGGL((embedding_sums_kernel<TYPE, G, VEC, false>), dim3((unsigned)blocks), dim3(256), 0, s, p, w, t, by);
    hipLaunchKernelGGL((embedding_join_kernel<G, false>), dim3((unsigned)blocks), dim3(256), 0, s, p, w, t, by);
  }
  if (p.q) hipLaunchKernelGGL((embedding_inner_kernel<TYPE, G, VEC>), dim3((unsigned)looks), dim3(256), 0, s, p, w, t);
  const long long samples = (long long)p.M * p.b;
  if (!p.n && !p.q) return hipGetLastError();
  if (p.T < 256 || samples > 1 << 20) hipLaunchKernelGGL((embedding_finish_kernel<1>), dim3((unsigned)((samples + 3) / 4)), dim3(256), 0, s, p, w, t);
  else hipLaunchKernelGGL((embedding_finish_kernel<4>), dim3((unsigned)samples), dim3(256), 0, s, p, w, t);
  return hipGetLastError();
}
template <int TYPE, bool VEC> hipError_t backward_group(const EmbeddingP &p, const SumPlan &w, const SumBuffers &t, hipStream_t s) {
  return w.group == 16 ? backward_launches<TYPE, 16, VEC>(p, w, t, s) : backward_launches<TYPE, 64, VEC>(p, w, t, s);
}

}  // namespace

hipError_t launch_embedding(const EmbeddingP &p, hipStream_t s) {
  switch (p.ttype) {
    case TYPE_F32: forward_from<TYPE_F32>(p, s); break;
    case TYPE_BF16: forward_from<TYPE_BF16>(p, s); break;
    default: forward_from<TYPE_F16>(p, s);
  }
  return hipGetLastError();
}

size_t embedding_backward_bytes(const EmbeddingP &p, bool want_n, bool want_q) {
  return pieces(p, sort_plan(p), sum_plan(p), want_n, want_q).total;
}

hipError_t launch_embedding_backward(const EmbeddingP &p, void *workspace, hipStream_t s) {
  const SortPlan o = sort_plan(p);
  const SumPlan w = sum_plan(p);
  const Pieces at = pieces(p, o, w, p.n != nullptr, p.q != nullptr);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  auto words = [&](size_t off) { return reinterpret_cast<uint32_t *>(ws + off); };
  auto floats = [&](size_t off) { return reinterpret_cast<float *>(ws + off); };
  const SortBuffers b = {{words(at.key[0]), words(at.key[1])}, {words(at.pos[0]), words(at.pos[1])}, words(at.count)};
  const long long cells = (long long)p.M * p.V * p.D;
  const int sorting = p.M * o.nb, filling = (int)std::max(1LL, std::min(cells / 4096, 2048LL));
  const dim3 grid(sorting + filling);
  if (o.nb == 1) {
    hipLaunchKernelGGL(sort_deal_kernel, grid, dim3(256), 0, s, p, o, b, 0, o.passes, (Fill{0, 1}));
  } else {
    for (int pass = 0; pass < o.passes; ++pass) {
      hipLaunchKernelGGL(sort_count_kernel, grid, dim3(256), 0, s, p, o, b, pass, (Fill{2 * pass, 2 * o.passes}));
      hipLaunchKernelGGL(sort_deal_kernel, grid, dim3(256), 0, s, p, o, b, pass, pass + 1, (Fill{2 * pass + 1, 2 * o.passes}));
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int last = (o.passes - 1) & 1;
  const SumBuffers t = {b.key[last], b.pos[last], floats(at.head), floats(at.tail), floats(at.shead), floats(at.stail), floats(at.share), floats(at.inner)};
  const bool vec = rows_of_vectors(p.dy, p.type, p.sy, p.ldy, p.D);
  switch (p.type) {
    case TYPE_F32: return vec ? backward_group<TYPE_F32, true>(p, w, t, s) : backward_group<TYPE_F32, false>(p, w, t, s);
    case TYPE_BF16: return vec ? backward_group<TYPE_BF16, true>(p, w, t, s) : backward_group<TYPE_BF16, false>(p, w, t, s);
    default: return vec ? backward_group<TYPE_F16, true>(p, w, t, s) : backward_group<TYPE_F16, false>(p, w, t, s);
  }
}

}  // namespace absk
