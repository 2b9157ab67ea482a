// Layer norm, its gradients, and the statistics that the batch tests take of them.
//
//   mu = mean_d x,  r = 1 / sqrt(mean_d (x - mu)^2 + eps),  xh = (x - mu) r,  y = xh gamma + beta
//   h = dy gamma,  dx = r (h - mean_d h - xh mean_d(h xh))
//   sample i (T rows):  g_i = (sum_t dy xh, sum_t dy),   gbar = mean_i g_i,   n_i = ||g_i||^2,   q_i = <g_i, gbar>
//
// All of it is bound by memory: forward reads x and writes y, backward reads x and dy and writes dx (8 x 8192 rows of 2048 in bf16: 108 us
// and 168, 5.0 and 4.8 TB/s; 90 us where half of x is still in a cache).  A row lives in the
// registers of a group of G lanes (16 to 512, V vectors of 8 values to a lane), so it is read once; gains, biases and
// the sums for gbar stay in the registers of the lanes that own their columns, over all rows of a block.  A block leaves
// one partial of (sum dy xh, sum dy), and a second launch adds the partials in order: no atomics, the same bits every time.
// The gradient of a gain is no outer product, so n_i has no factored form: samples of several rows are summed in
// registers by the block that has all of their rows, or from the partials where a sample is spread over blocks.
#include <algorithm>
#include <cstring>
#include <type_traits>
#include "device_utils.h"
#include "ops.h"
#include "typed_mem.h"

namespace absk {
namespace {

// ---- groups of lanes -----------------------------------------------------------------------------------------------

// Sum over the 16 lanes of a DPP row, over a wavefront: every lane has it.
template <int G> __device__ __forceinline__ float lanes_sum(float v) {
  static_assert(G == 16 || G == 64, "a row or a wavefront");
  v += dpp<0xB1>(v);                              // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);                              // quad_perm [2,3,0,1]
  v += dpp<0x141>(v);                             // row_half_mirror
  v += dpp<0x140>(v);                             // row_mirror
  if (G == 64) {
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
  }
  return v;
}

constexpr int ln_threads(int G) { return G > 256 ? G : 256; }      // of a block

// Sums of N values over the group.  G >= 256: through LDS, one barrier a call (`turn` picks one of two buffers, so that the
// next call's values do not meet this one's readers); every thread of the block takes part.
template <int G, int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float *sm, int turn) {      // sm: 2 N floats to a wavefront
  constexpr int W = G > 64 ? G / 64 : 4;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum<(G < 64 ? G : 64)>(v[i]);
  if (G <= 64) return;
  float *s = sm + (turn & 1) * N * W;
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i * W + wave] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0f;
#pragma unroll
    for (int h = 0; h < W; h += 4) {
      const float4 f = *reinterpret_cast<const float4 *>(s + i * W + h);
      v[i] += (f.x + f.y) + (f.z + f.w);
    }
  }
}

// Columns of lane l in a row: 16-byte vectors that lie side by side over the lanes, of 16-bit values (v G + l) 8 + e, of fp32
// ((2 v + e / 4) G + l) 4 + e % 4.
template <int TYPE, int G> __device__ __forceinline__ int col_of(int v, int e, int l) {
  return TYPE == TYPE_F32 ? ((2 * v + (e >> 2)) * G + l) * 4 + (e & 3) : (v * G + l) * 8 + e;
}

// Results are not read again here: non-temporal stores (16-bit rows of 2048: forward 116 -> 101 us for 134 M values, backward 204 -> 194;
// non-temporal loads cost more than they give where the inputs are still in a cache).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool VEC> __device__ __forceinline__ void st_once(void *p, uint4 v) {
  const u32x4 w = {v.x, v.y, v.z, v.w};
  if constexpr (VEC) __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p));
  else __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any *>(p));
}

// q without its first k values of BYTES, moved down, zeros behind them (k <= 16 / BYTES)
template <int BYTES> __device__ __forceinline__ uint4 move_down(uint4 q, int k) {
  if (BYTES == 2) {
    const uint32_t s = 16 * (k & 1);
    q = make_uint4(__builtin_amdgcn_alignbit(q.y, q.x, s), __builtin_amdgcn_alignbit(q.z, q.y, s), __builtin_amdgcn_alignbit(q.w, q.z, s), q.w >> s);
    k >>= 1;
  }
  const bool one = k & 1, two = k & 2, all = k & 4;        // words
  q = make_uint4(one ? q.y : q.x, one ? q.z : q.y, one ? q.w : q.z, one ? 0u : q.w);
  q = make_uint4(two ? q.z : q.x, two ? q.w : q.y, two ? 0u : q.z, two ? 0u : q.w);
  return make_uint4(all ? 0u : q.x, all ? 0u : q.y, all ? 0u : q.z, all ? 0u : q.w);
}

// 16 bytes of a row of D values of BYTES from column c on, zeros beyond the row; nothing outside the row is read.  VEC: whole vectors at
// 16-byte places.  Else a vector that would pass the row's end is the row's last one, moved down.
// (Every lane loads, from a column of the row where it has none: loads behind branches wait for each other.)
template <int BYTES, bool VEC> __device__ __forceinline__ uint4 load16(const void *p, long long at, int c, int D) {
  constexpr int N = 16 / BYTES;
  if constexpr (VEC) {
    const bool in = c < D;
    const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const unsigned char *>(p) + (at + (in ? c : 0)) * BYTES);
    return make_uint4(in ? q.x : 0u, in ? q.y : 0u, in ? q.z : 0u, in ? q.w : 0u);
  }
  const unsigned char *row = static_cast<const unsigned char *>(p) + at * BYTES;
  if (D < N) {                                    // (no row this short has such a vector)
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (c + e < D) {
        if constexpr (BYTES == 4) w[e] = reinterpret_cast<const uint32_t *>(row)[c + e];
        else w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c + e] << (16 * (e & 1));
      }
    return make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    const int from = min(c, D - N), k = min(c - from, N);
    return move_down<BYTES>(load16_any(row + (long long)from * BYTES), k);
  }
}

// What a lane holds of a row as it comes from memory
template <int TYPE, int V> struct Raw { uint4 q[V * (TYPE == TYPE_F32 ? 2 : 1)]; };

template <int TYPE, int G, int V, bool VEC>
__device__ __forceinline__ void load_raw(Raw<TYPE, V> &r, const void *p, long long at, int D, int l) {
  constexpr int PER = TYPE == TYPE_F32 ? 2 : 1, N = 8 / PER;        // vectors of a lane's eight, values of a vector
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int h = 0; h < PER; ++h) r.q[v * PER + h] = load16<16 / N, VEC>(p, at, col_of<TYPE, G>(v, N * h, l), D);
}

// From here on the values count as unknown, so that what was computed from them is computed again and not kept in registers.
template <int TYPE, int V> __device__ __forceinline__ void forget(Raw<TYPE, V> &r) {
#pragma unroll
  for (auto &q : r.q) asm volatile("" : "+v"(q.x), "+v"(q.y), "+v"(q.z), "+v"(q.w));
}
template <int TYPE, int V> __device__ __forceinline__ void raw_vals(const Raw<TYPE, V> &r, int v, float (&f)[8]) {
  if constexpr (TYPE == TYPE_F32) {
    const uint4 a = r.q[2 * v], b = r.q[2 * v + 1];
    f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
    f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
  } else {
    unpack8(r.q[v], TYPE, f);
  }
}
// What a column's value is centred with: the row's mean, and beyond the row, where values are zeros, nothing: 1 / sqrt(eps) times a large
// mean may be infinite, and its product with dy = 0 NaN
template <int TYPE, int G, bool VEC> __device__ __forceinline__ float mean_at(int v, int e, int l, int D, float mean) {
  constexpr int N = TYPE == TYPE_F32 ? 4 : 8;              // (whole vectors are in the row or not)
  return col_of<TYPE, G>(v, VEC ? e & ~(N - 1) : e, l) < D ? mean : 0.0f;
}
template <int TYPE, int G, bool VEC>
__device__ __forceinline__ void store_vals(void *p, long long at, int D, int l, int v, const float (&f)[8]) {
  constexpr int PER = TYPE == TYPE_F32 ? 2 : 1, N = 8 / PER;
#pragma unroll
  for (int h = 0; h < PER; ++h) {
    const int c = col_of<TYPE, G>(v, N * h, l);
    if (VEC ? c < D : c + N <= D) {
      if constexpr (TYPE == TYPE_F32)
        st_once<VEC>(static_cast<float *>(p) + at + c, make_uint4(__float_as_uint(f[4 * h]), __float_as_uint(f[4 * h + 1]), __float_as_uint(f[4 * h + 2]), __float_as_uint(f[4 * h + 3])));
      else
        st_once<VEC>(static_cast<uint16_t *>(p) + at + c, pack8(TYPE, f));
    } else if (!VEC) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c + e < D) store_from_f32(p, TYPE, at + c + e, f[N * h + e]);
    }
  }
}
// Gains, biases or batch gradients (fp32, or with PARAM == TYPE the rows' type) of a lane's columns; null: zeros
template <int TYPE, int PARAM, int G, int V, bool VEC>
__device__ __forceinline__ void load_param_as(float (&f)[V][8], const void *p, long long at, int D, int l) {
  const bool whole = VEC && !((reinterpret_cast<uintptr_t>(p) + at * (PARAM == TYPE_F32 ? 4 : 2)) & 15);
  auto load = [&](auto W) {
    constexpr bool w = decltype(W)::value;
    if constexpr (PARAM == TYPE) {
      Raw<TYPE, V> r;
      load_raw<TYPE, G, V, w>(r, p, at, D, l);
#pragma unroll
      for (int v = 0; v < V; ++v) raw_vals<TYPE, V>(r, v, f[v]);
    } else {                                      // fp32 beside 16-bit rows: two vectors to one of theirs
      Raw<TYPE_F32, V> r;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int h = 0; h < 2; ++h) r.q[2 * v + h] = load16<4, w>(p, at, col_of<TYPE, G>(v, 4 * h, l), D);
#pragma unroll
      for (int v = 0; v < V; ++v) raw_vals<TYPE_F32, V>(r, v, f[v]);
    }
  };
  if constexpr (!VEC) {
    load(std::false_type{});
  } else if (whole) {
    load(std::true_type{});
  } else {                                        // (whole vectors of rows beside unaligned gains)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = col_of<TYPE, G>(v, e, l);
        const bool in = c < D;
        const float got = load_as_f32(p, PARAM, at + (in ? c : 0));
        f[v][e] = in ? got : 0.0f;
      }
  }
}
template <int TYPE, int G, int V, bool VEC>
__device__ __forceinline__ void load_param(float (&f)[V][8], const void *p, int type, long long at, int D, int l) {
  if (!p) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[v][e] = 0.0f;
  } else if (type == TYPE_F32) {
    load_param_as<TYPE, TYPE_F32, G, V, VEC>(f, p, at, D, l);
  } else {
    load_param_as<TYPE, TYPE, G, V, VEC>(f, p, at, D, l);
  }
}

// ---- forward -------------------------------------------------------------------------------------------------------

// nb blocks per replica; a group takes every (nb GP)-th row
template <int TYPE, int G, int V, bool VEC>
__global__ void __launch_bounds__(ln_threads(G)) ln_forward_kernel(const LayerNormP p, const int nb) {
  constexpr int GP = ln_threads(G) / G;
  __shared__ __attribute__((aligned(16))) float sm[ln_threads(G) / 32];
  const int m = blockIdx.x / nb, j = blockIdx.x - m * nb, gid = threadIdx.x / G, l = threadIdx.x % G;
  const long long rows = (long long)p.b * p.T;
  const int D = p.D;
  const float n = (float)D;                       // (divided by, not multiplied with its inverse: rows of one value have variance 0)
  int turn = 0;
  const long long step = (long long)nb * GP;
  long long r = (long long)j * GP + gid;
  Raw<TYPE, V> next;                              // (the next row is on its way while a row is worked on)
  if (r < rows) load_raw<TYPE, G, V, VEC>(next, p.x, m * p.sx + r * p.ldx, D, l);
  float ga[V][8], be[V][8];
  load_param<TYPE, G, V, VEC>(ga, p.gamma, p.ptype, (long long)m * D, D, l);
  load_param<TYPE, G, V, VEC>(be, p.beta, p.ptype, (long long)m * D, D, l);
  for (; r < rows; r += step) {
    const Raw<TYPE, V> raw = next;
    if (r + step < rows) load_raw<TYPE, G, V, VEC>(next, p.x, m * p.sx + (r + step) * p.ldx, D, l);
    float x[V][8], s[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw_vals<TYPE, V>(raw, v, x[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += x[v][e];        // (zeros beyond the row)
    }
    group_sums<G, 1>(s, sm, turn++);
    const float mean = s[0] / n;
    s[0] = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = col_of<TYPE, G>(v, e, l) < D ? x[v][e] - mean : 0.0f;
        x[v][e] = d;
        s[0] = fmaf(d, d, s[0]);
      }
    group_sums<G, 1>(s, sm, turn++);
    const float rstd = 1.0f / sqrtf(s[0] / n + p.eps);
    if (l == 0) {
      if (p.mean) p.mean[m * rows + r] = mean;
      if (p.rstd) p.rstd[m * rows + r] = rstd;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] = fmaf(x[v][e] * rstd, ga[v][e], be[v][e]);
      store_vals<TYPE, G, VEC>(p.y, m * p.sy + r * p.ldy, D, l, v, x[v]);
    }
  }
}

// Rows longer than the registers of a block hold: three passes over the row, the later two out of the caches.  A launch takes LN_LONG_ROWS rows:
// a grid counts its threads in 32 bits.  (Blocks that take several rows one after the other need 1.1 to 1.2 times as long.)
constexpr int LN_LONG_ROWS = 1 << 18;
__global__ void __launch_bounds__(256) ln_forward_long_kernel(const LayerNormP p, const long long first) {
  __shared__ __attribute__((aligned(16))) float sm[8];
  const long long rows = (long long)p.b * p.T, i = first + blockIdx.x, m = i / rows, r = i - m * rows;
  const long long xa = m * p.sx + r * p.ldx, ya = m * p.sy + r * p.ldy, pa = m * p.D;
  const float n = (float)p.D;
  float s[1] = {0.0f};
  for (int c = threadIdx.x; c < p.D; c += 256) s[0] += load_as_f32(p.x, p.type, xa + c);
  group_sums<256, 1>(s, sm, 0);
  const float mean = s[0] / n;
  s[0] = 0.0f;
  for (int c = threadIdx.x; c < p.D; c += 256) {
    const float d = load_as_f32(p.x, p.type, xa + c) - mean;
    s[0] = fmaf(d, d, s[0]);
  }
  group_sums<256, 1>(s, sm, 1);
  const float rstd = 1.0f / sqrtf(s[0] / n + p.eps);
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[m * rows + r] = mean;
    if (p.rstd) p.rstd[m * rows + r] = rstd;
  }
  for (int c = threadIdx.x; c < p.D; c += 256) {
    const float xh = (load_as_f32(p.x, p.type, xa + c) - mean) * rstd;
    store_from_f32(p.y, p.type, ya + c, fmaf(xh, load_as_f32(p.gamma, p.ptype, pa + c), p.beta ? load_as_f32(p.beta, p.ptype, pa + c) : 0.0f));
  }
}

// ---- backward ------------------------------------------------------------------------------------------------------

enum { STAT_NONE = 0, STAT_ROW = 1, STAT_SAMPLE = 2 };   // n_i: not here; of samples that are one row; of samples of several

// How the rows of a replica are dealt to its nb blocks: `per` whole samples each, a sample to a group (chunks == 0; without statistics
// every row is a sample), or a sample's rows in `chunks` blocks of `per` rows.
struct LnSplit {
  int samples, T, nb, chunks, per;
  int tiles;             // column tiles of a row longer than a block's registers
  float *part;           // [M nb][2][D] partial sums of dy xh and dy
  float *npart;          // [tiles][M samples] partial n (tiles > 1 or chunks > 0)
  const float *sums;     // [M rows][2] mean_d h, mean_d(h xh) of long rows
};

template <int TYPE, int G, int V, bool VEC, int R, int STAT, bool LONG>
__global__ void __launch_bounds__(ln_threads(G), V == 1 && TYPE != TYPE_F32 && STAT != STAT_SAMPLE ? 4 : 1) ln_backward_kernel(const LayerNormP p, const LnSplit w) {
  constexpr int GP = ln_threads(G) / G;
  constexpr int NS = STAT == STAT_NONE ? 2 : 3;
  static_assert(!LONG || G == 256, "a tile of a long row is a block's");
  __shared__ __attribute__((aligned(16))) float sm[2 * R * NS * (ln_threads(G) / 64)];
  __shared__ float comb[GP > 1 ? GP * G * V * 8 : 1];
  const int bid = LONG ? blockIdx.x / w.tiles : blockIdx.x, tile = LONG ? blockIdx.x - bid * w.tiles : 0;
  const int m = bid / w.nb, j = bid - m * w.nb, gid = threadIdx.x / G, l = threadIdx.x % G;
  const int c0 = tile * G * V * 8, D = min(p.D - c0, G * V * 8);      // this block's columns
  const long long rows = (long long)p.b * p.T;
  const float inv = 1.0f / (float)p.D;
  // the group's rows: count of them, the q-th at row(q); samples end where t == T - 1
  long long first, count, hop;
  const int T = w.T;
  if (w.chunks > 0) {
    const int i = j / w.chunks, ch = j - i * w.chunks;
    const long long r0 = (long long)i * T + (long long)ch * w.per, r1 = min(r0 + w.per, (long long)(i + 1) * T);
    first = r0 + gid;
    count = first < r1 ? (r1 - first + GP - 1) / GP : 0;
    hop = GP;
  } else {
    const long long i0 = (long long)j * w.per + gid, i1 = min((long long)(j + 1) * w.per, (long long)w.samples);
    first = i0 * T;
    count = i0 < i1 ? (i1 - i0 + GP - 1) / GP * T : 0;
    hop = 0;                                      // rows of a sample, then the sample GP further on
  }
  float ga[V][8], tw[V][8], tb[V][8], gw[STAT == STAT_SAMPLE ? V : 1][8], gb[STAT == STAT_SAMPLE ? V : 1][8];
  load_param<TYPE, G, V, VEC>(ga, p.gamma, p.ptype, (long long)m * p.D + c0, D, l);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      tw[v][e] = tb[v][e] = 0.0f;
      if (STAT == STAT_SAMPLE) gw[v][e] = gb[v][e] = 0.0f;
    }
  const bool bias = p.dbeta != nullptr;
  int turn = 0, t = 0;
  long long row = first;
  // R rows at a time: their loads are under way together (of the first row again where there are fewer), and one exchange adds up what
  // all of them need
  for (long long q = 0; q < count; q += R, ++turn) {
    Raw<TYPE, V> rx[R], ry[R];
    float mean[R], rstd[R], s[R * NS];
    long long at[R];
    bool ends[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const bool in = q + k < count;
      const long long from = in ? row : first;
      load_raw<TYPE, G, V, VEC>(rx[k], p.x, m * p.sx + from * p.ldx + c0, D, l);
      load_raw<TYPE, G, V, VEC>(ry[k], p.dy, m * p.sy + from * p.ldy + c0, D, l);
      mean[k] = p.mean[m * rows + from];
      rstd[k] = p.rstd[m * rows + from];
      at[k] = in ? row : -1;
      ends[k] = in && t == T - 1;
      if (hop) row += hop;
      else if (ends[k]) { t = 0; row += (long long)(GP - 1) * T + 1; }
      else { ++t; ++row; }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float s1 = 0.0f, s2 = 0.0f, sn = 0.0f;
      if (at[k] >= 0) {                           // (a branch, so that rows are worked on one after the other: all at once take twice the registers)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float x[8], dy[8];
          raw_vals<TYPE, V>(rx[k], v, x);
          raw_vals<TYPE, V>(ry[k], v, dy);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float xh = (x[e] - mean_at<TYPE, G, VEC>(v, e, l, D, mean[k])) * rstd[k], h = dy[e] * ga[v][e], dw = dy[e] * xh;
            s1 += h;
            s2 = fmaf(h, xh, s2);
            if (STAT == STAT_SAMPLE) { gw[v][e] += dw; gb[v][e] += dy[e]; }
            else { tw[v][e] += dw; tb[v][e] += dy[e]; }
            if (STAT == STAT_ROW) {
              sn = fmaf(dw, dw, sn);
              if (bias) sn = fmaf(dy[e], dy[e], sn);
            }
          }
        }
        if (STAT == STAT_SAMPLE && ends[k]) {
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              sn = fmaf(gw[v][e], gw[v][e], sn);
              if (bias) sn = fmaf(gb[v][e], gb[v][e], sn);
              tw[v][e] += gw[v][e]; tb[v][e] += gb[v][e];
              gw[v][e] = gb[v][e] = 0.0f;
            }
        }
      }
      s[k * NS] = s1;
      s[k * NS + 1] = s2;
      if (NS == 3) s[k * NS + 2] = sn;
    }
    if (!LONG || NS == 3) group_sums<G, R * NS>(s, sm, turn);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (at[k] < 0) continue;
      forget(rx[k]);                              // (more work-groups to a CU: rows of 2048 205 -> 190 us)
      forget(ry[k]);
      float a = s[k * NS] * inv, c = s[k * NS + 1] * inv;
      if (LONG) { a = w.sums[(m * rows + at[k]) * 2]; c = w.sums[(m * rows + at[k]) * 2 + 1]; }
      if (STAT != STAT_NONE && ends[k] && l == 0) {
        const long long i = (long long)m * p.b + at[k] / T;
        if (LONG) w.npart[(long long)tile * p.M * p.b + i] = s[k * NS + 2];
        else p.n[i] = s[k * NS + 2];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[8], dy[8], d[8];
        raw_vals<TYPE, V>(rx[k], v, x);
        raw_vals<TYPE, V>(ry[k], v, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float xh = (x[e] - mean[k]) * rstd[k];
          d[e] = rstd[k] * (fmaf(dy[e], ga[v][e], -a) - xh * c);
        }
        store_vals<TYPE, G, VEC>(p.dx, m * p.sdx + at[k] * p.lddx + c0, D, l, v, d);
      }
    }
  }
  // the block's partial: groups added in order through LDS
  float *out = w.part + ((long long)m * w.nb + j) * 2 * p.D + c0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (GP == 1) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = col_of<TYPE, G>(v, e, l);
          if (c < D) out[(long long)h * p.D + c] = h ? tb[v][e] : tw[v][e];
        }
    } else {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) comb[gid * G * V * 8 + col_of<TYPE, G>(v, e, l)] = h ? tb[v][e] : tw[v][e];
      __syncthreads();
      for (int c = threadIdx.x; c < D; c += 256) {
        float a = 0.0f;
#pragma unroll
        for (int g = 0; g < GP; ++g) a += comb[g * G * V * 8 + c];
        out[(long long)h * p.D + c] = a;
      }
    }
  }
}

// mean_d h and mean_d(h xh) of long rows
__global__ void __launch_bounds__(256) ln_row_sums_kernel(const LayerNormP p, float *sums) {
  __shared__ __attribute__((aligned(16))) float sm[16];
  const long long rows = (long long)p.b * p.T, m = blockIdx.x / rows, r = blockIdx.x - m * rows;
  const float mean = p.mean[m * rows + r], rstd = p.rstd[m * rows + r], inv = 1.0f / (float)p.D;
  float s[2] = {0.0f, 0.0f};
  for (int c = threadIdx.x; c < p.D; c += 256) {
    const float h = load_as_f32(p.dy, p.type, m * p.sy + r * p.ldy + c) * load_as_f32(p.gamma, p.ptype, m * p.D + c);
    s[0] += h;
    s[1] = fmaf(h, (load_as_f32(p.x, p.type, m * p.sx + r * p.ldx + c) - mean) * rstd, s[1]);
  }
  group_sums<256, 2>(s, sm, 0);
  if (threadIdx.x == 0) { sums[blockIdx.x * 2LL] = s[0] * inv; sums[blockIdx.x * 2LL + 1] = s[1] * inv; }
}

// Sample spread over blocks: g_i = sum of its chunks' partials, left in the first of them; n_i's share of 256 columns.
__global__ void __launch_bounds__(256) ln_sample_kernel(const LayerNormP p, const LnSplit w, const int tiles) {
  __shared__ double sm[4];
  const int i = blockIdx.x / tiles, tile = blockIdx.x - i * tiles, c = tile * 256 + threadIdx.x;      // i = m b + sample
  float *part = w.part + (long long)i * w.chunks * 2 * p.D;
  float g = 0.0f;
  if (c < 2 * p.D) {
#pragma unroll 8
    for (int k = 0; k < w.chunks; ++k) g += part[(long long)k * 2 * p.D + c];
    part[c] = g;
  }
  const double n = block_sum<4>(c < (p.dbeta ? 2 : 1) * p.D ? (double)g * g : 0.0, sm);
  if (threadIdx.x == 0 && w.npart) w.npart[(long long)tile * p.M * p.b + i] = (float)n;
}

// gbar = (1 / b) sum of the partials j step, j < count, in order; further blocks add n_i's shares.
constexpr int FIN = 8;                   // wavefronts of a block, each with a part of the partials
__global__ void __launch_bounds__(FIN * 64) ln_finish_kernel(const LayerNormP p, const LnSplit w, const int count, const int step, const int colblocks, const int nshares) {
  __shared__ float sm[FIN][64];
  const int nfin = colblocks * p.M;
  if ((int)blockIdx.x >= nfin) {
    const long long i = (blockIdx.x - nfin) * (FIN * 64LL) + threadIdx.x, n = (long long)p.M * p.b;
    if (i >= n) return;
    float a = 0.0f;
    for (int k = 0; k < nshares; ++k) a += w.npart[k * n + i];
    p.n[i] = a;
    return;
  }
  const int m = blockIdx.x / colblocks, c = (blockIdx.x - m * colblocks) * 64 + (threadIdx.x & 63), q = threadIdx.x >> 6;
  const int per = (count + FIN - 1) / FIN, j1 = min(count, (q + 1) * per);
  const float *part = w.part + (long long)m * w.nb * 2 * p.D + c;
  float a = 0.0f;
  if (c < 2 * p.D) {
#pragma unroll 8
    for (int j = q * per; j < j1; ++j) a += part[(long long)j * step * 2 * p.D];
  }
  sm[q][threadIdx.x & 63] = a;
  __syncthreads();
  if (q == 0 && c < 2 * p.D) {
    const int k = threadIdx.x & 63;
    float g = 0.0f;
#pragma unroll
    for (int f = 0; f < FIN; ++f) g += sm[f][k];
    g *= 1.0f / (float)p.b;
    if (c < p.D) p.dgamma[(long long)m * p.D + c] = g;
    else if (p.dbeta) p.dbeta[(long long)m * p.D + c - p.D] = g;
  }
}

// q_i from the sums that ln_sample_kernel left
__global__ void __launch_bounds__(256) ln_inner_partials_kernel(const LayerNormP p, const LnSplit w) {
  __shared__ double sm[4];
  const int i = blockIdx.x, m = i / p.b;
  const float *g = w.part + (long long)i * w.chunks * 2 * p.D;
  double a = 0.0;
  for (int c = threadIdx.x; c < p.D; c += 256) {
    a += (double)g[c] * p.dgamma[(long long)m * p.D + c];
    if (p.dbeta) a += (double)g[p.D + c] * p.dbeta[(long long)m * p.D + c];
  }
  a = block_sum<4>(a, sm);
  if (threadIdx.x == 0) p.q[i] = (float)a;
}

// q_i from a second look at the rows: sum_t sum_d dy (xh gbar_gamma + gbar_beta).  gbar stays in a group's registers, which takes
// every (nb GP)-th sample of a replica.
template <int TYPE, int G, int V, bool VEC>
__global__ void __launch_bounds__(ln_threads(G)) ln_inner_rows_kernel(const LayerNormP p, const int nb) {
  constexpr int GP = ln_threads(G) / G;
  __shared__ __attribute__((aligned(16))) float sm[ln_threads(G) / 32];
  const int m = blockIdx.x / nb, j = blockIdx.x - m * nb, gid = threadIdx.x / G, l = threadIdx.x % G, D = p.D;
  const long long rows = (long long)p.b * p.T;
  float gw[V][8], gb[V][8];
  load_param<TYPE, G, V, VEC>(gw, p.dgamma, TYPE_F32, (long long)m * D, D, l);
  load_param<TYPE, G, V, VEC>(gb, p.dbeta, TYPE_F32, (long long)m * D, D, l);
  int turn = 0;
  for (long long i = j * GP + gid; i < p.b; i += nb * GP) {
    float s[1] = {0.0f};
    for (int t = 0; t < p.T; ++t) {
      const long long r = i * p.T + t;
      Raw<TYPE, V> rx, ry;
      load_raw<TYPE, G, V, VEC>(rx, p.x, m * p.sx + r * p.ldx, D, l);
      load_raw<TYPE, G, V, VEC>(ry, p.dy, m * p.sy + r * p.ldy, D, l);
      const float mean = p.mean[m * rows + r], rstd = p.rstd[m * rows + r];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[8], dy[8];
        raw_vals<TYPE, V>(rx, v, x);
        raw_vals<TYPE, V>(ry, v, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(dy[e], fmaf((x[e] - mean_at<TYPE, G, VEC>(v, e, l, D, mean)) * rstd, gw[v][e], gb[v][e]), s[0]);
      }
    }
    group_sums<G, 1>(s, sm, turn++);
    if (l == 0) p.q[(long long)m * p.b + i] = s[0];
  }
}

// The same of long rows, a wavefront to a sample
__global__ void __launch_bounds__(256) ln_inner_long_kernel(const LayerNormP p) {
  const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long long)p.b * p.T;
  if (i >= (long long)p.M * p.b) return;
  const int l = threadIdx.x & 63;
  const long long m = i / p.b, r0 = (i - m * p.b) * p.T;
  float a = 0.0f;
  for (int t = 0; t < p.T; ++t) {
    const long long r = r0 + t, xa = m * p.sx + r * p.ldx, ya = m * p.sy + r * p.ldy;
    const float mean = p.mean[m * rows + r], rstd = p.rstd[m * rows + r];
    for (int c = l; c < p.D; c += 64) {
      const float xh = (load_as_f32(p.x, p.type, xa + c) - mean) * rstd;
      a = fmaf(load_as_f32(p.dy, p.type, ya + c), fmaf(xh, p.dgamma[m * p.D + c], p.dbeta ? p.dbeta[m * p.D + c] : 0.0f), a);
    }
  }
  a = lanes_sum<64>(a);
  if (l == 0) p.q[i] = a;
}

// ---- choices -------------------------------------------------------------------------------------------------------

constexpr int LN_MAX_D = 8192;           // longest row that a block's registers hold
// Blocks of the backward pass: two to a CU of 256 threads, one of 512.  Their loads keep memory as busy as those of more blocks, which leave
// more partials and, where registers hold only two or three of them on a CU, a last round (8 x 8192 rows of 2048: 512 blocks 170 us, 768
// 184, 1024 176; 4 x 4096 rows of 4096 98, 107, 118).  Whole samples make fewer where their number is just past a multiple of the blocks
// (n_i of 512 samples of 64 rows of 2048 79 us, of 513 in 257 blocks of two 106, of 600 121).
constexpr int LN_BLOCKS = 512;

// lanes and vectors to a row: 16 x 1, 64 x 1, 64 x 2, 256 x 1, 256 x 2, 512 x 2 (256 x 4 fill the registers with one row: gradients of
// 2 x 8 x 512 rows of 8192 in bf16 114 us, here 99; 5 x 219 x 13 of 4507 in fp16 with q_i 465, here 280)
int ln_shape(int D) { return D <= 128 ? 0 : D <= 512 ? 1 : D <= 1024 ? 2 : D <= 2048 ? 3 : D <= 4096 ? 4 : 5; }
int ln_groups(int D) { return D <= 128 ? 16 : D <= 1024 ? 4 : 1; }      // to a block
int ln_rows_at_once(int D) { return D > LN_MAX_D ? 4 : D > 2048 ? 2 : D > 1024 ? 4 : D > 512 ? 2 : 4; }      // of a group, backward

int ln_sample_tiles(const LayerNormP &p) { return (2 * p.D + 255) / 256; }

LnSplit ln_split(const LayerNormP &p, bool want, bool want_q) {
  LnSplit w;
  std::memset(&w, 0, sizeof(w));
  const long long rows = (long long)p.b * p.T, all = (long long)p.M * p.b;
  const int groups = ln_groups(p.D), once = ln_rows_at_once(p.D);
  w.tiles = p.D > LN_MAX_D ? (p.D + 2047) / 2048 : 1;
  // (blocks of 512 threads are alone on their CU)
  const long long blocks = std::max(1, LN_BLOCKS / (w.tiles > 1 ? w.tiles : p.D > 4096 ? 2 : 1)), most = std::max(1LL, blocks / p.M);
  const long long few = (long long)once * groups;            // rows of a block at least: one round of its groups' loads
  w.samples = want ? p.b : (int)rows; w.T = want ? p.T : 1;
  // Blocks to a sample, whose partials a further launch adds, or samples to a group: what the partials cost (a launch, and bytes as five rows
  // have) against groups left idle, and against the second look at the rows that q_i takes otherwise.  us, blocks to a sample against samples
  // to a group: n_i of 5 x 2 samples of 124 rows of 345 14 / 106, 12 x 90 of 227 of 251 172 / 325, 16 x 64 of 64 of 512 42 / 52, but 8 x 32 of
  // 16 of 2048 28 / 22 and 16 x 512 of 64 of 96 66 / 60; with q_i 16 x 512 of 32 of 512 191 / 255, 16 x 128 of 64 of 512 85 / 119, but
  // 16 x 1024 of 32 of 96 98 / 91.
  const bool idle = w.T >= 4 * once && all * (w.T >= 32 || groups > 1 ? 2 : 4) <= blocks * groups, less = w.T >= 128 && all <= blocks * groups;
  const bool fits = all * ln_sample_tiles(p) <= 1 << 23;     // (a grid counts its threads in 32 bits)
  if (want && fits && (idle || less || (want_q && w.T >= 32 && w.T >= few))) {
    // one round of rows to each of sixteen blocks, then up to four
    const long long rounds = (w.T + few - 1) / few;
    w.chunks = (int)std::max(1LL, std::min(blocks / all, std::min(rounds, std::max(16LL, (rounds + 3) / 4))));
    w.per = (int)((w.T + (long long)w.chunks - 1) / w.chunks);
    w.chunks = (int)((w.T + (long long)w.per - 1) / w.per);
    w.nb = w.samples * w.chunks;
    return w;
  }
  const long long nb = std::max(1LL, std::min(most, (rows + few - 1) / few));
  w.per = (int)((w.samples + nb - 1) / nb);
  w.nb = (int)((w.samples + (long long)w.per - 1) / w.per);
  return w;
}

struct LnPieces { size_t part, npart, sums, total; };
LnPieces ln_pieces(const LayerNormP &p, const LnSplit &w, bool want_n) {
  LnPieces q;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o = (o + bytes + 255) / 256 * 256; return r; };
  q.part = take((size_t)p.M * w.nb * 2 * p.D * 4);
  q.npart = take(want_n ? (size_t)p.M * p.b * 4 * (w.chunks > 0 ? ln_sample_tiles(p) : w.tiles > 1 ? w.tiles : 0) : 0);
  q.sums = take(w.tiles > 1 ? (size_t)p.M * p.b * p.T * 8 : 0);
  q.total = o;
  return q;
}

template <int TYPE, int G, int V, bool VEC, int R, bool LONG>
hipError_t backward_stat(const LayerNormP &p, const LnSplit &w, bool want_n, hipStream_t s) {
  const long long blocks = (long long)p.M * w.nb * w.tiles;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(ln_threads(G));
  if (!want_n || w.chunks > 0) hipLaunchKernelGGL((ln_backward_kernel<TYPE, G, V, VEC, R, STAT_NONE, LONG>), grid, block, 0, s, p, w);
  else if (w.T == 1) hipLaunchKernelGGL((ln_backward_kernel<TYPE, G, V, VEC, R, STAT_ROW, LONG>), grid, block, 0, s, p, w);
  else hipLaunchKernelGGL((ln_backward_kernel<TYPE, G, V, VEC, R, STAT_SAMPLE, LONG>), grid, block, 0, s, p, w);
  return hipGetLastError();
}
template <int TYPE, bool VEC>
hipError_t backward_shape(const LayerNormP &p, const LnSplit &w, bool want_n, hipStream_t s) {
  if (w.tiles > 1) return backward_stat<TYPE, 256, 1, VEC, 4, true>(p, w, want_n, s);
  switch (ln_shape(p.D)) {
    case 0: return backward_stat<TYPE, 16, 1, VEC, 4, false>(p, w, want_n, s);
    case 1: return backward_stat<TYPE, 64, 1, VEC, 4, false>(p, w, want_n, s);
    case 2: return backward_stat<TYPE, 64, 2, VEC, 2, false>(p, w, want_n, s);
    case 3: return backward_stat<TYPE, 256, 1, VEC, 4, false>(p, w, want_n, s);
    case 4: return backward_stat<TYPE, 256, 2, VEC, 2, false>(p, w, want_n, s);
    default: return backward_stat<TYPE, 512, 2, VEC, 2, false>(p, w, want_n, s);
  }
}

// Blocks per replica of the kernels whose groups take one row or sample after the other
int ln_row_blocks(const LayerNormP &p, long long items, int groups) {
  return (int)std::max(1LL, std::min((items + groups - 1) / groups, (4LL * LN_BLOCKS + p.M - 1) / p.M));
}
struct Forward {
  template <int TYPE, int G, int V, bool VEC> static void go(const LayerNormP &p, hipStream_t s) {
    const int nb = ln_row_blocks(p, (long long)p.b * p.T, ln_threads(G) / G);
    hipLaunchKernelGGL((ln_forward_kernel<TYPE, G, V, VEC>), dim3((unsigned)((long long)nb * p.M)), dim3(ln_threads(G)), 0, s, p, nb);
  }
};
struct Inner {
  template <int TYPE, int G, int V, bool VEC> static void go(const LayerNormP &p, hipStream_t s) {
    const int nb = ln_row_blocks(p, p.b, ln_threads(G) / G);
    hipLaunchKernelGGL((ln_inner_rows_kernel<TYPE, G, V, VEC>), dim3((unsigned)((long long)nb * p.M)), dim3(ln_threads(G)), 0, s, p, nb);
  }
};
template <class K, int TYPE, bool VEC> void by_shape(const LayerNormP &p, hipStream_t s) {
  switch (ln_shape(p.D)) {
    case 0: return K::template go<TYPE, 16, 1, VEC>(p, s);
    case 1: return K::template go<TYPE, 64, 1, VEC>(p, s);
    case 2: return K::template go<TYPE, 64, 2, VEC>(p, s);
    case 3: return K::template go<TYPE, 256, 1, VEC>(p, s);
    case 4: return K::template go<TYPE, 256, 2, VEC>(p, s);
    default: return K::template go<TYPE, 512, 2, VEC>(p, s);
  }
}
template <class K> hipError_t by_type(const LayerNormP &p, bool vec, hipStream_t s) {
  switch (p.type) {
    case TYPE_F32: vec ? by_shape<K, TYPE_F32, true>(p, s) : by_shape<K, TYPE_F32, false>(p, s); break;
    case TYPE_BF16: vec ? by_shape<K, TYPE_BF16, true>(p, s) : by_shape<K, TYPE_BF16, false>(p, s); break;
    default: vec ? by_shape<K, TYPE_F16, true>(p, s) : by_shape<K, TYPE_F16, false>(p, s);
  }
  return hipGetLastError();
}

}  // namespace

size_t layer_norm_backward_bytes(const LayerNormP &p, bool want_n, bool want_q) {
  return ln_pieces(p, ln_split(p, want_n || want_q, want_q), want_n).total;
}

hipError_t launch_layer_norm(const LayerNormP &p, hipStream_t s) {
  const long long rows = (long long)p.b * p.T;
  if (rows == 0) return hipSuccess;
  if (rows * p.M > 0x7fffffff) return hipErrorInvalidValue;
  if (p.D > LN_MAX_D) {
    for (long long first = 0; first < rows * p.M; first += LN_LONG_ROWS)
      hipLaunchKernelGGL(ln_forward_long_kernel, dim3((unsigned)std::min<long long>(rows * p.M - first, LN_LONG_ROWS)), dim3(256), 0, s, p, first);
    return hipGetLastError();
  }
  return by_type<Forward>(p, rows_of_vectors(p.x, p.type, p.sx, p.ldx, p.D) && rows_of_vectors(p.y, p.type, p.sy, p.ldy, p.D), s);
}

hipError_t launch_layer_norm_backward(const LayerNormP &p, void *workspace, hipStream_t s) {
  const long long rows = (long long)p.b * p.T;
  if (rows * p.M > 0x7fffffff) return hipErrorInvalidValue;
  const bool want_n = p.n != nullptr, want = want_n || p.q;
  LnSplit w = ln_split(p, want, p.q != nullptr);
  const LnPieces at = ln_pieces(p, w, want_n);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  w.part = reinterpret_cast<float *>(ws + at.part);
  w.npart = want_n ? reinterpret_cast<float *>(ws + at.npart) : nullptr;
  if (w.tiles > 1) {
    float *sums = reinterpret_cast<float *>(ws + at.sums);
    hipLaunchKernelGGL(ln_row_sums_kernel, dim3((unsigned)(rows * p.M)), dim3(256), 0, s, p, sums);
    w.sums = sums;
  }
  const bool vec = rows_of_vectors(p.x, p.type, p.sx, p.ldx, p.D) && rows_of_vectors(p.dy, p.type, p.sy, p.ldy, p.D) &&
                   rows_of_vectors(p.dx, p.type, p.sdx, p.lddx, p.D);
  hipError_t e;
  switch (p.type) {
    case TYPE_F32: e = vec ? backward_shape<TYPE_F32, true>(p, w, want_n, s) : backward_shape<TYPE_F32, false>(p, w, want_n, s); break;
    case TYPE_BF16: e = vec ? backward_shape<TYPE_BF16, true>(p, w, want_n, s) : backward_shape<TYPE_BF16, false>(p, w, want_n, s); break;
    default: e = vec ? backward_shape<TYPE_F16, true>(p, w, want_n, s) : backward_shape<TYPE_F16, false>(p, w, want_n, s); break;
  }
  if (e != hipSuccess) return e;
  int nshares = 0;
  if (w.chunks > 0) {
    nshares = ln_sample_tiles(p);
    hipLaunchKernelGGL(ln_sample_kernel, dim3((unsigned)((long long)p.M * p.b * nshares)), dim3(256), 0, s, p, w, nshares);
    if (!want_n) nshares = 0;
  } else if (w.tiles > 1 && want_n) {
    nshares = w.tiles;
  }
  const int colblocks = (2 * p.D + 63) / 64;
  const int count = w.chunks > 0 ? w.samples : w.nb, step = std::max(1, w.chunks);
  const long long nblocks = nshares ? ((long long)p.M * p.b + FIN * 64 - 1) / (FIN * 64) : 0;
  hipLaunchKernelGGL(ln_finish_kernel, dim3((unsigned)((long long)colblocks * p.M + nblocks)), dim3(FIN * 64), 0, s, p, w, count, step, colblocks, nshares);
  if (p.q) {
    if (w.chunks > 0) hipLaunchKernelGGL(ln_inner_partials_kernel, dim3((unsigned)((long long)p.M * p.b)), dim3(256), 0, s, p, w);
    else if (p.D > LN_MAX_D) hipLaunchKernelGGL(ln_inner_long_kernel, dim3((unsigned)(((long long)p.M * p.b + 3) / 4)), dim3(256), 0, s, p);
    else return by_type<Inner>(p, vec, s);
  }
  return hipGetLastError();
}

}  // namespace absk
