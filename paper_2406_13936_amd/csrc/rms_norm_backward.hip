// Gradients of the root-mean-square norm (rms_norm.hip) and the statistics that the batch tests take of its gain's.
//
//   hh = h r,  u = dy w,  dx = dh + r (u - hh mean_d(u hh))      (of x and of the residual alike; dh: what else arrives at h)
//   sample i (T rows):  g_i = sum_t dy hh,  gbar = mean_i g_i,  n_i = ||g_i||^2,  q_i = <g_i, gbar>
//
// Bound by memory: h, dy and dh are read, dx written, once each.  As in layer_norm.hip a row stays in the registers of a group of lanes,
// the lanes that own a column keep its part of gbar over all rows of a block, every block leaves one partial, and a second launch
// adds them in order.  8 x 16 samples of 512 rows of 2048 in bf16 with dh and n_i: 211 us, 5.1 TB/s.  Arithmetic and sums are fp32; of samples spread over blocks n_i is added in fp64 over 256 columns at a time.
#include <algorithm>
#include <cstring>
#include "device_utils.h"
#include "ops.h"
#include "row_groups.h"

namespace absk {
namespace {

enum { STAT_NONE = 0, STAT_ROW = 1, STAT_SAMPLE = 2 };   // n_i: not here; of samples that are one row; of samples of several

// How the rows of a replica are dealt to its nb blocks: `per` whole samples each, a sample to a group (chunks == 0; without statistics
// every row is a sample), or a sample's rows in `chunks` blocks of `per` rows.
struct RmsSplit {
  int samples, T, nb, chunks, per;
  int tiles;             // column tiles of a row longer than a block's registers
  float *part;           // [M nb][D] partial sums of dy hh
  float *npart;          // [tiles][M samples] partial n (tiles > 1 or chunks > 0)
  const float *sums;     // [M rows] mean_d(u hh) of long rows
};

template <int TYPE, int G, int V, bool VEC, int R, int STAT, bool ADD, bool LONG>
__global__ void __launch_bounds__(ln_threads(G), V == 1 && TYPE != TYPE_F32 && STAT != STAT_SAMPLE ? 4 : 1) rms_backward_kernel(const RmsNormP p, const RmsSplit w) {
  constexpr int GP = ln_threads(G) / G;
  constexpr int NS = STAT == STAT_NONE ? 1 : 2;
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
  float ga[V][8], tw[V][8], gw[STAT == STAT_SAMPLE ? V : 1][8];
  load_param<TYPE, G, V, VEC>(ga, p.w, p.ptype, (long long)m * p.D + c0, D, l);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      tw[v][e] = 0.0f;
      if (STAT == STAT_SAMPLE) gw[v][e] = 0.0f;
    }
  int turn = 0, t = 0;
  long long row = first;
  // R rows at a time: their loads are under way together (of the first row again where there are fewer), and one exchange adds up what
  // all of them need
  for (long long q = 0; q < count; q += R, ++turn) {
    Raw<TYPE, V> rx[R], ry[R], rz[ADD ? R : 1];
    float rstd[R], s[R * NS];
    long long at[R];
    bool ends[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const bool in = q + k < count;
      const long long from = in ? row : first;
      load_raw<TYPE, G, V, VEC>(rx[k], p.x, m * p.sx + from * p.ldx + c0, D, l);
      load_raw<TYPE, G, V, VEC>(ry[k], p.dy, m * p.sy + from * p.ldy + c0, D, l);
      if (ADD) load_raw<TYPE, G, V, VEC>(rz[k], p.res, m * p.sr + from * p.ldr + c0, D, l);
      rstd[k] = p.rstd[m * rows + from];
      at[k] = in ? row : -1;
      ends[k] = in && t == T - 1;
      if (hop) row += hop;
      else if (ends[k]) { t = 0; row += (long long)(GP - 1) * T + 1; }
      else { ++t; ++row; }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float s2 = 0.0f, sn = 0.0f;
      if (at[k] >= 0) {                           // (a branch, so that rows are worked on one after the other)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float x[8], dy[8];
          raw_vals<TYPE, V>(rx[k], v, x);
          raw_vals<TYPE, V>(ry[k], v, dy);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float hh = x[e] * rstd[k], dw = dy[e] * hh;
            s2 = fmaf(dy[e] * ga[v][e], hh, s2);
            if (STAT == STAT_SAMPLE) gw[v][e] += dw;
            else tw[v][e] += dw;
            if (STAT == STAT_ROW) sn = fmaf(dw, dw, sn);
          }
        }
        if (STAT == STAT_SAMPLE && ends[k]) {
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              sn = fmaf(gw[v][e], gw[v][e], sn);
              tw[v][e] += gw[v][e];
              gw[v][e] = 0.0f;
            }
        }
      }
      s[k * NS] = s2;
      if (NS == 2) s[k * NS + 1] = sn;
    }
    if (!LONG || NS == 2) group_sums<G, R * NS>(s, sm, turn);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (at[k] < 0) continue;
      forget(rx[k]);                              // (more work-groups to a CU)
      forget(ry[k]);
      const float c = LONG ? w.sums[m * rows + at[k]] : s[k * NS] * inv;
      if (STAT != STAT_NONE && ends[k] && l == 0) {
        const long long i = (long long)m * p.b + at[k] / T;
        if (LONG) w.npart[(long long)tile * p.M * p.b + i] = s[k * NS + NS - 1];
        else p.n[i] = s[k * NS + NS - 1];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[8], dy[8], d[8], z[8];
        raw_vals<TYPE, V>(rx[k], v, x);
        raw_vals<TYPE, V>(ry[k], v, dy);
        if (ADD) raw_vals<TYPE, V>(rz[ADD ? k : 0], v, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float g = fmaf(-(x[e] * rstd[k]), c, dy[e] * ga[v][e]);
          d[e] = ADD ? fmaf(rstd[k], g, z[e]) : rstd[k] * g;
        }
        store_vals<TYPE, G, VEC>(p.dx, m * p.sh + at[k] * p.ldh + c0, D, l, v, d);
      }
    }
  }
  // the block's partial: groups added in order through LDS
  float *out = w.part + ((long long)m * w.nb + j) * p.D + c0;
  if (GP == 1) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = col_of<TYPE, G>(v, e, l);
        if (c < D) out[c] = tw[v][e];
      }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) comb[gid * G * V * 8 + col_of<TYPE, G>(v, e, l)] = tw[v][e];
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += 256) {
      float a = 0.0f;
#pragma unroll
      for (int g = 0; g < GP; ++g) a += comb[g * G * V * 8 + c];
      out[c] = a;
    }
  }
}

// mean_d(u hh) of long rows
__global__ void __launch_bounds__(256) rms_row_sums_kernel(const RmsNormP p, float *sums, const long long first) {
  __shared__ __attribute__((aligned(16))) float sm[8];
  const long long rows = (long long)p.b * p.T, i = first + blockIdx.x, m = i / rows, r = i - m * rows;
  const float rstd = p.rstd[i], inv = 1.0f / (float)p.D;
  float s[1] = {0.0f};
  for (int c = threadIdx.x; c < p.D; c += 256)
    s[0] = fmaf(load_as_f32(p.dy, p.type, m * p.sy + r * p.ldy + c) * load_as_f32(p.w, p.ptype, m * p.D + c), load_as_f32(p.x, p.type, m * p.sx + r * p.ldx + c) * rstd, s[0]);
  group_sums<256, 1>(s, sm, 0);
  if (threadIdx.x == 0) sums[i] = s[0] * inv;
}

// Sample spread over blocks: g_i = sum of its chunks' partials, left in the first of them; n_i's share of 256 columns.
__global__ void __launch_bounds__(256) rms_sample_kernel(const RmsNormP p, const RmsSplit w, const int tiles) {
  __shared__ double sm[4];
  const int i = blockIdx.x / tiles, tile = blockIdx.x - i * tiles, c = tile * 256 + threadIdx.x;      // i = m b + sample
  float *part = w.part + (long long)i * w.chunks * p.D;
  float g = 0.0f;
  if (c < p.D) {
#pragma unroll 8
    for (int k = 0; k < w.chunks; ++k) g += part[(long long)k * p.D + c];
    part[c] = g;
  }
  const double n = block_sum<4>((double)g * g, sm);
  if (threadIdx.x == 0 && w.npart) w.npart[(long long)tile * p.M * p.b + i] = (float)n;
}

// gbar = (1 / b) sum of the partials j step, j < count, in order; further blocks add n_i's shares.
constexpr int FIN = 8;                   // wavefronts of a block, each with a part of the partials
__global__ void __launch_bounds__(FIN * 64) rms_finish_kernel(const RmsNormP p, const RmsSplit w, const int count, const int step, const int colblocks, const int nshares) {
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
  const int m = blockIdx.x / colblocks, k = threadIdx.x & 63, c = (blockIdx.x - m * colblocks) * 64 + k, q = threadIdx.x >> 6;
  const int per = (count + FIN - 1) / FIN, j1 = min(count, (q + 1) * per);
  const float *part = w.part + (long long)m * w.nb * p.D + c;
  float a = 0.0f;
  if (c < p.D) {
#pragma unroll 8
    for (int j = q * per; j < j1; ++j) a += part[(long long)j * step * p.D];
  }
  sm[q][k] = a;
  __syncthreads();
  if (q == 0 && c < p.D) {
    float g = 0.0f;
#pragma unroll
    for (int f = 0; f < FIN; ++f) g += sm[f][k];
    p.dw[(long long)m * p.D + c] = g * (1.0f / (float)p.b);
  }
}

// q_i from the sums that rms_sample_kernel left
__global__ void __launch_bounds__(256) rms_inner_partials_kernel(const RmsNormP p, const RmsSplit w) {
  __shared__ double sm[4];
  const int i = blockIdx.x, m = i / p.b;
  const float *g = w.part + (long long)i * w.chunks * p.D;
  double a = 0.0;
  for (int c = threadIdx.x; c < p.D; c += 256) a += (double)g[c] * p.dw[(long long)m * p.D + c];
  a = block_sum<4>(a, sm);
  if (threadIdx.x == 0) p.q[i] = (float)a;
}

// q_i from a second look at the rows: sum_t sum_d dy hh gbar.  gbar stays in a group's registers, which takes every (nb GP)-th sample
// of a replica.
template <int TYPE, int G, int V, bool VEC>
__global__ void __launch_bounds__(ln_threads(G)) rms_inner_rows_kernel(const RmsNormP p, const int nb) {
  constexpr int GP = ln_threads(G) / G;
  __shared__ __attribute__((aligned(16))) float sm[ln_threads(G) / 32];
  const int m = blockIdx.x / nb, j = blockIdx.x - m * nb, gid = threadIdx.x / G, l = threadIdx.x % G, D = p.D;
  const long long rows = (long long)p.b * p.T;
  float gw[V][8];
  load_param<TYPE, G, V, VEC>(gw, p.dw, TYPE_F32, (long long)m * D, D, l);
  int turn = 0;
  for (long long i = j * GP + gid; i < p.b; i += nb * GP) {
    float s[1] = {0.0f};
    for (int t = 0; t < p.T; ++t) {
      const long long r = i * p.T + t;
      Raw<TYPE, V> rx, ry;
      load_raw<TYPE, G, V, VEC>(rx, p.x, m * p.sx + r * p.ldx, D, l);
      load_raw<TYPE, G, V, VEC>(ry, p.dy, m * p.sy + r * p.ldy, D, l);
      const float rstd = p.rstd[m * rows + r];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[8], dy[8];
        raw_vals<TYPE, V>(rx, v, x);
        raw_vals<TYPE, V>(ry, v, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(dy[e] * (x[e] * rstd), gw[v][e], s[0]);
      }
    }
    group_sums<G, 1>(s, sm, turn++);
    if (l == 0) p.q[(long long)m * p.b + i] = s[0];
  }
}

// The same of long rows, a wavefront to a sample
__global__ void __launch_bounds__(256) rms_inner_long_kernel(const RmsNormP p) {
  const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long long)p.b * p.T;
  if (i >= (long long)p.M * p.b) return;
  const int l = threadIdx.x & 63;
  const long long m = i / p.b, r0 = (i - m * p.b) * p.T;
  float a = 0.0f;
  for (int t = 0; t < p.T; ++t) {
    const long long r = r0 + t;
    const float rstd = p.rstd[m * rows + r];
    for (int c = l; c < p.D; c += 64)
      a = fmaf(load_as_f32(p.dy, p.type, m * p.sy + r * p.ldy + c) * (load_as_f32(p.x, p.type, m * p.sx + r * p.ldx + c) * rstd), p.dw[m * p.D + c], a);
  }
  a = lanes_sum<64>(a);
  if (l == 0) p.q[i] = a;
}

// ---- choices -------------------------------------------------------------------------------------------------------

int rms_groups(int D) { return D <= 128 ? 16 : D <= 1024 ? 4 : 1; }      // to a block
int rms_rows_at_once(int D) { return D > RMS_MAX_D ? 4 : D > 2048 ? 2 : D > 1024 ? 4 : D > 512 ? 2 : 4; }      // of a group
int rms_sample_tiles(const RmsNormP &p) { return (p.D + 255) / 256; }

// The rule of layer norm's gradients (ln_split, whose comments have both sides of each line measured): the same reads and partials to a row
RmsSplit rms_split(const RmsNormP &p, bool want, bool want_q) {
  RmsSplit w;
  std::memset(&w, 0, sizeof(w));
  const long long rows = (long long)p.b * p.T, all = (long long)p.M * p.b;
  const int groups = rms_groups(p.D), once = rms_rows_at_once(p.D);
  w.tiles = p.D > RMS_MAX_D ? (p.D + 2047) / 2048 : 1;
  const long long blocks = std::max(1, RMS_BLOCKS / (w.tiles > 1 ? w.tiles : p.D > 4096 ? 2 : 1)), most = std::max(1LL, blocks / p.M);
  const long long few = (long long)once * groups;            // rows of a block at least: one round of its groups' loads
  w.samples = want ? p.b : (int)rows; w.T = want ? p.T : 1;
  const bool idle = w.T >= 4 * once && all * (w.T >= 32 || groups > 1 ? 2 : 4) <= blocks * groups, less = w.T >= 128 && all <= blocks * groups;
  const bool fits = all * rms_sample_tiles(p) <= 1 << 23;    // (a grid counts its threads in 32 bits)
  if (want && fits && (idle || less || (want_q && w.T >= 32 && w.T >= few))) {
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

struct RmsPieces { size_t part, npart, sums, total; };
RmsPieces rms_pieces(const RmsNormP &p, const RmsSplit &w, bool want_n) {
  RmsPieces q;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t r = o; o = (o + bytes + 255) / 256 * 256; return r; };
  q.part = take((size_t)p.M * w.nb * p.D * 4);
  q.npart = take(want_n ? (size_t)p.M * p.b * 4 * (w.chunks > 0 ? rms_sample_tiles(p) : w.tiles > 1 ? w.tiles : 0) : 0);
  q.sums = take(w.tiles > 1 ? (size_t)p.M * p.b * p.T * 4 : 0);
  q.total = o;
  return q;
}

template <int TYPE, int G, int V, bool VEC, int R, bool LONG, bool ADD>
hipError_t backward_stat(const RmsNormP &p, const RmsSplit &w, bool want_n, hipStream_t s) {
  const long long blocks = (long long)p.M * w.nb * w.tiles;
  if (blocks > 0x7fffffff / ln_threads(G)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(ln_threads(G));
  if (!want_n || w.chunks > 0) hipLaunchKernelGGL((rms_backward_kernel<TYPE, G, V, VEC, R, STAT_NONE, ADD, LONG>), grid, block, 0, s, p, w);
  else if (w.T == 1) hipLaunchKernelGGL((rms_backward_kernel<TYPE, G, V, VEC, R, STAT_ROW, ADD, LONG>), grid, block, 0, s, p, w);
  else hipLaunchKernelGGL((rms_backward_kernel<TYPE, G, V, VEC, R, STAT_SAMPLE, ADD, LONG>), grid, block, 0, s, p, w);
  return hipGetLastError();
}
template <int TYPE, int G, int V, bool VEC, int R, bool LONG>
hipError_t backward_add(const RmsNormP &p, const RmsSplit &w, bool want_n, hipStream_t s) {
  return p.res ? backward_stat<TYPE, G, V, VEC, R, LONG, true>(p, w, want_n, s) : backward_stat<TYPE, G, V, VEC, R, LONG, false>(p, w, want_n, s);
}
template <int TYPE, bool VEC>
hipError_t backward_shape(const RmsNormP &p, const RmsSplit &w, bool want_n, hipStream_t s) {
  if (w.tiles > 1) return backward_add<TYPE, 256, 1, VEC, 4, true>(p, w, want_n, s);
  switch (rms_shape(p.D)) {
    case 0: return backward_add<TYPE, 16, 1, VEC, 4, false>(p, w, want_n, s);
    case 1: return backward_add<TYPE, 64, 1, VEC, 4, false>(p, w, want_n, s);
    case 2: return backward_add<TYPE, 64, 2, VEC, 2, false>(p, w, want_n, s);
    case 3: return backward_add<TYPE, 256, 1, VEC, 4, false>(p, w, want_n, s);
    case 4: return backward_add<TYPE, 256, 2, VEC, 2, false>(p, w, want_n, s);
    default: return backward_add<TYPE, 512, 2, VEC, 2, false>(p, w, want_n, s);
  }
}
template <int TYPE, int G, int V, bool VEC> void inner_shape(const RmsNormP &p, hipStream_t s) {
  const long long groups = ln_threads(G) / G;
  const int nb = (int)std::max(1LL, std::min((p.b + groups - 1) / groups, (4LL * RMS_BLOCKS + p.M - 1) / p.M));
  hipLaunchKernelGGL((rms_inner_rows_kernel<TYPE, G, V, VEC>), dim3((unsigned)((long long)nb * p.M)), dim3(ln_threads(G)), 0, s, p, nb);
}
template <int TYPE, bool VEC> void inner_by_length(const RmsNormP &p, hipStream_t s) {
  switch (rms_shape(p.D)) {
    case 0: return inner_shape<TYPE, 16, 1, VEC>(p, s);
    case 1: return inner_shape<TYPE, 64, 1, VEC>(p, s);
    case 2: return inner_shape<TYPE, 64, 2, VEC>(p, s);
    case 3: return inner_shape<TYPE, 256, 1, VEC>(p, s);
    case 4: return inner_shape<TYPE, 256, 2, VEC>(p, s);
    default: return inner_shape<TYPE, 512, 2, VEC>(p, s);
  }
}

}  // namespace

size_t rms_norm_backward_bytes(const RmsNormP &p, bool want_n, bool want_q) {
  return rms_pieces(p, rms_split(p, want_n || want_q, want_q), want_n).total;
}

hipError_t launch_rms_norm_backward(const RmsNormP &p, void *workspace, hipStream_t s) {
  const long long rows = (long long)p.b * p.T;
  if (rows * p.M > 0x7fffffff) return hipErrorInvalidValue;
  const bool want_n = p.n != nullptr, want = want_n || p.q;
  RmsSplit w = rms_split(p, want, p.q != nullptr);
  const RmsPieces at = rms_pieces(p, w, want_n);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  w.part = reinterpret_cast<float *>(ws + at.part);
  w.npart = want_n ? reinterpret_cast<float *>(ws + at.npart) : nullptr;
  if (w.tiles > 1) {
    float *sums = reinterpret_cast<float *>(ws + at.sums);
    for (long long first = 0; first < rows * p.M; first += 1 << 18)      // (a grid counts its threads in 32 bits)
      hipLaunchKernelGGL(rms_row_sums_kernel, dim3((unsigned)std::min<long long>(rows * p.M - first, 1 << 18)), dim3(256), 0, s, p, sums, first);
    w.sums = sums;
  }
  const bool vec = rows_of_vectors(p.x, p.type, p.sx, p.ldx, p.D) && rows_of_vectors(p.dy, p.type, p.sy, p.ldy, p.D) &&
                   rows_of_vectors(p.dx, p.type, p.sh, p.ldh, p.D) && (!p.res || rows_of_vectors(p.res, p.type, p.sr, p.ldr, p.D));
  hipError_t e;
  switch (p.type) {
    case TYPE_F32: e = vec ? backward_shape<TYPE_F32, true>(p, w, want_n, s) : backward_shape<TYPE_F32, false>(p, w, want_n, s); break;
    case TYPE_BF16: e = vec ? backward_shape<TYPE_BF16, true>(p, w, want_n, s) : backward_shape<TYPE_BF16, false>(p, w, want_n, s); break;
    default: e = vec ? backward_shape<TYPE_F16, true>(p, w, want_n, s) : backward_shape<TYPE_F16, false>(p, w, want_n, s); break;
  }
  if (e != hipSuccess) return e;
  int nshares = 0;
  if (w.chunks > 0) {
    nshares = rms_sample_tiles(p);
    hipLaunchKernelGGL(rms_sample_kernel, dim3((unsigned)((long long)p.M * p.b * nshares)), dim3(256), 0, s, p, w, nshares);
    if (!want_n) nshares = 0;
  } else if (w.tiles > 1 && want_n) {
    nshares = w.tiles;
  }
  const int colblocks = (p.D + 63) / 64;
  const int count = w.chunks > 0 ? w.samples : w.nb, step = std::max(1, w.chunks);
  const long long nblocks = nshares ? ((long long)p.M * p.b + FIN * 64 - 1) / (FIN * 64) : 0;
  hipLaunchKernelGGL(rms_finish_kernel, dim3((unsigned)((long long)colblocks * p.M + nblocks)), dim3(FIN * 64), 0, s, p, w, count, step, colblocks, nshares);
  if (p.q) {
    if (w.chunks > 0) hipLaunchKernelGGL(rms_inner_partials_kernel, dim3((unsigned)((long long)p.M * p.b)), dim3(256), 0, s, p, w);
    else if (p.D > RMS_MAX_D) hipLaunchKernelGGL(rms_inner_long_kernel, dim3((unsigned)(((long long)p.M * p.b + 3) / 4)), dim3(256), 0, s, p);
    else switch (p.type) {
      case TYPE_F32: vec ? inner_by_length<TYPE_F32, true>(p, s) : inner_by_length<TYPE_F32, false>(p, s); break;
      case TYPE_BF16: vec ? inner_by_length<TYPE_BF16, true>(p, s) : inner_by_length<TYPE_BF16, false>(p, s); break;
      default: vec ? inner_by_length<TYPE_F16, true>(p, s) : inner_by_length<TYPE_F16, false>(p, s);
    }
  }
  return hipGetLastError();
}

}  // namespace absk
