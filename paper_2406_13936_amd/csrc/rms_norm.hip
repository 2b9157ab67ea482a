// Root-mean-square norm behind the addition of a residual, with a result of the rows' type or in 8 bits (e4m3) with a scale to a row.
//
//   h = x + residual, rounded to its type (what the next layers add to);  r = 1 / sqrt(mean_d h^2 + eps),  y = h r w
//   in 8 bits:  c = max(max_d |y| / 448, 2^-100),  y / c rounded to e4m3
//
// y is made of the h that is stored, so that the backward pass, which reads h, differentiates what was computed.  Bound by memory: x and
// the residual are read, h and y written, once each.  A row lives in the registers of 16 to 512 lanes as in layer_norm.hip; the sum of
// squares and the largest |h w| are exchanged together, as r only scales them: one exchange a row.  8 x 8192 rows of 2048 in bf16 with a residual: 203 us,
// 5.3 TB/s; in 8 bits 201 to 206, 4.6 TB/s, of which exact ties are 15.
#include <algorithm>
#include <cstring>
#include "device_utils.h"
#include "ops.h"
#include "row_groups.h"

namespace absk {
namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr float SMALLEST_SCALE = 0x1p-100f;      // (its inverse is finite)

// NaN where results are infinite or NaN: an infinite maximum stands for infinities or NaN in the row or its gains (a row's NaN are in rstd, too), and r is
// infinite where a row's squares are all below fp32's range and eps is 0
__device__ __forceinline__ float scale_of(float rstd, double most) {
  // (in fp64: the maximum may be beyond fp32's range, or among its last bits, where r times it is not)
  const float c = (float)((double)rstd * most * (1.0 / E4M3_MAX));
  return c < SMALLEST_SCALE ? SMALLEST_SCALE : c < __builtin_inff() ? c : __builtin_nanf("");
}
// y / c = 448 h w / max |h w|, in which r has cancelled, is rounded to e4m3 as if it were exact, ties to even: products of two 16-bit values are often just
// between two of e4m3's, and in fp32 one value in a million came out on the other side of a border.
struct Quotient {
  double by, most;                               // 448 / max |h w|, or r / c where c is the smallest scale; then there is no `most`
  __device__ __forceinline__ Quotient(float rstd, float c, double most_) : by(c > SMALLEST_SCALE ? (double)E4M3_MAX / most_ : (double)rstd / (double)c), most(c > SMALLEST_SCALE ? most_ : 0.0) {}
  // in fp32, cut off, the last bit set if anything was: as good as the value itself to a rounding to fewer bits
  __device__ __forceinline__ float of(double hw) const {
    const float f = (float)(hw * by);            // at most half a step of fp32 away
    // |f| most - 448 |h w|: both products are exact (51 bits of the second, and one rounding of the difference keeps its sign)
    const double over = fma(fabs((double)f), most, -(double)E4M3_MAX * fabs(hw));
    if (most == 0.0 || over == 0.0 || !(fabsf(f) < __builtin_inff())) return f;
    const uint32_t u = __float_as_uint(f);
    return __uint_as_float((over > 0.0 ? u - 1 : u) | 1u);
  }
};
// four values in e4m3, to the nearest, ties to even (the machine's conversion)
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Are there infinities or NaN among a lane's gains?  (The maximum of |h w| would pass over NaN; the lane's is infinite then.)
// Gains of zero become the smallest normal value: an infinity times it is infinite, not a NaN that the maximum passes over, and of anything else the
// quotient is below sqrt(D) 2^-126 / 2^-100 and rounds to zero as before.
template <int V> __device__ __forceinline__ bool look_at_gains(float (&w)[V][8]) {
  bool odd = false;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      odd |= !(fabsf(w[v][e]) < __builtin_inff());
      w[v][e] = w[v][e] == 0.0f ? copysignf(0x1p-126f, w[v][e]) : w[v][e];
    }
  return odd;
}

// Sum and, if MAX, maximum over the group; sm: 6 floats to a wavefront, `turn` as in group_sums
template <int G, bool MAX> __device__ __forceinline__ void group_sum_max(float &s, double &m, float *sm, int turn) {
  if (!MAX) {
    float v[1] = {s};
    group_sums<G, 1>(v, sm, turn);
    s = v[0];
    return;
  }
  constexpr int W = G > 64 ? G / 64 : 4;
  s = lanes_sum<(G < 64 ? G : 64)>(s);
#pragma unroll
  for (int o = 1; o < (G < 64 ? G : 64); o <<= 1) m = fmax(m, __shfl_xor(m, o, 64));
  if (G <= 64) return;
  double *most = reinterpret_cast<double *>(sm) + (turn & 1) * W;
  float *at = sm + 4 * W + (turn & 1) * W;
  if ((threadIdx.x & 63) == 0) { at[threadIdx.x >> 6] = s; most[threadIdx.x >> 6] = m; }
  __syncthreads();
  s = 0.0f;
  m = 0.0;
#pragma unroll
  for (int h = 0; h < W; h += 4) {               // (in the order of group_sums: the same bits)
    s += (at[h] + at[h + 1]) + (at[h + 2] + at[h + 3]);
    m = fmax(m, fmax(fmax(most[h], most[h + 1]), fmax(most[h + 2], most[h + 3])));
  }
}

// The lane's eight values v of a row in e4m3; whole: vectors of a row that are all in it or not, at places that their stores may take
template <int TYPE, int G>
__device__ __forceinline__ void store_e4m3(void *p, long long at, int D, int l, int v, const float (&f)[8], bool whole) {
  uint8_t *row = static_cast<uint8_t *>(p) + at;
  const uint32_t lo = pack4_e4m3(f[0], f[1], f[2], f[3]), hi = pack4_e4m3(f[4], f[5], f[6], f[7]);
  const int c0 = col_of<TYPE, G>(v, 0, l), c4 = col_of<TYPE, G>(v, 4, l);
  if (whole) {
    if (TYPE != TYPE_F32) {
      if (c0 < D) *reinterpret_cast<uint2 *>(row + c0) = make_uint2(lo, hi);
    } else {
      if (c0 < D) *reinterpret_cast<uint32_t *>(row + c0) = lo;
      if (c4 < D) *reinterpret_cast<uint32_t *>(row + c4) = hi;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (c0 + e < D) row[c0 + e] = (uint8_t)(lo >> (8 * e));
      if (c4 + e < D) row[c4 + e] = (uint8_t)(hi >> (8 * e));
    }
  }
}

// nb blocks per replica; a group takes every (nb GP)-th row
template <int TYPE, int G, int V, bool VEC, bool ADD, bool EIGHT>
__global__ void __launch_bounds__(ln_threads(G)) rms_forward_kernel(const RmsNormP p, const int nb) {
  constexpr int GP = ln_threads(G) / G;
  __shared__ __attribute__((aligned(16))) float sm[ln_threads(G) / 64 * 6];
  const int m = blockIdx.x / nb, j = blockIdx.x - m * nb, gid = threadIdx.x / G, l = threadIdx.x % G;
  const long long rows = (long long)p.b * p.T, step = (long long)nb * GP;
  const int D = p.D;
  const float n = (float)D;
  const bool whole = VEC && !(((reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)p.sy | (uintptr_t)p.ldy)) & 7);
  int turn = 0;
  long long r = (long long)j * GP + gid;
  Raw<TYPE, V> nx, nr;                            // (the next row is on its way while a row is worked on)
  if (r < rows) {
    load_raw<TYPE, G, V, VEC>(nx, p.x, m * p.sx + r * p.ldx, D, l);
    if (ADD) load_raw<TYPE, G, V, VEC>(nr, p.res, m * p.sr + r * p.ldr, D, l);
  }
  float w[V][8];
  load_param<TYPE, G, V, VEC>(w, p.w, p.ptype, (long long)m * D, D, l);
  const bool odd = EIGHT && look_at_gains<V>(w);
  // G >= 256: every thread of the block goes through every exchange (one group to a block: they agree on r)
  for (; r < rows; r += step) {
    const Raw<TYPE, V> rx = nx, rr = nr;
    if (r + step < rows) {
      load_raw<TYPE, G, V, VEC>(nx, p.x, m * p.sx + (r + step) * p.ldx, D, l);
      if (ADD) load_raw<TYPE, G, V, VEC>(nr, p.res, m * p.sr + (r + step) * p.ldr, D, l);
    }
    float h[V][8], s = 0.0f;
    double most = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw_vals<TYPE, V>(rx, v, h[v]);
      if (ADD) {
        float q[8];
        raw_vals<TYPE, V>(rr, v, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] += q[e];
        if (TYPE != TYPE_F32) unpack8(pack8(TYPE, h[v]), TYPE, h[v]);
        store_vals<TYPE, G, VEC>(p.h, m * p.sh + r * p.ldh, D, l, v, h[v]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {               // (zeros beyond the row)
        s = fmaf(h[v][e], h[v][e], s);
        if (EIGHT) most = fmax(most, fabs((double)h[v][e] * w[v][e]));
      }
    }
    if (odd) most = __builtin_inff();
    group_sum_max<G, EIGHT>(s, most, sm, turn++);
    const float rstd = 1.0f / sqrtf(s / n + p.eps);
    const float c = EIGHT ? scale_of(rstd, most) : 0.0f;
    const Quotient quotient(rstd, c, EIGHT ? most : 1.0);
    if (l == 0) {
      if (p.rstd) p.rstd[m * rows + r] = rstd;
      if (EIGHT) p.scale[m * rows + r] = c;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) h[v][e] = EIGHT ? quotient.of((double)h[v][e] * w[v][e]) : (h[v][e] * rstd) * w[v][e];
      if (EIGHT) store_e4m3<TYPE, G>(p.y, m * p.sy + r * p.ldy, D, l, v, h[v], whole);
      else store_vals<TYPE, G, VEC>(p.y, m * p.sy + r * p.ldy, D, l, v, h[v]);
    }
  }
}

// Rows longer than the registers of a block hold: a second pass over h as it was stored, out of the caches (a thread reads what it wrote).
// A launch takes RMS_LONG_ROWS rows: a grid counts its threads in 32 bits.
constexpr int RMS_LONG_ROWS = 1 << 18;
__global__ void __launch_bounds__(256) rms_forward_long_kernel(const RmsNormP p, const int eight, const long long first) {
  __shared__ __attribute__((aligned(16))) float sm[24];
  const long long rows = (long long)p.b * p.T, i = first + blockIdx.x, m = i / rows, r = i - m * rows;
  const long long xa = m * p.sx + r * p.ldx, ra = m * p.sr + r * p.ldr, ha = m * p.sh + r * p.ldh, ya = m * p.sy + r * p.ldy, pa = m * p.D;
  float s = 0.0f;
  double most = 0.0;
  bool odd = false;
  for (int c = threadIdx.x; c < p.D; c += 256) {
    float h = load_as_f32(p.x, p.type, xa + c);
    if (p.res) {
      h += load_as_f32(p.res, p.type, ra + c);
      store_from_f32(p.h, p.type, ha + c, h);
      h = load_as_f32(p.h, p.type, ha + c);
    }
    s = fmaf(h, h, s);
    if (eight) {
      const float w = load_as_f32(p.w, p.ptype, pa + c);
      odd |= !(fabsf(w) < __builtin_inff()) || !(fabsf(h) < __builtin_inff());
      most = fmax(most, fabs((double)h * w));
    }
  }
  if (odd) most = __builtin_inff();
  group_sum_max<256, true>(s, most, sm, 0);
  const float rstd = 1.0f / sqrtf(s / (float)p.D + p.eps), scale = scale_of(rstd, most);
  const Quotient quotient(rstd, scale, most);
  if (threadIdx.x == 0) {
    if (p.rstd) p.rstd[m * rows + r] = rstd;
    if (eight) p.scale[m * rows + r] = scale;
  }
  for (int c = threadIdx.x; c < p.D; c += 256) {
    const float h = p.res ? load_as_f32(p.h, p.type, ha + c) : load_as_f32(p.x, p.type, xa + c), w = load_as_f32(p.w, p.ptype, pa + c);
    if (eight) static_cast<uint8_t *>(p.y)[ya + c] = (uint8_t)pack4_e4m3(quotient.of((double)h * w), 0.0f, 0.0f, 0.0f);
    else store_from_f32(p.y, p.type, ya + c, (h * rstd) * w);
  }
}

template <int TYPE, int G, int V, bool VEC> void forward_shape(const RmsNormP &p, hipStream_t s) {
  const long long groups = ln_threads(G) / G, rows = (long long)p.b * p.T;
  const int nb = (int)std::max(1LL, std::min((rows + groups - 1) / groups, (4LL * RMS_BLOCKS + p.M - 1) / p.M));
  const dim3 grid((unsigned)((long long)nb * p.M)), block(ln_threads(G));
  if (p.scale) {
    if (p.res) hipLaunchKernelGGL((rms_forward_kernel<TYPE, G, V, VEC, true, true>), grid, block, 0, s, p, nb);
    else hipLaunchKernelGGL((rms_forward_kernel<TYPE, G, V, VEC, false, true>), grid, block, 0, s, p, nb);
  } else {
    if (p.res) hipLaunchKernelGGL((rms_forward_kernel<TYPE, G, V, VEC, true, false>), grid, block, 0, s, p, nb);
    else hipLaunchKernelGGL((rms_forward_kernel<TYPE, G, V, VEC, false, false>), grid, block, 0, s, p, nb);
  }
}
template <int TYPE, bool VEC> void forward_by_length(const RmsNormP &p, hipStream_t s) {
  switch (rms_shape(p.D)) {
    case 0: return forward_shape<TYPE, 16, 1, VEC>(p, s);
    case 1: return forward_shape<TYPE, 64, 1, VEC>(p, s);
    case 2: return forward_shape<TYPE, 64, 2, VEC>(p, s);
    case 3: return forward_shape<TYPE, 256, 1, VEC>(p, s);
    case 4: return forward_shape<TYPE, 256, 2, VEC>(p, s);
    default: return forward_shape<TYPE, 512, 2, VEC>(p, s);
  }
}

}  // namespace

hipError_t launch_rms_norm(const RmsNormP &p, hipStream_t s) {
  const long long rows = (long long)p.b * p.T;
  if (rows * p.M > 0x7fffffff) return hipErrorInvalidValue;
  if (p.D > RMS_MAX_D) {
    for (long long first = 0; first < rows * p.M; first += RMS_LONG_ROWS)
      hipLaunchKernelGGL(rms_forward_long_kernel, dim3((unsigned)std::min<long long>(rows * p.M - first, RMS_LONG_ROWS)), dim3(256), 0, s, p, p.scale != nullptr, first);
    return hipGetLastError();
  }
  const bool vec = rows_of_vectors(p.x, p.type, p.sx, p.ldx, p.D) &&
                   (!p.res || (rows_of_vectors(p.res, p.type, p.sr, p.ldr, p.D) && rows_of_vectors(p.h, p.type, p.sh, p.ldh, p.D))) &&
                   (p.scale || rows_of_vectors(p.y, p.type, p.sy, p.ldy, p.D));
  switch (p.type) {
    case TYPE_F32: vec ? forward_by_length<TYPE_F32, true>(p, s) : forward_by_length<TYPE_F32, false>(p, s); break;
    case TYPE_BF16: vec ? forward_by_length<TYPE_BF16, true>(p, s) : forward_by_length<TYPE_BF16, false>(p, s); break;
    default: vec ? forward_by_length<TYPE_F16, true>(p, s) : forward_by_length<TYPE_F16, false>(p, s);
  }
  return hipGetLastError();
}

}  // namespace absk
