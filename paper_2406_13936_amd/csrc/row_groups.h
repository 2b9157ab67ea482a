// Rows of values in the registers of a group of lanes: loads and stores of rows of any alignment and width, gains beside them, sums
// over the group (layer_norm.hip, rms_norm.hip).
#pragma once
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

}  // namespace
}  // namespace absk
