// Values of a type known at run time or compile time (fp32, bf16, fp16) in memory, as fp32 in registers.
#pragma once
#include "device_utils.h"
#include "ops.h"

namespace absk {
namespace {

__device__ __forceinline__ float f16_val(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
__device__ __forceinline__ uint16_t f16_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ float load_as_f32(const void *p, int type, long long i) {
  if (type == TYPE_F32) return static_cast<const float *>(p)[i];
  const uint16_t h = static_cast<const uint16_t *>(p)[i];
  return type == TYPE_BF16 ? bf2f(h) : f16_val(h);
}
__device__ __forceinline__ void store_from_f32(void *p, int type, long long i, float v) {
  if (type == TYPE_F32) static_cast<float *>(p)[i] = v;
  else static_cast<uint16_t *>(p)[i] = type == TYPE_BF16 ? f2bf(v) : f16_bits(v);
}
// eight 16-bit values of one 16-byte vector
__device__ __forceinline__ void unpack8(const uint4 q, int type, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = type == TYPE_BF16 ? __uint_as_float(w[e] << 16) : f16_val(w[e] & 0xffffu);
    v[2 * e + 1] = type == TYPE_BF16 ? __uint_as_float(w[e] & 0xffff0000u) : f16_val(w[e] >> 16);
  }
}
__device__ __forceinline__ uint4 pack8(int type, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    w[e] = type == TYPE_BF16 ? pack2bf(v[2 * e], v[2 * e + 1]) : (uint32_t)f16_bits(v[2 * e]) | ((uint32_t)f16_bits(v[2 * e + 1]) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// eight consecutive values at 16-byte aligned places, all of which exist
__device__ __forceinline__ void load8(const void *p, int type, long long i, float (&v)[8]) {
  if (type == TYPE_F32) {
    const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
    const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    unpack8(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + i), type, v);
  }
}
__device__ __forceinline__ void store8(void *p, int type, long long i, const float (&v)[8]) {
  if (type == TYPE_F32) {
    float *f = static_cast<float *>(p) + i;
    *reinterpret_cast<float4 *>(f) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(f + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) = pack8(type, v);
  }
}
// The same at places of the type's own alignment (the machine takes 16 bytes from anywhere)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ uint4 load16_any(const void *p) {
  const u32x4_any q = *static_cast<const u32x4_any *>(p);
  return make_uint4(q.x, q.y, q.z, q.w);
}
__device__ __forceinline__ void store16_any(void *p, uint4 v) {
  const u32x4_any q = {v.x, v.y, v.z, v.w};
  *static_cast<u32x4_any *>(p) = q;
}
__device__ __forceinline__ void load8_any(const void *p, int type, long long i, float (&v)[8]) {
  if (type == TYPE_F32) {
    const uint4 a = load16_any(static_cast<const float *>(p) + i), b = load16_any(static_cast<const float *>(p) + i + 4);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(w[e]);
  } else {
    unpack8(load16_any(static_cast<const uint16_t *>(p) + i), type, v);
  }
}
__device__ __forceinline__ void store8_any(void *p, int type, long long i, const float (&v)[8]) {
  if (type == TYPE_F32) {
    float *f = static_cast<float *>(p) + i;
    store16_any(f, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
    store16_any(f + 4, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
  } else {
    store16_any(static_cast<uint16_t *>(p) + i, pack8(type, v));
  }
}

}  // namespace

// rows that all start on 16 bytes and hold whole 16-byte vectors of eight 16-bit values (two of four fp32 ones)
inline bool rows_of_vectors(const void *p, int type, long long stride, long long ld, int n) {
  return !(n & 7) && !(reinterpret_cast<uintptr_t>(p) & 15) && !((stride * type_bytes(type)) & 15) && !((ld * type_bytes(type)) & 15);
}

}  // namespace absk
