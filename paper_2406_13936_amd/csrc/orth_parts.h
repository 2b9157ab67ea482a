// Pieces of the orthogonalisation shared by orthogonalize.hip (any size, one launch per product) and orthogonalize_small.hip
// (matrices that a work-group's LDS holds, one launch for everything).
#pragma once
#include "device_utils.h"
#include "ops.h"
#include "typed_mem.h"

namespace absk {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

namespace {

// eight values as fp16 and what that leaves
__device__ __forceinline__ void split8(const float (&v)[8], uint4 &hi, uint4 &lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint16_t h0 = f16_bits(v[2 * e]), h1 = f16_bits(v[2 * e + 1]);
    h[e] = (uint32_t)h0 | ((uint32_t)h1 << 16);
    l[e] = (uint32_t)f16_bits(v[2 * e] - f16_val(h0)) | ((uint32_t)f16_bits(v[2 * e + 1] - f16_val(h1)) << 16);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// Values (r, c) .. (r, c + 7) of what is orthogonalised, matrix z; zeros outside the matrix.  ADVANCE: v takes its step first (each value must be visited once so); else v is the new one.
template <bool ADVANCE>
__device__ __forceinline__ void load_u8(const OrthIn &in, int rows, int cols, int z, int r, int c, float (&u)[8]) {
  const long long g0 = z * in.sg + (long long)r * in.ldg + c, v0 = z * in.sv + (long long)r * cols + c;
  const float mu = in.momentum;
  if (r < rows && c + 8 <= cols) {
    load8_any(in.g, in.type, g0, u);
    if (in.v) {
      float v[8];
      load8_any(in.v, TYPE_F32, v0, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (ADVANCE) v[e] = fmaf(mu, v[e], u[e]);
        u[e] = in.nesterov ? fmaf(mu, v[e], u[e]) : v[e];
      }
      if (ADVANCE) store8_any(in.v, TYPE_F32, v0, v);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    u[e] = 0.0f;
    if (r < rows && c + e < cols) {
      u[e] = load_as_f32(in.g, in.type, g0 + e);
      if (in.v) {
        float v = in.v[v0 + e];
        if (ADVANCE) in.v[v0 + e] = v = fmaf(mu, v, u[e]);
        u[e] = in.nesterov ? fmaf(mu, v, u[e]) : v;
      }
    }
  }
}

}  // namespace
}  // namespace absk
