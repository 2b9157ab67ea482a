// Checks of operands that the operators' entry points share: types, alignment, strides, overlaps.
#pragma once
#include <algorithm>
#include <numeric>
#include <string>
#include "../../include/abs.h"
#include "api_status.h"
#include "ops.h"

namespace absk {
namespace {

bool known_type(int t) { return t >= ABS_TYPE_F32 && t <= ABS_TYPE_F16; }
bool aligned_to(const void *p, int bytes) { return !(reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)); }

// A [n][rows][cols] block in memory, `bytes` to a value.  Looked at as a whole (level 0), as what repeats in its longer step (1), or as rows (2)
struct Block {
  const void *p;
  int64_t n, stride, rows, ld, cols;
  int bytes;
  uintptr_t at() const { return reinterpret_cast<uintptr_t>(p); }
  int64_t over(int64_t count, int64_t step) const { return count > 1 ? step : 0; }
  int64_t longer() const { return std::max(over(n, stride), over(rows, ld)) * bytes; }
  // bytes of a piece, from its first value to behind its last, and what the distances between pieces are multiples of (0: one piece)
  uintptr_t length(int level) const {
    const int64_t matrices = over(n, stride) * (n - 1), lines = over(rows, ld) * (rows - 1);
    const bool by_matrix = over(n, stride) >= over(rows, ld);
    return (uintptr_t)(((level == 0 ? matrices + lines : level == 1 ? (by_matrix ? lines : matrices) : 0) + cols) * bytes);
  }
  uintptr_t pitch(int level) const {
    return (uintptr_t)(level == 0 ? 0 : level == 1 ? longer() : std::gcd(over(n, stride), over(rows, ld)) * bytes);
  }
};
Block piece(const void *p, int64_t values, int bytes) { return {p, 1, 0, 1, 0, values, bytes}; }
// Apart: one ends before the other begins, or all pieces of both begin at two places, with room for each, of spaces of one pitch
bool overlap(const Block &a, const Block &b) {
  const uintptr_t p = a.at(), q = b.at();
  if (p + a.length(0) <= q || q + b.length(0) <= p) return false;
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 3; ++j) {
      const uintptr_t space = std::gcd(a.pitch(i), b.pitch(j));
      if (!space) continue;
      const uintptr_t d = q >= p ? (q - p) % space : (space - (p - q) % space) % space;
      if (d >= a.length(i) && d + b.length(j) <= space) return false;
    }
  return true;
}
// Any of the outputs over an input or another output (absent ones: null)
template <size_t NO, size_t NI> bool outputs_overlap(const Block (&out)[NO], const Block (&in)[NI]) {
  for (size_t i = 0; i < NO; ++i) {
    if (!out[i].p) continue;
    for (const Block &x : in)
      if (x.p && overlap(out[i], x)) return true;
    for (size_t j = 0; j < i; ++j)
      if (out[j].p && overlap(out[i], out[j])) return true;
  }
  return false;
}
// rows that do not overlap, matrix after matrix or interleaved; offsets that 64 bits hold
bool strides_ok(int64_t n, int64_t stride, int64_t rows, int64_t ld, int64_t cols) {
  const int64_t big = (int64_t)1 << 46;
  if (ld < cols || ld >= big / rows || stride < 0 || stride >= big / n) return false;
  return n == 1 || stride >= (rows - 1) * ld + cols || (stride >= cols && ld >= (n - 1) * stride + cols);
}
abs_status hip_status(hipError_t e, const char *what) {
  return e == hipSuccess ? ABS_OK : set_error(ABS_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace
}  // namespace absk
