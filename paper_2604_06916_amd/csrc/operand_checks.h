// Checks of operands on the host, shared by the C-ABI entry points: sizes,
// strides, alignment, and what may not lie over what.
#pragma once

#include <stdint.h>

#include <numeric>

#include "solfp4.h"

namespace solfp4::checks {

constexpr int64_t kMaxDim = (int64_t)1 << 31;

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline bool type_ok(int type) { return type == SOLFP4_BF16 || type == SOLFP4_F16 || type == SOLFP4_F32; }

inline bool element_aligned(int type, const void* p) { return ((uintptr_t)p & (type == SOLFP4_F32 ? 3u : 1u)) == 0; }

inline int check_dims(int64_t a, int64_t b) {
  if (a < 0 || b < 0) return SOLFP4_EINVAL;
  if (a >= kMaxDim || b >= kMaxDim) return SOLFP4_ESHAPE;
  return SOLFP4_OK;
}

// Whether an operand of this many rows stays within kMaxSpan elements.
constexpr int64_t kMaxSpan = (int64_t)1 << 46;
inline bool span_ok(int64_t stride, int64_t rows) { return stride == 0 || rows - 1 <= kMaxSpan / stride; }

// Rows of an operand that the call reads or, with `written`, writes (whose
// rows must not overlap).
inline int check_rows(int type, const void* p, int64_t stride, int64_t rows, int64_t width, bool written) {
  if (!p || stride < 0) return SOLFP4_EINVAL;
  if (!span_ok(stride, rows)) return SOLFP4_ESHAPE;
  if (!element_aligned(type, p)) return SOLFP4_EALIGN;
  if (written && rows > 1 && stride < width) return SOLFP4_EINVAL;
  return SOLFP4_OK;
}

// What an operand covers: w bytes at p + i s0 + j s1, i < n0, j < n1.
struct Region {
  uintptr_t p;
  int64_t n0, s0, n1, s1, w;
  int64_t span0() const { return (n0 - 1) * s0 + w; }
  int64_t span1() const { return (n1 - 1) * s1 + w; }
};

// Whether two regions (every count at least 1) share no byte: one ends before
// the other begins, or they lie side by side as columns or heads of one
// buffer do, which shows in their offsets modulo the strides' common divisor.
inline bool apart(const Region& a, const Region& b) {
  const int64_t a_len = (a.n0 - 1) * a.s0 + a.span1(), b_len = (b.n0 - 1) * b.s0 + b.span1();
  if (!a_len || !b_len || a.p + (uint64_t)a_len <= b.p || b.p + (uint64_t)b_len <= a.p) return true;
  const int64_t d = (int64_t)(b.p - a.p);
  const auto beside = [d](int64_t g, int64_t wa, int64_t wb) {
    if (g <= 0) return false;
    const int64_t r = (d % g + g) % g;
    return r >= wa && r + wb <= g;
  };
  const auto step = [](int64_t n, int64_t s) { return n > 1 ? s : (int64_t)0; };
  const int64_t g0 = std::gcd(step(a.n0, a.s0), step(b.n0, b.s0)), g1 = std::gcd(step(a.n1, a.s1), step(b.n1, b.s1));
  return beside(g0, a.span1(), b.span1()) || beside(g1, a.span0(), b.span0()) || beside(std::gcd(g0, g1), a.w, b.w);
}

inline Region block_of(const void* p, int64_t bytes) { return {(uintptr_t)p, 1, 0, 1, 0, bytes}; }

inline Region rows_region(int type, const void* p, int64_t stride, int64_t rows, int64_t width) {
  const int64_t bytes = type == SOLFP4_F32 ? 4 : 2;
  return {(uintptr_t)p, p ? rows : 1, rows > 1 ? stride * bytes : 0, 1, 0, p ? width * bytes : 0};
}

// The two are one operand (each element is read before it is written) or apart.
inline bool same_or_apart(const Region& a, const Region& b) {
  return (a.p == b.p && a.n0 == b.n0 && a.s0 == b.s0 && a.w == b.w) || apart(a, b);
}

}  // namespace solfp4::checks
