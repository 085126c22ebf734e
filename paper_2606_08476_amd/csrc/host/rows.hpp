// What the calls on rows (rotary rows, head norms) check and prepare alike.
#pragma once

#include <cmath>
#include <cstdint>

#include "internal.hpp"

namespace fc {

// A range of rows in memory, in bytes.
struct Span {
  uintptr_t base;
  int64_t stride, width, rows;
  uintptr_t end() const { return base + uintptr_t((rows - 1) * stride + width); }
  bool same(const Span& o) const { return base == o.base && stride == o.stride; }
  // whether any row of one touches a row of the other (slices of one buffer, rows
  // the same stride apart, touch where their columns do)
  bool touches(const Span& o) const {
    if (!rows || !o.rows || end() <= o.base || o.end() <= base) return false;
    if (stride != o.stride) return true;
    // columns from a row's start here to the start of the other's next row
    const int64_t ahead = o.base >= base ? int64_t(o.base - base) % stride
                                         : (stride - int64_t(base - o.base) % stride) % stride;
    return ahead < width || ahead + o.width > stride;
  }
};

inline int check_rope(const fc_rope* r, int32_t d) {
  if (!r) return FC_OK;
  if (r->dim < 2 || r->dim > d || r->dim % 2)
    return fail(FC_ERR_INVALID_ARG, "rotated values must be even and from 2 to the head dim");
  if (!r->inv_freq) return fail(FC_ERR_INVALID_ARG, "inv_freq is null");
  if (!std::isfinite(r->amplitude)) return fail(FC_ERR_INVALID_ARG, "amplitude is not finite");
  for (int32_t i = 0; i < r->dim / 2; ++i)
    if (!(std::fabs(r->inv_freq[i]) <= FC_ROPE_FREQ_MAX))
      return fail(FC_ERR_INVALID_ARG, "inv_freq must be within FC_ROPE_FREQ_MAX");
  return FC_OK;
}

// Radians per position as turns modulo 1, 64-bit fixed point (|w| is within
// FC_ROPE_FREQ_MAX, checked before). (Long doubles are truncated without a change of the
// rounding mode by SSE3's store alone: with such changes n = 32 take up to 1.2 us.)
__attribute__((target("sse3"))) inline void turns(const double* w, int32_t n, uint64_t* turn) {
  constexpr long double kPerTurn = 0.15915494309189533576888376337251436L;
  for (int32_t i = 0; i < n; ++i) {
    const long double t = w[i] * kPerTurn;
    const long double f = t - static_cast<int>(t);  // of w's sign, exact
    turn[i] = static_cast<uint64_t>(static_cast<int64_t>(f * 9223372036854775808.0L)) << 1;
  }
}

}  // namespace fc
