#pragma once
// Scores of a scored view, in log2 units (gfx950).
//
// With x = scale q.k, a capped score is cap tanh(x / cap), and a biased one has
// slope_h * (query position - key position) subtracted. tanh(y) = 1 - 2r with r =
// 1 / (1 + e^2y), so with u = exp2(q.k * cap_in), cap_in = 2 scale log2(e) / cap:
//   s2 = cap2 - 2 cap2 r,  r = 1 / (1 + u),  cap2 = cap log2(e)
// (u overflows to infinity where the score is the cap: r = 0.) It takes two
// instructions of the quarter-rate unit and three others, and is off by about cap
// * 2^-22: with the caps allowed (at most 1024) by less than the rounding of P to
// bf16. The derivative, which the backward needs, is 1 - tanh^2 = 4 (r - r^2), with
// no cancellation where the score is small and r is near 1/2, and with a small
// relative error where r is small; near r = 1 (scores near -cap) it is off by 2^-22,
// as tanh itself is. The backward leaves the 4 to the final scale.
//
// The bias is one FMA where a query is a lane: fma(slope2, key position, off), slope2
// = slope log2(e), with the query's share -slope2 * position (and cap2) in off.
// Positions are counted in the document, exact in fp32 (a biased view's documents
// have at most 2^24 tokens). off is large far into a document, but the sum with a
// near key's share is exact to its own size: only the rounding of off itself is
// left, which all scores of the row have in common. It drops out of the softmax,
// and row_offset() gives what the row's LSE has to be corrected by.
#include "common.hpp"

namespace fck {

enum { kScoreCap = 1, kScoreBias = 2 };

inline int score_kind(float cap2, const float* slopes) {
  return (cap2 > 0.f ? kScoreCap : 0) | (slopes ? kScoreBias : 0);
}

// r of a product `x` (see above)
__device__ __forceinline__ float cap_r(float x, float cap_in) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * cap_in));
}

// off = cap2 - slope2 * pos of a row, rounded, and in `rest` what the rounding left
// out: the product's tail by FMA and the sum's by comparing both terms with it.
__device__ __forceinline__ float row_offset(float cap2, float slope2, float pos, float& rest) {
#pragma clang fp contract(off)
  const float ph = slope2 * pos, pl = __builtin_fmaf(slope2, pos, -ph);
  const float off = cap2 - ph, back = off - cap2;
  rest = ((cap2 - (off - back)) - (ph + back)) - pl;
  return off;
}

// The score of product x: c is cap_in (capped) or scale log2(e), off the bias
// (with cap2 added if capped).
template <int SC>
__device__ __forceinline__ float score_of(float x, float c, float cap2, float off) {
  if constexpr (SC & kScoreCap)
    return __builtin_fmaf(cap_r(x, c), -2.f * cap2, off);
  else
    return __builtin_fmaf(x, c, off);
}

}  // namespace fck
