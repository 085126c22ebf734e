#pragma once
// Scores of a scored view, in log2 units (gfx950).
//
// With x = scale q.k, a capped score is cap tanh(x / cap), and a biased one has
// slope_h * (query position - key position) subtracted. tanh(y) = 1 - 2r with r =
// 1 / (1 + e^2y), so with u = exp2(q.k * cap_in), cap_in = 2 scale log2(e) / cap:
//   s2 = cap2 - 2 cap2 r,  r = 1 / (1 + u),  cap2 = cap log2(e)
// (u overflows to infinity where the score is the cap: r = 0.) It takes two
// transcendental instructions (each the issue time of two) and three others, and is off
// by about cap * 2^-22: with the caps allowed (at most 1024) by less than the rounding of
// P to bf16. The derivative, which the backward needs, is 1 - tanh^2 = 4 (r - r^2), taken
// as 4 u r^2: exact relative to its own size at either end, where a difference would
// leave the rounding of r alone for scores near -cap (7% off at 7 caps; against the
// difference, one instruction more per score, a layer of 32/8 heads of 128 over 64K
// tokens and 8 ranks 2306 -> 2325 us). The backward leaves the 4 to the final scale.
//
// The bias is one FMA where a query is a lane: fma(slope2, key position, off), slope2
// = slope log2(e), with the query's share -slope2 * position (and cap2) in off.
// Positions are counted in the document, exact in fp32 (a biased view's documents
// have at most 2^24 tokens). off is large far into a document, but the sum with a
// near key's share is exact to its own size: only the rounding of off itself is
// left, which all scores of the row have in common. It drops out of the softmax,
// and row_offset() gives what the row's LSE has to be corrected by. That is up to 2^-24
// of slope * position, scores are as large, and their roundings leave the LSE up to
// four times 2^-24 of that off. (Counted from the workgroup's first row they would not, but
// a row's bits would depend on its tile, and the partial passes' on the call. dQ takes
// the LSE as given, so nothing drops out there: it does count from its first row.)
#include "common.hpp"
#include "launch.hpp"

#include <type_traits>

namespace fck {

// Kinds of views: what their scores are, and whether rows see windows.
enum { kScoreCap = 1, kScoreBias = 2, kScores = 3, kWindow = 4 };

inline int score_kind(float cap2, const float* slopes, const int32_t* win) {
  return (cap2 > 0.f ? kScoreCap : 0) | (slopes ? kScoreBias : 0) | (win ? kWindow : 0);
}
// go(std::integral_constant<int, kind>())
template <class F>
hipError_t with_kind(int kind, const F& go) {
  switch (kind) {
    case 0: return go(std::integral_constant<int, 0>());
    case 1: return go(std::integral_constant<int, 1>());
    case 2: return go(std::integral_constant<int, 2>());
    case 3: return go(std::integral_constant<int, 3>());
    case 4: return go(std::integral_constant<int, 4>());
    case 5: return go(std::integral_constant<int, 5>());
    case 6: return go(std::integral_constant<int, 6>());
    case 7: return go(std::integral_constant<int, 7>());
    default: return hipErrorInvalidValue;
  }
}

// r of a product `x` (see above)
__device__ __forceinline__ float cap_r(float x, float cap_in) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * cap_in));
}

// v_mul_legacy_f32, the product in which 0 times anything is 0: the compiler's intrinsic
// has no builtin, and in inline assembly it would not wait for exp2's or rcp's result.
extern "C" __device__ __attribute__((const)) float fck_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");

// r times 2^LOG2 and, times 2^(2 LOG2), r - r^2 = u r^2. (Where u is infinite r is 0,
// and so is the legacy product.)
template <int LOG2>
__device__ __forceinline__ float cap_r(float x, float cap_in, float& r_r2) {
  constexpr float k = 1.f / (1 << LOG2);
  const float u = __builtin_amdgcn_exp2f(x * cap_in);
  const float r = __builtin_amdgcn_rcpf(LOG2 ? __builtin_fmaf(u, k, k) : 1.f + u);
  r_r2 = fck_mul_legacy(u, r) * r;
  return r;
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

// Keys out of reach. With |x| <= B = scale log2(e) |q| |k| (and <= cap2) for every key
// of a source, and the row's own key among the local ones, a key at distance t has a
// weight of at most 2^(B + B_local - slope2 t): where that is under 2^-kReach, all
// such keys together (2^24 at most) are 2^-76 of the row's sum, 2^52 times less than
// its last bit, and are not visited. Norms are the largest of a head's rows, in
// kNormParts partial maxima of squares that launch_norms leaves (a NaN counts as
// infinite, so that nothing is out of reach of it).
constexpr float kReach = 100.f;

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int w = 32; w >= 1; w >>= 1) x = fmaxf(x, __shfl_xor(x, w));
  return x;
}

// Largest norm of a head's rows, for the wave.
__device__ __forceinline__ float head_norm(const float* norms, int head) {
  const f32x4 v = reinterpret_cast<const f32x4*>(norms + size_t(head) * kNormParts)[threadIdx.x & 63];
  return __builtin_sqrtf(wave_max(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]))));
}

// The bound B of a score's size, given the norms of q and k and scale log2(e).
template <int SC>
__device__ __forceinline__ float score_bound(float c, float qn, float kn, float cap2) {
  const float b = fabsf(c) * qn * kn * 1.001f;  // (the norms' own roundings)
  return (SC & kScoreCap) && b < INFINITY ? fminf(b, cap2) : b;
}

// Windowed views (kWindow). A query tile's key tiles are those of key_tiles; of a source's
// keys (indices ascend with positions) a row sees those from the first in its window up
// to itself or its receive limit, and those before `sink`. In the query-major kernels a
// lane has a row: its windows' starts are in LDS (a word per source and lane of 32, read
// on tiles that are masked), the tile's own bounds in scalar registers. (The table is
// read through the tile's first and last row; a table of those per item, one load
// instead of two in turn, was no faster.)
struct WindowTiles {
  KeyTiles recv, local;
  int sink_r, sink_l;    // ends of the sinks
  int last_r, last_l;    // the last row's windows begin here
};
__device__ __forceinline__ WindowTiles window_tiles(const int32_t* win, int q0, int q1, int r0, int r1, int l0,
                                                    int l1) {
  const int32_t* const a = win + 4 * size_t(q0);
  const int32_t* const b = win + 4 * size_t(q1 - 1);
  return {key_tiles(r0, r1, a[1], a[3]), key_tiles(l0, l1, a[0], a[2]), a[3], a[2], b[1], b[0]};
}
// Bytes of LDS for the rows' windows, and a lane's place there (`pair`: wave * 32 + row).
constexpr uint32_t kWindowLds = 128 * 8;
__device__ __forceinline__ void put_window(char* lds, int pair, const int32_t* win, int row) {
  *reinterpret_cast<uint2*>(lds + 8 * pair) =
      make_uint2(uint32_t(win[4 * size_t(row)]), uint32_t(win[4 * size_t(row) + 1]));
}

// A lane's 32 scores of a key tile (key k0 + 4 (lane / 32) + 8 (n / 4) + n % 4 for score n)
// as bits: those of keys before the t-th from k0 + 4 (lane / 32) on.
__device__ __forceinline__ uint32_t keys_below(int t) {
  t = min(max(t, 0), 64);
  const int n = 4 * (t >> 3) + min(t & 7, 4);
  return n ? 0xffffffffu >> (32 - n) : 0u;
}
// The scores that a row sees: before `rel`, and from `from` on or before `sink`. One
// register for all of a tile (three compared per score cost spills).
__device__ __forceinline__ uint32_t seen_keys(int rel, int from, int sink) {
  return keys_below(rel) & (~keys_below(from) | keys_below(sink));
}

// KV head of workgroup b, and its index among those of the head; `per` of them.
// Consecutive workgroups are on consecutive XCDs, so with eight KV heads each L2 serves
// one of them. Where reach makes heads unequal, the heads are dealt to the XCDs in
// turn, or (head_order) taken one after the other, the farthest reaching first, so
// that no long workgroup starts late. One after the other, a head's rows lie 2 KB
// apart and fewer of the memory's channels work at a time. Measured, an L2 per head /
// in turn / farthest first: one 98K-token document, 32/8 heads of 128, slopes 2^-1/4
// to 2^-8, queries scaled by 3, forward 3707 / 2226 / 1157 us, backward 10720 / 6002 /
// 3420; 64K tokens of mixed documents, 8 ranks, two passes 412 / 324 / 323, backward
// 1235 / 937 / 918, dK/dV alone 763 / 591 / 640; 16/8 heads of 64, 32K tokens, cap and
// bias, queries scaled by 3, forward 183 / 180 / 211, backward 500 / 404 / 371.
template <bool BIAS, class P>
__device__ __forceinline__ int kv_head(const P& p, int b, int per, int& rest) {
  if (BIAS && p.norms) {
    if (p.head_order) {
      rest = __builtin_amdgcn_readfirstlane(b % per);
      return __builtin_amdgcn_readfirstlane(p.head_order[b / per]);
    }
    rest = b / p.hkv;
    return __builtin_amdgcn_readfirstlane((b % p.hkv + rest) % p.hkv);
  }
  rest = b / p.hkv;
  return b % p.hkv;
}

// How far a row's keys reach (b: what is known of the exponent without the bias).
__device__ __forceinline__ float reach(float b, float slope2) {
  const float r = (b + kReach) / slope2;
  return r >= 0.f ? r : slope2 > 0.f && r < 0.f ? 0.f : INFINITY;
}

// First index of lo .. hi-1 whose position (ascending) is at least `cut`, hi if none;
// by the whole wave, 64 probes at a time.
__device__ __forceinline__ int first_at(const float* pos, int lo, int hi, float cut) {
  const int lane = threadIdx.x & 63;
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const int n = __popcll(__ballot(i < hi && pos[min(i, hi - 1)] < cut));
    if (step == 1 || n == 0) return lo + n;
    hi = min(hi, lo + n * step);
    lo += (n - 1) * step + 1;
  }
  return lo;
}

// The starts of a workgroup's received and local key ranges (r0 .. r1-1, l0 .. l1-1) moved
// up, by whole tiles of BN keys, to the first key within reach of any of its rows: cr
// and cl are this lane's positions under which a source's keys are out of reach
// (infinite for a lane without a row). `lds`: 10 words that are free. Contains barriers;
// two waves search, one range each, where there is anything to leave out.
template <int BN>
__device__ __forceinline__ void skip_far(char* lds, const float* recv_pos, const float* q_pos, float cr,
                                         float cl, int& r0, int r1, int& l0, int l1) {
  float* const cuts = reinterpret_cast<float*>(lds);
  const int wave = wave_id();
  cr = -wave_max(-cr);
  cl = -wave_max(-cl);
  if ((threadIdx.x & 63) == 0) {
    cuts[2 * wave] = cr;
    cuts[2 * wave + 1] = cl;
  }
  __syncthreads();
  float mr = cuts[0], ml = cuts[1];
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    mr = fminf(mr, cuts[2 * w]);
    ml = fminf(ml, cuts[2 * w + 1]);
  }
  if (mr > 0.f || ml > 0.f) {  // (no position is below 0)
    int* const at = reinterpret_cast<int*>(lds) + 8;
    if (wave < 2) {
      const int a = wave ? l0 : r0, b = wave ? l1 : r1;
      const int i = first_at(wave ? q_pos : recv_pos, a, b, wave ? ml : mr);
      at[wave] = i >= b ? b : a + (i - a) / BN * BN;
    }
    __syncthreads();
    r0 = __builtin_amdgcn_readfirstlane(at[0]);
    l0 = __builtin_amdgcn_readfirstlane(at[1]);
  }
  __syncthreads();  // before the words are used again
}

}  // namespace fck
