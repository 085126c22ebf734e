// Norms of queries and keys per head, with the rotation, in one pass over a rank's
// rows (gfx950): the forward's rows, the keys of the KV gather, and gradients.
//
// A head's row x of d values is normalised, weighted and rotated:
//   n = (x - m) s,  s = 1 / sqrt(mean (x - m)^2 + eps),  m = mean x or 0;
//   y = R(position) ((w + offset) n)          (R: rope.hip; rounded once, to bf16).
// Back, with g = R(-position) dy and a = (w + offset) g:
//   dw = sum over tokens (and heads that share w) of g n;
//   dx = s (a - [mean a] - n mean(a n))       (mean a where m is the mean).
// n and s are formed again from x, which is read for n anyway.
//
// Bound by HBM: every row is read and written once. U threads take a head's row, two
// 16-byte pieces of it each, as the rotation pairs them; what they add up goes round
// them by lane permutes. A thread keeps its head and its pieces for all the
// workgroup's rows, so that the weights and their gradients stay in registers;
// sines and cosines are in LDS, for all the heads of a row. A row is read a step ahead
// of its sums (a gather of 135K rows of 8x128 keys and values 215 -> 208 us), and the
// weights without a wait for each (208 -> 192).
// Measured, with cold inputs (a copy of 256 MiB: 5.4 TB/s): 8193 rows of 32/8x128
// queries, keys and values, 201 MB, 34-43 us, 4.7-5.9 TB/s; that gather, 1107 MB, 192-204
// us, 5.4-5.8 TB/s; gradients of 8193 query rows and 53237 key rows (32/8x128), 1033 MB,
// 181-190 us, 5.4-5.7 TB/s, and 10 us more for the weights' sums. The smallest calls are latency: 5.2 us
// for 1024 rows of 4/4x64, a launch's 3 us, then a read, the sums and a write in turn.
// (More waves per SIMD by launch bounds, 8 forward or 7 backward, spill: 192 -> 295 us,
// 190 -> 212 us.)
#include "common.hpp"
#include "norm.hpp"
#include "rows.hpp"

namespace fck {

// x of lane ^ 1, of lane ^ 2; with lanes of a quad (an eighth) alike: of its neighbour
template <int CTRL>
__device__ __forceinline__ float lane_swap(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Sum over U lanes side by side, in every one of them (the same bits).
template <int U>
__device__ __forceinline__ float sum_lanes(float x) {
  static_assert(U == 4 || U == 8 || U == 16, "lanes of a head");
  x += lane_swap<0xB1>(x);                       // quad_perm 1 0 3 2
  x += lane_swap<0x4E>(x);                       // quad_perm 2 3 0 1
  if constexpr (U >= 8) x += lane_swap<0x141>(x);   // row_half_mirror
  if constexpr (U >= 16) x += lane_swap<0x140>(x);  // row_mirror
  return x;
}

// A unit's two pieces of V values: where they start (vector layouts), and, odd halves,
// the places of pair j's values or of two of the rest.
template <int D, int LAYOUT, int V>
struct Unit {
  int u, ea, eb, half;
  bool pairs;  // kRopeHalves: the pieces are pairs' halves
  __device__ __forceinline__ Unit(int u_, bool rotate, int half_) : u(u_), half(rotate ? half_ : 0) {
    ea = V * u;
    eb = ea + D / 2;
    pairs = LAYOUT == kRopeHalves && ea < half;
    if (LAYOUT == kRopeHalves && half) {
      ea += pairs ? 0 : half;
      eb = pairs ? ea + half : ea + (D / 2 - half);
    }
  }
  __device__ __forceinline__ bool odd() const { return LAYOUT == kRopeHalvesOdd && half; }
  __device__ __forceinline__ int at_a(int j) const {
    if (odd()) {
      const int i = V * u + j;
      return i < half ? i : 2 * i;
    }
    return ea + j;
  }
  __device__ __forceinline__ int at_b(int j) const {
    if (odd()) {
      const int i = V * u + j;
      return i < half ? i + half : 2 * i + 1;
    }
    return eb + j;
  }
  // the pair that values j of a (and b) are turned by, and whether they are at all
  __device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const float* c, const float* s) const {
#pragma clang fp contract(off)
    if (!half) return;
    if constexpr (LAYOUT == kRopeNeighbours) {
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        auto one = [&](float& x0, float& x1, int i) {
          const float y0 = x0 * c[i] - x1 * s[i], y1 = x1 * c[i] + x0 * s[i];
          x0 = i < half ? y0 : x0;
          x1 = i < half ? y1 : x1;
        };
        one(a[2 * j], a[2 * j + 1], ea / 2 + j);
        one(b[2 * j], b[2 * j + 1], eb / 2 + j);
      }
    } else {
      // (what is not rotated is not multiplied either: 0 times an infinity beside it)
      const int i0 = LAYOUT == kRopeHalves ? ea : V * u;
      if (LAYOUT == kRopeHalves && !pairs) return;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const bool on = LAYOUT == kRopeHalves || i0 + j < half;
        const int i = on ? i0 + j : 0;
        const float x = a[j], y = b[j], cc = c[i], ss = s[i];
        const float xt = x * cc - y * ss, yt = y * cc + x * ss;
        a[j] = on ? xt : x;
        b[j] = on ? yt : y;
      }
    }
  }
};

// A unit's values, one by one (odd halves; elsewhere a piece is a load of its own).
template <int D, int LAYOUT, int V, bool F32>
__device__ __forceinline__ void load_odd(float (&a)[V], float (&b)[V], const Unit<D, LAYOUT, V>& un,
                                         const void* p, int64_t at) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    a[j] = load1<F32>(p, at + un.at_a(j));
    b[j] = load1<F32>(p, at + un.at_b(j));
  }
}
// Two pieces of V bf16 values as they are read.
template <int V, class W>
__device__ __forceinline__ void unpack(float (&a)[V], float (&b)[V], const W& x, const W& y) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    a[j] = __uint_as_float(j & 1 ? x[j / 2] & 0xffff0000u : x[j / 2] << 16);
    b[j] = __uint_as_float(j & 1 ? y[j / 2] & 0xffff0000u : y[j / 2] << 16);
  }
}
template <int D, int LAYOUT, int V, bool F32>
__device__ __forceinline__ void store_unit(const float (&a)[V], const float (&b)[V],
                                           const Unit<D, LAYOUT, V>& un, void* p, int64_t at) {
  if (un.odd()) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      store1<F32>(p, at + un.at_a(j), a[j]);
      store1<F32>(p, at + un.at_b(j), b[j]);
    }
  } else {
    store<F32>(p, at + un.ea, a);
    store<F32>(p, at + un.eb, b);
  }
}

// A head's row, in U threads' pieces, normalised in place; returns s. Squares that would
// leave fp32's range (values beyond 2^57 or so) are taken of x times 2^-70, `again`
// reading x anew: n is the same (eps is nothing beside them), and s, by which a
// gradient is multiplied, 2^-70 of the scaled values' s.
template <int D, int U, int V, class Again>
__device__ __forceinline__ float normalise(float (&a)[V], float (&b)[V], bool centred, float eps,
                                           const Again& again) {
  auto spread = [&]() {
    if (centred) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) m += a[j] * (1.f / D) + b[j] * (1.f / D);
      m = sum_lanes<U>(m);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        a[j] -= m;
        b[j] -= m;
      }
    }
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) q = __builtin_fmaf(b[j], b[j], __builtin_fmaf(a[j], a[j], q));
    return sum_lanes<U>(q);
  };
  float q = spread(), k = 1.f;
  if (__builtin_expect(__any(!(q < 0x1p120f)), 0)) {
    k = q < 0x1p120f ? 1.f : 0x1p-70f;
    again(a, b);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      a[j] *= k;
      b[j] *= k;
    }
    q = spread();
  }
  const float s = __builtin_amdgcn_rsqf(__builtin_fmaf(q, 1.f / D, eps * k * k));
#pragma unroll
  for (int j = 0; j < V; ++j) {
    a[j] *= s;
    b[j] *= s;
  }
  return s * k;
}

// This thread's weights (with the offset): 1 where there are none.
template <int D, int LAYOUT, int V>
__device__ __forceinline__ void load_weights(float (&wa)[V], float (&wb)[V], const NormRows& s,
                                             const Unit<D, LAYOUT, V>& un, int head, bool on) {
#pragma unroll
  for (int j = 0; j < V; ++j) wa[j] = wb[j] = 1.f;
  if (!s.norm || !on) return;
  const int64_t at = int64_t(head) * s.w_stride;
  // (one branch around all loads of a kind: a branch around each would wait for each)
  auto load = [&](auto f32) {
    constexpr bool F32 = decltype(f32)::value;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      wa[j] = load1<F32>(s.weight, at + un.at_a(j));
      wb[j] = load1<F32>(s.weight, at + un.at_b(j));
    }
  };
  if (!s.weight) return;
  if (s.w_bf16)
    load(std::false_type());
  else
    load(std::true_type());
#pragma unroll
  for (int j = 0; j < V; ++j) {
    wa[j] += s.offset;
    wb[j] += s.offset;
  }
}

// Sine and cosine of a turn's 64-bit fraction, the nearest fp32 values but for one in two
// thousand: the nearest quarter turns off, |x| <= pi / 4, Taylor's series to x^11 and x^12
// in 64 bits (what is left out is under 2^-36). The calls take as long as with sincospif of
// the fraction as fp32, or with sums in 32-bit pairs: a row's heads share its sines.
__device__ __forceinline__ void turn_sincos(uint64_t turn, float& sn, float& cs) {
  const uint32_t quarter = uint32_t((turn + (uint64_t(1) << 61)) >> 62);
  const uint64_t h = turn - (uint64_t(quarter) << 62);  // 2^-64 turns, -2^61 .. 2^61
  constexpr double k = 6.283185307179586476925286766559 * 0x1p-32;
  const double x = __builtin_fma(double(int32_t(h >> 32)), k, double(uint32_t(h)) * (k * 0x1p-32));
  const double z = x * x;
  double p = __builtin_fma(z, -1.0 / 39916800, 1.0 / 362880);
  p = __builtin_fma(z, p, -1.0 / 5040);
  p = __builtin_fma(z, p, 1.0 / 120);
  p = __builtin_fma(z, p, -1.0 / 6);
  const float s0 = float(__builtin_fma(x * z, p, x));
  double q = __builtin_fma(z, 1.0 / 479001600, -1.0 / 3628800);
  q = __builtin_fma(z, q, 1.0 / 40320);
  q = __builtin_fma(z, q, -1.0 / 720);
  q = __builtin_fma(z, q, 1.0 / 24);
  q = __builtin_fma(z, q, -0.5);
  const float c0 = float(__builtin_fma(z, q, 1.0));
  const bool swap = quarter & 1;
  const float a = swap ? c0 : s0, b = swap ? s0 : c0;
  sn = quarter & 2 ? -a : a;
  cs = (quarter + 1) & 2 ? -b : b;
}

// Which tensor, rows and heads a workgroup takes.
struct Share {
  NormRows s;
  int r0, r1, block, head0;  // rows; their number among the tensor's; first head
};
__device__ __forceinline__ Share share_of(const NormParams& p) {
  int blk = blockIdx.x;
  Share h;
  h.s = p.set[0];
#pragma unroll
  for (int i = 1; i < kNormSets; ++i)
    if (i < p.n_sets && blk >= h.s.blocks) {
      blk -= h.s.blocks;
      h.s = p.set[i];
    }
  h.block = blk / h.s.head_groups;
  h.head0 = blk % h.s.head_groups * h.s.group_heads;
  h.r0 = h.block * h.s.per_block;
  h.r1 = min(h.r0 + h.s.per_block, h.s.rows);
  return h;
}

// Sines and cosines of rows r0 .. r0+n-1 (n <= kNormRows). Contains barriers.
template <int D>
__device__ __forceinline__ void fill_turns(const NormParams& p, const NormRows& s, int r0, int n,
                                           float (&cs)[2][kNormRows * D / 2], int32_t* pos) {
  const int tid = threadIdx.x;
  __syncthreads();  // (the rows before have been turned)
  if (tid < n) pos[tid] = row_pos(s, p.seg, p.packed_pos, r0 + tid);
  __syncthreads();
  for (int i = tid; i < n * (D / 2); i += 256) {
    const int j = i % (D / 2);
    float c = 1.f, sn = 0.f;
    if (j < p.pairs) {
      const uint64_t turn = p.turn[j] * uint64_t(uint32_t(pos[i / (D / 2)]));
      turn_sincos(turn, sn, c);
      c *= p.amplitude;
      sn *= p.amplitude * p.sign;
    }
    cs[0][i] = c;
    cs[1][i] = sn;
  }
  __syncthreads();
}

template <int D, int LAYOUT>
__global__ __launch_bounds__(256) void norm_fwd_kernel(NormParams p) {
  constexpr int V = 8, U = norm_lanes(D, false);
  typedef uint32_t word __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(16))) float cs[2][kNormRows * D / 2];
  __shared__ int32_t pos[kNormRows], src[kNormBlock];
  const Share sh = share_of(p);
  const NormRows& s = sh.s;
  const int slot = threadIdx.x / U;
  const int row = slot / s.group_heads, head = sh.head0 + slot % s.group_heads;
  const bool on = row < s.step_rows && head < s.heads;
  const Unit<D, LAYOUT, V> un(threadIdx.x % U, s.rotate, p.pairs);
  // where this thread's pieces of row r are (a thread without one: of the first row)
  auto at = [&](int r, const auto& source) {
    const bool have = on && r < sh.r1;
    return source(have ? r : sh.r0) * s.in_stride + (have ? head : 0) * D;
  };
  auto listed = [&](int r) { return int64_t(s.in_gather ? s.in_gather[r] : r); };
  auto known = [&](int r) { return int64_t(src[r - sh.r0]); };
  if (int(threadIdx.x) < sh.r1 - sh.r0) src[threadIdx.x] = int32_t(listed(sh.r0 + int(threadIdx.x)));
  // a row's pieces are read a step ahead, the first before the sines
  const u16* const base = static_cast<const u16*>(s.in);
  word na = {}, nb = {};
  auto ahead = [&](int r, const auto& source) {
    if (un.odd()) return;
    const int64_t e = at(r, source);
    na = *reinterpret_cast<const word*>(base + e + un.ea);
    nb = *reinterpret_cast<const word*>(base + e + un.eb);
  };
  ahead(sh.r0 + row, listed);
  float wa[V], wb[V];
  load_weights(wa, wb, s, un, head, on);
  __syncthreads();
  const int chunk = kNormRows / s.step_rows * s.step_rows;
  for (int c0 = sh.r0; c0 < sh.r1; c0 += chunk) {
    const int c1 = min(c0 + chunk, sh.r1);
    if (s.rotate) fill_turns<D>(p, s, c0, c1 - c0, cs, pos);
    for (int q = c0; q < c1; q += s.step_rows) {
      const int r = q + row;
      const bool have = on && r < c1;
      const word xa = na, xb = nb;
      auto read = [&](float (&a)[V], float (&b)[V]) {
        if (un.odd())
          load_odd<D, LAYOUT, V, false>(a, b, un, s.in, at(r, known));
        else
          unpack(a, b, xa, xb);
      };
      if (q + s.step_rows < sh.r1) ahead(r + s.step_rows, known);
      float a[V], b[V];
      read(a, b);
      if (s.norm) {
        normalise<D, U>(a, b, s.centred, s.eps, read);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          a[j] *= wa[j];
          b[j] *= wb[j];
        }
      }
      if (!have) continue;
      un.turn(a, b, cs[0] + (r - c0) * (D / 2), cs[1] + (r - c0) * (D / 2));
      store_unit<D, LAYOUT, V, false>(a, b, un, s.out, int64_t(r) * s.out_stride + head * D);
    }
  }
}

template <int D, int LAYOUT, bool OUT32>
__global__ __launch_bounds__(256) void norm_bwd_kernel(NormParams p) {
  constexpr int V = 4, U = norm_lanes(D, true);
  typedef uint32_t word2 __attribute__((ext_vector_type(2)));
  __shared__ __attribute__((aligned(16))) float cs[2][kNormRows * D / 2];
  __shared__ __attribute__((aligned(16))) float dws[256 * 2 * V];
  __shared__ int32_t pos[kNormRows], src[kNormBlock];
  const Share sh = share_of(p);
  const NormRows& s = sh.s;
  const int slot = threadIdx.x / U;
  const int row = slot / s.group_heads, head = sh.head0 + slot % s.group_heads;
  const bool on = row < s.step_rows && head < s.heads;
  const Unit<D, LAYOUT, V> un(threadIdx.x % U, s.rotate, p.pairs);
  // where this thread's pieces of row r are (a thread without one: of the first row)
  auto in_at = [&](int r) {
    const bool have = on && r < sh.r1;
    return (have ? r : sh.r0) * s.in_stride + (have ? head : 0) * D;
  };
  auto x_at = [&](int r, const auto& source) {
    const bool have = on && r < sh.r1;
    return source(have ? r : sh.r0) * s.x_stride + (have ? head : 0) * D;
  };
  auto listed = [&](int r) { return int64_t(s.x_gather ? s.x_gather[r] : r); };
  auto known = [&](int r) { return int64_t(src[r - sh.r0]); };
  if (int(threadIdx.x) < sh.r1 - sh.r0) src[threadIdx.x] = int32_t(listed(sh.r0 + int(threadIdx.x)));
  // a row's pieces are read a step ahead, the first before the sines
  f32x4 ga = {}, gb = {};
  word2 ya = {}, yb = {};
  auto ahead = [&](int r, const auto& source) {
    if (un.odd()) return;
    const float* const g = static_cast<const float*>(s.in) + in_at(r);
    ga = *reinterpret_cast<const f32x4*>(g + un.ea);
    gb = *reinterpret_cast<const f32x4*>(g + un.eb);
    if (!s.norm) return;
    const u16* const x = static_cast<const u16*>(s.x) + x_at(r, source);
    ya = *reinterpret_cast<const word2*>(x + un.ea);
    yb = *reinterpret_cast<const word2*>(x + un.eb);
  };
  ahead(sh.r0 + row, listed);
  float wa[V], wb[V], da[V], db[V];
  load_weights(wa, wb, s, un, head, on);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < V; ++j) da[j] = db[j] = 0.f;
  const int chunk = kNormRows / s.step_rows * s.step_rows;
  for (int c0 = sh.r0; c0 < sh.r1; c0 += chunk) {
    const int c1 = min(c0 + chunk, sh.r1);
    if (s.rotate) fill_turns<D>(p, s, c0, c1 - c0, cs, pos);
    for (int q = c0; q < c1; q += s.step_rows) {
      const int r = q + row;
      const bool have = on && r < c1;
      const int rr = have ? r : c0;
      float a[V], b[V];
      if (un.odd()) {
        load_odd<D, LAYOUT, V, true>(a, b, un, s.in, in_at(r));
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          a[j] = ga[j];
          b[j] = gb[j];
        }
      }
      const word2 xa = ya, xb = yb;
      if (q + s.step_rows < sh.r1) ahead(r + s.step_rows, known);
      un.turn(a, b, cs[0] + (rr - c0) * (D / 2), cs[1] + (rr - c0) * (D / 2));
      if (s.norm) {
        auto read = [&](float (&na)[V], float (&nb)[V]) {
          if (un.odd())
            load_odd<D, LAYOUT, V, false>(na, nb, un, s.x, x_at(r, known));
          else
            unpack(na, nb, xa, xb);
        };
        float na[V], nb[V];
        read(na, nb);
        const float sc = normalise<D, U>(na, nb, s.centred, s.eps, read);
        float m = 0.f, mn = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (have) {
            da[j] = __builtin_fmaf(a[j], na[j], da[j]);
            db[j] = __builtin_fmaf(b[j], nb[j], db[j]);
          }
          a[j] *= wa[j];
          b[j] *= wb[j];
          m += a[j] + b[j];
          mn = __builtin_fmaf(b[j], nb[j], __builtin_fmaf(a[j], na[j], mn));
        }
        m = s.centred ? sum_lanes<U>(m) * (1.f / D) : 0.f;
        mn = sum_lanes<U>(mn) * (1.f / D);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          a[j] = (__builtin_fmaf(-mn, na[j], a[j]) - m) * sc;
          b[j] = (__builtin_fmaf(-mn, nb[j], b[j]) - m) * sc;
        }
      }
      if (have) store_unit<D, LAYOUT, V, OUT32>(a, b, un, s.out, int64_t(r) * s.out_stride + head * D);
    }
  }
  if (!s.part) return;
  // the threads' sums, added per value over the rows of a step and, where they share
  // the weights, over the heads, in one order
#pragma unroll
  for (int j = 0; j < V; ++j) {
    dws[slot * D + un.at_a(j)] = da[j];
    dws[slot * D + un.at_b(j)] = db[j];
  }
  __syncthreads();
  const int gh = s.group_heads, here = min(gh, s.heads - sh.head0);
  float* const out = s.part + int64_t(s.w_stride ? sh.block : sh.block * s.head_groups + sh.head0 / gh) * s.part_width;
  if (s.w_stride) {
    for (int i = threadIdx.x; i < here * D; i += 256) {
      float t = 0.f;
      for (int k = 0; k < s.step_rows; ++k) t += dws[k * gh * D + i];
      out[sh.head0 * D + i] = t;
    }
  } else {
    for (int i = threadIdx.x; i < D; i += 256) {
      float t = 0.f;
      for (int k = 0; k < s.step_rows * gh; ++k) t += dws[k * D + i];
      out[i] = t;
    }
  }
}

// kSumCols values and a slice of the rows per workgroup, added in 64 bits, rows by 16
// threads each: partial rows to a row per slice (FINAL false), and these, or few partial
// rows, to the gradient. Bound by the latency of reading what other XCDs wrote, twice. A
// second launch because anything else is slower: 10751 rows of 128 values (gradients of
// 64K tokens over 8 ranks, 32/8 heads) take 24 us in one launch of 32 values and every row
// per workgroup, 18 of eight values, 18 with the last slice's workgroup adding them up (whose
// fence writes back an L2 full of the gradients), and 10 in two.
template <bool FINAL>
__global__ __launch_bounds__(256) void norm_sum_kernel(NormSum x, NormSum y) {
  constexpr int Q = kSumCols / 4, R = 256 / Q, N = kSumRows / R;  // threads of a row; rows at a time
  __shared__ double t[R][kSumCols];
  int blk = blockIdx.x;
  const int nx = x.width / kSumCols * (FINAL ? 1 : x.slices);
  const NormSum s = blk < nx ? x : y;
  if (blk >= nx) blk -= nx;
  const int slices = FINAL ? 1 : s.slices;
  const int col = blk / slices, slice = blk % slices, tid = threadIdx.x;
  const int i = 4 * (tid % Q), k = tid / Q;
  const bool sums = FINAL && s.slices > 1;  // rows are slices' sums
  const int n = sums ? s.slices : s.n;
  const int r0 = int(int64_t(n) * slice / slices), r1 = int(int64_t(n) * (slice + 1) / slices);
  double sum[4] = {0, 0, 0, 0};
  auto add = [&](const auto* at, auto v) {
    typedef decltype(v) vec;
    for (int r = r0 + k; r < r1; r += N * R) {
      vec x4[N];
#pragma unroll
      for (int u = 0; u < N; ++u)
        if (r + R * u < r1) x4[u] = *reinterpret_cast<const vec*>(at + int64_t(r + R * u) * s.width);
#pragma unroll
      for (int u = 0; u < N; ++u)
        if (r + R * u < r1) {
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[j] += double(x4[u][j]);
        }
    }
  };
  typedef double f64x4 __attribute__((ext_vector_type(4)));
  if (sums)
    add(s.rows + kSumCols * col + i, f64x4{});
  else
    add(s.part + kSumCols * col + i, f32x4{});
#pragma unroll
  for (int j = 0; j < 4; ++j) t[k][i + j] = sum[j];
  __syncthreads();
  if (tid >= kSumCols) return;
  double v = 0;
  for (int j = 0; j < R; ++j) v += t[j][tid];
  const int at = kSumCols * col + tid;
  if constexpr (!FINAL)
    s.rows[int64_t(slice) * s.width + at] = v;
  else if (s.bf16)
    static_cast<u16*>(s.dw)[at] = f2bf(float(v));
  else
    static_cast<float*>(s.dw)[at] = float(v);
}

template <int D, int LAYOUT>
static void launch_norm_t(const NormParams& p, unsigned blocks, bool back, bool out_f32, hipStream_t s) {
  if (!back)
    hipLaunchKernelGGL((norm_fwd_kernel<D, LAYOUT>), dim3(blocks), dim3(256), 0, s, p);
  else if (out_f32)
    hipLaunchKernelGGL((norm_bwd_kernel<D, LAYOUT, true>), dim3(blocks), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((norm_bwd_kernel<D, LAYOUT, false>), dim3(blocks), dim3(256), 0, s, p);
}

template <int D>
static hipError_t launch_norm_d(const NormParams& p, int layout, bool back, bool out_f32, hipStream_t s) {
  int64_t blocks = 0;
  for (int i = 0; i < p.n_sets; ++i) blocks += p.set[i].blocks;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  const unsigned n = unsigned(blocks);
  switch (layout) {
    case kRopeHalves: launch_norm_t<D, kRopeHalves>(p, n, back, out_f32, s); break;
    case kRopeNeighbours: launch_norm_t<D, kRopeNeighbours>(p, n, back, out_f32, s); break;
    case kRopeHalvesOdd: launch_norm_t<D, kRopeHalvesOdd>(p, n, back, out_f32, s); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

static hipError_t launch_norm(const NormParams& p, int d, int layout, bool back, bool out_f32, hipStream_t s) {
  if (d == 64) return launch_norm_d<64>(p, layout, back, out_f32, s);
  if (d == 128) return launch_norm_d<128>(p, layout, back, out_f32, s);
  return hipErrorInvalidValue;
}
hipError_t launch_norm_fwd(const NormParams& p, int d, int layout, hipStream_t s) {
  return launch_norm(p, d, layout, false, false, s);
}
hipError_t launch_norm_bwd(const NormParams& p, int d, int layout, bool out_f32, hipStream_t s) {
  return launch_norm(p, d, layout, true, out_f32, s);
}

hipError_t launch_norm_sum(const NormSum& a, const NormSum& b, hipStream_t s) {
  // (those of few rows have no part in the first)
  NormSum many[2] = {a, b};
  for (NormSum& m : many)
    if (m.slices <= 1) m.width = 0;
  const int32_t first = many[0].width / kSumCols * many[0].slices + many[1].width / kSumCols * many[1].slices;
  if (first) {
    hipLaunchKernelGGL((norm_sum_kernel<false>), dim3(unsigned(first)), dim3(256), 0, s, many[0], many[1]);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const unsigned blocks = unsigned(a.width + b.width) / kSumCols;
  if (!blocks) return hipSuccess;
  hipLaunchKernelGGL((norm_sum_kernel<true>), dim3(blocks), dim3(256), 0, s, a, b);
  return hipGetLastError();
}

}  // namespace fck
