// Rotary positions of a rank's rows (gfx950): the forward's rows, the keys of the
// KV gather, and their gradients.
//
// Pair i of a head, (x_i, x_{i+m/2}) or (x_2i, x_2i+1) of its first m values, is
// turned by position * w_i and scaled by the amplitude:
//   y_a = A (x_a cos t - x_b sin t),  y_b = A (x_b cos t + x_a sin t);
// a gradient goes back with -t. The angle is counted in turns as a 64-bit fixed
// point number, position * (w_i / 2 pi) modulo 2^64: exact whatever the position,
// where an fp32 product is off by 0.01 radians at 2^18 tokens. Its upper 32 bits are
// the half turns that sincospi takes.
//
// Bound by HBM: every row is read and written once. A workgroup takes a few tokens
// of one tensor and puts their sines and cosines in LDS once, for every head (one
// per thread and four tokens or so; held per lane they would be computed once per
// eight heads). A thread then takes units of two 16-byte pieces of a head: a pair's
// two halves, or pieces half a head apart, read before either is written, so that
// rows may be rotated in place.
// Measured, 64K tokens over 8 ranks, 32/8 heads of 128: own rows (201 MB read and
// written, each byte once by the counters) 37 us, 5.4 TB/s; KV gather (436 MB) 82 us,
// 5.3; gradients to bf16 (856 MB) 153 us, 5.6. A copy of these sizes reaches 5.0 to 5.5.
#include "common.hpp"
#include "rope.hpp"

namespace fck {

// A piece of a row: 16 bytes of it, 8 bf16 or 4 fp32 values, as fp32.
template <bool F32>
struct Piece {
  static constexpr int V = F32 ? 4 : 8;
  typedef uint32_t word __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ void load(float (&x)[V], const void* p, int64_t e) {
    const word w = *reinterpret_cast<const word*>(static_cast<const char*>(p) + e * (16 / V));
#pragma unroll
    for (int j = 0; j < V; ++j)
      x[j] = __uint_as_float(F32 ? w[j] : j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
};
// V values stored, 16 bytes of fp32 or V of bf16, not to be kept in the L2: another
// kernel is the next to read them. Against plain stores: own rows of 32/8 heads of
// 128 over 64K tokens and 8 ranks 43.5 -> 39.2 us, their gather 87.9 -> 82.2.
template <bool F32, int V>
__device__ __forceinline__ void store(void* p, int64_t e, const float (&x)[V]) {
  constexpr int N = F32 ? V : V / 2;
  typedef uint32_t word __attribute__((ext_vector_type(N)));
  word w;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if constexpr (F32)
      w[j] = __float_as_uint(x[j]);
    else
      w[j] = uint32_t(f2bf(x[2 * j])) | uint32_t(f2bf(x[2 * j + 1])) << 16;
  }
  word* q = reinterpret_cast<word*>(static_cast<char*>(p) + e * (F32 ? 4 : 2));
  __builtin_nontemporal_store(w, q);
}

// The unaligned layout (halves that are no multiple of 8 values apart): single values.
template <bool F32>
__device__ __forceinline__ float load1(const void* p, int64_t e) {
  return F32 ? static_cast<const float*>(p)[e] : bf2f(static_cast<const u16*>(p)[e]);
}
template <bool F32>
__device__ __forceinline__ void store1(void* p, int64_t e, float x) {
  if constexpr (F32)
    static_cast<float*>(p)[e] = x;
  else
    static_cast<u16*>(p)[e] = f2bf(x);
}

template <int D, int LAYOUT, bool IN32, bool OUT32>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams p) {
  constexpr int V = Piece<IN32>::V, U = D / (2 * V);  // units of two pieces per head
  __shared__ __attribute__((aligned(16))) float cs[2][kRopeRows * D / 2];
  __shared__ int32_t pos[kRopeRows];
  // this workgroup's tensor and rows
  int blk = blockIdx.x;
  RopeRows s = p.set[0];
#pragma unroll
  for (int i = 1; i < kRopeSets; ++i)
    if (i < p.n_sets && blk >= s.blocks) {
      blk -= s.blocks;
      s = p.set[i];
    }
  const int r0 = blk * s.per_block, n = min(s.per_block, s.rows - r0);
  const int tid = threadIdx.x;
  if (s.rotate) {
    if (tid < n) {
      const int r = r0 + tid;
      int x = s.gpos[r];
      if (!p.packed_pos) {
        int i = s.first[r / 64];
        while (r >= p.seg[4 * i + s.end]) ++i;
        x -= p.seg[4 * i + 2];
      }
      pos[tid] = x;
    }
    __syncthreads();
    for (int i = tid; i < n * (D / 2); i += 256) {
      const int j = i % (D / 2);
      float c = 1.f, sn = 0.f;
      if (j < p.pairs) {
        const uint64_t turn = p.turn[j] * uint64_t(uint32_t(pos[i / (D / 2)]));
        sincospif(float(int32_t(turn >> 32)) * 0x1p-31f, &sn, &c);
        c *= p.amplitude;
        sn *= p.amplitude * p.sign;
      }
      cs[0][i] = c;
      cs[1][i] = sn;
    }
    __syncthreads();
  }

  const int hu = s.heads * U;  // units per row
  const int half = p.pairs;    // values between a pair's halves
  // unit q of row t; 256 units further with each step
  int t = tid / hu, q = tid % hu;
  for (int i = tid; i < n * hu; i += 256) {
    const int h = q / U, u = q % U;
    const int64_t src = s.gather ? s.gather[r0 + t] : r0 + t;
    const int64_t in = src * s.in_stride + h * D, out = int64_t(r0 + t) * s.out_stride + h * D;
    const float* c = cs[0] + t * (D / 2);
    const float* sn = cs[1] + t * (D / 2);
    t += s.step_t;
    q += s.step_q;
    if (q >= hu) {
      q -= hu;
      ++t;
    }
    if (LAYOUT == kRopeHalvesOdd && s.rotate) {
      for (int j = V * u; j < V * (u + 1); ++j) {
        // pair j, or values of the rest two by two
        const int ea = j < half ? j : 2 * j, eb = j < half ? j + half : 2 * j + 1;
        const float xa = load1<IN32>(s.in, in + ea), xb = load1<IN32>(s.in, in + eb);
        store1<OUT32>(s.out, out + ea, j < half ? xa * c[j] - xb * sn[j] : xa);
        store1<OUT32>(s.out, out + eb, j < half ? xb * c[j] + xa * sn[j] : xb);
      }
      continue;
    }
    // the unit's two pieces: pairs' halves where they are rotated so, elsewhere
    // pieces from either half of the values, so that the lanes' lie side by side
    int ea = V * u, eb = ea + D / 2;
    const bool pairs = LAYOUT == kRopeHalves && s.rotate && ea < half;
    if (LAYOUT == kRopeHalves && s.rotate) {
      ea += pairs ? 0 : half;
      eb = pairs ? ea + half : ea + (D / 2 - half);
    }
    float a[V], b[V];
    Piece<IN32>::load(a, s.in, in + ea);
    Piece<IN32>::load(b, s.in, in + eb);
    // (what is not rotated is not multiplied either: 0 times an infinity beside it)
    if (LAYOUT == kRopeNeighbours && s.rotate) {
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        auto turn = [&](float& x0, float& x1, int i) {
          const float y0 = x0 * c[i] - x1 * sn[i], y1 = x1 * c[i] + x0 * sn[i];
          x0 = i < half ? y0 : x0;
          x1 = i < half ? y1 : x1;
        };
        turn(a[2 * j], a[2 * j + 1], ea / 2 + j);
        turn(b[2 * j], b[2 * j + 1], eb / 2 + j);
      }
    }
    if (pairs) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float x = a[j], y = b[j], cc = c[ea + j], ss = sn[ea + j];
        a[j] = x * cc - y * ss;
        b[j] = y * cc + x * ss;
      }
    }
    store<OUT32>(s.out, out + ea, a);
    store<OUT32>(s.out, out + eb, b);
  }
}

template <int D, int LAYOUT>
static void launch_rope_t(const RopeParams& p, unsigned blocks, bool in_f32, bool out_f32,
                          hipStream_t s) {
  if (!in_f32)
    hipLaunchKernelGGL((rope_kernel<D, LAYOUT, false, false>), dim3(blocks), dim3(256), 0, s, p);
  else if (!out_f32)
    hipLaunchKernelGGL((rope_kernel<D, LAYOUT, true, false>), dim3(blocks), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((rope_kernel<D, LAYOUT, true, true>), dim3(blocks), dim3(256), 0, s, p);
}

template <int D>
static hipError_t launch_rope_d(const RopeParams& p, unsigned blocks, int layout, bool in_f32,
                                bool out_f32, hipStream_t s) {
  switch (layout) {
    case kRopeHalves: launch_rope_t<D, kRopeHalves>(p, blocks, in_f32, out_f32, s); break;
    case kRopeNeighbours: launch_rope_t<D, kRopeNeighbours>(p, blocks, in_f32, out_f32, s); break;
    case kRopeHalvesOdd: launch_rope_t<D, kRopeHalvesOdd>(p, blocks, in_f32, out_f32, s); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_rope(const RopeParams& p, int d, int layout, bool in_f32, bool out_f32,
                       hipStream_t s) {
  int64_t blocks = 0;
  for (int i = 0; i < p.n_sets; ++i) blocks += p.set[i].blocks;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffff || (!in_f32 && out_f32)) return hipErrorInvalidValue;
  if (d == 64) return launch_rope_d<64>(p, unsigned(blocks), layout, in_f32, out_f32, s);
  if (d == 128) return launch_rope_d<128>(p, unsigned(blocks), layout, in_f32, out_f32, s);
  return hipErrorInvalidValue;
}

}  // namespace fck
