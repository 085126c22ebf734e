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
// eight heads). A thread then takes 16 values of a head (eight pairs), in 16-byte
// pieces; a piece and its partner are read before either is written, so rows may be
// rotated in place.
#include "common.hpp"
#include "rope.hpp"

namespace fck {

// 8 values from / to memory, as fp32
template <bool F32>
__device__ __forceinline__ void load8(float (&x)[8], const void* p, int64_t e) {
  if constexpr (F32) {
    const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + e);
    const f32x4 a = q[0], b = q[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const u16*>(p) + e);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf2f(u16(v[j] & 0xffff));
      x[2 * j + 1] = bf2f(u16(v[j] >> 16));
    }
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t e, const float (&x)[8]) {
  if constexpr (F32) {
    f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + e);
    q[0] = f32x4{x[0], x[1], x[2], x[3]};
    q[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = uint32_t(f2bf(x[2 * j])) | uint32_t(f2bf(x[2 * j + 1])) << 16;
    *reinterpret_cast<uint4*>(static_cast<u16*>(p) + e) = make_uint4(v[0], v[1], v[2], v[3]);
  }
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
  constexpr int U = D / 16;  // units of 16 values per head
  __shared__ __attribute__((aligned(16))) float cs[2][kRopeRows * D / 2];
  __shared__ int32_t pos[kRopeRows];
  // this workgroup's tensor and rows
  int b = blockIdx.x;
  RopeRows s = p.set[0];
#pragma unroll
  for (int i = 1; i < kRopeSets; ++i)
    if (i < p.n_sets && b >= s.blocks) {
      b -= s.blocks;
      s = p.set[i];
    }
  const int r0 = b * s.per_block, n = min(s.per_block, s.rows - r0);
  const int tid = threadIdx.x;
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
  if (s.rotate) {
    for (int i = tid; i < n * (D / 2); i += 256) {
      const int j = i % (D / 2);
      float c = 1.f, sn = 0.f;
      if (j < p.pairs) {
        const uint64_t t = p.turn[j] * uint64_t(uint32_t(pos[i / (D / 2)]));
        sincospif(float(int32_t(t >> 32)) * 0x1p-31f, &sn, &c);
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
  for (int i = tid; i < n * hu; i += 256) {
    const int t = i / hu, h = (i % hu) / U, u = i % U;
    const int64_t src = s.gather ? s.gather[r0 + t] : r0 + t;
    const int64_t in = src * s.in_stride + h * D, out = int64_t(r0 + t) * s.out_stride + h * D;
    const float* c = cs[0] + t * (D / 2) + 8 * u;
    const float* sn = cs[1] + t * (D / 2) + 8 * u;
    if (LAYOUT == kRopeHalvesOdd && s.rotate) {
      for (int j = 0; j < 8; ++j) {
        const int q = 8 * u + j;  // pair q, or values of the rest two by two
        const int ea = q < half ? q : 2 * q, eb = q < half ? q + half : 2 * q + 1;
        const float xa = load1<IN32>(s.in, in + ea), xb = load1<IN32>(s.in, in + eb);
        store1<OUT32>(s.out, out + ea, xa * c[j] - xb * sn[j]);
        store1<OUT32>(s.out, out + eb, xb * c[j] + xa * sn[j]);
      }
      continue;
    }
    // the unit's two pieces of 8 values: halves apart where it is rotated so,
    // neighbours elsewhere
    int ea = 16 * u, eb = ea + 8;
    if (LAYOUT == kRopeHalves && s.rotate && 8 * u < half) {
      ea = 8 * u;
      eb = ea + half;
    }
    float a[8], bb[8];
    load8<IN32>(a, s.in, in + ea);
    load8<IN32>(bb, s.in, in + eb);
    if (s.rotate) {
      if (LAYOUT == kRopeNeighbours) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x0 = a[2 * j], x1 = a[2 * j + 1], y0 = bb[2 * j], y1 = bb[2 * j + 1];
          a[2 * j] = x0 * c[j] - x1 * sn[j];
          a[2 * j + 1] = x1 * c[j] + x0 * sn[j];
          bb[2 * j] = y0 * c[4 + j] - y1 * sn[4 + j];
          bb[2 * j + 1] = y1 * c[4 + j] + y0 * sn[4 + j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = a[j], y = bb[j];
          a[j] = x * c[j] - y * sn[j];
          bb[j] = y * c[j] + x * sn[j];
        }
      }
    }
    store8<OUT32>(s.out, out + ea, a);
    store8<OUT32>(s.out, out + eb, bb);
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
