// Backward attention, dQ kernel (gfx950), and the sum of a split query tile's
// parts; the per-workgroup body is in bwd_dq.hpp.
#include "bwd_dq.hpp"

namespace fck {

// Head dim 64: -D held in registers leaves two waves per SIMD, without it the
// four-heads tile runs three. It gains on many workgroups (64/16 heads over 64K
// tokens 1163 -> 1110 us, 32/8 over 32K 254 -> 247) and loses on few (32/8 over 16K
// 110 -> 118; D subtracted per score, 122); the other tiles, at or over the
// three-wave limit without it, are faster with -D held (8/8 heads over 32K 109
// against 112 us, 16/8 95 against 97).
template <int D, int HPW>
__global__ __launch_bounds__(256, D == 64 && HPW == 4 ? 3 : 2) void attn_bwd_dq_kernel(DqParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DqLds<D>::bytes];
  dq_tile<D, HPW, D == 64 && HPW != 4>(p, blockIdx.x, smem);
}

template <int D, int HPW, int SC>
__global__ __launch_bounds__(256, 2) void attn_bwd_dq_scored_kernel(DqParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DqLds<D, SC>::bytes];
  dq_tile<D, HPW, D == 64 && HPW != 4, SC>(p, blockIdx.x, smem);
}

// (Windows with slopes at head dim 128 take 257 registers and more.)
template <int D, int HPW, int KIND>
__global__ __launch_bounds__(256, D == 128 && (KIND & kScoreBias) ? 1 : 2) void attn_bwd_dq_window_kernel(DqParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DqLds<D, KIND>::bytes];
  dq_tile<D, HPW, D == 64 && HPW != 4, KIND>(p, blockIdx.x, smem);
}

template <int D, int SC>
static hipError_t launch_dq_d(const DqParams& p, int hpw, hipStream_t s) {
  const dim3 grid(unsigned(p.n_items) * p.hkv * p.head_chunks), block(256);
  auto go = [&](auto w) {
    constexpr int W = decltype(w)::value;
    if constexpr (SC & kWindow)
      hipLaunchKernelGGL((attn_bwd_dq_window_kernel<D, W, SC>), grid, block, 0, s, p);
    else if constexpr (SC)
      hipLaunchKernelGGL((attn_bwd_dq_scored_kernel<D, W, SC>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((attn_bwd_dq_kernel<D, W>), grid, block, 0, s, p);
  };
  switch (hpw) {
    case 1: go(std::integral_constant<int, 1>()); break;
    case 2: go(std::integral_constant<int, 2>()); break;
    case 4: go(std::integral_constant<int, 4>()); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int SC>
static hipError_t launch_dq_sc(const DqParams& p, int d, int hpw, hipStream_t s) {
  if (d == 64) return launch_dq_d<64, SC>(p, hpw, s);
  if (d == 128) return launch_dq_d<128, SC>(p, hpw, s);
  return hipErrorInvalidValue;
}

hipError_t launch_bwd_dq(const DqParams& p, int d, int heads_per_tile, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  return with_kind(score_kind(p.cap2, p.slopes, p.win),
                   [&](auto k) { return launch_dq_sc<decltype(k)::value>(p, d, heads_per_tile, s); });
}

// dQ of a query tile whose key range was split: the parts' slots added in
// slot order (key order), scaled and stored. A workgroup takes one wave's 32
// rows, a quarter of the columns per wave and four slots in flight at once, so
// that few tiles still spread over the chip: bound by the latency of its reads.
template <int D, int HPW>
__global__ __launch_bounds__(256) void dq_combine_kernel(DqParams p) {
  constexpr int RPW = 32 / HPW, KW = D / 32;  // KW: 16-byte pieces per lane
  __shared__ __attribute__((aligned(16))) float st[32 * D];
  const int lane = threadIdx.x & 63;
  const int qw = blockIdx.x & 3, b = blockIdx.x >> 2;  // the rows' wave, the tile
  const int kvh = b % p.hkv, rest = b / p.hkv, hc = rest % p.head_chunks;
  const int32_t* e = p.comb + 8 * (rest / p.head_chunks);
  const int q0 = e[0], q1 = e[1], first = e[2], n = e[3];
  if (q0 + qw * RPW >= q1) return;
  auto read = [&](f32x4 (&x)[KW], int s) {
    const size_t slot = (size_t(first + s) * p.head_chunks + hc) * p.hkv + kvh;
    const float* const o = p.part + (slot * 4 + qw) * (32 * D) + 256 * KW * wave_id() + 4 * lane;
#pragma unroll
    for (int k = 0; k < KW; ++k) x[k] = *reinterpret_cast<const f32x4*>(o + 256 * k);
  };
  f32x4 acc[KW], x[4][KW];
  auto add = [&](const f32x4 (&y)[KW]) {
#pragma unroll
    for (int k = 0; k < KW; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[k][j] += y[k][j];
  };
  read(acc, 0);
  for (int s = 1; s < n; s += 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) read(x[u], min(s + u, n - 1));
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s + u < n) add(x[u]);
  }
  store_rows_shared<D, RPW>(
      st,
      [&](int k) {
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (p.cap2 > 0.f ? 4.f * p.scale : p.scale) * acc[k][j];
        return v;
      },
      q0 + qw * RPW, q1, p.hq, kvh * p.group + hc * HPW, p.dq, nullptr);
}

template <int D>
static hipError_t launch_dq_combine_d(const DqParams& p, int hpw, hipStream_t s) {
  const dim3 grid(unsigned(p.n_comb) * p.hkv * p.head_chunks * 4), block(256);
  switch (hpw) {
    case 1: hipLaunchKernelGGL((dq_combine_kernel<D, 1>), grid, block, 0, s, p); break;
    case 2: hipLaunchKernelGGL((dq_combine_kernel<D, 2>), grid, block, 0, s, p); break;
    case 4: hipLaunchKernelGGL((dq_combine_kernel<D, 4>), grid, block, 0, s, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_dq_combine(const DqParams& p, int d, int hpw, hipStream_t s) {
  return d == 64 ? launch_dq_combine_d<64>(p, hpw, s) : launch_dq_combine_d<128>(p, hpw, s);
}

}  // namespace fck
