#pragma once
// Backward attention kernels (gfx950): the key-major dK/dV kernel, the
// whole deterministic backward pass (dK/dV and dQ workgroups) in one
// launch, and the non-deterministic pass (key tiles that also add dQ with
// atomics). The per-workgroup bodies are in bwd_dkdv.hpp and bwd_dq.hpp.
#include "bwd_dkdv.hpp"
#include "bwd_dq.hpp"

namespace fck {

// Query heads per dK/dV iteration: the most of 4, 2, 1 that divides the
// group.
static int heads_per_iteration(int group) { return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1; }

// (Three waves per SIMD at head dim 64, for which the residual branch gives up P's
// packed values. With two and the values: 64/16 heads of 64 over 64K tokens 1757
// us, 32/8 over 16K with queries scaled by 3, 216; now 1585 and 199. At 128 there
// are two either way, and the values kept are worth 286 -> 279 us, 32/8 heads
// over 8K tokens scaled by 3.)
template <int D, int HPI>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attn_bwd_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DkdvLds<D>::bytes];
  dkdv_tile<D, false, HPI, D == 64 ? kKeepDs : kKeepAll>(p, blockIdx.x, smem);
}
// (Scored: bounds for two waves per SIMD; at 64 the kernels take 157 to 168 registers,
// which leaves three, but for cap and bias over four heads (172). P's packed values are
// not kept, as at 128 up to 254 of 256 are taken. Against views without a score function,
// 32/8 heads of 128 over 64K tokens and 8 ranks, capped at 50: dK/dV 679 -> 816 us, dQ 474
// -> 587, the whole 1148 -> 1397. Beside each MFMA there are 8.0 vector instructions, 1.5
// of them transcendental, where without a cap there are 3.8 and 0.6. Counted, the matrix
// unit is busy 47% of the cycles and the vector unit 56%, both at once 19% (without a cap
// 61, 33 and 17): neither is full, two waves per SIMD leave them too little of each
// other's work to overlap. What was tried: r - r^2 unpacked by mixed FMAs, 16
// instructions less per tile and wave, and the score's steps a slot apart; neither gave
// 1%.)
template <int D, int HPI, int SC>
__global__ __launch_bounds__(256, 2) void attn_bwd_scored_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DkdvLds<D, false, SC>::bytes];
  dkdv_tile<D, false, HPI, kKeepDs, SC>(p, blockIdx.x, smem);
}

// (Windows with slopes at head dim 128, and capped with dQ by atomics for ungrouped heads,
// take over 256 registers: one wave per SIMD, without scratch memory. With slopes, two
// waves with 6 to 24 registers spilled are faster: the case below, window 1024, 907 us and
// 664, where windows alone take 550; window 4096, 1533 and 1115.)
// The whole backward, 32/8 heads of 128, 64K tokens and 8 ranks, window 1024: 531-550 us,
// 1.5 GB at 2.8 TB/s, matrix unit busy 45% of the cycles, vector unit 34%, both 13%; window
// 4096, 16K rows: 2945-3060, 63, 36 and 18%. Five products of what the rows see are 297
// GFLOP (2388); seven of them, the tiles' masked parts and the residuals make 478 (3405).
template <int D, int KIND, bool MORE = false>
constexpr int kWindowWaves = D == 128 && ((KIND & kScoreBias) || MORE) ? 1 : 2;
template <int D, int HPI, int KIND>
__global__ __launch_bounds__(256, (kWindowWaves<D, KIND>)) void attn_bwd_window_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DkdvLds<D, false, KIND>::bytes];
  dkdv_tile<D, false, HPI, kKeepDs, KIND>(p, blockIdx.x, smem);
}

// The non-deterministic backward pass: key tiles only, each also adding its
// share of dQ into p.dq (zeroed beforehand) with atomics.
// (kKeepNone where the registers are short. Kept values spilled 4 at head dim 128
// and two heads per iteration, 16/8 heads over 32K tokens 1114 us against 1107; at
// 64 their lack leaves three waves per SIMD, 16/8 heads over 16K tokens with
// queries scaled by 3, 462 against 443. At 128 with one or four heads they fit:
// 32/8 heads over 64K tokens 2421 us, without them 2450.)
template <int D, int HPI>
__global__ __launch_bounds__(256, 2) void attn_bwd_atomic_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DkdvLds<D, true>::bytes];
  dkdv_tile<D, true, HPI, D == 128 && HPI != 2 ? kKeepAll : kKeepNone>(p, blockIdx.x, smem);
}
template <int D, int HPI, int SC>
__global__ __launch_bounds__(256, 2) void attn_bwd_atomic_scored_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DkdvLds<D, true, SC>::bytes];
  dkdv_tile<D, true, HPI, kKeepNone, SC>(p, blockIdx.x, smem);
}

template <int D, int HPI, int KIND>
__global__ __launch_bounds__(256, (kWindowWaves<D, KIND, HPI == 1 && (KIND & kScoreCap)>)) void
attn_bwd_atomic_window_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[DkdvLds<D, true, KIND>::bytes];
  dkdv_tile<D, true, HPI, kKeepNone, KIND>(p, blockIdx.x, smem);
}

// The whole backward pass in one launch: the first n_dkdv workgroups take
// key tiles (dK/dV), the others query tiles (dQ); the dQ workgroups start
// as dK/dV ones finish, so neither pass leaves a tail of its own.
template <int D, int HPW, int HPI>
__global__ __launch_bounds__(256, 2) void attn_bwd_grid_kernel(BwdParams bp, DqParams dp, int n_dkdv) {
  constexpr uint32_t kBytes = DkdvLds<D>::bytes > DqLds<D>::bytes ? DkdvLds<D>::bytes : DqLds<D>::bytes;
  __shared__ __attribute__((aligned(16))) char smem[kBytes];
  const int b = blockIdx.x;
  if (b < n_dkdv)
    dkdv_tile<D, false, HPI, kKeepAll>(bp, b, smem);
  else
    dq_tile<D, HPW, D == 64>(dp, b - n_dkdv, smem);
}
template <int D, int HPW, int HPI, int SC>
__global__ __launch_bounds__(256, 2) void attn_bwd_grid_scored_kernel(BwdParams bp, DqParams dp,
                                                                      int n_dkdv) {
  constexpr uint32_t kKeys = DkdvLds<D, false, SC>::bytes, kRows = DqLds<D, SC>::bytes;
  __shared__ __attribute__((aligned(16))) char smem[kKeys > kRows ? kKeys : kRows];
  const int b = blockIdx.x;
  if (b < n_dkdv)
    dkdv_tile<D, false, HPI, kKeepDs, SC>(bp, b, smem);
  else
    dq_tile<D, HPW, D == 64, SC>(dp, b - n_dkdv, smem);
}

template <int D, int HPW, int HPI, int KIND>
__global__ __launch_bounds__(256, (kWindowWaves<D, KIND>)) void attn_bwd_grid_window_kernel(BwdParams bp,
                                                                                         DqParams dp,
                                                                                         int n_dkdv) {
  constexpr uint32_t kKeys = DkdvLds<D, false, KIND>::bytes, kRows = DqLds<D, KIND>::bytes;
  __shared__ __attribute__((aligned(16))) char smem[kKeys > kRows ? kKeys : kRows];
  const int b = blockIdx.x;
  if (b < n_dkdv)
    dkdv_tile<D, false, HPI, kKeepDs, KIND>(bp, b, smem);
  else
    dq_tile<D, HPW, D == 64, KIND>(dp, b - n_dkdv, smem);
}

// (HPW, the dQ workgroups' heads per tile, divides the group as HPI does,
// so HPW <= HPI)
template <int D, int SC>
static hipError_t launch_grid_d(const BwdParams& bp, const DqParams& dp, int hpw, hipStream_t s) {
  const int n_dkdv = bp.n_items * bp.hkv;
  const dim3 grid(unsigned(n_dkdv + dp.n_items * dp.hkv * dp.head_chunks)), block(256);
  const int hpi = heads_per_iteration(bp.group);
  auto go = [&](auto w, auto i) {
    constexpr int W = decltype(w)::value, I = decltype(i)::value;
    if constexpr (SC & kWindow)
      hipLaunchKernelGGL((attn_bwd_grid_window_kernel<D, W, I, SC>), grid, block, 0, s, bp, dp, n_dkdv);
    else if constexpr (SC)
      hipLaunchKernelGGL((attn_bwd_grid_scored_kernel<D, W, I, SC>), grid, block, 0, s, bp, dp, n_dkdv);
    else
      hipLaunchKernelGGL((attn_bwd_grid_kernel<D, W, I>), grid, block, 0, s, bp, dp, n_dkdv);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, 4> four;
  if (hpi == 4 && hpw == 4) go(four, four);
  else if (hpi == 4 && hpw == 2) go(two, four);
  else if (hpi == 4 && hpw == 1) go(one, four);
  else if (hpi == 2 && hpw == 2) go(two, two);
  else if (hpi == 2 && hpw == 1) go(one, two);
  else if (hpi == 1 && hpw == 1) go(one, one);
  else return hipErrorInvalidValue;
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || !dp.n_comb) return e;
  return launch_dq_combine(dp, D, hpw, s);
}

// the key-tile kernels (dK/dV alone, or with atomic dQ) for head dim D and
// the group's heads per iteration
template <template <int, int, int> class K, int D, int SC>
static hipError_t launch_keys_d(const BwdParams& p, hipStream_t s) {
  const dim3 grid(unsigned(p.n_items) * p.hkv), block(256);
  switch (heads_per_iteration(p.group)) {
    case 4: hipLaunchKernelGGL((K<D, 4, SC>::fn()), grid, block, 0, s, p); break;
    case 2: hipLaunchKernelGGL((K<D, 2, SC>::fn()), grid, block, 0, s, p); break;
    default: hipLaunchKernelGGL((K<D, 1, SC>::fn()), grid, block, 0, s, p); break;
  }
  return hipGetLastError();
}
template <int D, int HPI, int SC>
struct DkdvKernel {
  static constexpr auto fn() {
    if constexpr (SC & kWindow) return attn_bwd_window_kernel<D, HPI, SC>;
    else if constexpr (SC) return attn_bwd_scored_kernel<D, HPI, SC>;
    else return attn_bwd_kernel<D, HPI>;
  }
};
template <int D, int HPI, int SC>
struct AtomicKernel {
  static constexpr auto fn() {
    if constexpr (SC & kWindow) return attn_bwd_atomic_window_kernel<D, HPI, SC>;
    else if constexpr (SC) return attn_bwd_atomic_scored_kernel<D, HPI, SC>;
    else return attn_bwd_atomic_kernel<D, HPI>;
  }
};

// (one kind of view per source file)
template <int SC>
hipError_t launch_bwd_grid_sc(const BwdParams& bp, const DqParams& dp, int d, int hpw, hipStream_t s) {
  if (d == 64) return launch_grid_d<64, SC>(bp, dp, hpw, s);
  if (d == 128) return launch_grid_d<128, SC>(bp, dp, hpw, s);
  return hipErrorInvalidValue;
}
template <int SC>
hipError_t launch_bwd_keys_sc(const BwdParams& p, int d, bool atomic_dq, hipStream_t s) {
  if (d == 64)
    return atomic_dq ? launch_keys_d<AtomicKernel, 64, SC>(p, s) : launch_keys_d<DkdvKernel, 64, SC>(p, s);
  if (d == 128)
    return atomic_dq ? launch_keys_d<AtomicKernel, 128, SC>(p, s) : launch_keys_d<DkdvKernel, 128, SC>(p, s);
  return hipErrorInvalidValue;
}

}  // namespace fck
