// Forward attention (gfx950): the merge of a split view's chunks, the forward of
// views without a score function, and which kernel a call takes. The per-workgroup
// body is in fwd.hpp.
#include "fwd.hpp"

namespace fck {

// The chunks of a split view's query tiles, merged: a source's chunks in key
// order, then (FINAL) the local with the received partial, as the merge kernel
// would, or each source's partial by itself. A workgroup takes one wave's 32
// rows of an entry (q0 q1 first-slot received-chunks local-chunks 0 0 0), a
// quarter of the columns per wave and four chunks in flight at once: bound by
// the latency of its reads.
template <int D, int HPW, bool FINAL>
__global__ __launch_bounds__(256) void fwd_combine_kernel(FwdParams p) {
  constexpr int RPW = 32 / HPW, KW = D / 32;  // KW: 16-byte pieces per lane
  __shared__ __attribute__((aligned(16))) float st[32 * D];
  const int lane = threadIdx.x & 63, l31 = lane & 31;
  const int qw = blockIdx.x & 3, b = blockIdx.x >> 2;  // the rows' wave, the tile
  const int kvh = b % p.hkv, rest = b / p.hkv, hc = rest % p.head_chunks;
  const int32_t* e = p.comb + 8 * (rest / p.head_chunks);
  const int q0 = e[0], q1 = e[1], first = e[2], n_r = e[3], n_l = e[4];
  if (q0 + qw * RPW >= q1) return;
  auto read = [&](f32x4 (&x)[KW], float& l, int c) {
    const size_t sl = (size_t(first + c) * p.head_chunks + hc) * p.hkv + kvh;
    const float* const o = p.slots + (sl * 4 + qw) * (32 * D) + 256 * KW * wave_id() + 4 * lane;
#pragma unroll
    for (int k = 0; k < KW; ++k) x[k] = *reinterpret_cast<const f32x4*>(o + 256 * k);
    l = p.slot_lse[sl * 128 + 32 * qw + l31];
  };
  auto merge = [&](f32x4 (&a)[KW], float& la, const f32x4 (&x)[KW], float lx) {
    const Merge2 w = merge2(la, lx);
    la = w.lse;
#pragma unroll
    for (int k = 0; k < KW; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) a[k][j] = merge2_value(w, a[k][j], x[k][j]);
  };
  // chunks c0 .. c1-1 of one source
  auto source = [&](f32x4 (&a)[KW], float& la, int c0, int c1) __attribute__((always_inline)) {
    f32x4 x[4][KW];
    float lx[4];
    read(a, la, c0);
    for (int c = c0 + 1; c < c1; c += 4) {
#pragma unroll
      for (int u = 0; u < 4; ++u) read(x[u], lx[u], min(c + u, c1 - 1));
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c + u < c1) merge(a, la, x[u], lx[u]);
    }
  };
  const int h0 = kvh * p.group + hc * HPW;
  auto put = [&](const f32x4 (&a)[KW], float la, float* of, u16* ob, float* lse) {
    store_rows_shared<D, RPW>(st, [&](int k) { return a[k]; }, q0 + qw * RPW, q1, p.hq, h0, of, ob);
    const int qrow = q0 + qw * RPW + l31 % RPW;
    if (threadIdx.x < 32 && qrow < q1) lse[(size_t)(h0 + l31 / RPW) * p.t_q + qrow] = la;
  };
  f32x4 a[KW], r[KW];
  float la = -INFINITY, lr = -INFINITY;
  // (a source with no chunk: an empty partial)
#pragma unroll
  for (int k = 0; k < KW; ++k) a[k] = r[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool local = FINAL || p.o_f32, recv = FINAL || p.o_f32_recv;
  if (local && n_l > 0) source(a, la, n_r, n_r + n_l);
  if (recv && n_r > 0) source(r, lr, 0, n_r);
  if constexpr (FINAL) {
    merge(a, la, r, lr);
    put(a, la, p.o_f32, p.o_bf16, p.lse);
  } else {
    if (local) put(a, la, p.o_f32, nullptr, p.lse);
    __syncthreads();
    if (recv) put(r, lr, p.o_f32_recv, nullptr, p.lse_recv);
  }
}

template <int D>
static hipError_t launch_combine_d(const FwdParams& p, int hpw, hipStream_t s) {
  const dim3 grid(unsigned(p.n_comb) * p.hkv * p.head_chunks * 4), block(256);
#define FC_COMBINE(W)                                                            \
  if (p.o_bf16)                                                                  \
    hipLaunchKernelGGL((fwd_combine_kernel<D, W, true>), grid, block, 0, s, p);  \
  else                                                                           \
    hipLaunchKernelGGL((fwd_combine_kernel<D, W, false>), grid, block, 0, s, p)
  switch (hpw) {
    case 1: FC_COMBINE(1); break;
    case 2: FC_COMBINE(2); break;
    case 4: FC_COMBINE(4); break;
    default: return hipErrorInvalidValue;
  }
#undef FC_COMBINE
  return hipGetLastError();
}
hipError_t launch_fwd_combine(const FwdParams& p, int d, int hpw, hipStream_t s) {
  return d == 64 ? launch_combine_d<64>(p, hpw, s) : launch_combine_d<128>(p, hpw, s);
}

template hipError_t launch_fwd_sc<0>(const FwdParams&, int, int, int, hipStream_t);
// (in attn_fwd_cap.hip, attn_fwd_bias.hip and attn_fwd_cap_bias.hip)
extern template hipError_t launch_fwd_sc<1>(const FwdParams&, int, int, int, hipStream_t);
extern template hipError_t launch_fwd_sc<2>(const FwdParams&, int, int, int, hipStream_t);
extern template hipError_t launch_fwd_sc<3>(const FwdParams&, int, int, int, hipStream_t);

hipError_t launch_fwd(const FwdParams& p, int d, int heads_per_tile, bool final_out,
                      hipStream_t s) {
  if (p.n_items == 0 && p.n_units == 0) return hipSuccess;
  // (a captured partial pass may be replayed on any stream, where no event
  // orders its use of the view's slots)
  bool slots = p.slots != nullptr;
  if (slots && !p.o_bf16) {
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &st) != hipSuccess || st != hipStreamCaptureStatusNone) {
      (void)hipGetLastError();
      slots = false;
    }
  }
  const int out = slots           ? kOutUnit
                  : p.chunk       ? kOutChunks
                  : p.o_f32_recv  ? (final_out ? kOutMerged : kOutPaired)
                  : final_out     ? kOutFinal
                                  : kOutPartial;
  if (p.norms && final_out) {
    const hipError_t e = launch_norms(p.norms, nullptr, p.k_loc, p.k_recv, p.t_q, p.t_r, p.hq, p.hkv, d, s);
    if (e != hipSuccess) return e;
  }
  switch (score_kind(p.cap2, p.slopes)) {
    case 0: return launch_fwd_sc<0>(p, d, heads_per_tile, out, s);
    case kScoreCap: return launch_fwd_sc<kScoreCap>(p, d, heads_per_tile, out, s);
    case kScoreBias: return launch_fwd_sc<kScoreBias>(p, d, heads_per_tile, out, s);
    default: return launch_fwd_sc<kScoreCap | kScoreBias>(p, d, heads_per_tile, out, s);
  }
}

}  // namespace fck
