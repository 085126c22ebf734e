// Backward attention (gfx950): the kernels of views without a score function, and
// which kernel a call takes. The kernels are in bwd.hpp.
#include "bwd.hpp"

namespace fck {

template hipError_t launch_bwd_grid_sc<0>(const BwdParams&, const DqParams&, int, int, hipStream_t);
template hipError_t launch_bwd_keys_sc<0>(const BwdParams&, int, bool, hipStream_t);
// (in attn_bwd_cap.hip, attn_bwd_bias.hip, attn_bwd_cap_bias.hip, and the same of windows)
extern template hipError_t launch_bwd_grid_sc<1>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<1>(const BwdParams&, int, bool, hipStream_t);
extern template hipError_t launch_bwd_grid_sc<2>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<2>(const BwdParams&, int, bool, hipStream_t);
extern template hipError_t launch_bwd_grid_sc<3>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<3>(const BwdParams&, int, bool, hipStream_t);
extern template hipError_t launch_bwd_grid_sc<4>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<4>(const BwdParams&, int, bool, hipStream_t);
extern template hipError_t launch_bwd_grid_sc<5>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<5>(const BwdParams&, int, bool, hipStream_t);
extern template hipError_t launch_bwd_grid_sc<6>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<6>(const BwdParams&, int, bool, hipStream_t);
extern template hipError_t launch_bwd_grid_sc<7>(const BwdParams&, const DqParams&, int, int, hipStream_t);
extern template hipError_t launch_bwd_keys_sc<7>(const BwdParams&, int, bool, hipStream_t);

// the row norms that a biased backward's reach goes by
static hipError_t norms_first(const BwdParams& p, int d, hipStream_t s) {
  if (!p.norms) return hipSuccess;
  return launch_norms(p.norms, p.q, p.k_loc, p.k_recv, p.t_q, p.t_r, p.hq, p.hkv, d, s);
}

hipError_t launch_bwd_grid(const BwdParams& bp, const DqParams& dp, int d, int heads_per_tile,
                           hipStream_t s) {
  if (bp.n_items == 0 && dp.n_items == 0) return hipSuccess;
  if (const hipError_t e = norms_first(bp, d, s); e != hipSuccess) return e;
  return with_kind(score_kind(bp.cap2, bp.slopes, bp.win), [&](auto k) {
    return launch_bwd_grid_sc<decltype(k)::value>(bp, dp, d, heads_per_tile, s);
  });
}

static hipError_t launch_keys(const BwdParams& p, int d, bool atomic_dq, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  if (const hipError_t e = norms_first(p, d, s); e != hipSuccess) return e;
  return with_kind(score_kind(p.cap2, p.slopes, p.win),
                   [&](auto k) { return launch_bwd_keys_sc<decltype(k)::value>(p, d, atomic_dq, s); });
}
hipError_t launch_bwd_atomic(const BwdParams& p, int d, hipStream_t s) {
  return launch_keys(p, d, true, s);
}
hipError_t launch_bwd(const BwdParams& p, int d, hipStream_t s) {
  return launch_keys(p, d, false, s);
}

}  // namespace fck
