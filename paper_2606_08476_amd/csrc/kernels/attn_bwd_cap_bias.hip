// Backward attention with capped scores and a distance bias (gfx950); the kernels are in bwd.hpp.
#include "bwd.hpp"

namespace fck {

template hipError_t launch_bwd_grid_sc<kScoreCap | kScoreBias>(const BwdParams&, const DqParams&, int, int, hipStream_t);
template hipError_t launch_bwd_keys_sc<kScoreCap | kScoreBias>(const BwdParams&, int, bool, hipStream_t);

}  // namespace fck
