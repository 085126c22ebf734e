// Forward attention with capped scores and a distance bias (gfx950); the per-workgroup body is in
// fwd.hpp.
#include "fwd.hpp"

namespace fck {

template hipError_t launch_fwd_sc<kScoreCap | kScoreBias>(const FwdParams&, int, int, int, hipStream_t);

}  // namespace fck
