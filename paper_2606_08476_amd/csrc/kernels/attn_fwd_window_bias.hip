// Forward attention with windows and a distance bias (gfx950); the per-workgroup body is in
// fwd.hpp.
#include "fwd.hpp"

namespace fck {

template hipError_t launch_fwd_sc<kWindow | kScoreBias>(const FwdParams&, int, int, int, hipStream_t);

}  // namespace fck
