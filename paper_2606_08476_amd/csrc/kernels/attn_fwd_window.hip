// Forward attention with windows (gfx950); the per-workgroup body is in
// fwd.hpp.
#include "fwd.hpp"

namespace fck {

template hipError_t launch_fwd_sc<kWindow>(const FwdParams&, int, int, int, hipStream_t);

}  // namespace fck
