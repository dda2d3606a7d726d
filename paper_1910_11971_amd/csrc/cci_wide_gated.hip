// Wide-tile kernels of the gated product H = act(X Wg^T) * (X Wu^T) (the
// method, work split and layouts are described at their body,
// cci_wide_body.hpp).
#include "cci_wide_block.hpp"

namespace cci {

bool wide_gated_supports(const BlockProduct& a) { return supports<kWGated>(a); }
hipError_t launch_wide_gated(const BlockProduct& a, int pt, hipStream_t s) { return launch_wide<kWGated>(a, pt, s); }

}  // namespace cci
