// Wide-tile kernels of the transposed product dX = dY . W_hat (the
// method, work split and layouts are described at their body,
// cci_wide_body.hpp).
#include "cci_wide_block.hpp"

namespace cci {

bool wide_back_supports(const BlockProduct& a) { return supports<kWBack>(a); }
hipError_t launch_wide_back(const BlockProduct& a, int pt, hipStream_t s) { return launch_wide<kWBack>(a, pt, s); }

}  // namespace cci
