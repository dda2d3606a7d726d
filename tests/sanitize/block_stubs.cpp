// Launcher stand-ins of the feed-forward block's operators for a host-only
// build of their C-ABI layer (cci_block_api.cpp): each records that it was
// reached and launches nothing.  Buffers are touched at their ends where their
// sizes are the interface's business (workspaces).
#include <hip/hip_runtime.h>

#include "../../include/cci.h"
#include "../../paper_1910_11971_amd/csrc/cci_block.hpp"

int g_block_launches = 0;
int g_fail_at = 0;  // the launch that reports an error (1: the next one; 0: none)

namespace cci {

static hipError_t reached() {
  ++g_block_launches;
  return g_fail_at > 0 && --g_fail_at == 0 ? hipErrorOutOfMemory : hipSuccess;
}
hipError_t launch_layernorm(const void*, DType, int64_t, int64_t, const float*, const float*, float, void*, float*,
                            float*, hipStream_t) {
  return reached();
}
int64_t layernorm_bwd_workspace(int64_t N, int64_t C) { return (N < 4 ? N : 4) * 2 * C * 4; }
hipError_t launch_layernorm_bwd(const void*, const void*, DType, int64_t N, int64_t C, const float*, const float*,
                                const float*, void*, float*, float*, void* ws, hipStream_t) {
  const int64_t n = layernorm_bwd_workspace(N, C);
  if (n > 0) static_cast<char*>(ws)[0] = static_cast<char*>(ws)[n - 1] = 1;
  return reached();
}
hipError_t launch_tile_gated(const BlockProduct&, hipStream_t) { return reached(); }
hipError_t launch_tile_plain(const BlockProduct&, hipStream_t) { return reached(); }
hipError_t launch_tile_back(const BlockProduct&, hipStream_t) { return reached(); }
hipError_t launch_tile_grad(const BlockProduct&, hipStream_t) { return reached(); }
bool spmm_without_matrix_cores(ProductArgs a) { return a.C % 32 != 0; }
bool wave_split_supports(const BlockProduct& a, bool gated, int wb) {
  return a.t == DType::BF16 && (gated ? wb >= 2 : a.C >= 16 * wb);
}
hipError_t launch_wave_split(const BlockProduct&, bool, int, int, hipStream_t) { return reached(); }
bool wide_gated_supports(const BlockProduct& a) { return a.t == DType::BF16 && a.C % 8 == 0 && a.O % 16 == 0; }
hipError_t launch_wide_gated(const BlockProduct&, int, hipStream_t) { return reached(); }
bool wide_back_supports(const BlockProduct& a) { return a.t == DType::BF16 && a.C % 8 == 0 && a.O % 8 == 0; }
hipError_t launch_wide_back(const BlockProduct&, int, hipStream_t) { return reached(); }
bool grad_mfma_supports(const void*, const void*, DType t, int64_t, int64_t C, int64_t O, int32_t G) {
  return t == DType::BF16 && C % 8 == 0 && O % 8 == 0 && 128 % G == 0;
}
hipError_t launch_grad_mfma_to(const void*, const void*, int64_t, int64_t, const uint8_t*, int64_t, int32_t, int32_t,
                               void*, DType, hipStream_t) {
  return reached();
}
hipError_t launch_gate_grad(const void*, const void*, DType, int64_t, int64_t, Act, void*, hipStream_t) {
  return reached();
}
int64_t adapter_part_bytes(int64_t N, int64_t, int64_t, int32_t R) { return N * R * 4; }
hipError_t launch_adapters(const AdapterArgs& a, hipStream_t) {
  static_cast<char*>(a.D)[0] = static_cast<char*>(a.D)[a.N * a.O * (a.d_t == DType::F32 ? 4 : 2) - 1] = 1;
  a.part[0] = a.part[a.N * a.R - 1] = 1.0f;
  return reached();
}

}  // namespace cci

// cci_spmm as the adapters call it: a stand-in, so that cci_api.cpp's launchers are not needed here.
extern "C" cci_status cci_spmm(const void*, cci_dtype, int64_t, int64_t, const void*, cci_dtype, const uint8_t*, int64_t,
                               int32_t, int32_t, const cci_epilogue* ep, void*, cci_dtype, void*) {
  cci::reached();
  return ep && ep->residual ? CCI_OK : CCI_EINVAL;
}
