// CCI-sparse product on the matrix cores: wide-tile kernels for large FC and
// stride-1 1x1 products (the method, work split and layouts are described at
// their body, cci_wide_body.hpp).
#include "cci_wide_body.hpp"

namespace cci {
namespace {

// (The body is a device function: with it inside the kernel template, the
// host pass of this compiler emitted no launch stubs for the kernels.)
template <typename YT, int PT, int UPL, int UE, bool FULL, bool BIGG, bool MASK>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
void wide_tile_kernel(WParams p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  wide_tile_body<kWPlain, YT, PT, UPL, UE, FULL, BIGG, MASK>(p, lds);
}

// Rows of X are pixels: FC, or a 1x1 convolution with unit stride and no
// padding over NHWC activations.
bool plain_rows(const ProductArgs& a) {
  if (!a.conv) return true;
  const ConvGeom& g = a.geom;
  return g.KH == 1 && g.KW == 1 && g.sh == 1 && g.sw == 1 && g.ph == 0 && g.pw == 0;
}

template <typename YT, int PT, int UPL, int UE, bool FULL, bool BIGG, bool MASK>
hipError_t launch_wu(const WParams& p, uint32_t grid, hipStream_t s) {
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t attr = set_lds_limit_once(
      lds_set, reinterpret_cast<const void*>(&wide_tile_kernel<YT, PT, UPL, UE, FULL, BIGG, MASK>), kLds);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((wide_tile_kernel<YT, PT, UPL, UE, FULL, BIGG, MASK>), dim3(grid), dim3(kThreads), kLds, s, p);
  return hipGetLastError();
}

template <typename YT, int PT, bool BIGG, int UPL>
hipError_t launch_wm(const WParams& p, uint32_t grid, hipStream_t s) {
  return p.rows_w == 8 * UPL ? launch_wu<YT, PT, UPL, 8, false, BIGG, false>(p, grid, s)
                             : launch_wu<YT, PT, UPL, 8, false, BIGG, true>(p, grid, s);
}

template <typename YT, int PT, bool BIGG>
hipError_t launch_wg(const WParams& p, uint32_t grid, hipStream_t s) {
  // packed elements per lane per chunk: rows_w (= 64 K / G)
  if (p.rows_w == 4) return launch_wu<YT, PT, 1, 4, false, BIGG, false>(p, grid, s);
  if (p.rows_w <= 8) return launch_wm<YT, PT, BIGG, 1>(p, grid, s);
  if (p.rows_w <= 16) return launch_wm<YT, PT, BIGG, 2>(p, grid, s);
  if (p.rows_w <= 32) return launch_wm<YT, PT, BIGG, 4>(p, grid, s);
  return launch_wu<YT, PT, 8, 8, false, BIGG, true>(p, grid, s);
}

template <typename YT, int PT>
hipError_t launch_wp(const WParams& p, uint32_t grid, hipStream_t s) {
  if (p.K == p.G) return launch_wu<YT, PT, 8, 8, true, false, false>(p, grid, s);
  return p.G > 16 ? launch_wg<YT, PT, true>(p, grid, s) : launch_wg<YT, PT, false>(p, grid, s);
}

// Pixels per workgroup tile: 256, or 128 when 256-pixel tiles would leave
// more than half of the CUs idle.
int tile_pixels(int64_t N, int64_t O) { return (N + 255) / 256 * (O / kTile) >= 128 ? 256 : 128; }

}  // namespace

bool wide_tile_supports(const ProductArgs& a) {
  if (a.x_t != DType::BF16 || a.val_t != DType::BF16) return false;
  if (!plain_rows(a)) return false;
  if (a.G < 1 || a.G > 64 || 64 % a.G != 0 || a.K < 1 || a.K > a.G) return false;
  if (a.C % kCK != 0 || a.O % kTile != 0 || a.N < 1) return false;
  const auto al = [](const void* q, uintptr_t m) { return (reinterpret_cast<uintptr_t>(q) & (m - 1)) == 0; };
  if (!al(a.X, 16) || !al(a.vals, 16) || !al(a.idx, 8) || !al(a.Y, 16)) return false;
  if ((a.scale && !al(a.scale, 16)) || (a.bias && !al(a.bias, 16)) || (a.residual && !al(a.residual, 16)))
    return false;
  // every buffer offset is 32-bit and stays below the out-of-range marker
  const int64_t lim = static_cast<int64_t>(kOOB);
  const int64_t packed = (a.O / a.G) * a.K * a.C;
  if (a.N * a.C * 2 >= lim || packed * 2 >= lim || a.N * a.O * (a.y_t == DType::F32 ? 4 : 2) >= lim) return false;
  return true;
}

hipError_t launch_wide_tile(const ProductArgs& a, hipStream_t s) {
  if (!wide_tile_supports(a)) return hipErrorInvalidConfiguration;
  WParams p{};
  p.X = static_cast<const uint16_t*>(a.X);
  p.vals = static_cast<const uint16_t*>(a.vals);
  p.idx = a.idx;
  p.scale = a.scale;
  p.bias = a.bias;
  p.residual = a.residual;
  p.Y = a.Y;
  const int64_t ysz = a.y_t == DType::F32 ? 4 : 2;
  const int64_t packed = (a.O / a.G) * a.K * a.C;
  p.x_bytes = static_cast<uint32_t>(a.N * a.C * 2);
  p.v_bytes = static_cast<uint32_t>(packed * 2);
  p.i_bytes = static_cast<uint32_t>(packed);
  p.y_bytes = static_cast<uint32_t>(a.N * a.O * ysz);
  p.N = static_cast<int32_t>(a.N);
  p.C = static_cast<int32_t>(a.C);
  p.O = static_cast<int32_t>(a.O);
  p.G = a.G;
  p.K = a.K;
  p.relu = a.relu;
  p.pitch = p.C;
  p.OW = p.O;
  const int tp = tile_pixels(a.N, a.O);
  p.npb = static_cast<int32_t>((a.N + tp - 1) / tp);
  p.nob = static_cast<int32_t>(a.O / kTile);
  p.nch = static_cast<int32_t>(a.C / kCK);
  p.rows_w = 64 * a.K / a.G;
  const int64_t grid = static_cast<int64_t>(p.npb) * p.nob;
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  p.grid8 = grid % 8 == 0 ? static_cast<int32_t>(grid / 8) : 0;
  // An XCD running P pixel blocks x (32 / P) output blocks fetches P blocks
  // of X (256 C bf16 each) and 32 / P blocks of packed rows (256 C K / G
  // values and indices, 3 bytes each): 2 beats 4 when 8 K / G < 4 / 3.
  p.pgr = 6 * a.K < a.G ? 2 : 4;
  const uint32_t g = static_cast<uint32_t>(grid);
  if (tp == 256) return a.y_t == DType::BF16 ? launch_wp<bf16_t, 8>(p, g, s) : launch_wp<float, 8>(p, g, s);
  return a.y_t == DType::BF16 ? launch_wp<bf16_t, 4>(p, g, s) : launch_wp<float, 4>(p, g, s);
}

}  // namespace cci
