// Launch of the wide-tile kernels of the feed-forward block: the gated product
// (cci_wide_gated.hip) and the transposed one (cci_wide_back.hip).
#pragma once

#include "cci_block.hpp"
#include "cci_wide_body.hpp"

namespace cci {
namespace {

template <int MODE, int PT, int UPL, int UE, bool BIGG, bool MASK>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void wide_block_kernel(WParams p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  wide_tile_body<MODE, bf16_t, PT, UPL, UE, false, BIGG, MASK>(p, lds);
}

template <int MODE, int PT, int UPL, int UE, bool BIGG, bool MASK>
hipError_t launch(const WParams& p, uint32_t grid, hipStream_t s) {
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t attr =
      set_lds_limit_once(lds_set, reinterpret_cast<const void*>(&wide_block_kernel<MODE, PT, UPL, UE, BIGG, MASK>), kLds);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((wide_block_kernel<MODE, PT, UPL, UE, BIGG, MASK>), dim3(grid), dim3(kThreads), kLds, s, p);
  return hipGetLastError();
}

template <int MODE, int PT, bool BIGG, int UPL>
hipError_t launch_m(const WParams& p, bool ragged, uint32_t grid, hipStream_t s) {
  return p.rows_w == 8 * UPL && !ragged ? launch<MODE, PT, UPL, 8, BIGG, false>(p, grid, s)
                                        : launch<MODE, PT, UPL, 8, BIGG, true>(p, grid, s);
}

template <int MODE, int PT, bool BIGG>
hipError_t launch_g(const WParams& p, bool ragged, uint32_t grid, hipStream_t s) {
  // packed elements per lane per chunk: rows_w (= 64 K / G)
  if (p.rows_w == 4 && !ragged) return launch<MODE, PT, 1, 4, BIGG, false>(p, grid, s);
  if (p.rows_w <= 8) return launch_m<MODE, PT, BIGG, 1>(p, ragged, grid, s);
  if (p.rows_w <= 16) return launch_m<MODE, PT, BIGG, 2>(p, ragged, grid, s);
  if (p.rows_w <= 32) return launch_m<MODE, PT, BIGG, 4>(p, ragged, grid, s);
  return launch<MODE, PT, 8, 8, BIGG, true>(p, grid, s);
}

// Reduction length, outputs of a row, and outputs of a tile.
struct Shape {
  int64_t red, out, tile;
};
template <int MODE>
Shape shape(const BlockProduct& a) {
  return MODE == kWGated ? Shape{a.C, a.O / 2, 128} : Shape{a.O, a.C, 256};
}

template <int MODE>
bool supports(const BlockProduct& a) {
  if (a.t != DType::BF16 || (MODE == kWBack && a.y_t != DType::BF16)) return false;
  const Shape q = shape<MODE>(a);
  if (a.G > 64 || 64 % a.G != 0 || q.red % 8 != 0 || q.out % 8 != 0 || a.N < 1) return false;
  // every buffer offset is 32-bit and stays below the out-of-range marker, also that of the last chunk's blank lanes
  const int64_t lim = static_cast<int64_t>(kOOB);
  const int64_t packed = a.O / a.G * a.K * a.C;
  if ((a.N + 1) * q.red * 2 + 4096 >= lim || (packed + 64 * a.C) * 2 >= lim || a.N * q.out * 4 >= lim) return false;
  return true;
}

template <int MODE>
hipError_t launch_wide(const BlockProduct& a, int pt, hipStream_t s) {
  if (!supports<MODE>(a)) return hipErrorInvalidConfiguration;
  const Shape q = shape<MODE>(a);
  WParams p{};
  p.X = static_cast<const uint16_t*>(MODE == kWGated ? a.X : a.dY);
  p.vals = static_cast<const uint16_t*>(a.vals);
  p.idx = a.idx;
  p.Y = a.Y;
  p.pre = a.pre;
  const int64_t packed = a.O / a.G * a.K * a.C;
  p.x_bytes = static_cast<uint32_t>(a.N * q.red * 2);
  p.v_bytes = static_cast<uint32_t>(packed * 2);
  p.i_bytes = static_cast<uint32_t>(packed);
  p.y_bytes = static_cast<uint32_t>(a.N * q.out * 2);
  p.N = static_cast<int32_t>(a.N);
  p.C = static_cast<int32_t>(q.red);
  p.O = static_cast<int32_t>(a.O);
  p.G = a.G;
  p.K = a.K;
  p.act = static_cast<int32_t>(a.act);
  p.pitch = static_cast<int32_t>(a.C);
  p.OW = static_cast<int32_t>(q.out);
  p.up = static_cast<int32_t>(MODE == kWGated ? a.O / 2 / a.G * a.K : 0);
  p.npb = static_cast<int32_t>((a.N + 32 * pt - 1) / (32 * pt));
  p.nob = static_cast<int32_t>((q.out + q.tile - 1) / q.tile);
  p.nch = static_cast<int32_t>((q.red + kCK - 1) / kCK);
  p.rows_w = 64 * a.K / a.G;
  const int64_t grid = static_cast<int64_t>(p.npb) * p.nob;
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  p.pgr = 6 * a.K < a.G ? 2 : 4;  // (as for the plain product)
  const bool ragged = q.red % kCK != 0 || q.out % q.tile != 0;
  const uint32_t g = static_cast<uint32_t>(grid);
  const bool big = a.G > (MODE == kWBack ? 8 : 16);
  if (pt == 4) return big ? launch_g<MODE, 4, true>(p, ragged, g, s) : launch_g<MODE, 4, false>(p, ragged, g, s);
  return big ? launch_g<MODE, 8, true>(p, ragged, g, s) : launch_g<MODE, 8, false>(p, ragged, g, s);
}

}  // namespace
}  // namespace cci
