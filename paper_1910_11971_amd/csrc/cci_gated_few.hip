// The gated product H = act(X Wg^T) * (X Wu^T) for few rows (N <= 64: a
// decoding batch), bf16.  Every packed weight meets at most 64 rows, so the
// packed bytes and the memory latency set the time: a workgroup of eight waves
// owns 16 outputs (16 gate and 16 up rows of the packing), wave w takes the
// 128-column chunks w, w + 8, ... of the reduction and keeps the loads of
// several in flight.  Per chunk a wave clears its 32 x 128 tile in LDS, writes
// the kept weights of its groups to their rows (Alg. 1's gG + idx, Sec. 3.2),
// reads the tile back as A fragments of v_mfma_f32_16x16x32_bf16 and
// multiplies them with up to four blocks of 16 rows of X.  The eight partial
// sums meet in LDS, where the gate and up sums of an output lie in one lane.
// Tile row r keeps its 16-byte unit u at 256 r + 16 (u ^ (r % 16)): the 16
// rows of a fragment read touch distinct bank slots.
#include <algorithm>

#include "cci_act.hpp"
#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kCols = 128, kUnits = kCols / 8, kSteps = kCols / 32;  // of a chunk
constexpr int kOut = 16;                                             // outputs of a workgroup
constexpr int kTile = 2 * kOut * kCols * 2;                          // bytes of a wave's tile

struct FParams {
  const uint16_t* X;
  const uint16_t* vals;
  const uint8_t* idx;
  void* H;
  void* pre;
  int64_t N, C, F;
  int32_t G, K, act;
};

template <int PL, int NB>
struct Fetch {
  Unit<bf16_t> v[PL];
  u32x2_t ix[PL];
  Unit<bf16_t> x[kSteps][NB];
};

// Chunks in flight per wave: as many as fit about 150 registers, at most 4.
constexpr int depth(int pl, int nb) {
  const int d = 150 / (pl * 6 + nb * kSteps * 4);
  return d < 1 ? 1 : d > 4 ? 4 : d;
}

// PL: packed units per lane of a chunk; ONE: that is all of them (else the rest is walked in passes).
template <int NB, int PL, bool ONE>
__global__ __launch_bounds__(kThreads, 2) void gated_few_kernel(FParams p) {
  constexpr int D = ONE ? depth(PL, NB) : 1;
  constexpr int kSums = 2 * NB * 64 * 16;
  __shared__ __attribute__((aligned(16))) uint8_t tiles[kWaves][kTile > kSums ? kTile : kSums];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lq = lane >> 4;
  const bf16_t* X = global_ptr<const bf16_t>(p.X);
  const bf16_t* vals = global_ptr<const bf16_t>(p.vals);
  const uint8_t* idx = global_ptr<const uint8_t>(p.idx);
  uint8_t* tile = tiles[w];
  const int64_t f0 = static_cast<int64_t>(blockIdx.x) * kOut;
  const int lim = static_cast<int>(min(static_cast<int64_t>(kOut), p.F - f0));
  // Packed rows: those of the groups that meet gate rows f0 .. f0 + lim - 1,
  // then the same of the up rows (F is a multiple of G).
  const int64_t g_lo = f0 / p.G;
  const int half = static_cast<int>((f0 + lim - 1) / p.G - g_lo + 1) * p.K;
  const int64_t up = p.F / p.G * p.K;  // packed rows from a gate row to its up row
  const int first = static_cast<int>(g_lo * p.G - f0);
  // unit v of the wave: packed row v / kUnits, columns 8 (v % kUnits) .. +7 of the chunk
  auto load_unit = [&](int64_t c0, int v, Unit<bf16_t>& val, u32x2_t& ix) __attribute__((always_inline)) {
    const int r = v / kUnits;
    const int64_t row = g_lo * p.K + (r < half ? r : r - half + up), c = c0 + 8 * (v % kUnits);
    const int64_t left = r < 2 * half ? p.C - c : 0;
    load_elems<8>(val, vals + row * p.C + c, left);
    load_elems<8>(ix, idx + row * p.C + c, left);
  };
  auto scatter = [&](int v, const Unit<bf16_t>& val, const u32x2_t& ix) __attribute__((always_inline)) {
    const int r = v / kUnits, u = v % kUnits;
    if (r >= 2 * half) return;
    const bool second = r >= half;
    const int row0 = first + (second ? r - half : r) / p.K * p.G;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = row0 + static_cast<int>((ix[e >> 2] >> (8 * (e & 3))) & 0xffu);
      if (t >= 0 && t < lim)
        *reinterpret_cast<uint16_t*>(tile + (second ? kOut * 256 : 0) + t * 256 + ((u ^ t) << 4) + 2 * e) =
            static_cast<uint16_t>(val.d[0][e >> 1] >> (16 * (e & 1)));
    }
  };
  auto fetch = [&](int64_t ch, Fetch<PL, NB>& f) __attribute__((always_inline)) {
    const int64_t c0 = ch * kCols;
    if constexpr (ONE) {
#pragma unroll
      for (int i = 0; i < PL; ++i) load_unit(c0, lane + 64 * i, f.v[i], f.ix[i]);
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int64_t n = 16 * nb + li, c = c0 + 32 * j + 8 * lq;
        load_elems<8>(f.x[j][nb], X + n * p.C + c, n < p.N ? p.C - c : 0);
      }
  };

  f32x4_t acc[2][NB];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[h][nb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int64_t nch = (p.C + kCols - 1) / kCols;
  Fetch<PL, NB> st[D];
#pragma unroll
  for (int d = 0; d < D; ++d)
    if (w + kWaves * d < nch) fetch(w + kWaves * d, st[d]);
  for (int64_t base = w; base < nch; base += kWaves * D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int64_t ch = base + kWaves * d;
      if (ch < nch) {
#pragma unroll
        for (int q = 0; q < kTile / 1024; ++q)
          *reinterpret_cast<u32x4_t*>(tile + q * 1024 + lane * 16) = u32x4_t{0u, 0u, 0u, 0u};
        asm volatile("" ::: "memory");  // the zeros come first; one wave's LDS writes stay in order
        if constexpr (ONE) {
#pragma unroll
          for (int i = 0; i < PL; ++i) scatter(lane + 64 * i, st[d].v[i], st[d].ix[i]);
        } else {
#pragma unroll 1
          for (int v = lane; v < 2 * half * kUnits; v += 64 * PL) {
#pragma unroll
            for (int i = 0; i < PL; ++i) load_unit(ch * kCols, v + 64 * i, st[d].v[i], st[d].ix[i]);
#pragma unroll
            for (int i = 0; i < PL; ++i) scatter(v + 64 * i, st[d].v[i], st[d].ix[i]);
          }
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            Unit<bf16_t> a;
            a.d[0] = *reinterpret_cast<const u32x4_t*>(tile + h * (kOut * 256) + li * 256 + (((4 * j + lq) ^ li) << 4));
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma(acc[h][nb], a, st[d].x[j][nb]);
          }
        asm volatile("" ::: "memory");  // the tile is read before it is cleared again
        if (ch + kWaves * D < nch) fetch(ch + kWaves * D, st[d]);
      }
    }
  }

  // ---- the waves' sums; wave nb finishes rows 16 nb .. +15 of X: lane (li, lq) holds outputs 4 lq .. +3 of row li
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) reinterpret_cast<f32x4_t*>(tile)[(h * NB + nb) * 64 + lane] = acc[h][nb];
  __syncthreads();
  if (w >= NB) return;
  f32x4_t s[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    s[h] = reinterpret_cast<const f32x4_t*>(tiles[0])[(h * NB + w) * 64 + lane];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) s[h] += reinterpret_cast<const f32x4_t*>(tiles[v])[(h * NB + w) * 64 + lane];
  }
  const int64_t n = 16 * w + li, f = f0 + 4 * lq;
  if (n >= p.N) return;
  const Act act = static_cast<Act>(p.act);
  const bool vec = p.F % 4 == 0;
  float g[4], u[4], h[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    g[r] = s[0][r];
    u[r] = s[1][r];
    h[r] = act_value(act, g[r]) * u[r];
  }
  store4<bf16_t>(global_ptr<bf16_t>(p.H) + n * p.F + f, h, p.F - f, vec);
  if (p.pre) {
    bf16_t* q = global_ptr<bf16_t>(p.pre) + n * 2 * p.F + f;
    store4<bf16_t>(q, g, p.F - f, vec);
    store4<bf16_t>(q + p.F, u, p.F - f, vec);
  }
}

template <int NB>
hipError_t launch(const FParams& p, int64_t rows, uint32_t grid, hipStream_t s) {
  const int64_t pl = (2 * rows * kUnits + 63) / 64;
  const auto kernel = pl <= 1 ? gated_few_kernel<NB, 1, true> : pl <= 2 ? gated_few_kernel<NB, 2, true>
                      : pl <= 4 ? gated_few_kernel<NB, 4, true> : gated_few_kernel<NB, 4, false>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

bool gated_few_supports(const BlockProduct& a) { return a.t == DType::BF16 && a.N <= 64; }

hipError_t launch_gated_few(const BlockProduct& a, hipStream_t s) {
  FParams p{};
  p.X = static_cast<const uint16_t*>(a.X);
  p.vals = static_cast<const uint16_t*>(a.vals);
  p.idx = a.idx;
  p.H = a.Y;
  p.pre = a.pre;
  p.N = a.N;
  p.C = a.C;
  p.F = a.O / 2;
  p.G = a.G;
  p.K = a.K;
  p.act = static_cast<int32_t>(a.act);
  const int64_t grid = (p.F + kOut - 1) / kOut;
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  const int64_t rows = groups_in(kOut, a.G) * a.K;  // packed rows behind 16 outputs, at most
  const uint32_t g = static_cast<uint32_t>(grid);
  return a.N <= 16 ? launch<1>(p, rows, g, s) : a.N <= 32 ? launch<2>(p, rows, g, s) : launch<4>(p, rows, g, s);
}

}  // namespace cci
