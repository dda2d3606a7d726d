// The bf16 products of a CCI-sparse feed-forward block over few tiles:
//   gated  H[n][f] = act(P[n][f]) P[n][F + f],  P = X . W_hat^T;
//   back   dX[n][c] = sum_o dY[n][o] W_hat[o][c].
// With few tiles of the output a workgroup's own latency and its LDS set the
// time.  The eight waves of a workgroup share one tile of 16 NT rows of X x 16
// WB rows of the expanded weight tile, not its outputs but its reduction:
// wave w takes the steps w, w + 8, ... of 128 / WB elements and holds the whole
// tile's sums.  So a wave never waits for another in the loop; every weight
// fragment read from LDS feeds NT MFMAs (waves that split the outputs of a 64 x
// 64 tile read 2.5 times the bytes per MFMA); the fragments of X come straight
// from memory, each once.  Loads run D steps ahead in registers; a step's
// weights (2048 entries) are expanded (zero fill, then every kept weight to its
// place: Alg. 1's row gG + idx, Sec. 3.2) into one of the wave's two LDS tiles
// while the MFMAs of the step before run.  The eight partial tiles meet in LDS
// at the end, added in the order of the waves.
// The LDS binds: a step is 4 zeroing stores, 8 per unit of kept entries and 4
// fragment reads, about 180 cycles whatever NT is.  Fewer rows than a tile
// holds cost nothing more; narrow tiles (WB) or fewer rows (NT) fill the CUs
// when there are few tiles (dX, 333 x 1000 -> 2728: 19.2 us on 258 tiles of 64
// rows, 11.4 on 473 of 32).
//
// Weight tile rows: gated 8 WB gate rows, then the up rows of the same
// outputs; back: columns c, the reduction element along the row.  LDS:
// element (row, k) at (row / 16) 32 KS + (k / 8) 256 + (row % 16) 16 + (k % 8) 2,
// the order of the MFMA fragments.
#include <type_traits>

#include "cci_act.hpp"
#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kGated = 0, kBack = 1;

struct SParams {
  const void* X;  // [N][ldx]
  const void* vals;
  const uint8_t* idx;
  void* Y;
  void* pre;
  int64_t N, C, O;
  int32_t G, K, y_f32, act;
  uint32_t nnb, nwb, grid;
};

constexpr int step_of(int wb) { return 128 / wb; }  // reduction elements of a step
template <int KS>
__device__ __forceinline__ uint32_t erow(uint32_t row) {
  return (row >> 4) * (32u * KS) + ((row & 15u) << 4);
}
__device__ __forceinline__ uint32_t ecol(uint32_t k) { return ((k >> 3) << 8) | ((k & 7u) << 1); }

// Row blocks of a pass of the final sum, and a wave's LDS: its two weight
// tiles, later its parts of the sums.
constexpr int sum_blocks(int nt) { return nt >= 2 ? 2 : 1; }
constexpr int kTile = 4096;
constexpr int wave_lds(int nt, int wb) {
  return wb * 1024 * sum_blocks(nt) > 2 * kTile ? wb * 1024 * sum_blocks(nt) : 2 * kTile;
}

// PL: packed units (8 columns of a packed row) of a lane and step; FIT: whole
// groups lie in a tile (gated: its rows, back: a step) and G is a power of
// two, so no entry has to be checked.
template <int MODE, int NT, int WB, int PL, bool FIT>
__global__ __launch_bounds__(kThreads, 2) void wave_split_kernel(SParams p) {
  constexpr int TN = 16 * NT, TW = 16 * WB;
  constexpr int R = MODE == kGated ? TW / 2 : TW;          // outputs of the tile along the weights
  constexpr int KS = step_of(WB), NK = KS / 32;            // a step's reduction elements and MFMA steps
  constexpr int UR = MODE == kGated ? KS / 8 : TW / 8;     // units of a packed row
  constexpr int D = NT * NK * 4 + PL * 6 <= 26 ? 4 : 2;    // steps in flight (registers)
  constexpr int NP = sum_blocks(NT), kLds = wave_lds(NT, WB);
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t li = lane & 15, lq = lane >> 4;
  uint8_t* tiles = lds + w * kLds;
  uint8_t* trash = lds + kWaves * kLds;  // entries of other tiles go here
  const bf16_t* X = global_ptr<const bf16_t>(p.X);
  const bf16_t* vals = global_ptr<const bf16_t>(p.vals);
  const uint8_t* idx = global_ptr<const uint8_t>(p.idx);

  // ---- tile of this workgroup: dispatch places workgroup b on XCD b % 8; an
  // XCD's workgroups run through bands of four row blocks x every weight block
  const uint32_t L = xcd_order(blockIdx.x, p.grid);
  const uint32_t per = 4u * p.nwb, band = L / per, within = L - band * per;
  const uint32_t rows = min(4u, p.nnb - 4u * band);
  const uint32_t wb = within / rows, nb = 4u * band + (within - wb * rows);
  // (back: a last tile of fewer columns starts earlier and computes some again)
  const int64_t n0 = static_cast<int64_t>(nb) * TN, w0 = MODE == kBack ? min(static_cast<int64_t>(wb) * R, p.C - R) : static_cast<int64_t>(wb) * R;
  const int64_t F = p.O / 2;
  const uint32_t red = static_cast<uint32_t>(MODE == kGated ? p.C : p.O);
  const uint32_t ldx = red;
  const int steps = static_cast<int>(red / KS);  // whole ones; a rest of the reduction is the last wave's turn after them

  // ---- X fragments: lane (li, lq) holds elements 8 lq .. +7 of row li of a
  // block.  Rows past the last read it again: their outputs are not stored.
  const char* xbase = reinterpret_cast<const char*>(X + n0 * ldx);
  uint32_t xoff[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
    xoff[n] = (static_cast<uint32_t>(min(static_cast<int64_t>(16 * n + li), p.N - 1 - n0)) * ldx + 8u * lq) * 2u;

  // ---- packed units.  Unit v of a step: packed row r = v / UR, its columns
  // 8 (v % UR) .. +7 of the step (gated) or of the tile (back).  Packed rows
  // count from the first group that meets the tile's gate rows, then from the
  // first that meets its up rows (gated), or from the step's first group.
  const uint32_t G = static_cast<uint32_t>(p.G);
  const uint32_t lim = MODE == kGated ? static_cast<uint32_t>(min(static_cast<int64_t>(R), F - w0)) : KS;
  const uint32_t g_gate = static_cast<uint32_t>(w0) / G;  // gated
  const int half = MODE == kGated ? static_cast<int>((static_cast<uint32_t>(w0) + lim - 1) / G - g_gate + 1) * p.K : 0;
  const uint32_t gps = MODE == kBack && FIT ? KS / G : 0;  // back: groups of a step, where they fit
  struct Span {
    uint32_t g_lo;  // first group
    int nrows;      // packed rows
    int first;      // g_lo G - first row (gated) or element of the step (back)
  };
  auto span_of = [&](int t) __attribute__((always_inline)) {
    if constexpr (MODE == kGated)
      return Span{g_gate, 2 * half, static_cast<int>(g_gate * G) - static_cast<int>(w0)};
    const uint32_t b = static_cast<uint32_t>(t) * KS, n = min(static_cast<uint32_t>(KS), red - b);
    if constexpr (FIT) return Span{static_cast<uint32_t>(t) * gps, static_cast<int>(n / G) * p.K, 0};
    const uint32_t lo = b / G;
    return Span{lo, static_cast<int>((b + n - 1) / G - lo + 1) * p.K, static_cast<int>(lo * G) - static_cast<int>(b)};
  };
  const int64_t up = F / p.G * p.K;  // packed rows from a gate row to its up row
  int grow[PL];                      // first row of a unit's group from its span's first (gated: of its half)
  bool second[PL];                   // gated: an up row
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const int r = (lane + 64 * i) / UR;
    second[i] = MODE == kGated && r >= half;
    grow[i] = (second[i] ? r - half : r) / p.K * p.G;
  }
  struct Set {
    Unit<bf16_t> x[NT][NK], v[PL];
    u32x2_t ix[PL];
  };
  // (The loop's loads have no branch: after one the compiler would wait for
  // every load in flight.)
  auto load = [&](int t, Set& s, auto rest) __attribute__((always_inline)) {
    constexpr bool kRest = decltype(rest)::value;  // a step of red % KS elements
    const uint32_t k0 = static_cast<uint32_t>(t) * KS;
    const char* xs = xbase + k0 * 2u;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const bf16_t* xp = reinterpret_cast<const bf16_t*>(xs + xoff[n]);
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        if constexpr (kRest)
          load_tail<8>(s.x[n][j], xp + 32 * j, static_cast<int>(red - k0) - 32 * j - 8 * static_cast<int>(lq));
        else
          load_full<8>(s.x[n][j], xp + 32 * j);
      }
    }
    const Span g = span_of(t);
    const int64_t c0 = MODE == kGated ? static_cast<int64_t>(k0) : w0;
    const int64_t at = static_cast<int64_t>(g.g_lo) * p.K * p.C + c0;
    const char* vb = reinterpret_cast<const char*>(vals + at);
    const uint8_t* ib = idx + at;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int v = lane + 64 * i, u = v % UR;
      // (a unit without a packed row reads the last one's and is not written)
      const int r = max(min(v / UR, g.nrows - 1), 0);
      const uint32_t row = static_cast<uint32_t>(MODE == kGated && r >= half ? r - half : r);
      const uint32_t off = row * static_cast<uint32_t>(p.C) + 8u * static_cast<uint32_t>(u);
      const int64_t far = MODE == kGated && r >= half ? up * p.C : 0;
      const bf16_t* vp = reinterpret_cast<const bf16_t*>(vb + 2 * far + 2u * off);
      const uint8_t* ip = ib + far + off;
      if constexpr (kRest && MODE == kGated) {
        load_tail<8>(s.v[i], vp, static_cast<int>(red - k0) - 8 * u);
        load_tail<8>(s.ix[i], ip, static_cast<int>(red - k0) - 8 * u);
      } else {
        load_full<8>(s.v[i], vp);
        load_full<8>(s.ix[i], ip);
      }
    }
  };
  // Order of a unit's entries: back, the rows of the packing over the eight
  // 16-byte slots of a column block; gated, the units of a row over a slot's words.
  const Shuffle sh = make_shuffle(MODE == kGated ? 2u * (static_cast<uint32_t>(lane) & 3u)
                                                 : static_cast<uint32_t>(lane / UR) & 7u);
  uint32_t eoff[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) eoff[e] = (MODE == kGated ? 2u : 16u) * (static_cast<uint32_t>(e) ^ sh.m);
  const uint32_t gmask = (G - 1u) * 0x01010101u;  // FIT: an index past its group stays in the tile
  auto expand = [&](int t, uint8_t* tile, Set& s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4_t*>(tile + i * 1024 + lane * 16) = u32x4_t{0u, 0u, 0u, 0u};
    asm volatile("" ::: "memory");  // the zeros come first; one wave's LDS writes stay in order
    const Span g = span_of(t);
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int v = lane + 64 * i;
      const uint32_t u = static_cast<uint32_t>(v % UR);
      const bool there = v / UR < g.nrows;
      const uint32_t row0 = static_cast<uint32_t>(g.first + grow[i]);
      const uint32_t r0 = second[i] ? static_cast<uint32_t>(R) : 0u;
      shuffle(sh, s.v[i], s.ix[i]);
      if constexpr (FIT) {
        if (there) {
          uint8_t* to = tile + (MODE == kGated ? erow<KS>(r0 + row0) + ecol(8 * u) : erow<KS>(8 * u) + ecol(row0));
          const u32x2_t im = {s.ix[i][0] & gmask, s.ix[i][1] & gmask};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t x = (im[e >> 2] >> (8 * (e & 3))) & 0xffu;
            const uint32_t at = (MODE == kGated ? (R > 16 ? erow<KS>(x) : x << 4) : ecol(x)) + eoff[e];
            *reinterpret_cast<uint16_t*>(to + at) = static_cast<uint16_t>(s.v[i].d[0][e >> 1] >> (16 * (e & 1)));
          }
        }
      } else {
        const uint32_t most = there ? lim : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t x = row0 + ((s.ix[i][e >> 2] >> (8 * (e & 3))) & 0xffu);
          const uint32_t at = (MODE == kGated ? erow<KS>(r0 + x) + ecol(8 * u) : erow<KS>(8 * u) + ecol(x)) + eoff[e];
          *reinterpret_cast<uint16_t*>(x < most ? tile + at : trash) =
              static_cast<uint16_t>(s.v[i].d[0][e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    asm volatile("" ::: "memory");
  };

  f32x4_t acc[WB][NT];
#pragma unroll
  for (int o = 0; o < WB; ++o)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[o][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const auto multiply = [&](const Unit<bf16_t> (&a)[4], const Set& s) __attribute__((always_inline)) {
#pragma unroll
    for (int o = 0; o < WB; ++o)
#pragma unroll
      for (int j = 0; j < NK; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) mma(acc[o][n], a[o * NK + j], s.x[n][j]);
  };
  const auto read = [&](const uint8_t* tile, Unit<bf16_t> (&a)[4]) __attribute__((always_inline)) {  // block o, MFMA step j at o NK + j
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i].d[0] = *reinterpret_cast<const u32x4_t*>(tile + i * 1024 + lane * 16);
    asm volatile("" ::: "memory");
  };

  // The wave's step i is w + 8 i, in set i % D and LDS tile i % 2.  Past the
  // end the last step is read again.
  Set set[D];
  const auto step = [&](int i) { return w + kWaves * i; };
  if (steps > 0) {
#pragma unroll
    for (int d = 0; d < D; ++d) load(min(step(d), steps - 1), set[d], std::false_type{});
    if (step(0) < steps) expand(step(0), tiles, set[0]);
  }
#pragma unroll 1
  for (int i0 = 0; step(i0) < steps; i0 += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int i = i0 + d;
      if (step(i) < steps) {
        Unit<bf16_t> a[4];
        read(tiles + (d & 1) * kTile, a);
        if (step(i + 1) < steps) expand(step(i + 1), tiles + ((d + 1) & 1) * kTile, set[(d + 1) % D]);
        multiply(a, set[d]);
      }
      load(min(step(i + D), steps - 1), set[d], std::false_type{});
    }
  }
  if (red % KS != 0 && w == steps % kWaves) {
    load(steps, set[0], std::true_type{});
    expand(steps, tiles, set[0]);
    Unit<bf16_t> a[4];
    read(tiles, a);
    multiply(a, set[0]);
  }

  // ---- the waves' sums, NP row blocks at a time: each wave parks its part,
  // then adds up one or more of the blocks (gated: a gate block and its up block)
  constexpr int kJobs = (MODE == kGated ? WB / 2 : WB) * NP;
  const auto parked = [&](int v, int o, int n) {
    return reinterpret_cast<f32x4_t*>(lds + v * kLds)[(o * NP + n) * 64 + lane];
  };
  const auto total = [&](int o, int n) __attribute__((always_inline)) {
    f32x4_t s = parked(0, o, n);
#pragma unroll
    for (int v = 1; v < kWaves; ++v) s += parked(v, o, n);
    return s;
  };
  const bool vec = (MODE == kGated ? F : p.C) % 4 == 0;
#pragma unroll
  for (int ps = 0; ps < NT / NP; ++ps) {
    __syncthreads();
#pragma unroll
    for (int o = 0; o < WB; ++o)
#pragma unroll
      for (int n = 0; n < NP; ++n)
        reinterpret_cast<f32x4_t*>(tiles)[(o * NP + n) * 64 + lane] = acc[o][ps * NP + n];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kJobs; j += kWaves) {
      const int job = j + w;
      if (job >= kJobs) break;
      const int n = job % NP, o = job / NP;
      const int64_t row = n0 + 16 * (ps * NP + n) + li, c = w0 + 16 * o + 4 * lq;
      if constexpr (MODE == kGated) {
        const f32x4_t sg = total(o, n), su = total(o + WB / 2, n);
        if (row < p.N) {
          const float g[4] = {sg[0], sg[1], sg[2], sg[3]}, u[4] = {su[0], su[1], su[2], su[3]};
          float h[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) h[r] = act_value(static_cast<Act>(p.act), g[r]) * u[r];
          store4<bf16_t>(global_ptr<bf16_t>(p.Y) + row * F + c, h, F - c, vec);
          if (p.pre) {
            bf16_t* q = global_ptr<bf16_t>(p.pre) + row * p.O + c;
            store4<bf16_t>(q, g, F - c, vec);
            store4<bf16_t>(q + F, u, F - c, vec);
          }
        }
      } else {
        const f32x4_t s = total(o, n);
        if (row < p.N) {
          const float v[4] = {s[0], s[1], s[2], s[3]};
          if (p.y_f32)
            store4<float>(global_ptr<float>(p.Y) + row * p.C + c, v, p.C - c, vec);
          else
            store4<bf16_t>(global_ptr<bf16_t>(p.Y) + row * p.C + c, v, p.C - c, vec);
        }
      }
    }
  }
}

template <int MODE, int NT, int WB, int PL, bool FIT>
hipError_t launch(SParams p, hipStream_t s) {
  const int64_t along = MODE == kGated ? p.O / 2 : p.C;
  constexpr int R = MODE == kGated ? 8 * WB : 16 * WB;
  const int64_t nnb = (p.N + 16 * NT - 1) / (16 * NT), nwb = (along + R - 1) / R;
  const uint32_t grid = static_cast<uint32_t>(nnb * nwb);
  p.nnb = static_cast<uint32_t>(nnb);
  p.nwb = static_cast<uint32_t>(nwb);
  p.grid = grid;
  constexpr int kLds = kWaves * wave_lds(NT, WB) + 16;
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t e =
      set_lds_limit_once(lds_set, reinterpret_cast<const void*>(&wave_split_kernel<MODE, NT, WB, PL, FIT>), kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((wave_split_kernel<MODE, NT, WB, PL, FIT>), dim3(grid), dim3(kThreads), kLds, s, p);
  return hipGetLastError();
}

// Packed units of a lane and step.
int64_t units(bool gated, int wb, int64_t G, int64_t K) {
  const int64_t rows = gated ? 2 * groups_in(8 * wb, G) * K : groups_in(step_of(wb), G) * K;
  return (rows * (gated ? step_of(wb) / 8 : 2 * wb) + 63) / 64;
}

template <int MODE, int NT, int WB>
hipError_t launch_pl(const SParams& p, hipStream_t s) {
  const bool fit = (p.G & (p.G - 1)) == 0 && p.G <= (MODE == kGated ? 8 * WB : step_of(WB));
  const int64_t pl = units(MODE == kGated, WB, p.G, p.K);
  if (fit) {
    if (pl <= 1) return launch<MODE, NT, WB, 1, true>(p, s);
    if (pl <= 2) return launch<MODE, NT, WB, 2, true>(p, s);
    return launch<MODE, NT, WB, 4, true>(p, s);
  }
  if (pl <= 2) return launch<MODE, NT, WB, 2, false>(p, s);
  return launch<MODE, NT, WB, 4, false>(p, s);
}

// rows: of a tile, 16, 32 or (back) 64.
template <int MODE, int WB>
hipError_t launch_wb(const SParams& p, int rows, hipStream_t s) {
  if (rows == 16) return launch_pl<MODE, 1, WB>(p, s);
  if (rows == 32) return launch_pl<MODE, 2, WB>(p, s);
  if constexpr (MODE == kBack) return launch_pl<MODE, 4, WB>(p, s);
  return hipErrorInvalidConfiguration;
}

template <int MODE>
hipError_t launch_nt(const BlockProduct& a, int wb, int rows, hipStream_t s) {
  SParams p{};
  p.X = MODE == kGated ? a.X : a.dY;
  p.vals = a.vals;
  p.idx = a.idx;
  p.Y = a.Y;
  p.pre = a.pre;
  p.N = a.N;
  p.C = a.C;
  p.O = a.O;
  p.G = a.G;
  p.K = a.K;
  p.y_f32 = a.y_t == DType::F32;
  p.act = static_cast<int32_t>(a.act);
  if (wb == 4) return launch_wb<MODE, 4>(p, rows, s);
  if (wb == 2) return launch_wb<MODE, 2>(p, rows, s);
  if constexpr (MODE == kBack) {
    if (wb == 1) return launch_wb<MODE, 1>(p, rows, s);
  }
  return hipErrorInvalidConfiguration;
}

}  // namespace

bool wave_split_supports(const BlockProduct& a, bool gated, int wb) {
  const int64_t out = gated ? a.O / 2 : a.C, width = (gated ? 8 : 16) * wb;
  if ((a.N + 15) / 16 * ((out + width - 1) / width) > kMostThreads / kThreads) return false;
  return a.t == DType::BF16 && a.N >= 1 && units(gated, wb, a.G, a.K) <= 4 &&
         (gated ? wb >= 2 : a.C >= 16 * wb);
}

hipError_t launch_wave_split(const BlockProduct& a, bool gated, int wb, int rows, hipStream_t s) {
  return gated ? launch_nt<kGated>(a, wb, rows, s) : launch_nt<kBack>(a, wb, rows, s);
}

}  // namespace cci
