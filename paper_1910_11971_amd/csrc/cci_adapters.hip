// Low-rank adapters of many requests: for row n with adapter a = rows[n],
//   D[n][o] = residual[n][o] + alpha[a] sum_r T[n][r] B[a][o][r],  T[n][r] = sum_c A[a][r][c] X[n][c];
// a row whose adapter is outside [0, L) gets the residual alone.  The shared
// projection then takes D as its residual, so the sum is rounded once more
// than the projection alone (D, in the output's type, is a small part of it).
//
// Both kernels work on tiles of 16 rows and walk over the distinct adapters
// among them: the matrix cores multiply all 16 rows by one adapter, and the
// rows that have it keep the result.  A prompt's tile has one or two; a
// decoding batch up to 16, whose weights have to be read in any case.
//   shrink  T: a workgroup of four waves sums one of S column ranges of one
//           tile, the waves taking turns at its 32-column steps, and adds the
//           four partial tiles in LDS.  With few tiles P workgroups share the
//           distinct adapters of one.  The S partial sums stay apart (fp32):
//           no atomics, equal calls give equal bits.
//   expand  a wave adds them up in order and multiplies by 64 rows of B.  With
//           bf16 operands T enters as the sum of two bf16 values (16 bits of
//           mantissa): it is not rounded to one.
// Adapter weights bind while decoding, X (shrink) and D (expand) for prompts.
#include <algorithm>

#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kRows = 16;       // rows of a tile
constexpr int kRankBlocks = 4;  // blocks of 16 ranks a shrink pass accumulates
constexpr int kOutBlocks = 4;   // blocks of 16 outputs of an expand wave

struct APlan {
  int32_t S, P;      // column ranges, workgroups sharing a tile's adapters
  int64_t tiles;
  int64_t cols;      // columns of a range (a multiple of 128)
};

struct AParams {
  const void* X;
  const void* A;
  const void* B;
  const float* alpha;
  const int32_t* rows;
  const void* residual;
  void* D;
  float* part;  // [S][N][R]
  int64_t N, C, O, L, cols;
  int32_t R, S, P, d_f32;
};

// The adapter of row n of the tile (-1: none), for lane n % 16.
__device__ __forceinline__ int32_t row_adapter(const AParams& p, int64_t n) {
  if (n >= p.N) return -1;
  const int32_t a = global_ptr<const int32_t>(p.rows)[n];
  return a >= 0 && a < p.L ? a : -1;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void shrink_kernel(AParams p) {
  __shared__ f32x4_t red[kWaves][kRankBlocks][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t li = lane & 15, lq = lane >> 4;
  const uint32_t per = static_cast<uint32_t>(p.S) * static_cast<uint32_t>(p.P);
  const uint32_t tile = blockIdx.x / per, rest = blockIdx.x - tile * per;
  const int32_t sl = static_cast<int32_t>(rest / p.P), turn = static_cast<int32_t>(rest % p.P);
  const int64_t n = static_cast<int64_t>(tile) * kRows + li;
  const int64_t c_lo = sl * p.cols, c_hi = min(p.C, c_lo + p.cols);
  const T* x = global_ptr<const T>(p.X) + min(n, p.N - 1) * p.C;  // (rows past the last have no adapter)
  const T* A = global_ptr<const T>(p.A);
  float* part = global_ptr<float>(p.part);
  const int32_t mine = row_adapter(p, n);
  const int rank_blocks = (p.R + 15) / 16;
  uint64_t todo = __ballot(mine >= 0) & 0xffffu;  // rows (lanes 0 .. 15) still to do
  for (int32_t ord = 0; todo; ++ord) {
    const int32_t a = __builtin_amdgcn_readfirstlane(__shfl(mine, __builtin_ctzll(todo)));
    todo &= ~__ballot(mine == a);
    if (ord % p.P != turn) continue;
    for (int rb0 = 0; rb0 < rank_blocks; rb0 += kRankBlocks) {
      f32x4_t acc[kRankBlocks];
#pragma unroll
      for (int b = 0; b < kRankBlocks; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const int nb = min(kRankBlocks, rank_blocks - rb0);
      const int64_t r0 = 16 * rb0 + li;
      const T* ar = A + static_cast<int64_t>(a) * p.R * p.C;
      for (int64_t c0 = c_lo + 32 * w; c0 < c_hi; c0 += 32 * kWaves) {
        const int64_t c = c0 + 8 * lq, left = p.C - c;
        const bool whole = c0 + 32 <= p.C;
        Unit<T> xf, af[kRankBlocks];
        load_part<8>(xf, x + c, left, whole);
#pragma unroll
        for (int b = 0; b < kRankBlocks; ++b)  // (ranks past the last read it again: their sums are not stored)
          if (b < nb) load_part<8>(af[b], ar + min(r0 + 16 * b, static_cast<int64_t>(p.R - 1)) * p.C + c, left, whole);
#pragma unroll
        for (int b = 0; b < kRankBlocks; ++b)
          if (b < nb) mma(acc[b], af[b], xf);
      }
      __syncthreads();  // the previous pass's sums are read
#pragma unroll
      for (int b = 0; b < kRankBlocks; ++b)
        if (b < nb) red[w][b][lane] = acc[b];
      __syncthreads();
      // wave w finishes block w: lane (li, lq) holds ranks 16 (rb0 + w) + 4 lq .. +3 of row li
      if (w < nb && mine == a) {
        const f32x4_t t = red[0][w][lane] + red[1][w][lane] + red[2][w][lane] + red[3][w][lane];
        const int64_t r = 16 * (rb0 + w) + 4 * lq;
        const float v[4] = {t[0], t[1], t[2], t[3]};
        store4<float>(part + (static_cast<int64_t>(sl) * p.N + n) * p.R + r, v, p.R - r, p.R % 4 == 0);
      }
    }
  }
}

// T as MFMA operands: fp32 as it is, bf16 as high part + low part.
struct Split {
  Unit<bf16_t> hi, lo;
};
__device__ __forceinline__ Split split(const float (&t)[8]) {
  Split s;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      hi[i] = f32_to_bf16_rne(t[e + i]);
      const float d = t[e + i] - bf16_to_f32(static_cast<uint16_t>(hi[i]));
      lo[i] = __builtin_isfinite(d) ? f32_to_bf16_rne(d) : 0u;  // (an infinite T stays infinite)
    }
    s.hi.d[0][e >> 1] = hi[0] | (hi[1] << 16);
    s.lo.d[0][e >> 1] = lo[0] | (lo[1] << 16);
  }
  return s;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void expand_kernel(AParams p, uint32_t nob) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t li = lane & 15, lq = lane >> 4;
  const uint32_t tile = blockIdx.x / nob, ob = blockIdx.x - tile * nob;
  const int64_t n = static_cast<int64_t>(tile) * kRows + li;
  const int64_t o0 = (static_cast<int64_t>(ob) * kWaves + w) * (16 * kOutBlocks);
  const T* B = global_ptr<const T>(p.B);
  const float* part = global_ptr<const float>(p.part);
  const int32_t mine = row_adapter(p, n);
  f32x4_t out[kOutBlocks];
#pragma unroll
  for (int b = 0; b < kOutBlocks; ++b) out[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  uint64_t todo = __ballot(mine >= 0) & 0xffffu;
  if (o0 >= p.O) return;
  while (todo) {
    const int32_t a = __builtin_amdgcn_readfirstlane(__shfl(mine, __builtin_ctzll(todo)));
    todo &= ~__ballot(mine == a);
    const float s = p.alpha ? global_ptr<const float>(p.alpha)[a] : 1.0f;
    f32x4_t acc[kOutBlocks];
#pragma unroll
    for (int b = 0; b < kOutBlocks; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int32_t rs = 0; rs < p.R; rs += 32) {
      const int32_t r0 = rs + 8 * static_cast<int32_t>(lq);
      // ranks r0 .. r0 + 7 of row li, the column ranges' sums added in order
      float t[8] = {};
      if (mine == a) {
        for (int32_t k = 0; k < p.S; ++k) {
          Unit<float> u;
          load_elems<8>(u, part + (static_cast<int64_t>(k) * p.N + n) * p.R + r0, p.R - r0);
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] += __uint_as_float(u.d[e >> 2][e & 3]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= s;
      }
      Unit<T> bf[kOutBlocks];
#pragma unroll
      for (int b = 0; b < kOutBlocks; ++b) {
        const int64_t o = min(o0 + 16 * b + li, p.O - 1);  // (outputs past the last are not stored)
        load_elems<8>(bf[b], B + (static_cast<int64_t>(a) * p.O + o) * p.R + r0, p.R - r0);
      }
      if constexpr (sizeof(T) == 2) {
        const Split q = split(t);
#pragma unroll
        for (int b = 0; b < kOutBlocks; ++b) {
          mma(acc[b], bf[b], q.lo);
          mma(acc[b], bf[b], q.hi);
        }
      } else {
        Unit<float> q;
#pragma unroll
        for (int e = 0; e < 8; ++e) q.d[e >> 2][e & 3] = __float_as_uint(t[e]);
#pragma unroll
        for (int b = 0; b < kOutBlocks; ++b) mma(acc[b], bf[b], q);
      }
    }
#pragma unroll
    for (int b = 0; b < kOutBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) out[b][r] = mine == a ? acc[b][r] : out[b][r];
  }
  if (n >= p.N) return;
  const bool vec = p.O % 4 == 0;
#pragma unroll
  for (int b = 0; b < kOutBlocks; ++b) {
    const int64_t o = o0 + 16 * b + 4 * lq, at = n * p.O + o;
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      v[r] = out[b][r];
      if (p.residual && o + r < p.O)
        v[r] += p.d_f32 ? global_ptr<const float>(p.residual)[at + r]
                        : bf16_to_f32(global_ptr<const uint16_t>(p.residual)[at + r]);
    }
    if (p.d_f32)
      store4<float>(global_ptr<float>(p.D) + at, v, p.O - o, vec);
    else
      store4<bf16_t>(global_ptr<bf16_t>(p.D) + at, v, p.O - o, vec);
  }
}

// expand for few rows: a workgroup has one row and 256 outputs, a lane one
// output, whose R weights meet T's row in LDS on the vector ALUs (fp32).  A
// decoding batch has nearly as many adapters as rows, and the matrix cores'
// walk over a tile's adapters is a chain of memory latencies: 32 rows, 16
// adapters, 4096 outputs, R = 16: 79 us there.
template <typename T>
__global__ __launch_bounds__(kThreads) void expand_rows_kernel(AParams p, uint32_t nob) {
  extern __shared__ __attribute__((aligned(16))) float t[];  // [R rounded up to 8]
  const int64_t n = blockIdx.x / nob;
  const int64_t o = static_cast<int64_t>(blockIdx.x - static_cast<uint32_t>(n) * nob) * kThreads + threadIdx.x;
  const int32_t a = __builtin_amdgcn_readfirstlane(row_adapter(p, n));
  float v = 0.0f;
  if (a >= 0) {
    const float* part = global_ptr<const float>(p.part);
    const float s = p.alpha ? global_ptr<const float>(p.alpha)[a] : 1.0f;
    const int32_t padded = (p.R + 7) & ~7;
    for (int32_t r = threadIdx.x; r < padded; r += kThreads) {
      float sum = 0.0f;
      if (r < p.R)
        for (int32_t k = 0; k < p.S; ++k) sum += part[(static_cast<int64_t>(k) * p.N + n) * p.R + r];
      t[r] = sum * s;
    }
    __syncthreads();
    if (o < p.O) {
      const T* b = global_ptr<const T>(p.B) + (static_cast<int64_t>(a) * p.O + o) * p.R;
      for (int32_t r = 0; r < p.R; r += 8) {
        Unit<T> u;
        load_elems<8>(u, b + r, p.R - r);
#pragma unroll
        for (int e = 0; e < 8; ++e) v = __builtin_fmaf(elem(u, e), t[r + e], v);
      }
    }
  }
  if (o >= p.O) return;
  const int64_t at = n * p.O + o;
  if (p.residual)
    v += p.d_f32 ? global_ptr<const float>(p.residual)[at] : bf16_to_f32(global_ptr<const uint16_t>(p.residual)[at]);
  if (p.d_f32)
    global_ptr<float>(p.D)[at] = v;
  else
    global_ptr<uint16_t>(p.D)[at] = f32_to_bf16_rne(v);
}

constexpr int64_t kFewRows = 64;  // expand on the vector ALUs up to so many rows

// About 512 workgroups: column ranges of at least 256 columns first, then,
// for a decoding batch's few tiles, workgroups that share the adapters.
APlan plan(int64_t N, int64_t C, int64_t L) {
  APlan q{};
  q.tiles = (N + kRows - 1) / kRows;
  const int64_t want = std::max<int64_t>(1, 512 / std::max<int64_t>(q.tiles, 1));
  const int64_t S = std::min<int64_t>(std::min<int64_t>(want, 16), (C + 255) / 256);
  q.cols = (C + S - 1) / S;
  q.cols = (q.cols + 127) / 128 * 128;
  q.S = static_cast<int32_t>((C + q.cols - 1) / q.cols);
  q.P = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(16, std::min(L, N)), want * 2 / q.S)));
  return q;
}

}  // namespace

int64_t adapter_part_bytes(int64_t N, int64_t C, int64_t L, int32_t R) { return plan(N, C, L).S * N * R * 4; }

hipError_t launch_adapters(const AdapterArgs& a, hipStream_t s) {
  const APlan q = plan(a.N, a.C, a.L);
  AParams p{};
  p.X = a.X;
  p.A = a.A;
  p.B = a.B;
  p.alpha = a.alpha;
  p.rows = a.rows;
  p.residual = a.residual;
  p.D = a.D;
  p.part = a.part;
  p.N = a.N;
  p.C = a.C;
  p.O = a.O;
  p.L = a.L;
  p.cols = q.cols;
  p.R = a.R;
  p.S = q.S;
  p.P = q.P;
  p.d_f32 = a.d_t == DType::F32;
  const int64_t g1 = q.tiles * q.S * q.P;
  const int64_t nob = (a.O + kWaves * 16 * kOutBlocks - 1) / (kWaves * 16 * kOutBlocks);
  if (g1 > 0x7fffffff || nob > 0x7fffffff || q.tiles > 0x7fffffff / nob) return hipErrorInvalidConfiguration;
  const dim3 grid1(static_cast<uint32_t>(g1)), grid2(static_cast<uint32_t>(q.tiles * nob));
  if (a.t == DType::F32)
    hipLaunchKernelGGL((shrink_kernel<float>), grid1, dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((shrink_kernel<bf16_t>), grid1, dim3(kThreads), 0, s, p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.N <= kFewRows) {
    const int64_t blocks = (a.O + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff / a.N) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>(a.N * blocks));
    const size_t lds = static_cast<size_t>((a.R + 7) & ~7) * 4;
    if (a.t == DType::F32)
      hipLaunchKernelGGL((expand_rows_kernel<float>), grid, dim3(kThreads), lds, s, p, static_cast<uint32_t>(blocks));
    else
      hipLaunchKernelGGL((expand_rows_kernel<bf16_t>), grid, dim3(kThreads), lds, s, p, static_cast<uint32_t>(blocks));
    return hipGetLastError();
  }
  if (a.t == DType::F32)
    hipLaunchKernelGGL((expand_kernel<float>), grid2, dim3(kThreads), 0, s, p, static_cast<uint32_t>(nob));
  else
    hipLaunchKernelGGL((expand_kernel<bf16_t>), grid2, dim3(kThreads), 0, s, p, static_cast<uint32_t>(nob));
  return hipGetLastError();
}

}  // namespace cci
