// Low-rank adapters of many requests: for row n with adapter a = rows[n],
//   D[n][o] = P[n][o] + residual[n][o] + alpha[a] sum_r T[n][r] B[a][o][r],  T[n][r] = sum_c A[a][r][c] X[n][c],
// P the shared projection; a row whose adapter is outside [0, L) has no third
// term.  P comes in fp32 and the sum is rounded once, to D's type: the
// adapters' term and the residual are as large as the projection, and where
// they cancel a sum of rounded terms would be off by far more than a rounding
// of its own.  (The other order, the projection adding a term that this file
// had left in the output's type, moves 50 MB less over 3001 x 4096 outputs in
// bf16, 131 us for the call and 140 now, and doubled the outputs' rounding.)
//
// Both kernels work on tiles of 16 RT rows and walk over the distinct adapters
// among them: the matrix cores multiply all rows by one adapter, and the rows
// that have it keep the result.  A prompt's tile has one or two (RT = 4: the
// adapter's fragments serve 64 rows); a decoding batch up to 16 in 16 rows,
// whose weights have to be read in any case.
//   shrink  T: a workgroup of four waves sums one of S column ranges of one
//           tile, the waves taking turns at its 32-column steps, and adds the
//           four partial tiles in LDS.  With few tiles P workgroups share the
//           distinct adapters of one.  The S partial sums stay apart (fp32):
//           no atomics, equal calls give equal bits.
//   expand  the workgroup adds them up in order into LDS, and a wave multiplies
//           by 64 rows of B.  With bf16 operands T enters as the sum of two
//           bf16 values (16 bits of mantissa): it is not rounded to one.
// Fragments read from rows of memory cost the L1 one access per lane and 16
// bytes; that and the latency of a chain of loads bind.  3001 rows, C = O =
// 4096, R = 32, runs of 377 rows: shrink 13.9 us (18.8 with tiles of 16 rows),
// expand 28, which reads 49 MB of P and writes 24.6 of D; 32 rows of 16 adapters, R = 16: 4.2
// and 5.3, two launches' own time for the most part.
#include <algorithm>
#include <type_traits>

#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kOutBlocks = 4;   // blocks of 16 outputs of an expand wave
constexpr int kOutTile = kWaves * 16 * kOutBlocks;  // outputs of its workgroup's block

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
  const float* base;     // P
  const void* residual;  // of D's type
  void* D;
  float* part;  // [S][N][R]
  int64_t N, C, O, L, cols;
  int32_t R, S, P, d_f32, relu;
};

// The adapter of row n (-1: none).
__device__ __forceinline__ int32_t row_adapter(const AParams& p, int64_t n) {
  if (n >= p.N) return -1;
  const int32_t a = global_ptr<const int32_t>(p.rows)[n];
  return a >= 0 && a < p.L ? a : -1;
}

// The distinct adapters of a tile's rows in turn: lane l has row l of the tile
// (lanes past the rows have none), and `todo` its rows still to do.
struct Walk {
  int32_t mine;
  uint64_t todo;
};
template <int RT>
__device__ __forceinline__ Walk start_walk(const AParams& p, int64_t n0, int lane) {
  const int32_t a = lane < 16 * RT ? row_adapter(p, n0 + lane) : -1;
  return Walk{a, __ballot(a >= 0)};
}
__device__ __forceinline__ int32_t next_adapter(Walk& k) {
  const int32_t a = __builtin_amdgcn_readfirstlane(__shfl(k.mine, __builtin_ctzll(k.todo)));
  k.todo &= ~__ballot(k.mine == a);
  return a;
}

// KB: blocks of 16 ranks of a pass.
template <typename T, int RT, int KB>
__global__ __launch_bounds__(kThreads) void shrink_kernel(AParams p) {
  __shared__ f32x4_t red[kWaves][KB][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t li = lane & 15, lq = lane >> 4;
  const uint32_t per = static_cast<uint32_t>(p.S) * static_cast<uint32_t>(p.P);
  const uint32_t tile = blockIdx.x / per, rest = blockIdx.x - tile * per;
  const int32_t sl = static_cast<int32_t>(rest / p.P), turn = static_cast<int32_t>(rest % p.P);
  const int64_t n0 = static_cast<int64_t>(tile) * (16 * RT);
  const int64_t c_lo = sl * p.cols, c_hi = min(p.C, c_lo + p.cols);
  const T* X = global_ptr<const T>(p.X);
  const T* A = global_ptr<const T>(p.A);
  float* part = global_ptr<float>(p.part);
  const T* x[RT];  // (rows past the last have no adapter)
  int32_t mine[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t n = n0 + 16 * t + li;
    x[t] = X + min(n, p.N - 1) * p.C;
    mine[t] = row_adapter(p, n);
  }
  const int rank_blocks = (p.R + 15) / 16;
  Walk walk = start_walk<RT>(p, n0, lane);
  for (int32_t ord = 0; walk.todo; ++ord) {
    const int32_t a = next_adapter(walk);
    if (ord % p.P != turn) continue;
    for (int rb0 = 0; rb0 < rank_blocks; rb0 += KB) {
      f32x4_t acc[KB][RT];
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const int nb = min(KB, rank_blocks - rb0);
      const T* ar[KB];  // (ranks past the last read it again: their sums are not stored)
#pragma unroll
      for (int b = 0; b < KB; ++b)
        ar[b] = A + (static_cast<int64_t>(a) * p.R + min(16 * (rb0 + b) + static_cast<int>(li), p.R - 1)) * p.C;
      // Steps of 32 columns, two at a time; the loads of whole ones have no
      // branch, so that all of them are in flight.
      struct Step {
        Unit<T> x[RT], a[KB];
      };
      auto load = [&](Step& q, int64_t c, auto tail) __attribute__((always_inline)) {
        constexpr bool kWhole = !decltype(tail)::value;
#pragma unroll
        for (int t = 0; t < RT; ++t) load_part<8>(q.x[t], x[t] + c, p.C - c, kWhole);
#pragma unroll
        for (int b = 0; b < KB; ++b) load_part<8>(q.a[b], ar[b] + c, p.C - c, kWhole);
      };
      auto multiply = [&](const Step& q) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int t = 0; t < RT; ++t) mma(acc[b][t], q.a[b], q.x[t]);
      };
      const int64_t whole = min(c_hi, p.C / 32 * 32);
      int64_t c0 = c_lo + 32 * w;
      Step q0, q1;
      for (; c0 + 32 * kWaves < whole; c0 += 64 * kWaves) {
        load(q0, c0 + 8 * lq, std::false_type{});
        load(q1, c0 + 32 * kWaves + 8 * lq, std::false_type{});
        multiply(q0);
        multiply(q1);
      }
      if (c0 < whole) {
        load(q0, c0 + 8 * lq, std::false_type{});
        multiply(q0);
        c0 += 32 * kWaves;
      }
      if (c0 < c_hi) {
        load(q0, c0 + 8 * lq, std::true_type{});
        multiply(q0);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        __syncthreads();  // the previous sums are read
#pragma unroll
        for (int b = 0; b < KB; ++b) red[w][b][lane] = acc[b][t];
        __syncthreads();
        // wave w finishes block w: lane (li, lq) holds ranks 16 (rb0 + w) + 4 lq .. +3 of row li
        if (w < nb && mine[t] == a) {
          const f32x4_t s = red[0][w][lane] + red[1][w][lane] + red[2][w][lane] + red[3][w][lane];
          const int64_t n = n0 + 16 * t + li, r = 16 * (rb0 + w) + 4 * lq;
          const float v[4] = {s[0], s[1], s[2], s[3]};
          store4<float>(part + (static_cast<int64_t>(sl) * p.N + n) * p.R + r, v, p.R - r, p.R % 4 == 0);
        }
      }
    }
  }
}

// The workgroup's sum of the column ranges' parts of `rows` rows from n0, times
// alpha, into t[row][pitch] (padded: R rounded up to 8; rows without an
// adapter and ranks past the last are 0).  A thread takes 4 ranks; the loads of
// four ranges are in flight together and added in the ranges' order.
__device__ __forceinline__ void sum_parts(const AParams& p, int64_t n0, int rows, int32_t padded, int32_t pitch, float* t) {
  const float* part = global_ptr<const float>(p.part);
  const int64_t next = p.N * p.R;  // from a range's part to the next
  const int32_t quads = padded / 4;
  for (int32_t i = threadIdx.x; i < rows * quads; i += kThreads) {
    const int32_t row = i / quads, r = 4 * (i - row * quads);
    const int64_t n = min(n0 + row, p.N - 1);
    const int32_t a = row_adapter(p, n0 + row);
    const float* q = part + n * p.R + r;  // (a row without an adapter has no parts: what is read there is not used)
    f32x4_t sum{0.f, 0.f, 0.f, 0.f};
    int32_t k = 0;
    for (; k + 4 <= p.S; k += 4) {
      f32x4_t v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) load_elems<4>(v[j], q + (k + j) * next, p.R - r);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += v[j];
    }
    for (; k < p.S; ++k) {
      f32x4_t v;
      load_elems<4>(v, q + k * next, p.R - r);
      sum += v;
    }
    if (p.alpha) sum *= global_ptr<const float>(p.alpha)[a >= 0 ? a : 0];
    if (a < 0) sum = f32x4_t{0.f, 0.f, 0.f, 0.f};
    *reinterpret_cast<f32x4_t*>(t + row * pitch + r) = sum;
  }
  __syncthreads();
}

// T as MFMA operands: fp32 as it is, bf16 as high part + low part.
struct Split {
  Unit<bf16_t> hi, lo;
};
__device__ __forceinline__ Split split(const float (&t)[8]) {
  Split s;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const uint32_t hi = pack_bf16(t[e], t[e + 1]);
    const float d0 = t[e] - __uint_as_float(hi << 16), d1 = t[e + 1] - __uint_as_float(hi & 0xffff0000u);
    s.hi.d[0][e >> 1] = hi;
    // (an infinite T stays infinite)
    s.lo.d[0][e >> 1] = pack_bf16(__builtin_isfinite(d0) ? d0 : 0.0f, __builtin_isfinite(d1) ? d1 : 0.0f);
  }
  return s;
}

// An output from its terms: the projection, the residual at `at` (if it is there) and the adapter's.
__device__ __forceinline__ float total(const AParams& p, float base, int64_t at, bool there, float term) {
  float v = base;
  if (p.residual && there)
    v += p.d_f32 ? global_ptr<const float>(p.residual)[at] : bf16_to_f32(global_ptr<const uint16_t>(p.residual)[at]);
  v += term;
  return p.relu && v <= 0.0f ? 0.0f : v;  // (a NaN stays)
}

// A workgroup has 16 RT rows and every `groups`-th block of 256 outputs.
template <typename T, int RT>
__global__ __launch_bounds__(kThreads) void expand_kernel(AParams p, uint32_t nob, uint32_t groups) {
  extern __shared__ __attribute__((aligned(16))) float tsum[];  // [16 RT][pitch]
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t li = lane & 15, lq = lane >> 4;
  const uint32_t tile = blockIdx.x / groups;
  const int64_t n0 = static_cast<int64_t>(tile) * (16 * RT);
  const T* B = global_ptr<const T>(p.B);
  const int32_t padded = (p.R + 7) & ~7, pitch = padded + 4;  // (16 rows' units in different banks)
  const Walk all = start_walk<RT>(p, n0, lane);
  int32_t mine[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) mine[t] = row_adapter(p, n0 + 16 * t + li);
  const bool vec = p.O % 4 == 0;
  bool summed = false;
  for (uint32_t ob = blockIdx.x - tile * groups; ob < nob; ob += groups) {
    const int64_t o0 = (static_cast<int64_t>(ob) * kWaves + w) * (16 * kOutBlocks);
    const auto load_b = [&](Unit<T> (&bf)[kOutBlocks], int32_t a, int32_t r0) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < kOutBlocks; ++b) {
        const int64_t o = min(o0 + 16 * b + li, p.O - 1);  // (outputs past the last are not stored)
        load_elems<8>(bf[b], B + (static_cast<int64_t>(a) * p.O + o) * p.R + r0, p.R - r0);
      }
    };
    Walk walk = all;
    Unit<T> bf[kOutBlocks];
    int32_t a = -1;
    if (walk.todo) {  // B of the first adapter, before the wait for the sums
      a = next_adapter(walk);
      load_b(bf, a, 8 * static_cast<int32_t>(lq));
    }
    if (!summed) sum_parts(p, n0, 16 * RT, padded, pitch, tsum);
    summed = true;
    f32x4_t out[kOutBlocks][RT];
#pragma unroll
    for (int b = 0; b < kOutBlocks; ++b)
#pragma unroll
      for (int t = 0; t < RT; ++t) out[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    while (a >= 0) {
      f32x4_t acc[kOutBlocks][RT];
#pragma unroll
      for (int b = 0; b < kOutBlocks; ++b)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int32_t rs = 0; rs < p.R; rs += 32) {
        const int32_t r0 = rs + 8 * static_cast<int32_t>(lq);
        if (rs > 0) load_b(bf, a, r0);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          // ranks r0 .. r0 + 7 of row li; a row of another adapter enters as 0 and is not kept
          const f32x4_t* q = reinterpret_cast<const f32x4_t*>(tsum + (16 * t + li) * pitch + min(r0, padded - 8));
          const f32x4_t q0 = q[0], q1 = q[1];
          const bool keep = r0 < p.R && mine[t] == a;
          float v[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = keep ? q0[e] : 0.0f;
            v[4 + e] = keep ? q1[e] : 0.0f;
          }
          if constexpr (sizeof(T) == 2) {
            const Split q = split(v);
#pragma unroll
            for (int b = 0; b < kOutBlocks; ++b) {
              mma(acc[b][t], bf[b], q.lo);
              mma(acc[b][t], bf[b], q.hi);
            }
          } else {
            Unit<float> q;
#pragma unroll
            for (int e = 0; e < 8; ++e) q.d[e >> 2][e & 3] = __float_as_uint(v[e]);
#pragma unroll
            for (int b = 0; b < kOutBlocks; ++b) mma(acc[b][t], bf[b], q);
          }
        }
      }
#pragma unroll
      for (int b = 0; b < kOutBlocks; ++b)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) out[b][t][r] = mine[t] == a ? acc[b][t][r] : out[b][t][r];
      a = -1;
      if (walk.todo) {
        a = next_adapter(walk);
        load_b(bf, a, 8 * static_cast<int32_t>(lq));
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t n = n0 + 16 * t + li;
      if (n >= p.N) continue;
#pragma unroll
      for (int b = 0; b < kOutBlocks; ++b) {
        const int64_t o = o0 + 16 * b + 4 * lq, at = n * p.O + o;
        f32x4_t base;
        load_elems<4>(base, global_ptr<const float>(p.base) + at, p.O - o);
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = total(p, base[r], at + r, o + r < p.O, out[b][t][r]);
        if (p.d_f32)
          store4<float>(global_ptr<float>(p.D) + at, v, p.O - o, vec);
        else
          store4<bf16_t>(global_ptr<bf16_t>(p.D) + at, v, p.O - o, vec);
      }
    }
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
    const int32_t padded = (p.R + 7) & ~7;
    sum_parts(p, n, 1, padded, padded, t);
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
  v = total(p, global_ptr<const float>(p.base)[at], at, true, v);
  if (p.d_f32)
    global_ptr<float>(p.D)[at] = v;
  else
    global_ptr<uint16_t>(p.D)[at] = f32_to_bf16_rne(v);
}

// Up to so many rows: tiles of 16 rows, and expand on the vector ALUs.
constexpr int64_t kFewRows = 64;

// About 512 workgroups (64-row tiles: 256): column ranges of at least 256
// columns first, then, for a decoding batch's few tiles, workgroups that share
// the adapters.
APlan plan(int64_t N, int64_t C, int64_t L) {
  APlan q{};
  const int64_t rows = N <= kFewRows ? 16 : 64;
  q.tiles = (N + rows - 1) / rows;
  const int64_t want = std::max<int64_t>(1, (N <= kFewRows ? 512 : 256) / std::max<int64_t>(q.tiles, 1));
  const int64_t S = std::min<int64_t>(std::min<int64_t>(want, 16), (C + 255) / 256);
  q.cols = (C + S - 1) / S;
  q.cols = (q.cols + 127) / 128 * 128;
  q.S = static_cast<int32_t>((C + q.cols - 1) / q.cols);
  q.P = static_cast<int32_t>(
      std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rows, std::min(L, N)), want * 2 / q.S)));
  return q;
}

template <typename T>
hipError_t launch_typed(const AdapterArgs& a, const APlan& q, const AParams& p, hipStream_t s) {
  const int64_t shrink = q.tiles * q.S * q.P;
  if (shrink > 0x7fffffff) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(shrink)), block(kThreads);
  const size_t row_bytes = static_cast<size_t>((a.R + 7) & ~7) * 4;
  if (a.N <= kFewRows) {
    const int64_t nob = (a.O + kThreads - 1) / kThreads;
    if (nob > 0x7fffffff / a.N) return hipErrorInvalidConfiguration;
    const auto kernel = a.R <= 16 ? shrink_kernel<T, 1, 1> : a.R <= 32 ? shrink_kernel<T, 1, 2> : shrink_kernel<T, 1, 4>;
    hipLaunchKernelGGL(kernel, grid, block, 0, s, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((expand_rows_kernel<T>), dim3(static_cast<uint32_t>(a.N * nob)), block, row_bytes, s, p,
                       static_cast<uint32_t>(nob));
    return hipGetLastError();
  }
  const int64_t nob = (a.O + kOutTile - 1) / kOutTile;
  const int64_t tiles32 = (a.N + 31) / 32;
  if (nob > 0x7fffffff / tiles32) return hipErrorInvalidConfiguration;
  const auto kernel = a.R <= 16 ? shrink_kernel<T, 4, 1> : shrink_kernel<T, 4, 2>;
  hipLaunchKernelGGL(kernel, grid, block, 0, s, p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  // tiles of 32 rows: their sums of up to 1024 ranks fit the LDS
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t e = set_lds_limit_once(lds_set, reinterpret_cast<const void*>(&expand_kernel<T, 2>), 32 * (1024 + 4) * 4);
  if (e != hipSuccess) return e;
  // one round of workgroups: each sums its rows' parts once for all of its blocks
  const int64_t groups = std::max<int64_t>(1, std::min(nob, 512 / tiles32));
  hipLaunchKernelGGL((expand_kernel<T, 2>), dim3(static_cast<uint32_t>(tiles32 * groups)), block, 32 * (row_bytes + 16), s, p,
                     static_cast<uint32_t>(nob), static_cast<uint32_t>(groups));
  return hipGetLastError();
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
  p.base = a.base;
  p.residual = a.residual;
  p.relu = a.relu;
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
  return a.t == DType::F32 ? launch_typed<float>(a, q, p, s) : launch_typed<bf16_t>(a, q, p, s);
}

}  // namespace cci
