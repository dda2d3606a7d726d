// Layer norm over rows of C elements, forward and backward.
//   forward   m = mean(x), s = 1 / sqrt(mean((x - m)^2) + eps), y = (x - m) s gamma + beta
//   backward  xh = (x - m) s, q = dy gamma,
//             dx = s (q - mean(q) - xh mean(q xh)), dgamma = sum_n dy xh, dbeta = sum_n dy
// HBM binds: forward reads and writes a row once, backward reads two and
// writes one.  A team of threads keeps its row in registers between the sums
// and the write; teams walk over rows and hold gamma and beta (forward), or
// gamma and the sums of the weight gradients (backward), in registers too.
// The mean m is taken first, and then the sums of d = x - m and d^2: rows far
// from zero do not cancel, and mean(d) is what the rounding of m left out
// (half a step of m, which may be as much as the row's deviation): the
// variance is mean(d^2) - mean(d)^2, the centred value d - mean(d).  Weight gradients are summed per team,
// over a workgroup's teams in LDS, and over the workgroups by a second kernel
// in a fixed order (no atomics: equal calls give equal bits).
// Rows too long for the registers are read again for every pass.
#include <algorithm>

#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kCUs = 256;
constexpr int kFwdThreads = 256;
// Threads of a backward workgroup: four teams, 1024 at most (more teams of short
// rows would add up longer in LDS than they save in partial sums: 1537 x 1001
// fp32 with sixteen 17 us).
constexpr int bwd_threads(int tpr) { return tpr <= 256 ? 4 * tpr : 1024; }
constexpr int kSumCols = 64, kSumGroups = 16;  // reduction of the partial weight gradients

// 8 fp32 values of an optional vector (null: `otherwise`).
__device__ __forceinline__ void load_vec(float (&v)[8], const float* p, int64_t c, int64_t left, float otherwise) {
  if (p) {
    Unit<float> u;
    load_elems<8>(u, p + c, left);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = elem(u, e);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = otherwise;
  }
}

// Sums over the TPR threads of a team, for every one of them.  `red` holds the
// workgroup's wave sums of one call; calls in turn use different ones, so that
// one barrier a call is enough.
template <int TPR, int THREADS, int NV>
__device__ __forceinline__ void team_sum(float (&v)[NV], float* red) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1)
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] += __shfl_xor(v[j], m);
  if constexpr (TPR > 64) {
    constexpr int kW = THREADS / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) red[j * kW + (threadIdx.x >> 6)] = v[j];
    }
    __syncthreads();
    const int first = threadIdx.x / TPR * (TPR / 64);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      v[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < TPR / 64; ++i) v[j] += red[j * kW + first + i];
    }
  }
}

// The value that deviations are taken from: near the mean, and for bf16 rows of
// 12 bits, so that x - m is exact (8 bits of x, fp32 holds 24) unless the mean
// is below 2^-12 of x.  From a mean of 24 bits every x of one binade would lose
// the same part of it: the mean of 4096 values of deviation 1 was off by 0.4
// u (u = 2^-24), 3 times an fp32 sum's error.  (An infinity, and a NaN that came
// from bf16, stay: their low bits are 0.)
template <typename T>
__device__ __forceinline__ float near_mean(float m) {
  if constexpr (sizeof(T) == 4) return m;
  return __uint_as_float((__float_as_uint(m) + 0x800u) & 0xfffff000u);
}

// 1 / sqrt(var + eps); a variance below 0 is rounding, and a NaN stays one.
__device__ __forceinline__ float deviation(float var, float eps) { return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps); }

// The mean from its first value and what that left out (of an infinite one: a NaN).
__device__ __forceinline__ float whole_mean(float m, float lost) { return __builtin_isfinite(m) ? m + lost : m; }

template <typename T, int TPR, int VPT>
__global__ __launch_bounds__(kFwdThreads > TPR ? kFwdThreads : TPR) void norm_kernel(
    const T* __restrict__ X, int64_t N, int64_t C, const float* __restrict__ gamma, const float* __restrict__ beta,
    float eps, T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int kThreads = kFwdThreads > TPR ? kFwdThreads : TPR, kTeams = kThreads / TPR;
  __shared__ float red1[kThreads / 64], red2[2 * (kThreads / 64)];
  const int t = threadIdx.x % TPR;
  const float len = static_cast<float>(C);
  const bool vec = C % 4 == 0;
  float ga[VPT][8], be[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i);
    load_vec(ga[i], gamma, c, C - c, 1.0f);
    load_vec(be[i], beta, c, C - c, 0.0f);
  }
  // every thread of a workgroup makes the same number of rounds (barriers)
  const int64_t rounds = (N + static_cast<int64_t>(gridDim.x) * kTeams - 1) / (static_cast<int64_t>(gridDim.x) * kTeams);
  for (int64_t k = 0; k < rounds; ++k) {
    const int64_t n = (k * gridDim.x + blockIdx.x) * kTeams + threadIdx.x / TPR;
    const bool on = n < N;
    Unit<T> x[VPT];
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i);
      load_elems<8>(x[i], X + n * C + c, on ? C - c : 0);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[0] += elem(x[i], e);
    team_sum<TPR, kThreads>(sum, red1);
    const float m = near_mean<T>(sum[0] / len);
    float sq[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t left = C - 8 * (t + static_cast<int64_t>(TPR) * i);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = e < left ? elem(x[i], e) - m : 0.0f;
        sq[0] += d;
        sq[1] += d * d;
      }
    }
    team_sum<TPR, kThreads>(sq, red2);
    const float lost = sq[0] / len;
    const float r = deviation(sq[1] / len - lost * lost, eps);
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          y[e] = (elem(x[i], 4 * h + e) - m - lost) * r * ga[i][4 * h + e] + be[i][4 * h + e];
        store4<T>(Y + n * C + c + 4 * h, y, C - c - 4 * h, vec);
      }
    }
    if (t == 0) {
      if (mean) mean[n] = whole_mean(m, lost);
      if (rstd) rstd[n] = r;
    }
  }
}

// Any C: a workgroup per row, which is read once per pass.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const T* __restrict__ X, int64_t N, int64_t C,
                                                         const float* __restrict__ gamma,
                                                         const float* __restrict__ beta, float eps, T* __restrict__ Y,
                                                         float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float red1[16], red2[2 * 16];
  const float len = static_cast<float>(C);
  const bool vec = C % 4 == 0;
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const T* x = X + n * C;
    float sum[1] = {0.0f}, sq[2] = {0.0f, 0.0f};
    for (int64_t c = 8 * threadIdx.x; c < C; c += 8 * 1024) {
      Unit<T> u;
      load_elems<8>(u, x + c, C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[0] += elem(u, e);
    }
    team_sum<1024, 1024>(sum, red1);
    const float m = near_mean<T>(sum[0] / len);
    for (int64_t c = 8 * threadIdx.x; c < C; c += 8 * 1024) {
      Unit<T> u;
      load_elems<8>(u, x + c, C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = e < C - c ? elem(u, e) - m : 0.0f;
        sq[0] += d;
        sq[1] += d * d;
      }
    }
    team_sum<1024, 1024>(sq, red2);
    const float lost = sq[0] / len;
    const float r = deviation(sq[1] / len - lost * lost, eps);
    for (int64_t c = 8 * threadIdx.x; c < C; c += 8 * 1024) {
      Unit<T> u;
      float ga[8], be[8];
      load_elems<8>(u, x + c, C - c);
      load_vec(ga, gamma, c, C - c, 1.0f);
      load_vec(be, beta, c, C - c, 0.0f);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (elem(u, 4 * h + e) - m - lost) * r * ga[4 * h + e] + be[4 * h + e];
        store4<T>(Y + n * C + c + 4 * h, y, C - c - 4 * h, vec);
      }
    }
    if (threadIdx.x == 0) {
      if (mean) mean[n] = whole_mean(m, lost);
      if (rstd) rstd[n] = r;
    }
  }
}

// part: [gridDim.x][2][C], the workgroup's sums of dgamma and dbeta (null: not wanted).
template <typename T, int TPR, int VPT>
__global__ __launch_bounds__(bwd_threads(TPR)) void norm_bwd_kernel(
    const T* __restrict__ dY, const T* __restrict__ X, int64_t N, int64_t C, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, T* __restrict__ dX, float* __restrict__ part) {
  constexpr int kBwdThreads = bwd_threads(TPR), kTeams = kBwdThreads / TPR;
  __shared__ float red[2][2 * (kBwdThreads / 64)];
  extern __shared__ __attribute__((aligned(16))) float sums[];  // [kTeams / 2][2][TPR * VPT * 8]
  const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
  const float len = static_cast<float>(C);
  const bool vec = C % 4 == 0;
  float ga[VPT][8], dg[VPT][8], db[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i);
    load_vec(ga[i], gamma, c, C - c, 1.0f);
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = db[i][e] = 0.0f;
  }
  const int64_t rounds = (N + static_cast<int64_t>(gridDim.x) * kTeams - 1) / (static_cast<int64_t>(gridDim.x) * kTeams);
  for (int64_t k = 0; k < rounds; ++k) {
    const int64_t n = (k * gridDim.x + blockIdx.x) * kTeams + team;
    const bool on = n < N;
    const float m = on ? mean[n] : 0.0f, r = on ? rstd[n] : 0.0f;
    Unit<T> x[VPT], y[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i), left = on ? C - c : 0;
      load_elems<8>(x[i], X + n * C + c, left);
      load_elems<8>(y[i], dY + n * C + c, left);
    }
    float s12[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // (dY reads as 0 past the row's end)
        const float dy = elem(y[i], e), xh = (elem(x[i], e) - m) * r, q = dy * ga[i][e];
        s12[0] += q;
        s12[1] += q * xh;
        dg[i][e] += dy * xh;
        db[i][e] += dy;
      }
    if (!dX) continue;
    team_sum<TPR, kBwdThreads>(s12, red[k & 1]);
    const float c1 = s12[0] / len, c2 = s12[1] / len;
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float xh = (elem(x[i], 4 * h + e) - m) * r, q = elem(y[i], 4 * h + e) * ga[i][4 * h + e];
          v[e] = r * (q - c1 - xh * c2);
        }
        store4<T>(dX + n * C + c + 4 * h, v, C - c - 4 * h, vec);
      }
    }
  }
  if (!part) return;
  // the teams' sums, halved until one team holds them
  constexpr int kRow = TPR * VPT * 8;
#pragma unroll
  for (int half = kTeams / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (team >= half && team < 2 * half) {
      float* p = sums + (team - half) * 2 * kRow;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {  // (element-major: consecutive threads on consecutive words)
          p[(i * 8 + e) * TPR + t] = dg[i][e];
          p[kRow + (i * 8 + e) * TPR + t] = db[i][e];
        }
    }
    __syncthreads();
    if (team < half) {
      const float* p = sums + team * 2 * kRow;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dg[i][e] += p[(i * 8 + e) * TPR + t];
          db[i][e] += p[kRow + (i * 8 + e) * TPR + t];
        }
    }
  }
  if (team == 0) {
    float* pg = part + static_cast<int64_t>(blockIdx.x) * 2 * C;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = 8 * (t + static_cast<int64_t>(TPR) * i);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float a[4] = {dg[i][4 * h], dg[i][4 * h + 1], dg[i][4 * h + 2], dg[i][4 * h + 3]};
        const float b[4] = {db[i][4 * h], db[i][4 * h + 1], db[i][4 * h + 2], db[i][4 * h + 3]};
        store4<float>(pg + c + 4 * h, a, C - c - 4 * h, vec);
        store4<float>(pg + C + c + 4 * h, b, C - c - 4 * h, vec);
      }
    }
  }
}

// Rows too long for that: mean(q) and mean(q xh) of every row first ...
template <typename T>
__global__ __launch_bounds__(1024) void norm_bwd_rows_kernel(const T* __restrict__ dY, const T* __restrict__ X,
                                                             int64_t N, int64_t C, const float* __restrict__ gamma,
                                                             const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, float* __restrict__ stats) {
  __shared__ float red[2][2 * 16];
  int64_t k = 0;
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const float m = mean[n], r = rstd[n];
    float s12[2] = {0.0f, 0.0f};
    for (int64_t c = 8 * threadIdx.x; c < C; c += 8 * 1024) {
      Unit<T> x, y;
      float ga[8];
      load_elems<8>(x, X + n * C + c, C - c);
      load_elems<8>(y, dY + n * C + c, C - c);
      load_vec(ga, gamma, c, C - c, 1.0f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = elem(y, e) * ga[e];
        s12[0] += q;
        s12[1] += q * ((elem(x, e) - m) * r);
      }
    }
    team_sum<1024, 1024>(s12, red[k++ & 1]);
    if (threadIdx.x == 0) {
      stats[2 * n] = s12[0] / static_cast<float>(C);
      stats[2 * n + 1] = s12[1] / static_cast<float>(C);
    }
  }
}

// ... then dX and the sums of a run of rows, 2048 columns a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void norm_bwd_cols_kernel(
    const T* __restrict__ dY, const T* __restrict__ X, int64_t N, int64_t C, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, const float* __restrict__ stats, T* __restrict__ dX,
    float* __restrict__ part, int64_t rows, uint32_t nrb) {
  const bool vec = C % 4 == 0;
  const uint32_t cb = blockIdx.x / nrb, rb = blockIdx.x - cb * nrb;
  const int64_t c = (static_cast<int64_t>(cb) * 256 + threadIdx.x) * 8;
  if (c >= C) return;
  float ga[8], dg[8] = {}, db[8] = {};
  load_vec(ga, gamma, c, C - c, 1.0f);
  const int64_t end = min(N, (rb + 1) * rows);
  for (int64_t n = rb * rows; n < end; ++n) {
    const float m = mean[n], r = rstd[n], c1 = dX ? stats[2 * n] : 0.0f, c2 = dX ? stats[2 * n + 1] : 0.0f;
    Unit<T> x, y;
    load_elems<8>(x, X + n * C + c, C - c);
    load_elems<8>(y, dY + n * C + c, C - c);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float dy = elem(y, 4 * h + e), xh = (elem(x, 4 * h + e) - m) * r;
        dg[4 * h + e] += dy * xh;
        db[4 * h + e] += dy;
        v[e] = r * (dy * ga[4 * h + e] - c1 - xh * c2);
      }
      if (dX) store4<T>(dX + n * C + c + 4 * h, v, C - c - 4 * h, vec);
    }
  }
  if (!part) return;
  float* pg = part + static_cast<int64_t>(rb) * 2 * C;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float a[4] = {dg[4 * h], dg[4 * h + 1], dg[4 * h + 2], dg[4 * h + 3]};
    const float b[4] = {db[4 * h], db[4 * h + 1], db[4 * h + 2], db[4 * h + 3]};
    store4<float>(pg + c + 4 * h, a, C - c - 4 * h, vec);
    store4<float>(pg + C + c + 4 * h, b, C - c - 4 * h, vec);
  }
}

// dgamma[c] = sum_p part[p][0][c], dbeta[c] = sum_p part[p][1][c], in a fixed order.
__global__ __launch_bounds__(kSumCols * kSumGroups) void norm_sums_kernel(const float* __restrict__ part, int32_t P,
                                                                         int64_t C, float* __restrict__ dgamma,
                                                                         float* __restrict__ dbeta) {
  __shared__ float red[kSumGroups][kSumCols];
  const int col = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols;
  // (in a loop: a launch has fewer than 2^32 threads)
  for (int64_t c0 = static_cast<int64_t>(blockIdx.x) * kSumCols; c0 < 2 * C; c0 += static_cast<int64_t>(gridDim.x) * kSumCols) {
    const int64_t c = c0 + col;  // of the 2 C sums
    float v = 0.0f;
    if (c < 2 * C) {
      constexpr int kAhead = 8;  // loads in flight
      int32_t p = grp;
      for (; p + (kAhead - 1) * kSumGroups < P; p += kAhead * kSumGroups) {
        float q[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) q[i] = part[static_cast<int64_t>(p + i * kSumGroups) * 2 * C + c];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v += q[i];
      }
      for (; p < P; p += kSumGroups) v += part[static_cast<int64_t>(p) * 2 * C + c];
    }
    __syncthreads();  // the previous columns' sums are read
    red[grp][col] = v;
    __syncthreads();
    if (grp != 0 || c >= 2 * C) continue;
#pragma unroll
    for (int i = 1; i < kSumGroups; ++i) v += red[i][col];
    if (c < C) {
      if (dgamma) dgamma[c] = v;
    } else if (dbeta) {
      dbeta[c - C] = v;
    }
  }
}

constexpr int64_t kFwdMost = 16384;  // longest rows kept in registers (backward: kNormBwdMost)

// Partial weight gradients at most: a workgroup of 16 waves a CU, two of 4 waves (short rows).
int64_t most_parts(int64_t C) { return C <= 1024 ? 2 * kCUs : kCUs; }

template <typename T, int TPR, int VPT>
hipError_t fwd(const void* X, int64_t N, int64_t C, const float* gamma, const float* beta, float eps, void* Y,
               float* mean, float* rstd, hipStream_t s) {
  constexpr int kThreads = kFwdThreads > TPR ? kFwdThreads : TPR;
  const int64_t wgs = (N + kThreads / TPR - 1) / (kThreads / TPR);
  const int64_t most = kCUs * (2048 / kThreads);  // resident at once
  hipLaunchKernelGGL((norm_kernel<T, TPR, VPT>), dim3(static_cast<uint32_t>(wgs < most ? wgs : most)), dim3(kThreads), 0, s,
                     static_cast<const T*>(X), N, C, gamma, beta, eps, static_cast<T*>(Y), mean, rstd);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd_typed(const void* X, int64_t N, int64_t C, const float* gamma, const float* beta, float eps, void* Y,
                     float* mean, float* rstd, hipStream_t s) {
  if (C > kFwdMost) {
    hipLaunchKernelGGL((norm_long_kernel<T>), dim3(static_cast<uint32_t>(N < 65536 ? N : 65536)), dim3(1024), 0, s,
                       static_cast<const T*>(X), N, C, gamma, beta, eps, static_cast<T*>(Y), mean, rstd);
    return hipGetLastError();
  }
  if (C <= 512) return fwd<T, 64, 1>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
  if (C <= 1024) return fwd<T, 64, 2>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
  if (C <= 2048) return fwd<T, 256, 1>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
  if (C <= 4096) return fwd<T, 256, 2>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
  if (C <= 8192) return fwd<T, 512, 2>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
  return fwd<T, 1024, 2>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
}

// Workgroups of the backward kernel: the partial sums it leaves.
int64_t bwd_parts(int64_t N, int64_t C) {
  const int64_t teams = C <= 4096 ? 4 : C <= 8192 ? 2 : 1;
  return std::min((N + teams - 1) / teams, most_parts(C));
}

template <typename T, int TPR, int VPT>
hipError_t bwd(const void* dY, const void* X, int64_t N, int64_t C, const float* gamma, const float* mean,
               const float* rstd, void* dX, float* part, int64_t parts, hipStream_t s) {
  constexpr int kBwdThreads = bwd_threads(TPR), kTeams = kBwdThreads / TPR;
  constexpr int kLds = kTeams / 2 * 2 * TPR * VPT * 8 * 4;
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t e = set_lds_limit_once(lds_set, reinterpret_cast<const void*>(&norm_bwd_kernel<T, TPR, VPT>), kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((norm_bwd_kernel<T, TPR, VPT>), dim3(static_cast<uint32_t>(parts)), dim3(kBwdThreads), kLds, s,
                     static_cast<const T*>(dY), static_cast<const T*>(X), N, C, gamma, mean, rstd, static_cast<T*>(dX),
                     part);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd_typed(const void* dY, const void* X, int64_t N, int64_t C, const float* gamma, const float* mean,
                     const float* rstd, void* dX, float* part, float* stats, int64_t parts, hipStream_t s) {
  if (C <= kNormBwdMost) {
    if (C <= 512) return bwd<T, 64, 1>(dY, X, N, C, gamma, mean, rstd, dX, part, parts, s);
    if (C <= 1024) return bwd<T, 64, 2>(dY, X, N, C, gamma, mean, rstd, dX, part, parts, s);
    if (C <= 2048) return bwd<T, 256, 1>(dY, X, N, C, gamma, mean, rstd, dX, part, parts, s);
    if (C <= 4096) return bwd<T, 256, 2>(dY, X, N, C, gamma, mean, rstd, dX, part, parts, s);
    if (C <= 8192) return bwd<T, 512, 2>(dY, X, N, C, gamma, mean, rstd, dX, part, parts, s);
    return bwd<T, 1024, 2>(dY, X, N, C, gamma, mean, rstd, dX, part, parts, s);
  }
  if (dX) {  // the weight gradients do not need the rows' means
    hipLaunchKernelGGL((norm_bwd_rows_kernel<T>), dim3(static_cast<uint32_t>(N < 65536 ? N : 65536)), dim3(1024), 0, s,
                       static_cast<const T*>(dY), static_cast<const T*>(X), N, C, gamma, mean, rstd, stats);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const int64_t rows = (N + parts - 1) / parts, cb = (C + 2047) / 2048;
  hipLaunchKernelGGL((norm_bwd_cols_kernel<T>), dim3(static_cast<uint32_t>(parts * cb)), dim3(256), 0, s,
                     static_cast<const T*>(dY), static_cast<const T*>(X), N, C, gamma, mean, rstd, stats,
                     static_cast<T*>(dX), part, rows, static_cast<uint32_t>(parts));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm(const void* X, DType t, int64_t N, int64_t C, const float* gamma, const float* beta,
                            float eps, void* Y, float* mean, float* rstd, hipStream_t s) {
  return t == DType::F32 ? fwd_typed<float>(X, N, C, gamma, beta, eps, Y, mean, rstd, s)
                         : fwd_typed<bf16_t>(X, N, C, gamma, beta, eps, Y, mean, rstd, s);
}

int64_t layernorm_bwd_workspace(int64_t N, int64_t C) {
  return (bwd_parts(N, C) * 2 * C + (C > kNormBwdMost ? 2 * N : 0)) * 4;
}

hipError_t launch_layernorm_bwd(const void* dY, const void* X, DType t, int64_t N, int64_t C, const float* gamma,
                                const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta,
                                void* workspace, hipStream_t s) {
  const bool weights = dgamma || dbeta;
  if (!dX && !weights) return hipSuccess;
  const int64_t parts = bwd_parts(N, C);
  float* part = weights ? static_cast<float*>(workspace) : nullptr;
  float* stats = C > kNormBwdMost ? static_cast<float*>(workspace) + parts * 2 * C : nullptr;
  if (N > 0) {
    const hipError_t e = t == DType::F32 ? bwd_typed<float>(dY, X, N, C, gamma, mean, rstd, dX, part, stats, parts, s)
                                         : bwd_typed<bf16_t>(dY, X, N, C, gamma, mean, rstd, dX, part, stats, parts, s);
    if (e != hipSuccess) return e;
  }
  if (!weights) return hipSuccess;
  const int64_t blocks = std::min<int64_t>((2 * C + kSumCols - 1) / kSumCols, int64_t(1) << 20);
  hipLaunchKernelGGL(norm_sums_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kSumCols * kSumGroups), 0, s, part, static_cast<int32_t>(parts), C, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace cci
