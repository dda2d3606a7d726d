// The products of a CCI-sparse feed-forward block on the matrix cores, for
// any sizes, groups and alignment of rows, in bf16 and fp32:
//   gated  H[n][f] = act(P[n][f]) P[n][F + f],  P = X . W_hat^T, the gate and
//          up weights one packing of the stacked [2F][C] matrix;
//   plain  Y = epilogue(X . W_hat^T);
//   back   dX[n][c] = sum_o dY[n][o] W_hat[o][c];
//   grad   dvals[g][k][c] = sum_n dY[n][gG + idx[g][k][c]] X[n][c].
// All but the last expand each chunk of packed groups to a dense tile in LDS
// (zero fill, then every kept weight to its place: Alg. 1's row gG + idx,
// Sec. 3.2), grad computes dense tiles of dY^T X and writes the kept entries; the matrix cores do G/K times the kept work at 32 times the vector
// ALUs' rate.
//
// A workgroup of four waves owns a TN x TW tile of outputs (TN rows of X, TW
// rows of the expanded weight tile: gated TW/2 outputs, whose gate and up
// rows alternate in runs of TW/4 so that both preactivations of an output
// end in one lane).  The reduction runs in chunks of 128 bytes a row (64
// bf16, 32 fp32) through two LDS buffers, the loads of the next chunk in
// registers: they need no alignment beyond their element's, and columns past
// the end become zeros.  Wave w expands tile rows [w TW/4, (w+1) TW/4) alone,
// so its zero fill and its writes are ordered by the LDS itself.
#include "cci_act.hpp"
#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kThreads = 256;   // of a team
constexpr int kRowBytes = 128;  // a tile row's chunk in LDS
constexpr int kGated = 0, kBack = 1, kGrad = 2, kPlain = 3;

template <typename T> constexpr int chunk_of = kRowBytes / static_cast<int>(sizeof(T));  // reduction elements of a chunk

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// LDS: element (row, k) of a tile sits in 16-byte slot k sizeof(T) / 16 of the
// row's 128 bytes, the slot XOR-ed with (row / 2) % 8, so that the 16 rows of
// a fragment read touch distinct bank slots.
__device__ __forceinline__ uint32_t slot_addr(uint32_t row, uint32_t slot) {
  return row * kRowBytes + ((slot ^ ((row >> 1) & 7u)) << 4);
}
template <typename T>
__device__ __forceinline__ uint32_t elem_addr(uint32_t row, uint32_t k) {
  const uint32_t b = k * static_cast<uint32_t>(sizeof(T));
  return slot_addr(row, b >> 4) + (b & 15u);
}
template <typename T>
__device__ __forceinline__ Unit<T> read_unit(const uint8_t* tile, uint32_t row, uint32_t u) {
  Unit<T> f;
#pragma unroll
  for (uint32_t h = 0; h < sizeof(T) / 2; ++h)
    f.d[h] = *reinterpret_cast<const u32x4_t*>(tile + slot_addr(row, u * (sizeof(T) / 2) + h));
  return f;
}
template <typename T>
__device__ __forceinline__ void write_unit(uint8_t* tile, uint32_t row, uint32_t u, const Unit<T>& f) {
#pragma unroll
  for (uint32_t h = 0; h < sizeof(T) / 2; ++h)
    *reinterpret_cast<u32x4_t*>(tile + slot_addr(row, u * (sizeof(T) / 2) + h)) = f.d[h];
}

struct TParams {
  const void* X;     // [N][ldx]: rows of the reduction operand (gated X, back dY, grad X)
  const void* dY;    // grad: [N][O]
  const void* vals;
  const uint8_t* idx;
  void* Y;
  void* pre;
  int64_t N, C, O;
  int32_t G, K;
  int32_t y_f32;     // plain, back, grad: Y (and residual) is fp32
  int32_t act, relu;
  const float* scale;
  const float* bias;
  const void* residual;
  uint32_t nnb, nwb;  // tile counts along TN and TW
  uint32_t grid8;     // grid / 8 when the grid is a multiple of 8, else 0
};

// PL: packed units per lane that are loaded a chunk ahead; 0: more, loaded
// where they are written.  TEAMS teams of four waves take turns at the chunks.
template <typename T, int MODE, int TN, int TW, int PL, int TEAMS>
__global__ __launch_bounds__(TEAMS * kThreads, TEAMS > 2 ? TEAMS : 2) void tile_kernel(TParams p) {
  constexpr int BK = chunk_of<T>, UPR = BK / 8;  // units of a row's chunk
  constexpr int kXTile = TN * kRowBytes, kWTile = TW * kRowBytes, kBuf = kXTile + kWTile;
  constexpr int TQ = TW / 4;                     // tile rows a wave expands
  constexpr int OT = TW / 32, NT = TN / 32;      // 16 x 16 blocks of a wave
  constexpr int XU = TN * UPR / kThreads;        // units of X a thread stages
  constexpr int UC = TQ / 8;                     // back: 8-column units of a packed row in a wave's columns
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int tid = threadIdx.x % kThreads, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  uint8_t* bufs = lds + team * (2 * kBuf);  // the team's two buffers
  const int wn = w & 1, wo = w >> 1;
  const T* X = global_ptr<const T>(p.X);
  const T* dY = global_ptr<const T>(p.dY);
  const T* vals = global_ptr<const T>(p.vals);
  const uint8_t* idx = global_ptr<const uint8_t>(p.idx);

  // ---- tile of this workgroup: dispatch places workgroup b on XCD b % 8; L
  // numbers the workgroups of one XCD consecutively, in bands of four row
  // blocks x every weight block, so that an XCD's L2 holds few of either.
  const uint32_t L = p.grid8 ? (blockIdx.x & 7u) * p.grid8 + (blockIdx.x >> 3) : blockIdx.x;
  const uint32_t per = 4u * p.nwb, band = L / per, within = L - band * per;
  const uint32_t rows = min(4u, p.nnb - 4u * band);
  const uint32_t wb = within / rows, nb = 4u * band + (within - wb * rows);
  const int64_t n0 = static_cast<int64_t>(nb) * TN;
  // first output of the tile along the weights: gated f, back c, plain and grad o
  const int64_t w0 = static_cast<int64_t>(wb) * (MODE == kGated ? TW / 2 : TW);
  const int64_t F = p.O / 2;
  constexpr bool kFwd = MODE == kGated || MODE == kPlain;
  const int64_t red = kFwd ? p.C : MODE == kBack ? p.O : p.N;  // reduction length
  const int64_t ldx = MODE == kBack ? p.O : p.C;
  const int nch = static_cast<int>((red + BK - 1) / BK);

  // ---- staging of X (gated, back: rows n0 .. of the reduction operand)
  Unit<T> xu[MODE == kGrad ? 1 : XU];
  auto load_x = [&](int ch) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad) {
#pragma unroll
      for (int i = 0; i < XU; ++i) {
        const int v = tid + kThreads * i, row = v / UPR, u = v % UPR;
        const int64_t k = static_cast<int64_t>(ch) * BK + 8 * u;
        load_elems<8>(xu[i], X + (n0 + row) * ldx + k, n0 + row < p.N ? red - k : 0);
      }
    }
  };
  auto store_x = [&](uint8_t* buf) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad) {
#pragma unroll
      for (int i = 0; i < XU; ++i) {
        const int v = tid + kThreads * i;
        write_unit<T>(buf, static_cast<uint32_t>(v / UPR), static_cast<uint32_t>(v % UPR), xu[i]);
      }
    }
  };

  // ---- grad: both operands are sample-major; a thread loads 4 columns of 8
  // samples and writes them transposed, 8 samples of a column to a unit.
  using Quad = std::conditional_t<sizeof(T) == 2, u32x2_t, u32x4_t>;
  Quad qx[MODE == kGrad ? 8 : 1], qy[MODE == kGrad ? 8 : 1];
  auto load_quads = [&](Quad (&q)[MODE == kGrad ? 8 : 1], const T* src, int64_t width, int64_t col0, int cols, int ch) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      const int cq = tid % (cols / 4), rg = tid / (cols / 4);
      const int64_t c = col0 + 4 * cq;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int64_t n = static_cast<int64_t>(ch) * BK + 8 * rg + r;
        load_elems<4>(q[r], src + n * width + c, n < p.N && rg < UPR ? width - c : 0);
      }
    }
  };
  auto store_quads = [&](uint8_t* tile, const Quad (&q)[MODE == kGrad ? 8 : 1], int cols) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      const int cq = tid % (cols / 4), rg = tid / (cols / 4);
      if (rg < UPR) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          Unit<T> f;
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              const uint32_t a = q[2 * m][j >> 1], b = q[2 * m + 1][j >> 1];
              f.d[0][m] = (j & 1) ? (a >> 16) | (b & 0xffff0000u) : (a & 0xffffu) | (b << 16);
            }
          } else {
#pragma unroll
            for (int m = 0; m < 8; ++m) f.d[m >> 2][m & 3] = q[m][j];
          }
          write_unit<T>(tile, static_cast<uint32_t>(4 * cq + j), static_cast<uint32_t>(rg), f);
        }
      }
    }
  };

  // ---- packed weights.  Unit v of a wave: 8 columns of packed row r, counted
  // from the first group that meets its rows (gated, plain) or the chunk (back).
  // Entry e of it goes to (tile row, reduction element)
  //   gated, plain (row0 + idx[e], 8 u + e) if row0 + idx[e] is among the wave's rows,
  //   back         (8 u + e, row0 + idx[e]) if row0 + idx[e] is in the chunk.
  const int64_t f0 = w0 + (MODE == kGated ? (w >> 1) * TQ : w * TQ);  // gated, plain: the wave's first output
  const int64_t wrow = f0 + (MODE == kGated && (w & 1) ? F : 0);      // and weight row
  const int64_t rest = max((MODE == kGated ? F : p.O) - f0, static_cast<int64_t>(0));
  const int lim = kFwd ? static_cast<int>(min(static_cast<int64_t>(TQ), rest)) : BK;
  constexpr int PU = PL > 0 ? PL : 1;
  Unit<T> pv[PU];
  u32x2_t pi[PU];
  int gl[PU];  // group of the unit's packed row, from the first
#pragma unroll
  for (int i = 0; i < PU; ++i) gl[i] = (lane + 64 * i) / (MODE == kBack ? UC : UPR) / p.K;
  struct Span {
    int64_t g_lo;  // first group
    int nrows;     // packed rows
    int first;     // g_lo G relative to the wave's rows / the chunk
  };
  auto span = [&](int ch) __attribute__((always_inline)) {
    const int64_t b = kFwd ? wrow : static_cast<int64_t>(ch) * BK;
    const int64_t last = kFwd ? b + lim - 1 : min(b + BK, p.O) - 1;
    Span s;
    s.g_lo = b / p.G;
    s.nrows = last >= b ? static_cast<int>(last / p.G - s.g_lo + 1) * p.K : 0;
    s.first = static_cast<int>(s.g_lo * p.G - b);
    return s;
  };
  const Span gspan = span(0);  // (gated, plain: the same in every chunk)
  auto load_unit = [&](const Span& s, int ch, int v, Unit<T>& val, u32x2_t& ix) __attribute__((always_inline)) {
    const int r = v / (MODE == kBack ? UC : UPR), u = v % (MODE == kBack ? UC : UPR);
    const int64_t c = kFwd ? static_cast<int64_t>(ch) * BK + 8 * u : w0 + w * TQ + 8 * u;
    const int64_t at = (s.g_lo * p.K + r) * p.C + c;
    const int64_t left = r < s.nrows ? p.C - c : 0;
    load_elems<8>(val, vals + at, left);
    load_elems<8>(ix, idx + at, left);
  };
  auto scatter = [&](uint8_t* wt, const Span& s, int v, int group, const Unit<T>& val, const u32x2_t& ix) __attribute__((always_inline)) {
    const int r = v / (MODE == kBack ? UC : UPR), u = v % (MODE == kBack ? UC : UPR);
    if (r >= s.nrows) return;
    const int row0 = s.first + group * p.G;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = row0 + static_cast<int>((ix[e >> 2] >> (8 * (e & 3))) & 0xffu);
      if (t >= 0 && t < lim) {
        const uint32_t at = kFwd ? elem_addr<T>(static_cast<uint32_t>(w * TQ + t), static_cast<uint32_t>(8 * u + e))
                                 : elem_addr<T>(static_cast<uint32_t>(w * TQ + 8 * u + e), static_cast<uint32_t>(t));
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<uint16_t*>(wt + at) = static_cast<uint16_t>(val.d[0][e >> 1] >> (16 * (e & 1)));
        else
          *reinterpret_cast<uint32_t*>(wt + at) = val.d[e >> 2][e & 3];
      }
    }
  };
  auto load_w = [&](int ch) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad && PL > 0) {
      const Span s = kFwd ? gspan : span(ch);
#pragma unroll
      for (int i = 0; i < PL; ++i) load_unit(s, ch, lane + 64 * i, pv[i], pi[i]);
    }
  };
  auto store_w = [&](uint8_t* wt, int ch) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad) {
#pragma unroll
      for (int i = 0; i < TQ / 8; ++i)
        *reinterpret_cast<u32x4_t*>(wt + w * TQ * kRowBytes + (i * 64 + lane) * 16) = u32x4_t{0u, 0u, 0u, 0u};
      asm volatile("" ::: "memory");  // the zeros come first; one wave's LDS writes stay in order
      const Span s = kFwd ? gspan : span(ch);
      if constexpr (PL > 0) {
#pragma unroll
        for (int i = 0; i < PL; ++i) scatter(wt, s, lane + 64 * i, gl[i], pv[i], pi[i]);
      } else {
        const int units = s.nrows * (MODE == kBack ? UC : UPR);
#pragma unroll 1
        for (int v = lane; v < units; v += 64) {
          load_unit(s, ch, v, pv[0], pi[0]);
          scatter(wt, s, v, v / (MODE == kBack ? UC : UPR) / p.K, pv[0], pi[0]);
        }
      }
    }
  };

  auto load_chunk = [&](int ch) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      load_quads(qy, dY, p.O, w0, TW, ch);
      load_quads(qx, X, p.C, n0, TN, ch);
    } else {
      load_x(ch);
      load_w(ch);
    }
  };
  auto store_chunk = [&](uint8_t* buf, int ch) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      store_quads(buf + kXTile, qy, TW);
      store_quads(buf, qx, TN);
    } else {
      store_x(buf);
      store_w(buf + kXTile, ch);
    }
  };

  f32x4_t acc[OT][NT];
#pragma unroll
  for (int o = 0; o < OT; ++o)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[o][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const uint32_t li = static_cast<uint32_t>(lane & 15), lq = static_cast<uint32_t>(lane >> 4);

  // the team's chunks are team, team + TEAMS, ...; every team makes the same number of rounds (barriers)
  const int rounds = (nch + TEAMS - 1) / TEAMS;
  const auto chunk = [&](int i) { return team + TEAMS * i; };
  if (chunk(0) < nch) {
    load_chunk(chunk(0));
    store_chunk(bufs, chunk(0));
    if (chunk(1) < nch) load_chunk(chunk(1));
  }
#pragma unroll 1
  for (int i = 0; i < rounds; ++i) {
    // round i's chunk is complete in its buffer, and nobody reads the one of round i - 1 any more
    lds_barrier();
    const uint8_t* cur = bufs + (i & 1) * kBuf;
    if (chunk(i + 1) < nch) {
      store_chunk(bufs + ((i + 1) & 1) * kBuf, chunk(i + 1));
      if (chunk(i + 2) < nch) load_chunk(chunk(i + 2));
    }
    if (chunk(i) >= nch) continue;
    const uint8_t* xt = cur;
    const uint8_t* wt = cur + kXTile;
#pragma unroll
    for (int ks = 0; ks < UPR / 4; ++ks) {
      Unit<T> a[OT], b[NT];
#pragma unroll
      for (int o = 0; o < OT; ++o) a[o] = read_unit<T>(wt, static_cast<uint32_t>(wo * (TW / 2) + 16 * o) + li, 4u * ks + lq);
#pragma unroll
      for (int n = 0; n < NT; ++n) b[n] = read_unit<T>(xt, static_cast<uint32_t>(wn * (TN / 2) + 16 * n) + li, 4u * ks + lq);
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int n = 0; n < NT; ++n) mma(acc[o][n], a[o], b[n]);
    }
  }

  // ---- the teams' sums, added in their order by the first
  if constexpr (TEAMS > 1) {
    lds_barrier();
    f32x4_t* park = reinterpret_cast<f32x4_t*>(bufs);
    if (team > 0) {
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int n = 0; n < NT; ++n) park[(o * NT + n) * kThreads + tid] = acc[o][n];
    }
    lds_barrier();
    if (team == 0) {
#pragma unroll
      for (int t = 1; t < TEAMS; ++t)
#pragma unroll
        for (int o = 0; o < OT; ++o)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            acc[o][n] += reinterpret_cast<const f32x4_t*>(lds + t * (2 * kBuf))[(o * NT + n) * kThreads + tid];
    } else if (MODE != kGrad) {
      return;
    }
  }

  // ---- a lane holds rows 4 lq .. +3 of each 16 x 16 block (weights) of column li (row of X)
  if constexpr (MODE == kGated) {
    const bool vec = F % 4 == 0;
    const Act act = static_cast<Act>(p.act);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t row = n0 + wn * (TN / 2) + 16 * n + li;
      if (row >= p.N) continue;
#pragma unroll
      for (int o = 0; o < OT / 2; ++o) {
        const int64_t f = w0 + wo * TQ + 16 * o + 4 * lq;
        float g[4], u[4], h[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          g[r] = acc[o][n][r];
          u[r] = acc[o + OT / 2][n][r];
          h[r] = act_value(act, g[r]) * u[r];
        }
        store4<T>(global_ptr<T>(p.Y) + row * F + f, h, F - f, vec);
        if (p.pre) {
          T* q = global_ptr<T>(p.pre) + row * p.O + f;
          store4<T>(q, g, F - f, vec);
          store4<T>(q + F, u, F - f, vec);
        }
      }
    }
  } else if constexpr (MODE == kPlain) {
    const bool vec = p.O % 4 == 0;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t row = n0 + wn * (TN / 2) + 16 * n + li;
      if (row >= p.N) continue;
#pragma unroll
      for (int o = 0; o < OT; ++o) {
        const int64_t c = w0 + wo * (TW / 2) + 16 * o + 4 * lq, at = row * p.O + c;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v[r] = acc[o][n][r];
          if (c + r >= p.O) continue;
          if (p.scale) v[r] *= global_ptr<const float>(p.scale)[c + r];
          if (p.bias) v[r] += global_ptr<const float>(p.bias)[c + r];
          if (p.residual)
            v[r] += p.y_f32 ? global_ptr<const float>(p.residual)[at + r]
                            : bf16_to_f32(global_ptr<const uint16_t>(p.residual)[at + r]);
          if (p.relu) v[r] = v[r] > 0.0f ? v[r] : (v[r] != v[r] ? v[r] : 0.0f);
        }
        if (p.y_f32)
          store4<float>(global_ptr<float>(p.Y) + at, v, p.O - c, vec);
        else
          store4<bf16_t>(global_ptr<bf16_t>(p.Y) + at, v, p.O - c, vec);
      }
    }
  } else if constexpr (MODE == kBack) {
    const bool vec = p.C % 4 == 0;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t row = n0 + wn * (TN / 2) + 16 * n + li;
      if (row >= p.N) continue;
#pragma unroll
      for (int o = 0; o < OT; ++o) {
        const int64_t c = w0 + wo * (TW / 2) + 16 * o + 4 * lq;
        const float v[4] = {acc[o][n][0], acc[o][n][1], acc[o][n][2], acc[o][n][3]};
        if (p.y_f32)
          store4<float>(global_ptr<float>(p.Y) + row * p.C + c, v, p.C - c, vec);
        else
          store4<bf16_t>(global_ptr<bf16_t>(p.Y) + row * p.C + c, v, p.C - c, vec);
      }
    }
  } else {
    // the dense tile goes to LDS column by column, and the kept entries of its rows from there to dvals
    constexpr int kPitch = TW + 4;
    float* park = reinterpret_cast<float*>(lds);
    lds_barrier();
    if (team == 0) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int o = 0; o < OT; ++o)
          *reinterpret_cast<f32x4_t*>(park + (wn * (TN / 2) + 16 * n + li) * kPitch + wo * (TW / 2) + 16 * o + 4 * lq) =
              acc[o][n];
    }
    lds_barrier();
    const int64_t o_end = min(w0 + TW, p.O);
    const int64_t g_lo = w0 / p.G;
    const int nrows = static_cast<int>((o_end - 1) / p.G - g_lo + 1) * p.K;
    const int first = static_cast<int>(g_lo * p.G - w0), lim_o = static_cast<int>(o_end - w0);
    const int c = tid % TN;
    if (n0 + c < p.C) {
#pragma unroll 1
      for (int r = threadIdx.x / TN; r < nrows; r += TEAMS * kThreads / TN) {
        const int64_t at = (g_lo * p.K + r) * p.C + n0 + c;
        const int o = first + (r / p.K) * p.G + static_cast<int>(idx[at]);
        if (o < 0 || o >= lim_o) continue;  // another tile's row
        const float v = park[c * kPitch + o];
        if (p.y_f32)
          global_ptr<float>(p.Y)[at] = v;
        else
          global_ptr<uint16_t>(p.Y)[at] = f32_to_bf16_rne(v);
      }
    }
  }
}

template <typename T, int MODE, int TN, int TW, int PL, int TEAMS>
hipError_t launch(const TParams& q, hipStream_t s) {
  TParams p = q;
  constexpr int kOperands = TEAMS * 2 * (TN + TW) * kRowBytes;
  constexpr int kPark = MODE == kGrad ? TN * (TW + 4) * 4 : 0;
  constexpr int kLds = kOperands > kPark ? kOperands : kPark;
  const int64_t along_n = MODE == kGrad ? p.C : p.N;
  const int64_t along_w = MODE == kBack ? p.C : p.O;
  const int64_t nnb = (along_n + TN - 1) / TN, nwb = (along_w + TW - 1) / TW;
  if (nnb > 0x7fffffff / 8 || nwb > 0x7fffffff / 8 || nnb * nwb > 0x7fffffff) return hipErrorInvalidConfiguration;
  const uint32_t grid = static_cast<uint32_t>(nnb * nwb);
  p.nnb = static_cast<uint32_t>(nnb);
  p.nwb = static_cast<uint32_t>(nwb);
  p.grid8 = grid % 8 == 0 ? grid / 8 : 0;
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t e = set_lds_limit_once(lds_set, reinterpret_cast<const void*>(&tile_kernel<T, MODE, TN, TW, PL, TEAMS>), kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tile_kernel<T, MODE, TN, TW, PL, TEAMS>), dim3(grid), dim3(TEAMS * kThreads), kLds, s, p);
  return hipGetLastError();
}

template <typename T, int MODE, int TN, int TW, int TEAMS>
hipError_t launch_pl(const TParams& p, hipStream_t s) {
  if constexpr (MODE == kGrad) {
    return launch<T, MODE, TN, TW, 0, TEAMS>(p, s);
  } else {
    // packed units of a wave and chunk, per lane
    const int64_t rows = groups_in(MODE == kBack ? chunk_of<T> : TW / 4, p.G) * p.K;
    const int64_t pl = (rows * (MODE == kBack ? TW / 32 : chunk_of<T> / 8) + 63) / 64;
    if (pl <= 1) return launch<T, MODE, TN, TW, 1, TEAMS>(p, s);
    if (pl <= 2) return launch<T, MODE, TN, TW, 2, TEAMS>(p, s);
    if (pl <= 4) return launch<T, MODE, TN, TW, 4, TEAMS>(p, s);
    return launch<T, MODE, TN, TW, 0, TEAMS>(p, s);
  }
}

template <typename T, int MODE>
hipError_t launch_tiles(const TParams& p, hipStream_t s) {
  const int64_t an = MODE == kGrad ? p.C : p.N, aw = MODE == kBack ? p.C : p.O;
  // 128 x 128 tiles unless they leave half of the CUs without one
  const int64_t big = (an + 127) / 128 * ((aw + 127) / 128);
  if (big >= 256) return launch_pl<T, MODE, 128, 128, 1>(p, s);
  // 64 x 64 tiles; up to two a CU, a memory latency per chunk binds, and teams share the chunks (as many as their
  // registers allow)
  const int64_t small = (an + 63) / 64 * ((aw + 63) / 64);
  const int64_t red = MODE == kBack ? p.O : MODE == kGrad ? p.N : p.C;
  if (small <= 512 && red >= 4 * chunk_of<T>) return launch_pl<T, MODE, 64, 64, sizeof(T) == 2 ? 4 : 2>(p, s);
  return launch_pl<T, MODE, 64, 64, 1>(p, s);
}

TParams params(const BlockProduct& a) {
  TParams p{};
  p.X = a.X;
  p.dY = a.dY;
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
  p.scale = a.scale;
  p.bias = a.bias;
  p.residual = a.residual;
  p.relu = a.relu;
  return p;
}

}  // namespace

hipError_t launch_tile_gated(const BlockProduct& a, hipStream_t s) {
  const TParams p = params(a);
  return a.t == DType::F32 ? launch_tiles<float, kGated>(p, s) : launch_tiles<bf16_t, kGated>(p, s);
}

hipError_t launch_tile_plain(const BlockProduct& a, hipStream_t s) {
  const TParams p = params(a);
  return a.t == DType::F32 ? launch_tiles<float, kPlain>(p, s) : launch_tiles<bf16_t, kPlain>(p, s);
}

hipError_t launch_tile_back(const BlockProduct& a, hipStream_t s) {
  BlockProduct b = a;
  b.X = a.dY;
  const TParams p = params(b);
  return a.t == DType::F32 ? launch_tiles<float, kBack>(p, s) : launch_tiles<bf16_t, kBack>(p, s);
}

hipError_t launch_tile_grad(const BlockProduct& a, hipStream_t s) {
  const TParams p = params(a);
  return a.t == DType::F32 ? launch_tiles<float, kGrad>(p, s) : launch_tiles<bf16_t, kGrad>(p, s);
}

}  // namespace cci
