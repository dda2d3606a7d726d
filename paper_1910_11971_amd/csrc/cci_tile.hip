// The products of a CCI-sparse feed-forward block on the matrix cores, for
// any sizes, groups and alignment of rows, in bf16 and fp32:
//   gated  H[n][f] = act(P[n][f]) P[n][F + f],  P = X . W_hat^T, the gate and
//          up weights one packing of the stacked [2F][C] matrix;
//   plain  Y = X . W_hat^T * scale + bias, in fp32;
//   back   dX[n][c] = sum_o dY[n][o] W_hat[o][c];
//   grad   dvals[g][k][c] = sum_n dY[n][gG + idx[g][k][c]] X[n][c].
// All but the last expand each chunk of packed groups to a dense tile in LDS
// (zero fill, then every kept weight to its place: Alg. 1's row gG + idx,
// Sec. 3.2), grad computes dense tiles of dY^T X and writes the kept entries.
// The matrix cores do G/K times the kept work, at 32 times the vector ALUs'
// rate in bf16.
//
// A workgroup of four waves owns a TN x TW tile of outputs (TN rows of X, TW
// rows of the expanded weight tile: gated TW/2 outputs, whose gate and up
// rows alternate in runs of TW/4 so that both preactivations of an output
// end in one lane).  The reduction runs in chunks of 128 bytes a row (64
// bf16, 32 fp32) through two LDS buffers, the loads of the next chunk in
// registers: they need no alignment beyond their element's, and columns past
// the end become zeros.  Wave w expands tile rows [w TW/4, (w+1) TW/4) alone,
// so its zero fill and its writes are ordered by the LDS itself.
// The LDS binds where tiles fill the chip (zero fill, one two-byte store per
// kept weight, fragment reads: gated 4096 x 4096 -> 8192, G = 16, K = 4: 815
// us, 480 on the wide tiles, both under the profiler), a memory latency per chunk where they do not
// (back, 777 x 5456 -> 1000: 166 us with one team of waves, 65 with four; 1424
// x 3584 -> 160: 23, and 39 before its loads at the last columns were whole).
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

// LDS layouts of a chunk, 128 bytes a row.
// Rows that are staged whole: 16-byte slot i of a row at slot i ^ (row / 2) % 8
// of its 128 bytes, so that the 16 rows of a fragment read touch distinct bank
// slots.
__device__ __forceinline__ uint32_t slot_addr(uint32_t row, uint32_t slot) {
  return row * kRowBytes + ((slot ^ ((row >> 1) & 7u)) << 4);
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
// The expanded weights, written entry by entry: 16-byte slots of 16 rows side
// by side, erow(row) + ecol(k).  A fragment read is 1 KiB in a row, and with
// whole groups in a tile an entry's address is its group's plus a shift of its
// index.
__device__ __forceinline__ uint32_t erow(uint32_t row) { return ((row >> 4) << 11) | ((row & 15u) << 4); }
template <typename T>
__device__ __forceinline__ uint32_t ecol(uint32_t k) {
  const uint32_t b = k * static_cast<uint32_t>(sizeof(T));
  return ((b >> 4) << 8) | (b & 15u);
}
template <typename T>
__device__ __forceinline__ Unit<T> read_expanded(const uint8_t* tile, uint32_t block, uint32_t u, uint32_t li) {
  Unit<T> f;
#pragma unroll
  for (uint32_t h = 0; h < sizeof(T) / 2; ++h)
    f.d[h] = *reinterpret_cast<const u32x4_t*>(tile + (block << 11) + ((u * (sizeof(T) / 2) + h) << 8) + (li << 4));
  return f;
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
  int32_t y_f32;     // back, grad: Y is fp32
  int32_t act;
  const float* scale;
  const float* bias;
  uint32_t nnb, nwb;  // tile counts along TN and TW
  uint32_t grid;      // workgroups of this launch
  uint32_t base;      // and of those before it
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
  const uint32_t L = p.base + xcd_order(blockIdx.x, p.grid);
  const uint32_t per = 4u * p.nwb, band = L / per, within = L - band * per;
  const uint32_t rows = min(4u, p.nnb - 4u * band);
  const uint32_t wb = within / rows, nb = 4u * band + (within - wb * rows);
  // First row of X of the tile, and first output along the weights: gated f,
  // back c, plain and grad o.  (Where columns of memory are the tile's, a last
  // tile of fewer starts earlier and computes some again, in the same order: its
  // loads are whole.)
  const int64_t along = MODE == kGrad ? p.C : p.N, across = MODE == kBack ? p.C : p.O;
  int64_t n0 = static_cast<int64_t>(nb) * TN, w0 = static_cast<int64_t>(wb) * (MODE == kGated ? TW / 2 : TW);
  if constexpr (MODE == kGrad) n0 = max(min(n0, along - TN), static_cast<int64_t>(0));
  if constexpr (MODE == kGrad || MODE == kBack) w0 = max(min(w0, across - TW), static_cast<int64_t>(0));
  const int64_t F = p.O / 2;
  constexpr bool kFwd = MODE == kGated || MODE == kPlain;
  const int64_t red = kFwd ? p.C : MODE == kBack ? p.O : p.N;  // reduction length
  const int64_t ldx = MODE == kBack ? p.O : p.C;
  const int nch = static_cast<int>((red + BK - 1) / BK);

  // Loads run ND chunks ahead of their use, in register sets taken in turn
  // (one set where two do not fit the registers).
  constexpr int ND = (MODE == kGrad || PL == 4) && (sizeof(T) == 4 || TEAMS == 4) ? 1 : 2;

  // ---- staging of X (gated, plain, back: rows n0 .. of the reduction operand).
  // Rows past the last read it again: their outputs are not stored.  Offsets
  // of lanes are 32-bit, from a row block's first row.
  Unit<T> xu[ND][MODE == kGrad ? 1 : XU];
  const char* xbase = reinterpret_cast<const char*>(X + (MODE == kGrad ? 0 : n0 * ldx));
  uint32_t xoff[MODE == kGrad ? 1 : XU];
  if constexpr (MODE != kGrad) {
#pragma unroll
    for (int i = 0; i < XU; ++i) {
      const int v = tid + kThreads * i;
      const uint32_t row = static_cast<uint32_t>(min(static_cast<int64_t>(v / UPR), p.N - 1 - n0));
      xoff[i] = (row * static_cast<uint32_t>(ldx) + 8u * (v % UPR)) * static_cast<uint32_t>(sizeof(T));
    }
  }
  auto load_x = [&](int ch, int set) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad) {
      const char* xc = xbase + static_cast<int64_t>(ch) * kRowBytes;
      if ((ch + 1) * static_cast<int64_t>(BK) <= red) {
#pragma unroll
        for (int i = 0; i < XU; ++i) load_full<8>(xu[set][i], reinterpret_cast<const T*>(xc + xoff[i]));
      } else {
#pragma unroll
        for (int i = 0; i < XU; ++i)
          load_tail<8>(xu[set][i], reinterpret_cast<const T*>(xc + xoff[i]),
                       red - static_cast<int64_t>(ch) * BK - 8 * ((tid + kThreads * i) % UPR));
      }
    }
  };
  auto store_x = [&](uint8_t* buf, int set) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad) {
#pragma unroll
      for (int i = 0; i < XU; ++i) {
        const int v = tid + kThreads * i;
        write_unit<T>(buf, static_cast<uint32_t>(v / UPR), static_cast<uint32_t>(v % UPR), xu[set][i]);
      }
    }
  };

  // ---- grad: both operands are sample-major; a thread loads 4 columns of 8
  // samples and writes them transposed, 8 samples of a column to a unit.
  using Quad = std::conditional_t<sizeof(T) == 2, u32x2_t, u32x4_t>;
  constexpr int kQuads = MODE == kGrad ? 8 : 1;
  Quad qx[ND][kQuads], qy[ND][kQuads];
  auto load_quads = [&](Quad (&q)[kQuads], const T* src, int64_t width, int64_t col0, int cols, int ch) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      const int cq = tid % (cols / 4), rg = min(tid / (cols / 4), UPR - 1);
      const char* qb = reinterpret_cast<const char*>(src + static_cast<int64_t>(ch) * BK * width + col0);
      const bool all = (ch + 1) * static_cast<int64_t>(BK) <= p.N;
      const int last = all ? BK - 1 : static_cast<int>(p.N - 1 - static_cast<int64_t>(ch) * BK);  // sample of the chunk
      if (all && col0 + cols <= width) {
        const uint32_t off = (static_cast<uint32_t>(8 * rg) * static_cast<uint32_t>(width) + 4u * cq) * static_cast<uint32_t>(sizeof(T));
        const uint32_t step = static_cast<uint32_t>(width) * static_cast<uint32_t>(sizeof(T));
#pragma unroll
        for (int r = 0; r < 8; ++r) load_full<4>(q[r], reinterpret_cast<const T*>(qb + (off + r * step)));
      } else {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const uint32_t off = (static_cast<uint32_t>(min(8 * rg + r, last)) * static_cast<uint32_t>(width) + 4u * cq) *
                               static_cast<uint32_t>(sizeof(T));
          load_tail<4>(q[r], reinterpret_cast<const T*>(qb + off), width - col0 - 4 * cq);
          if (8 * rg + r > last) q[r] = Quad{};  // a sample past the last adds nothing
        }
      }
    }
  };
  auto store_quads = [&](uint8_t* tile, const Quad (&q)[kQuads], int cols) __attribute__((always_inline)) {
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
  //   back         (8 u + e, row0 + idx[e]) if row0 + idx[e] is in the chunk,
  // and otherwise to a word that nobody reads.
  constexpr int kUnitsOfRow = MODE == kBack ? UC : UPR;
  const int64_t f0 = w0 + (MODE == kGated ? (w >> 1) * TQ : w * TQ);  // gated, plain: the wave's first output
  const int64_t wrow = f0 + (MODE == kGated && (w & 1) ? F : 0);      // and weight row
  const int64_t rest = max((MODE == kGated ? F : p.O) - f0, static_cast<int64_t>(0));
  const uint32_t lim = kFwd ? static_cast<uint32_t>(min(static_cast<int64_t>(TQ), rest)) : BK;
  constexpr int PU = PL > 0 ? PL : 1;
  Unit<T> pv[ND][PU];
  u32x2_t pi[ND][PU];
  int grow[PU];  // first row of the group of the unit's packed row, from the first group's
#pragma unroll
  for (int i = 0; i < PU; ++i) grow[i] = (lane + 64 * i) / kUnitsOfRow / p.K * p.G;
  struct Span {
    uint32_t g_lo;  // first group
    int nrows;      // packed rows
    int first;      // g_lo G relative to the wave's rows / the chunk
  };
  auto span = [&](uint32_t b, uint32_t n) __attribute__((always_inline)) {  // groups that meet rows b .. b + n - 1
    const uint32_t G = static_cast<uint32_t>(p.G);
    Span s{0, 0, 0};
    if (n > 0) {
      s.g_lo = b / G;
      s.nrows = static_cast<int>((b + n - 1) / G - s.g_lo + 1) * p.K;
      s.first = static_cast<int>(s.g_lo * G) - static_cast<int>(b);
    }
    return s;
  };
  // (gated, plain: the same in every chunk.  back: where G divides the chunk, the next chunk's groups follow)
  const Span span0 = kFwd ? span(static_cast<uint32_t>(wrow), lim) : span(0, min(static_cast<uint32_t>(BK), static_cast<uint32_t>(p.O)));
  const int gpc = MODE == kBack && BK % p.G == 0 ? BK / p.G : 0;  // back: groups per chunk
  auto span_of = [&](int ch) __attribute__((always_inline)) {
    if constexpr (kFwd) return span0;
    const uint32_t b = static_cast<uint32_t>(ch) * BK, n = min(static_cast<uint32_t>(BK), static_cast<uint32_t>(p.O) - b);
    if (gpc == 0) return span(b, n);
    // (the last chunk may be short: G divides O, and what is left of it)
    return Span{static_cast<uint32_t>(ch) * static_cast<uint32_t>(gpc),
                n == BK ? span0.nrows : static_cast<int>(n / static_cast<uint32_t>(p.G)) * p.K, 0};
  };
  // element offset of a unit from its span's first packed row (a unit without one reads the last and is not written)
  auto unit_off = [&](const Span& s, int v) __attribute__((always_inline)) {
    const uint32_t r = static_cast<uint32_t>(max(min(v / kUnitsOfRow, s.nrows - 1), 0));
    return r * static_cast<uint32_t>(p.C) + 8u * static_cast<uint32_t>(v % kUnitsOfRow);
  };
  auto load_unit = [&](const Span& s, int ch, int v, Unit<T>& val, u32x2_t& ix) __attribute__((always_inline)) {
    const int64_t c0 = kFwd ? static_cast<int64_t>(ch) * BK : w0 + w * TQ;
    const int64_t at = static_cast<int64_t>(s.g_lo) * p.K * p.C + c0;
    const uint32_t off = unit_off(s, v);
    const T* vb = vals + at;
    const uint8_t* ib = idx + at;
    if (c0 + (kFwd ? BK : TQ) <= p.C) {
      load_full<8>(val, reinterpret_cast<const T*>(reinterpret_cast<const char*>(vb) + off * static_cast<uint32_t>(sizeof(T))));
      load_full<8>(ix, ib + off);
    } else {
      const int64_t left = p.C - c0 - 8 * (v % kUnitsOfRow);
      load_tail<8>(val, vb + off, left);
      load_tail<8>(ix, ib + off, left);
    }
  };
  uint8_t* trash = lds + TEAMS * 2 * kBuf;
  // Whole groups lie in the wave's rows (gated, plain) or in a chunk (back) and
  // G is a power of two: no entry has to be checked, and its place is its
  // group's first plus idx rows, or plus idx elements of a row.
  const bool fit = (p.G & (p.G - 1)) == 0 && p.G <= (kFwd ? TQ : BK);
  const uint32_t gmask = static_cast<uint32_t>(p.G - 1) * 0x01010101u;  // (an index past its group stays in the tile)
  // Order of a unit's entries (bf16): back, the rows of the packing over the
  // 16-byte slots of a column block; else the units of a row over a slot's words.
  const Shuffle sh = make_shuffle(sizeof(T) != 2 ? 0u
                                  : kFwd         ? 2u * (static_cast<uint32_t>(lane) & 3u)
                                                 : static_cast<uint32_t>(lane / kUnitsOfRow) & 7u);
  uint32_t eoff[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) eoff[e] = kFwd ? ecol<T>(static_cast<uint32_t>(e) ^ sh.m) : 16u * (static_cast<uint32_t>(e) ^ sh.m);
  auto put = [&](uint8_t* to, const Unit<T>& val, int e) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(val.d[0][e >> 1] >> (16 * (e & 1)));
    else
      *reinterpret_cast<uint32_t*>(to) = val.d[e >> 2][e & 3];
  };
  auto scatter = [&](uint8_t* wt, const Span& s, int v, int row_of_group, Unit<T>& val, u32x2_t& ix) __attribute__((always_inline)) {
    const uint32_t u = static_cast<uint32_t>(v % kUnitsOfRow);
    if constexpr (sizeof(T) == 2) shuffle(sh, val, ix);
    const uint32_t row0 = static_cast<uint32_t>(s.first + row_of_group);  // the group's first row / element
    const bool there = v / kUnitsOfRow < s.nrows;
    const uint32_t r0 = static_cast<uint32_t>(w * TQ);
    if (fit) {
      if (!there) return;
      uint8_t* at = wt + (kFwd ? erow(r0 + row0) + ecol<T>(8 * u) : erow(r0 + 8 * u) + ecol<T>(row0));
      const u32x2_t im = {ix[0] & gmask, ix[1] & gmask};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t i = (im[e >> 2] >> (8 * (e & 3))) & 0xffu;
        const uint32_t step = kFwd ? (TQ > 16 ? erow(i) : i << 4) : ecol<T>(i);
        put(at + step + eoff[e], val, e);
      }
    } else {
      const uint32_t most = there ? lim : 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t t = row0 + ((ix[e >> 2] >> (8 * (e & 3))) & 0xffu);
        const uint32_t at = (kFwd ? erow(r0 + t) + ecol<T>(8 * u) : erow(r0 + 8 * u) + ecol<T>(t)) + eoff[e];
        put(t < most ? wt + at : trash, val, e);
      }
    }
  };
  auto load_w = [&](int ch, int set) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad && PL > 0) {
      const Span s = span_of(ch);
#pragma unroll
      for (int i = 0; i < PL; ++i) load_unit(s, ch, lane + 64 * i, pv[set][i], pi[set][i]);
    }
  };
  auto store_w = [&](uint8_t* wt, int ch, int set) __attribute__((always_inline)) {
    if constexpr (MODE != kGrad) {
#pragma unroll
      for (int i = 0; i < TQ / 8; ++i)
        *reinterpret_cast<u32x4_t*>(wt + w * TQ * kRowBytes + (i * 64 + lane) * 16) = u32x4_t{0u, 0u, 0u, 0u};
      asm volatile("" ::: "memory");  // the zeros come first; one wave's LDS writes stay in order
      const Span s = span_of(ch);
      if constexpr (PL > 0) {
#pragma unroll
        for (int i = 0; i < PL; ++i) scatter(wt, s, lane + 64 * i, grow[i], pv[set][i], pi[set][i]);
      } else {
        const int units = s.nrows * kUnitsOfRow;
#pragma unroll 1
        for (int v = lane; v < units; v += 64) {
          load_unit(s, ch, v, pv[0][0], pi[0][0]);
          scatter(wt, s, v, v / kUnitsOfRow / p.K * p.G, pv[0][0], pi[0][0]);
        }
      }
    }
  };

  auto load_chunk = [&](int ch, int set) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      load_quads(qy[set], dY, p.O, w0, TW, ch);
      load_quads(qx[set], X, p.C, n0, TN, ch);
    } else {
      load_x(ch, set);
      load_w(ch, set);
    }
  };
  auto store_chunk = [&](uint8_t* buf, int ch, int set) __attribute__((always_inline)) {
    if constexpr (MODE == kGrad) {
      store_quads(buf + kXTile, qy[set], TW);
      store_quads(buf, qx[set], TN);
    } else {
      store_x(buf, set);
      store_w(buf + kXTile, ch, set);
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
#pragma unroll
  for (int i = 0; i < ND; ++i)
    if (chunk(i) < nch) load_chunk(chunk(i), i);
  if (chunk(0) < nch) {
    store_chunk(bufs, chunk(0), 0);
    if (chunk(ND) < nch) load_chunk(chunk(ND), 0);
  }
  // Round i: its chunk is complete in its buffer, and nobody reads the one of
  // round i - 1 any more, which takes chunk i + 1 out of its registers (set
  // `next`), which take chunk i + 1 + ND.
  auto round = [&](int i, int next) __attribute__((always_inline)) {
    lds_barrier();
    const uint8_t* cur = bufs + (i & 1) * kBuf;
    if (chunk(i + 1) < nch) {
      store_chunk(bufs + ((i + 1) & 1) * kBuf, chunk(i + 1), next);
      if (chunk(i + 1 + ND) < nch) load_chunk(chunk(i + 1 + ND), next);
    }
    if (chunk(i) >= nch) return;
    const uint8_t* xt = cur;
    const uint8_t* wt = cur + kXTile;
#pragma unroll
    for (int ks = 0; ks < UPR / 4; ++ks) {
      Unit<T> a[OT], b[NT];
#pragma unroll
      for (int o = 0; o < OT; ++o) a[o] = MODE == kGrad
                   ? read_unit<T>(wt, static_cast<uint32_t>(wo * (TW / 2) + 16 * o) + li, 4u * ks + lq)
                   : read_expanded<T>(wt, static_cast<uint32_t>(wo * (TW / 32) + o), 4u * ks + lq, li);
#pragma unroll
      for (int n = 0; n < NT; ++n) b[n] = read_unit<T>(xt, static_cast<uint32_t>(wn * (TN / 2) + 16 * n) + li, 4u * ks + lq);
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int n = 0; n < NT; ++n) mma(acc[o][n], a[o], b[n]);
    }
  };
#pragma unroll 1
  for (int i = 0; i < rounds; i += ND) {
    round(i, ND - 1);
    if constexpr (ND == 2) {
      if (i + 1 < rounds) round(i + 1, 0);
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
        }
        store4<float>(global_ptr<float>(p.Y) + at, v, p.O - c, vec);
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
  constexpr int kLds = (kOperands > kPark ? kOperands : kPark) + 16;  // and the word for entries of other tiles
  const int64_t along_n = MODE == kGrad ? p.C : p.N;
  const int64_t along_w = MODE == kBack ? p.C : p.O;
  const int64_t nnb = (along_n + TN - 1) / TN, nwb = (along_w + TW - 1) / TW;
  if (nnb > 0x7fffffff / 8 || nwb > 0x7fffffff / 8 || nnb * nwb > 0x7fffffff) return hipErrorInvalidConfiguration;
  p.nnb = static_cast<uint32_t>(nnb);
  p.nwb = static_cast<uint32_t>(nwb);
  static std::atomic<int8_t> lds_set[kMaxDevices];
  const hipError_t e = set_lds_limit_once(lds_set, reinterpret_cast<const void*>(&tile_kernel<T, MODE, TN, TW, PL, TEAMS>), kLds);
  if (e != hipSuccess) return e;
  constexpr int64_t kMost = kMostThreads / (TEAMS * kThreads) / 8 * 8;  // workgroups of a launch
  for (int64_t first = 0; first < nnb * nwb; first += kMost) {
    p.base = static_cast<uint32_t>(first);
    p.grid = static_cast<uint32_t>(nnb * nwb - first < kMost ? nnb * nwb - first : kMost);
    hipLaunchKernelGGL((tile_kernel<T, MODE, TN, TW, PL, TEAMS>), dim3(p.grid), dim3(TEAMS * kThreads), kLds, s, p);
    if (const hipError_t f = hipGetLastError(); f != hipSuccess) return f;
  }
  return hipSuccess;
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
