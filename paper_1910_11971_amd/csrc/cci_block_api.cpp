// C ABI of the feed-forward block's operators: argument validation, kernel
// choice and error reporting.  Nothing here allocates, synchronises or keeps
// state.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/cci.h"
#include "cci_block.hpp"
#include "cci_check.hpp"

using namespace cci;

namespace {

// Row counts whose element offsets stay far inside 64 bits and whose grids fit.
cci_status check_rows(int64_t N, int64_t width) {
  if (N < 0) return fail(CCI_EINVAL, "N=%lld < 0", (long long)N);
  if (N > (int64_t(1) << 31) || N > (int64_t(1) << 40) / width) return fail(CCI_EINVAL, "N too large");
  return CCI_OK;
}

// Lanes of the product kernels address rows with 32-bit offsets.
constexpr int64_t kWidest = int64_t(1) << 20;

cci_status check_product(int64_t N, int64_t C, int64_t O, int32_t G, int32_t K) {
  if (cci_status s = check_groups(O, C, G, K)) return s;
  if (C > kWidest || O > kWidest)
    return fail(CCI_EINVAL, "C=%lld or %lld weight rows above 2^20", (long long)C, (long long)O);
  return check_rows(N, C > O ? C : O);
}

cci_status check_act(cci_act act) {
  switch (act) {
    case CCI_ACT_NONE:
    case CCI_ACT_RELU:
    case CCI_ACT_SILU:
    case CCI_ACT_GELU:
    case CCI_ACT_GELU_TANH: return CCI_OK;
  }
  return fail(CCI_EINVAL, "unknown activation %d", (int)act);
}

bool misaligned(const void* p) { return p && !aligned16(p); }

cci_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(CCI_EHIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return ok();
}

cci_status check_norm(cci_dtype t, int64_t N, int64_t C) {
  if (!dtype_ok(t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (C < 1 || C > (int64_t(1) << 31)) return fail(CCI_EINVAL, "C=%lld outside [1, 2^31]", (long long)C);
  return check_rows(N, C);
}

cci_status check_gated(cci_dtype t, int64_t N, int64_t C, int64_t F, int32_t G, int32_t K, cci_act act) {
  if (!dtype_ok(t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (cci_status s = check_groups(F, C, G, K)) return s;
  if (cci_status s = check_act(act)) return s;
  return check_product(N, C, 2 * F, G, K);
}

Act to_act(cci_act a) {
  switch (a) {
    case CCI_ACT_RELU: return Act::RELU;
    case CCI_ACT_SILU: return Act::SILU;
    case CCI_ACT_GELU: return Act::GELU;
    case CCI_ACT_GELU_TANH: return Act::GELU_TANH;
    default: return Act::NONE;
  }
}

cci_status check_adapters(int64_t N, int64_t C, int64_t O, int64_t L, int32_t R) {
  if (R < 1 || R > 1024) return fail(CCI_EINVAL, "R=%d outside [1, 1024]", R);
  if (L < 1 || L > (int64_t(1) << 31) - 1) return fail(CCI_EINVAL, "L=%lld outside [1, 2^31)", (long long)L);
  if (C < 1 || O < 1 || C > (int64_t(1) << 31) || O > (int64_t(1) << 31))
    return fail(CCI_EINVAL, "C=%lld or O=%lld outside [1, 2^31]", (long long)C, (long long)O);
  if (L > (int64_t(1) << 40) / R / (C > O ? C : O)) return fail(CCI_EINVAL, "L*R*max(C, O) too large");
  return check_rows(N, C > O ? C : O);
}

// Rows that a call takes at a time.  The projection waits in the workspace in
// fp32 for its adapters' term; slices keep that at 1 GiB, and inside the
// 32-bit offsets of the kernels that cci_spmm runs large products on.
int64_t adapter_slice(int64_t N, int64_t O) { return std::min(N, std::max<int64_t>(256, (int64_t(1) << 28) / O / 256 * 256)); }

size_t adapter_base_bytes(int64_t N, int64_t O) {
  return (static_cast<size_t>(adapter_slice(N, O)) * static_cast<size_t>(O) * sizeof(float) + 15) / 16 * 16;
}

// Projection and partial sums of a slice, whole or the last one.
size_t adapter_workspace(int64_t N, int64_t C, int64_t O, int64_t L, int32_t R) {
  if (N == 0) return 0;
  const int64_t rows = adapter_slice(N, O), last = N % rows;
  const int64_t part = std::max(adapter_part_bytes(rows, C, L, R), last ? adapter_part_bytes(last, C, L, R) : 0);
  return adapter_base_bytes(N, O) + static_cast<size_t>(part);
}

// Whether an fp32 product beside adapters runs on the tile kernels: cci_spmm
// has the vector ALUs alone for it.  Those take up to 256 rows in one pass over
// the packed weights, whose length (C K entries of a group, one after another)
// and kept multiply-adds set the time; from 257 rows on they are far behind.
// Tiles take a time per chunk of 32 columns and round of 256 tiles, whatever
// is kept.  us of a call, vector ALUs / tiles, and what is chosen:
//   640 -> 352, G = 8, K = 2    64 rows 14 / 28 v, 256 rows 30 / 34 v
//   640 -> 352, G = 32, K = 8   64 rows 33 / 30 t, 256 rows 56 / 36 t
//   256 -> 512, G = 8, K = 4    64 rows 12 / 19 v, 128 rows 22 / 25 v, 256 rows 28 / 25 t
//   1024 -> 1024, G = 16, K = 4 64 rows 28 / 37 v, 96 rows 44 / 45 v, 128 rows 51 / 43 t
//   1024 -> 1024, G = 16, K = 8 24 rows 28 / 37 v, 48 rows 42 / 37 t
//   4096 -> 4096, G = 16, K = 4 16 rows 82 / 109 v, 24 rows 116 / 111 t, 64 rows 277 / 114 t
//   320 -> 128, G = 8, K = 2    304 rows 273 / 28 t
// On 48 drawn shapes of 1 to 468 rows the choice takes 1.01 times the better form's time.
bool f32_on_tiles(const BlockProduct& p) {
  if (p.G != 2 && p.G != 4 && p.G != 8 && p.G != 16 && p.G != 32) return true;  // cci_spmm refuses them
  if (p.N > 256) return true;
  const double kept = static_cast<double>(p.N) * static_cast<double>(p.O) * static_cast<double>(p.C) * p.K / p.G;
  const double walk = static_cast<double>(p.C) * p.K * (p.G <= 16 ? 2.3e-3 : 4.1e-3);
  const double chunks = static_cast<double>((p.C + 31) / 32);
  const double filled = std::max(1.0, static_cast<double>(p.N) * static_cast<double>(p.O) / (256.0 * 64 * 64));
  return 3.0 + 0.9 * chunks * filled < walk + kept * (p.K == 1 ? 1.8e-6 : 0.85e-6);
}

// cci_spmm runs a product on kernels made for its shape, except in bf16 what
// it leaves to the vector ALUs, at 1/32 of the matrix cores' rate (239 x 3896
// -> 416, G = 32, K = 8: 271 us there, 28 here), and groups that it refuses.
// Rows that are not a multiple of 8 elements long have a form there that reads
// element by element.
bool tile_product(const BlockProduct& p) {
  if (p.t == DType::F32) return f32_on_tiles(p);
  if (p.C % 8 != 0 || p.O % 8 != 0) return true;
  ProductArgs a{};
  a.X = p.X;
  a.x_t = a.val_t = p.t;
  a.N = p.N;
  a.C = p.C;
  a.conv = false;
  a.vals = p.vals;
  a.idx = p.idx;
  a.O = p.O;
  a.G = p.G;
  a.K = p.K;
  a.Y = p.Y;
  a.y_t = p.y_t;
  a.scale = p.scale;
  a.bias = p.bias;
  return spmm_without_matrix_cores(a);
}

// ---------------------------------------------------------------------------
// Which kernels run a bf16 gated product or input gradient.  Each family has a
// time per piece of the reduction and round of workgroups over the 256 CUs,
// measured on 90 shapes with G = 4 .. 32 and K / G = 1/4 and 1/2 (us):
//   64 x 64 tiles, four teams of waves  1.25 a 4 chunks of 64, 3.5 a round
//   64 x 64 tiles, one team             0.95 a chunk for up to 1024 tiles
//   128 x 128 tiles                     1.1 a chunk, 1.4 for 257 .. 512 tiles, and so on by 512
//   wide tiles, 128 rows                1.07 a chunk, 256 rows 1.42
//   wave-split                          kSteps: a step of its eight waves, a round
// Both sides of the borders (tile / wide 128 / wide 256 / wave-split):
//   gated, C = 4096, F = 8192: 32 rows 25 / - / - / 17, 64 rows 24 / - / - / 28, 128 rows 48 / 68 / 94 / 51, 256 rows
//   70 / 69 / 95 / 96, 1024 rows 171 / 134 / 103 / 360; C = 2928, F = 4704, 70 rows 36 / - / - / 20;
//   dX, O = 8192, C = 4096: 256 rows 50 / 136 / 182 / 45, 1024 rows 144 / 137 / 181 / 164, 2048 rows 190 / 142 / 181 / 309.
// On 41 drawn shapes of up to 3400 rows the choice takes 1.01 times the best form's time (dX).

double rounds(int64_t tiles, int64_t at_once) { return static_cast<double>((tiles + at_once - 1) / at_once); }

enum Kind { kTiles, kWide128, kWide256, kWave4, kWave2, kWave1 };
struct Choice {
  Kind kind;
  double us;
  int rows;  // wave-split: of a tile
};
void consider(Choice& best, Kind kind, double us, int rows = 0) {
  if (us < best.us) best = Choice{kind, us, rows};
}

// out: the outputs of a row, per64 / per256: those of a 64- and a 256-row weight tile.
Choice tile_or_wide(const BlockProduct& p, int64_t red, int64_t out, int64_t per64, int64_t per256, bool wide) {
  const double chunks = static_cast<double>((red + 63) / 64);
  const int64_t t64 = (p.N + 63) / 64 * ((out + per64 - 1) / per64);
  const int64_t t128 = (p.N + 127) / 128 * ((out + 2 * per64 - 1) / (2 * per64));
  const double teams = static_cast<double>((red + 255) / 256);
  Choice best{kTiles,
              t128 >= 256  ? 4.0 + chunks * (t128 <= 256 ? 1.1 : 1.4 * rounds(t128, 512))
              : t64 <= 512 ? 1.0 + rounds(t64, 256) * (teams * 1.25 + 3.5)
                           : 4.0 + chunks * 0.95,
              0};
  if (wide) {
    const int64_t w = (out + per256 - 1) / per256;
    consider(best, kWide128, 4.0 + chunks * 1.07 * rounds((p.N + 127) / 128 * w, 256));
    consider(best, kWide256, 6.0 + chunks * 1.42 * rounds((p.N + 255) / 256 * w, 256));
  }
  return best;
}

// The best of the wave-split kernels' tiles (blocks of 16 rows, nt, and of weights, wb): us a step, a round and a
// call.  Half the rows take more than half the time, but fill the CUs where tiles are few, and two workgroups of the
// narrowest tile share a CU (short rounds).  64 / 32 rows, dX: 333 x 1000 -> 2728 19.2 / 11.4, 777 x 5456 -> 1000
// 29.5 / 35.1, 1424 x 3584 -> 160 22.9 / 15.5.
struct StepTime {
  double step, round, call;
};
constexpr StepTime kSteps[3][3] = {{{0.55, 4.0, 5.0}, {0.6, 4.0, 5.0}, {1.2, 4.0, 5.0}},    // nt = 1: wb = 4, 2, 1
                                   {{0.62, 1.5, 3.7}, {0.85, 6.0, 1.0}, {1.6, 6.0, 1.5}},    // nt = 2
                                   {{0.98, 5.0, 1.0}, {1.75, 4.8, 1.0}, {3.4, 6.0, 1.0}}};   // nt = 4
void consider_wave_split(Choice& best, const BlockProduct& p, bool gated) {
  const int64_t red = gated ? p.C : p.O, out = gated ? p.O / 2 : p.C;
  const int most = p.N <= 16 ? 1 : p.N <= 32 || gated ? 2 : 4;  // blocks of 16 rows
  for (int nt = most; nt >= (most == 4 ? 2 : most); nt -= 2) {
    for (const int wb : {4, 2, 1}) {
      if (!wave_split_supports(p, gated, wb)) continue;
      const int64_t ks = 128 / wb;  // elements of a step
      const StepTime& t = kSteps[nt / 2][wb == 4 ? 0 : wb == 2 ? 1 : 2];
      const double steps = static_cast<double>((red + 8 * ks - 1) / (8 * ks));
      const int64_t width = (gated ? 8 : 16) * wb, tiles = (p.N + 16 * nt - 1) / (16 * nt) * ((out + width - 1) / width);
      consider(best, wb == 4 ? kWave4 : wb == 2 ? kWave2 : kWave1,
               t.call + rounds(tiles, 256) * (steps * t.step + t.round), 16 * nt);
    }
  }
}

int wave_width(Kind kind) { return kind == kWave4 ? 4 : kind == kWave2 ? 2 : kind == kWave1 ? 1 : 0; }

hipError_t gated_product(const BlockProduct& p, hipStream_t st) {
  if (p.t != DType::BF16) return launch_tile_gated(p, st);
  Choice c = tile_or_wide(p, p.C, p.O / 2, 32, 128, wide_gated_supports(p));
  consider_wave_split(c, p, true);
  if (const int wb = wave_width(c.kind)) return launch_wave_split(p, true, wb, c.rows, st);
  return c.kind == kTiles ? launch_tile_gated(p, st) : launch_wide_gated(p, c.kind == kWide256 ? 8 : 4, st);
}

hipError_t input_gradient(const BlockProduct& p, hipStream_t st) {
  if (p.t != DType::BF16) return launch_tile_back(p, st);
  Choice c = tile_or_wide(p, p.O, p.C, 64, 256, wide_back_supports(p));
  consider_wave_split(c, p, false);
  if (const int wb = wave_width(c.kind)) return launch_wave_split(p, false, wb, c.rows, st);
  return c.kind == kTiles ? launch_tile_back(p, st) : launch_wide_back(p, c.kind == kWide256 ? 8 : 4, st);
}

}  // namespace

extern "C" {

cci_status cci_layernorm(const void* X, cci_dtype t, int64_t N, int64_t C, const float* gamma, const float* beta,
                         float eps, void* Y, float* mean, float* rstd, void* stream) {
  if (cci_status s = check_norm(t, N, C)) return s;
  if (!(eps >= 0.0f)) return fail(CCI_EINVAL, "eps must be >= 0");
  if (N == 0) return ok();
  if (!X || !Y) return fail(CCI_EINVAL, "null pointer");
  if (!aligned16(X) || !aligned16(Y) || misaligned(gamma) || misaligned(beta) || misaligned(mean) || misaligned(rstd))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  return launched(launch_layernorm(X, to_dt(t), N, C, gamma, beta, eps, Y, mean, rstd, static_cast<hipStream_t>(stream)),
                  "layer-norm");
}

cci_status cci_layernorm_bwd_workspace(int64_t N, int64_t C, size_t* bytes) {
  if (cci_status s = check_norm(CCI_F32, N, C)) return s;
  if (!bytes) return fail(CCI_EINVAL, "null output pointer");
  *bytes = static_cast<size_t>(layernorm_bwd_workspace(N, C));
  return ok();
}

cci_status cci_layernorm_bwd(const void* dY, const void* X, cci_dtype t, int64_t N, int64_t C, const float* gamma,
                             const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta,
                             void* workspace, size_t workspace_bytes, void* stream) {
  if (cci_status s = check_norm(t, N, C)) return s;
  if (N > 0 && (!dY || !X || !mean || !rstd)) return fail(CCI_EINVAL, "null pointer");
  const size_t need = dgamma || dbeta || C > kNormBwdMost ? static_cast<size_t>(layernorm_bwd_workspace(N, C)) : 0;
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(CCI_EINVAL, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : 0, need);
  if (misaligned(dY) || misaligned(X) || misaligned(gamma) || misaligned(mean) || misaligned(rstd) || misaligned(dX) ||
      misaligned(dgamma) || misaligned(dbeta) || misaligned(workspace))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  return launched(launch_layernorm_bwd(dY, X, to_dt(t), N, C, gamma, mean, rstd, dX, dgamma, dbeta, workspace,
                                       static_cast<hipStream_t>(stream)),
                  "layer-norm backward");
}

cci_status cci_gated_spmm(const void* X, cci_dtype t, int64_t N, int64_t C, const void* vals, const uint8_t* idx,
                          int64_t F, int32_t G, int32_t K, cci_act act, void* H, void* pre, void* stream) {
  if (cci_status s = check_gated(t, N, C, F, G, K, act)) return s;
  if (N == 0) return ok();
  if (!X || !vals || !idx || !H) return fail(CCI_EINVAL, "null pointer");
  if (!aligned16(X) || !aligned16(vals) || !aligned16(idx) || !aligned16(H) || misaligned(pre))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  BlockProduct p{};
  p.X = X;
  p.t = p.y_t = to_dt(t);
  p.N = N;
  p.C = C;
  p.vals = vals;
  p.idx = idx;
  p.O = 2 * F;
  p.G = G;
  p.K = K;
  p.act = to_act(act);
  p.Y = H;
  p.pre = pre;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return launched(gated_product(p, st), "gated product");
}

cci_status cci_spmm_t(const void* dY, cci_dtype t, int64_t N, int64_t O, const void* vals, const uint8_t* idx,
                      int64_t C, int32_t G, int32_t K, void* dX, cci_dtype dx_t, void* stream) {
  if (!dtype_ok(t) || !dtype_ok(dx_t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (t == CCI_F32 && dx_t != CCI_F32) return fail(CCI_EUNSUPPORTED, "an fp32 product has an fp32 output");
  if (cci_status s = check_product(N, C, O, G, K)) return s;
  if (N == 0) return ok();
  if (!dY || !vals || !idx || !dX) return fail(CCI_EINVAL, "null pointer");
  if (!aligned16(dY) || !aligned16(vals) || !aligned16(idx) || !aligned16(dX))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  BlockProduct p{};
  p.dY = dY;
  p.t = to_dt(t);
  p.N = N;
  p.C = C;
  p.vals = vals;
  p.idx = idx;
  p.O = O;
  p.G = G;
  p.K = K;
  p.Y = dX;
  p.y_t = to_dt(dx_t);
  return launched(input_gradient(p, static_cast<hipStream_t>(stream)), "transposed product");
}

cci_status cci_gated_spmm_bwd(const void* dH, const void* pre, const void* X, cci_dtype t, int64_t N, int64_t C,
                              const void* vals, const uint8_t* idx, int64_t F, int32_t G, int32_t K, cci_act act,
                              void* dpre, void* dX, void* dvals, cci_dtype dv_t, void* stream) {
  if (cci_status s = check_gated(t, N, C, F, G, K, act)) return s;
  if (!dtype_ok(dv_t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (t == CCI_F32 && dv_t != CCI_F32) return fail(CCI_EUNSUPPORTED, "an fp32 backward pass has fp32 gradients");
  if (N > 0 && (!dH || !pre || !dpre)) return fail(CCI_EINVAL, "null pointer");
  if (N > 0 && dX && !vals) return fail(CCI_EINVAL, "dX needs the packed values");
  if (N > 0 && dvals && !X) return fail(CCI_EINVAL, "dvals needs X");
  if (((N > 0 && dX) || dvals) && !idx) return fail(CCI_EINVAL, "null pointer");
  if (misaligned(dH) || misaligned(pre) || misaligned(X) || misaligned(vals) || misaligned(idx) || misaligned(dpre) ||
      misaligned(dX) || misaligned(dvals))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (N > 0) e = launch_gate_grad(dH, pre, to_dt(t), N, F, to_act(act), dpre, st);
  BlockProduct p{};
  p.X = X;
  p.dY = dpre;
  p.t = to_dt(t);
  p.N = N;
  p.C = C;
  p.vals = vals;
  p.idx = idx;
  p.O = 2 * F;
  p.G = G;
  p.K = K;
  if (e == hipSuccess && N > 0 && dX) {
    p.Y = dX;
    p.y_t = p.t;
    e = input_gradient(p, st);
  }
  if (e == hipSuccess && dvals) {
    p.Y = dvals;
    p.y_t = to_dt(dv_t);
    e = N >= 32 && grad_mfma_supports(dpre, X, p.t, N, C, 2 * F, G)
            ? launch_grad_mfma_to(dpre, X, N, C, idx, 2 * F, G, K, dvals, p.y_t, st)
            : launch_tile_grad(p, st);
  }
  return launched(e, "gated backward");
}

cci_status cci_spmm_adapters_workspace(int64_t N, int64_t C, int64_t O, int64_t L, int32_t R, cci_dtype y_t,
                                       size_t* bytes) {
  if (!dtype_ok(y_t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (cci_status s = check_adapters(N, C, O, L, R)) return s;
  if (!bytes) return fail(CCI_EINVAL, "null output pointer");
  *bytes = adapter_workspace(N, C, O, L, R);
  return ok();
}

cci_status cci_spmm_adapters(const void* X, cci_dtype x_t, int64_t N, int64_t C, const void* vals, cci_dtype val_t,
                             const uint8_t* idx, int64_t O, int32_t G, int32_t K, const cci_adapters* adapters,
                             const cci_epilogue* ep, void* Y, cci_dtype y_t, void* workspace, size_t workspace_bytes,
                             void* stream) {
  if (!dtype_ok(x_t) || !dtype_ok(val_t) || !dtype_ok(y_t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (x_t != val_t || (x_t == CCI_F32 && y_t != CCI_F32))
    return fail(CCI_EUNSUPPORTED, "dtype combination (x=%d, vals=%d, y=%d) not supported", x_t, val_t, y_t);
  if (cci_status s = check_product(N, C, O, G, K)) return s;
  if (!adapters) return fail(CCI_EINVAL, "null pointer");
  if (cci_status s = check_adapters(N, C, O, adapters->L, adapters->R)) return s;
  if (N == 0) return ok();
  if (!X || !vals || !idx || !Y || !adapters->A || !adapters->B || !adapters->rows)
    return fail(CCI_EINVAL, "null pointer");
  if (!aligned16(X) || !aligned16(vals) || !aligned16(idx) || !aligned16(Y) || !aligned16(adapters->A) ||
      !aligned16(adapters->B) || !aligned16(adapters->rows) || misaligned(adapters->alpha) || misaligned(workspace) ||
      (ep && (misaligned(ep->scale) || misaligned(ep->bias) || misaligned(ep->residual))))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  const size_t need = adapter_workspace(N, C, O, adapters->L, adapters->R);
  if (!workspace || workspace_bytes < need)
    return fail(CCI_EINVAL, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : 0, need);
  // the projection in fp32, then the adapters' term and the one rounding to Y's type
  float* base = static_cast<float*>(workspace);
  const cci_epilogue affine{ep ? ep->scale : nullptr, ep ? ep->bias : nullptr, nullptr, 0};
  BlockProduct p{};
  p.t = to_dt(x_t);
  p.C = C;
  p.vals = vals;
  p.idx = idx;
  p.O = O;
  p.G = G;
  p.K = K;
  p.Y = base;
  p.y_t = DType::F32;
  p.scale = affine.scale;
  p.bias = affine.bias;
  AdapterArgs a{};
  a.t = p.t;
  a.C = C;
  a.O = O;
  a.L = adapters->L;
  a.R = adapters->R;
  a.A = adapters->A;
  a.B = adapters->B;
  a.alpha = adapters->alpha;
  a.base = base;
  a.relu = ep ? ep->relu : 0;
  a.d_t = to_dt(y_t);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + adapter_base_bytes(N, O));
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t slice = adapter_slice(N, O);
  for (int64_t n = 0; n < N; n += slice) {
    p.X = a.X = static_cast<const char*>(X) + static_cast<size_t>(n * C) * dsize(x_t);
    p.N = a.N = std::min(slice, N - n);
    a.rows = adapters->rows + n;
    a.residual = ep && ep->residual ? static_cast<const char*>(ep->residual) + static_cast<size_t>(n * O) * dsize(y_t) : nullptr;
    a.D = static_cast<char*>(Y) + static_cast<size_t>(n * O) * dsize(y_t);
    const cci_status s =
        tile_product(p) ? launched(launch_tile_plain(p, st), "product")
                        : cci_spmm(p.X, x_t, p.N, C, vals, val_t, idx, O, G, K, &affine, base, CCI_F32, stream);
    if (s != CCI_OK) return s;
    if (const cci_status t = launched(launch_adapters(a, st), "adapter")) return t;
  }
  return ok();
}

}  // extern "C"
