// C ABI of the feed-forward block's operators: argument validation, kernel
// choice and error reporting.  Nothing here allocates, synchronises or keeps
// state.
#include <hip/hip_runtime.h>

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
  if (cci_status s = check_groups(2 * F, C, G, K)) return s;
  if (cci_status s = check_act(act)) return s;
  return check_rows(N, C > 2 * F ? C : 2 * F);
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

size_t adapter_d_bytes(int64_t N, int64_t O, cci_dtype y_t) {
  return (static_cast<size_t>(N) * static_cast<size_t>(O) * dsize(y_t) + 15) / 16 * 16;
}

// cci_spmm runs a product on kernels made for its shape, except where rows
// are not a multiple of 8 elements long (bf16: the vector ALUs, which do 1/32
// of the matrix cores' rate) and for groups that it refuses.
bool tile_product(cci_dtype t, int64_t C, int64_t O, int32_t G) {
  const bool mac = G == 2 || G == 4 || G == 8 || G == 16 || G == 32;
  return !mac || (t == CCI_BF16 && (C % 8 != 0 || O % 8 != 0));
}

hipError_t input_gradient(const BlockProduct& p, hipStream_t st) {
  return wide_back_supports(p) ? launch_wide_back(p, st) : launch_tile_back(p, st);
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
  const size_t need = static_cast<size_t>(layernorm_bwd_workspace(N, C));
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
  return launched(gated_few_supports(p)    ? launch_gated_few(p, st)
                  : wide_gated_supports(p) ? launch_wide_gated(p, st)
                                           : launch_tile_gated(p, st),
                  "gated product");
}

cci_status cci_spmm_t(const void* dY, cci_dtype t, int64_t N, int64_t O, const void* vals, const uint8_t* idx,
                      int64_t C, int32_t G, int32_t K, void* dX, cci_dtype dx_t, void* stream) {
  if (!dtype_ok(t) || !dtype_ok(dx_t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (t == CCI_F32 && dx_t != CCI_F32) return fail(CCI_EUNSUPPORTED, "an fp32 product has an fp32 output");
  if (cci_status s = check_groups(O, C, G, K)) return s;
  if (cci_status s = check_rows(N, C > O ? C : O)) return s;
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
  *bytes = N == 0 ? 0 : adapter_d_bytes(N, O, y_t) + static_cast<size_t>(adapter_part_bytes(N, C, L, R));
  return ok();
}

cci_status cci_spmm_adapters(const void* X, cci_dtype x_t, int64_t N, int64_t C, const void* vals, cci_dtype val_t,
                             const uint8_t* idx, int64_t O, int32_t G, int32_t K, const cci_adapters* adapters,
                             const cci_epilogue* ep, void* Y, cci_dtype y_t, void* workspace, size_t workspace_bytes,
                             void* stream) {
  if (!dtype_ok(x_t) || !dtype_ok(val_t) || !dtype_ok(y_t)) return fail(CCI_EINVAL, "unknown dtype code");
  if (x_t != val_t || (x_t == CCI_F32 && y_t != CCI_F32))
    return fail(CCI_EUNSUPPORTED, "dtype combination (x=%d, vals=%d, y=%d) not supported", x_t, val_t, y_t);
  if (cci_status s = check_groups(O, C, G, K)) return s;
  if (!adapters) return fail(CCI_EINVAL, "null pointer");
  if (cci_status s = check_adapters(N, C, O, adapters->L, adapters->R)) return s;
  if (N == 0) return ok();
  if (!X || !vals || !idx || !Y || !adapters->A || !adapters->B || !adapters->rows)
    return fail(CCI_EINVAL, "null pointer");
  if (!aligned16(X) || !aligned16(vals) || !aligned16(idx) || !aligned16(Y) || !aligned16(adapters->A) ||
      !aligned16(adapters->B) || !aligned16(adapters->rows) || misaligned(adapters->alpha) || misaligned(workspace) ||
      (ep && (misaligned(ep->scale) || misaligned(ep->bias) || misaligned(ep->residual))))
    return fail(CCI_EALIGN, "pointer not 16-byte aligned");
  const size_t d_bytes = adapter_d_bytes(N, O, y_t);
  const size_t need = d_bytes + static_cast<size_t>(adapter_part_bytes(N, C, adapters->L, adapters->R));
  if (!workspace || workspace_bytes < need)
    return fail(CCI_EINVAL, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : 0, need);
  AdapterArgs a{};
  a.X = X;
  a.t = to_dt(x_t);
  a.N = N;
  a.C = C;
  a.O = O;
  a.L = adapters->L;
  a.R = adapters->R;
  a.A = adapters->A;
  a.B = adapters->B;
  a.alpha = adapters->alpha;
  a.rows = adapters->rows;
  a.residual = ep ? ep->residual : nullptr;
  a.D = workspace;
  a.d_t = to_dt(y_t);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + d_bytes);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (cci_status s = launched(launch_adapters(a, st), "adapter")) return s;
  cci_epilogue with{ep ? ep->scale : nullptr, ep ? ep->bias : nullptr, workspace, ep ? ep->relu : 0};
  if (!tile_product(x_t, C, O, G))
    return cci_spmm(X, x_t, N, C, vals, val_t, idx, O, G, K, &with, Y, y_t, stream);
  BlockProduct p{};
  p.X = X;
  p.t = to_dt(x_t);
  p.N = N;
  p.C = C;
  p.vals = vals;
  p.idx = idx;
  p.O = O;
  p.G = G;
  p.K = K;
  p.Y = Y;
  p.y_t = to_dt(y_t);
  p.scale = with.scale;
  p.bias = with.bias;
  p.residual = with.residual;
  p.relu = with.relu;
  return launched(launch_tile_plain(p, st), "product");
}

}  // extern "C"
