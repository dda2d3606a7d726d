// Host-side launcher interface of the feed-forward block's operators (layer
// norm, gated product, transposed product, adapters) between their C ABI
// layer (cci_block_api.cpp) and the kernel translation units.  Every launcher
// assumes validated arguments and returns the HIP status of its launch.
#pragma once

#include "cci_launch.hpp"

namespace cci {

// Activations (the values of cci_act).
enum class Act { NONE = 0, RELU = 1, SILU = 2, GELU = 3, GELU_TANH = 4 };

// Layer norm over the last dimension.
hipError_t launch_layernorm(const void* X, DType t, int64_t N, int64_t C, const float* gamma, const float* beta,
                            float eps, void* Y, float* mean, float* rstd, hipStream_t s);
// The backward pass keeps rows of up to so many elements in registers; it needs no workspace for them where the weight
// gradients (dgamma and dbeta) are not wanted.
constexpr int64_t kNormBwdMost = 16384;
int64_t layernorm_bwd_workspace(int64_t N, int64_t C);
hipError_t launch_layernorm_bwd(const void* dY, const void* X, DType t, int64_t N, int64_t C, const float* gamma,
                                const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta,
                                void* workspace, hipStream_t s);

// Products over one CCI packing on the matrix cores, any sizes, G and K.
struct BlockProduct {
  const void* X;       // gated, plain, grad: X [N][C]
  const void* dY;      // back, grad: dY [N][O]
  DType t;
  int64_t N, C;
  const void* vals;    // [O/G][K][C] of t
  const uint8_t* idx;
  int64_t O;           // gated: 2 F
  int32_t G, K;
  Act act;             // gated
  void* Y;             // gated: H [N][O/2]; plain: [N][O]; back: dX [N][C]; grad: dvals [O/G][K][C]
  void* pre;           // gated: preactivations [N][O], or null
  DType y_t;           // plain, back, grad: type of Y
  const float* scale;  // plain: Y = (X . W_hat^T) * scale + bias (each may be null)
  const float* bias;
};
// Groups that meet any `span` rows starting at a multiple of it.
inline int64_t groups_in(int64_t span, int64_t G) {
  return span % G == 0 ? span / G : G % span == 0 ? 1 : (span - 2) / G + 2;
}

// cci_spmm would run this product on the sparse-MAC kernels, or refuse it (cci_api.cpp).
bool spmm_without_matrix_cores(ProductArgs a);

// bf16 gated products and input gradients over few tiles of up to 64 rows x
// 16 wb weight rows (wb 4, 2; input gradients also 1): 8 wb outputs (gated) or
// 16 wb columns.
bool wave_split_supports(const BlockProduct& a, bool gated, int wb);
hipError_t launch_wave_split(const BlockProduct& a, bool gated, int wb, int rows, hipStream_t s);
// bf16 gated products and input gradients in tiles of 32 pt rows (pt 4 or 8)
// x 128 outputs (gated) or 256 columns; 64 % G == 0, sizes in multiples of 8.
bool wide_gated_supports(const BlockProduct& a);
hipError_t launch_wide_gated(const BlockProduct& a, int pt, hipStream_t s);
bool wide_back_supports(const BlockProduct& a);
hipError_t launch_wide_back(const BlockProduct& a, int pt, hipStream_t s);
// Any gated product, plain product, input gradient and packed-value gradient.
hipError_t launch_tile_gated(const BlockProduct& a, hipStream_t s);
hipError_t launch_tile_plain(const BlockProduct& a, hipStream_t s);
hipError_t launch_tile_back(const BlockProduct& a, hipStream_t s);
hipError_t launch_tile_grad(const BlockProduct& a, hipStream_t s);

// launch_grad_mfma with the gradient in fp32 or bf16.
hipError_t launch_grad_mfma_to(const void* dY, const void* X, int64_t N, int64_t C, const uint8_t* idx, int64_t O,
                               int32_t G, int32_t K, void* dv, DType dv_t, hipStream_t s);

// Gradient of the preactivations of H = act(pre[:, :F]) * pre[:, F:].
hipError_t launch_gate_grad(const void* dH, const void* pre, DType t, int64_t N, int64_t F, Act act, void* dpre,
                            hipStream_t s);

// Low-rank adapters: D[n][o] = relu?(base[n][o] + residual[n][o] + alpha[a] sum_r (sum_c A[a][r][c] X[n][c]) B[a][o][r]),
// a = rows[n] (outside [0, L): without the third term).
struct AdapterArgs {
  const void* X;
  DType t;
  int64_t N, C, O, L;
  int32_t R;
  const void* A;
  const void* B;
  const float* alpha;
  const int32_t* rows;
  const float* base;     // the shared projection
  const void* residual;  // of D's type, or null; D may be the same memory
  int32_t relu;
  void* D;
  DType d_t;
  float* part;  // workspace of adapter_part_bytes()
};
int64_t adapter_part_bytes(int64_t N, int64_t C, int64_t L, int32_t R);
hipError_t launch_adapters(const AdapterArgs& a, hipStream_t s);

}  // namespace cci
