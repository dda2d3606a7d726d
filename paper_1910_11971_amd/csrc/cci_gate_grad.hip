// Gradient of the preactivations of the gated product H = act(g) u:
//   dg = dH u act'(g),  du = dH act(g).
// Both are rounded to the operands' type: the products behind them, dX and the
// packed gradient, take operands of that type on the matrix cores, and take
// them as they are returned.  (bf16: the products' error is 1.35 times that of
// fp32 dP, two independent roundings; dP in two bf16 parts would double both
// products, 329 and 263 us at 2048 x 4096 <- 8192.)
// Elementwise: 5 elements move per output, and HBM binds.  A lane owns eight
// consecutive outputs (16-byte loads and stores where rows are aligned): 2048
// x 8192 in bf16 32 us, 5.2 TB/s (the GELU 40: its erfc and exp bind there).
#include "cci_act.hpp"
#include "cci_block.hpp"
#include "cci_frag.hpp"

namespace cci {
namespace {

constexpr int kThreads = 256;

template <typename T, Act A>
__global__ __launch_bounds__(kThreads) void gate_grad_kernel(const T* __restrict__ dH, const T* __restrict__ pre,
                                                             int64_t N, int64_t F, uint32_t upr, int64_t units,
                                                             T* __restrict__ dpre) {
  const bool vec = F % 4 == 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t v = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; v < units; v += step) {
    const int64_t n = v / upr;
    const int64_t f = 8 * (v - n * upr), left = F - f;
    Unit<T> h, g, u;
    load_elems<8>(h, dH + n * F + f, left);
    load_elems<8>(g, pre + n * 2 * F + f, left);
    load_elems<8>(u, pre + n * 2 * F + F + f, left);
    T* q = dpre + n * 2 * F + f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float dg[4], du[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = 4 * half + r;
        float a, d;
        act_both<A>(elem(g, e), a, d);
        dg[r] = elem(h, e) * elem(u, e) * d;
        du[r] = elem(h, e) * a;
      }
      store4<T>(q + 4 * half, dg, left - 4 * half, vec);
      store4<T>(q + F + 4 * half, du, left - 4 * half, vec);
    }
  }
}

template <typename T, Act A>
hipError_t launch(const void* dH, const void* pre, int64_t N, int64_t F, void* dpre, hipStream_t s) {
  const int64_t upr = (F + 7) / 8, units = N * upr;
  const int64_t grid = (units + kThreads - 1) / kThreads;
  hipLaunchKernelGGL((gate_grad_kernel<T, A>), dim3(static_cast<uint32_t>(grid < 65536 ? grid : 65536)), dim3(kThreads),
                     0, s, static_cast<const T*>(dH), static_cast<const T*>(pre), N, F, static_cast<uint32_t>(upr), units,
                     static_cast<T*>(dpre));
  return hipGetLastError();
}

template <typename T>
hipError_t typed(const void* dH, const void* pre, int64_t N, int64_t F, Act act, void* dpre, hipStream_t s) {
  switch (act) {
    case Act::RELU: return launch<T, Act::RELU>(dH, pre, N, F, dpre, s);
    case Act::SILU: return launch<T, Act::SILU>(dH, pre, N, F, dpre, s);
    case Act::GELU: return launch<T, Act::GELU>(dH, pre, N, F, dpre, s);
    case Act::GELU_TANH: return launch<T, Act::GELU_TANH>(dH, pre, N, F, dpre, s);
    default: return launch<T, Act::NONE>(dH, pre, N, F, dpre, s);
  }
}

}  // namespace

hipError_t launch_gate_grad(const void* dH, const void* pre, DType t, int64_t N, int64_t F, Act act, void* dpre,
                            hipStream_t s) {
  return t == DType::F32 ? typed<float>(dH, pre, N, F, act, dpre, s) : typed<bf16_t>(dH, pre, N, F, act, dpre, s);
}

}  // namespace cci
