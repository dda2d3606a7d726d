// Drives the feed-forward block's entry points through their validation and
// choice of kernels (valid calls reach the stand-ins, invalid ones must fail
// before them) in a build with AddressSanitizer and
// UndefinedBehaviorSanitizer.  Exit status 0 and "block driver ok" on success.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <vector>

#include "../../include/cci.h"

extern int g_block_launches;
extern int g_fail_at;

namespace cci {
// (cci_api.cpp's error state)
static char message[512];
cci_status fail(cci_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(message, sizeof message, fmt, ap);
  va_end(ap);
  return s;
}
cci_status ok() {
  message[0] = '\0';
  return CCI_OK;
}
}  // namespace cci

static int failures = 0;
#define EXPECT(cond)                                                   \
  do {                                                                 \
    if (!(cond)) {                                                     \
      std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond);  \
      ++failures;                                                      \
    }                                                                  \
  } while (0)

alignas(16) static unsigned char buf[1 << 12];

int main() {
  void* P = buf;
  const uint8_t* I = buf;
  float* F = reinterpret_cast<float*>(buf);
  size_t n = 0;
  int before = g_block_launches;
  // every size goes through the choice of kernels without overflow, and reaches one launcher
  int calls = 0;
  for (int64_t N : {1, 31, 33, 100, 4096, 1 << 20})
    for (int64_t C : {1, 8, 1000, 4096, 1 << 20})
      for (int64_t f : {16, 4096, 1 << 19})
        for (cci_dtype t : {CCI_F32, CCI_BF16}) {
          EXPECT(cci_gated_spmm(P, t, N, C, P, I, f, 16, 4, CCI_ACT_SILU, P, nullptr, nullptr) == CCI_OK);
          EXPECT(cci_spmm_t(P, t, N, 2 * f, P, I, C, 16, 4, P, t, nullptr) == CCI_OK);
          calls += 2;
        }
  EXPECT(g_block_launches - before == calls);
  before = g_block_launches;
  EXPECT(cci_layernorm(P, CCI_BF16, 4, 8, F, nullptr, 0.0f, P, F, F, nullptr) == CCI_OK);
  EXPECT(cci_gated_spmm_bwd(P, P, P, CCI_BF16, 40, 8, P, I, 16, 8, 2, CCI_ACT_GELU, P, P, P, CCI_F32, nullptr) == CCI_OK);
  EXPECT(g_block_launches - before == 4);
  before = g_block_launches;
  EXPECT(cci_gated_spmm_bwd(P, P, nullptr, CCI_F32, 4, 8, P, I, 16, 8, 2, CCI_ACT_RELU, P, P, nullptr, CCI_F32, nullptr) == CCI_OK);
  EXPECT(cci_gated_spmm_bwd(nullptr, nullptr, nullptr, CCI_F32, 0, 8, nullptr, I, 16, 8, 2, CCI_ACT_NONE, nullptr,
                            nullptr, P, CCI_F32, nullptr) == CCI_OK);
  EXPECT(g_block_launches - before == 3);
  // workspaces: of exactly the size that is asked for, at their own sizes and one byte short
  for (int64_t N : {0, 1, 3, 100}) {
    EXPECT(cci_layernorm_bwd_workspace(N, 9, &n) == CCI_OK);
    std::vector<float> ws(n / 4 + 4);
    EXPECT(cci_layernorm_bwd(P, P, CCI_F32, N, 9, nullptr, F, F, P, F, F, ws.data(), n, nullptr) == CCI_OK);
    if (n > 0) EXPECT(cci_layernorm_bwd(P, P, CCI_F32, N, 9, nullptr, F, F, P, F, F, ws.data(), n - 1, nullptr) == CCI_EINVAL);
  }
  const cci_epilogue ep{F, F, P, 1};
  for (cci_dtype y : {CCI_BF16, CCI_F32})
    for (int64_t C : {8, 9}) {  // cci_spmm, and the tile kernels
      cci_adapters ad{P, P, F, reinterpret_cast<const int32_t*>(P), 3, 5};
      EXPECT(cci_spmm_adapters_workspace(7, C, 16, 3, 5, y, &n) == CCI_OK);
      char* ws = static_cast<char*>(aligned_alloc(16, (n + 15) / 16 * 16));
      before = g_block_launches;
      EXPECT(cci_spmm_adapters(P, CCI_BF16, 7, C, P, CCI_BF16, I, 16, 8, 2, &ad, &ep, P, y, ws, n, nullptr) == CCI_OK);
      EXPECT(cci_spmm_adapters(P, CCI_BF16, 7, C, P, CCI_BF16, I, 15, 3, 2, &ad, nullptr, P, y, ws, n, nullptr) == CCI_OK);
      EXPECT(g_block_launches - before == 4);
      EXPECT(cci_spmm_adapters(P, CCI_BF16, 7, C, P, CCI_BF16, I, 16, 8, 2, &ad, &ep, P, y, ws, n - 1, nullptr) == CCI_EINVAL);
      free(ws);
    }
  // a launch that fails ends the call with its error
  for (int at : {1, 2, 3}) {
    g_fail_at = at;
    EXPECT(cci_gated_spmm_bwd(P, P, P, CCI_BF16, 40, 8, P, I, 16, 8, 2, CCI_ACT_SILU, P, P, P, CCI_BF16, nullptr) == CCI_EHIP);
    EXPECT(g_fail_at == 0 && std::strlen(cci::message) > 0);
  }
  // refused before any launch
  before = g_block_launches;
  EXPECT(cci_layernorm(P, CCI_F32, 4, 8, nullptr, nullptr, NAN, P, nullptr, nullptr, nullptr) == CCI_EINVAL);
  EXPECT(cci_layernorm(P, CCI_F32, INT64_MAX, INT64_MAX, nullptr, nullptr, 1.0f, P, nullptr, nullptr, nullptr) == CCI_EINVAL);
  EXPECT(cci_layernorm_bwd_workspace(INT64_MAX / 2, 1 << 20, &n) == CCI_EINVAL);
  EXPECT(cci_gated_spmm(P, CCI_BF16, 4, 8, P, I, INT64_MAX / 8 * 8, 8, 2, CCI_ACT_SILU, P, nullptr, nullptr) == CCI_EINVAL);
  EXPECT(cci_gated_spmm(P, CCI_BF16, 4, (1 << 20) + 1, P, I, 16, 8, 2, CCI_ACT_SILU, P, nullptr, nullptr) == CCI_EINVAL);
  EXPECT(cci_gated_spmm(P, CCI_BF16, 4, 8, P, I, (1 << 19) + 8, 8, 2, CCI_ACT_SILU, P, nullptr, nullptr) == CCI_EINVAL);
  EXPECT(cci_spmm_t(P, CCI_BF16, INT64_MAX, 16, P, I, 8, 8, 2, P, CCI_BF16, nullptr) == CCI_EINVAL);
  EXPECT(cci_spmm_adapters_workspace(INT64_MAX, 8, 16, 3, 5, CCI_BF16, &n) == CCI_EINVAL);
  EXPECT(cci_spmm_adapters_workspace(4, 8, 16, INT64_MAX, 5, CCI_BF16, &n) == CCI_EINVAL);
  EXPECT(g_block_launches == before);
  if (failures) return 1;
  std::printf("block driver ok\n");
  return 0;
}
