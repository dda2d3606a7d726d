// Argument checks and error reporting shared by the files of the C ABI layer.
#pragma once

#include <stdint.h>

#include "../../include/cci.h"
#include "cci_launch.hpp"

namespace cci {

// Records the message of a failed call on the calling thread and returns its
// status; ok() clears the message.  (Defined in cci_api.cpp.)
cci_status fail(cci_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
cci_status ok();

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool dtype_ok(cci_dtype t) { return t == CCI_F32 || t == CCI_BF16; }

inline DType to_dt(cci_dtype t) { return t == CCI_F32 ? DType::F32 : DType::BF16; }

inline size_t dsize(cci_dtype t) { return t == CCI_F32 ? 4 : 2; }

inline cci_status check_groups(int64_t O, int64_t C, int32_t G, int32_t K) {
  if (G < 1 || G > 256) return fail(CCI_EINVAL, "G=%d outside [1, 256]", G);
  if (K < 1 || K > G) return fail(CCI_EINVAL, "K=%d outside [1, G=%d]", K, G);
  if (O < 1 || O % G != 0) return fail(CCI_EINVAL, "O=%lld is not a positive multiple of G=%d", (long long)O, G);
  if (C < 1) return fail(CCI_EINVAL, "C=%lld < 1", (long long)C);
  // packed arrays and grids are indexed with 64-bit offsets; keep element
  // counts well inside what the launch grids can cover
  if (O > (int64_t(1) << 31) || C > (int64_t(1) << 31) || O * C > (int64_t(1) << 40))
    return fail(CCI_EINVAL, "O*C too large");
  return CCI_OK;
}

}  // namespace cci
