// Checks of arguments that the calls on logits share (not part of the C ABI).
#pragma once
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "../../include/tfe.h"
#include "tfe_internal.h"

#define NEED(cond, ...)                                          \
  do {                                                           \
    if (!(cond)) return fail(TFE_ERR_INVALID_ARG, __VA_ARGS__);  \
  } while (0)
#define TRY(call)                      \
  do {                                 \
    const tfe_status st_ = (call);     \
    if (st_ != TFE_OK) return st_;     \
  } while (0)

namespace tfe {

inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline uintptr_t elem(int32_t dtype) { return dtype == TFE_BF16 ? 2 : 4; }

inline tfe_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return TFE_OK;
  return fail(TFE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// A matrix argument of `rows` rows of `cols` elements, `ld` apart.
inline tfe_status matrix(const void* p, int32_t dtype, int64_t ld, int64_t rows, int64_t cols,
                  const char* what) {
  NEED(dtype == TFE_F32 || dtype == TFE_BF16, "%s: unknown dtype %d", what, dtype);
  NEED(ld >= cols, "%s: pitch %lld below the row's %lld elements", what, (long long)ld,
       (long long)cols);
  NEED(ld < ((int64_t)1 << 31), "%s: pitch above 2^31", what);
  if (rows == 0) return TFE_OK;
  NEED(p, "%s: null", what);
  NEED(aligned(p, elem(dtype)), "%s: not aligned to its elements", what);
  return TFE_OK;
}

inline tfe_status space(const void* p, int64_t bytes, int64_t need) {
  if (need == 0) return TFE_OK;
  NEED(p, "null workspace");
  NEED(aligned(p, 16), "workspace not 16-byte aligned");
  NEED(bytes >= need, "workspace of %lld bytes, %lld needed", (long long)bytes, (long long)need);
  return TFE_OK;
}

}  // namespace tfe
