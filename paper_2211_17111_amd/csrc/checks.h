// Argument checks shared by the C entries of the row and logits operators.
#pragma once

#include <stdint.h>

#include "bevpool_rows.h"
#include "status.h"

namespace bevpool {

constexpr int64_t kIndexLimit = int64_t(1) << 31;

inline int check_dtype(int dtype, const char* what) {
  if (dtype != BEVPOOL_F32 && dtype != BEVPOOL_F16 && dtype != BEVPOOL_BF16)
    return fail(BEVPOOL_EDTYPE, "unknown %s %d", what, dtype);
  return BEVPOOL_OK;
}

inline int check_key_type(int key_type) {
  if (key_type != BEVPOOL_KEY_I32 && key_type != BEVPOOL_KEY_I64)
    return fail(BEVPOOL_EDTYPE, "unknown key type %d", key_type);
  return BEVPOOL_OK;
}

inline int check_stride(int64_t stride, const char* what) {
  if (stride < 0) return fail(BEVPOOL_EINVAL, "%s = %lld is negative", what, (long long)stride);
  return BEVPOOL_OK;
}

inline int check_workspace(const void* workspace, size_t bytes, size_t need, const char* what) {
  if (need > 0 && (workspace == nullptr || bytes < need))
    return fail(BEVPOOL_EWORKSPACE, "%s needs %zu workspace bytes, got %zu at %p", what, need,
                bytes, workspace);
  return BEVPOOL_OK;
}

}  // namespace bevpool

#define CHECK(call)                        \
  do {                                     \
    const int st_ = (call);                \
    if (st_ != BEVPOOL_OK) return st_;     \
  } while (0)
