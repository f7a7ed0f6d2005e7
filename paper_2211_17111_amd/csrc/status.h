// Status reporting shared by the C ABI's translation units.
#pragma once

#include <hip/hip_runtime_api.h>

#include "bevpool.h"

namespace bevpool {

// Records a message for the calling thread (bevpool_last_error) and returns status.
int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears the message and returns BEVPOOL_OK.
int ok();
// BEVPOOL_OK, or BEVPOOL_ELAUNCH with the HIP error's name.
int from_hip(hipError_t e, const char* what);

}  // namespace bevpool

#define REQUIRE_PTR(p)                                                           \
  do {                                                                           \
    if ((p) == nullptr) return bevpool::fail(BEVPOOL_EINVAL, #p " is NULL");     \
  } while (0)
