// C ABI of the logits operators (bevpool_logits.h): argument validation,
// workspace sizing and dispatch to the HIP launchers.  As in api.cpp,
// validation runs before any HIP call.

#include <hip/hip_runtime_api.h>

#include <cmath>

#include "bevpool_logits.h"
#include "checks.h"
#include "logits.h"

namespace {

using bevpool::check_dtype;
using bevpool::check_key_type;
using bevpool::check_stride;
using bevpool::check_workspace;
using bevpool::fail;
using bevpool::from_hip;
using bevpool::ok;

constexpr int64_t kMaxV = int64_t(1) << 20;

int check_sizes(int64_t rows, int64_t V, int32_t k, int32_t k_least, int32_t k_most, int dtype) {
  if (rows < 0) return fail(BEVPOOL_EINVAL, "rows = %lld is negative", (long long)rows);
  if (rows >= bevpool::kIndexLimit)
    return fail(BEVPOOL_EOVERFLOW, "rows = %lld exceeds 2^31-1", (long long)rows);
  if (V < 1) return fail(BEVPOOL_EINVAL, "V = %lld must be >= 1", (long long)V);
  if (V > kMaxV)
    return fail(BEVPOOL_EOVERFLOW, "V = %lld exceeds %lld", (long long)V, (long long)kMaxV);
  if (k < k_least || k > V)
    return fail(BEVPOOL_EINVAL, "k = %d outside [%d, V = %lld]", k, k_least, (long long)V);
  if (k > k_most) return fail(BEVPOOL_EOVERFLOW, "k = %d exceeds %d", k, k_most);
  return check_dtype(dtype, "dtype");
}

int check_logprobs(int64_t rows, int64_t V, int32_t k, int dtype) {
  return check_sizes(rows, V, k, 0, bevpool::kMaxAlternatives, dtype);
}

int check_distill(int64_t rows, int64_t V, int32_t k, int dtype) {
  return check_sizes(rows, V, k, 1, bevpool::kMaxTaught, dtype);
}

int check_rows(int64_t stride, float scale, int key_type) {
  CHECK(check_stride(stride, "logits_stride"));
  if (!(scale > 0.f) || !std::isfinite(scale))
    return fail(BEVPOOL_EINVAL, "scale = %g must be positive and finite", scale);
  if (!std::isfinite(bevpool::exponent_factor(scale)))
    return fail(BEVPOOL_EINVAL, "scale = %g: scale log2 e exceeds float32", scale);
  return check_key_type(key_type);
}

bevpool::LogitsRows rows_of(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                            int64_t stride, float scale, int key_type, const void* ids,
                            const float* teacher = nullptr, int renormalise = 0) {
  return bevpool::LogitsRows{rows,       stride, logits, ids,      teacher,         scale,
                             (int32_t)V, k,      dtype,  key_type, renormalise != 0};
}

}  // namespace

extern "C" {

int bevpool_logprobs_workspace_size(int64_t rows, int64_t V, int32_t k, int dtype, size_t* bytes) {
  CHECK(check_logprobs(rows, V, k, dtype));
  REQUIRE_PTR(bytes);
  *bytes = bevpool::logprobs_workspace(rows, V, k, dtype);
  return ok();
}

int bevpool_logprobs_forward(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                             int64_t logits_stride, float scale, int key_type, const void* ids,
                             float* stats, float* logprob, float* lse, float* entropy, float* top,
                             int32_t* top_ids, void* workspace, size_t workspace_bytes,
                             void* stream) {
  CHECK(check_logprobs(rows, V, k, dtype));
  CHECK(check_rows(logits_stride, scale, key_type));
  if (rows > 0) {
    REQUIRE_PTR(logits);
    REQUIRE_PTR(stats);
    if (logprob != nullptr) REQUIRE_PTR(ids);
    if (k > 0) {
      REQUIRE_PTR(top);
      REQUIRE_PTR(top_ids);
    }
  }
  CHECK(check_workspace(workspace, workspace_bytes,
                        bevpool::logprobs_workspace(rows, V, k, dtype), "logprobs_forward"));
  return from_hip(
      bevpool::launch_logprobs_forward(
          rows_of(rows, V, k, dtype, logits, logits_stride, scale, key_type, ids),
          bevpool::LogprobsOut{stats, logprob, lse, entropy, top, top_ids}, workspace,
          static_cast<hipStream_t>(stream)),
      "bevpool_logprobs_forward");
}

int bevpool_logprobs_backward(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                              int64_t logits_stride, float scale, int key_type, const void* ids,
                              const float* stats, const float* entropy, const int32_t* top_ids,
                              const float* grad_logprob, const float* grad_lse,
                              const float* grad_entropy, const float* grad_top, void* grad_logits,
                              void* stream) {
  CHECK(check_logprobs(rows, V, k, dtype));
  CHECK(check_rows(logits_stride, scale, key_type));
  if (rows > 0) {
    REQUIRE_PTR(logits);
    REQUIRE_PTR(stats);
    REQUIRE_PTR(grad_logits);
    if (grad_logprob != nullptr) REQUIRE_PTR(ids);
    if (grad_entropy != nullptr) REQUIRE_PTR(entropy);
    if (k > 0 && grad_top != nullptr) REQUIRE_PTR(top_ids);
  }
  return from_hip(
      bevpool::launch_logprobs_backward(
          rows_of(rows, V, k, dtype, logits, logits_stride, scale, key_type, ids),
          bevpool::LogprobsGrads{stats, entropy, top_ids, grad_logprob, grad_lse, grad_entropy,
                                 k > 0 ? grad_top : nullptr},
          grad_logits, static_cast<hipStream_t>(stream)),
      "bevpool_logprobs_backward");
}

int bevpool_distill_workspace_size(int64_t rows, int64_t V, int32_t k, int dtype, size_t* bytes) {
  CHECK(check_distill(rows, V, k, dtype));
  REQUIRE_PTR(bytes);
  *bytes = bevpool::distill_workspace(rows, V, k, dtype);
  return ok();
}

int bevpool_distill_forward(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                            int64_t logits_stride, float scale, int key_type, const void* ids,
                            const float* teacher, int renormalise, float* loss, float* stats,
                            void* workspace, size_t workspace_bytes, void* stream) {
  CHECK(check_distill(rows, V, k, dtype));
  CHECK(check_rows(logits_stride, scale, key_type));
  if (rows > 0) {
    REQUIRE_PTR(logits);
    REQUIRE_PTR(ids);
    REQUIRE_PTR(teacher);
    REQUIRE_PTR(loss);
    REQUIRE_PTR(stats);
  }
  CHECK(check_workspace(workspace, workspace_bytes, bevpool::distill_workspace(rows, V, k, dtype),
                        "distill_forward"));
  return from_hip(bevpool::launch_distill_forward(
                      rows_of(rows, V, k, dtype, logits, logits_stride, scale, key_type, ids,
                              teacher, renormalise),
                      loss, stats, workspace, static_cast<hipStream_t>(stream)),
                  "bevpool_distill_forward");
}

int bevpool_distill_backward(int64_t rows, int64_t V, int32_t k, int dtype, const float* grad_loss,
                             const void* logits, int64_t logits_stride, float scale, int key_type,
                             const void* ids, const float* teacher, int renormalise,
                             const float* stats, void* grad_logits, void* stream) {
  CHECK(check_distill(rows, V, k, dtype));
  CHECK(check_rows(logits_stride, scale, key_type));
  if (rows > 0) {
    REQUIRE_PTR(grad_loss);
    REQUIRE_PTR(logits);
    REQUIRE_PTR(ids);
    REQUIRE_PTR(teacher);
    REQUIRE_PTR(stats);
    REQUIRE_PTR(grad_logits);
  }
  return from_hip(bevpool::launch_distill_backward(
                      rows_of(rows, V, k, dtype, logits, logits_stride, scale, key_type, ids,
                              teacher, renormalise),
                      grad_loss, stats, grad_logits, static_cast<hipStream_t>(stream)),
                  "bevpool_distill_backward");
}

int bevpool_distill_step(int64_t rows, int64_t V, int32_t k, int dtype, const float* grad_loss,
                         const void* logits, int64_t logits_stride, float scale, int key_type,
                         const void* ids, const float* teacher, int renormalise, float* loss,
                         float* stats, void* grad_logits, void* workspace, size_t workspace_bytes,
                         void* stream) {
  CHECK(check_distill(rows, V, k, dtype));
  CHECK(check_rows(logits_stride, scale, key_type));
  if (rows > 0) {
    REQUIRE_PTR(grad_loss);
    REQUIRE_PTR(logits);
    REQUIRE_PTR(ids);
    REQUIRE_PTR(teacher);
    REQUIRE_PTR(loss);
    REQUIRE_PTR(stats);
    REQUIRE_PTR(grad_logits);
  }
  CHECK(check_workspace(workspace, workspace_bytes, bevpool::distill_workspace(rows, V, k, dtype),
                        "distill_step"));
  return from_hip(bevpool::launch_distill_step(
                      rows_of(rows, V, k, dtype, logits, logits_stride, scale, key_type, ids,
                              teacher, renormalise),
                      grad_loss, loss, stats, grad_logits, workspace,
                      static_cast<hipStream_t>(stream)),
                  "bevpool_distill_step");
}

}  // extern "C"
