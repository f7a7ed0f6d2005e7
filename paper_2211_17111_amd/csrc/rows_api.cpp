// C ABI of the row operators (bevpool_rows.h): argument validation, workspace
// sizing and dispatch to the HIP launchers.  As in api.cpp, validation runs
// before any HIP call.

#include <hip/hip_runtime_api.h>

#include "bevpool_rows.h"
#include "rows.h"
#include "status.h"

namespace {

using bevpool::fail;
using bevpool::from_hip;
using bevpool::ok;

constexpr int64_t kIndexLimit = int64_t(1) << 31;
constexpr int64_t kMaxC = int64_t(1) << 20;
constexpr int32_t kMaxExperts = 1024;
constexpr int32_t kMaxChosen = 64;

int check_dtype(int dtype, const char* what) {
  if (dtype != BEVPOOL_F32 && dtype != BEVPOOL_F16 && dtype != BEVPOOL_BF16)
    return fail(BEVPOOL_EDTYPE, "unknown %s %d", what, dtype);
  return BEVPOOL_OK;
}

int check_dtypes(int in_dtype, int out_dtype) {
  int st = check_dtype(in_dtype, "in_dtype");
  if (st == BEVPOOL_OK) st = check_dtype(out_dtype, "out_dtype");
  if (st != BEVPOOL_OK) return st;
  if (out_dtype != in_dtype && out_dtype != BEVPOOL_F32)
    return fail(BEVPOOL_EDTYPE, "out_dtype %d is neither in_dtype %d nor float32", out_dtype,
                in_dtype);
  return BEVPOOL_OK;
}

int check_keys(int64_t n, int64_t n_keys) {
  if (n < 0) return fail(BEVPOOL_EINVAL, "n = %lld is negative", (long long)n);
  if (n >= kIndexLimit) return fail(BEVPOOL_EOVERFLOW, "n = %lld exceeds 2^31-1", (long long)n);
  if (n_keys < 1) return fail(BEVPOOL_EINVAL, "n_keys = %lld must be >= 1", (long long)n_keys);
  if (n_keys >= kIndexLimit - 1)
    return fail(BEVPOOL_EOVERFLOW, "n_keys = %lld exceeds 2^31-2", (long long)n_keys);
  return BEVPOOL_OK;
}

int check_key_type(int key_type) {
  if (key_type != BEVPOOL_KEY_I32 && key_type != BEVPOOL_KEY_I64)
    return fail(BEVPOOL_EDTYPE, "unknown key type %d", key_type);
  return BEVPOOL_OK;
}

int check_columns(int64_t C) {
  if (C < 1) return fail(BEVPOOL_EINVAL, "C = %lld must be >= 1", (long long)C);
  if (C > kMaxC) return fail(BEVPOOL_EOVERFLOW, "C = %lld exceeds %lld", (long long)C, (long long)kMaxC);
  return BEVPOOL_OK;
}

int check_stride(int64_t stride, const char* what) {
  if (stride < 0) return fail(BEVPOOL_EINVAL, "%s = %lld is negative", what, (long long)stride);
  return BEVPOOL_OK;
}

// rows x k slots of C elements
int check_slots(int64_t rows, int32_t k, int64_t C) {
  if (rows < 0) return fail(BEVPOOL_EINVAL, "rows = %lld is negative", (long long)rows);
  if (k < 1) return fail(BEVPOOL_EINVAL, "k = %d must be >= 1", k);
  if (rows >= kIndexLimit || rows * k >= kIndexLimit)
    return fail(BEVPOOL_EOVERFLOW, "rows * k = %lld * %d exceeds 2^31-1", (long long)rows, k);
  return check_columns(C);
}

int check_route(int64_t rows, int32_t n_experts, int32_t k, int dtype, int64_t stride) {
  if (n_experts < 1) return fail(BEVPOOL_EINVAL, "n_experts = %d must be >= 1", n_experts);
  if (k < 1 || k > n_experts)
    return fail(BEVPOOL_EINVAL, "k = %d outside [1, n_experts = %d]", k, n_experts);
  if (n_experts > kMaxExperts)
    return fail(BEVPOOL_EOVERFLOW, "n_experts = %d exceeds %d", n_experts, kMaxExperts);
  if (k > kMaxChosen) return fail(BEVPOOL_EOVERFLOW, "k = %d exceeds %d", k, kMaxChosen);
  int st = check_slots(rows, k, 1);
  if (st == BEVPOOL_OK) st = check_dtype(dtype, "dtype");
  if (st == BEVPOOL_OK) st = check_stride(stride, "logits_stride");
  return st;
}

int check_workspace(const void* workspace, size_t bytes, size_t need, const char* what) {
  if (need > 0 && (workspace == nullptr || bytes < need))
    return fail(BEVPOOL_EWORKSPACE, "%s needs %zu workspace bytes, got %zu at %p", what, need,
                bytes, workspace);
  return BEVPOOL_OK;
}

int check_weight_dtype(int weight_dtype, int in_dtype) {
  int st = check_dtype(weight_dtype, "weight_dtype");
  if (st != BEVPOOL_OK) return st;
  if (weight_dtype != in_dtype && weight_dtype != BEVPOOL_F32)
    return fail(BEVPOOL_EDTYPE, "weight_dtype %d is neither in_dtype %d nor float32", weight_dtype,
                in_dtype);
  return BEVPOOL_OK;
}

// A launch holds fewer than 2^24 blocks of 256 threads: the kernels of the
// table's gradient have at most a quarter block per range of slots and 256
// elements of a row, beside those over the table.  (Only the expanded gradient
// of more elements than fit the device's memory comes near.)
int check_embed_grid(int64_t n, int64_t table_rows, int64_t C) {
  const int64_t ranges = bevpool::embed_layout(n, table_rows, C).ranges;
  if (ranges * ((C + 255) / 256) > (int64_t(1) << 24))
    return fail(BEVPOOL_EOVERFLOW, "n * C = %lld * %lld exceeds the gradient's launch", (long long)n,
                (long long)C);
  return BEVPOOL_OK;
}

#define CHECK(call)                        \
  do {                                     \
    const int st_ = (call);                \
    if (st_ != BEVPOOL_OK) return st_;     \
  } while (0)

}  // namespace

extern "C" {

int bevpool_sort_keys_workspace_size(int64_t n, int64_t n_keys, size_t* bytes) {
  CHECK(check_keys(n, n_keys));
  REQUIRE_PTR(bytes);
  *bytes = bevpool::sort_layout(n, n_keys).total;
  return ok();
}

int bevpool_sort_keys(int64_t n, int64_t n_keys, int key_type, const void* keys, int32_t* order,
                      int32_t* position, int32_t* offsets, void* workspace,
                      size_t workspace_bytes, void* stream) {
  CHECK(check_keys(n, n_keys));
  CHECK(check_key_type(key_type));
  if (n > 0) {
    REQUIRE_PTR(keys);
    REQUIRE_PTR(order);
    REQUIRE_PTR(position);
  }
  REQUIRE_PTR(offsets);
  CHECK(check_workspace(workspace, workspace_bytes, bevpool::sort_layout(n, n_keys).total,
                        "sort_keys"));
  return from_hip(bevpool::launch_sort_keys(n, n_keys, key_type, keys, order, position, offsets,
                                            nullptr, workspace, static_cast<hipStream_t>(stream)),
                  "bevpool_sort_keys");
}

int bevpool_route_forward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                          const void* logits, int64_t logits_stride, int renormalise,
                          float* weights, int32_t* ids, void* stream) {
  CHECK(check_route(rows, n_experts, k, dtype, logits_stride));
  if (rows > 0) {
    REQUIRE_PTR(logits);
    REQUIRE_PTR(weights);
    REQUIRE_PTR(ids);
  }
  return from_hip(bevpool::launch_route_forward(rows, n_experts, k, dtype, logits, logits_stride,
                                                renormalise != 0, weights, ids,
                                                static_cast<hipStream_t>(stream)),
                  "bevpool_route_forward");
}

int bevpool_route_backward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                           const float* grad_weights, const void* logits, int64_t logits_stride,
                           const float* weights, const int32_t* ids, int renormalise,
                           void* grad_logits, void* stream) {
  CHECK(check_route(rows, n_experts, k, dtype, logits_stride));
  if (rows > 0) {
    REQUIRE_PTR(grad_weights);
    if (!renormalise) REQUIRE_PTR(logits);
    REQUIRE_PTR(weights);
    REQUIRE_PTR(ids);
    REQUIRE_PTR(grad_logits);
  }
  return from_hip(bevpool::launch_route_backward(rows, n_experts, k, dtype, grad_weights, logits,
                                                 logits_stride, weights, ids, renormalise != 0,
                                                 grad_logits, static_cast<hipStream_t>(stream)),
                  "bevpool_route_backward");
}

int bevpool_dispatch_forward(int64_t rows, int32_t k, int64_t C, int64_t n_keys, int dtype,
                             const void* x, int64_t x_stride, int key_type, const void* ids,
                             int32_t* order, int32_t* position, int32_t* offsets, void* out,
                             void* workspace, size_t workspace_bytes, void* stream) {
  CHECK(check_slots(rows, k, C));
  CHECK(check_keys(rows * k, n_keys));
  CHECK(check_dtype(dtype, "dtype"));
  CHECK(check_key_type(key_type));
  CHECK(check_stride(x_stride, "x_stride"));
  if (rows > 0) {
    REQUIRE_PTR(x);
    REQUIRE_PTR(ids);
    REQUIRE_PTR(order);
    REQUIRE_PTR(position);
    REQUIRE_PTR(out);
  }
  REQUIRE_PTR(offsets);
  CHECK(check_workspace(workspace, workspace_bytes, bevpool::sort_layout(rows * k, n_keys).total,
                        "dispatch_forward"));
  return from_hip(bevpool::launch_dispatch_forward(rows, k, C, n_keys, dtype, x, x_stride, key_type,
                                                   ids, order, position, offsets, out, workspace,
                                                   static_cast<hipStream_t>(stream)),
                  "bevpool_dispatch_forward");
}

int bevpool_dispatch_rows(int64_t rows, int32_t k, int64_t C, int dtype, const void* x,
                          int64_t x_stride, const int32_t* position, const int32_t* kept,
                          void* out, void* stream) {
  CHECK(check_slots(rows, k, C));
  CHECK(check_dtype(dtype, "dtype"));
  CHECK(check_stride(x_stride, "x_stride"));
  if (rows > 0) {
    REQUIRE_PTR(x);
    REQUIRE_PTR(position);
    REQUIRE_PTR(kept);
    REQUIRE_PTR(out);
  }
  return from_hip(bevpool::launch_dispatch_rows(rows, k, C, dtype, x, x_stride, position, kept,
                                                out, static_cast<hipStream_t>(stream)),
                  "bevpool_dispatch_rows");
}

int bevpool_dispatch_backward(int64_t rows, int32_t k, int64_t C, int dtype, const void* grad_out,
                              int64_t grad_stride, const int32_t* position, const int32_t* kept,
                              void* grad_x, void* stream) {
  CHECK(check_slots(rows, k, C));
  CHECK(check_dtype(dtype, "dtype"));
  CHECK(check_stride(grad_stride, "grad_stride"));
  if (rows > 0) {
    REQUIRE_PTR(grad_out);
    REQUIRE_PTR(position);
    REQUIRE_PTR(kept);
    REQUIRE_PTR(grad_x);
  }
  return from_hip(bevpool::launch_combine_forward(rows, k, C, dtype, dtype, BEVPOOL_F32, grad_out,
                                                  grad_stride, nullptr, position, kept, grad_x,
                                                  static_cast<hipStream_t>(stream)),
                  "bevpool_dispatch_backward");
}

int bevpool_combine_forward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                            int weight_dtype, const void* in, int64_t in_stride,
                            const void* weights, const int32_t* position, const int32_t* kept,
                            void* out, void* stream) {
  CHECK(check_slots(rows, k, C));
  CHECK(check_dtypes(in_dtype, out_dtype));
  CHECK(check_weight_dtype(weight_dtype, in_dtype));
  CHECK(check_stride(in_stride, "in_stride"));
  if (rows > 0) {
    REQUIRE_PTR(in);
    REQUIRE_PTR(weights);
    REQUIRE_PTR(position);
    REQUIRE_PTR(kept);
    REQUIRE_PTR(out);
  }
  return from_hip(bevpool::launch_combine_forward(rows, k, C, in_dtype, out_dtype, weight_dtype,
                                                  in, in_stride, weights, position, kept, out,
                                                  static_cast<hipStream_t>(stream)),
                  "bevpool_combine_forward");
}

int bevpool_combine_backward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                             int weight_dtype, const void* grad_out, int64_t grad_stride,
                             const void* in, int64_t in_stride, const void* weights,
                             const int32_t* position, const int32_t* kept, void* grad_in,
                             void* grad_weights, void* stream) {
  CHECK(check_slots(rows, k, C));
  CHECK(check_dtypes(in_dtype, out_dtype));
  CHECK(check_weight_dtype(weight_dtype, in_dtype));
  CHECK(check_stride(grad_stride, "grad_stride"));
  CHECK(check_stride(in_stride, "in_stride"));
  if (rows > 0) {
    REQUIRE_PTR(grad_out);
    if (grad_weights != nullptr) REQUIRE_PTR(in);
    if (grad_in != nullptr) REQUIRE_PTR(weights);
    REQUIRE_PTR(position);
    REQUIRE_PTR(kept);
  }
  return from_hip(bevpool::launch_combine_backward(rows, k, C, in_dtype, out_dtype, weight_dtype,
                                                   grad_out, grad_stride, in, in_stride, weights,
                                                   position, kept, grad_in, grad_weights,
                                                   static_cast<hipStream_t>(stream)),
                  "bevpool_combine_backward");
}

int bevpool_embed_forward(int64_t n, int64_t table_rows, int64_t C, int in_dtype, int out_dtype,
                          const void* table, int64_t table_stride, int key_type, const void* ids,
                          float scale, void* out, void* stream) {
  CHECK(check_keys(n, table_rows));
  CHECK(check_columns(C));
  CHECK(check_dtypes(in_dtype, out_dtype));
  CHECK(check_key_type(key_type));
  CHECK(check_stride(table_stride, "table_stride"));
  if (n > 0) {
    REQUIRE_PTR(table);
    REQUIRE_PTR(ids);
    REQUIRE_PTR(out);
  }
  return from_hip(bevpool::launch_embed_forward(n, table_rows, C, in_dtype, out_dtype, table,
                                                table_stride, key_type, ids, scale, out,
                                                static_cast<hipStream_t>(stream)),
                  "bevpool_embed_forward");
}

int bevpool_embed_backward_workspace_size(int64_t n, int64_t table_rows, int64_t C,
                                          size_t* bytes) {
  CHECK(check_keys(n, table_rows));
  CHECK(check_columns(C));
  CHECK(check_embed_grid(n, table_rows, C));
  REQUIRE_PTR(bytes);
  *bytes = bevpool::embed_layout(n, table_rows, C).total;
  return ok();
}

int bevpool_embed_backward(int64_t n, int64_t table_rows, int64_t C, int in_dtype, int out_dtype,
                           const void* grad_out, int64_t grad_stride, int key_type,
                           const void* ids, float scale, void* grad_table, void* workspace,
                           size_t workspace_bytes, void* stream) {
  CHECK(check_keys(n, table_rows));
  CHECK(check_columns(C));
  CHECK(check_embed_grid(n, table_rows, C));
  if (in_dtype == BEVPOOL_F32)
    CHECK(check_dtype(out_dtype, "out_dtype"));
  else
    CHECK(check_dtypes(in_dtype, out_dtype));
  CHECK(check_key_type(key_type));
  CHECK(check_stride(grad_stride, "grad_stride"));
  if (n > 0) {
    REQUIRE_PTR(grad_out);
    REQUIRE_PTR(ids);
  }
  REQUIRE_PTR(grad_table);
  CHECK(check_workspace(workspace, workspace_bytes,
                        bevpool::embed_layout(n, table_rows, C).total, "embed_backward"));
  return from_hip(bevpool::launch_embed_backward(n, table_rows, C, in_dtype, out_dtype, grad_out,
                                                 grad_stride, key_type, ids, scale, grad_table,
                                                 workspace, static_cast<hipStream_t>(stream)),
                  "bevpool_embed_backward");
}

}  // extern "C"
