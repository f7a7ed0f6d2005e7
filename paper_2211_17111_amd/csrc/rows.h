// Internal interface between the row operators' C ABI (rows_api.cpp) and
// their HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "bevpool_rows.h"

namespace bevpool {

// Sort of n keys: `passes` radix passes of at most kSortBits bits over the
// keys 0 .. n_keys (n_keys = dropped).
constexpr int kSortBits = 10;
constexpr int kSortTile = 1024;
// Most slots that one workgroup sorts, in one pass and in several.
constexpr int kSmallSort = 4096, kSmallSortPasses = 8192;
struct SortLayout {
  size_t tile_counts, group_counts, totals;  // int32[digits] per tile, per group, in all
  size_t keys[2], vals[2];                   // int32[n] each, with several passes
  size_t total;                              // bytes
  int64_t tiles, groups;
  int bits, passes, digit_bits;
  bool small;  // one workgroup
};
SortLayout sort_layout(int64_t n, int64_t n_keys);

// position and sorted_keys (n_keys for a dropped slot) may be NULL, and offsets
// with several passes.
hipError_t launch_sort_keys(int64_t n, int64_t n_keys, int key_type, const void* keys,
                            int32_t* order, int32_t* position, int32_t* offsets,
                            int32_t* sorted_keys, void* workspace, hipStream_t stream);

hipError_t launch_route_forward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                                const void* logits, int64_t stride, bool renormalise,
                                float* weights, int32_t* ids, hipStream_t stream);
hipError_t launch_route_backward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                                 const float* grad_weights, const void* logits, int64_t stride,
                                 const float* weights, const int32_t* ids, bool renormalise,
                                 void* grad_logits, hipStream_t stream);

hipError_t launch_dispatch_forward(int64_t rows, int32_t k, int64_t C, int64_t n_keys, int dtype,
                                   const void* x, int64_t x_stride, int key_type, const void* ids,
                                   int32_t* order, int32_t* position, int32_t* offsets, void* out,
                                   void* workspace, hipStream_t stream);
hipError_t launch_dispatch_rows(int64_t rows, int32_t k, int64_t C, int dtype, const void* x,
                                int64_t x_stride, const int32_t* position, const int32_t* kept,
                                void* out, hipStream_t stream);
// weights may be NULL: every weight 1 (the dispatch's gradient).
hipError_t launch_combine_forward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                                  int weight_dtype, const void* in, int64_t in_stride,
                                  const void* weights, const int32_t* position,
                                  const int32_t* kept, void* out, hipStream_t stream);
hipError_t launch_combine_backward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                                   int weight_dtype, const void* grad_out, int64_t grad_stride,
                                   const void* in, int64_t in_stride, const void* weights,
                                   const int32_t* position, const int32_t* kept, void* grad_in,
                                   void* grad_weights, hipStream_t stream);

size_t layer_workspace(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts, int dtype);
hipError_t launch_expert_layer(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts,
                               int dtype, int weight_dtype, const void* x, int64_t x_stride,
                               const void* up, const void* down, const void* weights,
                               const int32_t* ids, void* out, void* workspace,
                               hipStream_t stream);

hipError_t launch_embed_forward(int64_t n, int64_t table_rows, int64_t C, int in_dtype,
                                int out_dtype, const void* table, int64_t table_stride,
                                int key_type, const void* ids, float scale, void* out,
                                hipStream_t stream);
struct EmbedLayout {
  size_t sort;                      // workspace of the sort
  size_t order, keys, offsets;  // int32[n], int32[n], int32[table_rows + 1]
  size_t partials;              // float[2 * ranges][C]
  size_t total;
  int64_t ranges;  // of RG sorted slots
  int32_t RG;
};
EmbedLayout embed_layout(int64_t n, int64_t table_rows, int64_t C);
hipError_t launch_embed_backward(int64_t n, int64_t table_rows, int64_t C, int in_dtype,
                                 int out_dtype, const void* grad_out, int64_t grad_stride,
                                 int key_type, const void* ids, float scale, void* grad_table,
                                 void* workspace, hipStream_t stream);

}  // namespace bevpool
