// Embedding lookup with a scale, and the table's gradient: the rows of each id
// summed through the ids' stable order, so that every table row is written
// once, by one owner, without atomics.  Bound by memory: the forward by the
// rows it writes, the gradient by the table it fills.

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

template <typename T, typename TO, typename TKey>
__global__ __launch_bounds__(kRowThreads) void k_embed(const T* __restrict__ table, int64_t stride,
                                                       RowSplit s, const TKey* __restrict__ ids,
                                                       int32_t table_rows, float scale,
                                                       TO* __restrict__ out) {
  constexpr int N = RowVec<T>::N;
  for_row_vectors<N>(s, [&](int64_t i, int32_t c) {
    const int32_t id = key_or_drop(ids, i, table_rows);
    const int left = s.C - c;
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = 0.f;
    if (id < table_rows) {
      load_row<T>(table + id * stride + c, left, v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= scale;
    }
    store_row<TO>(out + i * s.C + c, left, v);
  });
}

template <typename T, typename TO>
__global__ __launch_bounds__(kRowThreads) void k_embed_backward(
    const T* __restrict__ grad_out, int64_t stride, RowSplit s, int64_t n,
    const int32_t* __restrict__ order, const int32_t* __restrict__ offsets, float scale,
    TO* __restrict__ grad_table) {
  constexpr int N = RowVec<T>::N;
  for_row_vectors<N>(s, [&](int64_t v, int32_t c) {
    const int left = s.C - c;
    const int32_t end = offsets[v + 1];
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    for (int32_t q = offsets[v]; q < end; ++q) {
      float g[N];
      load_row<T>(grad_out + order[q] * stride + c, left, g);
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += g[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] *= scale;
    store_row<TO>(grad_table + v * s.C + c, left, acc);
  });
}

}  // namespace

hipError_t launch_embed_forward(int64_t n, int64_t table_rows, int64_t C, int in_dtype,
                                int out_dtype, const void* table, int64_t table_stride,
                                int key_type, const void* ids, float scale, void* out,
                                hipStream_t stream) {
  if (n == 0) return hipSuccess;
  by_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    const RowSplit s = row_split(n, C, RowVec<T>::N);
    auto go = [&](auto* keys) {
      k_embed<T, TO><<<row_grid(s), kRowThreads, 0, stream>>>(
          static_cast<const T*>(table), table_stride, s, keys, (int32_t)table_rows, scale,
          static_cast<TO*>(out));
    };
    if (key_type == BEVPOOL_KEY_I64) go(static_cast<const int64_t*>(ids));
    else go(static_cast<const int32_t*>(ids));
  });
  return hipGetLastError();
}

EmbedLayout embed_layout(int64_t n, int64_t table_rows, int64_t C) {
  (void)C;
  EmbedLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  L.sort = take(sort_layout(n, table_rows).total);
  L.order = take(sizeof(int32_t) * (size_t)n);
  L.position = take(sizeof(int32_t) * (size_t)n);
  L.offsets = take(sizeof(int32_t) * (size_t)(table_rows + 1));
  L.total = off;
  return L;
}

hipError_t launch_embed_backward(int64_t n, int64_t table_rows, int64_t C, int in_dtype,
                                 int out_dtype, const void* grad_out, int64_t grad_stride,
                                 int key_type, const void* ids, float scale, void* grad_table,
                                 void* workspace, hipStream_t stream) {
  const EmbedLayout L = embed_layout(n, table_rows, C);
  char* ws = static_cast<char*>(workspace);
  int32_t* order = reinterpret_cast<int32_t*>(ws + L.order);
  int32_t* position = reinterpret_cast<int32_t*>(ws + L.position);
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + L.offsets);
  const hipError_t e = launch_sort_keys(n, table_rows, key_type, ids, order, position, offsets,
                                        ws + L.sort, stream);
  if (e != hipSuccess) return e;
  by_any_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    const RowSplit s = row_split(table_rows, C, RowVec<T>::N);
    k_embed_backward<T, TO><<<row_grid(s), kRowThreads, 0, stream>>>(
        static_cast<const T*>(grad_out), grad_stride, s, n, order, offsets, scale,
        static_cast<TO*>(grad_table));
  });
  return hipGetLastError();
}

}  // namespace bevpool
