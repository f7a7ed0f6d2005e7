// Rows of float32, float16 or bfloat16 elements in 16-byte vectors, whatever
// their alignment, and the work split of kernels that run over (row, vector).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "bevpool_rows.h"
#include "device_utils.h"
#include "vec.h"

namespace bevpool {

typedef __bf16 bf16_t;

// A row of C elements begins wherever the caller's stride and C put it, so a
// vector is only as aligned as its element; the compiler then still emits one
// 16-byte access (the hardware takes any element alignment), and a row's
// last C % N elements go one by one.
template <typename T>
struct RowVec;
template <>
struct RowVec<float> {
  static constexpr int N = 4;
  typedef float type __attribute__((ext_vector_type(4), aligned(4)));
  typedef type four;
};
template <>
struct RowVec<half_t> {
  static constexpr int N = 8;
  typedef _Float16 type __attribute__((ext_vector_type(8), aligned(2)));
  typedef _Float16 four __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct RowVec<bf16_t> {
  static constexpr int N = 8;
  typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2)));
  typedef __bf16 four __attribute__((ext_vector_type(4), aligned(2)));
};

// v[0 .. M) = p[0 .. left), zeros past `left`.
template <typename T, int M>
__device__ __forceinline__ void load_row(const T* p, int left, float (&v)[M]) {
  using V = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N;
  static_assert(M % N == 0, "whole vectors");
  if (left >= M) {
#pragma unroll
    for (int b = 0; b < M; b += N) {
      const V t = *reinterpret_cast<const V*>(p + b);
#pragma unroll
      for (int e = 0; e < N; ++e) v[b + e] = (float)t[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < M; ++e) v[e] = e < left ? (float)p[e] : 0.f;
  }
}

// The vector at p as it is, zeros past `left`.  STREAM: the line is not wanted
// again (a hint to the caches).
template <typename T, bool STREAM = false>
__device__ __forceinline__ typename RowVec<T>::type load_raw(const T* p, int left) {
  using V = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N;
  if (left >= N) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    else return *reinterpret_cast<const V*>(p);
  }
  V t = {};
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < left) t[e] = p[e];
  return t;
}

// Whether rows that a kernel reads (and writes) once are streamed: not where
// they fit the eight L2s (32 MB), and not below four cache lines a row, where
// neighbouring rows share lines that other waves want.  Without and with, in
// microseconds: the combine of 200 MB of bfloat16 rows 57.8 and 73.9 at 80 bytes
// a row, 48.8 and 47.0 at 512, 48.4 and 46.9 at 4096, of 1.07 GB at 8192 bytes
// 242 and 214; its gradient 147 and 178, 100 and 87, 98 and 86, and with 20 MB
// of 512-byte rows 11.3 and 12.0.
inline bool stream_rows(int64_t rows, int64_t C, size_t element) {
  return C * (int64_t)element >= 512 && rows * C * (int64_t)element > (int64_t(32) << 20);
}

template <typename T, bool STREAM = false, int M>
__device__ __forceinline__ void store_row(T* p, int left, const float (&v)[M]) {
  constexpr int N = RowVec<T>::N < M ? RowVec<T>::N : M;  // (4 of a narrow type, from float32)
  using V = std::conditional_t<N == RowVec<T>::N, typename RowVec<T>::type, typename RowVec<T>::four>;
  static_assert(M % N == 0 && (N == RowVec<T>::N || N == 4), "whole vectors");
  if (left >= M) {
#pragma unroll
    for (int b = 0; b < M; b += N) {
      V t;
#pragma unroll
      for (int e = 0; e < N; ++e) t[e] = (T)v[b + e];
      if constexpr (STREAM) __builtin_nontemporal_store(t, reinterpret_cast<V*>(p + b));
      else *reinterpret_cast<V*>(p + b) = t;
    }
  } else {
#pragma unroll
    for (int e = 0; e < M; ++e)
      if (e < left) p[e] = (T)v[e];
  }
}

// Split of rows x cv vectors over blocks of kRowThreads: block (x, y) takes R
// rows from x R and vectors [y cvb, (y + 1) cvb) of each, one vector per
// thread and step.
constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / kWave;
struct RowSplit {
  int64_t rows;
  int32_t C;    // elements per row
  int32_t cv;   // vectors per row
  int32_t cvb;  // vectors of a row per block
  int32_t R;    // rows per block
  Divisor by;   // by cvb
};

// About `want` vectors per block, fewer when that would leave compute units
// without a block.
inline RowSplit row_split(int64_t rows, int64_t C, int vec, int want = 4 * kRowThreads) {
  RowSplit s;
  s.rows = rows;
  s.C = (int32_t)C;
  s.cv = (int32_t)((C + vec - 1) / vec);
  if (rows * s.cv < (int64_t)1024 * want) want = kRowThreads;
  const int64_t parts = (s.cv + want - 1) / want;
  s.cvb = (int32_t)((s.cv + parts - 1) / parts);
  s.R = (int32_t)std::max<int64_t>(1, want / s.cvb);
  s.by = divisor(s.cvb);
  return s;
}

// Blocks along x, at most: a launch holds fewer than 2^32 threads along a
// dimension, so kernels step through more rows than that.
constexpr int64_t kMaxBlocks = int64_t(1) << 22;

inline dim3 row_grid(const RowSplit& s) {
  return dim3((unsigned)std::min<int64_t>((s.rows + s.R - 1) / s.R, kMaxBlocks),
              (unsigned)((s.cv + s.cvb - 1) / s.cvb));
}

// First element of vector c of a row of C elements: a row's last vector ends
// with the row, over elements of the one before (two lanes then move or sum the
// same elements alike); a row shorter than a vector has one partial vector.
// Going through a row's last few elements one by one instead takes every wave
// that holds one along: rows of 1001 float16 elements, 4 slots a token, were
// dispatched in 31 us and are in 24.
template <int N>
__device__ __forceinline__ int32_t vector_start(int32_t c, int32_t C) {
  return min(c * N, max(C - N, 0));
}

// Calls f(row, first element) for every vector of this thread.
template <int N, class F>
__device__ __forceinline__ void for_row_vectors(const RowSplit& s, F f) {
  const int32_t c0 = blockIdx.y * s.cvb;
  for (int64_t row0 = (int64_t)blockIdx.x * s.R; row0 < s.rows; row0 += (int64_t)gridDim.x * s.R) {
    const int32_t rows = (int32_t)min<int64_t>(s.R, s.rows - row0);
    for (uint32_t i = threadIdx.x; i < (uint32_t)(rows * s.cvb); i += kRowThreads) {
      const uint32_t r = s.by.div(i);
      const int32_t c = c0 + (int32_t)(i - r * (uint32_t)s.cvb);
      if (c < s.cv) f(row0 + r, vector_start<N>(c, s.C));
    }
  }
}

// Calls f with a value of the element type(s) behind the code(s); the codes
// are checked at the C entry.
template <class F>
void by_type(int dtype, F f) {
  if (dtype == BEVPOOL_F32) f(float{});
  else if (dtype == BEVPOOL_F16) f(half_t{});
  else f(bf16_t{});
}
// (out_dtype is in_dtype or float32)
template <class F>
void by_types(int in_dtype, int out_dtype, F f) {
  by_type(in_dtype, [&](auto t) {
    if (out_dtype == in_dtype) f(t, t);
    else f(t, float{});
  });
}

// (equal types, or one of the two float32)
template <class F>
void by_any_types(int in_dtype, int out_dtype, F f) {
  if (in_dtype == BEVPOOL_F32) by_type(out_dtype, [&](auto t) { f(float{}, t); });
  else by_types(in_dtype, out_dtype, f);
}

// Key i of an array of int32 or int64 keys, n_keys when outside [0, n_keys).
template <typename TKey>
__device__ __forceinline__ int32_t key_or_drop(const TKey* keys, int64_t i, int32_t n_keys) {
  const TKey k = keys[i];
  return (k >= 0 && k < (TKey)n_keys) ? (int32_t)k : n_keys;
}

}  // namespace bevpool
