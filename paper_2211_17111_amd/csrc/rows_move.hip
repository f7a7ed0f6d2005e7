// Dispatch and combine of expert layers.  Everything goes by position, the
// place of slot (t, j) in expert order: a token's row is read once and written
// to its k places, and a token's k expert rows are read from theirs and summed
// in slot order, so that neither direction needs atomics.  Places behind
// *kept belong to dropped slots.  All of it is bound by memory: bytes per
// element moved against one multiply-add.

#include "device_utils.h"
#include "rows.h"
#include "rows_sort.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kSlots = 4;  // slots of a token whose places or rows a thread has in flight

// Stores vector c of token t's row at the places of its k slots (`place` gives
// them by slot), zeros for dropped ones.  The elements are moved as they are
// (T: an unsigned integer of their size).
template <typename T, typename V, int N, class Place>
__device__ __forceinline__ void move_vector(const T* __restrict__ x, int64_t x_stride,
                                            const RowSplit& s, int k, int64_t t, int32_t c,
                                            int32_t kept, Place place, T* __restrict__ out) {
  const int64_t n = s.rows * k;
  const T* p = x + t * x_stride + c;
  const int left = s.C - c;
  V v{};
  if (left >= N) {
    v = *reinterpret_cast<const V*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) v[e] = p[e];
  }
  for (int j0 = 0; j0 < k; j0 += kSlots) {
    int32_t pos[kSlots];
#pragma unroll
    for (int u = 0; u < kSlots; ++u) pos[u] = j0 + u < k ? place(t * k + j0 + u) : -1;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      if (pos[u] < 0 || pos[u] >= n) continue;
      const V w = pos[u] < kept ? v : V{};
      T* q = out + (int64_t)pos[u] * s.C + c;
      if (left >= N) {
        *reinterpret_cast<V*>(q) = w;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < left) q[e] = w[e];
      }
    }
  }
}

template <typename T, typename V, int N>
__global__ __launch_bounds__(kRowThreads) void k_dispatch(const T* __restrict__ x, int64_t x_stride,
                                                          RowSplit s, int k,
                                                          const int32_t* __restrict__ position,
                                                          const int32_t* __restrict__ kept_ptr,
                                                          T* __restrict__ out) {
  const int32_t kept = *kept_ptr;
  for_row_vectors<N>(s, [&](int64_t t, int32_t c) {
    move_vector<T, V, N>(x, x_stride, s, k, t, c, kept, [&](int64_t i) { return position[i]; }, out);
  });
}

// Few tokens (decoding): at most kSortTile slots and fewer than kMaxDigits
// keys.  Every block sorts all the slots in its LDS, the first one writes the
// order down, and each moves its rows: one launch.
template <typename T, typename V, int N, typename TKey>
__global__ __launch_bounds__(kRowThreads) void k_dispatch_small(
    const T* __restrict__ x, int64_t x_stride, RowSplit s, int k, const TKey* __restrict__ ids,
    int32_t n_keys, int digit_bits, int32_t* __restrict__ order, int32_t* __restrict__ position,
    int32_t* __restrict__ offsets, T* __restrict__ out) {
  static_assert(kRowThreads == kTileThreads, "a block is a tile");
  __shared__ int cnt[kTileWaves][kMaxDigits];
  __shared__ int s_scan[kTileWaves];
  __shared__ int32_t s_pos[kSortTile];
  __shared__ int32_t s_kept;
  const int n = (int)s.rows * k;
  const int digits = 1 << digit_bits;
  const bool writer = blockIdx.x == 0 && blockIdx.y == 0;
  int32_t key[kTileRounds], rank[kTileRounds];
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int i = tile_index(r);
    key[r] = i < n ? key_or_drop(ids, i, n_keys) : 0;
  }
  tile_ranks(key, n, 0, digit_bits, cnt, rank);
  const int per = max(1, digits / kTileThreads);
  int sum = 0;
#pragma unroll
  for (int q = 0; q < kDigitsPerThread; ++q) {
    const int d = threadIdx.x * per + q;
    if (q < per && d < digits)
#pragma unroll
      for (int w = 0; w < kTileWaves; ++w) sum += cnt[w][d];
  }
  int all;
  int at = block_exclusive_scan<kTileThreads, true>(sum, s_scan, &all);
#pragma unroll
  for (int q = 0; q < kDigitsPerThread; ++q) {
    const int d = threadIdx.x * per + q;
    if (q >= per || d >= digits) continue;
    if (writer && d <= n_keys) offsets[d] = at;
    if (d == n_keys) s_kept = at;
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) {
      const int c = cnt[w][d];
      cnt[w][d] = at;
      at += c;
    }
  }
  lds_barrier();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int i = tile_index(r);
    if (i >= n) continue;
    const int32_t pos = cnt[threadIdx.x / kWave][key[r]] + rank[r];
    s_pos[i] = pos;
    if (writer) {
      position[i] = pos;
      order[pos] = i;
    }
  }
  lds_barrier();
  const int32_t kept = s_kept;
  for_row_vectors<N>(s, [&](int64_t t, int32_t c) {
    move_vector<T, V, N>(x, x_stride, s, k, t, c, kept, [&](int64_t i) { return s_pos[i]; }, out);
  });
}

// Calls f with a value of the unsigned integer type of dtype's size, a vector
// of them and its length.
template <class F>
void by_element(int dtype, F f) {
  typedef uint32_t V4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint16_t V8 __attribute__((ext_vector_type(8), aligned(2)));
  if (dtype == BEVPOOL_F32) f(uint32_t{}, V4{}, std::integral_constant<int, 4>{});
  else f(uint16_t{}, V8{}, std::integral_constant<int, 8>{});
}

template <typename T>
__device__ __forceinline__ float weight_at(const void* w, bool f32, int64_t i) {
  return f32 ? static_cast<const float*>(w)[i] : (float)static_cast<const T*>(w)[i];
}

// out[t] = sum over kept j of w[t k + j] * in[position[t k + j]], w = 1 where
// weights is NULL.
template <typename T, typename TO, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void k_combine(const T* __restrict__ in, int64_t stride,
                                                         RowSplit s, int k,
                                                         const void* __restrict__ weights,
                                                         bool weights_f32,
                                                         const int32_t* __restrict__ position,
                                                         const int32_t* __restrict__ kept_ptr,
                                                         TO* __restrict__ out) {
  using V = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N;
  const int64_t n = s.rows * k;
  const int32_t kept = (int32_t)min<int64_t>(*kept_ptr, n);
  for_row_vectors<N>(s, [&](int64_t t, int32_t c) {
    const int left = s.C - c;
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    for (int j0 = 0; j0 < k; j0 += kSlots) {
      int32_t pos[kSlots];
      float w[kSlots];
      V v[kSlots];
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        const int64_t i = t * k + j0 + u;
        pos[u] = j0 + u < k ? position[i] : -1;
        w[u] = 1.f;
        if (weights != nullptr && j0 + u < k) w[u] = weight_at<T>(weights, weights_f32, i);
      }
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        v[u] = V{};
        if (pos[u] >= 0 && pos[u] < kept) v[u] = load_raw<T, STREAM>(in + pos[u] * stride + c, left);
      }
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        if (pos[u] < 0 || pos[u] >= kept) continue;  // (a dropped slot's weight may be anything)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = fmaf(w[u], (float)v[u][e], acc[e]);
      }
    }
    store_row<TO>(out + t * s.C + c, left, acc);
  });
}

// The gradients of a token's slots by a group of W lanes (a power of two, or
// the whole block): grad_out's row is read once for kSlots slots, their rows are
// in flight together, and each weight's gradient is a sum over the group.
template <typename T, typename TO, int W, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void k_combine_backward(
    const TO* __restrict__ grad_out, int64_t grad_stride, const T* __restrict__ in,
    int64_t in_stride, int64_t rows, int k, int C, const void* __restrict__ weights,
    bool weights_f32, const int32_t* __restrict__ position, const int32_t* __restrict__ kept_ptr,
    T* __restrict__ grad_in, void* __restrict__ grad_weights) {
  using V = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N;
  constexpr int kGroups = kRowThreads / W;
  __shared__ float s_dot[kRowWaves][kSlots];
  const int64_t n = rows * k;
  const int32_t kept = *kept_ptr;
  const int lane = threadIdx.x % W;
  const int cv = (C + N - 1) / N;
  for (int64_t t0 = (int64_t)blockIdx.x * kGroups; t0 < rows; t0 += (int64_t)gridDim.x * kGroups) {
    // (groups past the end go along for the sums, without slots)
    const int64_t t = min(t0 + threadIdx.x / W, rows - 1);
    const bool mine = t0 + threadIdx.x / W < rows;
    for (int j0 = 0; j0 < k; j0 += kSlots) {
      int32_t pos[kSlots];
      float w[kSlots], dot[kSlots];
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        const int64_t i = t * k + j0 + u;
        pos[u] = mine && j0 + u < k ? position[i] : -1;
        if (pos[u] >= n) pos[u] = -1;
        w[u] = dot[u] = 0.f;
        if (grad_in != nullptr && j0 + u < k) w[u] = weight_at<T>(weights, weights_f32, i);
      }
      for (int vec = lane; vec < cv; vec += W) {
        const int c = vector_start<N>(vec, C);
        const int left = C - c;
        const int again = vec * N - c;  // elements that the vector before has too
        float g[N];
        load_row<TO>(grad_out + t * grad_stride + c, left, g);
        V v[kSlots];
        if (grad_weights != nullptr) {
#pragma unroll
          for (int u = 0; u < kSlots; ++u) {
            v[u] = V{};
            if (pos[u] >= 0 && pos[u] < kept) v[u] = load_raw<T, STREAM>(in + pos[u] * in_stride + c, left);
          }
        }
        if (grad_in != nullptr) {
#pragma unroll
          for (int u = 0; u < kSlots; ++u) {
            if (pos[u] < 0) continue;
            float d[N];
#pragma unroll
            for (int e = 0; e < N; ++e) d[e] = pos[u] < kept ? w[u] * g[e] : 0.f;
            store_row<T, STREAM>(grad_in + (int64_t)pos[u] * C + c, left, d);
          }
        }
        if (grad_weights != nullptr) {
#pragma unroll
          for (int u = 0; u < kSlots; ++u) {
            if (pos[u] < 0 || pos[u] >= kept) continue;
#pragma unroll
            for (int e = 0; e < N; ++e)
              dot[u] = e >= again ? fmaf(g[e], (float)v[u][e], dot[u]) : dot[u];
          }
        }
      }
      if (grad_weights == nullptr) continue;
#pragma unroll
      for (int u = 0; u < kSlots; ++u)
#pragma unroll
        for (int o = min(W, kWave) / 2; o > 0; o >>= 1) dot[u] += __shfl_xor(dot[u], o, kWave);
      if constexpr (W > kWave) {
        __syncthreads();  // (the sums of the slots before have been read)
        if (threadIdx.x % kWave == 0)
#pragma unroll
          for (int u = 0; u < kSlots; ++u) s_dot[threadIdx.x / kWave][u] = dot[u];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
          dot[u] = s_dot[0][u];
#pragma unroll
          for (int b = 1; b < kRowWaves; ++b) dot[u] += s_dot[b][u];
        }
      }
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        if (lane != u % W || !mine || j0 + u >= k) continue;
        const int64_t i = t * k + j0 + u;
        if (weights_f32) static_cast<float*>(grad_weights)[i] = dot[u];
        else static_cast<T*>(grad_weights)[i] = (T)dot[u];
      }
    }
  }
}

// Lanes per token of the combine's gradient: no more than a row has vectors, a
// whole block for rows that fill it (their k slots then go through DRAM in
// whole rows: 16,384 tokens of 4 slots, C = 2048 in bfloat16, took 130 us by
// waves and 118 by blocks, and 111 since the rows are streamed) and where waves
// would leave the device empty (fewer than eight to a compute unit).
template <class F>
void by_lanes(int64_t rows, int64_t cv, F f) {
  if (cv >= kRowThreads || (cv > kWave && rows < 2048))
    f(std::integral_constant<int, kRowThreads>{});
  else if (cv > 32) f(std::integral_constant<int, kWave>{});
  else if (cv > 16) f(std::integral_constant<int, 32>{});
  else if (cv > 8) f(std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, 8>{});
}

}  // namespace

hipError_t launch_dispatch_rows(int64_t rows, int32_t k, int64_t C, int dtype, const void* x,
                                int64_t x_stride, const int32_t* position, const int32_t* kept,
                                void* out, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  by_element(dtype, [&](auto e, auto v, auto n) {
    using T = decltype(e);
    const RowSplit s = row_split(rows, C, n.value);
    k_dispatch<T, decltype(v), n.value><<<row_grid(s), kRowThreads, 0, stream>>>(
        static_cast<const T*>(x), x_stride, s, k, position, kept, static_cast<T*>(out));
  });
  return hipGetLastError();
}

hipError_t launch_dispatch_forward(int64_t rows, int32_t k, int64_t C, int64_t n_keys, int dtype,
                                   const void* x, int64_t x_stride, int key_type, const void* ids,
                                   int32_t* order, int32_t* position, int32_t* offsets, void* out,
                                   void* workspace, hipStream_t stream) {
  const int64_t n = rows * k;
  // One launch where a block can sort all the slots, two and more else.  In a
  // graph, one against two: 5.2 and 6.8 us for a token of 6 slots, C = 2048;
  // 7.4 and 9.3 for 128 tokens of 8, C = 4096; 9.8 and 8.0 for 1024 tokens of
  // one slot, whose second launch costs a caller 3 us more outside a graph.
  if (n == 0 || n > kSortTile || n_keys >= kMaxDigits) {
    const hipError_t e = launch_sort_keys(n, n_keys, key_type, ids, order, position, offsets,
                                          nullptr, workspace, stream);
    if (e != hipSuccess) return e;
    return launch_dispatch_rows(rows, k, C, dtype, x, x_stride, position, offsets + n_keys, out,
                                stream);
  }
  const int bits = sort_layout(n, n_keys).digit_bits;
  by_element(dtype, [&](auto e, auto v, auto w) {
    using T = decltype(e);
    const RowSplit s = row_split(rows, C, w.value);
    auto go = [&](auto* keys) {
      k_dispatch_small<T, decltype(v), w.value><<<row_grid(s), kRowThreads, 0, stream>>>(
          static_cast<const T*>(x), x_stride, s, k, keys, (int32_t)n_keys, bits, order, position,
          offsets, static_cast<T*>(out));
    };
    if (key_type == BEVPOOL_KEY_I64) go(static_cast<const int64_t*>(ids));
    else go(static_cast<const int32_t*>(ids));
  });
  return hipGetLastError();
}

hipError_t launch_combine_forward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                                  int weight_dtype, const void* in, int64_t in_stride,
                                  const void* weights, const int32_t* position,
                                  const int32_t* kept, void* out, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  by_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    const RowSplit s = row_split(rows, C, RowVec<T>::N);
    auto go = [&](auto hint) {
      k_combine<T, TO, hint.value><<<row_grid(s), kRowThreads, 0, stream>>>(
          static_cast<const T*>(in), in_stride, s, k, weights, weight_dtype == BEVPOOL_F32,
          position, kept, static_cast<TO*>(out));
    };
    if (stream_rows(rows * k, C, sizeof(T))) go(std::true_type{});
    else go(std::false_type{});
  });
  return hipGetLastError();
}

hipError_t launch_combine_backward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                                   int weight_dtype, const void* grad_out, int64_t grad_stride,
                                   const void* in, int64_t in_stride, const void* weights,
                                   const int32_t* position, const int32_t* kept, void* grad_in,
                                   void* grad_weights, hipStream_t stream) {
  if (rows == 0 || (grad_in == nullptr && grad_weights == nullptr)) return hipSuccess;
  by_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    by_lanes(rows, (C + RowVec<T>::N - 1) / RowVec<T>::N, [&](auto w) {
      constexpr int kGroups = kRowThreads / w.value;
      const dim3 grid((unsigned)std::min<int64_t>((rows + kGroups - 1) / kGroups, kMaxBlocks));
      auto go = [&](auto hint) {
        k_combine_backward<T, TO, w.value, hint.value><<<grid, kRowThreads, 0, stream>>>(
            static_cast<const TO*>(grad_out), grad_stride, static_cast<const T*>(in), in_stride,
            rows, k, (int)C, weights, weight_dtype == BEVPOOL_F32, position, kept,
            static_cast<T*>(grad_in), grad_weights);
      };
      if (stream_rows(rows * k, C, sizeof(T))) go(std::true_type{});
      else go(std::false_type{});
    });
  });
  return hipGetLastError();
}

}  // namespace bevpool
