// Dispatch and combine of expert layers.  Everything goes by position, the
// place of slot (t, j) in expert order: a token's row is read once and written
// to its k places, and a token's k expert rows are read from theirs and summed
// in slot order, so that neither direction needs atomics.  Places behind
// *kept belong to dropped slots.  All of it is bound by memory: bytes per
// element moved against one multiply-add.

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

// out[position[t k + j]] = x[t], zeros for dropped slots.  The elements are
// moved as they are (T: an unsigned integer of their size).
template <typename T, typename V, int N>
__global__ __launch_bounds__(kRowThreads) void k_dispatch(const T* __restrict__ x, int64_t x_stride,
                                                          RowSplit s, int k,
                                                          const int32_t* __restrict__ position,
                                                          const int32_t* __restrict__ kept_ptr,
                                                          T* __restrict__ out) {
  const int64_t n = s.rows * k;
  const int32_t kept = *kept_ptr;
  for_row_vectors<N>(s, [&](int64_t t, int32_t c) {
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
    for (int j = 0; j < k; ++j) {
      const int32_t pos = position[t * k + j];
      if (pos < 0 || pos >= n) continue;
      const V w = pos < kept ? v : V{};
      T* q = out + (int64_t)pos * s.C + c;
      if (left >= N) {
        *reinterpret_cast<V*>(q) = w;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < left) q[e] = w[e];
      }
    }
  });
}

template <typename T>
__device__ __forceinline__ float weight_at(const void* w, bool f32, int64_t i) {
  return f32 ? static_cast<const float*>(w)[i] : (float)static_cast<const T*>(w)[i];
}

// out[t] = sum over kept j of w[t k + j] * in[position[t k + j]], w = 1 where
// weights is NULL.
template <typename T, typename TO>
__global__ __launch_bounds__(kRowThreads) void k_combine(const T* __restrict__ in, int64_t stride,
                                                         RowSplit s, int k,
                                                         const void* __restrict__ weights,
                                                         bool weights_f32,
                                                         const int32_t* __restrict__ position,
                                                         const int32_t* __restrict__ kept_ptr,
                                                         TO* __restrict__ out) {
  constexpr int N = RowVec<T>::N;
  const int64_t n = s.rows * k;
  const int32_t kept = (int32_t)min<int64_t>(*kept_ptr, n);
  for_row_vectors<N>(s, [&](int64_t t, int32_t c) {
    const int left = s.C - c;
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    for (int j = 0; j < k; ++j) {
      const int32_t pos = position[t * k + j];
      if (pos < 0 || pos >= kept) continue;
      const float w = weights != nullptr ? weight_at<T>(weights, weights_f32, t * k + j) : 1.f;
      float v[N];
      load_row<T>(in + pos * stride + c, left, v);
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] = fmaf(w, v[e], acc[e]);
    }
    store_row<TO>(out + t * s.C + c, left, acc);
  });
}

// One wave per token: grad_in of its slots and the weights' gradients.
template <typename T, typename TO>
__global__ __launch_bounds__(kRowThreads) void k_combine_backward(
    const TO* __restrict__ grad_out, int64_t grad_stride, const T* __restrict__ in,
    int64_t in_stride, int64_t rows, int k, int C, const void* __restrict__ weights,
    bool weights_f32, const int32_t* __restrict__ position, const int32_t* __restrict__ kept_ptr,
    T* __restrict__ grad_in, void* __restrict__ grad_weights) {
  constexpr int N = RowVec<T>::N;
  const int64_t n = rows * k;
  const int32_t kept = *kept_ptr;
  const int lane = lane_id();
  for (int64_t t = (int64_t)blockIdx.x * kRowWaves + threadIdx.x / kWave; t < rows;
       t += (int64_t)gridDim.x * kRowWaves) {
    for (int j = 0; j < k; ++j) {
      const int32_t pos = position[t * k + j];
      if (pos < 0 || pos >= n) continue;
      const bool on = pos < kept;
      const float w = on && grad_in != nullptr ? weight_at<T>(weights, weights_f32, t * k + j) : 0.f;
      float dot = 0.f;
      for (int c = lane * N; c < C; c += kWave * N) {
        float g[N];
        load_row<TO>(grad_out + t * grad_stride + c, C - c, g);
        if (grad_weights != nullptr && on) {
          float v[N];
          load_row<T>(in + pos * in_stride + c, C - c, v);
  #pragma unroll
          for (int e = 0; e < N; ++e) dot = fmaf(g[e], v[e], dot);
        }
        if (grad_in != nullptr) {
  #pragma unroll
          for (int e = 0; e < N; ++e) g[e] = on ? w * g[e] : 0.f;
          store_row<T>(grad_in + (int64_t)pos * C + c, C - c, g);
        }
      }
      if (grad_weights != nullptr) {
  #pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) dot += __shfl_xor(dot, o, kWave);
        if (lane == 0) {
          if (weights_f32)
            static_cast<float*>(grad_weights)[t * k + j] = dot;
          else
            static_cast<T*>(grad_weights)[t * k + j] = (T)dot;
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_dispatch_rows(int64_t rows, int32_t k, int64_t C, int dtype, const void* x,
                                int64_t x_stride, const int32_t* position, const int32_t* kept,
                                void* out, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  typedef uint32_t V4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint16_t V8 __attribute__((ext_vector_type(8), aligned(2)));
  if (dtype == BEVPOOL_F32) {
    const RowSplit s = row_split(rows, C, 4);
    k_dispatch<uint32_t, V4, 4><<<row_grid(s), kRowThreads, 0, stream>>>(
        static_cast<const uint32_t*>(x), x_stride, s, k, position, kept,
        static_cast<uint32_t*>(out));
  } else {
    const RowSplit s = row_split(rows, C, 8);
    k_dispatch<uint16_t, V8, 8><<<row_grid(s), kRowThreads, 0, stream>>>(
        static_cast<const uint16_t*>(x), x_stride, s, k, position, kept,
        static_cast<uint16_t*>(out));
  }
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
    k_combine<T, TO><<<row_grid(s), kRowThreads, 0, stream>>>(
        static_cast<const T*>(in), in_stride, s, k, weights, weight_dtype == BEVPOOL_F32, position,
        kept, static_cast<TO*>(out));
  });
  return hipGetLastError();
}

hipError_t launch_combine_backward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                                   int weight_dtype, const void* grad_out, int64_t grad_stride,
                                   const void* in, int64_t in_stride, const void* weights,
                                   const int32_t* position, const int32_t* kept, void* grad_in,
                                   void* grad_weights, hipStream_t stream) {
  if (rows == 0 || (grad_in == nullptr && grad_weights == nullptr)) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((rows + kRowWaves - 1) / kRowWaves, kMaxBlocks));
  by_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    k_combine_backward<T, TO><<<grid, kRowThreads, 0, stream>>>(
        static_cast<const TO*>(grad_out), grad_stride, static_cast<const T*>(in), in_stride, rows,
        k, (int)C, weights, weight_dtype == BEVPOOL_F32, position, kept, static_cast<T*>(grad_in),
        grad_weights);
  });
  return hipGetLastError();
}

}  // namespace bevpool
