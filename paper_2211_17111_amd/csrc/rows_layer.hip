// Whole expert layer for a few tokens: two launches, the gated products of every
// slot with its expert's rows, then the weighted sums of their products.

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// <a, b> over n elements, the same in every lane.
template <typename TA, typename TB>
__device__ __forceinline__ float wave_dot(const TA* a, const TB* b, int n) {
  float s = 0.f;
  for (int i = lane_id(); i < n; i += kWave) s = fmaf((float)a[i], (float)b[i], s);
  return wave_sum(s);
}

// A wave takes one hidden value of a slot.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_layer_up(const T* __restrict__ x, int64_t x_stride,
                                                       const T* __restrict__ up,
                                                       const int32_t* __restrict__ ids, int k,
                                                       int C, int F, int E,
                                                       float* __restrict__ hidden) {
  const int s = blockIdx.y, f = blockIdx.x * kWaves + threadIdx.x / kWave;
  const int e = ids[s];
  if (e < 0 || e >= E || f >= F) return;
  const T* row = x + (int64_t)(s / k) * x_stride;
  const float gate = wave_dot(row, up + ((int64_t)e * 2 * F + f) * C, C);
  const float value = wave_dot(row, up + ((int64_t)e * 2 * F + F + f) * C, C);
  if (lane_id() == 0) hidden[(int64_t)s * F + f] = gate / (1.f + expf(-gate)) * value;
}

// A wave takes one output of a token.
template <typename T, typename TW>
__global__ __launch_bounds__(kThreads) void k_layer_down(const float* __restrict__ hidden,
                                                         const T* __restrict__ down,
                                                         const TW* __restrict__ weights,
                                                         const int32_t* __restrict__ ids, int k,
                                                         int C, int F, int E,
                                                         T* __restrict__ out) {
  const int t = blockIdx.y, c = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (c >= C) return;
  float sum = 0.f;
  for (int s = t * k; s < t * k + k; ++s) {
    const int e = ids[s];
    if (e < 0 || e >= E) continue;
    const float y = wave_dot(hidden + (int64_t)s * F, down + ((int64_t)e * C + c) * F, F);
    sum = fmaf((float)weights[s], y, sum);
  }
  if (lane_id() == 0) out[(int64_t)t * C + c] = (T)sum;
}

}  // namespace

size_t layer_workspace(int64_t rows, int32_t k, int64_t F, int) {
  return (size_t)(rows * k * F) * sizeof(float);
}

hipError_t launch_expert_layer(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts,
                               int dtype, int weight_dtype, const void* x, int64_t x_stride,
                               const void* up, const void* down, const void* weights,
                               const int32_t* ids, void* out, void* workspace,
                               hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  by_types(dtype, weight_dtype, [&](auto t, auto tw) {
    using T = decltype(t);
    using TW = decltype(tw);
    float* hidden = static_cast<float*>(workspace);
    const dim3 slots((unsigned)((F + kWaves - 1) / kWaves), (unsigned)(rows * k));
    k_layer_up<T><<<slots, kThreads, 0, stream>>>(static_cast<const T*>(x), x_stride,
                                                  static_cast<const T*>(up), ids, k, (int)C,
                                                  (int)F, n_experts, hidden);
    const dim3 tokens((unsigned)((C + kWaves - 1) / kWaves), (unsigned)rows);
    k_layer_down<T, TW><<<tokens, kThreads, 0, stream>>>(
        hidden, static_cast<const T*>(down), static_cast<const TW*>(weights), ids, k, (int)C,
        (int)F, n_experts, static_cast<T*>(out));
  });
  return hipGetLastError();
}

}  // namespace bevpool
