// Router of expert layers: the k largest logits of every token and their
// softmax weights, and the logits' gradient.
//
// One wave per row; lane l holds the logits l, l + 64, ... in registers, so
// the row is read once.  Each of the k rounds takes the largest remaining
// (logit, lower index first) with a butterfly over the wave; the maximum of
// the softmax is the first round's logit, its sum is formed in float32 over
// the registers.

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// Order of floats as unsigned integers; -0 and +0 are equal, NaN below -inf.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0;
  const uint32_t b = __float_as_uint(v + 0.f);  // (-0 + 0 = +0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kOrderMinusInf = 0x007fffffu;  // order_of(-inf)

__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void k_route_forward(const T* __restrict__ logits,
                                                            int64_t stride, int64_t rows, int E,
                                                            int k, bool renormalise,
                                                            float* __restrict__ weights,
                                                            int32_t* __restrict__ ids) {
  const int lane = lane_id();
  for (int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; row < rows;
       row += (int64_t)gridDim.x * kWaves) {
    const T* p = logits + row * stride;
    uint32_t o[V];
    float x[V];
    bool nan = false;
  #pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * kWave + lane;
      x[i] = e < E ? (float)p[e] : -INFINITY;
      nan |= x[i] != x[i];
      o[i] = order_of(x[i]);
    }
    nan = wave_ballot(nan) != 0;
    float m = 0.f, mine = 0.f;  // lane j keeps the j-th chosen logit's term
    int32_t id = -1;
    for (int j = 0; j < k; ++j) {
      uint64_t best = 0;
  #pragma unroll
      for (int i = 0; i < V; ++i) {
        const uint64_t c = ((uint64_t)o[i] << 32) | (uint32_t)~(i * kWave + lane);
        best = c > best ? c : best;
      }
  #pragma unroll
      for (int s = kWave / 2; s > 0; s >>= 1) {
        const uint64_t c = __shfl_xor((unsigned long long)best, s, kWave);
        best = c > best ? c : best;
      }
      const uint32_t bo = (uint32_t)(best >> 32);
      if (bo <= kOrderMinusInf) break;  // (nothing left to choose; the same in every lane)
      const int e = (int)~(uint32_t)best;
      const float v = value_of(bo);
      if (j == 0) m = v;
      if (lane == j) {
        id = e;
        mine = expf(v - m);
      }
  #pragma unroll
      for (int i = 0; i < V; ++i)
        if (i * kWave + lane == e) o[i] = 0;
    }
    float sum = mine;
    if (!renormalise) {
      sum = 0.f;
  #pragma unroll
      for (int i = 0; i < V; ++i) sum += x[i] > -INFINITY ? expf(x[i] - m) : 0.f;
    }
    sum = wave_sum(sum);
    if (lane < k) {
      float w = id >= 0 ? mine / sum : 0.f;
      if (nan) w = NAN;
      weights[row * k + lane] = w;
      ids[row * k + lane] = id;
    }
  }
}

// grad[e] of a row: the chosen experts' terms are looked up by every lane.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void k_route_backward(
    const float* __restrict__ grad_weights, const T* __restrict__ logits, int64_t stride,
    int64_t rows, int E, int k, const float* __restrict__ weights,
    const int32_t* __restrict__ ids, bool renormalise, T* __restrict__ grad) {
  const int lane = lane_id();
  for (int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; row < rows;
       row += (int64_t)gridDim.x * kWaves) {
    float w = 0.f, g = 0.f;
    int32_t id = -1;
    if (lane < k) {
      id = ids[row * k + lane];
      w = weights[row * k + lane];
      g = id >= 0 ? grad_weights[row * k + lane] : 0.f;
    }
    const float s = wave_sum(id >= 0 ? w * g : 0.f);
    float p[V], G[V];
  #pragma unroll
    for (int i = 0; i < V; ++i) p[i] = G[i] = 0.f;
    if (!renormalise) {
      float x[V], m = -INFINITY;
      bool nan = false;
  #pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = i * kWave + lane;
        x[i] = e < E ? (float)logits[row * stride + e] : -INFINITY;
        nan |= x[i] != x[i];
        m = fmaxf(m, x[i]);
      }
  #pragma unroll
      for (int q = kWave / 2; q > 0; q >>= 1) m = fmaxf(m, __shfl_xor(m, q, kWave));
      float sum = 0.f;
  #pragma unroll
      for (int i = 0; i < V; ++i) {
        p[i] = x[i] > -INFINITY ? expf(x[i] - m) : 0.f;
        sum += p[i];
      }
      sum = wave_sum(sum);
      nan = wave_ballot(nan) != 0;
  #pragma unroll
      for (int i = 0; i < V; ++i) p[i] = nan ? NAN : (sum > 0.f ? p[i] / sum : 0.f);
    }
    for (int j = 0; j < k; ++j) {
      const int32_t e = __shfl(id, j, kWave);
      const float gj = __shfl(g, j, kWave), wj = __shfl(w, j, kWave);
  #pragma unroll
      for (int i = 0; i < V; ++i)
        if (i * kWave + lane == e) {
          G[i] = gj;
          if (renormalise) p[i] = wj;
        }
    }
  #pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * kWave + lane;
      if (e < E) grad[row * E + e] = (T)(p[i] == 0.f ? 0.f : p[i] * (G[i] - s));
    }
  }
}

template <class F>
void by_width(int E, F f) {
  if (E <= 64) f(std::integral_constant<int, 1>{});
  else if (E <= 128) f(std::integral_constant<int, 2>{});
  else if (E <= 256) f(std::integral_constant<int, 4>{});
  else if (E <= 512) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
}

}  // namespace

hipError_t launch_route_forward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                                const void* logits, int64_t stride, bool renormalise,
                                float* weights, int32_t* ids, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((rows + kWaves - 1) / kWaves, kMaxBlocks));
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    by_width(n_experts, [&](auto v) {
      k_route_forward<T, v.value><<<grid, kThreads, 0, stream>>>(
          static_cast<const T*>(logits), stride, rows, n_experts, k, renormalise, weights, ids);
    });
  });
  return hipGetLastError();
}

hipError_t launch_route_backward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                                 const float* grad_weights, const void* logits, int64_t stride,
                                 const float* weights, const int32_t* ids, bool renormalise,
                                 void* grad_logits, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((rows + kWaves - 1) / kWaves, kMaxBlocks));
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    by_width(n_experts, [&](auto v) {
      k_route_backward<T, v.value><<<grid, kThreads, 0, stream>>>(
          grad_weights, static_cast<const T*>(logits), stride, rows, n_experts, k, weights, ids,
          renormalise, static_cast<T*>(grad_logits));
    });
  });
  return hipGetLastError();
}

}  // namespace bevpool
