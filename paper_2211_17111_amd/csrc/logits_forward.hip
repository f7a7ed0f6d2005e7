// Forward of the logits operators: statistics of every row's softmax, and from
// them log probabilities, entropy, alternatives and divergences.

#include "logits.h"
#include "logits_rows.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;

// Floats as unsigned integers in their order, +0 and -0 the same; 0, below all
// of them, for what is never chosen (-inf, NaN).
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // (-0 + 0 = +0)
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return v > -INFINITY ? o : 0;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

// A logit's order and its index in one number: larger logits are larger, of
// equal ones the lower index is.
__device__ __forceinline__ uint64_t pair_of(uint32_t order, int v) {
  return ((uint64_t)order << 32) | (uint32_t)~v;
}

template <class TEAM>
__device__ __forceinline__ uint64_t team_max(const TEAM& team, uint64_t v, uint64_t* scratch) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    const uint64_t other = __shfl_xor(v, o, kWave);
    v = other > v ? other : v;
  }
  if (lane_id() == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  for (int w = 0; w < TEAM::kWaves; ++w) v = scratch[w] > v ? scratch[w] : v;
  __syncthreads();
  return v;
}

// One alternative of a row, best (0: none).
__device__ __forceinline__ void write_alternative(const LogprobsOut& out, int64_t at, uint64_t best,
                                                  const Row& p) {
  const uint32_t order = (uint32_t)(best >> 32);
  out.top[at] = p.S != p.S ? NAN : order != 0 ? p.logprob(value_of(order)) : -INFINITY;
  out.top_ids[at] = order != 0 ? (int32_t) ~(uint32_t)best : -1;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprobs(LogitsRows in, LogprobsOut out, float c) {
  __shared__ float s_scratch[kThreads / kWave];
  __shared__ uint64_t s_pairs[kThreads / kWave];
  const Team<kThreads> team{s_scratch};
  for (int64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    Soft a = no_soft();
    for_logits(team, row, in.V, [&](const auto& x, int) { add<true>(a, x, c); });
    a = join<true>(team, a, c);
    const Row p = row_of(a, in.scale);
    if (threadIdx.x == 0) {
      out.stats[2 * t] = p.m;
      out.stats[2 * t + 1] = p.S;
      if (out.logprob != nullptr) {
        const int32_t id = id_at(in.ids, in.key_type, t, in.V);
        out.logprob[t] = id >= 0 ? p.logprob((float)row[id]) : 0.f;
      }
      if (out.lse != nullptr) out.lse[t] = p.S == 0.f ? -INFINITY : fmaf(p.scale, p.m, p.log_S);
      if (out.entropy != nullptr) out.entropy[t] = p.S == 0.f ? 0.f : fmaf(-kLn2, a.w / a.s, p.log_S);
    }
    uint64_t last = ~uint64_t(0);
    for (int j = 0; j < in.k; ++j) {
      uint64_t best = 0;
      for_logits(team, row, in.V, [&](const auto& x, int v0) {
#pragma unroll
        for (int i = 0; i < RowVec<T>::N; ++i) {
          const uint32_t o = order_of(x[i]);
          const uint64_t pair = pair_of(o, v0 + i);
          if (o != 0 && pair < last && pair > best) best = pair;
        }
      });
      last = best = team_max(team, best, s_pairs);
      if (threadIdx.x == 0) write_alternative(out, t * in.k + j, best, p);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill(LogitsRows in, float* __restrict__ loss,
                                                      float* __restrict__ stats, float c) {
  __shared__ float s_scratch[kThreads / kWave];
  const Team<kThreads> team{s_scratch};
  for (int64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    Soft a = no_soft();
    for_logits(team, row, in.V, [&](const auto& x, int) { add<false>(a, x, c); });
    a = join<false>(team, a, c);
    const Row p = row_of(a, in.scale);
    const Taught q = taught(team, in, t);
    const float d = divergence(team, in, t, row, p, q);
    if (threadIdx.x == 0) {
      stats[2 * t] = p.m;
      stats[2 * t + 1] = p.S;
      loss[t] = d;
    }
  }
}

dim3 row_blocks(int64_t rows) { return dim3((unsigned)std::min<int64_t>(rows, kMaxBlocks)); }

}  // namespace

size_t logprobs_workspace(int64_t, int64_t, int32_t, int) { return 0; }
size_t distill_workspace(int64_t, int64_t, int32_t, int) { return 0; }

hipError_t launch_logprobs_forward(const LogitsRows& in, const LogprobsOut& out, void*,
                                   hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    k_logprobs<decltype(t)><<<row_blocks(in.rows), kThreads, 0, stream>>>(
        in, out, exponent_factor(in.scale));
  });
  return hipGetLastError();
}

hipError_t launch_distill_forward(const LogitsRows& in, float* loss, float* stats, void*,
                                  hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    k_distill<decltype(t)><<<row_blocks(in.rows), kThreads, 0, stream>>>(
        in, loss, stats, exponent_factor(in.scale));
  });
  return hipGetLastError();
}

}  // namespace bevpool
