// Gradients of the logits operators.  Both are, at logit v of a row,
//   e_v (A + B u_v) + sum of g_j over the row's marked tokens j that are v,
// e_v = 2^(u_v) = S p_v: what differs is A, B and the marked tokens (the given
// token and the alternatives, or the teacher's).

#include "logits.h"
#include "logits_rows.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxMarked = 1 + (kMaxTaught > kMaxAlternatives ? kMaxTaught : kMaxAlternatives);

// The gradient of a row; `none`: zeros.
struct RowGradient {
  float m, A, B;
  bool none;
};

template <class TEAM>
__device__ __forceinline__ RowGradient gradient_of(const TEAM& team, const LogitsRows& in,
                                                   const LogprobsGrads& g, int64_t t, int32_t* ids,
                                                   float* values) {
  const float m = g.stats[2 * t], S = g.stats[2 * t + 1];
  const int32_t id = g.logprob != nullptr ? id_at(in.ids, in.key_type, t, in.V) : -1;
  const float gl = id >= 0 ? g.logprob[t] : 0.f;
  const float gz = g.lse != nullptr ? g.lse[t] : 0.f;
  const float gh = g.of_entropy != nullptr ? g.of_entropy[t] : 0.f;
  const int k = g.top != nullptr ? in.k : 0;
  float sum = 0.f, some = 0.f;
  for (int j = team.lane(); j < k; j += TEAM::kLanes) {
    const int32_t v = g.top_ids[t * in.k + j];
    const bool on = v >= 0 && v < in.V;
    const float own = on ? g.top[t * in.k + j] : 0.f;
    ids[1 + j] = on ? v : -1;
    values[1 + j] = own * in.scale;
    sum += own;
    some = own != 0.f ? 1.f : some;  // (a NaN is some)
  }
  if (team.lane() == 0) {
    ids[0] = id;
    values[0] = gl * in.scale;
  }
  if (k > 0) {
    sum = team.sum(sum);
    some = team.max(some);
  }
  RowGradient r;
  r.m = m;
  r.none = S == 0.f || (some == 0.f && gl == 0.f && gz == 0.f && gh == 0.f);
  const float by = in.scale / S;
  // log p + H = ln2 u + (H - log S)
  r.A = by * (gz - gl - sum - (gh != 0.f ? gh * (g.entropy[t] - logf(S)) : 0.f));
  r.B = -by * gh * kLn2;
  return r;
}

struct DistillGrads {
  const float *stats, *loss;  // loss: the outgoing gradient
};

template <class TEAM>
__device__ __forceinline__ RowGradient gradient_of(const TEAM& team, const LogitsRows& in,
                                                   const DistillGrads& g, int64_t t, int32_t* ids,
                                                   float* values) {
  const float m = g.stats[2 * t], S = g.stats[2 * t + 1];
  const float go = g.loss[t];
  const Taught q = taught(team, in, t);
  for (int j = team.lane(); j < in.k; j += TEAM::kLanes) {
    float l;
    const int32_t id = slot_of(in, t, j, &l);
    ids[j] = id;
    values[j] = id >= 0 && l != -INFINITY ? -go * in.scale * expf(l - q.shift) : 0.f;
  }
  RowGradient r;
  r.m = m;
  r.none = S == 0.f || go == 0.f || !q.any;
  r.A = in.scale * go * q.mass / S;
  r.B = 0.f;
  return r;
}

template <bool ENTROPY>
__device__ __forceinline__ float base_of(const RowGradient& r, float x, float c) {
  const float u = (x - r.m) * c;
  const float e = __builtin_amdgcn_exp2f(u);
  return ENTROPY ? e * fmaf(r.B, held(u), r.A) : e * r.A;
}

template <typename T, bool ENTROPY, class G>
__global__ __launch_bounds__(kThreads) void k_logits_gradient(LogitsRows in, G g, int marked,
                                                              T* __restrict__ grad, float c) {
  constexpr int N = RowVec<T>::N;
  __shared__ float s_scratch[kThreads / kWave];
  __shared__ int32_t s_ids[kMaxMarked];
  __shared__ float s_values[kMaxMarked];
  const Team<kThreads> team{s_scratch};
  for (int64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    const RowGradient r = gradient_of(team, in, g, t, s_ids, s_values);
    for (int v0 = team.lane() * N; v0 < in.V; v0 += kThreads * N) {
      float x[N] = {};
      if (!r.none) {
        load_row(row + v0, in.V - v0, x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = base_of<ENTROPY>(r, x[i], c);
      }
      store_row(out + v0, in.V - v0, x);
    }
    __syncthreads();  // (the marked tokens' values follow the others)
    if (!r.none) {
      for (int j = team.lane(); j < marked; j += kThreads) {
        const int32_t id = s_ids[j];
        if (id < 0) continue;
        float sum = 0.f;  // (a token marked twice: both write the same)
        for (int i = 0; i < marked; ++i) sum += s_ids[i] == id ? s_values[i] : 0.f;
        out[id] = (T)(base_of<ENTROPY>(r, (float)row[id], c) + sum);
      }
    }
    __syncthreads();
  }
}

dim3 row_blocks(int64_t rows) { return dim3((unsigned)std::min<int64_t>(rows, kMaxBlocks)); }

}  // namespace

hipError_t launch_logprobs_backward(const LogitsRows& in, const LogprobsGrads& g,
                                    void* grad_logits, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto entropy) {
      k_logits_gradient<T, entropy.value><<<row_blocks(in.rows), kThreads, 0, stream>>>(
          in, g, g.top != nullptr ? 1 + in.k : 1, static_cast<T*>(grad_logits),
          exponent_factor(in.scale));
    };
    if (g.of_entropy != nullptr) go(std::true_type{});
    else go(std::false_type{});
  });
  return hipGetLastError();
}

hipError_t launch_distill_backward(const LogitsRows& in, const float* grad_loss,
                                   const float* stats, void* grad_logits, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    k_logits_gradient<T, false><<<row_blocks(in.rows), kThreads, 0, stream>>>(
        in, DistillGrads{stats, grad_loss}, in.k, static_cast<T*>(grad_logits),
        exponent_factor(in.scale));
  });
  return hipGetLastError();
}

hipError_t launch_distill_step(const LogitsRows& in, const float* grad_loss, float* loss,
                               float* stats, void* grad_logits, void* workspace,
                               hipStream_t stream) {
  const hipError_t e = launch_distill_forward(in, loss, stats, workspace, stream);
  return e != hipSuccess ? e : launch_distill_backward(in, grad_loss, stats, grad_logits, stream);
}

}  // namespace bevpool
