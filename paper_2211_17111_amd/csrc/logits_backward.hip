// Gradients of the logits operators.  Both are, at logit v of a row,
//   e_v (A + B u_v) + sum of g_j over the row's marked tokens j that are v,
// e_v = 2^(u_v) = S p_v: what differs is A, B and the marked tokens (the given
// token and the alternatives, or the teacher's).

#include "logits.h"
#include "logits_rows.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // vectors of a thread in flight

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

// The teacher's share of a row's gradient, go the outgoing one.
template <class TEAM>
__device__ __forceinline__ void mark_taught(const TEAM& team, const LogitsRows& in, int64_t t,
                                            const Taught& q, float go, int32_t* ids, float* values) {
  for (int j = team.lane(); j < in.k; j += TEAM::kLanes) {
    float l;
    const int32_t id = slot_of(in, t, j, &l);
    ids[j] = id;
    values[j] = id >= 0 && l != -INFINITY ? -go * in.scale * expf(l - q.shift) : 0.f;
  }
}
__device__ __forceinline__ RowGradient taught_gradient(float m, float S, const Taught& q, float go,
                                                       float scale) {
  return RowGradient{m, scale * go * q.mass / S, 0.f, S == 0.f || go == 0.f || !q.any};
}

template <class TEAM>
__device__ __forceinline__ RowGradient gradient_of(const TEAM& team, const LogitsRows& in,
                                                   const DistillGrads& g, int64_t t, int32_t* ids,
                                                   float* values) {
  const Taught q = taught(team, in, t);
  mark_taught(team, in, t, q, g.loss[t], ids, values);
  return taught_gradient(g.stats[2 * t], g.stats[2 * t + 1], q, g.loss[t], in.scale);
}

template <bool ENTROPY>
__device__ __forceinline__ float base_of(const RowGradient& r, float x, float c) {
  const float u = (x - r.m) * c;
  const float e = __builtin_amdgcn_exp2f(u);
  return ENTROPY ? e * fmaf(r.B, held(u), r.A) : e * r.A;
}

// A whole vector of gradients.
template <typename T>
__device__ __forceinline__ void gradient_to(T* out, int i, const float (&x)[RowVec<T>::N]) {
  typename RowVec<T>::type raw;
#pragma unroll
  for (int e = 0; e < RowVec<T>::N; ++e) raw[e] = (T)x[e];
  *reinterpret_cast<typename RowVec<T>::type*>(out + i * RowVec<T>::N) = raw;
}

// The gradients behind a row's whole vectors, an element to a lane.
template <bool ENTROPY, typename T, class TEAM>
__device__ __forceinline__ void write_tail(const TEAM& team, const T* row, T* out,
                                           const RowGradient& r, int V, float c) {
  const int v = V / RowVec<T>::N * RowVec<T>::N + team.lane();
  if (v < V) out[v] = r.none ? (T)0.f : (T)base_of<ENTROPY>(r, (float)row[v], c);
}

// The marked tokens in [first, end), written over what they have without their
// marks.  (A token that is marked twice is written twice, with the same value.)
template <bool ENTROPY, typename T, class TEAM>
__device__ __forceinline__ void write_marked(const TEAM& team, const T* row, T* out,
                                             const RowGradient& r, const int32_t* ids,
                                             const float* values, int marked, int first, int end,
                                             float c) {
  for (int j = team.lane(); j < marked; j += TEAM::kLanes) {
    const int32_t id = ids[j];
    if (id < first || id >= end) continue;
    float sum = 0.f;
    for (int i = 0; i < marked; ++i) sum += ids[i] == id ? values[i] : 0.f;
    out[id] = (T)(base_of<ENTROPY>(r, (float)row[id], c) + sum);
  }
}

// Tokens and values of a team's marks, behind one another in LDS.
extern __shared__ int32_t s_marks[];

// ------------------------------------------------------------------ short rows

template <typename T, int L, int NV, bool ENTROPY, class G>
__global__ __launch_bounds__(kThreads) void k_short_gradient(LogitsRows in, G g, int marked,
                                                             T* __restrict__ grad, float c) {
  constexpr int N = RowVec<T>::N, kTeams = kThreads / L;
  const Team<L> team{nullptr};
  const int lane = team.lane(), whole = in.V / N;
  int32_t* ids = s_marks + threadIdx.x / L * 2 * marked;
  float* values = reinterpret_cast<float*>(ids + marked);
  for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < in.rows; t0 += (int64_t)gridDim.x * kTeams) {
    const int64_t t = t0 + threadIdx.x / L;
    if (t >= in.rows) break;  // (a wave's teams need one another nowhere)
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    Held<T, L, NV> held_row;
    held_row.load(row, in.V, lane);
    const RowGradient r = gradient_of(team, in, g, t, ids, values);
    held_row.each(lane, [&](const float (&x)[N], int i) {
      float y[N] = {};
      if (!r.none) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = base_of<ENTROPY>(r, x[e], c);
      }
      if (i < whole) gradient_to(out, i, y);
    });
    write_tail<ENTROPY>(team, row, out, r, in.V, c);
    if (!r.none) {
      team.sync();  // (the marked tokens' values follow the others)
      write_marked<ENTROPY>(team, row, out, r, ids, values, marked, 0, in.V, c);
    }
    team.sync();
  }
}

// ------------------------------------------------------------------- long rows

// A workgroup takes `length` vectors of a row, one of `parts`.
template <typename T, bool ENTROPY, class G>
__global__ __launch_bounds__(kThreads) void k_long_gradient(LogitsRows in, G g, int marked,
                                                            T* __restrict__ grad, float c,
                                                            int parts, int length) {
  constexpr int N = RowVec<T>::N;
  __shared__ float s_scratch[kThreads / kWave];
  const Team<kThreads> team{s_scratch};
  int32_t* ids = s_marks;
  float* values = reinterpret_cast<float*>(ids + marked);
  const int whole = in.V / N;
  for (int64_t b = blockIdx.x; b < in.rows * parts; b += gridDim.x) {
    const int64_t t = parts == 1 ? b : b / parts;
    const int first = (int)(b - t * parts) * length, end = min(first + length, whole);
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    const RowGradient r = gradient_of(team, in, g, t, ids, values);
    if (r.none) {
      const float zero[N] = {};
      for (int i = first + threadIdx.x; i < end; i += kThreads) gradient_to(out, i, zero);
    } else {
      for (int i0 = first + threadIdx.x; i0 < end; i0 += kThreads * kBatch) {
        typename RowVec<T>::type raw[kBatch] = {};
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int i = i0 + j * kThreads;
          if (i < end) raw[j] = *reinterpret_cast<const typename RowVec<T>::type*>(row + i * N);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int i = i0 + j * kThreads;
          float x[N];
          to_floats<T>(raw[j], x);
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = base_of<ENTROPY>(r, x[e], c);
          if (i < end) gradient_to(out, i, x);
        }
      }
    }
    const bool last = first + length >= whole;
    if (last) write_tail<ENTROPY>(team, row, out, r, in.V, c);
    __syncthreads();  // (the marked tokens' values follow the others)
    if (!r.none)
      write_marked<ENTROPY>(team, row, out, r, ids, values, marked, first * N, last ? in.V : end * N, c);
    __syncthreads();
  }
}

// ------------------------------------------------------------ loss and gradient

// Distillation's loss and gradient of rows that a team of L threads holds: the
// row is read once.
template <typename T, int L, int NV>
__global__ __launch_bounds__(L > kThreads ? L : kThreads) void k_distill_step(
    LogitsRows in, const float* __restrict__ grad_loss, float* __restrict__ loss,
    float* __restrict__ stats, T* __restrict__ grad, float c) {
  constexpr int N = RowVec<T>::N, kTeams = L > kThreads ? 1 : kThreads / L;
  __shared__ float s_scratch[L > kWave ? L / kWave : 1];
  const Team<L> team{s_scratch};
  const int lane = team.lane(), whole = in.V / N, marked = in.k;
  int32_t* ids = s_marks + (kTeams == 1 ? 0 : threadIdx.x / L * 2 * marked);
  float* values = reinterpret_cast<float*>(ids + marked);
  for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < in.rows; t0 += (int64_t)gridDim.x * kTeams) {
    const int64_t t = kTeams == 1 ? t0 : t0 + threadIdx.x / L;
    if (t >= in.rows) break;  // (only teams within a wave may lack a row)
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    Held<T, L, NV> held_row;
    held_row.load(row, in.V, lane);
    const Taught q = taught(team, in, t);
    const float go = grad_loss[t];
    mark_taught(team, in, t, q, go, ids, values);
    const Soft a = soft_of<false>(team, held_row, held_row.largest(), c);
    const Row p = row_of(a, in.scale);
    const RowGradient r = taught_gradient(p.m, p.S, q, go, in.scale);
    held_row.each(lane, [&](const float (&x)[N], int i) {
      float y[N] = {};
      if (!r.none) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = base_of<false>(r, x[e], c);
      }
      if (i < whole) gradient_to(out, i, y);
    });
    write_tail<false>(team, row, out, r, in.V, c);
    const float d = divergence(team, in, t, row, p, q);
    if (lane == 0) {
      loss[t] = d;
      stats[2 * t] = p.m;
      stats[2 * t + 1] = p.S;
    }
    team.sync();  // (the marked tokens' values follow the others)
    if (!r.none) write_marked<false>(team, row, out, r, ids, values, marked, 0, in.V, c);
    team.sync();
  }
}

// -------------------------------------------------------------------- launches

// Rows up to this many vectors are held by lanes.
constexpr int kShort = 512;

template <typename T, bool ENTROPY, class G>
void launch_gradient(const LogitsRows& in, const G& g, int marked, void* grad, hipStream_t stream) {
  const float c = exponent_factor(in.scale);
  const int vectors = vectors_of<T>(in.V);
  T* out = static_cast<T*>(grad);
  if (vectors <= kShort) {
    auto go = [&](auto lanes, auto held) {
      constexpr int kTeams = kThreads / lanes.value;
      const int64_t blocks = std::min<int64_t>((in.rows + kTeams - 1) / kTeams, kMaxBlocks);
      k_short_gradient<T, lanes.value, held.value, ENTROPY>
          <<<(unsigned)blocks, kThreads, kTeams * 8 * marked, stream>>>(in, g, marked, out, c);
    };
    constexpr std::integral_constant<int, 16> few;
    constexpr std::integral_constant<int, kWave> wave;
    if (vectors <= 16) go(few, std::integral_constant<int, 1>{});
    else if (vectors <= 32) go(few, std::integral_constant<int, 2>{});
    else if (vectors <= 64) go(few, std::integral_constant<int, 4>{});
    else if (vectors <= 128) go(wave, std::integral_constant<int, 2>{});
    else if (vectors <= 256) go(wave, std::integral_constant<int, 4>{});
    else go(wave, std::integral_constant<int, 8>{});
    return;
  }
  // (about four workgroups to a compute unit where rows are few)
  constexpr int kStep = kThreads * kBatch;
  const int batches = (vectors + kStep - 1) / kStep;  // (whole vectors, and a tail's place)
  const int want = (int)std::min<int64_t>((1024 + in.rows - 1) / in.rows, batches);
  const int length = (batches + want - 1) / want;
  const int parts = (batches + length - 1) / length;
  k_long_gradient<T, ENTROPY><<<(unsigned)std::min<int64_t>(in.rows * parts, kMaxBlocks), kThreads, 8 * marked, stream>>>(
      in, g, marked, out, c, parts, length * kStep);
}

}  // namespace

hipError_t launch_logprobs_backward(const LogitsRows& in, const LogprobsGrads& g,
                                    void* grad_logits, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  const int marked = g.top != nullptr ? 1 + in.k : 1;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    if (g.of_entropy != nullptr) launch_gradient<T, true>(in, g, marked, grad_logits, stream);
    else launch_gradient<T, false>(in, g, marked, grad_logits, stream);
  });
  return hipGetLastError();
}

hipError_t launch_distill_backward(const LogitsRows& in, const float* grad_loss,
                                   const float* stats, void* grad_logits, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    launch_gradient<decltype(t), false>(in, DistillGrads{stats, grad_loss}, in.k, grad_logits, stream);
  });
  return hipGetLastError();
}

hipError_t launch_distill_step(const LogitsRows& in, const float* grad_loss, float* loss,
                               float* stats, void* grad_logits, void* workspace,
                               hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  bool held = true;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    const int vectors = vectors_of<T>(in.V);
    auto go = [&](auto lanes, auto regs) {
      constexpr int L = lanes.value, kTeams = L > kThreads ? 1 : kThreads / L;
      const int64_t blocks = std::min<int64_t>((in.rows + kTeams - 1) / kTeams, kMaxBlocks);
      k_distill_step<T, L, regs.value><<<(unsigned)blocks, std::max(L, kThreads), kTeams * 8 * in.k, stream>>>(
          in, grad_loss, loss, stats, static_cast<T*>(grad_logits), exponent_factor(in.scale));
    };
    constexpr std::integral_constant<int, 16> few;
    constexpr std::integral_constant<int, kWave> wave;
    constexpr std::integral_constant<int, 256> block;
    constexpr std::integral_constant<int, 512> half;
    constexpr std::integral_constant<int, 1024> full;
    if (vectors <= 16) go(few, std::integral_constant<int, 1>{});
    else if (vectors <= 32) go(few, std::integral_constant<int, 2>{});
    else if (vectors <= 64) go(few, std::integral_constant<int, 4>{});
    else if (vectors <= 128) go(wave, std::integral_constant<int, 2>{});
    else if (vectors <= 256) go(wave, std::integral_constant<int, 4>{});
    else if (vectors <= 512) go(wave, std::integral_constant<int, 8>{});
    else if (vectors <= 1024) go(block, std::integral_constant<int, 4>{});
    else if (vectors <= 2048) go(block, std::integral_constant<int, 8>{});
    else if (vectors <= 4096) go(block, std::integral_constant<int, 16>{});
    else if (vectors <= 8192) go(half, std::integral_constant<int, 16>{});
    else if (vectors <= 16384) go(full, std::integral_constant<int, 16>{});
    else if (vectors <= 24576) go(full, std::integral_constant<int, 24>{});
    else held = false;
  });
  if (held) return hipGetLastError();
  const hipError_t e = launch_distill_forward(in, loss, stats, workspace, stream);
  return e != hipSuccess ? e : launch_distill_backward(in, grad_loss, stats, grad_logits, stream);
}

}  // namespace bevpool
