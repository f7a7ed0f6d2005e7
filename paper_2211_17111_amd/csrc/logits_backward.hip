// Gradients of the logits operators.  Both are, at logit v of a row,
//   e_v (A + B u_v) + sum of g_j over the row's marked tokens j that are v,
// e_v = 2^(u_v) = S p_v: what differs is A, B and the marked tokens (the given
// token and the alternatives, or the teacher's).
//
// A logit is read and its gradient written once, and that is what bounds them:
// 8192 rows of 65,536 bfloat16 take 412 us, 5.2 TB/s (a copy reaches 5.06); loss and
// gradient in one call read and write as much in 466.  The marked tokens are written
// again after their vectors.

#include "logits.h"
#include "logits_rows.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;    // vectors of a thread in flight
constexpr int kUnits = 256;  // compute units of the device

// The gradient of a row; `none`: zeros.
struct RowGradient {
  float m, A, B;
  bool none;
};

// Each of the following forms a row's gradient by a team, with its marked tokens
// and their g in LDS.
struct LogprobsGradient {
  LogprobsGrads g;

  template <class TEAM>
  __device__ __forceinline__ RowGradient of(const TEAM& team, const LogitsRows& in, int64_t t,
                                            int32_t* ids, float* values) const {
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
};

__device__ __forceinline__ RowGradient taught_gradient(float m, float S, const Taught& q, float go,
                                                       float scale) {
  return RowGradient{m, scale * go * q.mass / S, 0.f, S == 0.f || go == 0.f || !q.any};
}

// (KS slots to a lane)
template <int KS>
struct DistillGradient {
  const float *stats, *loss;  // loss: the outgoing gradient

  template <class TEAM>
  __device__ __forceinline__ RowGradient of(const TEAM& team, const LogitsRows& in, int64_t t,
                                            int32_t* ids, float* values) const {
    const float m = stats[2 * t], S = stats[2 * t + 1], go = loss[t];
    Slots<KS> slots;
    slots.load(team, in, t);
    slots.drop();
    const Taught q = taught(team, slots, in.renormalise);
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int j = i * TEAM::kLanes + team.lane();
      if (j >= in.k) continue;
      ids[j] = slots.id[i];
      values[j] = slot_gradient(slots, i, go, in.scale);
    }
    return taught_gradient(m, S, q, go, in.scale);
  }
};

template <bool ENTROPY>
__device__ __forceinline__ float base_of(const RowGradient& r, float x, float c) {
  const float u = (x - r.m) * c;
  const float e = __builtin_amdgcn_exp2f(u);
  return ENTROPY ? e * fmaf(r.B, held(u), r.A) : e * r.A;
}

// A whole vector of gradients.  STREAM: with the hint that it is not wanted again.
// Long rows take it, short ones do not; microseconds without and with it, forward
// and gradient: 2047 rows of 65,537 float16 199 and 172, 4096 of 131,072 bfloat16
// 655 and 608, 65,536 of 4096 422 and 439 (loss and gradient in one 288 and 325).
template <bool STREAM, typename T>
__device__ __forceinline__ void gradient_to(T* out, int i, const float (&x)[RowVec<T>::N]) {
  typename RowVec<T>::type raw;
#pragma unroll
  for (int e = 0; e < RowVec<T>::N; ++e) raw[e] = (T)x[e];
  auto* at = reinterpret_cast<typename RowVec<T>::type*>(out + i * RowVec<T>::N);
  if constexpr (STREAM) __builtin_nontemporal_store(raw, at);
  else *at = raw;
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

// The gradient of a row that a team holds.
template <bool ENTROPY, typename T, class TEAM, class H>
__device__ __forceinline__ void write_held(const TEAM& team, H& held_row, const T* row, T* out,
                                           const RowGradient& r, int V, float c) {
  const int whole = V / H::N;
  held_row.each(team.lane(), [&](const float (&x)[H::N], int i, int) {
    float y[H::N] = {};
    if (!r.none) {
#pragma unroll
      for (int e = 0; e < H::N; ++e) y[e] = base_of<ENTROPY>(r, x[e], c);
    }
    if (i < whole) gradient_to<false>(out, i, y);
  });
  write_tail<ENTROPY>(team, row, out, r, V, c);
}

template <typename T, int L, int NV, bool ENTROPY, class G>
__global__ __launch_bounds__(kThreads) void k_short_gradient(LogitsRows in, G g, int marked,
                                                             T* __restrict__ grad, float c) {
  constexpr int kTeams = kThreads / L;
  const Team<L> team{nullptr};
  int32_t* ids = s_marks + threadIdx.x / L * 2 * marked;
  float* values = reinterpret_cast<float*>(ids + marked);
  for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < in.rows; t0 += (int64_t)gridDim.x * kTeams) {
    const int64_t t = t0 + threadIdx.x / L;
    if (t >= in.rows) break;  // (a wave's teams need one another nowhere)
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    Held<T, L, NV> held_row;
    held_row.load(row, in.V, team.lane());
    const RowGradient r = g.of(team, in, t, ids, values);
    write_held<ENTROPY>(team, held_row, row, out, r, in.V, c);
    team.sync();  // (the marked tokens' values follow the others)
    if (!r.none) write_marked<ENTROPY>(team, row, out, r, ids, values, marked, 0, in.V, c);
    team.sync();
  }
}

// Distillation's loss and gradient of rows that teams of lanes hold, KS slots to a
// lane: the row is read once.
template <typename T, int L, int NV, int KS>
__global__ __launch_bounds__(kThreads) void k_short_step(LogitsRows in,
                                                         const float* __restrict__ grad_loss,
                                                         float* __restrict__ loss,
                                                         float* __restrict__ stats,
                                                         T* __restrict__ grad, float c) {
  constexpr int kTeams = kThreads / L;
  const Team<L> team{nullptr};
  const int lane = team.lane(), marked = in.k;
  int32_t* ids = s_marks + threadIdx.x / L * 2 * marked;
  float* values = reinterpret_cast<float*>(ids + marked);
  for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < in.rows; t0 += (int64_t)gridDim.x * kTeams) {
    const int64_t t = t0 + threadIdx.x / L;
    if (t >= in.rows) break;  // (a wave's teams need one another nowhere)
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    Slots<KS> slots;
    slots.load(team, in, t);
    const float go = grad_loss[t];
    Held<T, L, NV> held_row;
    held_row.load(row, in.V, lane);
    slots.drop();
    slots.load_logits(row);
    const Taught q = taught(team, slots, in.renormalise);
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int j = i * L + lane;
      if (j >= marked) continue;
      ids[j] = slots.id[i];
      values[j] = slot_gradient(slots, i, go, in.scale);
    }
    const Soft a = soft_of<false>(team, held_row, held_row.largest(team.lane()), c);
    const Row p = row_of(a, in.scale);
    const RowGradient r = taught_gradient(p.m, p.S, q, go, in.scale);
    write_held<false>(team, held_row, row, out, r, in.V, c);
    const float d = divergence(team, slots, p);
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

// ------------------------------------------------------------------- long rows

// Elements of a row of V before the first that begins a cache line (fewer than 64).
// Long gradients are written in vectors from there on, and these one by one: rows
// of any length begin anywhere, and waves whose stores share lines cost 2047 rows of
// 65,537 float16 120 us where whole lines take 108 (65,536: 107).
template <typename T>
__device__ __forceinline__ int head_of(const T* row, int V) {
  constexpr int kLine = 128;
  const int off = (int)(reinterpret_cast<uintptr_t>(row) % kLine / sizeof(T));
  return off == 0 ? 0 : min(V, kLine / (int)sizeof(T) - off);
}

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
  for (int64_t b = blockIdx.x; b < in.rows * parts; b += gridDim.x) {
    // (from the last row: what the forward read last is still in the memory-side
    // cache; 2999 rows of 50,021 float16, forward and gradient, 211 us from the
    // first and 206 from the last)
    const int64_t back = in.rows * parts - 1 - b;
    const int64_t t = parts == 1 ? back : back / parts;
    const int part = (int)(back - t * parts);
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    // the gradient's vectors begin behind its head, which is the first part's
    const int head = head_of(out, in.V), whole = (in.V - head) / N;
    const T* body = row + head;
    T* to = out + head;
    // (behind the head there may be nothing left for the last part but the tail)
    const int first = min(part * length, whole), end = min(first + length, whole);
    const RowGradient r = g.of(team, in, t, ids, values);
    if (part == 0 && (int)threadIdx.x < head)
      out[threadIdx.x] = r.none ? (T)0.f : (T)base_of<ENTROPY>(r, (float)row[threadIdx.x], c);
    if (r.none) {
      const float zero[N] = {};
      for (int i = first + threadIdx.x; i < end; i += kThreads) gradient_to<true>(to, i, zero);
    } else {
      for (int i0 = first + threadIdx.x; i0 < end; i0 += kThreads * kBatch) {
        typename RowVec<T>::type raw[kBatch] = {};
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int i = i0 + j * kThreads;
          if (i < end) raw[j] = *reinterpret_cast<const typename RowVec<T>::type*>(body + i * N);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int i = i0 + j * kThreads;
          float x[N];
          to_floats<T>(raw[j], x);
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = base_of<ENTROPY>(r, x[e], c);
          if (i < end) gradient_to<true>(to, i, x);
        }
      }
    }
    const bool last = part == parts - 1;
    if (last) write_tail<ENTROPY>(team, body, to, r, in.V - head, c);
    __syncthreads();  // (the marked tokens' values follow the others)
    if (!r.none)
      write_marked<ENTROPY>(team, row, out, r, ids, values, marked, part == 0 ? 0 : head + first * N,
                            last ? in.V : head + end * N, c);
    __syncthreads();
  }
}

// Distillation's loss and gradient of rows that a workgroup of L threads holds.  One
// of 1024 has a compute unit for itself, so it overlaps its own rows: as soon as a
// vector's gradient is formed, the vector of its next row is on its way into the
// same registers.  Nothing in between waits for memory: barriers order LDS only,
// and a marked token's gradient is written by the thread that wrote its vector.
template <typename T, int L, int NV>
__global__ __launch_bounds__(L) void k_long_step(LogitsRows in, const float* __restrict__ grad_loss,
                                                 float* __restrict__ loss,
                                                 float* __restrict__ stats, T* __restrict__ grad,
                                                 float c) {
  static_assert(L >= kMaxTaught, "a slot to a thread");
  constexpr int N = RowVec<T>::N;
  __shared__ float s_scratch[L / kWave];
  __shared__ int32_t s_first[L];  // of every thread's marks, and the next of each; -1 behind the last
  __shared__ int32_t s_next[kMaxTaught], s_ids[kMaxTaught];
  __shared__ float s_values[kMaxTaught], s_gradients[kMaxTaught];
  const Team<L> team{s_scratch};
  const int tid = threadIdx.x, whole = in.V / N, k = in.k;
  const T* logits = static_cast<const T*>(in.logits);
  int64_t t = blockIdx.x;
  Slots<1> slots;
  slots.load(team, in, t);
  float go = grad_loss[t];
  Held<T, L, NV> held_row;
  held_row.load(logits + t * in.stride, in.V, tid);
  for (;;) {
    const T* row = logits + t * in.stride;
    T* out = grad + t * (int64_t)in.V;
    slots.drop();
    slots.load_logits(row);
    const int32_t id = slots.id[0];
    s_first[tid] = -1;
    const Taught q = taught(team, slots, in.renormalise);
    if (tid < k) {
      s_ids[tid] = id;
      s_values[tid] = slot_gradient(slots, 0, go, in.scale);
    }
    const Soft a = soft_of<false>(team, held_row, held_row.largest(team.lane()), c);
    const Row p = row_of(a, in.scale);
    const RowGradient r = taught_gradient(p.m, p.S, q, go, in.scale);
    if (tid < k && id >= 0 && !r.none) {
      float sum = 0.f;  // (an id that occurs again: both have the same)
      for (int i = 0; i < k; ++i) sum += s_ids[i] == id ? s_values[i] : 0.f;
      s_gradients[tid] = base_of<false>(r, slots.x[0], c) + sum;
      s_next[tid] = atomicExch(&s_first[id < whole * N ? id / N % L : id - whole * N], tid);
    }
    const float d = divergence(team, slots, p);
    if (tid == 0) {
      loss[t] = d;
      stats[2 * t] = p.m;
      stats[2 * t + 1] = p.S;
    }
    const int64_t next = t + gridDim.x;
    const bool more = next < in.rows;
    const T* next_row = logits + (more ? next : t) * in.stride;
    if (more) {
      slots.load(team, in, next);
      go = grad_loss[next];
    }
    lds_barrier();  // (the marks are complete)
    int lane = tid;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (held_row.asked(j) && j * L >= whole) break;
      float x[N];
      held_row.part(j, lane, x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = r.none ? 0.f : base_of<false>(r, x[e], c);
      if (j * L + lane < whole) gradient_to<true>(out, j * L + lane, x);
      if (more) held_row.load_part(j, next_row, lane);
    }
    write_tail<false>(team, row, out, r, in.V, c);
    for (int j = s_first[tid]; j >= 0; j = s_next[j]) out[s_ids[j]] = (T)s_gradients[j];
    if (!more) break;
    held_row.load_tail(next_row, in.V);
    t = next;
    lds_barrier();  // (the marks have been read)
  }
}

// -------------------------------------------------------------------- launches

// Rows up to this many vectors are held by lanes.
constexpr int kShort = 512;

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f with the lanes to a row and the vectors of each; 16 lanes only for rows
// with few marks.
template <class F>
void by_length(int vectors, bool few_marks, F f) {
  if (few_marks && vectors <= 16) f(Int<16>{}, Int<1>{});
  else if (few_marks && vectors <= 32) f(Int<16>{}, Int<2>{});
  else if (few_marks && vectors <= 64) f(Int<16>{}, Int<4>{});
  else if (vectors <= 128) f(Int<kWave>{}, Int<2>{});
  else if (vectors <= 256) f(Int<kWave>{}, Int<4>{});
  else f(Int<kWave>{}, Int<8>{});
}

// Whether a short row has four slots to a lane instead of one: up to 32 of a row that
// 16 lanes hold, or up to 256 of one that a wave does.  (Loss and gradient of 28,133
// rows of 118 float32, by a wave and by 16 lanes: with 29 slots 34 us and 22, with 64
// 47 and 51.)
template <typename T>
bool four_slots(const LogitsRows& in) {
  static_assert(4 * kWave == kMaxTaught, "slots of a wave");
  return in.k > kWave || (in.k > 16 && in.k <= 32 && vectors_of<T>(in.V) <= 64);
}

template <int L>
unsigned team_blocks(int64_t rows) {
  constexpr int kTeams = kThreads / L;
  return (unsigned)std::min<int64_t>((rows + kTeams - 1) / kTeams, kMaxBlocks);
}

template <typename T, bool ENTROPY, class G>
void launch_short_gradient(const LogitsRows& in, const G& g, bool few_marks, int marked, void* grad,
                           hipStream_t stream) {
  by_length(vectors_of<T>(in.V), few_marks, [&](auto l, auto v) {
    constexpr int L = l.value;
    k_short_gradient<T, L, v.value, ENTROPY><<<team_blocks<L>(in.rows), kThreads, kThreads / L * 8 * marked, stream>>>(
        in, g, marked, static_cast<T*>(grad), exponent_factor(in.scale));
  });
}

template <typename T, bool ENTROPY, class G>
void launch_long_gradient(const LogitsRows& in, const G& g, int marked, void* grad, hipStream_t stream) {
  // (about four workgroups to a compute unit where rows are few)
  constexpr int kStep = kThreads * kBatch;
  const int batches = (vectors_of<T>(in.V) + kStep - 1) / kStep;
  const int want = (int)std::min<int64_t>((4 * kUnits + in.rows - 1) / in.rows, batches);
  const int length = (batches + want - 1) / want;
  const int parts = (batches + length - 1) / length;
  k_long_gradient<T, ENTROPY><<<(unsigned)std::min<int64_t>(in.rows * parts, kMaxBlocks), kThreads, 8 * marked, stream>>>(
      in, g, marked, static_cast<T*>(grad), exponent_factor(in.scale), parts, length * kStep);
}

}  // namespace

hipError_t launch_logprobs_backward(const LogitsRows& in, const LogprobsGrads& g,
                                    void* grad_logits, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  const int marked = g.top != nullptr ? 1 + in.k : 1;
  const LogprobsGradient own{g};
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto entropy) {
      if (vectors_of<T>(in.V) <= kShort)
        launch_short_gradient<T, entropy.value>(in, own, marked <= 17, marked, grad_logits, stream);
      else
        launch_long_gradient<T, entropy.value>(in, own, marked, grad_logits, stream);
    };
    if (g.of_entropy != nullptr) go(std::true_type{});
    else go(std::false_type{});
  });
  return hipGetLastError();
}

hipError_t launch_distill_backward(const LogitsRows& in, const float* grad_loss,
                                   const float* stats, void* grad_logits, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  const DistillGradient<1> own{stats, grad_loss};
  const DistillGradient<4> four{stats, grad_loss};
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    if (vectors_of<T>(in.V) > kShort) launch_long_gradient<T, false>(in, own, in.k, grad_logits, stream);
    else if (four_slots<T>(in)) launch_short_gradient<T, false>(in, four, in.k <= 32, in.k, grad_logits, stream);
    else launch_short_gradient<T, false>(in, own, in.k <= 16, in.k, grad_logits, stream);
  });
  return hipGetLastError();
}

hipError_t launch_distill_step(const LogitsRows& in, const float* grad_loss, float* loss,
                               float* stats, void* grad_logits, void* workspace,
                               hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  const float c = exponent_factor(in.scale);
  bool held = true;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    T* grad = static_cast<T*>(grad_logits);
    auto lanes = [&](auto slots, bool few_marks) {
      by_length(vectors_of<T>(in.V), few_marks, [&](auto l, auto v) {
        constexpr int L = l.value;
        k_short_step<T, L, v.value, slots.value><<<team_blocks<L>(in.rows), kThreads, kThreads / L * 8 * in.k, stream>>>(
            in, grad_loss, loss, stats, grad, c);
      });
    };
    auto block = [&](auto l, auto v) {
      constexpr int L = l.value;
      const int64_t blocks = std::min<int64_t>(in.rows, kUnits * (1024 / L));  // (held at once)
      k_long_step<T, L, v.value><<<(unsigned)blocks, L, 0, stream>>>(in, grad_loss, loss, stats, grad, c);
    };
    const int vectors = vectors_of<T>(in.V);
    if (vectors <= kShort) {
      if (four_slots<T>(in)) lanes(Int<4>{}, in.k <= 32);
      else lanes(Int<1>{}, in.k <= 16);
    } else if (vectors <= 1024) block(Int<256>{}, Int<4>{});
    else if (vectors <= 2048) block(Int<256>{}, Int<8>{});
    else if (vectors <= 4096) block(Int<256>{}, Int<16>{});
    else if (vectors <= 8192) block(Int<512>{}, Int<16>{});
    else if (vectors <= 16384 && in.rows >= 2 * kUnits) block(Int<1024>{}, Int<16>{});
    else held = false;
  });
  if (held) return hipGetLastError();
  const hipError_t e = launch_distill_forward(in, loss, stats, workspace, stream);
  return e != hipSuccess ? e : launch_distill_backward(in, grad_loss, stats, grad_logits, stream);
}

}  // namespace bevpool
