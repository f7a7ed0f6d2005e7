// Device helpers of the logits operators: teams of threads that share a row,
// softmax statistics that are joined, and what a row's values are made of.
//
// Everything that depends on a row goes through differences from its largest
// logit m, so that no value is lost to the logits' size: terms e^(scale (x - m))
// are taken as 2^u, u = (x - m) (scale log2 e), and a log probability is
// scale (x - m) - log S.
#pragma once

#include <hip/hip_runtime.h>
#include <float.h>
#include <stdint.h>

#include "device_utils.h"
#include "logits.h"
#include "rows_vec.h"

namespace bevpool {

constexpr float kLn2 = 0.693147181f;

// A team of L threads (a power of two): within a wave up to 64, a workgroup
// above.  `scratch`: LDS, a float for every wave of a workgroup's team.
template <int L>
struct Team {
  static constexpr int kLanes = L;
  static constexpr bool kBlock = L > kWave;
  static constexpr int kWaves = kBlock ? L / kWave : 1;
  float* scratch;

  __device__ __forceinline__ int lane() const { return threadIdx.x % L; }
  // Orders the team's accesses to LDS.
  __device__ __forceinline__ void sync() const {
    if constexpr (kBlock) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
  // f over all threads (f commutes), the same in each.
  template <class F>
  __device__ __forceinline__ float reduce(float v, F f) const {
    constexpr int W = kBlock ? kWave : L;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, kWave));
    if constexpr (kBlock) {
      if (lane_id() == 0) scratch[threadIdx.x / kWave] = v;
      lds_barrier();
      v = scratch[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v = f(v, scratch[w]);
      lds_barrier();  // (the scratch may be written again)
    }
    return v;
  }
  __device__ __forceinline__ float sum(float v) const {
    return reduce(v, [](float a, float b) { return a + b; });
  }
  __device__ __forceinline__ float max(float v) const {
    return reduce(v, [](float a, float b) { return fmaxf(a, b); });
  }
};

// Statistics of some of a row's logits: the largest (r, NaN not counted), the
// sum s of 2^u with u = c (x - r), and the sum w of u 2^u.  r begins at the
// lowest number, from which -inf lies at -inf: nothing but -inf leaves s at 0.
struct Soft {
  float r, s, w;
};
constexpr float kLowest = -FLT_MAX;
__device__ __forceinline__ Soft no_soft() { return Soft{kLowest, 0.f, 0.f}; }

// u, held where 2^u is 0 anyway, so that u 2^u is 0 there (a NaN stays one).
__device__ __forceinline__ float held(float u) {
  return __builtin_elementwise_maximum(u, -256.f);
}

// The statistics as seen from r (no smaller than a.r).
__device__ __forceinline__ Soft seen_from(const Soft& a, float r, float c) {
  const float u = held((a.r - r) * c);
  const float f = __builtin_amdgcn_exp2f(u);
  return Soft{r, a.s * f, fmaf(u, a.s, a.w) * f};
}

// Joins a team's statistics: the same in each thread.
template <bool ENTROPY, class TEAM>
__device__ __forceinline__ Soft join(const TEAM& team, Soft a, float c) {
  a = seen_from(a, team.max(a.r), c);
  a.s = team.sum(a.s);
  if constexpr (ENTROPY) a.w = team.sum(a.w);
  return a;
}

// Adds N logits (-inf for none); the largest of them.
template <bool ENTROPY, int N>
__device__ __forceinline__ float add(Soft& a, const float (&x)[N], float c) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
  if (top > a.r) {
    if constexpr (ENTROPY) {
      a = seen_from(a, top, c);
    } else {
      a.s *= __builtin_amdgcn_exp2f((a.r - top) * c);
      a.r = top;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float u = (x[i] - a.r) * c;
    const float e = __builtin_amdgcn_exp2f(u);
    a.s += e;
    if constexpr (ENTROPY) a.w = fmaf(e, held(u), a.w);
  }
  return top;
}

// Vector i of a row of V logits, -inf past its end.
template <typename T>
__device__ __forceinline__ typename RowVec<T>::type logits_at(const T* row, int i, int V) {
  using W = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N;
  if (i < V / N) return *reinterpret_cast<const W*>(row + i * N);
  W raw;
#pragma unroll
  for (int e = 0; e < N; ++e) raw[e] = i * N + e < V ? row[i * N + e] : (T)-INFINITY;
  return raw;
}
template <typename T>
inline __host__ __device__ int vectors_of(int64_t V) {
  return (int)((V + RowVec<T>::N - 1) / RowVec<T>::N);
}

template <typename T>
__device__ __forceinline__ void to_floats(const typename RowVec<T>::type& raw, float* x) {
#pragma unroll
  for (int e = 0; e < RowVec<T>::N; ++e) x[e] = (float)raw[e];
}

// A row of at most L NV vectors in the registers of a team: vector j L + l in
// part j of lane l; what lies behind the row's whole vectors is put in its place,
// and -inf behind the row's end, where a part is used.  Several passes go over the
// row; what one has converted is not to be kept for the next (it would take twice
// the registers), nor every vector's place, so each part begins with values that
// the compiler cannot know to be the same.
template <typename T, int L, int NV>
struct Held {
  static constexpr int N = RowVec<T>::N;
  typedef int32_t Raw __attribute__((ext_vector_type(4)));
  Raw raw[NV], tail;
  int whole, vectors;

  // Whether part j is asked if it holds logits: each is where several workgroups
  // share a compute unit (fewer registers, and short rows do nothing for the parts
  // that they lack), every fourth where one of 1024 threads has it for itself and
  // needs its parts to overlap.  Loss and gradient of bfloat16 rows, microseconds,
  // each / every fourth: 8192 of 65,536 (512 threads) 489 and 611, 4096 of 131,072
  // (1024 threads) 608 and 556.
  static constexpr bool asked(int j) { return L < 1024 || j % 4 == 0; }
  // (vectors behind the last whole one load that one; a row must have one)
  __device__ __forceinline__ void load_part(int j, const T* row, int lane) {
    raw[j] = __builtin_bit_cast(
        Raw, *reinterpret_cast<const typename RowVec<T>::type*>(row + min(j * L + lane, whole - 1) * N));
  }
  __device__ __forceinline__ void load_tail(const T* row, int V) {
    tail = __builtin_bit_cast(Raw, logits_at(row, whole, V));
  }
  __device__ __forceinline__ void load(const T* row, int V, int lane) {
    whole = V / N;
    vectors = vectors_of<T>(V);
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = Raw{};
    load_tail(row, V);
    if (whole == 0) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (asked(j) && j * L >= whole) break;
      load_part(j, row, lane);
    }
  }
  __device__ __forceinline__ void part(int j, int& lane, float (&x)[N]) {
    __asm__ volatile("" : "+v"(raw[j]), "+v"(lane));
    Raw own = raw[j];
    if ((j + 1) * L > whole) {
      typename RowVec<T>::type none;
#pragma unroll
      for (int e = 0; e < N; ++e) none[e] = (T)-INFINITY;
      const int i = j * L + lane;
      own = i < whole ? own : i == whole ? tail : __builtin_bit_cast(Raw, none);
    }
    to_floats<T>(__builtin_bit_cast(typename RowVec<T>::type, own), x);
  }
  // f(x[N], vector, part) for every part of the row, also for lanes behind its end.
  template <class F>
  __device__ __forceinline__ void each(int lane, F f) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (asked(j) && j * L >= vectors) break;
      float x[N];
      part(j, lane, x);
      f(x, j * L + lane, j);
    }
  }
  // The largest logit of this lane, -inf for none (NaN not counted).
  __device__ __forceinline__ float largest(int lane) {
    float m = -INFINITY;
    each(lane, [&](const float (&x)[N], int, int) {
#pragma unroll
      for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    });
    return m;
  }
};

// The statistics of a held row, the same in each thread; `largest` of this lane.
template <bool ENTROPY, class TEAM, class H>
__device__ __forceinline__ Soft soft_of(const TEAM& team, H& held_row, float largest, float c) {
  Soft a{fmaxf(team.max(largest), kLowest), 0.f, 0.f};
  held_row.each(team.lane(), [&](const float (&x)[H::N], int, int) {
#pragma unroll
    for (int i = 0; i < H::N; ++i) {
      const float u = (x[i] - a.r) * c;
      const float e = __builtin_amdgcn_exp2f(u);
      a.s += e;
      if constexpr (ENTROPY) a.w = fmaf(e, held(u), a.w);
    }
  });
  a.s = team.sum(a.s);
  if constexpr (ENTROPY) a.w = team.sum(a.w);
  return a;
}

// A row's distribution from its statistics: S is 0 for a row without one.
struct Row {
  float m, S, log_S, scale;
  __device__ __forceinline__ float logprob(float x) const {
    return S == 0.f ? -INFINITY : fmaf(scale, x - m, -log_S);
  }
};
__device__ __forceinline__ Row row_of(float m, float S, float scale) {
  return Row{m, S, S == 0.f ? -INFINITY : logf(S), scale};
}
// (a row that only -inf and NaN are in leaves r where it began)
__device__ __forceinline__ Row row_of(const Soft& a, float scale) {
  return row_of(a.s > 0.f || a.r > kLowest ? a.r : -INFINITY, a.s, scale);
}

// Id i of an array of int32 or int64 ids, -1 when outside [0, V).
__device__ __forceinline__ int32_t id_at(const void* ids, int key_type, int64_t i, int32_t V) {
  const int32_t v = key_type == BEVPOOL_KEY_I32
                        ? key_or_drop(static_cast<const int32_t*>(ids), i, V)
                        : key_or_drop(static_cast<const int64_t*>(ids), i, V);
  return v < V ? v : -1;
}

// A row's alternatives by their teacher, slot j in place j / L of lane j % L, and
// the student's logits for them: -1, -inf and 0 for a slot without an id.
template <int KS>
struct Slots {
  int32_t id[KS];
  float l[KS];  // log q: the teacher's log probability
  float x[KS];

  template <class TEAM>
  __device__ __forceinline__ void load(const TEAM& team, const LogitsRows& in, int64_t t) {
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int j = i * TEAM::kLanes + team.lane();
      id[i] = j < in.k ? id_at(in.ids, in.key_type, t * in.k + j, in.V) : -1;
      l[i] = j < in.k ? in.teacher[t * in.k + j] : -INFINITY;
    }
  }
  // (apart from their loading, so that it waits for nothing)
  __device__ __forceinline__ void drop() {
#pragma unroll
    for (int i = 0; i < KS; ++i) l[i] = id[i] >= 0 ? l[i] : -INFINITY;
  }
  template <typename T>
  __device__ __forceinline__ void load_logits(const T* row) {
#pragma unroll
    for (int i = 0; i < KS; ++i) x[i] = id[i] >= 0 ? (float)row[id[i]] : 0.f;
  }
};

// A teacher's side of a row: the sum of q_j = e^(l_j) and whether any slot is kept.
struct Taught {
  float mass;
  bool any;
};

// (Renormalised, l_j becomes its difference from the row's largest, less the log of
// the sum: two subtractions, since the sum of largest and log would be rounded by
// 2^-24 of what is added to all l_j, which has no part.)
template <class TEAM, int KS>
__device__ __forceinline__ Taught taught(const TEAM& team, Slots<KS>& slots, bool renormalise) {
  float top = -INFINITY, sum = 0.f, some = 0.f;
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    top = fmaxf(top, slots.l[i]);
    some = slots.l[i] == -INFINITY ? some : 1.f;  // (a NaN is some)
  }
  some = team.max(some);
  if (renormalise) {
    top = team.max(top);
    top = top > -INFINITY ? top : 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) slots.l[i] -= top;
  }
#pragma unroll
  for (int i = 0; i < KS; ++i) sum += expf(slots.l[i]);
  sum = team.sum(sum);
  if (renormalise && some > 0.f) {
    const float log_sum = logf(sum);
#pragma unroll
    for (int i = 0; i < KS; ++i) slots.l[i] -= log_sum;
    sum = sum == sum ? 1.f : sum;
  }
  return Taught{sum, some > 0.f};
}

// Divergence of the row's distribution from the teacher's.  (The difference of
// the log probabilities is taken in 64 bits: a student's that is beyond float32,
// for a logit of the type's lowest number, may have a small share.)
template <class TEAM, int KS>
__device__ __forceinline__ float divergence(const TEAM& team, const Slots<KS>& slots, const Row& p) {
  float loss = 0.f;
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    if (slots.l[i] == -INFINITY) continue;
    const float own = expf(slots.l[i]);
    const double behind = (double)p.scale * ((double)p.m - (double)slots.x[i]);
    if (own != 0.f)
      loss += p.S == 0.f ? INFINITY : (float)(own * (slots.l[i] + behind + p.log_S));
  }
  return team.sum(loss);
}

// What a slot adds to its token's gradient, go the row's outgoing one.
template <int KS>
__device__ __forceinline__ float slot_gradient(const Slots<KS>& slots, int i, float go, float scale) {
  return slots.l[i] == -INFINITY ? 0.f : -go * scale * expf(slots.l[i]);
}

}  // namespace bevpool
