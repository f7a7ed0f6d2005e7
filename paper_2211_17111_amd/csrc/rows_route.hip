// Router of expert layers: the k largest logits of every token and their
// softmax weights, and the logits' gradient.
//
// A group of L lanes takes a row (16 lanes up to 256 experts, a whole wave
// above) and holds its logits in registers, V to a lane, so the row is read
// once, in vectors.  Values are exchanged by rotations within 16 lanes (DPP, at
// the rate of plain vector instructions).  What bounds the forward is
// instructions: 640 vector, 130 scalar and 23 LDS ones a wave of four rows of 256
// logits (k = 8, softmax over all experts, counted).  So there are two ways to the k largest:
//   - k rounds that each find and strike out the largest;
//   - a list of the few logits that can be among them, ranked pair by pair.
// Microseconds of the forward, 32,768 rows of float32, weights renormalised,
// launches back to back in a graph,
// rounds / list:        k = 2       4          8          12         16
//   256 experts       7.3 / 8.1  9.4 / 8.4  14.3 / 9.9  19.2 / 15.3  24.1 / 26.8
//   64 experts        4.1 / 4.6  5.1 / 4.7   7.0 / 5.7   8.9 / 7.4   10.8 / 11.7
// so 4 to 12 choices take the list (33.5 MB of logits take 7 us).  Over all
// experts instead of renormalised: 11.2 for 9.9.  384 and 512 experts, k = 8, take
// 31 by rounds of a whole wave.
//
// The gradient needs no second softmax: the first chosen expert's weight is
// exp(0) / sum, so p_e = exp(l_e - l_first) w_first.  The chosen experts' terms
// go to their places through LDS.  13.4 us for the same rows (67 MB), 8.3 where the
// weights are renormalised and no logit is read.

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxChosen = 64;
constexpr int kListFrom = 4, kListTo = 12;  // choices that are listed, see above

// Floats as unsigned integers in their order, +0 and -0 the same; kNone, below
// all of them, for what is never chosen (-inf, NaN) or already taken.
constexpr uint32_t kNone = 0;
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // (-0 + 0 = +0)
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return v > -INFINITY ? o : kNone;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

// e^d for d <= 0.  The hardware's exponential gives no subnormal numbers, so it
// is taken of half the exponent, h = d log2(e) / 2, and squared.  h is rounded to
// 24 bits, which alone would be a relative error that grows with |d|: the rest
// r = d - 2 ln(2) h is what one step of the constant and of h leave, and e^r is
// 1 + r to far below a rounding.  Measured error of a weight e^d / (1 + e^d):
// at most 5.7 x 2^-24 for d from -1 to -85 (without r: 18 at -20, 65 at -85).
// d is held where e^d is 0 already, so that r stays finite; a NaN stays one.
__device__ __forceinline__ float exp_of(float d) {
  constexpr double k2Ln2 = 1.3862943611198906;
  constexpr float kHigh = (float)k2Ln2, kLow = (float)(k2Ln2 - (double)kHigh);
  d = __builtin_elementwise_maximum(d, -256.f);
  const float h = d * 0.72134752f;
  const float r = fmaf(h, -kLow, fmaf(h, -kHigh, d));
  const float p = __builtin_amdgcn_exp2f(h);
  return p * fmaf(p, r, p);
}

// The value of the lane ROR lanes on, within 16 lanes.
template <int ROR, class T>
__device__ __forceinline__ T rotate16(T v) {
  static_assert(sizeof(T) == 4, "one register");
  const int r = __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + ROR, 0xf, 0xf, true);
  return __builtin_bit_cast(T, r);
}

// The value of the lane N lanes below, within 16 lanes; 0 where there is none.
template <int N>
__device__ __forceinline__ int shift16(int v) {
  return __builtin_amdgcn_update_dpp(0, v, 0x110 + N, 0xf, 0xf, true);
}

// Orders the wave's accesses to LDS that its lanes exchange.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// f over all lanes of a group, the same in each (f commutes, and every level
// pairs the same values on both sides).
template <int L, class T, class F>
__device__ __forceinline__ T group_reduce(T v, F f) {
  v = f(v, rotate16<8>(v));
  v = f(v, rotate16<4>(v));
  v = f(v, rotate16<2>(v));
  v = f(v, rotate16<1>(v));
  if constexpr (L == kWave) {
    v = f(v, __shfl_xor(v, 16, kWave));
    v = f(v, __shfl_xor(v, 32, kWave));
  }
  return v;
}

template <int L>
__device__ __forceinline__ float group_sum(float v) {
  return group_reduce<L>(v, [](float a, float b) { return a + b; });
}

template <int L>
__device__ __forceinline__ bool group_any(bool v) {
  const uint64_t m = wave_ballot(v);
  if constexpr (L == kWave) return m != 0;
  return (m >> (threadIdx.x % kWave / L * L) & ((uint64_t(1) << L) - 1)) != 0;
}

// The logits of lane l: runs of B neighbours, so that a lane loads vectors and
// the group's are next to each other.  Register i holds expert first(l) +
// offset(i).
template <typename T, int L, int V>
struct Held {
  static constexpr int B = V < RowVec<T>::N ? V : RowVec<T>::N;
  typedef T Run __attribute__((ext_vector_type(B)));
  __device__ static __forceinline__ int offset(int i) { return i / B * L * B + i % B; }
  __device__ static __forceinline__ int first(int l) { return l * B; }
  __device__ static __forceinline__ void load(const T* row, int E, int l, float (&x)[V]) {
#pragma unroll
    for (int b = 0; b < V; b += B) {
      const int e0 = first(l) + offset(b);
      if (e0 + B <= E) {
        Run t;
        __builtin_memcpy(&t, row + e0, sizeof(t));
#pragma unroll
        for (int i = 0; i < B; ++i) x[b + i] = (float)t[i];
      } else {
#pragma unroll
        for (int i = 0; i < B; ++i) x[b + i] = e0 + i < E ? (float)row[e0 + i] : -INFINITY;
      }
    }
  }
  __device__ static __forceinline__ void store(T* row, int E, int l, const float (&x)[V]) {
#pragma unroll
    for (int b = 0; b < V; b += B) {
      const int e0 = first(l) + offset(b);
      if (e0 + B <= E) {
        Run t;
#pragma unroll
        for (int i = 0; i < B; ++i) t[i] = (T)x[b + i];
        __builtin_memcpy(row + e0, &t, sizeof(t));
      } else {
#pragma unroll
        for (int i = 0; i < B; ++i)
          if (e0 + i < E) row[e0 + i] = (T)x[b + i];
      }
    }
  }
};

// A logit's order and its expert in one number: larger logits are larger, of
// equal ones the lower expert is.
__device__ __forceinline__ uint64_t pair_of(uint32_t order, int e) {
  return ((uint64_t)order << 32) | (uint32_t)~e;
}

// Number of the 16 lanes whose value is no smaller than this one's.
template <int R = 15>
__device__ __forceinline__ int lanes_ahead(uint32_t v) {
  if constexpr (R == 0) return 1;
  else return (rotate16<R>(v) >= v) + lanes_ahead<R - 1>(v);
}

// The chosen of a group's row, spread over its lanes: in register q of a lane
// the logit's order (kNone: nothing), its expert and its place among the k.
template <int Q>
struct Chosen {
  uint32_t order[Q];
  int32_t id[Q];
  int32_t place[Q];
};

// Most candidates of a row that choose_listed ranks.
constexpr int kListed = 32;

// Any k: k rounds take the largest logit and, of equal ones, the lowest expert,
// each by a reduction over the group, and strike it out.  Chosen j is lane
// j % L's, in register j / L.
template <int L, int V, class H, int Q>
__device__ __forceinline__ void choose_in_rounds(uint32_t (&o)[V], int k, int lane, Chosen<Q>& c) {
  const int base = H::first(lane);
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    c.order[q] = kNone;
    c.id[q] = -1;
    c.place[q] = q * L + lane;
  }
#pragma unroll
  for (int q = 0; q < Q; ++q)
    for (int j = 0; j < min(L, k - q * L); ++j) {
      uint32_t top = o[0];
#pragma unroll
      for (int i = 1; i < V; ++i) top = max(top, o[i]);
      top = group_reduce<L>(top, [](uint32_t a, uint32_t b) { return max(a, b); });
      int at = INT32_MAX;
#pragma unroll
      for (int i = V - 1; i >= 0; --i) at = o[i] == top ? H::offset(i) : at;
      at = at == INT32_MAX ? at : at + base;
      at = group_reduce<L>(at, [](int a, int b) { return min(a, b); });
      if (lane == j) {
        c.order[q] = top;
        c.id[q] = at;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = H::offset(i) == at - base ? kNone : o[i];
    }
}

// k < 16 of a row held by 16 lanes.  At least k logits are no smaller than the
// k-th largest of the lanes' maxima, so only logits from there on can be
// chosen: a few more than k, unless many are equal.  They are listed in LDS and
// each is ranked against the others.  False (for the whole wave) where a row
// has more than kListed candidates.
template <int V, class H, int Q>
__device__ __forceinline__ bool choose_listed(const uint32_t (&o)[V], int k, int lane,
                                              uint64_t* list, Chosen<Q>& c) {
  static_assert(Q * 16 == kListed, "a register for every candidate");
  uint32_t top = o[0];
#pragma unroll
  for (int i = 1; i < V; ++i) top = max(top, o[i]);
  const int ahead = lanes_ahead(top);
  const uint32_t from = max(1u, group_reduce<16>(ahead >= k ? top : kNone, [](uint32_t a, uint32_t b) {
                              return max(a, b);
                            }));
  int mine = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) mine += o[i] >= from;
  int pos = mine;  // inclusive sum over the lanes, then exclusive
  pos += shift16<1>(pos);
  pos += shift16<2>(pos);
  pos += shift16<4>(pos);
  pos += shift16<8>(pos);
  pos -= mine;
  const int total = group_reduce<16>(mine, [](int a, int b) { return a + b; });
  if (wave_ballot(total > kListed) != 0) return false;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (o[i] >= from) list[pos++] = pair_of(o[i], H::first(lane) + H::offset(i));
  wave_lds_fence();
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int at = q * 16 + lane;
    c.order[q] = kNone;
    c.id[q] = -1;
    c.place[q] = at;  // (past the list: an empty place, where it is below k)
    if (at >= total) continue;
    const uint64_t own = list[at];
    int place = 0;
#pragma unroll 4
    for (int r = 0; r < total; ++r) place += list[r] > own;
    c.place[q] = place;
    if (place >= k) continue;
    c.order[q] = (uint32_t)(own >> 32);
    c.id[q] = (int32_t) ~(uint32_t)own;
  }
  wave_lds_fence();  // (the list has been read)
  return true;
}

template <typename T, int L, int V, bool LISTED>
__global__ __launch_bounds__(kThreads) void k_route_forward(const T* __restrict__ logits,
                                                            int64_t stride, int64_t rows, int E,
                                                            int k, bool renormalise,
                                                            float* __restrict__ weights,
                                                            int32_t* __restrict__ ids) {
  using H = Held<T, L, V>;
  constexpr int kRows = kThreads / L;
  constexpr int Q = (LISTED ? kListed : kMaxChosen) / L;
  __shared__ uint64_t s_list[LISTED ? kRows : 1][kListed];
  const int lane = threadIdx.x % L;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < rows; row0 += (int64_t)gridDim.x * kRows) {
    // (every lane stays for the exchanges; groups past the end repeat the last row)
    const int64_t row = min(row0 + threadIdx.x / L, rows - 1);
    float x[V];
    H::load(logits + row * stride, E, lane, x);
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) nan |= x[i] != x[i];
    nan = group_any<L>(nan);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) m = fmaxf(m, x[i]);
    m = group_reduce<L>(m, [](float a, float b) { return fmaxf(a, b); });
    m = m > -INFINITY ? m : 0.f;  // (so that every barred logit lies at -inf from it)
    float sum = 0.f;
    if (!renormalise) {
#pragma unroll
      for (int i = 0; i < V; ++i) sum += exp_of(x[i] - m);
    }
    uint32_t o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = order_of(x[i]);
    Chosen<Q> c;
    bool done = false;
    if constexpr (LISTED) done = choose_listed<V, H>(o, k, lane, s_list[threadIdx.x / L], c);
    if (!done) {
      if constexpr (LISTED) {  // (rare: the row is loaded again rather than kept in registers)
        H::load(logits + row * stride, E, lane, x);
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = order_of(x[i]);
      }
      choose_in_rounds<L, V, H>(o, k, lane, c);
    }
    float term[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      term[q] = c.order[q] != kNone ? exp_of(value_of(c.order[q]) - m) : 0.f;
      if (renormalise) sum += term[q];
    }
    sum = group_sum<L>(sum);
    if (row0 + threadIdx.x / L >= rows) continue;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (c.place[q] >= k) continue;
      const bool on = c.order[q] != kNone;
      float w = on ? term[q] / sum : 0.f;
      if (nan) w = NAN;
      weights[row * k + c.place[q]] = w;
      ids[row * k + c.place[q]] = on ? c.id[q] : -1;
    }
  }
}

template <typename T, int L, int V>
__global__ __launch_bounds__(kThreads) void k_route_backward(
    const float* __restrict__ grad_weights, const T* __restrict__ logits, int64_t stride,
    int64_t rows, int E, int k, const float* __restrict__ weights,
    const int32_t* __restrict__ ids, bool renormalise, T* __restrict__ grad) {
  using H = Held<T, L, V>;
  constexpr int kRows = kThreads / L;
  constexpr int Q = kMaxChosen / L;
  __shared__ float s_term[kRows][L * V];  // by register: term of expert at (lane, i) at i L + lane
  const int lane = threadIdx.x % L;
  const int group = threadIdx.x / L;
  float* mine = s_term[group];
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < rows; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = min(row0 + group, rows - 1);
    float x[V];
    if (!renormalise) H::load(logits + row * stride, E, lane, x);
    int32_t id[Q];
    float w[Q], g[Q];
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = q * L + lane;
      id[q] = j < k ? ids[row * k + j] : -1;
      if (id[q] >= E) id[q] = -1;  // (names no expert, like a negative one)
      w[q] = j < k ? weights[row * k + j] : 0.f;
      g[q] = j < k ? grad_weights[row * k + j] : 0.f;
      if (id[q] >= 0) s += w[q] * g[q];
    }
    s = group_sum<L>(s);
#pragma unroll
    for (int i = 0; i < V; ++i) mine[i * L + lane] = 0.f;
    wave_lds_fence();
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (id[q] >= 0) {
        const int run = id[q] / H::B;  // expert -> (lane, register)
        const int i = run / L * H::B + id[q] % H::B;
        mine[i * L + run % L] = renormalise ? w[q] * (g[q] - s) : g[q];
      }
    wave_lds_fence();
    float out[V];
    if (renormalise) {
#pragma unroll
      for (int i = 0; i < V; ++i) out[i] = mine[i * L + lane];
    } else {
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, x[i]);
      m = group_reduce<L>(m, [](float a, float b) { return fmaxf(a, b); });
      m = m > -INFINITY ? m : 0.f;
      const float w0 = weights[row * k];  // 1 / sum, 0 where no expert could be chosen
#pragma unroll
      for (int i = 0; i < V; ++i) {
        // (a NaN, or an infinite logit, has made w0 a NaN)
        const float p = exp_of(x[i] - m) * w0;
        out[i] = p == 0.f ? 0.f : p * (mine[i * L + lane] - s);
      }
    }
    if (row0 + group < rows) H::store(grad + row * E, E, lane, out);
    wave_lds_fence();  // (the terms have been read)
  }
}

// Calls f with the lanes per row and the logits per lane.
template <class F>
void by_width(int E, F f) {
  constexpr std::integral_constant<int, 16> row16;
  constexpr std::integral_constant<int, kWave> wave;
  if (E <= 16) f(row16, std::integral_constant<int, 1>{});
  else if (E <= 32) f(row16, std::integral_constant<int, 2>{});
  else if (E <= 64) f(row16, std::integral_constant<int, 4>{});
  else if (E <= 128) f(row16, std::integral_constant<int, 8>{});
  else if (E <= 256) f(row16, std::integral_constant<int, 16>{});
  else if (E <= 512) f(wave, std::integral_constant<int, 8>{});
  else f(wave, std::integral_constant<int, 16>{});
}

}  // namespace

hipError_t launch_route_forward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                                const void* logits, int64_t stride, bool renormalise,
                                float* weights, int32_t* ids, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    by_width(n_experts, [&](auto l, auto v) {
      constexpr int L = l.value, V = v.value;
      constexpr int kRows = kThreads / L;
      const dim3 grid((unsigned)std::min<int64_t>((rows + kRows - 1) / kRows, kMaxBlocks));
      auto go = [&](auto listed) {
        k_route_forward<T, L, V, listed.value><<<grid, kThreads, 0, stream>>>(
            static_cast<const T*>(logits), stride, rows, n_experts, k, renormalise, weights, ids);
      };
      if constexpr (L == 16) {
        if (k >= kListFrom && k <= kListTo) {
          go(std::true_type{});
          return;
        }
      }
      go(std::false_type{});
    });
  });
  return hipGetLastError();
}

hipError_t launch_route_backward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                                 const float* grad_weights, const void* logits, int64_t stride,
                                 const float* weights, const int32_t* ids, bool renormalise,
                                 void* grad_logits, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    by_width(n_experts, [&](auto l, auto v) {
      constexpr int kRows = kThreads / l.value;
      const dim3 grid((unsigned)std::min<int64_t>((rows + kRows - 1) / kRows, kMaxBlocks));
      k_route_backward<T, l.value, v.value><<<grid, kThreads, 0, stream>>>(
          grad_weights, static_cast<const T*>(logits), stride, rows, n_experts, k, weights, ids,
          renormalise, static_cast<T*>(grad_logits));
    });
  });
  return hipGetLastError();
}

}  // namespace bevpool
