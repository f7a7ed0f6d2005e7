// Whole expert layer for a few tokens: two launches, the gated products of every
// slot with its expert's rows, then the weighted sums of their products.
//
// Both are products of an expert's rows with the columns of its few slots, on the
// matrix cores: 16 rows by 16 slots a tile, rows straight from memory into the
// registers (each is used once), slots' columns out of the caches.  The weights
// are read once for all slots of an expert, and what bounds the layer is reading
// them.  A wave takes 128 bytes of each of its 16 rows at a time; the waves of a
// workgroup take turns along the rows, and their sums are joined in LDS.
//
// hidden lies between the launches.  For 16-bit types it is held as two values of
// the type, hidden = high + low, with a product each: one alone would be a rounding
// as large as the output's own, and both cost 2 F values a slot beside 3 F C a
// weight matrix.

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kTile = 16;          // rows and slots of a tile
constexpr int kMaxSlots = 1024;
constexpr int kUpWaves = 8;
constexpr int kDownWaves = 16;
constexpr int kMaxLayerExperts = 1024;

typedef float Tile __attribute__((ext_vector_type(4)));

// A lane's part of 16 rows (or slots): row lane % 16, N neighbours from lane / 16 * N.
template <typename T>
using Part = typename RowVec<T>::type;

// sum += rows x slots over the 4 N elements that 64 lanes hold of each.  Lane
// l's results are rows 4 (l / 16) .. + 3 of slot l % 16.
__device__ __forceinline__ void multiply(Tile& sum, const Part<bf16_t>& a, const Part<bf16_t>& b) {
  typedef __bf16 V __attribute__((ext_vector_type(8)));
  sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16((V)a, (V)b, sum, 0, 0, 0);
}
__device__ __forceinline__ void multiply(Tile& sum, const Part<half_t>& a, const Part<half_t>& b) {
  typedef _Float16 V __attribute__((ext_vector_type(8)));
  sum = __builtin_amdgcn_mfma_f32_16x16x32_f16((V)a, (V)b, sum, 0, 0, 0);
}
__device__ __forceinline__ void multiply(Tile& sum, const Part<float>& a, const Part<float>& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], sum, 0, 0, 0);
}

// Elements of a row that a wave takes at a time: two parts, 128 bytes.
template <typename T>
constexpr int kChunk = 8 * RowVec<T>::N;

template <typename T, bool CHECK>
__device__ __forceinline__ Part<T> part_at(const T* row, int at, int n) {
  if constexpr (CHECK) {
    if (at >= n) return Part<T>{};
    return load_raw(row + at, n - at);
  }
  return *reinterpret_cast<const Part<T>*>(row + at);
}

// Orders the wave's accesses to LDS that its lanes exchange.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// hidden of a slot: F values, for 16-bit types F high ones and F low ones.
template <typename T>
constexpr int kPieces = sizeof(T) == 4 ? 1 : 2;

template <typename T>
__device__ __forceinline__ void store_hidden(T* at, int64_t low, float v) {
  const T high = (T)v;
  *at = high;
  if constexpr (kPieces<T> == 2)  // (an infinite one has no rest)
    at[low] = __builtin_isinf((float)high) ? (T)0.f : (T)(v - (float)high);
}

// Workgroup (x, y): hidden values [16 x, 16 x + 16) of the slots of one expert, y
// itself, or by_slot the expert of slot y if it is the first of its slots.
template <typename T, int NT>
__global__ __launch_bounds__(kUpWaves * kWave, 4) void k_layer_up(
    const T* __restrict__ x, int64_t x_stride, const T* __restrict__ up,
    const int32_t* __restrict__ ids, int n, Divisor by_k, int C, int F, int E, bool by_slot,
    T* __restrict__ hidden) {
  __shared__ int16_t s_slots[kMaxSlots];
  __shared__ float s_part[kUpWaves][2][kTile * kTile];
  const int e = by_slot ? ids[blockIdx.y] : (int)blockIdx.y;
  if (e < 0 || e >= E) return;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  int count = 0;  // (every wave makes the same list)
  for (int s0 = 0; s0 < n; s0 += kWave) {
    const bool mine = s0 + lane < n && ids[s0 + lane] == e;
    const uint64_t mask = wave_ballot(mine);
    if (by_slot && count == 0 && mask != 0 && s0 + __builtin_ctzll(mask) != (int)blockIdx.y) return;
    if (mine) s_slots[count + rank_below(mask)] = (int16_t)(s0 + lane);
    count += __popcll(mask);
  }
  if (count == 0) return;
  wave_lds_fence();

  const int r = lane % kTile, q = lane / kTile;
  constexpr int N = RowVec<T>::N, K = kChunk<T>;
  const int f0 = blockIdx.x * kTile;
  const T* gate_row = up + ((int64_t)e * 2 * F + min(f0 + r, F - 1)) * C;
  const T* value_row = gate_row + (int64_t)F * C;
  for (int first = 0; first < count; first += NT * kTile) {
    const T* token[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int s = first + t * kTile + r;
      token[t] = s < count ? x + (int64_t)by_k.div(s_slots[s]) * x_stride : nullptr;
    }
    Tile gate[NT] = {}, value[NT] = {};
    auto step = [&](auto check, auto steps, int k0) {
      constexpr bool CHECK = check.value;
      constexpr int S = 2 * steps.value;
      Part<T> g[S], v[S];
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const int at = k0 + i / 2 * kUpWaves * K + (i % 2 * 4 + q) * N;
        g[i] = part_at<T, CHECK>(gate_row, at, C);
        v[i] = part_at<T, CHECK>(value_row, at, C);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (first + t * kTile >= count) break;
        Part<T> b[S] = {};
        if (token[t] != nullptr) {
#pragma unroll
          for (int i = 0; i < S; ++i)
            b[i] = part_at<T, CHECK>(token[t], k0 + i / 2 * kUpWaves * K + (i % 2 * 4 + q) * N, C);
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
          multiply(gate[t], g[i], b[i]);
          multiply(value[t], v[i], b[i]);
        }
      }
    };
    constexpr std::integral_constant<int, 2> several;
    constexpr std::integral_constant<int, 1> single;
    int k0 = wave * K;
    for (; k0 + kUpWaves * K + K <= C; k0 += 2 * kUpWaves * K) step(std::false_type{}, several, k0);
    for (; k0 + K <= C; k0 += kUpWaves * K) step(std::false_type{}, single, k0);
    if (k0 < C) step(std::true_type{}, single, k0);

#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (first + t * kTile >= count) break;
      __syncthreads();  // (what was there has been read)
      *reinterpret_cast<Tile*>(&s_part[wave][0][lane * 4]) = gate[t];
      *reinterpret_cast<Tile*>(&s_part[wave][1][lane * 4]) = value[t];
      __syncthreads();
      const int i = threadIdx.x;
      if (i < kTile * kTile) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int w = 0; w < kUpWaves; ++w) {
          a += s_part[w][0][i];
          b += s_part[w][1][i];
        }
        const int f = f0 + i / 4 / kTile * 4 + i % 4, s = first + t * kTile + i / 4 % kTile;
        if (f < F && s < count)
          store_hidden(hidden + (int64_t)s_slots[s] * kPieces<T> * F + f, F, a / (1.f + expf(-a)) * b);
      }
    }
  }
}

// Workgroup x: outputs [16 x, 16 x + 16) of all tokens.
template <typename T, typename TW>
__global__ __launch_bounds__(kDownWaves * kWave) void k_layer_down(
    const T* __restrict__ hidden, const T* __restrict__ down, const TW* __restrict__ weights,
    const int32_t* __restrict__ ids, int n, int k, Divisor by_k, int C, int F, int E,
    T* __restrict__ out) {
  constexpr int kThreads = kDownWaves * kWave;
  constexpr int N = RowVec<T>::N, K = kChunk<T>;
  constexpr int kPitch = kTile + 1;
  __shared__ int s_count[kMaxLayerExperts];   // slots of an expert, then where they begin
  __shared__ int16_t s_slots[kMaxSlots];      // in the order of their experts
  __shared__ int16_t s_expert[kMaxSlots + 1], s_first[kMaxSlots + 1];  // of every group
  __shared__ int s_scan[kDownWaves];
  __shared__ float s_part[kDownWaves][kTile * kTile];
  extern __shared__ float s_sums[];  // n x kPitch: weighted products of every slot
  const int lane = lane_id(), wave = threadIdx.x / kWave;

  // The slots by expert.  (The order of an expert's slots is any: each has a
  // column of its own.)
  const int s = threadIdx.x;
  if (s < E) s_count[s] = 0;
  lds_barrier();
  int id = s < n ? ids[s] : -1;
  if (id >= E) id = -1;
  const int arrival = id >= 0 ? atomicAdd(&s_count[id], 1) : 0;
  lds_barrier();
  const int own = s < E ? s_count[s] : 0;
  int total;
  const int before = block_exclusive_scan<kThreads, true>(own + ((own > 0) << 16), s_scan, &total);
  const int groups = total >> 16;
  if (s < E) {
    s_count[s] = before & 0xffff;
    if (own > 0) {
      s_expert[before >> 16] = (int16_t)s;
      s_first[before >> 16] = (int16_t)(before & 0xffff);
    }
  }
  if (s == 0) s_first[groups] = (int16_t)(total & 0xffff);
  lds_barrier();
  if (id >= 0) s_slots[s_count[id] + arrival] = (int16_t)s;
  lds_barrier();

  const int r = lane % kTile, q = lane / kTile;
  const int c0 = blockIdx.x * kTile;
  // A tile's sum over the chunks of this wave: first, first + every, ...
  auto product = [&](int group, int slot0, int chunk0, int every) {
    const T* row = down + ((int64_t)s_expert[group] * C + min(c0 + r, C - 1)) * F;
    const bool on = slot0 + r < s_first[group + 1];
    const T* high = hidden + (int64_t)s_slots[on ? slot0 + r : slot0] * kPieces<T> * F;
    Tile sum = {};
    auto step = [&](auto check, auto steps, int k0) {
      constexpr bool CHECK = check.value;
      constexpr int S = 2 * steps.value;
      Part<T> a[S], b[kPieces<T>][S] = {};
#pragma unroll
      for (int i = 0; i < S; ++i)
        a[i] = part_at<T, CHECK>(row, k0 + i / 2 * every * K + (i % 2 * 4 + q) * N, F);
      if (on) {
#pragma unroll
        for (int p = 0; p < kPieces<T>; ++p)
#pragma unroll
          for (int i = 0; i < S; ++i)
            b[p][i] = part_at<T, CHECK>(high + p * F, k0 + i / 2 * every * K + (i % 2 * 4 + q) * N, F);
      }
#pragma unroll
      for (int p = 0; p < kPieces<T>; ++p)
#pragma unroll
        for (int i = 0; i < S; ++i) multiply(sum, a[i], b[p][i]);
    };
    constexpr std::integral_constant<int, 2> several;
    constexpr std::integral_constant<int, 1> single;
    int k0 = chunk0 * K;
    for (; k0 + every * K + K <= F; k0 += 2 * every * K) step(std::false_type{}, several, k0);
    for (; k0 + K <= F; k0 += every * K) step(std::false_type{}, single, k0);
    if (k0 < F) step(std::true_type{}, single, k0);
    return sum;
  };

  if (groups >= kDownWaves) {  // a group to a wave
    for (int g = wave; g < groups; g += kDownWaves)
      for (int slot0 = s_first[g]; slot0 < s_first[g + 1]; slot0 += kTile) {
        const Tile sum = product(g, slot0, 0, 1);
        if (slot0 + r < s_first[g + 1]) {
          const int slot = s_slots[slot0 + r];
          const float w = (float)weights[slot];
#pragma unroll
          for (int i = 0; i < 4; ++i) s_sums[slot * kPitch + 4 * q + i] = w * sum[i];
        }
      }
  } else {  // the waves share a group's rows
    for (int g = 0; g < groups; ++g)
      for (int slot0 = s_first[g]; slot0 < s_first[g + 1]; slot0 += kTile) {
        *reinterpret_cast<Tile*>(&s_part[wave][lane * 4]) = product(g, slot0, wave, kDownWaves);
        __syncthreads();
        const int i = threadIdx.x;
        if (i < kTile * kTile && slot0 + i / 4 % kTile < s_first[g + 1]) {
          const int slot = s_slots[slot0 + i / 4 % kTile];
          float sum = 0.f;
#pragma unroll
          for (int w = 0; w < kDownWaves; ++w) sum += s_part[w][i];
          s_sums[slot * kPitch + i / 4 / kTile * 4 + i % 4] = (float)weights[slot] * sum;
        }
        __syncthreads();
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n / k * kTile; i += kThreads) {
    const int t = i / kTile, c = i % kTile;
    if (c0 + c >= C) continue;
    float sum = 0.f;
    for (int j = t * k; j < t * k + k; ++j) {
      const int e = ids[j];
      if (e >= 0 && e < E) sum += s_sums[j * kPitch + c];
    }
    out[(int64_t)t * C + c0 + c] = (T)sum;
  }
}

}  // namespace

size_t layer_workspace(int64_t rows, int32_t k, int64_t F, int dtype) {
  return (size_t)(rows * k * F) * sizeof(float);  // (two 16-bit pieces take as much)
}

hipError_t launch_expert_layer(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts,
                               int dtype, int weight_dtype, const void* x, int64_t x_stride,
                               const void* up, const void* down, const void* weights,
                               const int32_t* ids, void* out, void* workspace,
                               hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  const int n = (int)(rows * k);
  const Divisor by_k = divisor(k);
  by_types(dtype, weight_dtype, [&](auto t, auto tw) {
    using T = decltype(t);
    using TW = decltype(tw);
    T* hidden = static_cast<T*>(workspace);
    const bool by_slot = n <= n_experts;
    const dim3 up_grid((unsigned)((F + kTile - 1) / kTile), (unsigned)(by_slot ? n : n_experts));
    auto go = [&](auto tiles) {
      k_layer_up<T, tiles.value><<<up_grid, kUpWaves * kWave, 0, stream>>>(
          static_cast<const T*>(x), x_stride, static_cast<const T*>(up), ids, n, by_k, (int)C,
          (int)F, n_experts, by_slot, hidden);
    };
    // (an expert's slots: a token chooses it once, as a rule)
    if (rows <= kTile) go(std::integral_constant<int, 1>{});
    else if (rows <= 2 * kTile) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 4>{});
    k_layer_down<T, TW><<<(unsigned)((C + kTile - 1) / kTile), kDownWaves * kWave,
                          n * (kTile + 1) * sizeof(float), stream>>>(
        hidden, static_cast<const T*>(down), static_cast<const TW*>(weights), ids, n, k, by_k,
        (int)C, (int)F, n_experts, static_cast<T*>(out));
  });
  return hipGetLastError();
}

}  // namespace bevpool
