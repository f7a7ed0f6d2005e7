// Whole expert layer for a few tokens: two launches, the gated products of every
// slot with its expert's rows, then the weighted sums of their products (and a
// third that joins these, where few columns are cut into shares).
//
// Both are products of an expert's rows with the columns of its few slots, on the
// matrix cores: 16 rows by 16 slots a tile, rows straight from memory into the
// registers (each is used once), slots' columns out of the caches.  The weights
// are read once for all slots of an expert, and what bounds the layer is reading
// them.  A wave takes 128 bytes of each of its 16 rows at a time; the waves of a
// workgroup take turns along the rows, and their sums are joined in LDS.  64 tokens,
// 8 of 128 experts, C 4096, F 1280, bfloat16: up 2.6 GB in 474 us (5.5 TB/s), down 1.3
// GB in 317 (4.2).
//
// hidden lies between the launches, in float32 whatever the layer's type, and meets
// down's rows in float32 products: a sum's intermediate has float32's range and digits,
// and its F values a slot are little beside 3 F C of the weights.  (Two values of the
// 16-bit type, a product each, took as many bytes and 306 us there, but were infinite
// past 65504 and lost digits below 2^-3 in float16, and had 16 digits in bfloat16.)

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
constexpr int kUnits = 256;           // compute units of the device
constexpr int kPitch = kTile + 1;     // of a slot's sums in LDS
constexpr int kSumBytes = kMaxSlots * kPitch * sizeof(float);

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
// The same with slots of float32, whatever the rows' type.
template <typename T>
__device__ __forceinline__ void multiply(Tile& sum, const Part<T>& a, const float (&b)[RowVec<T>::N]) {
#pragma unroll
  for (int i = 0; i < RowVec<T>::N; ++i)
    sum = __builtin_amdgcn_mfma_f32_16x16x4f32((float)a[i], b[i], sum, 0, 0, 0);
}
// The same of the first 4 FEW of 16 slots, in a quarter of the time for every four:
// 16 products of four slots by four rows, one for each quarter of 16 lanes, which is
// given the slots of lanes 4 u .. + 3 of these (the broadcast 2, u).  Lane l's results
// are row l % 16 of slots 4 u .. + 3, over the elements that its 16 lanes hold.  (A
// tile of 16 slots, with four in it on the average: the layer above 835 us, by fours 801.)
template <typename T, int FEW>
__device__ __forceinline__ void multiply_few(Tile (&sum)[FEW], const Part<T>& a, const float (&b)[RowVec<T>::N]) {
  static_assert(FEW <= 2, "broadcasts");
#pragma unroll
  for (int i = 0; i < RowVec<T>::N; ++i) {
    sum[0] = __builtin_amdgcn_mfma_f32_4x4x1f32(b[i], (float)a[i], sum[0], 2, 0, 0);
    if constexpr (FEW > 1) sum[1] = __builtin_amdgcn_mfma_f32_4x4x1f32(b[i], (float)a[i], sum[1], 2, 1, 0);
  }
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

// Workgroup (x, y): 16 hidden values of the slots of one expert, from 16 x on, y
// itself, or by_slot the expert of slot y if it is the first of its slots.  HALF: 8
// values from 8 x on, whose gates and values are the two halves of one tile, where
// workgroups are few.  STEPS chunks of a wave are in flight together.
template <typename T, int NT, int STEPS, bool HALF>
__global__ __launch_bounds__(kUpWaves * kWave, 4) void k_layer_up(
    const T* __restrict__ x, int64_t x_stride, const T* __restrict__ up,
    const int32_t* __restrict__ ids, int n, Divisor by_k, int C, int F, int E, bool by_slot,
    float* __restrict__ hidden) {
  constexpr int kRows = HALF ? kTile / 2 : kTile;  // hidden values
  constexpr int kTiles = HALF ? 1 : 2;             // of rows: gates and values
  __shared__ int16_t s_slots[kMaxSlots];
  __shared__ float s_part[kUpWaves][kTiles][kTile * kTile];
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
  const int f0 = blockIdx.x * kRows;
  const T* row[kTiles];
#pragma unroll
  for (int h = 0; h < kTiles; ++h)
    row[h] = up + ((int64_t)e * 2 * F + (HALF ? r / kRows : h) * F + min(f0 + r % kRows, F - 1)) * C;
  for (int first = 0; first < count; first += NT * kTile) {
    const T* token[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int s = first + t * kTile + r;
      token[t] = s < count ? x + (int64_t)by_k.div(s_slots[s]) * x_stride : nullptr;
    }
    Tile sum[kTiles][NT] = {};
    auto step = [&](auto check, auto steps, int k0) {
      constexpr bool CHECK = check.value;
      constexpr int S = 2 * steps.value;
      auto place = [&](int i) { return k0 + i / 2 * kUpWaves * K + (i % 2 * 4 + q) * N; };
      Part<T> a[kTiles][S];
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int h = 0; h < kTiles; ++h) a[h][i] = part_at<T, CHECK>(row[h], place(i), C);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (first + t * kTile >= count) break;
        Part<T> b[S] = {};
        if (token[t] != nullptr) {
#pragma unroll
          for (int i = 0; i < S; ++i) b[i] = part_at<T, CHECK>(token[t], place(i), C);
        }
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
          for (int h = 0; h < kTiles; ++h) multiply(sum[h][t], a[h][i], b[i]);
      }
    };
    constexpr std::integral_constant<int, STEPS> several;
    constexpr std::integral_constant<int, 1> single;
    int k0 = wave * K;
    for (; k0 + (STEPS - 1) * kUpWaves * K + K <= C; k0 += STEPS * kUpWaves * K)
      step(std::false_type{}, several, k0);
    if constexpr (STEPS > 2) {
      constexpr std::integral_constant<int, 2> two;
      for (; k0 + kUpWaves * K + K <= C; k0 += 2 * kUpWaves * K) step(std::false_type{}, two, k0);
    }
    for (; k0 + K <= C; k0 += kUpWaves * K) step(std::false_type{}, single, k0);
    if (k0 < C) step(std::true_type{}, single, k0);

#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (first + t * kTile >= count) break;
      __syncthreads();  // (what was there has been read)
#pragma unroll
      for (int h = 0; h < kTiles; ++h) *reinterpret_cast<Tile*>(&s_part[wave][h][lane * 4]) = sum[h][t];
      __syncthreads();
      // (element 4 l + i of a tile is row 4 (l / 16) + i of slot l % 16)
      const int i = threadIdx.x;
      if (i < kRows * kTile) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int w = 0; w < kUpWaves; ++w) {
          a += s_part[w][0][i];
          b += HALF ? s_part[w][0][i + kRows * kTile] : s_part[w][kTiles - 1][i];
        }
        const int f = f0 + i / 4 / kTile * 4 + i % 4, s = first + t * kTile + i / 4 % kTile;
        if (f < F && s < count)
          hidden[(int64_t)s_slots[s] * F + f] = a / (1.f + expf(-a)) * b;
      }
    }
  }
}

// Workgroup (x, y): outputs [16 x, 16 x + 16) of all tokens, from every gridDim.y-th
// of the items that the experts' products are cut into, a wave to an item: an
// expert with slots (a group), and one of P parts of its rows' chunks.  Where
// several workgroups share the items (few columns would leave compute units idle),
// their sums go to `shares`, which a third launch adds up in their order.  (Adding
// up by the last of them to arrive took 97 us where this launch took 17, at one token
// of 6 experts, C 2048, F 1024, where it takes 11 now and the third 3: its fences
// write back the caches.)
template <typename T, typename TW, int NT>
__global__ __launch_bounds__(kDownWaves * kWave) void k_layer_down(
    const float* __restrict__ hidden, const T* __restrict__ down, const TW* __restrict__ weights,
    const int32_t* __restrict__ ids, int n, int k, int C, int F, int E, int P,
    float* __restrict__ shares, T* __restrict__ out) {
  constexpr int kThreads = kDownWaves * kWave;
  constexpr int N = RowVec<T>::N, K = kChunk<T>;
  __shared__ int s_count[kMaxLayerExperts];   // slots of an expert, then where they begin
  __shared__ int16_t s_slots[kMaxSlots];      // in the order of their experts
  __shared__ int16_t s_expert[kMaxSlots + 1], s_first[kMaxSlots + 1];  // of every group
  __shared__ int s_scan[kDownWaves];
  extern __shared__ float s_sums[];  // P x n x kPitch: weighted products of every slot
  const int lane = lane_id(), wave = threadIdx.x / kWave;

  // The slots by expert.  (The order of an expert's slots is any: each has a
  // column of its own.)
  const int s = threadIdx.x;
  if (s < E) s_count[s] = 0;
  for (int i = s; i < P * n * kPitch; i += kThreads) s_sums[i] = 0.f;
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
  for (int item = blockIdx.y * kDownWaves + wave; item < groups * P; item += gridDim.y * kDownWaves) {
    const int group = item / P, part = item - group * P, end = s_first[group + 1];
    const T* row = down + ((int64_t)s_expert[group] * C + min(c0 + r, C - 1)) * F;
    // FEW: at most 4 FEW slots; otherwise up to 16 NT of them in a turn.
    auto turn = [&](auto few, int first) {
      constexpr int FEW = few.value, TILES = FEW > 0 ? 1 : NT;
      int slots[TILES];  // of this lane, -1 for none
#pragma unroll
      for (int t = 0; t < TILES; ++t) slots[t] = first + t * kTile + r < end ? s_slots[first + t * kTile + r] : -1;
      Tile sum[FEW > 0 ? FEW : NT] = {};
      auto step = [&](auto check, auto steps, int k0) {
        constexpr bool CHECK = check.value;
        constexpr int S = 2 * steps.value;
        auto place = [&](int i) { return k0 + i / 2 * P * K + (i % 2 * 4 + q) * N; };
        Part<T> a[S];
#pragma unroll
        for (int i = 0; i < S; ++i) a[i] = part_at<T, CHECK>(row, place(i), F);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
          if (first + t * kTile >= end) break;
          const float* slot = hidden + (int64_t)slots[t] * F;
#pragma unroll
          for (int i = 0; i < S; ++i) {
            float b[N] = {};
            if (slots[t] >= 0) {
#pragma unroll
              for (int p = 0; p < N; p += 4) {
                const Part<float> v = part_at<float, CHECK>(slot, place(i) + p, F);
#pragma unroll
                for (int j = 0; j < 4; ++j) b[p + j] = v[j];
              }
            }
            if constexpr (FEW > 0) multiply_few<T, FEW>(sum, a[i], b);
            else multiply<T>(sum[t], a[i], b);
          }
        }
      };
      constexpr std::integral_constant<int, 4> several;
      constexpr std::integral_constant<int, 2> two;
      constexpr std::integral_constant<int, 1> single;
      int k0 = part * K;  // every P-th chunk
      if constexpr (TILES == 1)
        for (; k0 + 3 * P * K + K <= F; k0 += 4 * P * K) step(std::false_type{}, several, k0);
      for (; k0 + P * K + K <= F; k0 += 2 * P * K) step(std::false_type{}, two, k0);
      for (; k0 + K <= F; k0 += P * K) step(std::false_type{}, single, k0);
      if (k0 < F) step(std::true_type{}, single, k0);
      if constexpr (FEW > 0) {
#pragma unroll
        for (int u = 0; u < FEW; ++u) {
          float v = 0.f;  // (lane 16 q + r keeps row r of slot q)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float all = sum[u][i];
            all += __shfl_xor(all, 16, kWave);
            all += __shfl_xor(all, 32, kWave);
            v = q == i ? all : v;
          }
          if (first + 4 * u + q < end) {
            const int slot = s_slots[first + 4 * u + q];
            s_sums[(part * n + slot) * kPitch + r] = (float)weights[slot] * v;
          }
        }
      } else {
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
          if (slots[t] < 0) continue;
          const float w = (float)weights[slots[t]];
#pragma unroll
          for (int i = 0; i < 4; ++i) s_sums[(part * n + slots[t]) * kPitch + 4 * q + i] = w * sum[t][i];
        }
      }
    };
    const int begin = s_first[group];
    if (end - begin <= 4) turn(std::integral_constant<int, 1>{}, begin);
    else if (end - begin <= 8) turn(std::integral_constant<int, 2>{}, begin);
    else
      for (int first = begin; first < end; first += NT * kTile) turn(std::integral_constant<int, 0>{}, first);
  }
  __syncthreads();
  const int rows = n / k;
  for (int i = threadIdx.x; i < rows * kTile; i += kThreads) {
    const int t = i / kTile, c = c0 + i % kTile;
    if (c >= C) continue;
    float sum = 0.f;
    for (int j = t * k; j < t * k + k; ++j)
      for (int p = 0; p < P; ++p) sum += s_sums[(p * n + j) * kPitch + i % kTile];
    if (gridDim.y > 1) shares[((int64_t)blockIdx.y * rows + t) * C + c] = sum;
    else out[(int64_t)t * C + c] = (T)sum;
  }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_layer_join(const float* __restrict__ shares,
                                                            int count, int outputs,
                                                            T* __restrict__ out) {
  const int i = blockIdx.x * kRowThreads + threadIdx.x;
  if (i >= outputs) return;
  float sum = 0.f;
#pragma unroll 8
  for (int y = 0; y < count; ++y) sum += shares[(int64_t)y * outputs + i];
  out[i] = (T)sum;
}

// How the second launch is cut, see there; workgroups to a row of them, and parts.
struct DownCut {
  int tiles, shares, P;
};
DownCut down_cut(int64_t n, int64_t C, int64_t F, int64_t E, int dtype) {
  const int64_t chunk = dtype == BEVPOOL_F32 ? kChunk<float> : kChunk<half_t>;
  const int64_t tiles = (C + kTile - 1) / kTile, chunks = (F + chunk - 1) / chunk;
  const int64_t groups = std::min(n, E);  // (at most)
  // a workgroup to a compute unit, each wave with a chunk at least
  const int64_t shares = std::max<int64_t>(
      1, std::min<int64_t>((kUnits + tiles - 1) / tiles, groups * chunks / kDownWaves));
  // an item to a wave, as far as the sums of all parts fit LDS
  const int64_t room = kSumBytes / ((int64_t)sizeof(float) * kPitch * n);
  const int64_t P = std::max<int64_t>(1, std::min({kDownWaves * shares / groups, chunks, room}));
  return DownCut{(int)tiles, (int)shares, (int)P};
}

// Bytes of hidden, behind which the shares lie.
size_t hidden_bytes(int64_t n, int64_t F) { return (n * F * sizeof(float) + 15) / 16 * 16; }

}  // namespace

size_t layer_workspace(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts, int dtype) {
  if (rows == 0) return 0;
  const DownCut cut = down_cut(rows * k, C, F, n_experts, dtype);
  return hidden_bytes(rows * k, F) + (cut.shares > 1 ? cut.shares * rows * C * sizeof(float) : 0) + 16;  // (16: alignment)
}

hipError_t launch_expert_layer(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts,
                               int dtype, int weight_dtype, const void* x, int64_t x_stride,
                               const void* up, const void* down, const void* weights,
                               const int32_t* ids, void* out, void* workspace,
                               hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  const int n = (int)(rows * k);
  const Divisor by_k = divisor(k);
  const DownCut cut = down_cut(n, C, F, n_experts, dtype);
  char* base = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 15) & ~uintptr_t(15));
  float* hidden = reinterpret_cast<float*>(base);
  float* shares = reinterpret_cast<float*>(base + hidden_bytes(n, F));
  by_types(dtype, weight_dtype, [&](auto t, auto tw) {
    using T = decltype(t);
    using TW = decltype(tw);
    const bool by_slot = n <= n_experts;
    const int columns = by_slot ? n : n_experts;
    auto up_rows = [&](auto tiles, auto steps, auto half) {
      constexpr int kRows = half.value ? kTile / 2 : kTile;
      k_layer_up<T, tiles.value, steps.value, half.value>
          <<<dim3((unsigned)((F + kRows - 1) / kRows), (unsigned)columns), kUpWaves * kWave, 0, stream>>>(
              static_cast<const T*>(x), x_stride, static_cast<const T*>(up), ids, n, by_k, (int)C,
              (int)F, n_experts, by_slot, hidden);
    };
    // (few slots on a launch of less than two workgroups to a compute unit: one token
    // of 6 experts, C 2048, F 1024, 12.7 us and 15.6 with whole tiles)
    const bool half = (F + kTile - 1) / kTile * std::min(n, n_experts) < 2 * kUnits;
    constexpr std::integral_constant<int, 2> two;
    constexpr std::integral_constant<int, 4> four;
    auto go = [&](auto tiles) {
      bool done = false;
      if constexpr (tiles.value == 1) {
        if (half) up_rows(tiles, four, std::true_type{});
        done = half;
      }
      if (!done) up_rows(tiles, two, std::false_type{});
      k_layer_down<T, TW, tiles.value><<<dim3(cut.tiles, cut.shares), kDownWaves * kWave,
                                         cut.P * n * kPitch * sizeof(float), stream>>>(
          hidden, static_cast<const T*>(down), static_cast<const TW*>(weights), ids, n, k, (int)C,
          (int)F, n_experts, cut.P, shares, static_cast<T*>(out));
    };
    // An expert's slots: a token chooses it once, as a rule, and four times as many
    // as on the average are rare.  (What does not fit is done in another turn.)
    const int64_t likely = std::min<int64_t>(rows, 4 * (int64_t)n / n_experts + 1);
    if (likely <= kTile) go(std::integral_constant<int, 1>{});
    else if (likely <= 2 * kTile) go(two);
    else go(four);
    if (cut.shares > 1) {
      const int outputs = (int)(rows * C);  // (at most 2^26)
      k_layer_join<T><<<(outputs + kRowThreads - 1) / kRowThreads, kRowThreads, 0, stream>>>(
          shares, cut.shares, outputs, static_cast<T*>(out));
    }
  });
  return hipGetLastError();
}

}  // namespace bevpool
