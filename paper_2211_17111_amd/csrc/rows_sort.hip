// Stable sort of keys (expert ids, row ids) with their slots as the trace: the
// analogue of the plan's sort for keys that a model gives anew on every call.
//
// The keys 0 .. n_keys (n_keys = dropped) are sorted by radix passes of at
// most 10 bits, so expert ids take one pass and the ids of a large table two:
//   hist      the digit counts of every tile of 2048 slots
//   scan      per digit, the counts of the tiles before each tile, and the total
//   scatter   every slot to its digit's start (a scan of the totals), plus the
//             earlier tiles' count, plus its rank in the tile
// A slot's rank in its tile comes from wave ballots (one per digit bit finds
// the lanes of equal digit) and counters per wave and digit, all in slot
// order: the sort is stable and every result the same on every run.  The last
// pass writes order and position.  With one pass the starts of the digits are
// the offsets; else every key's offset is searched in the sorted keys.

#include <algorithm>

#include "device_utils.h"
#include "rows.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRounds = kSortTile / kThreads;  // 64-slot rounds of a wave
constexpr int kWaveSpan = kRounds * kWave;     // slots of a wave, consecutive
constexpr int kMaxDigits = 1 << kSortBits;

__global__ __launch_bounds__(256) void k_zero_i32(int32_t* __restrict__ a, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) a[i] = 0;
}

template <typename TKey>
__global__ __launch_bounds__(kThreads) void k_keys_hist(const TKey* __restrict__ keys, int64_t n,
                                                        int32_t n_keys, int shift, int digit_bits,
                                                        int32_t* __restrict__ hist) {
  __shared__ int h[kMaxDigits];
  const int digits = 1 << digit_bits;
  for (int i = threadIdx.x; i < digits; i += kThreads) h[i] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = base + r * kThreads + threadIdx.x;
    if (i < n) atomicAdd(&h[(key_or_drop(keys, i, n_keys) >> shift) & (digits - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < digits; i += kThreads)
    hist[(int64_t)blockIdx.x * digits + i] = h[i];
}

// One digit per thread; hist becomes the exclusive prefix over the tiles.
__global__ __launch_bounds__(kWave) void k_keys_scan(int32_t* __restrict__ hist, int64_t tiles,
                                                     int digits, int32_t* __restrict__ totals) {
  const int d = blockIdx.x * kWave + threadIdx.x;
  if (d >= digits) return;
  int sum = 0;
  constexpr int kBatch = 8;  // loads in flight
  int64_t t = 0;
  for (; t + kBatch <= tiles; t += kBatch) {
    int32_t c[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) c[u] = hist[(t + u) * digits + d];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      hist[(t + u) * digits + d] = sum;
      sum += c[u];
    }
  }
  for (; t < tiles; ++t) {
    const int32_t c = hist[t * digits + d];
    hist[t * digits + d] = sum;
    sum += c;
  }
  totals[d] = sum;
}

// `slots` NULL: the slot is the key's index (first pass).  The last pass sets
// order and position, the others keys_out and slots_out; keys_out is also set
// in a last pass whose sorted keys are searched for the offsets.  offsets is
// set in an only pass.
template <typename TKey>
__global__ __launch_bounds__(kThreads) void k_keys_scatter(
    const TKey* __restrict__ keys, const int32_t* __restrict__ slots, int64_t n, int32_t n_keys,
    int shift, int digit_bits, const int32_t* __restrict__ hist, const int32_t* __restrict__ totals,
    int32_t* __restrict__ keys_out, int32_t* __restrict__ slots_out,
    int32_t* __restrict__ position, int32_t* __restrict__ offsets) {
  __shared__ int cnt[kWaves][kMaxDigits];
  __shared__ int s_scan[kWaves];
  const int digits = 1 << digit_bits;
  for (int w = 0; w < kWaves; ++w)
    for (int i = threadIdx.x; i < digits; i += kThreads) cnt[w][i] = 0;
  __syncthreads();

  const int lane = lane_id();
  const int wid = threadIdx.x / kWave;
  const int64_t base = (int64_t)blockIdx.x * kSortTile + (int64_t)wid * kWaveSpan;
  int32_t key[kRounds], rank[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = base + r * kWave + lane;
    const bool valid = i < n;
    key[r] = valid ? key_or_drop(keys, i, n_keys) : 0;
    const int digit = (key[r] >> shift) & (digits - 1);
    uint64_t same = wave_ballot(valid);
    for (int b = 0; b < digit_bits; ++b) {
      const bool bit = (digit >> b) & 1;
      const uint64_t m = wave_ballot(bit);
      same &= bit ? m : ~m;
    }
    const int below = rank_below(same);
    const int prior = cnt[wid][digit];
    if (valid && below == 0) cnt[wid][digit] = prior + __popcll(same);
    rank[r] = prior + below;
  }
  __syncthreads();
  // starts of the digits: thread t scans digits [t * per, (t + 1) * per)
  constexpr int kPer = kMaxDigits / kThreads;
  int tot[kPer];
  int sum = 0;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int d = threadIdx.x * kPer + q;
    tot[q] = d < digits ? totals[d] : 0;
    sum += tot[q];
  }
  int all;
  int start = block_exclusive_scan<kThreads>(sum, s_scan, &all);
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int d = threadIdx.x * kPer + q;
    if (d < digits) {
      int at = start + hist[(int64_t)blockIdx.x * digits + d];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const int c = cnt[w][d];
        cnt[w][d] = at;
        at += c;
      }
      if (offsets != nullptr && blockIdx.x == 0 && d <= n_keys) offsets[d] = start;
    }
    start += tot[q];
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = base + r * kWave + lane;
    if (i >= n) continue;
    const int32_t pos = cnt[wid][(key[r] >> shift) & (digits - 1)] + rank[r];
    const int32_t slot = slots != nullptr ? slots[i] : (int32_t)i;
    slots_out[pos] = slot;
    if (keys_out != nullptr) keys_out[pos] = key[r];
    if (position != nullptr) position[slot] = pos;
  }
}

// offsets[v] = number of sorted keys below v, v = 0 .. n_keys
__global__ __launch_bounds__(256) void k_keys_offsets(const int32_t* __restrict__ keys, int64_t n,
                                                      int32_t n_keys,
                                                      int32_t* __restrict__ offsets) {
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (v > n_keys) return;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (keys[mid] < v) lo = mid + 1; else hi = mid;
  }
  offsets[v] = (int32_t)lo;
}

}  // namespace

SortLayout sort_layout(int64_t n, int64_t n_keys) {
  SortLayout L{};
  L.bits = 1;
  while ((int64_t(1) << L.bits) <= n_keys) ++L.bits;
  L.passes = (L.bits + kSortBits - 1) / kSortBits;
  L.digit_bits = (L.bits + L.passes - 1) / L.passes;
  L.tiles = (n + kSortTile - 1) / kSortTile;
  size_t off = 0;
  auto take = [&](int64_t ints) {
    const size_t o = off;
    off += (sizeof(int32_t) * (size_t)ints + 255) & ~size_t(255);
    return o;
  };
  if (n > 0) {
    L.hist = take(L.tiles << L.digit_bits);
    L.totals = take(int64_t(1) << L.digit_bits);
    if (L.passes > 1)
      for (int i = 0; i < 2; ++i) {
        L.keys[i] = take(n);
        L.vals[i] = take(n);
      }
  }
  L.total = off;
  return L;
}

hipError_t launch_sort_keys(int64_t n, int64_t n_keys, int key_type, const void* keys,
                            int32_t* order, int32_t* position, int32_t* offsets,
                            int32_t* sorted_keys, void* workspace, hipStream_t stream) {
  const unsigned ogrid = (unsigned)((n_keys + 1 + 255) / 256);
  if (n == 0) {
    k_zero_i32<<<ogrid, 256, 0, stream>>>(offsets, n_keys + 1);
    return hipGetLastError();
  }
  const SortLayout L = sort_layout(n, n_keys);
  char* ws = static_cast<char*>(workspace);
  auto W = [&](size_t o) { return reinterpret_cast<int32_t*>(ws + o); };
  int32_t *hist = W(L.hist), *totals = W(L.totals);
  const int32_t nk = (int32_t)n_keys;
  const int digits = 1 << L.digit_bits;
  const dim3 grid((unsigned)L.tiles);
  const unsigned sgrid = (unsigned)((digits + kWave - 1) / kWave);
  const int32_t* in_keys = nullptr;
  const int32_t* in_slots = nullptr;
  for (int p = 0; p < L.passes; ++p) {
    const int shift = p * L.digit_bits;
    const bool last = p == L.passes - 1;
    int32_t* out_keys = last && sorted_keys != nullptr ? sorted_keys
                        : L.passes > 1                ? W(L.keys[p & 1])
                                                       : nullptr;
    int32_t* out_slots = last ? order : W(L.vals[p & 1]);
    int32_t* pos = last ? position : nullptr;
    int32_t* off = L.passes == 1 ? offsets : nullptr;
    auto pass = [&](auto* k) {
      k_keys_hist<<<grid, kThreads, 0, stream>>>(k, n, nk, shift, L.digit_bits, hist);
      k_keys_scan<<<sgrid, kWave, 0, stream>>>(hist, L.tiles, digits, totals);
      k_keys_scatter<<<grid, kThreads, 0, stream>>>(k, in_slots, n, nk, shift, L.digit_bits, hist,
                                                    totals, out_keys, out_slots, pos, off);
    };
    if (p > 0)
      pass(in_keys);
    else if (key_type == BEVPOOL_KEY_I64)
      pass(static_cast<const int64_t*>(keys));
    else
      pass(static_cast<const int32_t*>(keys));
    in_keys = out_keys;
    in_slots = out_slots;
  }
  if (L.passes > 1) k_keys_offsets<<<ogrid, 256, 0, stream>>>(in_keys, n, nk, offsets);
  return hipGetLastError();
}

}  // namespace bevpool
