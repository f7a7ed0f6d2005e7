// Stable sort of keys (expert ids, row ids) with their slots as the trace: the
// analogue of the plan's sort for keys that a model gives anew on every call.
//
// The keys 0 .. n_keys (n_keys = dropped) are sorted by radix passes of at
// most 10 bits, so expert ids take one pass and the ids of a large table two.
// A slot's rank among the equal digits of its tile comes from wave ballots (one
// per digit bit finds the lanes of equal digit) and counters per wave and digit,
// all in slot order: the sort is stable and every result the same on every run.
//
// Up to 4096 slots, and up to 8192 that take several passes, one workgroup does
// all passes in LDS.  More slots are cut into tiles of 1024, eight to a group,
// and every pass is
//   hist      per group, the digit counts of its tiles, summed over the tiles
//             before each, and the group's counts
//   (scan     per digit, the sum over the groups before each group, and over
//             all, where there are more than 32 groups)
//   scatter   every slot to its digit's start, plus the count in earlier groups
//             and tiles, plus its rank in the tile
// The last pass writes order, position and the sorted keys.  With one pass the
// starts of the digits are the offsets; else every key's offset is searched in
// the sorted keys.
//
// A call costs its chain of small launches, far from its bytes (1.5 MB for
// 131,072 slots).
// Microseconds per sort, launches back to back in a graph, with 128 and with
// 131,072 keys (two passes and the search):
//   slots            64   1024   4096   8192  16384  131072  1000000
//   128 keys        4.0    4.6    6.9    9.1    9.5    10.2     24.7
//   131,072 keys    8.9   10.8   16.5   24.2   28.5    33.9     88.8
// At 8192 slots one workgroup takes 10.6 with 128 keys, and tiles take 26.9 with
// 131,072.

#include <algorithm>

#include "device_utils.h"
#include "rows.h"
#include "rows_sort.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

constexpr int kGroupTiles = 8;
constexpr int kGroup = kSortTile * kGroupTiles;  // slots of a hist block
constexpr int kFusedGroups = 32;                 // most groups that a scatter block adds up itself

__global__ __launch_bounds__(256) void k_zero_i32(int32_t* __restrict__ a, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) a[i] = 0;
}

// tile_counts[tile][digit]: the digit's count in the earlier tiles of the
// group; group_counts[group][digit]: in the whole group.
template <typename TKey>
__global__ __launch_bounds__(kSortTile) void k_keys_hist(const TKey* __restrict__ keys, int64_t n,
                                                         int32_t n_keys, int shift, int digit_bits,
                                                         int32_t* __restrict__ tile_counts,
                                                         int32_t* __restrict__ group_counts) {
  __shared__ int h[kGroupTiles][kMaxDigits];
  const int digits = 1 << digit_bits;
  const int64_t base = (int64_t)blockIdx.x * kGroup;
  const int t = threadIdx.x;
  int32_t key[kGroupTiles];
#pragma unroll
  for (int k = 0; k < kGroupTiles; ++k) {
    const int64_t i = base + k * kSortTile + t;
    key[k] = i < n ? key_or_drop(keys, i, n_keys) : -1;
  }
  for (int i = t; i < kGroupTiles * kMaxDigits; i += kSortTile) (&h[0][0])[i] = 0;
  lds_barrier();
#pragma unroll
  for (int k = 0; k < kGroupTiles; ++k)
    if (key[k] >= 0) atomicAdd(&h[k][(key[k] >> shift) & (digits - 1)], 1);
  lds_barrier();
  if (t < digits) {
    int sum = 0;
#pragma unroll
    for (int k = 0; k < kGroupTiles; ++k) {
      tile_counts[((int64_t)blockIdx.x * kGroupTiles + k) * digits + t] = sum;
      sum += h[k][t];
    }
    group_counts[(int64_t)blockIdx.x * digits + t] = sum;
  }
}

// One digit per thread; group_counts becomes the exclusive sum over the groups.
__global__ __launch_bounds__(kWave) void k_keys_scan(int32_t* __restrict__ group_counts,
                                                     int64_t groups, int digits,
                                                     int32_t* __restrict__ totals) {
  const int d = blockIdx.x * kWave + threadIdx.x;
  if (d >= digits) return;
  int sum = 0;
  constexpr int kBatch = 16;  // loads in flight
  for (int64_t g = 0; g < groups; g += kBatch) {
    int32_t c[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) c[u] = g + u < groups ? group_counts[(g + u) * digits + d] : 0;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (g + u < groups) group_counts[(g + u) * digits + d] = sum;
      sum += c[u];
    }
  }
  totals[d] = sum;
}

// `slots` NULL: the slot is the key's index (first pass).  totals NULL: the
// groups' counts have not been summed.  position, keys_out and offsets may be
// NULL.
template <typename TKey>
__global__ __launch_bounds__(kTileThreads) void k_keys_scatter(
    const TKey* __restrict__ keys, const int32_t* __restrict__ slots, int64_t n, int32_t n_keys,
    int shift, int digit_bits, const int32_t* __restrict__ tile_counts,
    const int32_t* __restrict__ group_counts, const int32_t* __restrict__ totals, int groups,
    int32_t* __restrict__ keys_out, int32_t* __restrict__ slots_out,
    int32_t* __restrict__ position, int32_t* __restrict__ offsets) {
  __shared__ int cnt[kTileWaves][kMaxDigits];
  __shared__ int s_scan[kTileWaves];
  const int digits = 1 << digit_bits;
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  const int n_tile = (int)min<int64_t>(kSortTile, n - base);
  int32_t key[kTileRounds], slot[kTileRounds], rank[kTileRounds];
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int i = tile_index(r);
    key[r] = i < n_tile ? key_or_drop(keys, base + i, n_keys) : 0;
    slot[r] = i < n_tile ? (slots != nullptr ? slots[base + i] : (int32_t)(base + i)) : 0;
  }
  // this thread's digits t per .. t per + per - 1: their counts in all slots
  // and in the earlier groups and tiles
  const int per = max(1, digits / kTileThreads);
  const int mine = blockIdx.x / kGroupTiles;
  int tot[kDigitsPerThread], before[kDigitsPerThread];
#pragma unroll
  for (int q = 0; q < kDigitsPerThread; ++q) {
    const int d = threadIdx.x * per + q;
    tot[q] = before[q] = 0;
    if (q >= per || d >= digits) continue;
    before[q] = tile_counts[(int64_t)blockIdx.x * digits + d];
    if (totals != nullptr) {
      tot[q] = totals[d];
      before[q] += group_counts[(int64_t)mine * digits + d];
    } else {
#pragma unroll 8
      for (int g = 0; g < groups; ++g) {
        const int c = group_counts[(int64_t)g * digits + d];
        tot[q] += c;
        before[q] += g < mine ? c : 0;
      }
    }
  }
  tile_ranks(key, n_tile, shift, digit_bits, cnt, rank);
  int sum = 0;
#pragma unroll
  for (int q = 0; q < kDigitsPerThread; ++q) sum += tot[q];
  int all;
  int start = block_exclusive_scan<kTileThreads, true>(sum, s_scan, &all);
#pragma unroll
  for (int q = 0; q < kDigitsPerThread; ++q) {
    const int d = threadIdx.x * per + q;
    if (q >= per || d >= digits) continue;
    int at = start + before[q];
    int c[kTileWaves];
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) c[w] = cnt[w][d];
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) {
      cnt[w][d] = at;
      at += c[w];
    }
    if (offsets != nullptr && blockIdx.x == 0 && d <= n_keys) offsets[d] = start;
    start += tot[q];
  }
  lds_barrier();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    if (tile_index(r) >= n_tile) continue;
    const int32_t pos = cnt[threadIdx.x / kWave][(key[r] >> shift) & (digits - 1)] + rank[r];
    slots_out[pos] = slot[r];
    if (keys_out != nullptr) keys_out[pos] = key[r];
    if (position != nullptr) position[slot[r]] = pos;
  }
}

// All passes over at most ROUNDS * 1024 slots in one workgroup.
constexpr int kSmallThreads = 1024;
constexpr int kSmallWaves = kSmallThreads / kWave;

template <typename TKey, int ROUNDS>
__global__ __launch_bounds__(kSmallThreads) void k_keys_small(
    const TKey* __restrict__ keys, int32_t n, int32_t n_keys, int passes, int digit_bits,
    int32_t* __restrict__ order, int32_t* __restrict__ position, int32_t* __restrict__ offsets,
    int32_t* __restrict__ sorted_keys) {
  __shared__ __attribute__((aligned(4))) uint16_t cnt[kSmallWaves][kMaxDigits];  // (a wave has few slots)
  __shared__ int32_t s_start[kMaxDigits];
  __shared__ int s_scan[kSmallWaves];
  __shared__ int32_t s_key[ROUNDS * kSmallThreads];
  __shared__ uint16_t s_slot[ROUNDS * kSmallThreads], s_pos[ROUNDS * kSmallThreads];
  const int t = threadIdx.x;
  const int wid = t / kWave, lane = t % kWave;
  const int digits = 1 << digit_bits;
  const int rounds = (n + kSmallThreads - 1) / kSmallThreads;
  const int base = wid * rounds * kWave + lane;  // the wave's slots are consecutive
  int32_t key[ROUNDS];
  uint32_t slot[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = base + r * kWave;
    const bool on = r < rounds && i < n;
    key[r] = on ? key_or_drop(keys, i, n_keys) : 0;
    slot[r] = (uint32_t)i;
  }
  for (int p = 0; p < passes; ++p) {
    const int shift = p * digit_bits;
    for (int i = t; i < kSmallWaves * kMaxDigits / 2; i += kSmallThreads)
      reinterpret_cast<uint32_t*>(cnt)[i] = 0;
    lds_barrier();
    if (p > 0) {
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) {
        const int i = base + r * kWave;
        if (r >= rounds || i >= n) continue;
        key[r] = s_key[i];
        slot[r] = s_slot[i];
      }
    }
    int32_t rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      rank[r] = 0;
      if (r >= rounds) continue;  // (uniform)
      const bool on = base + r * kWave < n;
      const int digit = (key[r] >> shift) & (digits - 1);
      const uint64_t same = same_digit(digit, on, digit_bits);
      const int below = rank_below(same);
      const int prior = cnt[wid][digit];
      if (on && below == 0) cnt[wid][digit] = (uint16_t)(prior + __popcll(same));
      rank[r] = prior + below;
    }
    lds_barrier();
    int tot = 0;  // digit t: the waves' offsets within the digit, and its count
    if (t < digits) {
      int c[kSmallWaves];
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) c[w] = cnt[w][t];
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) {
        cnt[w][t] = (uint16_t)tot;
        tot += c[w];
      }
    }
    int all;
    const int start = block_exclusive_scan<kSmallThreads, true>(tot, s_scan, &all);
    if (t < digits) s_start[t] = start;
    if (passes == 1 && t <= n_keys && t < digits) offsets[t] = start;
    lds_barrier();
    const bool last = p == passes - 1;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (r >= rounds || base + r * kWave >= n) continue;
      const int digit = (key[r] >> shift) & (digits - 1);
      const int pos = s_start[digit] + cnt[wid][digit] + rank[r];
      s_key[pos] = key[r];
      s_slot[pos] = (uint16_t)slot[r];
      if (last) s_pos[slot[r]] = (uint16_t)pos;
    }
    lds_barrier();
  }
  // (out of LDS in order: one unit's scattered stores took 5 us for 4096 slots)
  for (int i = t; i < n; i += kSmallThreads) {
    order[i] = s_slot[i];
    if (position != nullptr) position[i] = s_pos[i];
    if (sorted_keys != nullptr) sorted_keys[i] = s_key[i];
  }
}

// offsets[v] = number of sorted keys below v, v = 0 .. n_keys
__global__ __launch_bounds__(256) void k_keys_offsets(const int32_t* __restrict__ keys, int64_t n,
                                                      int32_t n_keys,
                                                      int32_t* __restrict__ offsets) {
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (v <= n_keys) offsets[v] = (int32_t)keys_below(keys, n, v);
}

}  // namespace

SortLayout sort_layout(int64_t n, int64_t n_keys) {
  SortLayout L{};
  L.bits = 1;
  while ((int64_t(1) << L.bits) <= n_keys) ++L.bits;
  L.passes = (L.bits + kSortBits - 1) / kSortBits;
  L.digit_bits = (L.bits + L.passes - 1) / L.passes;
  L.tiles = (n + kSortTile - 1) / kSortTile;
  L.groups = (n + kGroup - 1) / kGroup;
  size_t off = 0;
  auto take = [&](int64_t ints) {
    const size_t o = off;
    off += (sizeof(int32_t) * (size_t)ints + 255) & ~size_t(255);
    return o;
  };
  L.small = n <= (L.passes > 1 ? kSmallSortPasses : kSmallSort);
  if (!L.small) {
    L.tile_counts = take((L.groups * kGroupTiles) << L.digit_bits);
    L.group_counts = take(L.groups << L.digit_bits);
    L.totals = take(int64_t(1) << L.digit_bits);
    if (L.passes > 1)
      for (int i = 0; i < 2; ++i) {
        L.keys[i] = take(n);
        L.vals[i] = take(n);
      }
  } else if (n > 0 && L.passes > 1) {
    L.keys[0] = take(n);  // (sorted, for the offsets)
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
  const int32_t nk = (int32_t)n_keys;
  if (L.small) {
    int32_t* sorted = sorted_keys != nullptr ? sorted_keys : L.passes > 1 ? W(L.keys[0]) : nullptr;
    auto run = [&](auto* k, auto rounds) {
      k_keys_small<std::remove_const_t<std::remove_pointer_t<decltype(k)>>, rounds.value>
          <<<1, kSmallThreads, 0, stream>>>(k, (int32_t)n, nk, L.passes, L.digit_bits, order,
                                            position, offsets, sorted);
    };
    auto go = [&](auto* k) {
      if (n <= kSmallSort) run(k, std::integral_constant<int, kSmallSort / kSmallThreads>{});
      else run(k, std::integral_constant<int, kSmallSortPasses / kSmallThreads>{});
    };
    if (key_type == BEVPOOL_KEY_I64) go(static_cast<const int64_t*>(keys));
    else go(static_cast<const int32_t*>(keys));
    if (L.passes > 1 && offsets != nullptr)
      k_keys_offsets<<<ogrid, 256, 0, stream>>>(sorted, n, nk, offsets);
    return hipGetLastError();
  }
  int32_t *tile_counts = W(L.tile_counts), *group_counts = W(L.group_counts);
  int32_t* totals = L.groups > kFusedGroups ? W(L.totals) : nullptr;
  const int digits = 1 << L.digit_bits;
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
      k_keys_hist<<<(unsigned)L.groups, kSortTile, 0, stream>>>(k, n, nk, shift, L.digit_bits,
                                                                tile_counts, group_counts);
      if (totals != nullptr)
        k_keys_scan<<<(unsigned)((digits + kWave - 1) / kWave), kWave, 0, stream>>>(
            group_counts, L.groups, digits, totals);
      k_keys_scatter<<<(unsigned)L.tiles, kTileThreads, 0, stream>>>(
          k, in_slots, n, nk, shift, L.digit_bits, tile_counts, group_counts, totals,
          (int)L.groups, out_keys, out_slots, pos, off);
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
  if (L.passes > 1 && offsets != nullptr)
    k_keys_offsets<<<ogrid, 256, 0, stream>>>(in_keys, n, nk, offsets);
  return hipGetLastError();
}

}  // namespace bevpool
