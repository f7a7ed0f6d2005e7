// Stable ranks of a tile of keys by one radix digit, shared by the key sort
// and the dispatch that sorts few slots itself.
#pragma once

#include "device_utils.h"
#include "rows.h"

namespace bevpool {

constexpr int kMaxDigits = 1 << kSortBits;
constexpr int kTileThreads = 256;
constexpr int kTileWaves = kTileThreads / kWave;
constexpr int kTileRounds = kSortTile / kTileThreads;  // rounds of 64 slots of a wave
constexpr int kDigitsPerThread = kMaxDigits / kTileThreads;

// Number of the n sorted keys below v.
__device__ __forceinline__ int64_t keys_below(const int32_t* keys, int64_t n, int64_t v) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (keys[mid] < v) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// The tile's slot that this thread holds in round r: a wave's are consecutive.
__device__ __forceinline__ int tile_index(int r) {
  return (int)(threadIdx.x / kWave) * kTileRounds * kWave + r * kWave + (int)(threadIdx.x % kWave);
}

// Lanes that are `on` and hold the same digit: for each bit, those whose bit
// is this lane's (its sign over a word turns the ballot around).
__device__ __forceinline__ uint64_t same_digit(int digit, bool on, int digit_bits) {
  const uint64_t all = wave_ballot(on);
  uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
  for (int b = 0; b < kSortBits; ++b) {
    if (b >= digit_bits) break;
    const uint32_t bit = (uint32_t)((int32_t)((uint32_t)digit << (31 - b)) >> 31);
    const uint64_t m = wave_ballot(bit != 0);
    lo &= ~((uint32_t)m ^ bit);
    hi &= ~((uint32_t)(m >> 32) ^ bit);
  }
  return lo | (uint64_t)hi << 32;
}

// rank[r]: the number of equal digits in earlier slots of the wave; cnt[w][d]:
// the digit's count in wave w.  Ends with a barrier; all threads call it.
__device__ __forceinline__ void tile_ranks(const int32_t (&key)[kTileRounds], int n_tile, int shift,
                                           int digit_bits, int (*cnt)[kMaxDigits],
                                           int32_t (&rank)[kTileRounds]) {
  const int digits = 1 << digit_bits;
  const int wid = threadIdx.x / kWave;
  for (int w = 0; w < kTileWaves; ++w)
    for (int d = threadIdx.x; d < digits; d += kTileThreads) cnt[w][d] = 0;
  lds_barrier();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const bool on = tile_index(r) < n_tile;
    const int digit = (key[r] >> shift) & (digits - 1);
    const uint64_t same = same_digit(digit, on, digit_bits);
    const int below = rank_below(same);
    const int prior = cnt[wid][digit];
    if (on && below == 0) cnt[wid][digit] = prior + __popcll(same);
    rank[r] = prior + below;
  }
  lds_barrier();
}

}  // namespace bevpool
