// Forward of the logits operators: statistics of every row's softmax, and from
// them log probabilities, entropy, alternatives and divergences.
//
// Every logit is read once, and reading is what bounds rows that are many or
// long.  Short rows are held in the registers of 16 or 64 lanes.  Longer ones are
// streamed by workgroups, each thread with its own running maximum and sums;
// where there are few of them, a row is cut into parts, whose statistics (and
// alternatives) a second launch joins.
//
// Alternatives: at least k logits are no smaller than the k-th largest of some
// (disjoint) groups' maxima, so only logits from there on can be chosen: a few
// more than k, unless many are equal or the groups are few.  The maxima are
// by-products of the statistics.  The candidates are listed in LDS and each is
// ranked against the others; a row with more candidates than the list holds takes
// k rounds, each of which finds the next in order.
//
// Measured: 8192 rows of 65,536 bfloat16 183 us, 5.9 TB/s (float32 6.1; at 65,537,
// where vectors lie across cache lines, 4.8 and 6.1), 190 with the entropy; 4096
// rows of 131,072 with 20 alternatives 195 us, 5.5 TB/s; 24,000 rows of 118 float32
// with their divergence 6 us.  (Beginning each row's vectors at a cache line would
// make a row's sums depend on where it lies.)

#include "logits.h"
#include "logits_rows.h"

namespace bevpool {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;       // vectors of a thread in flight
constexpr int kMaxParts = 64;
constexpr int kMaxBatches = 16;  // of a part whose alternatives are wanted

// Floats as unsigned integers in their order, +0 and -0 the same; 0, below all
// of them, for what is never chosen (-inf, NaN).
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // (-0 + 0 = +0)
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return v > -INFINITY ? o : 0;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

// A logit's order and its index in one number: larger logits are larger, of
// equal ones the lower index is; 0 for what is never chosen.
__device__ __forceinline__ uint64_t pair_of(float x, int v) {
  const uint32_t o = order_of(x);
  return o != 0 ? ((uint64_t)o << 32) | (uint32_t)~v : 0;
}

template <int L>
__device__ __forceinline__ uint64_t lanes_max(uint64_t v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) {
    const uint64_t other = __shfl_xor(v, o, kWave);
    v = other > v ? other : v;
  }
  return v;
}

// A value that at least k of a wave's 64 R values are no smaller than, and as few
// more as can be: -inf where fewer than k are above it.  (Its order is found bit by
// bit, the values counted by ballots.)
template <int R>
__device__ __forceinline__ float wave_threshold(const uint32_t (&order)[R], int k) {
  uint32_t from = 0;
  for (uint32_t bit = 1u << 31; bit != 0; bit >>= 1) {
    int count = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) count += __popcll(wave_ballot(order[r] >= (from | bit)));
    if (count >= k) from |= bit;
    if (count == k) break;
  }
  return from > order_of(-FLT_MAX) ? value_of(from) : -INFINITY;
}

// The same for k <= 16 values of 16 lanes, one each: the k-th largest.
__device__ __forceinline__ float team_threshold(float v, int k) {
  const int lane = threadIdx.x % 16;
  int ahead = 0;
#pragma unroll
  for (int o = 1; o < 16; ++o) {
    const float other = __shfl_xor(v, o, kWave);
    ahead += other > v || (other == v && (lane ^ o) < lane);
  }
  float m = ahead == k - 1 ? v : -INFINITY;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
  return m;
}

// What a forward writes of a row.  `Own` is what it needs beside the statistics:
// loaded ahead of the logits, so that nothing waits for it behind them.
struct LogprobsRow {
  LogprobsOut out;
  static constexpr bool kEntropy = true;

  struct Own {
    int32_t id;
    float x;
  };
  template <typename T, class TEAM>
  __device__ __forceinline__ Own ahead(const TEAM& team, const LogitsRows& in, int64_t t, const T* row) const {
    Own own{-1, 0.f};
    if (out.logprob != nullptr && team.lane() == 0) {
      own.id = id_at(in.ids, in.key_type, t, in.V);
      if (own.id >= 0) own.x = (float)row[own.id];
    }
    return own;
  }
  template <class TEAM>
  __device__ __forceinline__ void finish(const TEAM& team, const LogitsRows&, int64_t t, const Own& own,
                                         const Soft& a, const Row& p) const {
    if (team.lane() != 0) return;
    out.stats[2 * t] = p.m;
    out.stats[2 * t + 1] = p.S;
    if (out.logprob != nullptr) out.logprob[t] = own.id >= 0 ? p.logprob(own.x) : 0.f;
    if (out.lse != nullptr) out.lse[t] = p.S == 0.f ? -INFINITY : fmaf(p.scale, p.m, p.log_S);
    if (out.entropy != nullptr) out.entropy[t] = p.S == 0.f ? 0.f : fmaf(-kLn2, a.w / a.s, p.log_S);
  }
  // Alternative j of row t (0: none).
  __device__ __forceinline__ void alternative(int64_t at, uint64_t pair, const Row& p) const {
    const uint32_t order = (uint32_t)(pair >> 32);
    out.top[at] = p.S != p.S ? NAN : order != 0 ? p.logprob(value_of(order)) : -INFINITY;
    out.top_ids[at] = order != 0 ? (int32_t) ~(uint32_t)pair : -1;
  }
};

// KS slots to a lane.
template <int KS>
struct DistillRow {
  float *loss, *stats;
  static constexpr bool kEntropy = false;

  using Own = Slots<KS>;
  template <typename T, class TEAM>
  __device__ __forceinline__ Own ahead(const TEAM& team, const LogitsRows& in, int64_t t, const T* row) const {
    Own own;
    own.load(team, in, t);
    own.drop();
    own.load_logits(row);
    return own;
  }
  template <class TEAM>
  __device__ __forceinline__ void finish(const TEAM& team, const LogitsRows& in, int64_t t, Own own,
                                         const Soft&, const Row& p) const {
    taught(team, own, in.renormalise);
    const float d = divergence(team, own, p);
    if (team.lane() != 0) return;
    stats[2 * t] = p.m;
    stats[2 * t + 1] = p.S;
    loss[t] = d;
  }
  __device__ __forceinline__ void alternative(int64_t, uint64_t, const Row&) const {}
};

// Writes the k best of n listed pairs by f(place, pair), 0 for a place that none
// takes.
template <class TEAM, class F>
__device__ __forceinline__ void rank_pairs(const TEAM& team, const uint64_t* list, int n, int k, F f) {
  for (int i = team.lane(); i < n; i += TEAM::kLanes) {
    const uint64_t own = list[i];
    int place = 0;
#pragma unroll 4
    for (int r = 0; r < n; ++r) place += list[r] > own;
    if (place < k) f(place, own);
  }
  for (int j = n + team.lane(); j < k; j += TEAM::kLanes) f(j, uint64_t(0));
}

// ------------------------------------------------------------------ short rows

// Rows held by teams of L lanes.
template <typename T, int L, int NV, bool TOP, class ROW>
__global__ __launch_bounds__(kThreads) void k_short_rows(LogitsRows in, ROW out, float c) {
  constexpr int kTeams = kThreads / L;
  constexpr int kListed = TOP ? 2048 / kTeams : 1;
  __shared__ uint64_t s_list[kTeams][kListed];
  __shared__ int s_count[kTeams];
  const Team<L> team{nullptr};
  const int own = threadIdx.x / L, lane = team.lane();
  for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < in.rows; t0 += (int64_t)gridDim.x * kTeams) {
    const int64_t t = t0 + own;
    if (t >= in.rows) break;  // (a wave's teams need one another nowhere)
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    const auto ahead = out.ahead(team, in, t, row);
    Held<T, L, NV> x;
    x.load(row, in.V, lane);
    const float largest = x.largest(lane);
    const Soft a = soft_of<ROW::kEntropy>(team, x, largest, c);
    const Row p = row_of(a, in.scale);
    out.finish(team, in, t, ahead, a, p);
    if constexpr (TOP) {
      const int k = in.k;
      constexpr int N = RowVec<T>::N;
      int n = 0;
      if constexpr (L == kWave) {
        // from the vectors' maxima, or where these may be too few from the logits
        constexpr bool kSingle = NV == 2;
        uint32_t order[kSingle ? NV * N : NV] = {};
        x.each(lane, [&](const auto& v, int, int j) {
          if constexpr (kSingle) {
#pragma unroll
            for (int e = 0; e < N; ++e) order[j * N + e] = order_of(v[e]);
          } else {
            float top = v[0];
#pragma unroll
            for (int e = 1; e < N; ++e) top = fmaxf(top, v[e]);
            order[j] = order_of(top);
          }
        });
        const float from = wave_threshold(order, k);
        x.each(lane, [&](const auto& v, int i, int) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const bool on = v[e] >= from && v[e] > -INFINITY;
            const uint64_t mask = wave_ballot(on);
            if (mask == 0) continue;
            const int at = n + rank_below(mask);
            if (on && at < kListed) s_list[own][at] = pair_of(v[e], i * N + e);
            n += __popcll(mask);
          }
        });
        team.sync();
      } else {
        const float from = team_threshold(largest, k);
        if (lane == 0) s_count[own] = 0;
        team.sync();
        x.each(lane, [&](const auto& v, int i, int) {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (v[e] >= from && v[e] > -INFINITY) {
              const int at = atomicAdd(&s_count[own], 1);
              if (at < kListed) s_list[own][at] = pair_of(v[e], i * N + e);
            }
        });
        team.sync();
        n = s_count[own];
      }
      if (n <= kListed) {
        rank_pairs(team, s_list[own], n, k, [&](int j, uint64_t pair) { out.alternative(t * k + j, pair, p); });
      } else {
        uint64_t last = ~uint64_t(0);
        for (int j = 0; j < k; ++j) {
          uint64_t best = 0;
          x.each(lane, [&](const auto& v, int i, int) {
#pragma unroll
            for (int e = 0; e < RowVec<T>::N; ++e) {
              const uint64_t pair = pair_of(v[e], i * RowVec<T>::N + e);
              best = pair < last && pair > best ? pair : best;
            }
          });
          last = best = lanes_max<L>(best);
          if (lane == 0) out.alternative(t * k + j, best, p);
        }
      }
      team.sync();  // (the list has been read)
    }
  }
}

// ------------------------------------------------------------------- long rows

// Statistics of a part of a row; behind them in the workspace lie the k best of
// every part, in order.
struct Part {
  float r, s, w;
};
struct Parts {
  int64_t total;  // rows * count
  int32_t count;  // of a row
  int32_t length;  // vectors, whole batches
  Part* soft;
  uint64_t* pairs;
};

template <typename T, bool ENTROPY, bool TOP, class ROW>
__global__ __launch_bounds__(kThreads) void k_row_parts(LogitsRows in, ROW out, float c, Parts parts) {
  constexpr int N = RowVec<T>::N;
  constexpr int kStep = kThreads * kBatch;
  constexpr int kEntries = TOP ? kMaxBatches * kThreads : 1;
  constexpr int kListed = kEntries / 2;
  // the maxima of every thread's batches, and once these are looked through the list
  __shared__ union {
    float maxima[kEntries];
    uint64_t list[TOP ? kListed : 1];
  } s;
  __shared__ uint16_t s_batches[kEntries];
  __shared__ float s_largest[kThreads], s_scratch[kThreads / kWave], s_from;
  __shared__ uint64_t s_best[kThreads / kWave];
  __shared__ int s_count[2];
  const Team<kThreads> team{s_scratch};
  const int tid = threadIdx.x;
  const int vectors = vectors_of<T>(in.V), whole = in.V / N;
  for (int64_t b = blockIdx.x; b < parts.total; b += gridDim.x) {
    const int64_t t = parts.count == 1 ? b : b / parts.count;
    const int first = (int)(b - t * parts.count) * parts.length;
    const int end = min(first + parts.length, vectors);
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    typename ROW::Own ahead;
    if (parts.count == 1) ahead = out.ahead(team, in, t, row);
    Soft a = no_soft();
    float largest = -INFINITY;
    int batch = 0;
    for (int i0 = first; i0 < end; i0 += kStep, ++batch) {
      typename RowVec<T>::type raw[kBatch];
      if (i0 + kStep <= min(end, whole)) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          raw[j] = *reinterpret_cast<const typename RowVec<T>::type*>(row + (int64_t)(i0 + j * kThreads + tid) * N);
      } else {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int i = i0 + j * kThreads + tid;
          raw[j] = logits_at(row, i, i < end ? in.V : 0);
        }
      }
      float x[kBatch * N];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) to_floats<T>(raw[j], x + j * N);
      const float top = add<ENTROPY>(a, x, c);
      if constexpr (TOP) {
        s.maxima[batch * kThreads + tid] = top;
        largest = fmaxf(largest, top);
      }
    }
    if constexpr (TOP) {
      s_largest[tid] = largest;
      if (tid < 2) s_count[tid] = 0;
    }
    a = join<ENTROPY>(team, a, c);
    Row p = row_of(a, in.scale);
    if (parts.count == 1) {
      out.finish(team, in, t, ahead, a, p);
    } else if (tid == 0) {
      parts.soft[b] = Part{a.r, a.s, a.w};
    }
    if constexpr (TOP) {
      const int k = in.k;
      auto put = [&](int j, uint64_t pair) {
        if (parts.count == 1) out.alternative(t * k + j, pair, p);
        else parts.pairs[b * k + j] = pair;
      };
      const int lane = lane_id();  // (join's barriers lie behind the maxima)
      if (tid < kWave) {
        uint32_t order[kThreads / kWave];
#pragma unroll
        for (int w = 0; w < kThreads / kWave; ++w) order[w] = order_of(s_largest[w * kWave + lane]);
        const float threshold = wave_threshold(order, k);
        if (tid == 0) s_from = threshold;
      }
      lds_barrier();
      const float from = s_from;
      for (int i = 0; i < batch; ++i) {
        const float top = s.maxima[i * kThreads + tid];
        if (top >= from && top > -INFINITY) s_batches[atomicAdd(&s_count[0], 1)] = (uint16_t)(i * kThreads + tid);
      }
      __syncthreads();
      const int items = s_count[0] * kBatch;
      for (int i = tid; i < items; i += kThreads) {
        const int at = s_batches[i / kBatch];
        const int v = first + (at / kThreads * kBatch + i % kBatch) * kThreads + at % kThreads;
        if (v >= end) continue;
        float x[N];
        to_floats<T>(logits_at(row, v, in.V), x);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (x[e] >= from && x[e] > -INFINITY) {
            const int place = atomicAdd(&s_count[1], 1);
            if (place < kListed) s.list[place] = pair_of(x[e], v * N + e);
          }
      }
      __syncthreads();
      const int n = s_count[1];
      if (n <= kListed) {
        rank_pairs(team, s.list, n, k, put);
      } else {
        uint64_t last = ~uint64_t(0);
        for (int j = 0; j < k; ++j) {
          uint64_t best = 0;
          for (int v = first + tid; v < end; v += kThreads) {
            float x[N];
            to_floats<T>(logits_at(row, v, in.V), x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const uint64_t pair = pair_of(x[e], v * N + e);
              best = pair < last && pair > best ? pair : best;
            }
          }
          best = lanes_max<kWave>(best);
          if (lane == 0) s_best[tid / kWave] = best;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < kThreads / kWave; ++w) best = s_best[w] > best ? s_best[w] : best;
          last = best;
          if (tid == 0) put(j, best);
          __syncthreads();
        }
      }
      __syncthreads();  // (the lists have been read)
    }
  }
}

// Joins a row's parts: a workgroup to a row.
template <typename T, bool ENTROPY, bool TOP, class ROW>
__global__ __launch_bounds__(kThreads) void k_join_parts(LogitsRows in, ROW out, float c, Parts parts) {
  constexpr int kListed = TOP ? kMaxParts * kMaxAlternatives : 1;
  __shared__ uint64_t s_list[kListed];
  __shared__ float s_scratch[kThreads / kWave];
  __shared__ int s_count;
  const Team<kThreads> team{s_scratch};
  const int tid = threadIdx.x, lane = lane_id(), count = parts.count;
  for (int64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
    const T* row = static_cast<const T*>(in.logits) + t * in.stride;
    const auto ahead = out.ahead(team, in, t, row);
    Soft a = no_soft();
    if (tid < count) {
      const Part own = parts.soft[t * count + tid];
      a = Soft{own.r, own.s, own.w};
    }
    if (tid == 0) s_count = 0;
    a = join<ENTROPY>(team, a, c);
    const Row p = row_of(a, in.scale);
    out.finish(team, in, t, ahead, a, p);
    if constexpr (TOP) {
      // The lists are in order: the least of the parts' m-th, m parts >= k, has k
      // pairs no smaller than itself.
      const int k = in.k, m = (k + count - 1) / count;
      const uint64_t* pairs = parts.pairs + t * count * k;
      uint64_t from = lane < count ? pairs[lane * k + m - 1] : ~uint64_t(0);
      from = ~lanes_max<kWave>(~from);
      for (int i = tid; i < count * k; i += kThreads) {
        const uint64_t pair = pairs[i];
        if (pair != 0 && pair >= from) s_list[atomicAdd(&s_count, 1)] = pair;
      }
      __syncthreads();
      rank_pairs(team, s_list, s_count, k, [&](int j, uint64_t pair) { out.alternative(t * k + j, pair, p); });
    }
    __syncthreads();
  }
}

// -------------------------------------------------------------------- launches

// Rows up to this many vectors are held by lanes.
constexpr int kShort = 512;

// How rows of `vectors` are cut: into parts of whole batches, so that there are
// about four workgroups to a compute unit, and batches enough for the maxima of a
// part that alternatives are chosen from.  A part has at least kLeastBatches: a row
// of no more is not cut, since a second launch costs more than these take (one row
// of 32,000 bfloat16 with 8 alternatives 8.9 us whole, 11.9 in two parts, 11.2 in
// four).  For rows that are cut anyway the least length matters less; microseconds
// with at least 2, 4 and 8 batches: one row of 131,072 with 8 alternatives 11.8,
// 12.7 and 14.1, 16 with 20 14.0, 15.6 and 17.9, 128 19.7, 18.8 and 20.1.
constexpr int kLeastBatches = 4;
struct Cut {
  int32_t count, length;
};
Cut cut_of(int64_t rows, int vectors, int k) {
  constexpr int kStep = kThreads * kBatch;
  const int batches = (vectors + kStep - 1) / kStep;
  int64_t count = rows > 0 ? (1024 + rows - 1) / rows : 1;
  if (k > 0) count = std::max<int64_t>(count, (batches + kMaxBatches - 1) / kMaxBatches);
  count = std::min<int64_t>({count, batches, kMaxParts});
  const int length = std::min(batches, std::max(kLeastBatches, (int)((batches + count - 1) / count)));
  return Cut{(batches + length - 1) / length, length * kStep};
}

int row_vectors(int64_t V, int dtype) {
  return dtype == BEVPOOL_F32 ? vectors_of<float>(V) : vectors_of<half_t>(V);
}

size_t forward_workspace(int64_t rows, int64_t V, int k, int dtype) {
  const int vectors = row_vectors(V, dtype);
  if (vectors <= kShort) return 0;
  const Cut cut = cut_of(rows, vectors, k);
  if (cut.count == 1) return 0;
  return rows * cut.count * (sizeof(Part) + k * sizeof(uint64_t)) + 16;  // (16: alignment)
}

// Rows that lanes hold; SMALL: what a row has beside its logits fits 16 lanes.
template <typename T, bool TOP, class SMALL, class ROW>
void launch_short(const LogitsRows& in, bool small, const SMALL& few_out, const ROW& out, hipStream_t stream) {
  const float c = exponent_factor(in.scale);
  const int vectors = vectors_of<T>(in.V);
  auto go = [&](auto lanes, auto held, const auto& row) {
    constexpr int kTeams = kThreads / lanes.value;
    const int64_t blocks = std::min<int64_t>((in.rows + kTeams - 1) / kTeams, kMaxBlocks);
    k_short_rows<T, lanes.value, held.value, TOP><<<(unsigned)blocks, kThreads, 0, stream>>>(in, row, c);
  };
  constexpr std::integral_constant<int, 16> few;
  constexpr std::integral_constant<int, kWave> wave;
  if (small && vectors <= 16) go(few, std::integral_constant<int, 1>{}, few_out);
  else if (small && vectors <= 32) go(few, std::integral_constant<int, 2>{}, few_out);
  else if (small && vectors <= 64) go(few, std::integral_constant<int, 4>{}, few_out);
  else if (vectors <= 128) go(wave, std::integral_constant<int, 2>{}, out);
  else if (vectors <= 256) go(wave, std::integral_constant<int, 4>{}, out);
  else go(wave, std::integral_constant<int, 8>{}, out);
}

template <typename T, bool ENTROPY, bool TOP, class ROW>
void launch_long(const LogitsRows& in, const ROW& out, void* workspace, hipStream_t stream) {
  const float c = exponent_factor(in.scale);
  const int vectors = vectors_of<T>(in.V);
  const Cut cut = cut_of(in.rows, vectors, TOP ? in.k : 0);
  Parts parts{in.rows * cut.count, cut.count, cut.length, nullptr, nullptr};
  if (cut.count > 1) {
    const uintptr_t at = (reinterpret_cast<uintptr_t>(workspace) + 15) & ~uintptr_t(15);
    parts.pairs = reinterpret_cast<uint64_t*>(at);
    parts.soft = reinterpret_cast<Part*>(parts.pairs + (TOP ? parts.total * in.k : 0));
  }
  k_row_parts<T, ENTROPY, TOP><<<(unsigned)std::min<int64_t>(parts.total, kMaxBlocks), kThreads, 0, stream>>>(
      in, out, c, parts);
  if (cut.count > 1)
    k_join_parts<T, ENTROPY, TOP><<<(unsigned)std::min<int64_t>(in.rows, kMaxBlocks), kThreads, 0, stream>>>(
        in, out, c, parts);
}

}  // namespace

size_t logprobs_workspace(int64_t rows, int64_t V, int32_t k, int dtype) {
  return forward_workspace(rows, V, k, dtype);
}
size_t distill_workspace(int64_t rows, int64_t V, int32_t, int dtype) {
  return forward_workspace(rows, V, 0, dtype);
}

hipError_t launch_logprobs_forward(const LogitsRows& in, const LogprobsOut& out, void* workspace,
                                   hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    const LogprobsRow row{out};
    const bool top = in.k > 0, entropy = out.entropy != nullptr;
    if (vectors_of<T>(in.V) <= kShort) {
      if (top) launch_short<T, true>(in, in.k <= 16, row, row, stream);
      else launch_short<T, false>(in, true, row, row, stream);
    } else if (entropy) {
      if (top) launch_long<T, true, true>(in, row, workspace, stream);
      else launch_long<T, true, false>(in, row, workspace, stream);
    } else {
      if (top) launch_long<T, false, true>(in, row, workspace, stream);
      else launch_long<T, false, false>(in, row, workspace, stream);
    }
  });
  return hipGetLastError();
}

hipError_t launch_distill_forward(const LogitsRows& in, float* loss, float* stats, void* workspace,
                                  hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  by_type(in.dtype, [&](auto t) {
    using T = decltype(t);
    const DistillRow<1> row{loss, stats};
    const DistillRow<4> four{loss, stats};  // (32 slots to 16 lanes, 256 to a wave)
    static_assert(4 * kWave == kMaxTaught, "slots of a wave");
    if (vectors_of<T>(in.V) > kShort) launch_long<T, false, false>(in, row, workspace, stream);
    else if (in.k <= 16) launch_short<T, false>(in, true, row, row, stream);
    else if (in.k <= 32) launch_short<T, false>(in, true, four, row, stream);
    else if (in.k <= kWave) launch_short<T, false>(in, false, row, row, stream);
    else launch_short<T, false>(in, false, four, four, stream);
  });
  return hipGetLastError();
}

}  // namespace bevpool
