// Embedding lookup with a scale, and the table's gradient: the rows of each id
// summed through the ids' stable order, so that every table row is written by
// one owner, without atomics.  Bound by memory: the forward by the
// rows it writes, the gradient by the table it fills.

#include "device_utils.h"
#include "rows.h"
#include "rows_sort.h"
#include "rows_vec.h"

namespace bevpool {

namespace {

template <typename T, typename TO, typename TKey>
__global__ __launch_bounds__(kRowThreads) void k_embed(const T* __restrict__ table, int64_t stride,
                                                       RowSplit s, const TKey* __restrict__ ids,
                                                       int32_t table_rows, float scale,
                                                       TO* __restrict__ out) {
  constexpr int N = RowVec<T>::N;
  for_row_vectors<N>(s, [&](int64_t i, int32_t c) {
    const int32_t id = key_or_drop(ids, i, table_rows);
    const int left = s.C - c;
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = 0.f;
    if (id < table_rows) {
      load_row<T>(table + id * stride + c, left, v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= scale;
    }
    store_row<TO>(out + i * s.C + c, left, v);
  });
}

// Table gradient.  The sorted slots are cut into equal ranges of RG, whatever
// ids they hold: a few ids are very frequent and most occur once or never, so
// work assigned by id would wait for the frequent ones.
//
//   k_embed_ranges  a lane group walks its range with kInFlight rows in flight
//                   and stores the sum of every id whose slots lie in the
//                   range.  The sum of an id that comes from the range before
//                   is that range's partial 2 r, of one that starts here and
//                   goes on into the next 2 r + 1 (float32 rows).
//   k_embed_rest    blocks of ids fill the rows of ids that do not occur;
//                   lane groups, one to a range, add up the partials of the id
//                   that starts in the range and goes on, in range order; the
//                   block's groups share an id of many partials and add their
//                   sums in group order.
//
// Measured with 16,384 ids of a text (the most frequent 917 times) and a
// bfloat16 table of 131072 x 4096 (1.07 GB): ranges 45 us, rest 172 us (its fill
// runs at 6.0 TB/s), where one owner per table row took 1866 us.
struct Ranges {
  const int32_t* order;
  const int32_t* keys;     // of the sorted slots
  int32_t* offsets;        // [n_keys + 1]
  float* partials;         // [2 * ranges][C]
  int64_t n;               // slots
  int64_t ranges;
  int32_t RG;
  int32_t n_keys;
  int32_t C;
};

constexpr int kInFlight = 8;   // rows a lane group has in flight
constexpr int kJoinFlight = 4;  // and partials

template <typename T, typename TO, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void k_embed_ranges(const T* __restrict__ grad_out,
                                                              int64_t stride, Ranges a,
                                                              unsigned range_blocks, int32_t W,
                                                              int32_t tiles, float scale,
                                                              TO* __restrict__ grad_table) {
  using V = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N;
  if (blockIdx.x >= range_blocks) {  // (an id to a thread, where the sort has not left the offsets)
    const int64_t v = (int64_t)(blockIdx.x - range_blocks) * kRowThreads + threadIdx.x;
    if (v <= a.n_keys) a.offsets[v] = (int32_t)keys_below(a.keys, a.n, v);
    return;
  }
  // group of W lanes: one range, vectors [tile W, tile W + W) of its rows
  const int group = threadIdx.x / W;
  const int G = kRowThreads / W;
  if (group >= G) return;
  const int64_t item = (int64_t)blockIdx.x * G + group;
  const int64_t r = item / tiles;
  if (r >= a.ranges) return;
  const int vec = (int)(item - r * tiles) * W + threadIdx.x - group * W;
  if (vec * N >= a.C) return;
  const int c = vector_start<N>(vec, a.C);
  const int left = a.C - c;
  const int64_t p0 = r * a.RG;
  const int32_t m = (int32_t)min<int64_t>(a.RG, a.n - p0);
  const int32_t before = p0 > 0 ? a.keys[p0 - 1] : -1;
  const int32_t after = p0 + m < a.n ? a.keys[p0 + m] : -1;
  const int32_t* order = a.order + p0;
  const int32_t* keys = a.keys + p0;
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  int32_t cur = keys[0];
  if (cur >= a.n_keys) return;  // (dropped slots, like all behind them)
  auto flush = [&]() {
    if (cur >= a.n_keys) {
      // (dropped slots at the end of the kept ones)
    } else if (cur == before || cur == after) {
      const int64_t slot = 2 * r + (cur == before ? 0 : 1);
      store_row<float>(a.partials + slot * a.C + c, left, acc);
    } else if (cur >= 0) {
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] *= scale;
      store_row<TO>(grad_table + (int64_t)cur * a.C + c, left, acc);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
  };
  for (int32_t q0 = 0; q0 < m; q0 += kInFlight) {
    V g[kInFlight];
    int32_t key[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int32_t q = min(q0 + u, m - 1);  // (a repeat past the end, not added)
      key[u] = keys[q];
      g[u] = load_raw<T, STREAM>(grad_out + order[q] * stride + c, left);
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (q0 + u >= m) break;
      if (key[u] != cur) {
        flush();
        cur = key[u];
      }
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += (float)g[u][e];
    }
  }
  flush();
}

// Adds the n partials from j0 on, `step` apart, of an id that starts in range r.
template <int N>
__device__ __forceinline__ void add_partials(const Ranges& a, int64_t r, int64_t j0, int64_t step,
                                             int64_t n, int c, float (&acc)[N]) {
  // (the second partial of the range where it starts, the first of the others)
  auto at = [&](int64_t j) { return a.partials + (2 * (r + j) + (j == 0 ? 1 : 0)) * a.C + c; };
  int64_t j = j0;
  for (; j + (kJoinFlight - 1) * step < n; j += kJoinFlight * step) {
    float g[kJoinFlight][N];
#pragma unroll
    for (int u = 0; u < kJoinFlight; ++u) load_row<float>(at(j + u * step), a.C - c, g[u]);
#pragma unroll
    for (int u = 0; u < kJoinFlight; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += g[u][e];
  }
  for (; j < n; j += step) {
    float g[N];
    load_row<float>(at(j), a.C - c, g);
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] += g[e];
  }
}

// Blocks [0, fill): rows of ids that do not occur.  The others: ranges of one
// tile of W vectors of 4 elements, one to each of the block's G lane groups;
// a group joins an id of a few partials, the whole block one of more.
template <typename TO>
__global__ __launch_bounds__(kRowThreads) void k_embed_rest(RowSplit s, Ranges a, int64_t fill,
                                                            int32_t W, int32_t tiles, float scale,
                                                            TO* __restrict__ grad_table) {
  if (blockIdx.x < fill) {
    constexpr int N = RowVec<TO>::N;
    const float zero[N] = {};
    const int32_t parts = (s.cv + s.cvb - 1) / s.cvb;
    const int32_t c0 = (int32_t)(blockIdx.x % parts) * s.cvb;
    for (int64_t row0 = (int64_t)(blockIdx.x / parts) * s.R; row0 < s.rows;
         row0 += fill / parts * s.R) {
      const int32_t items = (int32_t)min<int64_t>(s.R, s.rows - row0) * s.cvb;
      for (uint32_t i = threadIdx.x; i < (uint32_t)items; i += kRowThreads) {
        const uint32_t q = s.by.div(i);
        const int32_t vec = c0 + (int32_t)(i - q * (uint32_t)s.cvb);
        const int32_t c = vector_start<N>(vec, s.C);
        const int64_t v = row0 + q;
        if (vec < s.cv && a.offsets[v] == a.offsets[v + 1])
          store_row<TO>(grad_table + v * s.C + c, s.C - c, zero);
      }
    }
    return;
  }
  constexpr int N = 4;
  constexpr int kMaxGroups = kRowThreads;
  __shared__ float s_sum[kRowThreads][N + 1];
  __shared__ int32_t s_many[kMaxGroups];  // partials that the block has to join for each group, or 0
  const int G = kRowThreads / W;
  const int group = threadIdx.x / W;
  const int64_t item = blockIdx.x - fill;
  const int64_t r0 = item / tiles * G;
  const int vec = (int)(item % tiles) * W + threadIdx.x - group * W;
  const bool on = group < G && vec * N < a.C;
  const int c = vector_start<N>(vec, a.C);
  // the id that starts in range r and goes on: its number of partials, or 0
  auto partials_from = [&](int64_t r, int32_t& v) -> int64_t {
    const int64_t p1 = (r + 1) * a.RG;  // first slot of the next range
    if (r >= a.ranges || p1 >= a.n) return 0;
    v = a.keys[p1];
    if (a.keys[p1 - 1] != v || v < 0 || v >= a.n_keys) return 0;
    const int32_t begin = a.offsets[v], end = a.offsets[v + 1];
    if (begin < p1 - a.RG || begin >= p1 || end <= p1) return 0;  // (it starts in an earlier range)
    return (end - 1) / a.RG - r + 1;
  };
  auto finish = [&](int32_t v, float (&acc)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] *= scale;
    store_row<TO>(grad_table + (int64_t)v * a.C + c, a.C - c, acc);
  };
  int32_t v = 0;
  const int64_t n = group < G ? partials_from(r0 + group, v) : 0;
  if (on && n > 0 && n <= kJoinFlight) {
    float acc[N] = {};
    add_partials<N>(a, r0 + group, 0, 1, n, c, acc);
    finish(v, acc);
  }
  if (group < G && threadIdx.x == group * W) s_many[group] = n > kJoinFlight ? (int32_t)n : 0;
  __syncthreads();
  for (int q = 0; q < G; ++q) {
    const int32_t many = s_many[q];
    if (many == 0) continue;  // (uniform over the block)
    float acc[N] = {};
    if (on) add_partials<N>(a, r0 + q, group, G, many, c, acc);
#pragma unroll
    for (int e = 0; e < N; ++e) s_sum[threadIdx.x][e] = acc[e];
    __syncthreads();
    if (group == 0 && on) {
      for (int g = 1; g < G; ++g)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += s_sum[g * W + threadIdx.x][e];
      finish(a.keys[(r0 + q + 1) * a.RG], acc);
    }
    __syncthreads();  // (the sums have been read)
  }
}

// Slots per range.  A long range is a long chain of loads for its group, a
// short one leaves more partials: 8 until the groups (about 512 elements wide)
// are 8,192, then longer ones; and up to a third of an id's mean count, at most
// 64, where every id has many slots to join.  Microseconds of the whole
// gradient (with its sort) with ranges of 8, 16, 32, 64 and 128 slots, launches
// back to back in a graph on ids of which none is padding:
//   16,384 slots, 131,072 ids (text), C = 4096, bfloat16   272  268  266  284  319  (takes 16)
//   130,160 slots, 16,384 ids (even), C = 80, float32       44   43   50   63   90  (16)
//   2,048 slots, 32,000 ids (text), C = 1024, bfloat16      27   31   39   56   88  (8)
//   65,536 slots, 1,000 ids (even), C = 1024, bfloat16      68   61   55   67   95  (32)
//   65,536 slots, 3 ids, C = 512, float32                  177  112   78   75   97  (64)
int32_t range_slots(int64_t n, int64_t n_keys, int64_t C) {
  const int64_t tiles = (C + 511) / 512;
  int32_t RG = 8;
  while (RG < 128 && n * tiles / RG > 8192) RG *= 2;
  while (RG < 64 && RG < n / n_keys / 3) RG *= 2;
  return RG;
}

}  // namespace

hipError_t launch_embed_forward(int64_t n, int64_t table_rows, int64_t C, int in_dtype,
                                int out_dtype, const void* table, int64_t table_stride,
                                int key_type, const void* ids, float scale, void* out,
                                hipStream_t stream) {
  if (n == 0) return hipSuccess;
  by_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    const RowSplit s = row_split(n, C, RowVec<T>::N);
    auto go = [&](auto* keys) {
      k_embed<T, TO><<<row_grid(s), kRowThreads, 0, stream>>>(
          static_cast<const T*>(table), table_stride, s, keys, (int32_t)table_rows, scale,
          static_cast<TO*>(out));
    };
    if (key_type == BEVPOOL_KEY_I64) go(static_cast<const int64_t*>(ids));
    else go(static_cast<const int32_t*>(ids));
  });
  return hipGetLastError();
}

EmbedLayout embed_layout(int64_t n, int64_t table_rows, int64_t C) {
  EmbedLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  L.sort = take(sort_layout(n, table_rows).total);
  L.order = take(sizeof(int32_t) * (size_t)n);
  L.keys = take(sizeof(int32_t) * (size_t)n);
  L.offsets = take(sizeof(int32_t) * (size_t)(table_rows + 1));
  L.RG = range_slots(n, table_rows, C);
  L.ranges = (n + L.RG - 1) / L.RG;
  L.partials = take(L.ranges > 1 ? sizeof(float) * 2 * (size_t)L.ranges * (size_t)C : 0);
  L.total = off;
  return L;
}

hipError_t launch_embed_backward(int64_t n, int64_t table_rows, int64_t C, int in_dtype,
                                 int out_dtype, const void* grad_out, int64_t grad_stride,
                                 int key_type, const void* ids, float scale, void* grad_table,
                                 void* workspace, hipStream_t stream) {
  const EmbedLayout L = embed_layout(n, table_rows, C);
  char* ws = static_cast<char*>(workspace);
  int32_t* order = reinterpret_cast<int32_t*>(ws + L.order);
  int32_t* keys = reinterpret_cast<int32_t*>(ws + L.keys);
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + L.offsets);
  const bool search = n > 0 && sort_layout(n, table_rows).passes > 1;
  const hipError_t e = launch_sort_keys(n, table_rows, key_type, ids, order, nullptr,
                                        search ? nullptr : offsets, keys, ws + L.sort, stream);
  if (e != hipSuccess) return e;
  const Ranges a{order, keys, offsets, reinterpret_cast<float*>(ws + L.partials), n,
                 L.ranges, L.RG, (int32_t)table_rows, (int32_t)C};
  // lanes of a group and column tiles, for vectors of `per` elements
  auto lanes = [&](int64_t per, int64_t* tiles) {
    const int64_t cv = (C + per - 1) / per;
    *tiles = (cv + kWave - 1) / kWave;
    return (int32_t)((cv + *tiles - 1) / *tiles);
  };
  by_any_types(in_dtype, out_dtype, [&](auto ti, auto to) {
    using T = decltype(ti);
    using TO = decltype(to);
    TO* out = static_cast<TO*>(grad_table);
    int64_t tiles;
    if (n > 0) {
      const int32_t W = lanes(RowVec<T>::N, &tiles);
      const int64_t G = kRowThreads / W;
      const int64_t blocks = (L.ranges * tiles + G - 1) / G;
      const int64_t searches = search ? table_rows / kRowThreads + 1 : 0;
      auto go = [&](auto hint) {
        k_embed_ranges<T, TO, hint.value>
            <<<(unsigned)(blocks + searches), kRowThreads, 0, stream>>>(
                static_cast<const T*>(grad_out), grad_stride, a, (unsigned)blocks, W,
                (int32_t)tiles, scale, out);
      };
      if (stream_rows(n, C, sizeof(T))) go(std::true_type{});
      else go(std::false_type{});
    }
    const RowSplit s = row_split(table_rows, C, RowVec<TO>::N);
    const int64_t parts = (s.cv + s.cvb - 1) / s.cvb;
    const int64_t fill = std::min((s.rows + s.R - 1) / s.R, std::max<int64_t>(1, kMaxBlocks / parts)) * parts;
    const int32_t W = lanes(4, &tiles);
    const int64_t G = kRowThreads / W;
    const int64_t joins = L.ranges > 1 ? (L.ranges + G - 1) / G * tiles : 0;
    k_embed_rest<TO><<<(unsigned)(fill + joins), kRowThreads, 0, stream>>>(
        s, a, fill, W, (int32_t)tiles, scale, out);
  });
  return hipGetLastError();
}

}  // namespace bevpool
