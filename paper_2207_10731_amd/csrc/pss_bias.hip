// Learned relative position bias by buckets: scores + table[bucket], and the
// table's gradient.
#include "pss_rows.hpp"

namespace pss {

constexpr int kBiasThreads = 256;
constexpr int kBiasWaves = kBiasThreads / kWave;
constexpr int kMaxStart = 1 << 29;  // of q_starts
constexpr int kMaxNear = 1024;      // last border that lists and windows of distances hold

// Position of query 0 of batch b.  Positions stay below 3 * 2^29 and keys
// below 2^30: differences fit 32 bits.
__device__ __forceinline__ int32_t first_position(const BiasArgs& a, int64_t b) {
  int32_t s = a.q_starts != nullptr ? a.q_starts[b] : 0;
  s = s < 0 ? 0 : (s > kMaxStart ? kMaxStart : s);
  return static_cast<int32_t>(a.q_start) + s;
}

__device__ __forceinline__ float table_entry(const BiasArgs& a, int64_t i) {
  return a.table_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.table)[i])
                      : static_cast<const float*>(a.table)[i];
}
// Keys from k on, as an int; a lane takes 16 bytes of them at a time (kVec).
__device__ __forceinline__ int keys_left(int64_t k, int64_t K) { return static_cast<int>(K - k); }
// Elements of a row's last vector.
template <typename T>
__device__ __forceinline__ int key_rest(int64_t K) {
  return static_cast<int>(K) & (kVec<T> - 1);
}

// ---------------------------------------------------------------------------
// Forward, few queries (new tokens): 16 bytes of keys a lane.  Buckets are
// ranges of distances: keys beyond the last border (nearly all of a long cache)
// need no search.  A wavefront that has others copies the borders to LDS and, up to
// distances of 1024, makes a list of buckets there, a search to each distance and
// not to each key; farther, keys whose ends share a bucket need two searches.
// 64 x 16 x 1 x 4096 bfloat16: 7.1 us a call (a search to each key near the query
// 9.9), 16 x 32 x 1 x 32768: 14.6 us, 4.6 TB/s (19.7).  Both are one shape again and
// again; with a cache that grows by a token a call the first takes 9.4 (the host 7.1
// us instead of 6.0, and lengths that fill no tile).  Its kernel alone takes 7.6 us,
// not bound by memory (2.7) but by a chain: start positions, borders, list of
// buckets, table.
// ---------------------------------------------------------------------------
constexpr int kRowPieces = 4;

// WIDE: 64 lanes or more to a row, so that a wavefront has one.  A lane takes U pieces
// of keys, tx apart.
template <typename T, bool ENDS, bool PAST, bool WIDE, int U>
__global__ __launch_bounds__(kBiasThreads) void bias_row_kernel(const BiasArgs a,
                                                                const BucketMap map, const int tx,
                                                                const uint32_t k_tiles,
                                                                const uint32_t per) {
  constexpr int V = kVec<T>;
  constexpr End kEnd = ENDS ? End::kPieces : End::kWhole;
  __shared__ int32_t all_borders[kBiasWaves][kMaxBuckets];
  __shared__ uint8_t all_lists[kBiasWaves][kMaxNear];
  const int rest = key_rest<T>(a.K);
  const int x = threadIdx.x & (tx - 1), y = threadIdx.x / tx;
  const uint32_t kt = blockIdx.x % k_tiles;
  uint32_t row = tile_of(per, k_tiles) * (kBiasThreads / tx) + y;
  if (WIDE) row = __builtin_amdgcn_readfirstlane(row);
  const bool any = row < static_cast<uint32_t>(a.B * a.H * a.Q);
  if (WIDE && !any) return;
  const uint32_t bh = row / static_cast<uint32_t>(a.Q), q = row - bh * static_cast<uint32_t>(a.Q);
  const uint32_t b = bh / static_cast<uint32_t>(a.H), h = bh - b * static_cast<uint32_t>(a.H);
  const int64_t k0 = static_cast<int64_t>(kt) * U * tx * V;  // the tile's
  const T* in = static_cast<const T*>(a.in) + b * a.in_stride[0] + h * a.in_stride[1] +
                q * a.in_stride[2] + k0;
  T* out = static_cast<T*>(a.out) + b * a.out_stride[0] + h * a.out_stride[1] + q * a.out_stride[2] + k0;
  typename Vec<T>::type raw[U];
  int len[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    len[i] = any ? keys_left(k0 + (i * tx + x) * V, a.K) : 0;
    if (a.in != nullptr) raw[i] = load_vec<kEnd>(in + (i * tx + x) * V, len[i], rest);
  }
  const FarBuckets far = map.far;
  const int32_t pos = any ? first_position(a, b) + static_cast<int32_t>(q) : 0;
  const float t_behind = any ? table_entry(a, static_cast<int64_t>(far.behind) * a.H + h) : 0.f;
  const float t_ahead = any ? table_entry(a, static_cast<int64_t>(far.ahead) * a.H + h) : 0.f;
  int32_t* borders = all_borders[threadIdx.x >> 6];
  uint8_t* list = all_lists[threadIdx.x >> 6];
  const bool listed = far.near <= kMaxNear;
  bool copied = false;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int32_t rel = static_cast<int32_t>(k0) + (i * tx + x) * V - pos;
    const bool is_behind = rel + V - 1 <= -far.near;
    const bool is_near = len[i] > 0 && !is_behind && rel < far.from;
    float v[V];
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = is_behind ? t_behind : t_ahead;
    if (__any(is_near)) {
      if (!copied) {
        for (int j = threadIdx.x & (kWave - 1); j < map.side; j += kWave) borders[j] = map.borders[j];
        wave_lds_fence();
        if (listed) {
          for (int n = threadIdx.x & (kWave - 1); n < far.near; n += kWave)
            list[n] = static_cast<uint8_t>(bucket_of(-n, borders, map.side, map.both));
          wave_lds_fence();
        }
        copied = true;
      }
      if (is_near && listed) {
        int j[V];
#pragma unroll
        for (int u = 0; u < V; ++u) {
          const int32_t r = rel + u, n = r < 0 ? -r : r;
          const bool in_list = n < far.near && r < far.from;
          j[u] = list[in_list ? n : 0] + (r > 0 ? map.side : 0);
          if (!in_list) j[u] = r < far.from ? far.behind : far.ahead;
        }
#pragma unroll
        for (int u = 0; u < V; ++u) v[u] = table_entry(a, static_cast<int64_t>(j[u]) * a.H + h);
      } else if (is_near) {
        const int j0 = bucket_of(rel, borders, map.side, map.both);
        // behind the query buckets fall with the key, ahead of it they rise: equal
        // ends on one side of it hold all between
        const bool one = j0 == bucket_of(rel + V - 1, borders, map.side, map.both) &&
                         (rel >= 0 || rel + V - 1 <= 0);
        v[0] = table_entry(a, static_cast<int64_t>(j0) * a.H + h);
#pragma unroll
        for (int u = 1; u < V; ++u) v[u] = v[0];
        if (!one) {
#pragma unroll
          for (int u = 1; u < V; ++u)
            v[u] = table_entry(
                a, static_cast<int64_t>(bucket_of(rel + u, borders, map.side, map.both)) * a.H + h);
        }
      }
    }
    if (a.in != nullptr) {
      raw[i] = settle<kEnd>(raw[i], len[i], rest);
#pragma unroll
      for (int u = 0; u < V; ++u) v[u] += widen(raw[i][u]);
    }
    store_vec<ENDS, PAST>(out + (i * tx + x) * V, v, len[i]);
  }
}

// ---------------------------------------------------------------------------
// Forward, many queries.  The bias of a tile of queries and keys depends on
// key - query alone: a block writes the table's entries for the tile's
// differences to LDS once (tile's keys + queries of them, not keys x queries),
// and a lane reads for 8 queries and its keys the few that they take (8 keys: 15).
// The first scores are on their way meanwhile.  Short sequences: a block takes
// several (batch, head) pairs, a window of differences to each (as many as leave 2
// blocks to a CU: 1000 x 8 x 20 x 20 bfloat16 9 us, 19 with 8 blocks to a CU).
// Bound by memory, the scores read and written: 4 x 16 x 2048 x 2048 bfloat16
// 174 us, 6.2 TB/s (a bucket search to every element: 1162 us), float32 348 us, 6.2
// TB/s.  Rows that end inside a vector: 8 x 16 x 511 x 517 bfloat16 43 us, 3.1 TB/s,
// float32 69 us, 3.9 TB/s.
// ---------------------------------------------------------------------------
constexpr int kStep = 8;  // queries of a lane

struct BiasTile {
  uint32_t pairs;    // (batch, head) pairs of a block
  uint32_t groups;   // of lanes to a pair
  uint32_t q_tiles;  // of a pair
  uint32_t k_tiles;
  uint32_t per;      // tile_of
};

template <typename T, int TX, End E, bool PAST>
__global__ __launch_bounds__(kBiasThreads) void bias_tile_kernel(const BiasArgs a,
                                                                 const BucketMap map,
                                                                 const BiasTile tl) {
  constexpr int V = kVec<T>, TY = kBiasThreads / TX, kKeys = TX * V;
  __shared__ int32_t borders[kMaxBuckets];
  __shared__ float column[kMaxBuckets];
  __shared__ float windows[TY * (kKeys + kStep)];
  const uint32_t tile = tile_of(tl.per, tl.k_tiles), kt = blockIdx.x % tl.k_tiles;
  const uint32_t pt = tile / tl.q_tiles, qt = tile - pt * tl.q_tiles;
  const uint32_t H = static_cast<uint32_t>(a.H), all = static_cast<uint32_t>(a.B * a.H);
  const uint32_t bh0 = pt * tl.pairs;
  if (bh0 >= all) return;
  const int rows = static_cast<int>(tl.groups) * kStep;  // of a pair's tile
  const int64_t q0 = static_cast<int64_t>(qt) * rows, k0 = static_cast<int64_t>(kt) * kKeys;
  const int x = threadIdx.x % TX;
  const uint32_t y = threadIdx.x / TX;
  const uint32_t pair = tl.pairs == 1 ? 0 : y / tl.groups;
  const uint32_t bh = bh0 + pair, b = bh / H, h = bh - b * H;
  const bool mine = pair < tl.pairs && bh < all;
  const int64_t k = k0 + x * V;
  const int len = mine ? keys_left(k, a.K) : 0;
  const int rest = key_rest<T>(a.K);
  const int row = static_cast<int>(y - pair * tl.groups) * kStep;
  const int64_t q = q0 + row;
  const T* in = static_cast<const T*>(a.in) + b * a.in_stride[0] + h * a.in_stride[1] + k;
  typename Vec<T>::type raw[kStep];
  if (a.in != nullptr) {
#pragma unroll
    for (int j = 0; j < kStep; ++j)
      raw[j] = load_vec<E>(in + (q + j) * a.in_stride[2], q + j < a.Q ? len : 0, rest);
  }
  for (int i = threadIdx.x; i < map.num; i += kBiasThreads) {
    if (i < map.side) borders[i] = map.borders[i];
    if (tl.pairs == 1) column[i] = table_entry(a, static_cast<int64_t>(i) * a.H + h);
  }
  __syncthreads();
  const int size = kKeys + rows;  // of a window, with one more than it needs
  // difference of its first entry: the tile's first key, its last query
  const int32_t rel0 = static_cast<int32_t>(k0 - q0 - (rows - 1));
  const FarBuckets far = map.far;
  const auto bucket = [&](int32_t rel) {
    if (rel <= -far.near) return far.behind;
    return rel >= far.from ? far.ahead : bucket_of(rel, borders, map.side, map.both);
  };
  if (tl.pairs == 1) {
    const int32_t rel = rel0 - first_position(a, b);
    for (int i = threadIdx.x; i < size - 1; i += kBiasThreads) windows[i] = column[bucket(rel + i)];
  } else {
    for (uint32_t i = threadIdx.x; i < tl.pairs * size; i += kBiasThreads) {
      const uint32_t w = i / size, bh1 = bh0 + w, b1 = bh1 / H;
      if (bh1 >= all) break;
      const int32_t rel = rel0 - first_position(a, b1) + static_cast<int32_t>(i - w * size);
      windows[i] = table_entry(a, static_cast<int64_t>(bucket(rel)) * a.H + bh1 - b1 * H);
    }
  }
  __syncthreads();
  if (len <= 0 || q >= a.Q) return;
  const float* window = windows + pair * size;
  T* out = static_cast<T*>(a.out) + b * a.out_stride[0] + h * a.out_stride[1] + k;
  // bias of query q + j and key k + u: near[7 + u - j]
  const int at = x * V + rows - 1 - row - (kStep - 1);
  float near[V + kStep - 1];
#pragma unroll
  for (int i = 0; i < V + kStep - 1; ++i) near[i] = window[at + i];
#pragma unroll
  for (int j = 0; j < kStep; ++j) {
    if (q + j >= a.Q) break;
    float v[V];
    if (a.in != nullptr) raw[j] = settle<E>(raw[j], len, rest);
#pragma unroll
    for (int u = 0; u < V; ++u) {
      v[u] = near[kStep - 1 + u - j];
      if (a.in != nullptr) v[u] += widen(raw[j][u]);
    }
    store_vec<E != End::kWhole, PAST>(out + (q + j) * a.out_stride[2], v, len);
  }
}

// Lanes along the keys, `vec` keys each, `least` to `most`: as many as there are
// keys, but several tiles of fewer lanes where more than an eighth of the lanes
// would have none (511 x 517 bfloat16, 65 vectors in tiles of 16 lanes instead of
// 128).
static int key_lanes(int64_t K, int vec, int least, int most) {
  const int64_t pieces = (K + vec - 1) / vec;
  int tx = least;
  while (tx < pieces && tx < most) tx *= 2;
  const auto lanes = [&](int t) { return (pieces + t - 1) / t * t; };
  int64_t fewest = lanes(tx);
  for (int t = tx / 2; t >= 16 && t >= least; t /= 2) fewest = lanes(t) < fewest ? lanes(t) : fewest;
  while (lanes(tx) > fewest + fewest / 8) tx /= 2;
  return tx;
}

// launch(whether the results go past the caches)
template <typename F>
static hipError_t by_store(bool past, F launch) {
  return past ? launch(std::true_type{}) : launch(std::false_type{});
}

template <typename T>
static hipError_t launch_bias_t(const BiasArgs& a, const BucketMap& map, hipStream_t stream) {
  const dim3 block(kBiasThreads);
  const int tx = key_lanes(a.K, kVec<T>, 4, kBiasThreads), ty = kBiasThreads / tx;
  const int64_t keys = static_cast<int64_t>(tx) * kVec<T>;
  const int64_t k_tiles = (a.K + keys - 1) / keys, bh = a.B * a.H;
  // (several narrow bfloat16 rows to a wavefront that are not whole lines: 9% slower
  // past the caches)
  const bool past = bh * a.Q * a.K * static_cast<int64_t>(sizeof(T)) > kPastBytes &&
                    (sizeof(T) == 4 || tx >= kWave || a.K % 32 == 0);
  if (a.Q < kStep && bh * a.Q <= INT32_MAX) {
    // several pieces a lane, as long as they leave 2 blocks to a CU (16 x 32 x 1 x 32768
    // float32 26 against 30 us)
    int pieces = 1, lanes = tx;
    for (int n = kRowPieces; n > 1 && pieces == 1; n /= 2) {
      const int64_t step = n * kVec<T>;  // keys of a lane
      if (a.K < step * kWave) continue;
      const int t = key_lanes(a.K, static_cast<int>(step), kWave, kBiasThreads);
      const int64_t rows = kBiasThreads / t, across = step * t;
      if ((bh * a.Q + rows - 1) / rows * ((a.K + across - 1) / across) < 512) continue;
      pieces = n;
      lanes = t;
    }
    const int64_t rows = kBiasThreads / lanes, across = static_cast<int64_t>(lanes) * pieces * kVec<T>;
    const int64_t tiles = (a.K + across - 1) / across;
    const TileGrid tg = tile_grid((bh * a.Q + rows - 1) / rows, tiles);
    if (!tg.fits) return hipErrorInvalidConfiguration;
    const auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, tg.grid, block, 0, stream, a, map, lanes,
                         static_cast<uint32_t>(tiles), tg.per);
      return hipGetLastError();
    };
    const auto with_ends = [&](auto ends) {
      return by_store(past, [&](auto to) {
        if (lanes < kWave) return launch(bias_row_kernel<T, ends.value, to.value, false, 1>);
        return with_const<1, 2, kRowPieces>(pieces, [&](auto n) {
          return launch(bias_row_kernel<T, ends.value, to.value, true, n.value>);
        });
      });
    };
    return a.K % kVec<T> ? with_ends(std::true_type{}) : with_ends(std::false_type{});
  }
  BiasTile tl;
  tl.pairs = 1;
  tl.groups = ty;
  int64_t q_tiles = 1;
  const int64_t q_steps = (a.Q + kStep - 1) / kStep;
  if (k_tiles == 1 && 2 * q_steps <= ty) {
    tl.groups = static_cast<uint32_t>(q_steps);
    tl.pairs = ty / tl.groups;  // fewer if that leaves less than 2 blocks to a CU
    while (tl.pairs > 1 && bh < 512 * static_cast<int64_t>(tl.pairs)) tl.pairs /= 2;
  } else {
    q_tiles = (q_steps + ty - 1) / ty;
  }
  const int64_t tiles = (bh + tl.pairs - 1) / tl.pairs * q_tiles;
  const TileGrid tg = tile_grid(tiles, k_tiles);
  // (tile_of of a slice past the end stays below 2^32 too)
  if (!tg.fits || tiles > INT32_MAX) return hipErrorInvalidConfiguration;
  tl.q_tiles = static_cast<uint32_t>(q_tiles);
  tl.k_tiles = static_cast<uint32_t>(k_tiles);
  tl.per = tg.per;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, tg.grid, block, 0, stream, a, map, tl);
    return hipGetLastError();
  };
  return with_const<4, 8, 16, 32, 64, 128, 256>(tx, [&](auto lanes) {
    constexpr int TX = lanes.value;
    return by_store(past, [&](auto to) {
      if (a.K % kVec<T> == 0) return launch(bias_tile_kernel<T, TX, End::kWhole, to.value>);
      // the lane with a row's end has the elements before it in its own wavefront,
      // unless it is the first one
      if (a.K / kVec<T> % (TX < kWave ? TX : kWave) != 0)
        return launch(bias_tile_kernel<T, TX, End::kOverlap, to.value>);
      return launch(bias_tile_kernel<T, TX, End::kPieces, to.value>);
    });
  });
}

hipError_t launch_bias(bool bf16, const BiasArgs& a, const BucketMap& map, hipStream_t stream) {
  return bf16 ? launch_bias_t<uint16_t>(a, map, stream) : launch_bias_t<float>(a, map, stream);
}

// ---------------------------------------------------------------------------
// The table's gradient.  All pairs at one difference key - query share a
// bucket, and all beyond the last border share one on each side: a wavefront
// keeps one sum per difference up to that border (near) in its window in LDS
// and the two far sums in registers, over all of its rows, whatever their
// batch.  A lane takes V keys (16 bytes) of QU queries at a time.  Such blocks of
// elements that are far are summed whole; in a near one the V x QU elements lie
// on V + QU - 1 diagonals, summed in registers first and added to the window V at
// a time, so that no two lanes of a group share a difference (lane x's begin V x
// above lane 0's), one group after the other.  At the end every
// bucket, a range of differences, sums its part of the window.  Every sum
// has a fixed order.  Bound by memory, one read of the gradient: 4 x 16 x 2048 x
// 2048 bfloat16 93 us, 5.8 TB/s (5 for the blocks' sums); small calls by their
// launches.
// ---------------------------------------------------------------------------
// Units that one block takes alone (1 x 16 x 128 x 128 bfloat16: 7.6 against 9.7 us a
// call; twice as many, 16 x 8 x 1 x 512: 11.6 against 9.6).
constexpr int kAloneUnits = 2 * kBiasWaves;
constexpr int kNearPad = 2 * kStep;   // differences a near block reaches beyond it

// Differences key - query that bucket j holds, lo .. hi (hi < lo: none).
__device__ __forceinline__ void bucket_range(int j, const int32_t* borders, const BucketMap& map,
                                             int32_t* lo, int32_t* hi) {
  const bool ahead = map.both && j >= map.side;
  const int i = ahead ? j - map.side : j;
  const int32_t n0 = borders[i], n1 = i + 1 < map.side ? borders[i + 1] : INT32_MAX;
  if (ahead) {
    *lo = n0 < 1 ? 1 : n0;
    *hi = n1 - 1;
  } else {
    *lo = 1 - n1;
    // keys ahead of the query count as distance 0 on a single side
    *hi = !map.both && n0 == 0 && n1 > 0 ? INT32_MAX : -n0;
  }
}


// at[i] += diag[i] (i < V + QU - 1) from lanes whose `at` are V apart, within
// groups that take turns: from the top, V at a time, so that no two lanes add to
// one element at once.  The wavefront's lanes take part together.
template <int V, int N, int GROUPS>
__device__ __forceinline__ void add_diagonals(float* at, const float diag[N], bool mine, int group) {
  for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
    for (int top = N - 1; top >= 0; top -= V) {
      if (mine && group == g) {
#pragma unroll
        for (int i = top; i > top - V && i >= 0; --i) at[i] += diag[i];
      }
      wave_lds_fence();
    }
  }
}

struct NearShape {
  int tx;           // lanes of a group: they share rows
  int qu;           // queries of a lane's step, beside 8 / qu pieces of keys
  int64_t q_steps;  // steps of qu queries of one sequence
  int64_t k_steps;  // steps of keys
  int64_t units;    // of a wavefront: a step of each of its groups
  int blocks;       // of a head
  int window;       // floats of a wavefront's window
};
static bool is_near(const BucketMap& map) { return map.borders[map.side - 1] <= kMaxNear; }
static NearShape near_shape(bool bf16, const BiasArgs& a, const BucketMap& map) {
  NearShape s;
  const int vec = bf16 ? kVec<uint16_t> : kVec<float>;
  s.tx = key_lanes(a.K, vec, 8, kWave);
  s.qu = kStep;
  while (s.qu > 1 && s.qu / 2 >= a.Q) s.qu /= 2;
  const int64_t keys = static_cast<int64_t>(s.tx) * vec * (kStep / s.qu);
  const int groups = kWave / s.tx;
  s.q_steps = (a.Q + s.qu - 1) / s.qu;
  s.k_steps = (a.K + keys - 1) / keys;
  s.units = (a.B * s.q_steps + groups - 1) / groups * s.k_steps;
  // a unit a wavefront, up to 8 blocks to a CU over all heads; few are one block's,
  // which saves the sum's launch
  const int64_t want = s.units <= kAloneUnits ? 1 : (s.units + kBiasWaves - 1) / kBiasWaves;
  const int64_t most = 2048 / a.H < 1 ? 1 : 2048 / a.H;
  s.blocks = static_cast<int>(want < most ? want : most);
  const int near = map.borders[map.side - 1];
  s.window = near + kNearPad + (map.both ? near : 0) + kNearPad + 1;
  return s;
}

template <typename T, int TX, int QU, End E>
__global__ __launch_bounds__(kBiasThreads) void bias_grad_near_kernel(
    const BiasArgs a, const BucketMap map, const uint32_t q_steps, const uint32_t k_steps,
    const int64_t units, const int window, float* __restrict__ part,
    float* __restrict__ grad_table) {
  constexpr int V = kVec<T>, KU = kStep / QU, kGroups = kWave / TX;
  extern __shared__ float windows[];  // [wavefront][window]
  __shared__ int32_t borders[kMaxBuckets];
  __shared__ float far[2][kBiasWaves];
  for (int i = threadIdx.x; i < map.side; i += kBiasThreads) borders[i] = map.borders[i];  // the end's
  const int near = map.far.near;
  const int ahead = map.far.from;          // differences from here on are far
  const int zero = near + kNearPad;                        // window[zero]: difference 0
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = lane % TX, group = lane / TX;
  float* mine = windows + wave * window;
  for (int i = lane; i < window; i += kWave) mine[i] = 0.f;
  wave_lds_fence();
  const uint32_t h = blockIdx.y;
  // the wavefront's units: rows of steps, each k_steps long
  const int64_t waves = static_cast<int64_t>(gridDim.x) * kBiasWaves;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kBiasWaves + wave;
  const int64_t each = units / waves, more = units - each * waves;
  int64_t unit = w * each + (w < more ? w : more);
  const int64_t end = unit + each + (w < more ? 1 : 0);
  uint32_t row = static_cast<uint32_t>(unit / k_steps);
  uint32_t kt = static_cast<uint32_t>(unit - static_cast<int64_t>(row) * k_steps);
  const uint32_t rows = static_cast<uint32_t>(a.B) * q_steps;
  const int rest = key_rest<T>(a.K);
  float behind_sum = 0.f, ahead_sum = 0.f;
  for (; unit < end; ++unit) {
    const uint32_t r = row * kGroups + group;  // this group's step
    const uint32_t b = r / q_steps;
    const int64_t q = static_cast<int64_t>(r - b * q_steps) * QU;
    const int left = r < rows ? (a.Q - q < QU ? static_cast<int>(a.Q - q) : QU) : 0;
    const int64_t k0 = (static_cast<int64_t>(kt) * KU * TX + x) * V;
    const T* in = static_cast<const T*>(a.in) + b * a.in_stride[0] + h * a.in_stride[1] +
                  q * a.in_stride[2] + k0;
    typename Vec<T>::type raw[KU][QU];
#pragma unroll
    for (int c = 0; c < KU; ++c) {
      const int len = keys_left(k0 + c * (TX * V), a.K);
#pragma unroll
      for (int j = 0; j < QU; ++j)
        raw[c][j] = load_vec<E>(in + j * a.in_stride[2] + c * (TX * V), j < left ? len : 0, rest);
    }
    const int32_t pos = (left > 0 ? first_position(a, b) : 0) + static_cast<int32_t>(q);
#pragma unroll
    for (int c = 0; c < KU; ++c) {
      const int32_t k = static_cast<int32_t>(k0) + c * (TX * V);
      // the block's differences: low .. high
      const int32_t low = k - (pos + QU - 1), high = k + V - 1 - pos;
      const bool is_behind = high <= -near, is_ahead = low >= ahead;
      const bool is_near = !is_behind && !is_ahead && left > 0 && k < a.K;
      float diag[V + QU - 1];  // of low + i
#pragma unroll
      for (int i = 0; i < V + QU - 1; ++i) diag[i] = 0.f;
#pragma unroll
      for (int j = 0; j < QU; ++j) {
        raw[c][j] = settle<E>(raw[c][j], j < left ? keys_left(k, a.K) : 0, rest);
#pragma unroll
        for (int u = 0; u < V; ++u) diag[QU - 1 + u - j] += widen(raw[c][j][u]);
      }
      if (!is_near) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V + QU - 1; ++i) sum += diag[i];
        if (is_behind) behind_sum += sum; else ahead_sum += sum;
      }
      if (__any(is_near)) {
        add_diagonals<V, V + QU - 1, kGroups>(mine + zero + low, diag, is_near, group);
      }
    }
    if (++kt == k_steps) {
      kt = 0;
      ++row;
    }
  }
  behind_sum = wave_sum(behind_sum);
  ahead_sum = wave_sum(ahead_sum);
  if (lane == 0) {
    far[0][wave] = behind_sum;
    far[1][wave] = ahead_sum;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < window; i += kBiasThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kBiasWaves; ++k) v += windows[k * window + i];
    windows[i] = v;
  }
  __syncthreads();
  const int behind_bucket = map.far.behind, ahead_bucket = map.far.ahead;
  for (int j = wave; j < map.num; j += kBiasWaves) {
    int32_t lo, hi;
    bucket_range(j, borders, map, &lo, &hi);
    lo = lo < -zero ? -zero : lo;
    hi = hi > window - 1 - zero ? window - 1 - zero : hi;
    float v = 0.f;
    for (int i = lo + lane; i <= hi; i += kWave) v += windows[zero + i];
    v = wave_sum(v);
#pragma unroll
    for (int k = 0; k < kBiasWaves; ++k) {
      if (j == behind_bucket) v += far[0][k];
      if (j == ahead_bucket) v += far[1][k];
    }
    if (lane != 0) continue;
    if (gridDim.x == 1)  // no others to join
      grad_table[j * a.H + h] = v;
    else  // [head][bucket][block]
      part[(static_cast<int64_t>(h) * map.num + j) * gridDim.x + blockIdx.x] = v;
  }
}

// ---------------------------------------------------------------------------
// The same for maps with borders farther than that: the window holds the
// differences of one tile of keys and up to 64 queries, and every tile sums its
// buckets (8 x 16 x 512 x 512 bfloat16, 64 buckets to distance 3000: 58 us; 32 buckets
// to 128, by the form above: 21.  4 x 16 x 2048 x 2048: 115 and 93).
constexpr int kMaxGradRows = 64;  // queries of one group's tile

struct FarShape {
  int tx;           // lanes of a group
  int rows;         // queries of a group
  int64_t k_tiles;  // of one (b, h)
  int64_t q_tiles;  // blocks of groups along the queries of one (b, h, k tile)
};
static FarShape far_shape(bool bf16, const BiasArgs& a) {
  FarShape s;
  const int vec = bf16 ? kVec<uint16_t> : kVec<float>;
  s.tx = key_lanes(a.K, vec, 16, kWave);
  const int groups = kBiasThreads / s.tx;
  const int64_t keys = static_cast<int64_t>(s.tx) * vec;
  s.k_tiles = (a.K + keys - 1) / keys;
  // many queries, as long as they leave 8 blocks to a CU
  s.rows = kMaxGradRows;
  while (s.rows > kStep &&
         a.B * a.H * s.k_tiles * ((a.Q + groups * s.rows - 1) / (groups * s.rows)) < 2048)
    s.rows /= 2;
  s.q_tiles = (a.Q + groups * s.rows - 1) / (groups * s.rows);
  return s;
}

template <typename T, int TX, End E>
__global__ __launch_bounds__(kBiasThreads) void bias_grad_far_kernel(
    const BiasArgs a, const BucketMap map, const int rows, const int64_t q_tiles,
    const int64_t k_tiles, const uint32_t per, float* __restrict__ part) {
  constexpr int V = kVec<T>, kGroups = kBiasThreads / TX, kKeys = TX * V;
  constexpr int kWaveGroups = kWave / TX, kDiagonals = V + kStep - 1;
  __shared__ float windows[kGroups][kKeys + kMaxGradRows];
  __shared__ int32_t borders[kMaxBuckets];
  __shared__ float sums[kBiasWaves][kMaxBuckets];
  const uint32_t blk = tile_of(per, 1);
  const int64_t kt = blk % k_tiles, qt = blk / k_tiles % q_tiles, bh = blk / (k_tiles * q_tiles);
  const int64_t b = bh / a.H, h = bh - b * a.H;
  if (b >= a.B) return;
  const int x = threadIdx.x % TX, group = threadIdx.x / TX;
  for (int i = x; i < kKeys + kMaxGradRows; i += TX) windows[group][i] = 0.f;
  for (int i = threadIdx.x; i < map.side; i += kBiasThreads) borders[i] = map.borders[i];
  __syncthreads();
  const int64_t q0 = (qt * kGroups + group) * rows, k = kt * kKeys + x * V;
  const int len = keys_left(k, a.K), rest = key_rest<T>(a.K);
  const T* in = static_cast<const T*>(a.in) + b * a.in_stride[0] + h * a.in_stride[1] + k;
  for (int s = 0; s < rows; s += kStep) {
    const int64_t q = q0 + s;
    typename Vec<T>::type raw[kStep];
#pragma unroll
    for (int j = 0; j < kStep; ++j)
      raw[j] = load_vec<E>(in + (q + j) * a.in_stride[2], q + j < a.Q ? len : 0, rest);
    float diag[kDiagonals];  // of difference k - q - 7 + i
#pragma unroll
    for (int i = 0; i < kDiagonals; ++i) diag[i] = 0.f;
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      raw[j] = settle<E>(raw[j], q + j < a.Q ? len : 0, rest);
#pragma unroll
      for (int u = 0; u < V; ++u) diag[kStep - 1 + u - j] += widen(raw[j][u]);
    }
    // groups have windows of their own: no turns
    add_diagonals<V, kDiagonals, 1>(windows[group] + x * V + rows - kStep - s, diag, true, 0);
  }
  __syncthreads();
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const int32_t first = first_position(a, b);
  for (int j = 0; j < map.num; ++j) {
    int32_t lo, hi;
    bucket_range(j, borders, map, &lo, &hi);
    float v = 0.f;
    bool any = false;
#pragma unroll
    for (int g = 0; g < kWaveGroups; ++g) {
      const int at = wave * kWaveGroups + g;
      // difference of windows[at][0]: the tile's first key, the group's last query
      const int64_t rel0 = kt * kKeys - ((qt * kGroups + at) * rows + rows - 1) - first;
      const int64_t from = lo - rel0 < 0 ? 0 : lo - rel0;
      const int64_t to = hi - rel0 >= kKeys + rows - 1 ? kKeys + rows - 2 : hi - rel0;
      if (from > to) continue;
      any = true;
      for (int i = static_cast<int>(from) + lane; i <= to; i += kWave) v += windows[at][i];
    }
    if (any) v = wave_sum(v);
    if (lane == 0) sums[wave][j] = v;
  }
  __syncthreads();
  // [head][bucket][batch, tile]
  const int64_t parts = a.B * q_tiles * k_tiles;
  for (int j = threadIdx.x; j < map.num; j += kBiasThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kBiasWaves; ++w) v += sums[w][j];
    part[(h * map.num + j) * parts + (b * q_tiles + qt) * k_tiles + kt] = v;
  }
}

// A block an entry of the table.
__global__ __launch_bounds__(kBiasThreads) void bias_sum_kernel(const float* __restrict__ part,
                                                                const int64_t parts, const int num,
                                                                const int64_t heads,
                                                                float* __restrict__ out) {
  __shared__ float lds[kBiasWaves];
  const int64_t h = blockIdx.x / num;
  const int j = static_cast<int>(blockIdx.x % num);
  float v = 0.f;
  for (int64_t i = threadIdx.x; i < parts; i += kBiasThreads) v += part[blockIdx.x * parts + i];
  v = wave_sum(v);
  if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = 0.f;
    for (int w = 0; w < kBiasWaves; ++w) v += lds[w];
    out[j * heads + h] = v;
  }
}

// Parts of one entry (0: one block writes the entries), and whether the grids hold
// the call.
static int64_t grad_parts(bool bf16, const BiasArgs& a, const BucketMap& map) {
  if (is_near(map)) {
    const int blocks = near_shape(bf16, a, map).blocks;
    return blocks > 1 ? blocks : 0;
  }
  const FarShape s = far_shape(bf16, a);
  return a.B * s.q_tiles * s.k_tiles;
}
bool bias_grad_fits(bool bf16, const BiasArgs& a, const BucketMap& map) {
  if (a.H * map.num > INT32_MAX) return false;
  if (is_near(map)) {
    const NearShape s = near_shape(bf16, a, map);
    return a.B <= INT32_MAX / s.q_steps;
  }
  const FarShape s = far_shape(bf16, a);
  return a.B * a.H <= INT32_MAX / s.q_tiles / s.k_tiles;
}

size_t bias_grad_workspace_bytes(bool bf16, const BiasArgs& a, const BucketMap& map) {
  return static_cast<size_t>(a.H * map.num * grad_parts(bf16, a, map)) * sizeof(float);
}

// f(how rows of K keys end): gradients are only read, so that a row of a vector or
// more may always be read with the elements before its end.
template <typename T, typename F>
static hipError_t by_key_end(int64_t K, F f) {
  if (K % kVec<T> == 0) return f(std::integral_constant<End, End::kWhole>{});
  return K > kVec<T> ? f(std::integral_constant<End, End::kOverlap>{})
                     : f(std::integral_constant<End, End::kPieces>{});
}
template <typename T>
static hipError_t launch_near(const BiasArgs& a, const BucketMap& map, const NearShape& s,
                              float* part, float* grad_table, hipStream_t stream) {
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(s.blocks, static_cast<uint32_t>(a.H)), dim3(kBiasThreads),
                       kBiasWaves * s.window * sizeof(float), stream, a, map,
                       static_cast<uint32_t>(s.q_steps), static_cast<uint32_t>(s.k_steps), s.units,
                       s.window, part, grad_table);
    return hipGetLastError();
  };
  return by_key_end<T>(a.K, [&](auto end) {
    return with_const<8, 16, 32, 64>(s.tx, [&](auto lanes) {
      constexpr End E = end.value;
      if constexpr (E == End::kPieces && lanes.value != 8) {
        return hipErrorInvalidValue;  // not reached: less than a vector of keys has 8 lanes
      } else {
        return with_const<1, 2, 4, 8>(s.qu, [&](auto qu) {
          return launch(bias_grad_near_kernel<T, lanes.value, qu.value, E>);
        });
      }
    });
  });
}
template <typename T>
static hipError_t launch_far(const BiasArgs& a, const BucketMap& map, const FarShape& s, float* part,
                             hipStream_t stream) {
  const TileGrid tg = tile_grid(a.B * a.H * s.q_tiles * s.k_tiles, 1);  // (bias_grad_fits)
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, tg.grid, dim3(kBiasThreads), 0, stream, a, map, s.rows, s.q_tiles,
                       s.k_tiles, tg.per, part);
    return hipGetLastError();
  };
  return by_key_end<T>(a.K, [&](auto end) {
    return with_const<16, 32, 64>(s.tx, [&](auto lanes) {
      constexpr End E = end.value;
      if constexpr (E == End::kPieces && lanes.value != 16) {
        return hipErrorInvalidValue;  // not reached: less than a vector of keys has 16 lanes
      } else {
        return launch(bias_grad_far_kernel<T, lanes.value, E>);
      }
    });
  });
}
template <typename T>
static hipError_t launch_grad_t(const BiasArgs& a, const BucketMap& map, float* part,
                                float* grad_table, hipStream_t stream) {
  return is_near(map) ? launch_near<T>(a, map, near_shape(sizeof(T) == 2, a, map), part, grad_table,
                                       stream)
                      : launch_far<T>(a, map, far_shape(sizeof(T) == 2, a), part, stream);
}

hipError_t launch_bias_grad(bool bf16, const BiasArgs& a, const BucketMap& map, void* workspace,
                            float* grad_table, hipStream_t stream) {
  float* part = static_cast<float*>(workspace);
  const hipError_t e = bf16 ? launch_grad_t<uint16_t>(a, map, part, grad_table, stream)
                            : launch_grad_t<float>(a, map, part, grad_table, stream);
  if (e != hipSuccess || grad_parts(bf16, a, map) == 0) return e;
  hipLaunchKernelGGL(bias_sum_kernel, dim3(static_cast<uint32_t>(a.H * map.num)), dim3(kBiasThreads), 0,
                     stream, part, grad_parts(bf16, a, map), map.num, a.H, grad_table);
  return hipGetLastError();
}

}  // namespace pss
