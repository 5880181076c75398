// Operators on rows: dropout from a counter-based generator, layer norm and
// its backward pass.
#include "pss_rows.hpp"

namespace pss {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kMaxWaves = 16;  // of a block that takes a row together
constexpr int kSpanCols = kWave * kLanePiece;  // columns of a wavefront's span

// Columns from c on, as an int (a span has at most 512).
__device__ __forceinline__ int cols_left(int64_t c, int64_t cols) {
  return cols - c > INT32_MAX ? INT32_MAX : static_cast<int>(cols - c);
}

// Which of the block's groups of G lanes: one value a wavefront for G = 64, so that
// a row's addresses stay out of the lanes' registers.
template <int G>
__device__ __forceinline__ int group_of() {
  const int g = threadIdx.x / G;
  return G == kWave ? __builtin_amdgcn_readfirstlane(g) : g;
}

// Lanes to a row: as many as its pieces of 8, up to a wavefront.
static int row_lanes(int64_t cols) {
  const int64_t pieces = (cols + kLanePiece - 1) / kLanePiece;
  int g = 1;
  while (g < pieces && g < kWave) g *= 2;
  return g;
}

// f(a T, whether rows of `cols` end inside a vector)
template <typename F>
static hipError_t by_row_type(bool bf16, int64_t cols, F f) {
  const std::true_type yes;
  const std::false_type no;
  if (bf16) return cols % kVec<uint16_t> ? f(uint16_t{}, yes) : f(uint16_t{}, no);
  return cols % kVec<float> ? f(float{}, yes) : f(float{}, no);
}

// ---------------------------------------------------------------------------
// out = residual + D(x): a span of a row to a group of G lanes.  Ten rounds of the
// generator make the numbers of 8 elements, about 60 instructions that the loads
// hide: bound by memory, 2 row arrays or 3.  32768 x 4096 bfloat16 with residual:
// 121 us, 6.6 TB/s; 16384 x 3328 float32: 68 us, 6.4 TB/s (a large copy: 6.2).
// ---------------------------------------------------------------------------
template <typename T, int G, bool ENDS, bool PAST>
__global__ __launch_bounds__(kRowThreads) void dropout_kernel(const RowsIn x, const RowsIn residual,
                                                              const RowsOut out, const int64_t rows,
                                                              const int64_t cols,
                                                              const uint32_t spans,
                                                              const uint32_t per, const Drop drop) {
  typedef Span<T, G, ENDS> S;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const uint32_t tile = tile_of(per, spans), span = blockIdx.x % spans;
  const int lane = threadIdx.x % G;
  const int64_t r = static_cast<int64_t>(tile) * (kRowThreads / G) + group_of<G>();
  const int64_t c = static_cast<int64_t>(span) * (G * kLanePiece);
  if (r >= rows) return;
  const int left = cols_left(c, cols);
  S a, b;
  a.load(static_cast<const T*>(x.p) + r * x.stride + c, lane, left);
  if (residual.p != nullptr)
    b.load(static_cast<const T*>(residual.p) + r * residual.stride + c, lane, left);
  float v[kLanePiece];
  a.settle_end(lane, left);
  a.widen_to(v);
  if (drop.t) S::drop(v, drop, n, span * G, static_cast<uint32_t>(r), lane);
  if (residual.p != nullptr) {
    float q[kLanePiece];
    b.settle_end(lane, left);
    b.widen_to(q);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] += q[u];
  }
  S::template store<PAST>(static_cast<T*>(out.p) + r * out.stride + c, v, lane, left);
}

// Kernels whose stores gain past the caches: those of whole lines, which a
// wavefront's bfloat16 rows fill and float32 ones (in two stores, a span's halves)
// if they are wide (norm of 1048576 x 16 float32 without residual: 40 us past them,
// 32 through them; of 524288 x 64: 47 and 50).
template <typename T, int G, bool ENDS>
constexpr bool kGainsPast = sizeof(T) == 2 || G == kWave || (!ENDS && G >= 8);
// launch(whether the results go past the caches)
template <typename T, int G, bool ENDS, typename F>
static hipError_t by_store(int64_t elements, F launch) {
  if constexpr (kGainsPast<T, G, ENDS>) {
    if (elements * static_cast<int64_t>(sizeof(T)) > kPastBytes) return launch(std::true_type{});
  }
  return launch(std::false_type{});
}

template <typename T, bool ENDS>
static hipError_t launch_dropout_t(const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                                   int64_t rows, int64_t cols, const Drop& drop,
                                   hipStream_t stream) {
  const int g = row_lanes(cols);
  const int64_t spans = (cols + g * kLanePiece - 1) / (g * kLanePiece);
  const int64_t tiles = (rows * g + kRowThreads - 1) / kRowThreads;
  const TileGrid tg = tile_grid(tiles, spans);
  if (!tg.fits) return hipErrorInvalidConfiguration;
  // (float32 with a residual: 3 to 6% slower past the caches)
  const int64_t stored = sizeof(T) == 4 && residual.p != nullptr ? 0 : rows * cols;
  return with_const<1, 2, 4, 8, 16, 32, 64>(g, [&](auto lanes) {
    constexpr int G = lanes.value;
    return by_store<T, G, ENDS>(stored, [&](auto past) {
      hipLaunchKernelGGL((dropout_kernel<T, G, ENDS, past.value>), tg.grid, dim3(kRowThreads), 0,
                         stream, x, residual, out, rows, cols, static_cast<uint32_t>(spans), tg.per,
                         drop);
      return hipGetLastError();
    });
  });
}

hipError_t launch_dropout(bool bf16, const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                          int64_t rows, int64_t cols, const Drop& drop, hipStream_t stream) {
  return by_row_type(bf16, cols, [&](auto t, auto ends) {
    return launch_dropout_t<decltype(t), ends.value>(x, residual, out, rows, cols, drop, stream);
  });
}

// ---------------------------------------------------------------------------
// Layer norm.  Rows of up to 16384 columns are read once and stay in
// registers: up to 1024 columns a group of lanes takes a row, beyond that a block
// of as many wavefronts as the row fills.  Groups and blocks walk over rows, with
// the row after the present one already requested and the weights in
// registers.  Bound by memory: 2 to 4 row arrays read or written.  425984 x 128
// float32: 71 us, 6.2 TB/s; 16384 x 4096 bfloat16 with residual and dropout:
// 100 us, 5.4 TB/s (a block a row that reads it three times: 909 and 175 us).
// ---------------------------------------------------------------------------

// What a row needs of one span.
template <typename T, int G, bool ENDS>
struct NormSpan {
  Span<T, G, ENDS> x, q;
  __device__ __forceinline__ void load(const NormArgs& a, int64_t r, int64_t c, int lane, int left,
                                       bool there = true) {
    x.load(static_cast<const T*>(a.x.p) + r * a.x.stride + c, lane, left, there);
    if (a.residual.p != nullptr)
      q.load(static_cast<const T*>(a.residual.p) + r * a.residual.stride + c, lane, left, there);
  }
  // s = residual + D(x)
  __device__ __forceinline__ void sum_to(float v[kLanePiece], const NormArgs& a, const Drop& drop,
                                         uint64_t n, int64_t r, int64_t c, int lane, int left) {
    x.settle_end(lane, left);
    x.widen_to(v);
    if (drop.t)
      Span<T, G, ENDS>::drop(v, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r),
                             lane);
    if (a.residual.p != nullptr) {
      float w[kLanePiece];
      q.settle_end(lane, left);
      q.widen_to(w);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) v[u] += w[u];
    }
  }
};

template <typename T, int G, bool ENDS, bool PAST>
__device__ __forceinline__ void norm_store(float v[kLanePiece], const NormArgs& a, int64_t r,
                                           int64_t c, int lane, int left, float mean, float rstd,
                                           const float w[kLanePiece], const float b[kLanePiece]) {
  typedef Span<T, G, ENDS> S;
  if (a.sum.p != nullptr)
    S::template store<PAST>(static_cast<T*>(a.sum.p) + r * a.sum.stride + c, v, lane, left);
#pragma unroll
  for (int u = 0; u < kLanePiece; ++u) v[u] = (v[u] - mean) * rstd * w[u] + b[u];
  S::template store<PAST>(static_cast<T*>(a.out.p) + r * a.out.stride + c, v, lane, left);
}

__device__ __forceinline__ void norm_store_stats(const NormArgs& a, int64_t r, float mean,
                                                 float rstd) {
  if (a.mean != nullptr) a.mean[r] = mean;
  if (a.rstd != nullptr) a.rstd[r] = rstd;
}

// Squares of a span's elements about `mean`.
template <typename T, int G, bool ENDS>
__device__ __forceinline__ float squares(const float v[kLanePiece], int lane, int left, float mean) {
  float sq = 0.f;
#pragma unroll
  for (int u = 0; u < kLanePiece; ++u) {
    const int at = ENDS ? u : u / kVec<T> * kVec<T>;  // whole vectors are in or out
    const float e = Span<T, G, ENDS>::col(lane, at) < left ? v[u] - mean : 0.f;
    sq += e * e;
  }
  return sq;
}

// A group of G lanes a row, NP spans.  AHEAD: the next row is requested before the
// present one's sums.  (4 wavefronts to a SIMD: at most 128 registers.)
template <typename T, int G, bool ENDS, bool PAST, int NP, bool AHEAD>
__global__ __launch_bounds__(kRowThreads, 4) void norm_group_kernel(const NormArgs a, const Drop drop) {
  constexpr int kRows = kRowThreads / G, kSpan = G * kLanePiece;
  const int lane = threadIdx.x % G;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + group_of<G>();
  NormSpan<T, G, ENDS> in[NP], next[NP];
  float w[NP][kLanePiece], b[NP][kLanePiece];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    in[i].load(a, r, i * kSpan, lane, cols - i * kSpan, r < a.rows);
    Span<T, G, ENDS>::weights(w[i], a.weight, a.weight_bf16, i * kSpan, lane, cols - i * kSpan, 1.f);
    Span<T, G, ENDS>::weights(b[i], a.bias, a.weight_bf16, i * kSpan, lane, cols - i * kSpan, 0.f);
  }
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.rows; r0 += step, r += step) {
    if (AHEAD && r0 + step < a.rows) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        next[i].load(a, r + step, i * kSpan, lane, cols - i * kSpan, r + step < a.rows);
    }
    float v[NP][kLanePiece], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      in[i].sum_to(v[i], a, drop, n, r, i * kSpan, lane, cols - i * kSpan);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum += v[i][u];
    }
    const float mean = group_sum<G>(sum) * inv;
#pragma unroll
    for (int i = 0; i < NP; ++i) sq += squares<T, G, ENDS>(v[i], lane, cols - i * kSpan, mean);
    const float rstd = 1.f / sqrtf(group_sum<G>(sq) * inv + a.eps);
    if (r < a.rows) {
      if (lane == 0) norm_store_stats(a, r, mean, rstd);
#pragma unroll
      for (int i = 0; i < NP; ++i)
        norm_store<T, G, ENDS, PAST>(v[i], a, r, i * kSpan, lane, cols - i * kSpan, mean, rstd, w[i], b[i]);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (AHEAD)
        in[i] = next[i];
      else
        in[i].load(a, r + step, i * kSpan, lane, cols - i * kSpan, r + step < a.rows);
    }
  }
}

// Wavefront k of n has the spans at columns (i n + k) * kSpanCols, i < NP: how many
// elements of a row of `cols`.
template <int NP>
__device__ __forceinline__ float part_size(int k, int n, int cols) {
  int e = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int left = cols - (i * n + k) * kSpanCols;
    e += left < 0 ? 0 : (left > kSpanCols ? kSpanCols : left);
  }
  return static_cast<float>(e);
}

// A block a row.  Every wavefront takes mean and squares of its own part; the
// parts are joined through LDS with one barrier a row (the squares about the
// common mean are those about each part's plus the part's size times the square
// of its mean's distance).
template <typename T, int TH, bool ENDS, bool PAST, int NP, bool AHEAD>
__global__ __launch_bounds__(TH, 4) void norm_block_kernel(const NormArgs a, const Drop drop) {
  __shared__ float lds[2][2][kMaxWaves];
  const int lane = threadIdx.x & (kWave - 1), wave = group_of<kWave>();
  const int waves = blockDim.x >> 6;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  int64_t r = blockIdx.x;
  NormSpan<T, kWave, ENDS> in[NP], next[NP];
  float w[NP][kLanePiece], b[NP][kLanePiece];
  int c[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    c[i] = (i * waves + wave) * kSpanCols;
    in[i].load(a, r, c[i], lane, cols - c[i]);
    Span<T, kWave, ENDS>::weights(w[i], a.weight, a.weight_bf16, c[i], lane, cols - c[i], 1.f);
    Span<T, kWave, ENDS>::weights(b[i], a.bias, a.weight_bf16, c[i], lane, cols - c[i], 0.f);
  }
  const float my_size = part_size<NP>(wave, waves, cols);
  const float inv_part = my_size > 0.f ? 1.f / my_size : 0.f;
  const int other = lane % kMaxWaves;  // the part this lane joins
  const float size = other < waves ? part_size<NP>(other, waves, cols) : 0.f;
  int turn = 0;
  for (; r < a.rows; r += gridDim.x, turn ^= 1) {
    const int64_t after = r + gridDim.x;
    if (AHEAD && after < a.rows) {
#pragma unroll
      for (int i = 0; i < NP; ++i) next[i].load(a, after, c[i], lane, cols - c[i]);
    }
    float v[NP][kLanePiece], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      in[i].sum_to(v[i], a, drop, n, r, c[i], lane, cols - c[i]);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum += v[i][u];
    }
    const float part = wave_sum(sum) * inv_part;
#pragma unroll
    for (int i = 0; i < NP; ++i) sq += squares<T, kWave, ENDS>(v[i], lane, cols - c[i], part);
    sq = wave_sum(sq);
    if (lane == 0) {
      lds[turn][0][wave] = part;
      lds[turn][1][wave] = sq;
    }
    __syncthreads();  // the other half of lds is free again at the next row's
    const float their_mean = other < waves ? lds[turn][0][other] : 0.f;
    const float their_sq = other < waves ? lds[turn][1][other] : 0.f;
    const float mean = group_sum<kMaxWaves>(size * their_mean) * inv;
    const float away = size > 0.f ? their_mean - mean : 0.f;  // (a square may overflow)
    const float var = group_sum<kMaxWaves>(their_sq + size * (away * away)) * inv;
    const float rstd = 1.f / sqrtf(var + a.eps);
    if (threadIdx.x == 0) norm_store_stats(a, r, mean, rstd);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      norm_store<T, kWave, ENDS, PAST>(v[i], a, r, c[i], lane, cols - c[i], mean, rstd, w[i], b[i]);
      if (AHEAD)
        in[i] = next[i];
      else if (after < a.rows)
        in[i].load(a, after, c[i], lane, cols - c[i]);
    }
  }
}

// Sums of two values over the block, in every thread, in a fixed order.
__device__ __forceinline__ void block_sum2(float& a, float& b, float* lds) {
  a = wave_sum(a);
  b = wave_sum(b);
  const int w = threadIdx.x >> 6;
  __syncthreads();  // the last values are read
  if ((threadIdx.x & (kWave - 1)) == 0) {
    lds[w] = a;
    lds[kRowWaves + w] = b;
  }
  __syncthreads();
  a = b = 0.f;
#pragma unroll
  for (int i = 0; i < kRowWaves; ++i) {
    a += lds[i];
    b += lds[kRowWaves + i];
  }
}

// Wider rows: a block a row, which it reads three times (sum, squares about the
// mean, result), the last two from L2.  Nothing is stored before the last pass,
// where every element is read by the lane that then stores its results.  1024 x
// 30000 float32: 92 us, 2.7 TB/s of the two arrays, bound by the three reads one
// after the other (a request in flight to each lane); with residual and dropout 180
// us, the mask made three times.
template <typename T, bool ENDS, bool PAST>
__global__ __launch_bounds__(kRowThreads, 4) void norm_wide_kernel(const NormArgs a, const Drop drop) {
  __shared__ float lds[2 * kRowWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t first = group_of<kWave>() * kSpanCols, step = kRowWaves * kSpanCols;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const float inv = 1.f / static_cast<float>(a.cols);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float sum = 0.f, zero = 0.f;
#pragma unroll 1
    for (int64_t c = first; c < a.cols; c += step) {
      NormSpan<T, kWave, ENDS> in;
      float v[kLanePiece];
      in.load(a, r, c, lane, cols_left(c, a.cols));
      in.sum_to(v, a, drop, n, r, c, lane, cols_left(c, a.cols));
      float piece = 0.f;  // of its own: a long row's chain of additions is 8 times shorter
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) piece += v[u];
      sum += piece;
    }
    block_sum2(sum, zero, lds);
    const float mean = sum * inv;
    float sq = 0.f;
#pragma unroll 1
    for (int64_t c = first; c < a.cols; c += step) {
      NormSpan<T, kWave, ENDS> in;
      float v[kLanePiece];
      in.load(a, r, c, lane, cols_left(c, a.cols));
      in.sum_to(v, a, drop, n, r, c, lane, cols_left(c, a.cols));
      sq += squares<T, kWave, ENDS>(v, lane, cols_left(c, a.cols), mean);
    }
    block_sum2(sq, zero, lds);
    const float rstd = 1.f / sqrtf(sq * inv + a.eps);
    if (threadIdx.x == 0) norm_store_stats(a, r, mean, rstd);
#pragma unroll 1
    for (int64_t c = first; c < a.cols; c += step) {
      NormSpan<T, kWave, ENDS> in;
      float v[kLanePiece], w[kLanePiece], b[kLanePiece];
      const int left = cols_left(c, a.cols);
      in.load(a, r, c, lane, left);
      in.sum_to(v, a, drop, n, r, c, lane, left);
      Span<T, kWave, ENDS>::weights(w, a.weight, a.weight_bf16, c, lane, left, 1.f);
      Span<T, kWave, ENDS>::weights(b, a.bias, a.weight_bf16, c, lane, left, 0.f);
      norm_store<T, kWave, ENDS, PAST>(v, a, r, c, lane, left, mean, rstd, w, b);
    }
  }
}

// Which kernel takes rows of `cols` columns, and how many of its wavefronts a
// CU holds (by their registers).
struct RowForm {
  int lanes;  // of a row: a group (<= 64), else a block of that many threads
  int spans;  // of a lane; 0: the wide kernel
  int waves;  // of a CU
};
constexpr int kHeld = 16;     // wavefronts of 128 registers
constexpr int kHeldBf16 = 20;  // of the forward's bfloat16 kernel of one span

// Blocks of whole wavefronts beyond 1024 columns, one or two spans a lane.  Two hold
// more rows on a CU but need more registers: bfloat16 takes them for half as many
// rows again (8192 x 4096: 28 against 34 us; 25000 x 1300, 8 rows against 6: 45
// against 37), float32, whose spans are twice the bytes, only where a CU would be
// left with one row (4096 x 8192: 49 against 55 us; 8192 x 4096 with residual and
// dropout, 4 rows against 2: 100 against 94; the others without either).  Two-span
// blocks of an odd number of wavefronts leave a
// SIMD without its share (8192 x 4104 float32: 5 wavefronts 57 us, 6 54).
static RowForm norm_form(bool bf16, int64_t cols) {
  const int64_t n = (cols + kLanePiece - 1) / kLanePiece;
  if (n <= kWave) return {row_lanes(cols), 1, kHeld};
  if (n <= 2 * kWave) return {kWave, 2, kHeld};
  const int64_t w1 = (n + kWave - 1) / kWave, half = (n + 2 * kWave - 1) / (2 * kWave);
  const int64_t w2 = half > 1 ? (half + 1) / 2 * 2 : 1;
  if (w2 > kMaxWaves) return {kRowThreads, 0, kRowWaves};
  const int64_t held = bf16 ? kHeldBf16 : kHeld;
  const int64_t rows1 = w1 <= kMaxWaves ? held / w1 : 0, rows2 = kHeld / w2;
  const bool two = rows1 == 0 || (bf16 ? 2 * rows2 >= 3 * rows1 : rows1 == 1 && rows2 > 1);
  if (two) return {static_cast<int>(w2) * kWave, 2, kHeld};
  return {static_cast<int>(w1) * kWave, 1, static_cast<int>(held)};
}
// Blocks that walk rows: what the CUs hold, with as many rows to each (a last
// round of a few rows takes as long as the others: norm of 16000 x 2500 float32
// without residual 55 against 57 us).  Narrow rows, many to a block, fill the CUs instead (backward of 53248 x
// 128 float32 20.9 against 21.6 us).
static uint32_t row_blocks(const RowForm& f, int64_t rows) {
  const bool group = f.lanes <= kWave;
  const int64_t per_block = group ? kRowThreads / f.lanes : 1;
  const int64_t want = (rows + per_block - 1) / per_block;
  const int64_t held = int64_t{256} * (f.waves * kWave / (group ? kRowThreads : f.lanes));
  const int64_t rounds = (want + held - 1) / held;
  if (f.lanes < kWave && rounds > 2) return static_cast<uint32_t>(held);
  return static_cast<uint32_t>((want + rounds - 1) / rounds);
}

// The forward of rows of whole vectors: groups take a row and are done, or two
// without a residual, rather than walk over the array, where the results go past the
// caches and for bfloat16 with a residual (262144 x 128 with residual and dropout:
// float32 90 against 96 us, bfloat16 50 against 53; without, float32 45 against 47; but
// 65536 x 256 float32, results through the caches, 52 against 50).  Half-empty bfloat16
// spans (40000 x 520) lose by it, and so do rows that end inside a vector.
template <typename T, bool ENDS, bool PAST>
static uint32_t norm_blocks(const RowForm& f, const NormArgs& a) {
  const uint32_t walking = row_blocks(f, a.rows);
  const bool gains = PAST || (sizeof(T) == 2 && a.residual.p != nullptr);
  if (ENDS || !gains || f.lanes > kWave || (sizeof(T) == 2 && f.spans == 2)) return walking;
  const int64_t each = (kRowThreads / f.lanes) * (a.residual.p != nullptr ? 1 : 2);
  const int64_t blocks = (a.rows + each - 1) / each;
  return blocks < kGridBlocks ? static_cast<uint32_t>(blocks) : walking;
}

template <typename T, bool ENDS>
static hipError_t launch_norm_t(const NormArgs& a, const Drop& drop, hipStream_t stream) {
  const RowForm f = norm_form(sizeof(T) == 2, a.cols);
  const dim3 block(f.lanes <= kWave ? kRowThreads : f.lanes);
  constexpr bool kAhead2 = sizeof(T) == 2;  // two float32 spans ahead: too many registers
  const auto launch = [&](auto kernel, uint32_t blocks) {
    hipLaunchKernelGGL(kernel, dim3(blocks), block, 0, stream, a, drop);
    return hipGetLastError();
  };
  if (f.lanes < kWave) {
    return with_const<1, 2, 4, 8, 16, 32>(f.lanes, [&](auto lanes) {
      constexpr int G = lanes.value;
      return by_store<T, G, ENDS>(a.rows * a.cols, [&](auto past) {
        return launch(norm_group_kernel<T, G, ENDS, past.value, 1, true>,
                      norm_blocks<T, ENDS, past.value>(f, a));
      });
    });
  }
  return by_store<T, kWave, ENDS>(a.rows * a.cols, [&](auto past) {
    constexpr bool PAST = past.value;
    if (f.spans == 0)
      return launch(norm_wide_kernel<T, ENDS, PAST>, static_cast<uint32_t>(a.rows < 2048 ? a.rows : 2048));
    const uint32_t blocks = norm_blocks<T, ENDS, PAST>(f, a);
    if (f.lanes == kWave)
      return f.spans == 1 ? launch(norm_group_kernel<T, kWave, ENDS, PAST, 1, true>, blocks)
                          : launch(norm_group_kernel<T, kWave, ENDS, PAST, 2, kAhead2>, blocks);
    if (f.spans == 1) return launch(norm_block_kernel<T, 1024, ENDS, PAST, 1, true>, blocks);
    return f.lanes <= 512 ? launch(norm_block_kernel<T, 512, ENDS, PAST, 2, kAhead2>, blocks)
                          : launch(norm_block_kernel<T, 1024, ENDS, PAST, 2, false>, blocks);
  });
}

hipError_t launch_norm(bool bf16, const NormArgs& a, const Drop& drop, hipStream_t stream) {
  return by_row_type(bf16, a.cols, [&](auto t, auto ends) {
    return launch_norm_t<decltype(t), ends.value>(a, drop, stream);
  });
}

// ---------------------------------------------------------------------------
// Backward.  Each block adds what its rows give to the weight's and bias's
// gradients in registers and writes them to its own row of parts
// ([blocks][2][cols]); sum_parts_kernel adds the blocks' rows in order.  A few
// rows are one block's, which writes the gradients themselves.
// Bound by memory: 3 to 5 row arrays.  16384 x 4096 bfloat16 with residual and
// dropout: 125 us, 5.4 TB/s (122 and 5 for the parts' sum in calls one after the other;
// 105 for a first one, before whose stores none wait to reach memory); 53248 x 128
// float32: 21 us (18 and 4), 3.9 TB/s.  (Stored past the caches: 3 to 16% slower.)
// ---------------------------------------------------------------------------

// Where a block's sums go: element c of block k's at weight[k * 2 * cols + c] (of
// one block: the gradients); null: not wanted.
struct SumsOut {
  float* weight = nullptr;
  float* bias = nullptr;
};

// rstd for the sums over a span, whose lanes past the row's end have h = 0 and z =
// -mean * rstd: 0 where that overflows and 0 * z would be NaN.  The forward keeps such
// values of constant rows alone, where z is 0 with any rstd (one element a rounding
// away from the mean leaves |mean| * rstd at about 2^40 at most).  (A test of each
// element's column instead: backward of 8192 x 4099 bfloat16 83 against 74 us.)
__device__ __forceinline__ float sums_rstd(float mean, float rstd) {
  return isfinite(mean * rstd) ? rstd : 0.f;
}

// What a row needs of one span.
template <typename T, int G, bool ENDS>
struct GradSpan {
  Span<T, G, ENDS> dy, s, up;
  __device__ __forceinline__ void load(const NormGradArgs& a, int64_t r, int64_t c, int lane,
                                       int left, bool there = true) {
    dy.load(static_cast<const T*>(a.grad.p) + r * a.grad.stride + c, lane, left, there);
    s.load(static_cast<const T*>(a.s.p) + r * a.s.stride + c, lane, left, there);
    if (a.grad_sum.p != nullptr)
      up.load(static_cast<const T*>(a.grad_sum.p) + r * a.grad_sum.stride + c, lane, left, there);
  }
  // The row's two sums, and this span's part of the gradients over rows.
  __device__ __forceinline__ void sums(const float w[kLanePiece], float mean, float rstd, float& sh,
                                       float& shz, float gw[kLanePiece], float gb[kLanePiece],
                                       int lane, int left) {
    float d[kLanePiece], z[kLanePiece];
    dy.settle_end(lane, left);
    s.settle_end(lane, left);
    dy.widen_to(d);
    s.widen_to(z);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) {
      z[u] = (z[u] - mean) * rstd;
      const float h = d[u] * w[u];
      sh += h;
      shz += h * z[u];
      gw[u] += d[u] * z[u];
      gb[u] += d[u];
    }
  }
  // The row's gradient from the means m1 of h and m2 of h * z, plus what
  // reaches the sum from elsewhere; stored, dropped out for grad_x.  (float32: h
  // and z are made again, registers for them cost more than the arithmetic;
  // bfloat16: z with the sums' rstd, so that the sums' z are kept.)
  __device__ __forceinline__ void finish(const float w[kLanePiece], float mean, float rstd,
                                         float z_rstd, float m1, float m2, const NormGradArgs& a, const Drop& drop,
                                         uint64_t n, int64_t r, int64_t c, int lane, int left) {
    typedef Span<T, G, ENDS> S;
    float d[kLanePiece], z[kLanePiece];
    if (sizeof(T) == 4) {
      dy.renew();
      s.renew();
      z_rstd = rstd;
    }
    dy.widen_to(d);
    s.widen_to(z);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) {
      z[u] = (z[u] - mean) * z_rstd;
      d[u] = rstd * (d[u] * w[u] - m1 - z[u] * m2);
    }
    if (a.grad_sum.p != nullptr) {
      up.settle_end(lane, left);
      up.widen_to(z);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) d[u] += z[u];
    }
    if (a.grad_residual.p != nullptr)
      S::template store<false>(static_cast<T*>(a.grad_residual.p) + r * a.grad_residual.stride + c, d,
                               lane, left);
    if (a.grad_x.p != nullptr) {
      if (drop.t)
        S::drop(d, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r), lane);
      S::template store<false>(static_cast<T*>(a.grad_x.p) + r * a.grad_x.stride + c, d, lane, left);
    }
  }
};

// A group of G lanes a row, as in norm_group_kernel; a lane keeps its columns'
// weights and gradient sums for all of its rows.
template <typename T, int G, bool ENDS, int NP>
__global__ __launch_bounds__(kRowThreads, NP == 1 ? 4 : 2) void norm_grad_group_kernel(const NormGradArgs a,
                                                                      const Drop drop,
                                                                      const SumsOut sums) {
  constexpr int kRows = kRowThreads / G, kSpan = G * kLanePiece;
  __shared__ float lds[kRowWaves][NP * kSpan];
  const int lane = threadIdx.x % G, wave = threadIdx.x >> 6;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + group_of<G>();
  GradSpan<T, G, ENDS> in[NP], next[NP];
  float w[NP][kLanePiece], gw[NP][kLanePiece], gb[NP][kLanePiece];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    in[i].load(a, r, i * kSpan, lane, cols - i * kSpan, r < a.rows);
    Span<T, G, ENDS>::weights(w[i], a.weight, a.weight_bf16, i * kSpan, lane, cols - i * kSpan, 1.f);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) gw[i][u] = gb[i][u] = 0.f;
  }
  float mean = r < a.rows ? a.mean[r] : 0.f, rstd = r < a.rows ? a.rstd[r] : 0.f;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.rows; r0 += step, r += step) {
    float next_mean = 0.f, next_rstd = 0.f;
    if (r0 + step < a.rows) {
      const bool more = r + step < a.rows;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        next[i].load(a, r + step, i * kSpan, lane, cols - i * kSpan, more);
      if (more) {
        next_mean = a.mean[r + step];
        next_rstd = a.rstd[r + step];
      }
    }
    const float z_rstd = sums_rstd(mean, rstd);
    float sh = 0.f, shz = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) in[i].sums(w[i], mean, z_rstd, sh, shz, gw[i], gb[i], lane, cols - i * kSpan);
    const float m1 = group_sum<G>(sh) * inv, m2 = group_sum<G>(shz) * inv;
    if (r < a.rows) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        in[i].finish(w[i], mean, rstd, z_rstd, m1, m2, a, drop, n, r, i * kSpan, lane, cols - i * kSpan);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) in[i] = next[i];
    mean = next_mean;
    rstd = next_rstd;
  }
  // the groups of a wavefront, then the wavefronts
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = which ? sums.bias : sums.weight;
    if (out == nullptr) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        float v = which ? gb[i][u] : gw[i][u];
#pragma unroll
        for (int m = G; m < kWave; m <<= 1) v += __shfl_xor(v, m);
        if ((threadIdx.x & (kWave - 1)) < G) lds[wave][i * kSpan + Span<T, G, ENDS>::col(lane, u)] = v;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += kRowThreads) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < kRowWaves; ++k) v += lds[k][c];
      out[static_cast<int64_t>(blockIdx.x) * 2 * cols + c] = v;
    }
  }
}

// A block a row: its wavefronts' two sums are joined through LDS with one
// barrier a row.
template <typename T, int TH, bool ENDS, int NP>
__global__ __launch_bounds__(TH) void norm_grad_block_kernel(const NormGradArgs a, const Drop drop,
                                                             const SumsOut sums) {
  __shared__ float lds[2][2][kMaxWaves];
  const int lane = threadIdx.x & (kWave - 1), wave = group_of<kWave>();
  const int waves = blockDim.x >> 6;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  int64_t r = blockIdx.x;
  GradSpan<T, kWave, ENDS> in[NP], next[NP];
  float w[NP][kLanePiece], gw[NP][kLanePiece], gb[NP][kLanePiece];
  int c[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    c[i] = (i * waves + wave) * kSpanCols;
    in[i].load(a, r, c[i], lane, cols - c[i]);
    Span<T, kWave, ENDS>::weights(w[i], a.weight, a.weight_bf16, c[i], lane, cols - c[i], 1.f);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) gw[i][u] = gb[i][u] = 0.f;
  }
  const int other = lane % kMaxWaves;
  float mean = a.mean[r], rstd = a.rstd[r];
  int turn = 0;
  for (; r < a.rows; r += gridDim.x, turn ^= 1) {
    const int64_t after = r + gridDim.x;
    const bool more = after < a.rows;
    if (more) {
#pragma unroll
      for (int i = 0; i < NP; ++i) next[i].load(a, after, c[i], lane, cols - c[i]);
    }
    const float next_mean = more ? a.mean[after] : 0.f, next_rstd = more ? a.rstd[after] : 0.f;
    const float z_rstd = sums_rstd(mean, rstd);
    float sh = 0.f, shz = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) in[i].sums(w[i], mean, z_rstd, sh, shz, gw[i], gb[i], lane, cols - c[i]);
    sh = wave_sum(sh);
    shz = wave_sum(shz);
    if (lane == 0) {
      lds[turn][0][wave] = sh;
      lds[turn][1][wave] = shz;
    }
    __syncthreads();  // the other half of lds is free again at the next row's
    const float m1 = group_sum<kMaxWaves>(other < waves ? lds[turn][0][other] : 0.f) * inv;
    const float m2 = group_sum<kMaxWaves>(other < waves ? lds[turn][1][other] : 0.f) * inv;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      in[i].finish(w[i], mean, rstd, z_rstd, m1, m2, a, drop, n, r, c[i], lane, cols - c[i]);
      in[i] = next[i];
    }
    mean = next_mean;
    rstd = next_rstd;
  }
  const int64_t mine = static_cast<int64_t>(blockIdx.x) * 2 * cols;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    if (sums.weight != nullptr)
      Span<T, kWave, ENDS>::template store<false>(sums.weight + mine + c[i], gw[i], lane, cols - c[i]);
    if (sums.bias != nullptr)
      Span<T, kWave, ENDS>::template store<false>(sums.bias + mine + c[i], gb[i], lane, cols - c[i]);
  }
}

// Wider rows, which are read twice (2048 x 16384 float32 without residual: 123 us, 3.3
// TB/s of the three arrays).  First the rows' two means (m1 and m2, [2][rows] of
// scratch) ...
template <typename T, bool ENDS>
__global__ __launch_bounds__(kRowThreads) void norm_grad_means_kernel(const NormGradArgs a,
                                                                      float* __restrict__ means) {
  __shared__ float lds[2 * kRowWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t begin = group_of<kWave>() * kSpanCols, step = kRowWaves * kSpanCols;
  const float inv = 1.f / static_cast<float>(a.cols);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float mean = a.mean[r], rstd = sums_rstd(mean, a.rstd[r]);
    float sh = 0.f, shz = 0.f;
    for (int64_t c = begin; c < a.cols; c += step) {
      const int left = cols_left(c, a.cols);
      Span<T, kWave, ENDS> g, s;
      float dy[kLanePiece], z[kLanePiece], w[kLanePiece];
      g.load(static_cast<const T*>(a.grad.p) + r * a.grad.stride + c, lane, left);
      s.load(static_cast<const T*>(a.s.p) + r * a.s.stride + c, lane, left);
      Span<T, kWave, ENDS>::weights(w, a.weight, a.weight_bf16, c, lane, left, 1.f);
      g.settle_end(lane, left);
      s.settle_end(lane, left);
      g.widen_to(dy);
      s.widen_to(z);
      float ph = 0.f, phz = 0.f;
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const float h = dy[u] * w[u];
        ph += h;
        phz += h * ((z[u] - mean) * rstd);
      }
      sh += ph;
      shz += phz;
    }
    block_sum2(sh, shz, lds);
    if (threadIdx.x == 0) {
      means[r] = sh * inv;
      means[a.rows + r] = shz * inv;
    }
  }
}
// ... then tiles of columns, a wavefront a span of them: block y takes rows y, y +
// gridDim.y, ... and keeps its columns' gradient sums in registers.
template <typename T, bool ENDS>
__global__ __launch_bounds__(kRowThreads) void norm_grad_tile_kernel(
    const NormGradArgs a, const Drop drop, const float* __restrict__ means, const SumsOut sums) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * kRowWaves + group_of<kWave>()) * kSpanCols;
  if (c >= a.cols) return;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int left = cols_left(c, a.cols);
  float w[kLanePiece], gw[kLanePiece], gb[kLanePiece];
  Span<T, kWave, ENDS>::weights(w, a.weight, a.weight_bf16, c, lane, left, 1.f);
#pragma unroll
  for (int u = 0; u < kLanePiece; ++u) gw[u] = gb[u] = 0.f;
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    GradSpan<T, kWave, ENDS> in;
    in.load(a, r, c, lane, left);
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sh = 0.f, shz = 0.f;
    in.sums(w, mean, rstd, sh, shz, gw, gb, lane, left);
    in.finish(w, mean, rstd, rstd, means[r], means[a.rows + r], a, drop, n, r, c, lane, left);
  }
  const int64_t mine = static_cast<int64_t>(blockIdx.y) * 2 * a.cols + c;
  if (sums.weight != nullptr)
    Span<T, kWave, ENDS>::template store<false>(sums.weight + mine, gw, lane, left);
  if (sums.bias != nullptr)
    Span<T, kWave, ENDS>::template store<false>(sums.bias + mine, gb, lane, left);
}

// Sums the blocks' parts: COLS columns a block, 1024 / COLS threads to each, which
// request 8 parts at a time and add them in order; joined in two steps.
constexpr int kSumThreads = 1024, kSumAhead = 8;
constexpr int kWideSums = 2048;  // columns from which on a block takes 32 of them, else 16
template <int COLS>
__global__ __launch_bounds__(kSumThreads) void sum_parts_kernel(const float* __restrict__ part,
                                                                const int parts, const int64_t cols,
                                                                float* __restrict__ weight,
                                                                float* __restrict__ bias) {
  constexpr int kGroups = kSumThreads / COLS, kJoin = 8;
  __shared__ float lds[kGroups][COLS + 1], joined[kJoin][COLS + 1];
  const int x = threadIdx.x % COLS, y = threadIdx.x / COLS;
  const int64_t step = static_cast<int64_t>(gridDim.x) * COLS;
  for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * COLS; i0 < 2 * cols; i0 += step) {
    const int64_t i = i0 + x;
    float v = 0.f;
    if (i < 2 * cols) {
      for (int k = y; k < parts; k += kGroups * kSumAhead) {
        float t[kSumAhead];
#pragma unroll
        for (int m = 0; m < kSumAhead; ++m) {
          const int at = k + m * kGroups;
          t[m] = at < parts ? part[at * 2 * cols + i] : 0.f;
        }
#pragma unroll
        for (int m = 0; m < kSumAhead; ++m) v += t[m];
      }
    }
    lds[y][x] = v;
    __syncthreads();
    if (y < kJoin) {
      v = 0.f;
#pragma unroll
      for (int k = 0; k < kGroups / kJoin; ++k) v += lds[y * (kGroups / kJoin) + k][x];
      joined[y][x] = v;
    }
    __syncthreads();
    float* out = i < cols ? weight : bias;
    if (y == 0 && i < 2 * cols && out != nullptr) {
      v = 0.f;
#pragma unroll
      for (int k = 0; k < kJoin; ++k) v += joined[k][x];
      out[i < cols ? i : i - cols] = v;
    }
  }
}

// One span a lane takes up to 128 registers, two bfloat16 ones up to 170: blocks of
// two are for rows that one span does not cover (4000 x 9000 bfloat16 without
// residual: 56 us, the wide form 91; float32 they would spill, 217 against 208 with
// residual and dropout).  Five wavefronts a block leave a SIMD without its share: 6
// (16000 x 2500 bfloat16 without residual: 69 against 86 us).
constexpr int kGradWaves2 = 12;
static RowForm grad_form(bool bf16, int64_t cols) {
  const int64_t n = (cols + kLanePiece - 1) / kLanePiece;
  if (n <= kWave) return {row_lanes(cols), 1, kHeld};
  if (n <= 2 * kWave) return {kWave, 2, kHeld / 2};
  const int64_t w = (n + kWave - 1) / kWave, w1 = w > 3 ? (w + 1) / 2 * 2 : w;
  if (w1 <= kMaxWaves) return {static_cast<int>(w1) * kWave, 1, kHeld};
  const int64_t w2 = (n + 2 * kWave - 1) / (2 * kWave);
  if (bf16 && w2 <= kGradWaves2) return {static_cast<int>(w2) * kWave, 2, kGradWaves2};
  return {kRowThreads, 0, kRowWaves};
}

// Parts: blocks that walk rows (one alone, which saves the sum's launch, for up to
// kAlone rows to a group of lanes: 4 x 4096 bfloat16 8.5 against 11.2 us a call; 8 rows
// to it take 13.9 against 11.3); of the wide form, the blocks that share a tile of
// columns (8 blocks to a CU over all tiles).
constexpr int kAlone = 4;
static int norm_grad_parts(bool bf16, int64_t rows, int64_t cols) {
  const RowForm f = grad_form(bf16, cols);
  if (f.spans != 0) {
    const int64_t together = f.lanes <= kWave ? kRowThreads / f.lanes : 1;
    return rows <= kAlone * together ? 1 : static_cast<int>(row_blocks(f, rows));
  }
  const int64_t tiles = (cols + kRowWaves * kSpanCols - 1) / (kRowWaves * kSpanCols);
  const int64_t want = tiles < 2048 ? 2048 / tiles : 1;
  return static_cast<int>(rows < want ? rows : want);
}

size_t norm_grad_workspace_bytes(bool bf16, int64_t rows, int64_t cols, bool sums) {
  const int parts = norm_grad_parts(bf16, rows, cols);
  const size_t part = sums && parts > 1 ? static_cast<size_t>(parts) * 2 * cols : 0;
  return (part + (grad_form(bf16, cols).spans == 0 ? 2 * static_cast<size_t>(rows) : 0)) *
         sizeof(float);
}

template <typename T, bool ENDS>
static hipError_t launch_norm_grad_t(const NormGradArgs& a, const Drop& drop, const SumsOut& sums,
                                     float* means, int parts, hipStream_t stream) {
  const RowForm f = grad_form(sizeof(T) == 2, a.cols);
  const dim3 grid(parts), block(f.lanes <= kWave ? kRowThreads : f.lanes);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, drop, sums);
    return hipGetLastError();
  };
  if (f.spans == 0) {
    const int64_t most = 2048;
    hipLaunchKernelGGL((norm_grad_means_kernel<T, ENDS>),
                       dim3(static_cast<uint32_t>(a.rows < most ? a.rows : most)), block, 0, stream,
                       a, means);
    const int64_t tiles = (a.cols + kRowWaves * kSpanCols - 1) / (kRowWaves * kSpanCols);
    hipLaunchKernelGGL((norm_grad_tile_kernel<T, ENDS>), dim3(static_cast<uint32_t>(tiles), parts), block, 0,
                       stream, a, drop, means, sums);
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 2) {
    if (f.lanes > kWave && f.spans == 2)
      return launch(norm_grad_block_kernel<T, kGradWaves2 * kWave, ENDS, 2>);
  }
  if (f.lanes > kWave) return launch(norm_grad_block_kernel<T, 1024, ENDS, 1>);
  if (f.spans == 2) return launch(norm_grad_group_kernel<T, kWave, ENDS, 2>);
  return with_const<1, 2, 4, 8, 16, 32, 64>(f.lanes, [&](auto lanes) {
    return launch(norm_grad_group_kernel<T, lanes.value, ENDS, 1>);
  });
}

hipError_t launch_norm_grad(bool bf16, const NormGradArgs& a, const Drop& drop, void* workspace,
                            hipStream_t stream) {
  const int parts = norm_grad_parts(bf16, a.rows, a.cols);
  float* part = static_cast<float*>(workspace);
  float* means = part;
  SumsOut sums = {a.grad_weight, a.grad_bias};
  const bool join = parts > 1 && (a.grad_weight != nullptr || a.grad_bias != nullptr);
  if (join) {
    sums = {part, part + a.cols};
    means = part + static_cast<size_t>(parts) * 2 * a.cols;
  }
  hipError_t e = by_row_type(bf16, a.cols, [&](auto t, auto ends) {
    return launch_norm_grad_t<decltype(t), ends.value>(a, drop, sums, means, parts, stream);
  });
  if (e == hipSuccess && join) {
    // whole lines of columns where they leave enough blocks (16384 x 2048 bfloat16
    // without residual: 43.0 against 45.5 us for the call; 3000 x 1000: 12.2 against
    // 11.9)
    e = with_const<16, 32>(a.cols >= kWideSums ? 32 : 16, [&](auto wide) {
      constexpr int COLS = wide.value;
      const int64_t blocks = (2 * a.cols + COLS - 1) / COLS;
      hipLaunchKernelGGL(sum_parts_kernel<COLS>,
                         dim3(static_cast<uint32_t>(blocks < kGridBlocks ? blocks : kGridBlocks - 1)),
                         dim3(kSumThreads), 0, stream, part, parts, a.cols, a.grad_weight,
                         a.grad_bias);
      return hipGetLastError();
    });
  }
  return e;
}

}  // namespace pss
