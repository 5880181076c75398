// Operators on rows: dropout from a counter-based generator, layer norm and
// its backward pass.
#include "pss_rows.hpp"

namespace pss {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kNormBlocks = 256 * 8;  // blocks that walk rows: 8 to a CU

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

// Columns from c on, as an int (a span has at most 512).
__device__ __forceinline__ int cols_left(int64_t c, int64_t cols) {
  return cols - c > INT32_MAX ? INT32_MAX : static_cast<int>(cols - c);
}

// Lanes to a row: as many as its pieces of 8, up to a wavefront.
static int row_lanes(int64_t cols) {
  const int64_t pieces = (cols + kLanePiece - 1) / kLanePiece;
  int g = 1;
  while (g < pieces && g < kWave) g *= 2;
  return g;
}

// ---------------------------------------------------------------------------
// out = residual + D(x): a span of a row to a group of G lanes.
// ---------------------------------------------------------------------------
template <typename T, int G>
__global__ __launch_bounds__(kRowThreads) void dropout_kernel(const RowsIn x, const RowsIn residual,
                                                              const RowsOut out, const int64_t rows,
                                                              const int64_t cols,
                                                              const uint32_t spans, const Drop drop,
                                                              const bool stream) {
  typedef Span<T, G> S;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const uint32_t tile = blockIdx.x / spans, span = blockIdx.x - tile * spans;
  const int lane = threadIdx.x % G;
  const int64_t r = static_cast<int64_t>(tile) * (kRowThreads / G) + threadIdx.x / G;
  const int64_t c = static_cast<int64_t>(span) * (G * kLanePiece);
  if (r >= rows) return;
  const int left = cols_left(c, cols);
  S a, b;
  a.load(static_cast<const T*>(x.p) + r * x.stride + c, lane, left);
  if (residual.p != nullptr)
    b.load(static_cast<const T*>(residual.p) + r * residual.stride + c, lane, left);
  float v[kLanePiece];
  a.widen_to(v);
  if (drop.t) S::drop(v, drop, n, span * G, static_cast<uint32_t>(r), lane);
  if (residual.p != nullptr) {
    float q[kLanePiece];
    b.widen_to(q);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] += q[u];
  }
  S::store(static_cast<T*>(out.p) + r * out.stride + c, v, lane, left, stream);
}

// Results of more than this are stored past the caches.
constexpr int64_t kStreamBytes = int64_t{32} << 20;
static bool streams(bool bf16, int64_t rows, int64_t cols) {
  return rows * cols * (bf16 ? 2 : 4) > kStreamBytes;
}

template <typename T>
static hipError_t launch_dropout_t(const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                                   int64_t rows, int64_t cols, const Drop& drop,
                                   hipStream_t stream) {
  const int g = row_lanes(cols);
  const int64_t spans = (cols + g * kLanePiece - 1) / (g * kLanePiece);
  const int64_t tiles = (rows * g + kRowThreads - 1) / kRowThreads;
  if (tiles > INT32_MAX / spans) return hipErrorInvalidConfiguration;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(tiles * spans)), dim3(kRowThreads), 0,
                       stream, x, residual, out, rows, cols, static_cast<uint32_t>(spans), drop,
                       streams(sizeof(T) == 2, rows, cols));
    return hipGetLastError();
  };
  switch (g) {
    case 1: return launch(dropout_kernel<T, 1>);
    case 2: return launch(dropout_kernel<T, 2>);
    case 4: return launch(dropout_kernel<T, 4>);
    case 8: return launch(dropout_kernel<T, 8>);
    case 16: return launch(dropout_kernel<T, 16>);
    case 32: return launch(dropout_kernel<T, 32>);
    default: return launch(dropout_kernel<T, 64>);
  }
}

hipError_t launch_dropout(bool bf16, const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                          int64_t rows, int64_t cols, const Drop& drop, hipStream_t stream) {
  return bf16 ? launch_dropout_t<uint16_t>(x, residual, out, rows, cols, drop, stream)
              : launch_dropout_t<float>(x, residual, out, rows, cols, drop, stream);
}

// ---------------------------------------------------------------------------
// Layer norm.
// ---------------------------------------------------------------------------

// s of one span: residual + D(x).
template <typename T, int G>
__device__ __forceinline__ void norm_input(float v[kLanePiece], const NormArgs& a, const Drop& drop,
                                           uint64_t n, int64_t r, int64_t c, int lane, int left) {
  Span<T, G> x, q;
  x.load(static_cast<const T*>(a.x.p) + r * a.x.stride + c, lane, left);
  if (a.residual.p != nullptr)
    q.load(static_cast<const T*>(a.residual.p) + r * a.residual.stride + c, lane, left);
  x.widen_to(v);
  if (drop.t)
    Span<T, G>::drop(v, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r),
                     lane);
  if (a.residual.p != nullptr) {
    float w[kLanePiece];
    q.widen_to(w);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] += w[u];
  }
}

template <typename T, int G>
__device__ __forceinline__ void norm_store(float v[kLanePiece], const NormArgs& a, int64_t r,
                                           int64_t c, int lane, int left, float mean, float rstd,
                                           const float w[kLanePiece], const float b[kLanePiece]) {
  typedef Span<T, G> S;
  if (a.sum.p != nullptr)
    S::store(static_cast<T*>(a.sum.p) + r * a.sum.stride + c, v, lane, left, a.stream);
#pragma unroll
  for (int u = 0; u < kLanePiece; ++u) v[u] = (v[u] - mean) * rstd * w[u] + b[u];
  S::store(static_cast<T*>(a.out.p) + r * a.out.stride + c, v, lane, left, a.stream);
}

__device__ __forceinline__ void norm_store_stats(const NormArgs& a, int64_t r, float mean, float rstd) {
  if (a.mean != nullptr) a.mean[r] = mean;
  if (a.rstd != nullptr) a.rstd[r] = rstd;
}

// Rows of any width: a block a row, which it reads three times (sum, squares
// about the mean, result).  Nothing is stored before the last pass, where
// every element is read by the lane that then stores its results.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void norm_wide_kernel(const NormArgs a, const Drop drop) {
  constexpr int kSpan = kWave * kLanePiece;
  __shared__ float lds[2 * kRowWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t first = (threadIdx.x >> 6) * kSpan, step = kRowWaves * kSpan;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const float inv = 1.f / static_cast<float>(a.cols);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float sum = 0.f, zero = 0.f;
    for (int64_t c = first; c < a.cols; c += step) {
      float v[kLanePiece];
      norm_input<T, kWave>(v, a, drop, n, r, c, lane, cols_left(c, a.cols));
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum += v[u];
    }
    block_sum2(sum, zero, lds);
    const float mean = sum * inv;
    float sq = 0.f;
    for (int64_t c = first; c < a.cols; c += step) {
      float v[kLanePiece];
      const int left = cols_left(c, a.cols);
      norm_input<T, kWave>(v, a, drop, n, r, c, lane, left);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const float e = Span<T, kWave>::col(lane, u) < left ? v[u] - mean : 0.f;
        sq += e * e;
      }
    }
    block_sum2(sq, zero, lds);
    const float rstd = 1.f / sqrtf(sq * inv + a.eps);
    if (threadIdx.x == 0) norm_store_stats(a, r, mean, rstd);
    for (int64_t c = first; c < a.cols; c += step) {
      float v[kLanePiece], w[kLanePiece], b[kLanePiece];
      const int left = cols_left(c, a.cols);
      norm_input<T, kWave>(v, a, drop, n, r, c, lane, left);
      Span<T, kWave>::weights(w, a.weight, a.weight_bf16, c, lane, left, 1.f);
      Span<T, kWave>::weights(b, a.bias, a.weight_bf16, c, lane, left, 0.f);
      norm_store<T, kWave>(v, a, r, c, lane, left, mean, rstd, w, b);
    }
  }
}

// Rows whose elements stay in registers, by groups of G lanes of a wavefront
// (G * NP pieces cover a row): read once, mean and squares about it from the
// registers.  A group walks its rows with its weights in registers.
template <typename T, int G, int NP>
__global__ __launch_bounds__(kRowThreads) void norm_group_kernel(const NormArgs a, const Drop drop) {
  constexpr int kRows = kRowThreads / G, kSpan = G * kLanePiece;
  const int lane = threadIdx.x % G;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  float w[NP][kLanePiece], b[NP][kLanePiece];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    Span<T, G>::weights(w[i], a.weight, a.weight_bf16, i * kSpan, lane, cols - i * kSpan, 1.f);
    Span<T, G>::weights(b[i], a.bias, a.weight_bf16, i * kSpan, lane, cols - i * kSpan, 0.f);
  }
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.rows;
       r0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t r = r0 + threadIdx.x / G;
    const bool mine = r < a.rows;
    float v[NP][kLanePiece], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      norm_input<T, G>(v[i], a, drop, n, r, i * kSpan, lane, mine ? cols - i * kSpan : 0);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum += v[i][u];
    }
    const float mean = group_sum<G>(sum) * inv;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const float e = i * kSpan + Span<T, G>::col(lane, u) < cols ? v[i][u] - mean : 0.f;
        sq += e * e;
      }
    const float rstd = 1.f / sqrtf(group_sum<G>(sq) * inv + a.eps);
    if (!mine) continue;
    if (lane == 0) norm_store_stats(a, r, mean, rstd);
#pragma unroll
    for (int i = 0; i < NP; ++i)
      norm_store<T, G>(v[i], a, r, i * kSpan, lane, cols - i * kSpan, mean, rstd, w[i], b[i]);
  }
}

// The same by a whole block a row.  Every wavefront takes mean and squares of
// its own part; the parts are joined through LDS with one barrier a row (the
// squares about the common mean are those about each part's plus the part's
// size times the square of its mean's distance).
template <typename T, int TH, int NP>
__global__ __launch_bounds__(TH) void norm_block_kernel(const NormArgs a, const Drop drop) {
  constexpr int kWaves = TH / kWave, kSpan = kWave * kLanePiece;
  __shared__ float lds[2][2 * kWaves];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  float w[NP][kLanePiece], b[NP][kLanePiece];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * kWaves + wave) * kSpan;
    Span<T, kWave>::weights(w[i], a.weight, a.weight_bf16, c, lane, cols - c, 1.f);
    Span<T, kWave>::weights(b[i], a.bias, a.weight_bf16, c, lane, cols - c, 0.f);
  }
  // elements of wavefront k's part
  const auto size = [&](int k) {
    int e = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int left = cols - (i * kWaves + k) * kSpan;
      e += left < 0 ? 0 : (left > kSpan ? kSpan : left);
    }
    return static_cast<float>(e);
  };
  const float inv_part = size(wave) > 0.f ? 1.f / size(wave) : 0.f;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    float v[NP][kLanePiece], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * kWaves + wave) * kSpan;
      norm_input<T, kWave>(v[i], a, drop, n, r, c, lane, cols - c);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum += v[i][u];
    }
    const float part = wave_sum(sum) * inv_part;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const int c = (i * kWaves + wave) * kSpan + Span<T, kWave>::col(lane, u);
        const float e = c < cols ? v[i][u] - part : 0.f;
        sq += e * e;
      }
    sq = wave_sum(sq);
    if (lane == 0) {
      lds[turn][wave] = part;
      lds[turn][kWaves + wave] = sq;
    }
    __syncthreads();  // the other half of lds is free again at the next row's
    float mean = 0.f, var = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) mean += size(k) * lds[turn][k];
    mean *= inv;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float away = lds[turn][k] - mean;
      var += lds[turn][kWaves + k] + size(k) * (away * away);
    }
    const float rstd = 1.f / sqrtf(var * inv + a.eps);
    if (threadIdx.x == 0) norm_store_stats(a, r, mean, rstd);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * kWaves + wave) * kSpan;
      norm_store<T, kWave>(v[i], a, r, c, lane, cols - c, mean, rstd, w[i], b[i]);
    }
  }
}

static uint32_t row_grid(int64_t rows, int per_block, int most) {
  const int64_t want = (rows + per_block - 1) / per_block;
  return static_cast<uint32_t>(want < most ? want : most);
}

template <typename T, int G, int NP>
static hipError_t launch_norm_group(const NormArgs& a, const Drop& drop, hipStream_t stream) {
  hipLaunchKernelGGL((norm_group_kernel<T, G, NP>),
                     dim3(row_grid(a.rows, kRowThreads / G, kNormBlocks)), dim3(kRowThreads), 0,
                     stream, a, drop);
  return hipGetLastError();
}
template <typename T, int TH, int NP>
static hipError_t launch_norm_block(const NormArgs& a, const Drop& drop, hipStream_t stream) {
  hipLaunchKernelGGL((norm_block_kernel<T, TH, NP>),
                     dim3(row_grid(a.rows, 1, kNormBlocks * kRowThreads / TH)), dim3(TH), 0, stream,
                     a, drop);
  return hipGetLastError();
}

template <typename T>
static hipError_t launch_norm_t(const NormArgs& a, const Drop& drop, hipStream_t stream) {
  const int64_t pieces = (a.cols + kLanePiece - 1) / kLanePiece;
  if (pieces <= 1) return launch_norm_group<T, 1, 1>(a, drop, stream);
  if (pieces <= 2) return launch_norm_group<T, 2, 1>(a, drop, stream);
  if (pieces <= 4) return launch_norm_group<T, 4, 1>(a, drop, stream);
  if (pieces <= 8) return launch_norm_group<T, 8, 1>(a, drop, stream);
  if (pieces <= 16) return launch_norm_group<T, 16, 1>(a, drop, stream);
  if (pieces <= 32) return launch_norm_group<T, 32, 1>(a, drop, stream);
  if (pieces <= 64) return launch_norm_group<T, 64, 1>(a, drop, stream);
  if (pieces <= 128) return launch_norm_group<T, 64, 2>(a, drop, stream);
  if (pieces <= 256) return launch_norm_block<T, 256, 1>(a, drop, stream);
  if (pieces <= 512) return launch_norm_block<T, 256, 2>(a, drop, stream);
  if (pieces <= 1024) return launch_norm_block<T, 512, 2>(a, drop, stream);
  if (pieces <= 2048) return launch_norm_block<T, 1024, 2>(a, drop, stream);
  hipLaunchKernelGGL(norm_wide_kernel<T>, dim3(row_grid(a.rows, 1, kNormBlocks)), dim3(kRowThreads), 0,
                     stream, a, drop);
  return hipGetLastError();
}

hipError_t launch_norm(bool bf16, const NormArgs& args, const Drop& drop, hipStream_t stream) {
  NormArgs a = args;
  a.stream = streams(bf16, a.rows, a.cols);
  return bf16 ? launch_norm_t<uint16_t>(a, drop, stream) : launch_norm_t<float>(a, drop, stream);
}

// ---------------------------------------------------------------------------
// Backward.  Each block adds what its rows give to the weight's and bias's
// gradients to its own row of `part` ([blocks][2][cols]), and
// sum_parts_kernel adds the blocks' rows in order.
// ---------------------------------------------------------------------------

// What a row needs of one span, all read ahead of its sums.
template <typename T, int G>
struct GradSpan {
  Span<T, G> dy, s, up;
  __device__ __forceinline__ void load(const NormGradArgs& a, int64_t r, int64_t c, int lane,
                                       int left) {
    dy.load(static_cast<const T*>(a.grad.p) + r * a.grad.stride + c, lane, left);
    s.load(static_cast<const T*>(a.s.p) + r * a.s.stride + c, lane, left);
    if (a.grad_sum.p != nullptr)
      up.load(static_cast<const T*>(a.grad_sum.p) + r * a.grad_sum.stride + c, lane, left);
  }
};

// The row's gradient d, plus what reaches the sum from elsewhere (up); stored,
// dropped out for grad_x.
template <typename T, int G>
__device__ __forceinline__ void norm_grad_store(float d[kLanePiece], const Span<T, G>& up,
                                                const NormGradArgs& a, const Drop& drop, uint64_t n,
                                                int64_t r, int64_t c, int lane, int left) {
  typedef Span<T, G> S;
  if (a.grad_sum.p != nullptr) {
    float q[kLanePiece];
    up.widen_to(q);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) d[u] += q[u];
  }
  if (a.grad_residual.p != nullptr)
    S::store(static_cast<T*>(a.grad_residual.p) + r * a.grad_residual.stride + c, d, lane, left,
             a.stream);
  if (a.grad_x.p != nullptr) {
    if (drop.t)
      S::drop(d, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r), lane);
    S::store(static_cast<T*>(a.grad_x.p) + r * a.grad_x.stride + c, d, lane, left, a.stream);
  }
}

// Narrow rows, by groups of G lanes as in norm_group_kernel: a lane keeps its
// columns' weights and gradient sums in registers for all of its rows.
template <typename T, int G, int NP>
__global__ __launch_bounds__(kRowThreads) void norm_grad_group_kernel(const NormGradArgs a,
                                                                      const Drop drop,
                                                                      float* part) {
  constexpr int kRows = kRowThreads / G, kSpan = G * kLanePiece;
  __shared__ float lds[kRowWaves][NP * kSpan];
  const int lane = threadIdx.x % G, wave = threadIdx.x >> 6;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  float w[NP][kLanePiece], gw[NP][kLanePiece], gb[NP][kLanePiece];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    Span<T, G>::weights(w[i], a.weight, a.weight_bf16, i * kSpan, lane, cols - i * kSpan, 1.f);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) gw[i][u] = gb[i][u] = 0.f;
  }
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.rows;
       r0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t r = r0 + threadIdx.x / G;
    const bool mine = r < a.rows;
    const float mean = mine ? a.mean[r] : 0.f, rstd = mine ? a.rstd[r] : 0.f;
    GradSpan<T, G> in[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) in[i].load(a, r, i * kSpan, lane, mine ? cols - i * kSpan : 0);
    float dy[NP][kLanePiece], z[NP][kLanePiece], sh = 0.f, shz = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      in[i].dy.widen_to(dy[i]);
      in[i].s.widen_to(z[i]);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        z[i][u] = (z[i][u] - mean) * rstd;
        const float h = dy[i][u] * w[i][u];
        sh += h;
        shz += h * z[i][u];
        gw[i][u] += dy[i][u] * z[i][u];
        gb[i][u] += dy[i][u];
      }
    }
    const float m1 = group_sum<G>(sh) * inv, m2 = group_sum<G>(shz) * inv;
    if (!mine) continue;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      float d[kLanePiece];
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) d[u] = rstd * (dy[i][u] * w[i][u] - m1 - z[i][u] * m2);
      norm_grad_store<T, G>(d, in[i].up, a, drop, n, r, i * kSpan, lane, cols - i * kSpan);
    }
  }
  if (part == nullptr) return;
  // the groups of a wavefront, then the wavefronts
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        float v = which ? gb[i][u] : gw[i][u];
#pragma unroll
        for (int m = G; m < kWave; m <<= 1) v += __shfl_xor(v, m);
        if ((threadIdx.x & (kWave - 1)) < G) lds[wave][i * kSpan + Span<T, G>::col(lane, u)] = v;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += kRowThreads) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < kRowWaves; ++k) v += lds[k][c];
      part[(static_cast<int64_t>(blockIdx.x) * 2 + which) * cols + c] = v;
    }
  }
}

// A block a row: its wavefronts' two sums are joined through LDS with one
// barrier a row.
template <typename T, int TH, int NP>
__global__ __launch_bounds__(TH) void norm_grad_block_kernel(const NormGradArgs a, const Drop drop,
                                                             float* part) {
  constexpr int kWaves = TH / kWave, kSpan = kWave * kLanePiece;
  __shared__ float lds[2][2 * kWaves];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const int cols = static_cast<int>(a.cols);
  const float inv = 1.f / static_cast<float>(cols);
  float w[NP][kLanePiece], gw[NP][kLanePiece], gb[NP][kLanePiece];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * kWaves + wave) * kSpan;
    Span<T, kWave>::weights(w[i], a.weight, a.weight_bf16, c, lane, cols - c, 1.f);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) gw[i][u] = gb[i][u] = 0.f;
  }
  int turn = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const float mean = a.mean[r], rstd = a.rstd[r];
    GradSpan<T, kWave> in[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * kWaves + wave) * kSpan;
      in[i].load(a, r, c, lane, cols - c);
    }
    float dy[NP][kLanePiece], z[NP][kLanePiece], sh = 0.f, shz = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      in[i].dy.widen_to(dy[i]);
      in[i].s.widen_to(z[i]);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        z[i][u] = (z[i][u] - mean) * rstd;
        const float h = dy[i][u] * w[i][u];
        sh += h;
        shz += h * z[i][u];
        gw[i][u] += dy[i][u] * z[i][u];
        gb[i][u] += dy[i][u];
      }
    }
    sh = wave_sum(sh);
    shz = wave_sum(shz);
    if (lane == 0) {
      lds[turn][wave] = sh;
      lds[turn][kWaves + wave] = shz;
    }
    __syncthreads();  // the other half of lds is free again at the next row's
    float m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      m1 += lds[turn][k];
      m2 += lds[turn][kWaves + k];
    }
    m1 *= inv;
    m2 *= inv;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = (i * kWaves + wave) * kSpan;
      float d[kLanePiece];
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) d[u] = rstd * (dy[i][u] * w[i][u] - m1 - z[i][u] * m2);
      norm_grad_store<T, kWave>(d, in[i].up, a, drop, n, r, c, lane, cols - c);
    }
  }
  if (part == nullptr) return;
  float* mine = part + static_cast<int64_t>(blockIdx.x) * 2 * cols;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = (i * kWaves + wave) * kSpan;
    Span<T, kWave>::store(mine + c, gw[i], lane, cols - c, false);
    Span<T, kWave>::store(mine + cols + c, gb[i], lane, cols - c, false);
  }
}

// Rows of any width: a block reads its row twice (sums, result) and keeps its
// gradient sums in its row of `part`, each element always by the same thread.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void norm_grad_wide_kernel(const NormGradArgs a,
                                                                     const Drop drop, float* part) {
  constexpr int kSpan = kWave * kLanePiece;
  __shared__ float lds[2 * kRowWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t begin = (threadIdx.x >> 6) * kSpan, step = kRowWaves * kSpan;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const float inv = 1.f / static_cast<float>(a.cols);
  float* pw = part + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
  float* pb = pw + a.cols;
  bool first = true;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sh = 0.f, shz = 0.f;
    for (int64_t c = begin; c < a.cols; c += step) {
      const int left = cols_left(c, a.cols);
      Span<T, kWave> g, s;
      float dy[kLanePiece], z[kLanePiece], w[kLanePiece];
      g.load(static_cast<const T*>(a.grad.p) + r * a.grad.stride + c, lane, left);
      s.load(static_cast<const T*>(a.s.p) + r * a.s.stride + c, lane, left);
      Span<T, kWave>::weights(w, a.weight, a.weight_bf16, c, lane, left, 1.f);
      g.widen_to(dy);
      s.widen_to(z);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const float h = dy[u] * w[u];
        sh += h;
        shz += h * ((z[u] - mean) * rstd);
      }
    }
    block_sum2(sh, shz, lds);
    const float m1 = sh * inv, m2 = shz * inv;
    for (int64_t c = begin; c < a.cols; c += step) {
      const int left = cols_left(c, a.cols);
      GradSpan<T, kWave> in;
      float dy[kLanePiece], z[kLanePiece], w[kLanePiece], d[kLanePiece];
      in.load(a, r, c, lane, left);
      Span<T, kWave>::weights(w, a.weight, a.weight_bf16, c, lane, left, 1.f);
      in.dy.widen_to(dy);
      in.s.widen_to(z);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        z[u] = (z[u] - mean) * rstd;
        d[u] = rstd * (dy[u] * w[u] - m1 - z[u] * m2);
      }
      norm_grad_store<T, kWave>(d, in.up, a, drop, n, r, c, lane, left);
      if (part != nullptr) {
#pragma unroll
        for (int u = 0; u < kLanePiece; ++u) {
          const int at = Span<T, kWave>::col(lane, u);
          if (at < left) {
            pw[c + at] = (first ? 0.f : pw[c + at]) + dy[u] * z[u];
            pb[c + at] = (first ? 0.f : pb[c + at]) + dy[u];
          }
        }
      }
    }
    first = false;
  }
}

// Sums the blocks' parts: 32 columns a block, 32 threads of partial sums each,
// joined in order.
constexpr int kSumCols = 32, kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void sum_parts_kernel(const float* part, const int blocks,
                                                                const int64_t cols, float* weight,
                                                                float* bias) {
  constexpr int kParts = kSumThreads / kSumCols;
  __shared__ float lds[kParts][kSumCols + 1];
  const int x = threadIdx.x % kSumCols, y = threadIdx.x / kSumCols;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kSumCols + x;
  float v = 0.f;
  if (i < 2 * cols)
    for (int k = y; k < blocks; k += kParts) v += part[k * 2 * cols + i];
  lds[y][x] = v;
  __syncthreads();
  if (y != 0 || i >= 2 * cols) return;
  float* out = i < cols ? weight : bias;
  if (out == nullptr) return;
  v = 0.f;
#pragma unroll
  for (int k = 0; k < kParts; ++k) v += lds[k][x];
  out[i < cols ? i : i - cols] = v;
}

// Form of the backward's rows and its blocks: 4 of 256 threads to a CU, fewer
// where the parts would exceed 64 MB.
struct GradForm {
  int threads;   // of a block
  int lanes;     // of a row (threads: a block a row)
  int pieces;    // of a lane; 0: the wide kernel
};
static GradForm grad_form(int64_t cols) {
  const int64_t n = (cols + kLanePiece - 1) / kLanePiece;
  if (n <= 64) {
    int g = 1;
    while (g < n) g *= 2;
    return {kRowThreads, g, 1};
  }
  if (n <= 128) return {kRowThreads, kWave, 2};
  if (n <= 256) return {256, 256, 1};
  if (n <= 512) return {256, 256, 2};
  if (n <= 1024) return {512, 512, 2};
  if (n <= 2048) return {1024, 1024, 2};
  return {kRowThreads, kRowThreads, 0};
}
static int norm_grad_blocks(int64_t rows, int64_t cols) {
  const GradForm f = grad_form(cols);
  const int per_block = f.threads / f.lanes;
  const int64_t most = (int64_t{1} << 23) / cols;
  int64_t n = (rows + per_block - 1) / per_block;
  const int64_t fill = int64_t{4} * 256 * kRowThreads / f.threads;
  n = n < fill ? n : fill;
  return static_cast<int>(n < most ? n : (most < 1 ? 1 : most));
}

size_t norm_grad_workspace_bytes(int64_t rows, int64_t cols) {
  return static_cast<size_t>(norm_grad_blocks(rows, cols)) * 2 * cols * sizeof(float);
}

template <typename T>
static void launch_norm_grad_t(const NormGradArgs& a, const Drop& drop, float* part, int blocks,
                               hipStream_t stream) {
  const GradForm f = grad_form(a.cols);
  const dim3 grid(blocks), block(f.threads);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, drop, part);
  };
  switch (f.pieces == 0 ? 0 : f.lanes * f.pieces) {
    case 1: return launch(norm_grad_group_kernel<T, 1, 1>);
    case 2: return launch(norm_grad_group_kernel<T, 2, 1>);
    case 4: return launch(norm_grad_group_kernel<T, 4, 1>);
    case 8: return launch(norm_grad_group_kernel<T, 8, 1>);
    case 16: return launch(norm_grad_group_kernel<T, 16, 1>);
    case 32: return launch(norm_grad_group_kernel<T, 32, 1>);
    case 64: return launch(norm_grad_group_kernel<T, 64, 1>);
    case 128: return launch(norm_grad_group_kernel<T, 64, 2>);
    case 256: return launch(norm_grad_block_kernel<T, 256, 1>);
    case 512: return launch(norm_grad_block_kernel<T, 256, 2>);
    case 1024: return launch(norm_grad_block_kernel<T, 512, 2>);
    case 2048: return launch(norm_grad_block_kernel<T, 1024, 2>);
    default: return launch(norm_grad_wide_kernel<T>);
  }
}

hipError_t launch_norm_grad(bool bf16, const NormGradArgs& args, const Drop& drop, void* workspace,
                            hipStream_t stream) {
  NormGradArgs a = args;
  a.stream = streams(bf16, a.rows, a.cols);
  const bool sums = a.grad_weight != nullptr || a.grad_bias != nullptr;
  const int blocks = norm_grad_blocks(a.rows, a.cols);
  float* part = sums ? static_cast<float*>(workspace) : nullptr;
  if (bf16)
    launch_norm_grad_t<uint16_t>(a, drop, part, blocks, stream);
  else
    launch_norm_grad_t<float>(a, drop, part, blocks, stream);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && sums) {
    hipLaunchKernelGGL(sum_parts_kernel,
                       dim3(static_cast<uint32_t>((2 * a.cols + kSumCols - 1) / kSumCols)),
                       dim3(kSumThreads), 0, stream, part, blocks, a.cols, a.grad_weight,
                       a.grad_bias);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace pss
