// Operators on rows: dropout from a counter-based generator, layer norm and
// its backward pass.
#include "pss_rows.hpp"

namespace pss {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / kWave;

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

__device__ __forceinline__ int piece_len(int64_t c, int64_t cols) {
  return cols - c < kLanePiece ? static_cast<int>(cols - c) : kLanePiece;
}

// ---------------------------------------------------------------------------
// out = residual + D(x): one lane, one piece.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kRowThreads) void dropout_kernel(const RowsIn x, const RowsIn residual,
                                                              const RowsOut out, const int64_t rows,
                                                              const int64_t cols, const Drop drop) {
  const int64_t pieces = (cols + kLanePiece - 1) / kLanePiece, all = rows * pieces;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRowThreads;
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x; i < all; i += step) {
    const int64_t r = i / pieces, c = (i - r * pieces) * kLanePiece;
    const int len = piece_len(c, cols);
    float v[kLanePiece];
    load8(v, static_cast<const T*>(x.p) + r * x.stride + c, len);
    if (drop.t) drop8(v, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r));
    if (residual.p != nullptr) {
      float q[kLanePiece];
      load8(q, static_cast<const T*>(residual.p) + r * residual.stride + c, len);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) v[u] += q[u];
    }
    store8(static_cast<T*>(out.p) + r * out.stride + c, v, len);
  }
}

static uint32_t piece_grid(int64_t pieces) {
  const int64_t want = (pieces + kRowThreads - 1) / kRowThreads;
  const int64_t cap = 256 * 32;
  return static_cast<uint32_t>(want < 1 ? 1 : (want > cap ? cap : want));
}

hipError_t launch_dropout(bool bf16, const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                          int64_t rows, int64_t cols, const Drop& drop, hipStream_t stream) {
  const dim3 grid(piece_grid(rows * ((cols + kLanePiece - 1) / kLanePiece))), block(kRowThreads);
  if (bf16)
    hipLaunchKernelGGL(dropout_kernel<uint16_t>, grid, block, 0, stream, x, residual, out, rows,
                       cols, drop);
  else
    hipLaunchKernelGGL(dropout_kernel<float>, grid, block, 0, stream, x, residual, out, rows, cols,
                       drop);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Layer norm.
// ---------------------------------------------------------------------------

// s of one piece: residual + D(x).
template <typename T>
__device__ __forceinline__ void norm_input8(float v[kLanePiece], const NormArgs& a, const Drop& drop,
                                            uint64_t n, int64_t r, int64_t c, int len) {
  load8(v, static_cast<const T*>(a.x.p) + r * a.x.stride + c, len);
  if (drop.t) drop8(v, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r));
  if (a.residual.p != nullptr) {
    float q[kLanePiece];
    load8(q, static_cast<const T*>(a.residual.p) + r * a.residual.stride + c, len);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] += q[u];
  }
}

// Rows of any width: a block a row, which it reads three times (sum, squares
// about the mean, result).  Nothing is stored before the last pass, where
// every element is read by the lane that then stores its results.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void norm_wide_kernel(const NormArgs a, const Drop drop) {
  __shared__ float lds[2 * kRowWaves];
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const float inv = 1.f / static_cast<float>(a.cols);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float sum = 0.f, zero = 0.f;
    for (int64_t c = threadIdx.x * kLanePiece; c < a.cols; c += kRowThreads * kLanePiece) {
      float v[kLanePiece];
      norm_input8<T>(v, a, drop, n, r, c, piece_len(c, a.cols));
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum += v[u];
    }
    block_sum2(sum, zero, lds);
    const float mean = sum * inv;
    float sq = 0.f;
    for (int64_t c = threadIdx.x * kLanePiece; c < a.cols; c += kRowThreads * kLanePiece) {
      float v[kLanePiece];
      const int len = piece_len(c, a.cols);
      norm_input8<T>(v, a, drop, n, r, c, len);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const float e = u < len ? v[u] - mean : 0.f;
        sq += e * e;
      }
    }
    block_sum2(sq, zero, lds);
    const float rstd = 1.f / sqrtf(sq * inv + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean != nullptr) a.mean[r] = mean;
      if (a.rstd != nullptr) a.rstd[r] = rstd;
    }
    for (int64_t c = threadIdx.x * kLanePiece; c < a.cols; c += kRowThreads * kLanePiece) {
      float v[kLanePiece], w[kLanePiece], b[kLanePiece];
      const int len = piece_len(c, a.cols);
      norm_input8<T>(v, a, drop, n, r, c, len);
      load_weights8(w, a.weight, a.weight_bf16, c, len, 1.f);
      load_weights8(b, a.bias, a.weight_bf16, c, len, 0.f);
      if (a.sum.p != nullptr) store8(static_cast<T*>(a.sum.p) + r * a.sum.stride + c, v, len);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) v[u] = (v[u] - mean) * rstd * w[u] + b[u];
      store8(static_cast<T*>(a.out.p) + r * a.out.stride + c, v, len);
    }
  }
}

hipError_t launch_norm(bool bf16, const NormArgs& a, const Drop& drop, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(a.rows < 8192 ? a.rows : 8192)), block(kRowThreads);
  if (bf16)
    hipLaunchKernelGGL(norm_wide_kernel<uint16_t>, grid, block, 0, stream, a, drop);
  else
    hipLaunchKernelGGL(norm_wide_kernel<float>, grid, block, 0, stream, a, drop);
  return hipGetLastError();
}

// Backward, rows of any width: block i takes rows i, i + blocks, ... and adds
// its part of the weight's and bias's gradients to its own row of `part`
// ([blocks][2][cols], each element always by the same thread); sum_parts_kernel
// then adds the blocks' parts in order.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void norm_grad_wide_kernel(const NormGradArgs a,
                                                                     const Drop drop, float* part) {
  __shared__ float lds[2 * kRowWaves];
  const uint64_t n = drop.t ? drop_offset(drop) : 0;
  const float inv = 1.f / static_cast<float>(a.cols);
  float* pw = part + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
  float* pb = pw + a.cols;
  bool first = true;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* g = static_cast<const T*>(a.grad.p) + r * a.grad.stride;
    const T* s = static_cast<const T*>(a.s.p) + r * a.s.stride;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sh = 0.f, shz = 0.f;
    for (int64_t c = threadIdx.x * kLanePiece; c < a.cols; c += kRowThreads * kLanePiece) {
      const int len = piece_len(c, a.cols);
      float dy[kLanePiece], z[kLanePiece], w[kLanePiece];
      load8(dy, g + c, len);
      load8(z, s + c, len);
      load_weights8(w, a.weight, a.weight_bf16, c, len, 1.f);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        const float h = dy[u] * w[u];
        sh += h;
        shz += h * ((z[u] - mean) * rstd);
      }
    }
    block_sum2(sh, shz, lds);
    const float m1 = sh * inv, m2 = shz * inv;
    for (int64_t c = threadIdx.x * kLanePiece; c < a.cols; c += kRowThreads * kLanePiece) {
      const int len = piece_len(c, a.cols);
      float dy[kLanePiece], z[kLanePiece], w[kLanePiece], d[kLanePiece];
      load8(dy, g + c, len);
      load8(z, s + c, len);
      load_weights8(w, a.weight, a.weight_bf16, c, len, 1.f);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) {
        z[u] = (z[u] - mean) * rstd;
        d[u] = rstd * (dy[u] * w[u] - m1 - z[u] * m2);
      }
      if (a.grad_sum.p != nullptr) {
        float q[kLanePiece];
        load8(q, static_cast<const T*>(a.grad_sum.p) + r * a.grad_sum.stride + c, len);
#pragma unroll
        for (int u = 0; u < kLanePiece; ++u) d[u] += q[u];
      }
      if (a.grad_residual.p != nullptr)
        store8(static_cast<T*>(a.grad_residual.p) + r * a.grad_residual.stride + c, d, len);
      if (a.grad_x.p != nullptr) {
        if (drop.t) drop8(d, drop, n, static_cast<uint32_t>(c / kLanePiece), static_cast<uint32_t>(r));
        store8(static_cast<T*>(a.grad_x.p) + r * a.grad_x.stride + c, d, len);
      }
      if (part != nullptr) {
#pragma unroll
        for (int u = 0; u < kLanePiece; ++u)
          if (u < len) {
            pw[c + u] = (first ? 0.f : pw[c + u]) + dy[u] * z[u];
            pb[c + u] = (first ? 0.f : pb[c + u]) + dy[u];
          }
      }
    }
    first = false;
  }
}

__global__ __launch_bounds__(kRowThreads) void sum_parts_kernel(const float* part, const int blocks,
                                                                const int64_t cols, float* weight,
                                                                float* bias) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x;
  if (i >= 2 * cols) return;
  float* out = i < cols ? weight : bias;
  if (out == nullptr) return;
  float v = 0.f;
  for (int k = 0; k < blocks; ++k) v += part[k * 2 * cols + i];
  out[i < cols ? i : i - cols] = v;
}

// Blocks of the backward: at most 2 to a CU, and at most 64 MB of parts.
static int norm_grad_blocks(int64_t rows, int64_t cols) {
  const int64_t most = (int64_t{1} << 23) / cols;
  const int64_t n = rows < 512 ? rows : 512;
  return static_cast<int>(n < most ? n : (most < 1 ? 1 : most));
}

size_t norm_grad_workspace_bytes(int64_t rows, int64_t cols) {
  return static_cast<size_t>(norm_grad_blocks(rows, cols)) * 2 * cols * sizeof(float);
}

hipError_t launch_norm_grad(bool bf16, const NormGradArgs& a, const Drop& drop, void* workspace,
                            hipStream_t stream) {
  const bool sums = a.grad_weight != nullptr || a.grad_bias != nullptr;
  const int blocks = norm_grad_blocks(a.rows, a.cols);
  float* part = sums ? static_cast<float*>(workspace) : nullptr;
  const dim3 grid(blocks), block(kRowThreads);
  if (bf16)
    hipLaunchKernelGGL(norm_grad_wide_kernel<uint16_t>, grid, block, 0, stream, a, drop, part);
  else
    hipLaunchKernelGGL(norm_grad_wide_kernel<float>, grid, block, 0, stream, a, drop, part);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && sums) {
    hipLaunchKernelGGL(sum_parts_kernel,
                       dim3(static_cast<uint32_t>((2 * a.cols + kRowThreads - 1) / kRowThreads)),
                       block, 0, stream, part, blocks, a.cols, a.grad_weight, a.grad_bias);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace pss
