// Learned relative position bias by buckets: scores + table[bucket], and the
// table's gradient.
#include "pss_rows.hpp"

namespace pss {

constexpr int kBiasThreads = 256;
constexpr int kBiasWaves = kBiasThreads / kWave;
constexpr int kMaxStart = 1 << 29;  // of q_starts

// Position of query 0 of batch b.
__device__ __forceinline__ int32_t first_position(const BiasArgs& a, int64_t b) {
  int32_t s = a.q_starts != nullptr ? a.q_starts[b] : 0;
  s = s < 0 ? 0 : (s > kMaxStart ? kMaxStart : s);
  return static_cast<int32_t>(a.q_start) + s;
}

template <typename T>
__global__ __launch_bounds__(kBiasThreads) void bias_kernel(const BiasArgs a, const BucketMap map) {
  __shared__ int32_t borders[kMaxBuckets];
  for (int i = threadIdx.x; i < map.side; i += kBiasThreads) borders[i] = map.borders[i];
  __syncthreads();
  const int64_t all = a.B * a.H * a.Q * a.K;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kBiasThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBiasThreads + threadIdx.x; i < all; i += step) {
    const int64_t row = i / a.K, k = i - row * a.K;
    const int64_t bh = row / a.Q, q = row - bh * a.Q;
    const int64_t b = bh / a.H, h = bh - b * a.H;
    const int32_t rel = static_cast<int32_t>(k) - first_position(a, b) - static_cast<int32_t>(q);
    const int j = bucket_of(rel, borders, map.side, map.both);
    float v = a.table_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.table)[j * a.H + h])
                           : static_cast<const float*>(a.table)[j * a.H + h];
    if (a.in != nullptr) {
      float x[kLanePiece];
      load8(x, static_cast<const T*>(a.in) + b * a.in_stride[0] + h * a.in_stride[1] +
                   q * a.in_stride[2] + k, 1);
      v += x[0];
    }
    float y[kLanePiece] = {v};
    store8(static_cast<T*>(a.out) + b * a.out_stride[0] + h * a.out_stride[1] + q * a.out_stride[2] +
               k, y, 1);
  }
}

hipError_t launch_bias(bool bf16, const BiasArgs& a, const BucketMap& map, hipStream_t stream) {
  const int64_t want = (a.B * a.H * a.Q * a.K + kBiasThreads - 1) / kBiasThreads;
  const dim3 grid(static_cast<uint32_t>(want < 8192 ? want : 8192)), block(kBiasThreads);
  if (bf16)
    hipLaunchKernelGGL(bias_kernel<uint16_t>, grid, block, 0, stream, a, map);
  else
    hipLaunchKernelGGL(bias_kernel<float>, grid, block, 0, stream, a, map);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The table's gradient.  All pairs at one distance share a bucket, so a block
// first sums along diagonals: a lane owns 8 neighbouring values of
// key - query and walks the queries of its tile, reading the 8 elements of
// each row that lie at them.  Then every bucket, a range of distances,
// sums its diagonals.  Every sum has a fixed order.
// ---------------------------------------------------------------------------
constexpr int kDiagonals = kBiasThreads * kLanePiece;  // of one block
constexpr int kGradRows = 64;                      // queries of one block

struct GradShape {
  int64_t tiles;   // query tiles of one (b, h)
  int64_t chunks;  // windows of kDiagonals diagonals of one tile
};
static GradShape grad_shape(const BiasArgs& a) {
  const int64_t rows = a.Q < kGradRows ? a.Q : kGradRows;
  return {(a.Q + kGradRows - 1) / kGradRows, (a.K + rows - 1 + kDiagonals - 1) / kDiagonals};
}

// Values lo .. hi of key - query that bucket j holds (hi < lo: none).
__device__ __forceinline__ void bucket_range(int j, const BucketMap& map, int64_t* lo, int64_t* hi) {
  const bool ahead = map.both && j >= map.side;
  const int i = ahead ? j - map.side : j;
  const int64_t n0 = map.borders[i];
  const int64_t n1 = i + 1 < map.side ? map.borders[i + 1] : (int64_t{1} << 40);
  if (ahead) {
    *lo = n0 < 1 ? 1 : n0;
    *hi = n1 - 1;
  } else {
    *lo = 1 - n1;
    // keys ahead of the query count as distance 0 on a single side
    *hi = !map.both && n0 == 0 && n1 > 0 ? (int64_t{1} << 40) : -n0;
  }
}

template <typename T>
__global__ __launch_bounds__(kBiasThreads) void bias_grad_kernel(const BiasArgs a,
                                                                 const BucketMap map,
                                                                 const int64_t tiles,
                                                                 const int64_t chunks,
                                                                 float* __restrict__ part) {
  __shared__ float diag[kDiagonals];
  const int64_t blk = blockIdx.x;
  const int64_t chunk = blk % chunks, tile = blk / chunks % tiles, bh = blk / (chunks * tiles);
  const int64_t b = bh / a.H, h = bh - b * a.H;
  const int64_t q0 = tile * kGradRows, q1 = q0 + kGradRows < a.Q ? q0 + kGradRows : a.Q;
  // first diagonal of the window: key 0 of the tile's last query
  const int64_t base = -(q1 - 1) + chunk * kDiagonals;  // key index - query index
  const int64_t mine = base + threadIdx.x * kLanePiece;
  const T* g = static_cast<const T*>(a.in) + b * a.in_stride[0] + h * a.in_stride[1];
  float sum[kLanePiece] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t q = q0; q < q1; ++q) {
    const int64_t k = q + mine;
    const T* p = g + q * a.in_stride[2] + k;
    if (k >= 0 && k + kLanePiece <= a.K) {
      float v[kLanePiece];
      load8(v, p, kLanePiece);
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u) sum[u] += v[u];
    } else {
#pragma unroll
      for (int u = 0; u < kLanePiece; ++u)
        if (k + u >= 0 && k + u < a.K) {
          float v[kLanePiece];
          load8(v, p + u, 1);
          sum[u] += v[0];
        }
    }
  }
#pragma unroll
  for (int u = 0; u < kLanePiece; ++u) diag[threadIdx.x * kLanePiece + u] = sum[u];
  __syncthreads();
  // positions: key - query = index difference - first position
  const int64_t rel0 = base - first_position(a, b);
  const int lane = threadIdx.x & (kWave - 1);
  for (int j = threadIdx.x >> 6; j < map.num; j += kBiasWaves) {
    int64_t lo, hi;
    bucket_range(j, map, &lo, &hi);
    lo = lo - rel0 < 0 ? 0 : lo - rel0;
    hi = hi - rel0 >= kDiagonals ? kDiagonals - 1 : hi - rel0;
    float v = 0.f;
    for (int64_t i = lo + lane; i <= hi; i += kWave) v += diag[i];
    v = wave_sum(v);
    // [head][batch, tile, window][bucket]
    if (lane == 0)
      part[((h * a.B + b) * tiles * chunks + tile * chunks + chunk) * map.num + j] = v;
  }
}

__global__ __launch_bounds__(kBiasThreads) void bias_sum_kernel(const float* __restrict__ part,
                                                                const int64_t parts, const int num,
                                                                const int64_t heads,
                                                                float* __restrict__ out) {
  __shared__ float lds[kBiasWaves];
  const int64_t h = blockIdx.x / num;
  const int j = static_cast<int>(blockIdx.x % num);
  float v = 0.f;
  for (int64_t i = threadIdx.x; i < parts; i += kBiasThreads) v += part[(h * parts + i) * num + j];
  v = wave_sum(v);
  if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = 0.f;
    for (int w = 0; w < kBiasWaves; ++w) v += lds[w];
    out[j * heads + h] = v;
  }
}

bool bias_grad_fits(const BiasArgs& a, const BucketMap& map) {
  const GradShape s = grad_shape(a);
  return a.H * map.num <= INT32_MAX && a.B * a.H <= INT32_MAX / s.tiles / s.chunks;
}

size_t bias_grad_workspace_bytes(const BiasArgs& a, const BucketMap& map) {
  const GradShape s = grad_shape(a);
  return static_cast<size_t>(a.B * a.H * s.tiles * s.chunks) * map.num * sizeof(float);
}

hipError_t launch_bias_grad(bool bf16, const BiasArgs& a, const BucketMap& map, void* workspace,
                            float* grad_table, hipStream_t stream) {
  const GradShape s = grad_shape(a);
  const int64_t blocks = a.B * a.H * s.tiles * s.chunks;
  float* part = static_cast<float*>(workspace);
  const dim3 grid(static_cast<uint32_t>(blocks)), block(kBiasThreads);
  if (bf16)
    hipLaunchKernelGGL(bias_grad_kernel<uint16_t>, grid, block, 0, stream, a, map, s.tiles, s.chunks,
                       part);
  else
    hipLaunchKernelGGL(bias_grad_kernel<float>, grid, block, 0, stream, a, map, s.tiles, s.chunks,
                       part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(bias_sum_kernel, dim3(static_cast<uint32_t>(a.H * map.num)), block, 0, stream,
                     part, a.B * s.tiles * s.chunks, map.num, a.H, grad_table);
  return hipGetLastError();
}

}  // namespace pss
