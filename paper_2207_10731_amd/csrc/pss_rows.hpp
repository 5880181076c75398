// Operators on rows and the relative position bias (internal to the library):
// their launchers, rows of float32 or bfloat16 elements in pieces of 8, the
// counter-based dropout mask and the position buckets (host and device).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pss_kernels.hpp"

namespace pss {

constexpr int kLanePiece = 8;  // elements a lane takes at a time: 16 bytes of bfloat16

// A row argument: R rows of C consecutive elements, `stride` apart.  A null
// address stands for an argument that is not there.
struct RowsIn {
  const void* p = nullptr;
  int64_t stride = 0;
};
struct RowsOut {
  void* p = nullptr;
  int64_t stride = 0;
};

// The mask of one call: t of the 2^16 numbers are dropped (0: there is no
// dropout), the others scaled.
struct Drop {
  uint32_t k0 = 0, k1 = 0;
  uint64_t offset = 0;
  const uint64_t* step = nullptr;
  uint32_t t = 0;
  float scale = 1.f;
};

struct NormArgs {
  RowsIn x, residual;
  RowsOut out, sum;
  const void* weight = nullptr;
  const void* bias = nullptr;
  bool weight_bf16 = false;
  float eps = 0.f;
  float* mean = nullptr;
  float* rstd = nullptr;
  int64_t rows = 0, cols = 0;
};

struct NormGradArgs {
  RowsIn grad, s, grad_sum;
  RowsOut grad_x, grad_residual;
  const void* weight = nullptr;
  bool weight_bf16 = false;
  const float* mean = nullptr;
  const float* rstd = nullptr;
  float* grad_weight = nullptr;
  float* grad_bias = nullptr;
  int64_t rows = 0, cols = 0;
};

// Position buckets: `num` in all, one side's `side` borders.
constexpr int kMaxBuckets = 256;
struct BucketMap {
  int32_t num = 0, side = 0, both = 0;
  int32_t borders[kMaxBuckets];
};

struct BiasArgs {
  int64_t B = 0, H = 0, Q = 0, K = 0;
  int64_t q_start = 0;
  const int32_t* q_starts = nullptr;
  const void* in = nullptr;  // scores, or the gradient of out
  int64_t in_stride[3] = {0, 0, 0};
  void* out = nullptr;
  int64_t out_stride[3] = {0, 0, 0};
  const void* table = nullptr;
  bool table_bf16 = false;
};

// Bucket of a key `rel` positions ahead of its query (rel <= 0: behind it).
PSS_HD int bucket_of(int64_t rel, const int32_t* borders, int side, bool both) {
  const bool ahead = both && rel > 0;
  const int64_t n = rel < 0 ? -rel : (both ? rel : 0);
  int lo = 0, hi = side - 1;  // the largest j with borders[j] <= n (borders[0] = 0)
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (borders[mid] <= n) lo = mid; else hi = mid - 1;
  }
  return ahead ? side + lo : lo;
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): ten rounds, each two 32 x
// 32 -> 64 bit products whose high halves are xored with the other words and
// the round's key.
PSS_HD void philox4x32(uint32_t c[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c[0];
    const uint64_t b = static_cast<uint64_t>(0xCD9E8D57u) * c[2];
    c[0] = static_cast<uint32_t>(b >> 32) ^ c[1] ^ k0;
    c[1] = static_cast<uint32_t>(b);
    c[2] = static_cast<uint32_t>(a >> 32) ^ c[3] ^ k1;
    c[3] = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// Numbers of the 8 elements of piece c8 of row r: element u is the low (even
// u) or high half of word u / 2.
PSS_HD void drop_words(uint32_t w[4], uint32_t k0, uint32_t k1, uint64_t n, uint32_t c8,
                       uint32_t r) {
  w[0] = c8;
  w[1] = r;
  w[2] = static_cast<uint32_t>(n);
  w[3] = static_cast<uint32_t>(n >> 32);
  philox4x32(w, k0, k1);
}
PSS_HD uint32_t drop_number(const uint32_t w[4], int u) {
  return (u & 1) ? w[u >> 1] >> 16 : w[u >> 1] & 0xffffu;
}

__device__ __forceinline__ uint64_t drop_offset(const Drop& d) {
  return d.offset + (d.step != nullptr ? *d.step : 0u);
}

// v = D(v) for piece c8 of row r (n: drop_offset of the call).  A dropped
// element is 0 whatever it held.
__device__ __forceinline__ void drop8(float v[kLanePiece], const Drop& d, uint64_t n, uint32_t c8,
                                      uint32_t r) {
  uint32_t w[4];
  drop_words(w, d.k0, d.k1, n, c8, r);
#pragma unroll
  for (int u = 0; u < kLanePiece; ++u) v[u] = drop_number(w, u) < d.t ? 0.f : v[u] * d.scale;
}

typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t h8_any __attribute__((ext_vector_type(8), aligned(2)));

// n (1 .. 8) elements from p on; the others of the piece are 0.  Whole pieces
// take 16-byte loads whatever their alignment: the memory system takes those
// at any element.
__device__ __forceinline__ void load8(float v[kLanePiece], const float* p, int n) {
  if (n >= kLanePiece) {
    const f4_any a = *reinterpret_cast<const f4_any*>(p);
    const f4_any b = *reinterpret_cast<const f4_any*>(p + 4);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v[u] = a[u];
      v[u + 4] = b[u];
    }
  } else {
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] = u < n ? p[u] : 0.f;
  }
}
__device__ __forceinline__ void load8(float v[kLanePiece], const uint16_t* p, int n) {
  if (n >= kLanePiece) {
    const h8_any a = *reinterpret_cast<const h8_any*>(p);
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] = bf16_to_f32(a[u]);
  } else {
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] = u < n ? bf16_to_f32(p[u]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* p, const float v[kLanePiece], int n) {
  if (n >= kLanePiece) {
    f4_any a, b;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      a[u] = v[u];
      b[u] = v[u + 4];
    }
    *reinterpret_cast<f4_any*>(p) = a;
    *reinterpret_cast<f4_any*>(p + 4) = b;
  } else {
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u)
      if (u < n) p[u] = v[u];
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float v[kLanePiece], int n) {
  if (n >= kLanePiece) {
    h8_any a;
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) a[u] = f32_to_bf16_rne(v[u]);
    *reinterpret_cast<h8_any*>(p) = a;
  } else {
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u)
      if (u < n) p[u] = f32_to_bf16_rne(v[u]);
  }
}

// Weights (bf16: their storage) of a piece; null: `fill`.
__device__ __forceinline__ void load_weights8(float v[kLanePiece], const void* w, bool bf16, int64_t c,
                                              int n, float fill) {
  if (w == nullptr) {
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] = fill;
  } else if (bf16) {
    load8(v, static_cast<const uint16_t*>(w) + c, n);
  } else {
    load8(v, static_cast<const float*>(w) + c, n);
  }
}

// Sum over the wavefront, in every lane, in a fixed order.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// Host-side launchers.
//
// Operators on rows (pss_rows.hip) of float32 or bfloat16 elements; rows,
// cols > 0.
hipError_t launch_dropout(bool bf16, const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                          int64_t rows, int64_t cols, const Drop& drop, hipStream_t stream);
hipError_t launch_norm(bool bf16, const NormArgs& a, const Drop& drop, hipStream_t stream);
// workspace: norm_grad_workspace_bytes, null when neither weight nor bias gradient
// is wanted.
size_t norm_grad_workspace_bytes(int64_t rows, int64_t cols);
hipError_t launch_norm_grad(bool bf16, const NormGradArgs& a, const Drop& drop, void* workspace,
                            hipStream_t stream);

// Relative position bias (pss_bias.hip); every size > 0.
hipError_t launch_bias(bool bf16, const BiasArgs& a, const BucketMap& map, hipStream_t stream);
// bias_grad_fits: as many blocks as a grid can have.
bool bias_grad_fits(const BiasArgs& a, const BucketMap& map);
size_t bias_grad_workspace_bytes(const BiasArgs& a, const BucketMap& map);
hipError_t launch_bias_grad(bool bf16, const BiasArgs& a, const BucketMap& map, void* workspace,
                            float* grad_table, hipStream_t stream);

}  // namespace pss
