// Operators on rows and the relative position bias (internal to the library):
// their launchers, rows of float32 or bfloat16 elements in pieces of 8, the
// counter-based dropout mask and the position buckets (host and device).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
// Those of the differences key - query that need no search: beyond the last border,
// and ahead of the query on a single side.
struct FarBuckets {
  int32_t behind = 0, ahead = 0;  // of differences <= -near, >= from
  int32_t near = 0, from = 0;
};
struct BucketMap {
  int32_t num = 0, side = 0, both = 0;
  FarBuckets far;  // ahead of the borders: a kernel needs them before those
  int32_t borders[kMaxBuckets];
};
inline FarBuckets far_buckets(const BucketMap& map) {
  FarBuckets f;
  f.near = map.borders[map.side - 1];
  f.behind = map.side - 1;
  f.from = map.both ? (f.near > 1 ? f.near : 1) : 0;
  f.ahead = map.num - 1;
  if (!map.both) {  // the last of the buckets from distance 0 on
    f.ahead = 0;
    while (f.ahead + 1 < map.side && map.borders[f.ahead + 1] <= 0) ++f.ahead;
  }
  return f;
}

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
template <typename I>
PSS_HD int bucket_of(I rel, const int32_t* borders, int side, bool both) {
  const bool ahead = both && rel > 0;
  const I n = rel < 0 ? -rel : (both ? rel : 0);
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

// Vectors in memory: 16-byte loads and stores at any element (the memory system
// takes them at any alignment of whole elements).
typedef float f2_any __attribute__((ext_vector_type(2), aligned(4)));
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t w1_any __attribute__((aligned(2)));
typedef uint32_t w2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint16_t h4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint16_t h8_any __attribute__((ext_vector_type(8), aligned(2)));
template <typename T>
struct Vec;  // 16 bytes of T
template <>
struct Vec<float> {
  typedef f4_any type;
};
template <>
struct Vec<uint16_t> {
  typedef h8_any type;
};
template <typename T>
constexpr int kVec = 16 / static_cast<int>(sizeof(T));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return bf16_to_f32(x); }

// The end of a row whose length is not a whole number of vectors: n of its last
// vector's elements, n = rest (the same in every lane).  kOverlap: one load that
// also takes elements before them, moved down when the vector is used (settle), by
// which time it has arrived; for rows of at least a vector that one wavefront
// alone reads and writes (a result stored in place by another one may be there).
// kPieces: loads of 8, 4 and 2 bytes.  Rows of whole vectors need neither, and
// kernels of their own save the registers (norm of 32768 x 1024 bfloat16: 28 us,
// with the code for ends 33).
enum class End { kWhole, kOverlap, kPieces };

__device__ __forceinline__ f4_any load_end(const float* p, int rest) {
  f4_any x = {0.f, 0.f, 0.f, 0.f};
  if (rest & 2) {
    const f2_any a = __builtin_nontemporal_load(reinterpret_cast<const f2_any*>(p));
    x[0] = a[0];
    x[1] = a[1];
  }
  if (rest & 1) x[2] = __builtin_nontemporal_load(p + (rest & 2));
  return x;
}
__device__ __forceinline__ h8_any load_end(const uint16_t* p, int rest) {
  uint32_t w[4] = {0, 0, 0, 0};
  if (rest & 4) {
    const w2_any a = __builtin_nontemporal_load(reinterpret_cast<const w2_any*>(p));
    w[0] = a[0];
    w[1] = a[1];
  }
  if (rest & 2) w[2] = __builtin_nontemporal_load(reinterpret_cast<const w1_any*>(p + (rest & 4)));
  if (rest & 1) w[3] = __builtin_nontemporal_load(p + (rest & 6));
  h8_any x;
  __builtin_memcpy(&x, w, 16);
  return x;
}

// Rows are read once: past the caches (their lines are not kept for others),
// which for a large copy of float32 is 6.2 against 5.8 TB/s.  n elements from p
// on (kVec or more: all, 0 or less: none); the others are 0 once it is settled.
template <End E, typename T>
__device__ __forceinline__ typename Vec<T>::type load_vec(const T* p, int n, int rest) {
  typedef typename Vec<T>::type V;
  if (E == End::kOverlap && n < kVec<T>) p += rest - kVec<T>;
  if (E == End::kPieces ? n >= kVec<T> : n > 0)
    return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  V x = 0;
  if (E == End::kPieces && n > 0) x = load_end(p, rest);
  return x;
}

template <End E>
__device__ __forceinline__ f4_any settle(f4_any x, int n, int rest) {
  if (E == End::kWhole || n <= 0 || n >= 4) return x;
  if (E == End::kOverlap) {
    const int by = 4 - rest;
    if (by & 1) x = f4_any{x[1], x[2], x[3], 0.f};
    if (by & 2) x = f4_any{x[2], x[3], 0.f, 0.f};
  } else if (!(rest & 2)) {
    x = f4_any{x[2], 0.f, 0.f, 0.f};
  }
  return x;
}
template <End E>
__device__ __forceinline__ h8_any settle(h8_any x, int n, int rest) {
  if (E == End::kWhole || n <= 0 || n >= 8) return x;
  uint32_t w[4];
  __builtin_memcpy(w, &x, 16);
  if (E == End::kOverlap) {
    const int by = 8 - rest;
    if (by & 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = w[i] >> 16 | (i < 3 ? w[i + 1] << 16 : 0);
    }
    if (by & 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = i < 3 ? w[i + 1] : 0;
    }
    if (by & 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = i < 2 ? w[i + 2] : 0;
    }
  } else {
    if (!(rest & 2)) {
      w[2] = w[3];
      w[3] = 0;
    }
    if (!(rest & 4)) {
      w[0] = w[2];
      w[1] = w[3];
      w[2] = w[3] = 0;
    }
  }
  __builtin_memcpy(&x, w, 16);
  return x;
}

// Two floats as bfloat16 bits, to nearest even (one instruction).
typedef float f2_v __attribute__((ext_vector_type(2)));
typedef __bf16 b2_v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const b2_v b = __builtin_convertvector(f2_v{lo, hi}, b2_v);
  uint32_t u;
  __builtin_memcpy(&u, &b, 4);
  return u;
}
__device__ __forceinline__ f4_any narrow(const float* v, float) {
  return f4_any{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ h8_any narrow(const float* v, uint16_t) {
  h8_any a;
#pragma unroll
  for (int u = 0; u < 8; u += 2) {
    const uint32_t w = bf16_pair(v[u], v[u + 1]);
    a[u] = static_cast<uint16_t>(w);
    a[u + 1] = static_cast<uint16_t>(w >> 16);
  }
  return a;
}
// Stores of a row's end by halves of the vector.
__device__ __forceinline__ void store_end(float* p, f4_any a, int n) {
  if (n & 2) *reinterpret_cast<f2_any*>(p) = f2_any{a[0], a[1]};
  if (n & 1) p[n & 2] = n & 2 ? a[2] : a[0];
}
__device__ __forceinline__ void store_end(uint16_t* p, h8_any a, int n) {
  uint32_t w[4];
  __builtin_memcpy(w, &a, 16);
  if (n & 4) {
    *reinterpret_cast<w2_any*>(p) = w2_any{w[0], w[1]};
    p += 4;
    w[0] = w[2];
    w[1] = w[3];
  }
  if (n & 2) {
    *reinterpret_cast<w1_any*>(p) = w[0];
    p += 2;
    w[0] = w[1];
  }
  if (n & 1) *p = static_cast<uint16_t>(w[0]);
}
// PAST: past the caches; ENDS: n may be below kVec and above 0.  (PAST is a
// kernel's own: of two kinds of store in one kernel the compiler makes one.)
template <bool ENDS, bool PAST, typename T>
__device__ __forceinline__ void store_vec(T* p, const float* v, int n) {
  typedef typename Vec<T>::type V;
  const V a = narrow(v, T{});
  if (ENDS ? n >= kVec<T> : n > 0) {
    if constexpr (PAST)
      __builtin_nontemporal_store(a, reinterpret_cast<V*>(p));
    else
      *reinterpret_cast<V*>(p) = a;
  } else if (ENDS && n > 0) {
    store_end(p, a, n);
  }
}

// A span: G * 8 consecutive columns of a row, 8 of them to each of G
// neighbouring lanes, laid out so that the lanes of one load or store are
// 16 bytes apart: a bfloat16 lane has columns 8 lane .. 8 lane + 7, a float32 lane
// 4 lane .. 4 lane + 3 and the same of the span's second half (32 bytes apart a
// large float32 copy runs at 5.2 to 5.9 TB/s, 16 apart at 5.8 to 6.2).
// ENDS: rows may end inside a vector.
template <typename T, int G, bool ENDS>
struct Span {
  static constexpr End kEnd = !ENDS ? End::kWhole : (G > 1 && G < kWave ? End::kOverlap : End::kPieces);
  static constexpr int kParts = kLanePiece / kVec<T>;
  typename Vec<T>::type q[kParts];

  static __device__ __forceinline__ int col(int lane, int u) {
    return u / kVec<T> * (G * kVec<T>) + lane * kVec<T> + u % kVec<T>;
  }
  // Elements of the last vector of a row that ends `left` columns on.
  static __device__ __forceinline__ int rest(int left) { return left & (kVec<T> - 1); }
  // p: the span's first column; left: columns from there to the row's end; there:
  // false for a row past the last.
  __device__ __forceinline__ void load(const T* p, int lane, int left, bool there = true) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int c = col(lane, i * kVec<T>);
      q[i] = load_vec<kEnd>(p + c, there ? left - c : 0, rest(left));
    }
  }
  // Before the span's elements are used.
  __device__ __forceinline__ void settle_end(int lane, int left) {
#pragma unroll
    for (int i = 0; i < kParts; ++i)
      q[i] = settle<kEnd>(q[i], left - col(lane, i * kVec<T>), rest(left));
  }
  // From here on the compiler takes the span as new: values made from it before
  // are made again rather than kept in registers.
  __device__ __forceinline__ void renew() {
    static_assert(sizeof(q) % 4 == 0, "whole registers");
    uint32_t word[sizeof(q) / 4];
    __builtin_memcpy(word, q, sizeof(q));
#pragma unroll
    for (unsigned i = 0; i < sizeof(q) / 4; ++i) asm("" : "+v"(word[i]));
    __builtin_memcpy(q, word, sizeof(q));
  }
  __device__ __forceinline__ void widen_to(float v[kLanePiece]) const {
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] = widen(q[u / kVec<T>][u % kVec<T>]);
  }
  template <bool PAST, typename O>
  static __device__ __forceinline__ void store(O* p, const float v[kLanePiece], int lane, int left) {
    constexpr int V = kVec<O> < kVec<T> ? kVec<O> : kVec<T>;  // consecutive columns
#pragma unroll
    for (int u = 0; u < kLanePiece; u += V)
      store_vec<ENDS, PAST>(p + col(lane, u), v + u, left - col(lane, u));
  }
  // Weights (bf16: their storage) from column c0 on in the span's layout; null:
  // `fill`.  Other blocks read them too: through the caches, in fours.
  static __device__ __forceinline__ void weights(float v[kLanePiece], const void* w, bool bf16,
                                                 int64_t c0, int lane, int left, float fill) {
#pragma unroll
    for (int u = 0; u < kLanePiece; u += 4) {
      const int c = col(lane, u);
      const bool whole = c + 4 <= left;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[u + k] = fill;
      if (w == nullptr) continue;
      if (bf16) {
        const uint16_t* p = static_cast<const uint16_t*>(w) + c0 + c;
        if (whole) {
          const h4_any x = *reinterpret_cast<const h4_any*>(p);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[u + k] = bf16_to_f32(x[k]);
        } else if (ENDS) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + k < left) v[u + k] = bf16_to_f32(p[k]);
        }
      } else {
        const float* p = static_cast<const float*>(w) + c0 + c;
        if (whole) {
          const f4_any x = *reinterpret_cast<const f4_any*>(p);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[u + k] = x[k];
        } else if (ENDS) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + k < left) v[u + k] = p[k];
        }
      }
    }
  }
  // v = D(v) in row r of the span at piece c8 (n: drop_offset of the call).  A
  // dropped element is 0 whatever it held.  A float32 lane has halves of two
  // pieces, which a pair of lanes shares: the even lane makes the numbers of the
  // first, the odd one those of the second, and they exchange halves.  The
  // lanes of a group take part together.
  static __device__ __forceinline__ void drop(float v[kLanePiece], const Drop& d, uint64_t n,
                                              uint32_t c8, uint32_t r, int lane) {
    uint32_t w[4];
    if constexpr (kParts == 1 || G == 1) {
      drop_words(w, d.k0, d.k1, n, c8 + lane, r);
    } else {
      const bool odd = lane & 1;
      drop_words(w, d.k0, d.k1, n, c8 + (odd ? G / 2 : 0) + lane / 2, r);
      const uint32_t give0 = odd ? w[0] : w[2], give1 = odd ? w[1] : w[3];
      const uint32_t got0 = __builtin_amdgcn_update_dpp(0, give0, 0xb1, 0xf, 0xf, true);
      const uint32_t got1 = __builtin_amdgcn_update_dpp(0, give1, 0xb1, 0xf, 0xf, true);
      if (odd) {
        w[0] = got0;
        w[1] = got1;
      } else {
        w[2] = got0;
        w[3] = got1;
      }
    }
#pragma unroll
    for (int u = 0; u < kLanePiece; ++u) v[u] = drop_number(w, u) < d.t ? 0.f : v[u] * d.scale;
  }
};

// Sum over groups of G neighbouring lanes (a power of two), the same bits in
// every lane of a group; every lane of the wavefront takes part.  Within 16
// lanes by data-parallel moves: halves that hold equal sums are exchanged by
// quad permutations and mirrored rows, so that lane i adds what lane i ^ m has.
template <int CTRL>
__device__ __forceinline__ float add_moved(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  if (G > 1) v = add_moved<0xb1>(v);   // quad_perm 1,0,3,2
  if (G > 2) v = add_moved<0x4e>(v);   // quad_perm 2,3,0,1
  if (G > 4) v = add_moved<0x141>(v);  // row_half_mirror
  if (G > 8) v = add_moved<0x140>(v);  // row_mirror
  if (G > 16) v += __shfl_xor(v, 16);
  if (G > 32) v += __shfl_xor(v, 32);
  return v;
}
__device__ __forceinline__ float wave_sum(float v) { return group_sum<kWave>(v); }

// Results of more than this are stored past the caches.  The call itself gains 3 to 13%
// at nearly every size; a next call that reads the results loses as long as the
// memory-side cache (256 MB) would have held them.  Which of the two a program has the library
// cannot see; below 64 MB the results are taken to be read next.  us through / past
// the caches by the size of one result, rows of 4096 bfloat16, scores 512 x 1024:
//                                   72 MB        128 MB       256 MB       512 MB
//   norm                         30.0 / 28.6  50.0 / 47.6   102 / 95     193 / 184
//   norm, dropout of its result  53.3 / 54.6  88.3 / 90.9   173 / 178    373 / 350
//   residual, dropout, norm      57.5 / 55.7   104 / 100    212 / 204    455 / 428
//   the same, norm of both       94.1 / 98.1   162 / 172    353 / 348    771 / 724
//   dropout                      28.0 / 25.3  48.3 / 42.7   92.8 / 82.3  181 / 163
//   dropout, norm of its result  54.5 / 54.6  90.9 / 90.7   180 / 174    382 / 355
//   position bias                             48.4 / 46.4   94.4 / 89.6  187 / 176
//   bias, its table's gradient                72.0 / 78.9   133 / 144    276 / 270
// (Float32 gains 3 to 19% alone; its chains lose up to 7% at 72 and 128 MB, lie between
// 7% slower and 10% faster at 256 and gain from 384 on.)
constexpr int64_t kPastBytes = int64_t{64} << 20;

// f(the constant that n equals); n is one of them.
template <int N, int... MORE, typename F>
auto with_const(int n, F f) {
  if constexpr (sizeof...(MORE) > 0) {
    if (n != N) return with_const<MORE...>(n, f);
  }
  return f(std::integral_constant<int, N>{});
}

// Workgroups in one dimension of a grid: it holds fewer than 2^32 work-items
// (a larger one is cut to its low 32 bits without an error).
constexpr int64_t kGridBlocks = 1 << 22;  // of up to 1024 threads less one
constexpr int64_t kGridSlices = 65535;    // of the second dimension

// tiles x parts workgroups: grid.x holds `per` tiles of `parts` each, grid.y as many
// such slices as it takes (tile_of; the last slice may lie past the end).
struct TileGrid {
  dim3 grid;
  uint32_t per = 0;
  bool fits = false;
};
inline TileGrid tile_grid(int64_t tiles, int64_t parts) {
  TileGrid g;
  const int64_t most = parts < kGridBlocks ? (kGridBlocks - 1) / parts : 1;
  const int64_t per = tiles < most ? tiles : most, slices = (tiles + per - 1) / per;
  g.fits = parts < kGridBlocks && slices <= kGridSlices;
  g.grid = dim3(static_cast<uint32_t>(per * parts), static_cast<uint32_t>(slices));
  g.per = static_cast<uint32_t>(per);
  return g;
}
__device__ __forceinline__ uint32_t tile_of(uint32_t per, uint32_t parts) {
  return blockIdx.y * per + blockIdx.x / parts;
}

// Host-side launchers.
//
// Operators on rows (pss_rows.hip) of float32 or bfloat16 elements; rows,
// cols > 0.
hipError_t launch_dropout(bool bf16, const RowsIn& x, const RowsIn& residual, const RowsOut& out,
                          int64_t rows, int64_t cols, const Drop& drop, hipStream_t stream);
hipError_t launch_norm(bool bf16, const NormArgs& a, const Drop& drop, hipStream_t stream);
// workspace: norm_grad_workspace_bytes (may be 0); sums: a weight or bias gradient
// is wanted.
size_t norm_grad_workspace_bytes(bool bf16, int64_t rows, int64_t cols, bool sums);
hipError_t launch_norm_grad(bool bf16, const NormGradArgs& a, const Drop& drop, void* workspace,
                            hipStream_t stream);

// Relative position bias (pss_bias.hip); every size > 0.
hipError_t launch_bias(bool bf16, const BiasArgs& a, const BucketMap& map, hipStream_t stream);
// bias_grad_fits: as many blocks as a grid can have.
bool bias_grad_fits(bool bf16, const BiasArgs& a, const BucketMap& map);
size_t bias_grad_workspace_bytes(bool bf16, const BiasArgs& a, const BucketMap& map);
hipError_t launch_bias_grad(bool bf16, const BiasArgs& a, const BucketMap& map, void* workspace,
                            float* grad_table, hipStream_t stream);

}  // namespace pss
