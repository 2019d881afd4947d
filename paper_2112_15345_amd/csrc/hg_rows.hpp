// Shared by the kernels that walk over rows (hg_norm.hip, hg_layer_norm.hip, hg_quantize.hip):
// how threads share a row, its loads and stores, rows by ID, 8-bit results.
#pragma once

#include "hg_dense.hpp"

namespace hg {
namespace {

constexpr int kBlock = 256;
// Blocks of a walk over the rows: 8 on each of 256 compute units going forward; fewer
// going backward, where each leaves a part of dweight.
constexpr int64_t kResident = 2048;
constexpr int64_t kParts = 1024;

// Threads that share a row, and how to reduce over them.  Past a wavefront each
// reduction goes through one of two LDS buffers in turn, so that one barrier is enough.
template <int G>
struct Group {
  static constexpr int kRows = kBlock / G;  // rows of a block at a time
  static constexpr int kLds = G > 64 ? 4 * (kBlock / 64) : 1;
  float *red;  // LDS [kLds]
  int turn = 0;
  __device__ explicit Group(float *lds) : red(lds) {}
  // Sums of two values.
  __device__ __forceinline__ void sum(float &a, float &b) {
    a = lanes_sum<(G < 64 ? G : 64)>(a);
    b = lanes_sum<(G < 64 ? G : 64)>(b);
    if (G > 64) {
      float *const r = red + (turn ^= 1) * 2 * (kBlock / 64);
      if ((threadIdx.x & 63) == 0) {
        r[threadIdx.x >> 6] = a;
        r[kBlock / 64 + (threadIdx.x >> 6)] = b;
      }
      __syncthreads();
      a = b = 0.0f;
#pragma unroll
      for (int i = 0; i < kBlock / 64; ++i) {
        a += r[i];
        b += r[kBlock / 64 + i];
      }
    }
  }
  __device__ __forceinline__ float sum(float v) {
    float none = 0.0f;
    sum(v, none);
    return v;
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) {
    v = lanes_max_bits<(G < 64 ? G : 64)>(v);
    if (G > 64) {
      float *const r = red + (turn ^= 1) * 2 * (kBlock / 64);
      if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = __uint_as_float(v);
      __syncthreads();
      v = 0;
#pragma unroll
      for (int i = 0; i < kBlock / 64; ++i) v = ::max(v, __float_as_uint(r[i]));
    }
    return v;
  }
};

// The largest magnitude as bits: NaN is above infinity, so it is kept.
__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A scale that takes magnitudes up to amax to 448 (e4m3) or 127 (integers).
template <bool kIntegers = false>
__device__ __forceinline__ float scale_of(uint32_t amax) {
  const float a = __uint_as_float(amax);
  // (not fmax: it would drop a NaN)
  const float c = kIntegers ? a * (1.0f / 127.0f) : a / 448.0f;
  if (kIntegers && !(c < INFINITY)) return __builtin_nanf("");
  return c < 0x1p-126f ? 0x1p-126f : c;
}

// Four values in 8 bits, rounded to nearest even; |v| <= 448 or NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// N bytes of words, n (>= 1) of them in memory.
template <int N>
__device__ __forceinline__ void store_words(uint8_t *p, const uint32_t *w, int n) {
  if (n >= N) {
    __builtin_memcpy(p, w, N);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = uint8_t(w[i / 4] >> (8 * (i % 4)));
  }
}

template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t *p, const float *v, int n) {
  uint32_t w[V / 4];
#pragma unroll
  for (int i = 0; i < V / 4; ++i)
    w[i] = pack_e4m3(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  store_words<V>(p, w, n);
}

// Integers have neither NaN nor infinities: a row (or group) that has one is zeros with a
// scale of NaN, so that what it stands for is NaN.
__device__ __forceinline__ bool is_broken(uint32_t amax) { return amax >= 0x7f800000u; }

// Four values as 8-bit integers, rounded to nearest even; |v| <= 127.5.  The sum with 1.5 2^23
// has the integer in its low bits.
__device__ __forceinline__ uint32_t pack_i8(float a, float b, float c, float d) {
  const auto bits = [](float v) { return __float_as_uint(v + 12582912.0f); };
  const uint32_t ab = __builtin_amdgcn_perm(bits(b), bits(a), 0x0c0c0400u);
  const uint32_t cd = __builtin_amdgcn_perm(bits(d), bits(c), 0x04000c0cu);
  return ab | cd;
}

// V values of a vector over the columns, in float32 or T (HG_DT_NONE: all `none`).
template <typename T>
__device__ __forceinline__ void load_columns(const void *p, int32_t dtype, float none, int64_t c,
                                             int n, float *w) {
  constexpr int V = kVec<T>;
  if (dtype == HG_DT_NONE) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = none;
  } else if (dtype == HG_DT_F32) {
    Vec<float, V> t;
    t.load(static_cast<const float *>(p) + c, n);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = t.e[i];
  } else {
    Vec<T> t;
    t.load(static_cast<const T *>(p) + c, n);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = float(t.e[i]);
  }
}

// The row that position i stands for: its place in x, or -1 where the id is out of
// range.
struct Source {
  const int64_t *ids;
  int64_t rows;
  __device__ __forceinline__ int64_t at(int64_t i) const {
    if (!ids) return i;
    const int64_t v = ids[i];
    return v >= 0 && v < rows ? v : -1;
  }
};

template <typename T>
__device__ __forceinline__ void fill_nan(Vec<T> &t) {
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) t.e[j] = T(__builtin_nanf(""));
}

// One vector (n > 0 elements of it) of a row of x; its elements past n are 0.
template <typename T, Move M = Move::kStreamed>
__device__ __forceinline__ void load_x(const void *x, int64_t stride, int64_t at, int c, int n,
                                       Vec<T> &t) {
  if (at >= 0) {
    t.template load<M>(static_cast<const T *>(x) + at * stride + c, n);
  } else {
    fill_nan(t);
#pragma unroll
    for (int j = 0; j < kVec<T>; ++j)
      if (j >= n) t.e[j] = T(0.0f);
  }
}

template <typename T>
__device__ __forceinline__ void store_row(T *p, const float *v, int n) {
  Vec<T> t;
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) t.e[j] = T(v[j]);
  t.template store<Move::kStreamed>(p, n);
}

// How a row is shared: f.template run<G, NV>().
template <typename F>
hipError_t by_vectors(int64_t vecs, F f) {
  if (vecs <= 8) return f.template run<8, 1>();
  if (vecs <= 16) return f.template run<16, 1>();
  if (vecs <= 32) return f.template run<32, 1>();
  if (vecs <= 64) return f.template run<64, 1>();
  if (vecs <= 128) return f.template run<64, 2>();
  if (vecs <= 256) return f.template run<64, 4>();
  if (vecs <= 512) return f.template run<256, 2>();
  if (vecs <= 1024) return f.template run<256, 4>();
  return f.template run<256, 0>();
}
template <typename T, typename F>
hipError_t by_dim(int64_t dim, F f) {
  return by_vectors(ceil_div<int64_t>(dim, kVec<T>), f);
}

}  // namespace
}  // namespace hg
