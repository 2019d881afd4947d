// Rows kept in 8-bit integers, and what they stand for.
//
//   c = max(max |x| (1 / 127), 2^-126) over a row, or over each group of 128 columns,  q = x / c rounded
//   x = q c
//
// The quotient is the float32 one, rounded to the nearest integer, of two as near the even one: so
// that the integers are the definition's bit for bit.  A product with 1 / c rounds to the same integer
// unless it lies within kNear of a middle between two, and only there is it divided.
//
// Bound by memory once few enough instructions are left for an element (65537 x 1024 in bfloat16, in
// groups: 67 us with 8 elements a lane, float32 maxima and a 64-bit division for each group): a lane
// takes kWide neighbours, the largest magnitude is taken of 16-bit halves, and the position in the row
// is counted up.
#include "hg_rows.hpp"

namespace hg {
namespace {

// Of r, a reciprocal of c within 2^-23: |RN(x r) - RN(x / c)| is at most 2^-23 + 2 x 2^-24 of 127,
// below 2^-15.
constexpr float kNear = 0x1p-15f;

// i / per and i % per.  (The division of 64 bits takes some 100 instructions, of 32 some 20.)
struct Place {
  int64_t row, part;
};
__device__ __forceinline__ Place place_of(int64_t i, int64_t per) {
  if ((i | per) >> 32 == 0) {
    const uint32_t row = uint32_t(i) / uint32_t(per);
    return Place{int64_t(row), int64_t(uint32_t(i) - row * uint32_t(per))};
  }
  return Place{i / per, i % per};
}

// Neighbours of a row that a lane takes: 16 bytes of integers; 8 of float32.
template <typename T>
constexpr int kWide = sizeof(T) == 2 ? 16 : 8;

// The largest magnitude's bits as a float32's (of 16-bit types: as their own, two at a time).
template <typename T, int N>
__device__ __forceinline__ uint32_t largest(const Vec<T, N> &x, uint32_t before) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  uint32_t w[N * sizeof(T) / 4];
  __builtin_memcpy(w, x.e, sizeof(w));
#pragma unroll
  for (int k = 0; k < int(N * sizeof(T) / 4); ++k) {
    if constexpr (sizeof(T) == 4)
      before = max(before, w[k] & 0x7fffffffu);
    else
      before = __builtin_bit_cast(
          uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, before),
                                              __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu)));
  }
  return before;
}
template <typename T>
__device__ __forceinline__ uint32_t as_f32_bits(uint32_t m) {
  if constexpr (sizeof(T) == 4) {
    return m;
  } else {
    const uint16_t top = uint16_t(max(m & 0xffffu, m >> 16));
    return __float_as_uint(float(__builtin_bit_cast(T, top)));
  }
}

// N (a multiple of 4) of the values as integers; zeros where the group is broken.
template <int N>
__device__ __forceinline__ void integers(const float *x, float c, float f, bool broken,
                                         uint32_t *w) {
  float q[N];
  float off = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    q[k] = x[k] * f;
    off = fmaxf(off, fabsf(q[k] - rintf(q[k])));
  }
  if (off > 0.5f - kNear) {
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = x[k] / c;
  }
#pragma unroll
  for (int k = 0; k < N / 4; ++k)
    w[k] = broken ? 0 : pack_i8(q[4 * k], q[4 * k + 1], q[4 * k + 2], q[4 * k + 3]);
}

// G lanes take a group of columns: `groups` of `width` columns a row.  NV times kWide neighbours a
// lane hold it; walks over the groups, the next one's loads in flight while this one is written.
template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_quantize(hg_quantize_args A, int64_t groups,
                                                     int64_t width) {
  constexpr int V = kWide<T>;
  constexpr int kRows = Group<G>::kRows;
  __shared__ float red[Group<G>::kLds];
  Group<G> grp(red);
  const int lane = threadIdx.x % G;
  const int64_t all = A.rows * groups, step = int64_t(gridDim.x) * kRows;
  const Place by = place_of(step, groups);
  int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / G;
  Place at = place_of(i, groups), next = at;
  Vec<T, V> x[NV];
  const auto load = [&](Place p) {
    const int64_t c0 = p.part * width;
    const int n = int(min(width, A.dim - c0));
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      if (c < n)
        x[v].template load<Move::kStreamed>(static_cast<const T *>(A.x) + p.row * A.x_stride + c0 + c,
                                            n - c);
      else
        __builtin_memset(x[v].e, 0, sizeof(x[v].e));
    }
  };
  if (i < all) load(at);
  for (; i < all; i += step, at = next) {
    const int64_t c0 = at.part * width;
    const int n = int(min(width, A.dim - c0));
    uint32_t amax = 0;
    Vec<T, V> now[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      now[v] = x[v];
      amax = largest<T, V>(now[v], amax);
    }
    next = Place{at.row + by.row, at.part + by.part};
    if (next.part >= groups) next = Place{next.row + 1, next.part - groups};
    if (i + step < all) load(next);
    amax = grp.max(as_f32_bits<T>(amax));
    const bool broken = is_broken(amax);
    const float c = scale_of<true>(amax), f = __builtin_amdgcn_rcpf(c);
    if (lane == 0) A.scale[i] = c;
    uint8_t *const q = reinterpret_cast<uint8_t *>(A.q) + at.row * A.q_stride + c0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int j = (v * G + lane) * V;
      if (j < n) {
        float h[V];
        uint32_t w[V / 4];
#pragma unroll
        for (int k = 0; k < V; ++k) h[k] = float(now[v].e[k]);
        integers<V>(h, c, f, broken, w);
        store_words<V>(q + j, w, n - j);
      }
    }
  }
}

// Rows that do not fit in a block's registers: read twice.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_quantize_long(hg_quantize_args A) {
  constexpr int V = kVec<T>;
  __shared__ float red[Group<kBlock>::kLds];
  Group<kBlock> grp(red);
  const uint32_t dim = uint32_t(A.dim);
  for (int64_t i = blockIdx.x; i < A.rows; i += gridDim.x) {
    const T *const x = static_cast<const T *>(A.x) + i * A.x_stride;
    uint8_t *const q = reinterpret_cast<uint8_t *>(A.q) + i * A.q_stride;
    uint32_t amax = 0;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      Vec<T> t;
      t.load(x + c, dim - c);
#pragma unroll
      for (int j = 0; j < V; ++j) amax = max(amax, mag(float(t.e[j])));
    }
    amax = grp.max(amax);
    const float s = scale_of<true>(amax), f = __builtin_amdgcn_rcpf(s);
    if (threadIdx.x == 0) A.scale[i] = s;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      Vec<T> t;
      t.load(x + c, dim - c);
      float h[V];
      uint32_t w[V / 4];
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = float(t.e[j]);
      integers<V>(h, s, f, is_broken(amax), w);
      store_words<V>(q + c, w, dim - c);
    }
  }
}

// 16 bytes of the result a lane, so that a store's lanes write whole lines, kAhead of them in flight;
// zeros from column `cols` to out_cols.  (Rows that a product reads next stay in the caches: 16385 x 1024
// x 4096's backward pass 436 us, 460 where they were streamed past them.)
template <typename O, Move M>
__global__ __launch_bounds__(kBlock) void k_dequantize(Kept K, int64_t rows, int64_t cols,
                                                       int64_t out_cols, O *out, int64_t stride) {
  constexpr int N = kVec<O>, kAhead = 4;
  const int64_t across = (out_cols + N - 1) / N, all = rows * across;
  for (int64_t t0 = int64_t(blockIdx.x) * kBlock * kAhead + threadIdx.x; t0 < all;
       t0 += int64_t(gridDim.x) * kBlock * kAhead) {
    Place p[kAhead];
    float v[kAhead][N];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t t = t0 + u * kBlock;
      p[u] = place_of(min(t, all - 1), across);
      p[u].part *= N;
      K.load<N>(p[u].row, p[u].part, int(max<int64_t>(0, min<int64_t>(N, cols - p[u].part))), v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (t0 + u * kBlock >= all) break;
      Vec<O, N> o;
#pragma unroll
      for (int k = 0; k < N; ++k) o.e[k] = O(v[u][k]);
      o.template store<M>(out + p[u].row * stride + p[u].part,
                                        int(min<int64_t>(N, out_cols - p[u].part)));
    }
  }
}

template <typename T>
struct Quantize {
  const hg_quantize_args &A;
  hipStream_t stream;
  template <int G, int NV>
  hipError_t run() const {
    if constexpr (NV == 0) {
      hipLaunchKernelGGL((k_quantize_long<T>),
                         dim3(unsigned(std::min<int64_t>(A.rows, 65536))), dim3(kBlock), 0, stream,
                         A);
    } else {
      const int64_t groups = A.group ? ceil_div<int64_t>(A.dim, A.group) : 1;
      const int64_t blocks = ceil_div<int64_t>(A.rows * groups, Group<G>::kRows);
      hipLaunchKernelGGL((k_quantize<T, G, NV>), dim3(unsigned(std::min(blocks, kResident))),
                         dim3(kBlock), 0, stream, A, groups, A.group ? A.group : A.dim);
    }
    return hipGetLastError();
  }
};

template <typename T>
hipError_t quantize(const hg_quantize_args &A, hipStream_t stream) {
  const int64_t width = A.group ? std::min<int64_t>(A.group, A.dim) : A.dim;
  return by_vectors(ceil_div<int64_t>(width, kWide<T>), Quantize<T>{A, stream});
}

template <typename O>
hipError_t dequantize(const Kept &K, int64_t rows, int64_t cols, int64_t out_cols, O *out,
                      int64_t stride, bool read_next, hipStream_t stream) {
  const int64_t blocks = ceil_div<int64_t>(rows * ceil_div<int64_t>(out_cols, kVec<O>), kBlock * 4);
  const dim3 grid(unsigned(std::min(blocks, kMostBlocks))), block(kBlock);
  if (read_next)
    hipLaunchKernelGGL((k_dequantize<O, Move::kCached>), grid, block, 0, stream, K, rows, cols,
                       out_cols, out, stride);
  else
    hipLaunchKernelGGL((k_dequantize<O, Move::kStreamed>), grid, block, 0, stream, K, rows, cols,
                       out_cols, out, stride);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const hg_quantize_args &A, hipStream_t stream) {
  if (A.rows <= 0) return hipSuccess;
  switch (A.dtype) {
    case HG_DT_F32: return quantize<float>(A, stream);
    case HG_DT_F16: return quantize<_Float16>(A, stream);
    default: return quantize<__bf16>(A, stream);
  }
}

hipError_t launch_dequantize(const Kept &K, int64_t rows, int64_t cols, int64_t out_cols,
                             int32_t dtype, void *out, int64_t stride, bool read_next,
                             hipStream_t stream) {
  if (rows <= 0 || out_cols <= 0) return hipSuccess;
  switch (dtype) {
    case HG_DT_F32:
      return dequantize(K, rows, cols, out_cols, static_cast<float *>(out), stride, read_next, stream);
    case HG_DT_F16:
      return dequantize(K, rows, cols, out_cols, static_cast<_Float16 *>(out), stride, read_next,
                        stream);
    default:
      return dequantize(K, rows, cols, out_cols, static_cast<__bf16 *>(out), stride, read_next,
                        stream);
  }
}

}  // namespace hg
