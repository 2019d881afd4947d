// Root-mean-square norm with the residual's addition, and its backward pass.
//
//   h = x + r,  s = 1 / sqrt(mean(h^2) + eps),  y = h s w
//   dx = s (g - h s^2 mean(g h)) + dsum with g = dy w,  dw = sum_i dy h s
//
// Bound by memory: a row is read once, kept in registers, reduced, and written
// once.  A group of 8 to 64 lanes, or a block, takes a row; each lane holds up to
// kMaxVecs vectors of 16 bytes of it.  Rows longer than that are read twice.
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

__device__ __forceinline__ float scale_of(uint32_t amax) {
  const float a = __uint_as_float(amax);
  // (not fmax: it would drop a NaN)
  const float c = a / 448.0f;
  return c < 0x1p-126f ? 0x1p-126f : c;
}

// Four values in 8 bits, rounded to nearest even; |v| <= 448 or NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t *p, const float *v, int n) {
  uint32_t w[V / 4];
#pragma unroll
  for (int i = 0; i < V / 4; ++i)
    w[i] = pack_e4m3(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  if (n >= V) {
    __builtin_memcpy(p, w, V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = uint8_t(w[i / 4] >> (8 * (i % 4)));
  }
}

template <typename T>
__device__ __forceinline__ void load_weight(const hg_norm_args &A, int64_t c, int n, float *w) {
  constexpr int V = kVec<T>;
  if (A.weight_dtype == HG_DT_NONE) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = 1.0f;
  } else if (A.weight_dtype == HG_DT_F32) {
    Vec<float, V> t;
    t.load(static_cast<const float *>(A.weight) + c, n);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = t.e[i];
  } else {
    Vec<T> t;
    t.load(static_cast<const T *>(A.weight) + c, n);
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

// NV vectors a lane hold the row (NV > 0).  Groups walk over the rows and load the next
// one while this one is reduced and written.
template <typename T, int G, int NV, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_rms_norm(hg_norm_args A) {
  constexpr int V = kVec<T>;
  constexpr int kRows = Group<G>::kRows;
  __shared__ float red[Group<G>::kLds];
  Group<G> grp(red);
  const int lane = threadIdx.x % G;
  const int dim = int(A.dim);
  const float inv = 1.0f / float(dim);
  const Source src{A.ids, A.x_rows};
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / G;
  float w[NV][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) w[v][j] = 0.0f;
    if (c < dim) load_weight<T>(A, c, dim - c, w[v]);
  }
  Vec<T> x[NV], r[NV];
  auto load = [&](int64_t row, int64_t at) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      if (c < dim) {
        load_x<T>(A.x, A.x_stride, at, c, dim - c, x[v]);
        if (A.residual)
          r[v].template load<Move::kStreamed>(
              static_cast<const T *>(A.residual) + row * A.residual_stride + c, dim - c);
      }
    }
  };
  int64_t next_at = i + step < A.rows ? src.at(i + step) : 0;
  if (i < A.rows) load(i, src.at(i));
  // (a group of 64 lanes or fewer leaves on its own; a larger one is the block)
  for (; i < A.rows; i += step) {
    T *const y = static_cast<T *>(A.y) + i * A.y_stride;
    uint8_t *const y8 = static_cast<uint8_t *>(A.y) + i * A.y_stride;
    float h[NV][V];
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool in = (v * G + lane) * V < dim;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[v][j] = in ? float(x[v].e[j]) : 0.0f;
        if (A.residual && in) h[v][j] += float(r[v].e[j]);
        ss += h[v][j] * h[v][j];
      }
    }
    if (i + step < A.rows) {
      load(i + step, next_at);
      next_at = i + 2 * step < A.rows ? src.at(i + 2 * step) : 0;
    }
    if (A.sum) {
      T *const sum = static_cast<T *>(A.sum) + i * A.sum_stride;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        if (c < dim) store_row<T>(sum + c, h[v], dim - c);
      }
    }
    const float s = rsqrtf(grp.sum(ss) * inv + A.eps);
    uint32_t amax = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[v][j] = h[v][j] * s * w[v][j];
        if (E4M3 && c + j < dim) amax = max(amax, mag(h[v][j]));
      }
      if (!E4M3 && c < dim) store_row<T>(y + c, h[v], dim - c);
    }
    if (E4M3) {
      const float sc = scale_of(grp.max(amax));
      const float f = 1.0f / sc;
      if (lane == 0) A.scale[i] = sc;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        if (c < dim) {
#pragma unroll
          for (int j = 0; j < V; ++j) h[v][j] *= f;
          store_e4m3<V>(y8 + c, h[v], dim - c);
        }
      }
    }
  }
}

// Rows that do not fit in a block's registers: a block reads its row twice (three
// times for an 8-bit output).
template <typename T, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_rms_norm_long(hg_norm_args A) {
  constexpr int V = kVec<T>;
  __shared__ float red[Group<kBlock>::kLds];
  Group<kBlock> grp(red);
  // (counted without a sign: near the end of the longest rows a step passes 2^31)
  const uint32_t dim = uint32_t(A.dim);
  for (int64_t i = blockIdx.x; i < A.rows; i += gridDim.x) {
    const int64_t at = Source{A.ids, A.x_rows}.at(i);
    auto load_h = [&](uint32_t c, float *h) {
      Vec<T> t;
      load_x<T, Move::kCached>(A.x, A.x_stride, at, c, dim - c, t);
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = float(t.e[j]);
      if (A.residual) {
        t.load(static_cast<const T *>(A.residual) + i * A.residual_stride + c, dim - c);
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] += float(t.e[j]);
      }
    };
    float ss = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      float h[V];
      load_h(c, h);
#pragma unroll
      for (int j = 0; j < V; ++j) ss += h[j] * h[j];
    }
    const float s = rsqrtf(grp.sum(ss) / float(dim) + A.eps);
    float f = 1.0f;
    if (E4M3) {
      uint32_t amax = 0;
      for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
        float h[V], w[V];
        load_h(c, h);
        load_weight<T>(A, c, dim - c, w);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j < dim - c) amax = max(amax, mag(h[j] * s * w[j]));
      }
      const float sc = scale_of(grp.max(amax));
      f = 1.0f / sc;
      if (threadIdx.x == 0) A.scale[i] = sc;
    }
    // (a lane reads what it overwrites before it does, and no other lane's)
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      const int n = dim - c;
      float h[V], w[V];
      load_h(c, h);
      load_weight<T>(A, c, n, w);
      if (A.sum) store_row<T>(static_cast<T *>(A.sum) + i * A.sum_stride + c, h, n);
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = h[j] * s * w[j] * f;
      if (E4M3)
        store_e4m3<V>(static_cast<uint8_t *>(A.y) + i * A.y_stride + c, h, n);
      else
        store_row<T>(static_cast<T *>(A.y) + i * A.y_stride + c, h, n);
    }
  }
}

// The backward pass.  Groups walk over the rows as going forward, and keep their lanes'
// columns' parts of dweight in registers; a block adds its groups' in LDS and writes one
// part, which launch_sum_parts adds in order.  The two row sums are taken together.
template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_rms_norm_grad(hg_norm_grad_args A) {
  constexpr int V = kVec<T>;
  constexpr int kRows = Group<G>::kRows;
  __shared__ float red[Group<G>::kLds];
  __shared__ float wide[kRows > 1 ? kBlock * V : 1];
  Group<G> grp(red);
  const int lane = threadIdx.x % G;
  const int dim = int(A.dim);
  const float inv = 1.0f / float(dim);
  const Source src{A.ids, A.x_rows};
  const int64_t step = int64_t(gridDim.x) * kRows;
  hg_norm_args N{};  // the forward's view of the weight
  N.weight = A.weight;
  N.weight_dtype = A.weight_dtype;
  float dw[NV][V], w[NV][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) dw[v][j] = w[v][j] = 0.0f;
    if (c < dim) load_weight<T>(N, c, dim - c, w[v]);
  }
  Vec<T> x[NV], d[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < V; ++j) x[v].e[j] = d[v].e[j] = T(0.0f);
  auto load = [&](int64_t row, int64_t at) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      if (c < dim) {
        load_x<T>(A.x, A.x_stride, at, c, dim - c, x[v]);
        d[v].template load<Move::kStreamed>(static_cast<const T *>(A.dy) + row * A.dy_stride + c,
                                            dim - c);
      }
    }
  };
  int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / G;
  int64_t next_at = i + step < A.rows ? src.at(i + step) : 0;
  if (i < A.rows) load(i, src.at(i));
  for (; i < A.rows; i += step) {
    Vec<T> ds[NV];
    if (A.dsum && A.dx) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        if (c < dim)
          ds[v].template load<Move::kStreamed>(
              static_cast<const T *>(A.dsum) + i * A.dsum_stride + c, dim - c);
      }
    }
    float ss = 0.0f, gh = 0.0f;
    Vec<T> xc[NV], dc[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      xc[v] = x[v];
      dc[v] = d[v];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = float(xc[v].e[j]);
        ss += h * h;
        gh += float(dc[v].e[j]) * w[v][j] * h;
      }
    }
    if (i + step < A.rows) {
      load(i + step, next_at);
      next_at = i + 2 * step < A.rows ? src.at(i + 2 * step) : 0;
    }
    grp.sum(ss, gh);
    const float s = rsqrtf(ss * inv + A.eps);
    const float k = gh * inv * s * s;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = float(xc[v].e[j]), dy = float(dc[v].e[j]);
        dw[v][j] += dy * (h * s);
        o[j] = s * (dy * w[v][j] - h * k);
      }
      if (A.dx && c < dim) {
        if (A.dsum) {
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] += float(ds[v].e[j]);
        }
        store_row<T>(static_cast<T *>(A.dx) + i * A.dx_stride + c, o, dim - c);
      }
    }
  }
  if (!A.dweight) return;
  float *const part = static_cast<float *>(A.workspace) + int64_t(blockIdx.x) * dim;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
    if constexpr (kRows > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) wide[threadIdx.x * V + j] = dw[v][j];
      __syncthreads();
      if (threadIdx.x < G) {
        for (int r = 1; r < kRows; ++r)
#pragma unroll
          for (int j = 0; j < V; ++j) dw[v][j] += wide[(r * G + lane) * V + j];
      }
    }
    if ((kRows == 1 || threadIdx.x < G) && c < dim) {
      Vec<float, V> t;
#pragma unroll
      for (int j = 0; j < V; ++j) t.e[j] = dw[v][j];
      t.store(part + c, dim - c);
    }
  }
}

// The same for rows that do not fit: read twice, dweight's part kept in the workspace.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_rms_norm_grad_long(hg_norm_grad_args A) {
  constexpr int V = kVec<T>;
  __shared__ float red[Group<kBlock>::kLds];
  Group<kBlock> grp(red);
  const uint32_t dim = uint32_t(A.dim);
  const Source src{A.ids, A.x_rows};
  hg_norm_args N{};
  N.weight = A.weight;
  N.weight_dtype = A.weight_dtype;
  float *const part =
      A.dweight ? static_cast<float *>(A.workspace) + int64_t(blockIdx.x) * dim : nullptr;
  if (part)
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V)
      for (int j = 0; j < V && c + j < dim; ++j) part[c + j] = 0.0f;
  for (int64_t i = blockIdx.x; i < A.rows; i += gridDim.x) {
    const int64_t at = src.at(i);
    const T *const dy = static_cast<const T *>(A.dy) + i * A.dy_stride;
    float ss = 0.0f, gh = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      float w[V];
      Vec<T> d, x;
      d.load(dy + c, dim - c);
      load_x<T, Move::kCached>(A.x, A.x_stride, at, c, dim - c, x);
      load_weight<T>(N, c, dim - c, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = float(x.e[j]);
        ss += h * h;
        gh += float(d.e[j]) * w[j] * h;
      }
    }
    grp.sum(ss, gh);
    const float inv = 1.0f / float(dim);
    const float s = rsqrtf(ss * inv + A.eps);
    const float k = gh * inv * s * s;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      const int n = dim - c;
      float w[V], o[V];
      Vec<T> d, x;
      d.load(dy + c, n);
      load_x<T, Move::kCached>(A.x, A.x_stride, at, c, n, x);
      load_weight<T>(N, c, n, w);
      if (part)
        for (int j = 0; j < V && j < n; ++j)
          part[c + j] += float(d.e[j]) * (float(x.e[j]) * s);
      if (A.dx) {
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = s * (float(d.e[j]) * w[j] - float(x.e[j]) * k);
        if (A.dsum) {
          Vec<T> t;
          t.load(static_cast<const T *>(A.dsum) + i * A.dsum_stride + c, n);
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] += float(t.e[j]);
        }
        store_row<T>(static_cast<T *>(A.dx) + i * A.dx_stride + c, o, n);
      }
    }
  }
}

// 32 columns a block, 32 threads for each, which take turns over the parts and are
// added in LDS: a thread then has few loads that follow each other (1024 parts, 128
// columns: 4 us, where 4 threads for a column took 65).
__global__ __launch_bounds__(1024) void k_sum_parts(const float *__restrict__ part, int64_t parts,
                                                    int64_t n, float *__restrict__ out) {
  __shared__ float red[32][33];
  const int col = threadIdx.x & 31, turn = threadIdx.x >> 5;
  for (int64_t first = int64_t(blockIdx.x) * 32; first < n; first += int64_t(gridDim.x) * 32) {
    const int64_t j = first + col;
    float s = 0.0f;
    if (j < n) {
#pragma unroll 8
      for (int64_t p = turn; p < parts; p += 32) s += part[p * n + j];
    }
    if (first != int64_t(blockIdx.x) * 32) __syncthreads();  // the last columns' have been read
    red[turn][col] = s;
    __syncthreads();
    // (a wavefront now has two columns: their 32 sums, added in a fixed tree)
    const float v = lanes_sum<32>(red[threadIdx.x & 31][threadIdx.x >> 5]);
    const int64_t o = first + (threadIdx.x >> 5);
    if ((threadIdx.x & 31) == 0 && o < n) out[o] = v;
  }
}

// How a row is shared: f.template run<G, NV>().
template <typename T, typename F>
hipError_t by_dim(int64_t dim, F f) {
  const int64_t vecs = ceil_div<int64_t>(dim, kVec<T>);
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

template <typename T, bool E4M3>
struct Forward {
  const hg_norm_args &A;
  hipStream_t stream;
  template <int G, int NV>
  hipError_t run() const {
    const int64_t blocks = ceil_div<int64_t>(A.rows, Group<G>::kRows);
    if constexpr (NV == 0) {
      hipLaunchKernelGGL((k_rms_norm_long<T, E4M3>),
                         dim3(unsigned(blocks < 65536 ? blocks : 65536)), dim3(kBlock), 0, stream,
                         A);
    } else {
      hipLaunchKernelGGL((k_rms_norm<T, G, NV, E4M3>),
                         dim3(unsigned(blocks < kResident ? blocks : kResident)), dim3(kBlock), 0,
                         stream, A);
    }
    return hipGetLastError();
  }
};

template <typename T>
struct Backward {
  const hg_norm_grad_args &A;
  hipStream_t stream;
  template <int G, int NV>
  hipError_t run() const {
    const int64_t blocks = ceil_div<int64_t>(A.rows, Group<G>::kRows);
    const int64_t most = rms_norm_grad_parts(A.rows);
    const int64_t grid = blocks < most ? blocks : most;
    if constexpr (NV == 0)
      hipLaunchKernelGGL((k_rms_norm_grad_long<T>), dim3(unsigned(grid)), dim3(kBlock), 0, stream,
                         A);
    else
      hipLaunchKernelGGL((k_rms_norm_grad<T, G, NV>), dim3(unsigned(grid)), dim3(kBlock), 0,
                         stream, A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !A.dweight) return e;
    return launch_sum_parts(static_cast<const float *>(A.workspace), grid, A.dim, A.dweight,
                            stream);
  }
};

template <typename T>
hipError_t forward(const hg_norm_args &A, hipStream_t stream) {
  if (A.out_dtype == HG_DT_E4M3) return by_dim<T>(A.dim, Forward<T, true>{A, stream});
  return by_dim<T>(A.dim, Forward<T, false>{A, stream});
}

}  // namespace

hipError_t launch_sum_parts(const float *part, int64_t parts, int64_t n, float *out,
                            hipStream_t stream) {
  if (n <= 0) return hipSuccess;
  const int64_t blocks = std::min(ceil_div<int64_t>(n, 32), kMostBlocks);
  hipLaunchKernelGGL(k_sum_parts, dim3(unsigned(blocks)), dim3(1024), 0, stream, part, parts, n,
                     out);
  return hipGetLastError();
}

// Parts of dweight: blocks of the backward pass, at most.
int64_t rms_norm_grad_parts(int64_t rows) {
  return rows < kParts ? rows : kParts;
}

hipError_t launch_rms_norm(const hg_norm_args &A, hipStream_t stream) {
  if (A.rows <= 0) return hipSuccess;
  switch (A.dtype) {
    case HG_DT_F32: return forward<float>(A, stream);
    case HG_DT_F16: return forward<_Float16>(A, stream);
    default: return forward<__bf16>(A, stream);
  }
}

hipError_t launch_rms_norm_grad(const hg_norm_grad_args &A, hipStream_t stream) {
  if (A.rows <= 0) return A.dweight ? launch_sum_parts(nullptr, 0, A.dim, A.dweight, stream)
                                    : hipSuccess;
  switch (A.dtype) {
    case HG_DT_F32: return by_dim<float>(A.dim, Backward<float>{A, stream});
    case HG_DT_F16: return by_dim<_Float16>(A.dim, Backward<_Float16>{A, stream});
    default: return by_dim<__bf16>(A.dim, Backward<__bf16>{A, stream});
  }
}

}  // namespace hg
