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

// Threads that share a row, and how to add over them.
template <int G>
struct Group {
  static constexpr int kRows = kBlock / G;  // rows of a block
  float *red;                               // LDS, for G > 64
  __device__ __forceinline__ float sum(float v) const {
    v = lanes_sum<(G < 64 ? G : 64)>(v);
    if (G > 64) {
      __syncthreads();  // red may hold an earlier reduction that is still read
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < kBlock / 64; ++i) v += red[i];
    }
    return v;
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) const {
    v = lanes_max<(G < 64 ? G : 64)>(v);
    if (G > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = __uint_as_float(v);
      __syncthreads();
      v = 0;
#pragma unroll
      for (int i = 0; i < kBlock / 64; ++i) v = ::max(v, __float_as_uint(red[i]));
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

// h of one vector of row i; bad: the id is out of range.
template <typename T>
__device__ __forceinline__ void load_h(const hg_norm_args &A, int64_t i, int64_t at, bool bad,
                                       int64_t c, int n, float *h) {
  constexpr int V = kVec<T>;
  Vec<T> t;
  if (bad) {
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = j < n ? __builtin_nanf("") : 0.0f;
  } else {
    t.load(static_cast<const T *>(A.x) + at * A.x_stride + c, n);
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = float(t.e[j]);
  }
  if (A.residual) {
    t.load(static_cast<const T *>(A.residual) + i * A.residual_stride + c, n);
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] += float(t.e[j]);
  }
}

template <typename T>
__device__ __forceinline__ void store_row(T *p, const float *v, int n) {
  Vec<T> t;
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) t.e[j] = T(v[j]);
  t.store(p, n);
}

// NV vectors a lane hold the row; NV == 0: the row is read twice instead.
template <typename T, int G, int NV, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_rms_norm(hg_norm_args A) {
  constexpr int V = kVec<T>;
  __shared__ float red[kBlock / 64];
  const Group<G> grp{red};
  const int64_t i = int64_t(blockIdx.x) * Group<G>::kRows + threadIdx.x / G;
  const int lane = threadIdx.x % G;
  if (i >= A.rows) return;  // whole groups: no block barrier follows for G <= 64, and kRows is 1 past it
  const int dim = int(A.dim);
  const int64_t at = A.ids ? A.ids[i] : i;
  const bool bad = A.ids && (at < 0 || at >= A.x_rows);
  const float inv = 1.0f / float(dim);
  T *const y = static_cast<T *>(A.y) + i * A.y_stride;
  uint8_t *const y8 = static_cast<uint8_t *>(A.y) + i * A.y_stride;
  T *const sum = A.sum ? static_cast<T *>(A.sum) + i * A.sum_stride : nullptr;
  if constexpr (NV > 0) {
    float h[NV][V];
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      const int n = dim - c;
      if (n > 0) {
        load_h<T>(A, i, at, bad, c, n, h[v]);
        if (sum) store_row<T>(sum + c, h[v], n);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) h[v][j] = 0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < V; ++j) ss += h[v][j] * h[v][j];
    const float s = rsqrtf(grp.sum(ss) * inv + A.eps);
    uint32_t amax = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      const int n = dim - c;
      if (n > 0) {
        float w[V];
        load_weight<T>(A, c, n, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          h[v][j] = h[v][j] * s * w[j];
          if (E4M3 && j < n) amax = max(amax, mag(h[v][j]));
        }
        if (!E4M3) store_row<T>(y + c, h[v], n);
      }
    }
    if (E4M3) {
      const float sc = scale_of(grp.max(amax));
      if (lane == 0) A.scale[i] = sc;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        if (c < dim) {
#pragma unroll
          for (int j = 0; j < V; ++j) h[v][j] = h[v][j] / sc;
          store_e4m3<V>(y8 + c, h[v], dim - c);
        }
      }
    }
  } else {
    float ss = 0.0f;
    for (int c = lane * V; c < dim; c += G * V) {
      float h[V];
      load_h<T>(A, i, at, bad, c, dim - c, h);
#pragma unroll
      for (int j = 0; j < V; ++j) ss += h[j] * h[j];
    }
    const float s = rsqrtf(grp.sum(ss) * inv + A.eps);
    float sc = 1.0f;
    if (E4M3) {
      uint32_t amax = 0;
      for (int c = lane * V; c < dim; c += G * V) {
        float h[V], w[V];
        load_h<T>(A, i, at, bad, c, dim - c, h);
        load_weight<T>(A, c, dim - c, w);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j < dim - c) amax = max(amax, mag(h[j] * s * w[j]));
      }
      sc = scale_of(grp.max(amax));
      if (lane == 0) A.scale[i] = sc;
    }
    // (a lane reads what it overwrites before it does, and no other lane's)
    for (int c = lane * V; c < dim; c += G * V) {
      const int n = dim - c;
      float h[V], w[V];
      load_h<T>(A, i, at, bad, c, n, h);
      load_weight<T>(A, c, n, w);
      if (sum) store_row<T>(sum + c, h, n);
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = E4M3 ? h[j] * s * w[j] / sc : h[j] * s * w[j];
      if (E4M3)
        store_e4m3<V>(y8 + c, h, n);
      else
        store_row<T>(y + c, h, n);
    }
  }
}

// The backward pass.  Every group walks over rows and keeps its lanes' columns'
// parts of dweight in registers; a block adds its groups' in LDS and writes one
// part per block, which launch_sum_parts adds in order.
template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_rms_norm_grad(hg_norm_grad_args A) {
  constexpr int V = kVec<T>;
  constexpr int kRows = Group<G>::kRows;
  __shared__ float red[kBlock / 64];
  __shared__ float wide[kRows > 1 ? kBlock * V : 1];
  const Group<G> grp{red};
  const int lane = threadIdx.x % G;
  const int dim = int(A.dim);
  const float inv = 1.0f / float(dim);
  float *const part =
      A.dweight ? static_cast<float *>(A.workspace) + int64_t(blockIdx.x) * dim : nullptr;
  hg_norm_args N{};  // the forward's view of the rows and the weight
  N.x = A.x;
  N.x_stride = A.x_stride;
  N.weight = A.weight;
  N.weight_dtype = A.weight_dtype;
  constexpr int NR = NV > 0 ? NV : 1;
  float dw[NR][V], w[NR][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) dw[v][j] = w[v][j] = 0.0f;
    if (c < dim) load_weight<T>(N, c, dim - c, w[v]);
  }
  if (NV == 0 && part)
    for (int c = lane * V; c < dim; c += G * V)
      for (int j = 0; j < V && c + j < dim; ++j) part[c + j] = 0.0f;
  for (int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / G; i < A.rows;
       i += int64_t(gridDim.x) * kRows) {
    const int64_t at = A.ids ? A.ids[i] : i;
    const bool bad = A.ids && (at < 0 || at >= A.x_rows);
    const T *const dy = static_cast<const T *>(A.dy) + i * A.dy_stride;
    const T *const ds = A.dsum ? static_cast<const T *>(A.dsum) + i * A.dsum_stride : nullptr;
    T *const dx = A.dx ? static_cast<T *>(A.dx) + i * A.dx_stride : nullptr;
    float ss = 0.0f, gh = 0.0f;
    if constexpr (NV > 0) {
      float h[NV][V];
      Vec<T> d[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        const int n = dim - c;
        if (n > 0) {
          d[v].load(dy + c, n);
          load_h<T>(N, i, at, bad, c, n, h[v]);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) h[v][j] = 0.0f, d[v].e[j] = T(0.0f);
        }
      }
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          ss += h[v][j] * h[v][j];
          gh += float(d[v].e[j]) * w[v][j] * h[v][j];
        }
      const float s = rsqrtf(grp.sum(ss) * inv + A.eps);
      const float k = grp.sum(gh) * inv * s * s;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        const int n = dim - c;
        if (n > 0) {
#pragma unroll
          for (int j = 0; j < V; ++j) dw[v][j] += float(d[v].e[j]) * (h[v][j] * s);
          if (dx) {
            float o[V];
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = s * (float(d[v].e[j]) * w[v][j] - h[v][j] * k);
            if (ds) {
              Vec<T> t;
              t.load(ds + c, n);
#pragma unroll
              for (int j = 0; j < V; ++j) o[j] += float(t.e[j]);
            }
            store_row<T>(dx + c, o, n);
          }
        }
      }
    } else {
      for (int c = lane * V; c < dim; c += G * V) {
        float h[V], wt[V];
        Vec<T> d;
        d.load(dy + c, dim - c);
        load_h<T>(N, i, at, bad, c, dim - c, h);
        load_weight<T>(N, c, dim - c, wt);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          ss += h[j] * h[j];
          gh += float(d.e[j]) * wt[j] * h[j];
        }
      }
      const float s = rsqrtf(grp.sum(ss) * inv + A.eps);
      const float k = grp.sum(gh) * inv * s * s;
      for (int c = lane * V; c < dim; c += G * V) {
        const int n = dim - c;
        float h[V], wt[V], o[V];
        Vec<T> d;
        d.load(dy + c, n);
        load_h<T>(N, i, at, bad, c, n, h);
        load_weight<T>(N, c, n, wt);
        if (part)
          for (int j = 0; j < V && j < n; ++j) part[c + j] += float(d.e[j]) * (h[j] * s);
        if (dx) {
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] = s * (float(d.e[j]) * wt[j] - h[j] * k);
          if (ds) {
            Vec<T> t;
            t.load(ds + c, n);
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] += float(t.e[j]);
          }
          store_row<T>(dx + c, o, n);
        }
      }
    }
  }
  if constexpr (NV > 0) {
    if (!part) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      if constexpr (kRows > 1) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) wide[threadIdx.x * V + j] = dw[v][j];
        __syncthreads();
        if (threadIdx.x < G && c < dim) {
          for (int r = 1; r < kRows; ++r)
#pragma unroll
            for (int j = 0; j < V; ++j) dw[v][j] += wide[(r * G + lane) * V + j];
          Vec<float, V> t;
#pragma unroll
          for (int j = 0; j < V; ++j) t.e[j] = dw[v][j];
          t.store(part + c, dim - c);
        }
      } else if (c < dim) {
        Vec<float, V> t;
#pragma unroll
        for (int j = 0; j < V; ++j) t.e[j] = dw[v][j];
        t.store(part + c, dim - c);
      }
    }
  }
}

// 64 columns a block: a wavefront reads 64 neighbours of a part, four take turns.
__global__ __launch_bounds__(256) void k_sum_parts(const float *__restrict__ part, int64_t parts,
                                                   int64_t n, float *__restrict__ out) {
  __shared__ float red[256];
  const int64_t j = int64_t(blockIdx.x) * 64 + (threadIdx.x & 63);
  float s = 0.0f;
  if (j < n)
    for (int64_t p = threadIdx.x >> 6; p < parts; p += 4) s += part[p * n + j];
  red[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 64 && j < n)
    out[j] = red[threadIdx.x] + red[threadIdx.x + 64] + red[threadIdx.x + 128] +
             red[threadIdx.x + 192];
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
    hipLaunchKernelGGL((k_rms_norm<T, G, NV, E4M3>), dim3(unsigned(blocks)), dim3(kBlock), 0,
                       stream, A);
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
    const int64_t most = A.dweight ? rms_norm_grad_parts(A.rows, A.dim) : 2048;
    const int64_t grid = blocks < most ? blocks : most;
    hipLaunchKernelGGL((k_rms_norm_grad<T, G, NV>), dim3(unsigned(grid)), dim3(kBlock), 0, stream,
                       A);
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
  hipLaunchKernelGGL(k_sum_parts, dim3(unsigned(ceil_div<int64_t>(n, 64))), dim3(256), 0, stream,
                     part, parts, n, out);
  return hipGetLastError();
}

// Parts of dweight: blocks of the backward pass, at most.
int64_t rms_norm_grad_parts(int64_t rows, int64_t dim) {
  (void)dim;
  return rows < 1024 ? rows : 1024;
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
