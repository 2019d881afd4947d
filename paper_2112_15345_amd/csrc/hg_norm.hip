// Root-mean-square norm with the residual's addition, and its backward pass.
//
//   h = x + r,  s = 1 / sqrt(mean(h^2) + eps),  y = h s w
//   dx = s (g - h s^2 mean(g h)) + dsum with g = dy w,  dw = sum_i dy h s
//
// Bound by memory: a row is read once, kept in registers, reduced, and written
// once.  A group of 8 to 64 lanes, or a block, takes a row; each lane holds up to
// kMaxVecs vectors of 16 bytes of it.  Rows longer than that are read twice.
#include "hg_rows.hpp"

namespace hg {
namespace {

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
    if (c < dim) load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w[v]);
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
        load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w);
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
      load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, n, w);
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
  float dw[NV][V], w[NV][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) dw[v][j] = w[v][j] = 0.0f;
    if (c < dim) load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w[v]);
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
      load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w);
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
      load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, n, w);
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
// Columns from n1 on go to out2.
__global__ __launch_bounds__(1024) void k_sum_parts(const float *__restrict__ part, int64_t parts,
                                                    int64_t n, float *__restrict__ out, int64_t n1,
                                                    float *__restrict__ out2) {
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
    if ((threadIdx.x & 31) == 0 && o < n) (o < n1 ? out[o] : out2[o - n1]) = v;
  }
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
  return launch_sum_parts(part, parts, n, out, 0, nullptr, stream);
}
hipError_t launch_sum_parts(const float *part, int64_t parts, int64_t n1, float *out, int64_t n2,
                            float *out2, hipStream_t stream) {
  const int64_t n = n1 + n2;
  if (n <= 0) return hipSuccess;
  const int64_t blocks = std::min(ceil_div<int64_t>(n, 32), kMostBlocks);
  hipLaunchKernelGGL(k_sum_parts, dim3(unsigned(blocks)), dim3(1024), 0, stream, part, parts, n,
                     out, n1, out2);
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
