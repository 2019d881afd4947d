// Layer norm with the residual's addition, and its backward pass.
//
//   h = x + r,  d = h - mean(h),  s = 1 / sqrt(mean(d^2) + eps),  y = d s w + b
//   g = dy w,  n = d s,  dx = s (g - mean(g) - n mean(g n)) + dsum
//   dw = sum_i dy n,  db = sum_i dy
//
// Bound by memory.  A row is read once and kept in registers, where its mean and then the squares
// around it are summed (the sum of squares alone would lose the variance of rows far from 0), and
// written once.  A group of 8 to 64 lanes, or a block, takes a row, as in the root-mean-square
// norm; rows that do not fit in its registers are read again from the caches.  65537 x 1024 in
// bfloat16 with the residual: 95 us, 5.7 TB/s; the backward pass of 16385 x 4096 111 us, 4.8 TB/s.
#include "hg_rows.hpp"

namespace hg {
namespace {

// How a row of vecs vectors is shared: f.template run<G, NV>().  Of 65 to 128 it is a block's where
// there are at most `few` rows, of more always (us in a graph, in bfloat16 with residual, a
// wavefront's / a block's: 1024 columns, 1 row 3.6 / 2.7, 512 4.2 / 3.5, 1024 4.4 / 4.4, 2048 5.2 /
// 5.8, 8192 14.7 / 16.2; 2048 columns, 1 row 5.8 / 2.8, 1024 7.1 / 5.3, 8192 33.6 / 26.7; going
// backward 1024 columns, 1 row 7.5 / 5.4, 512 9.3 / 8.0, 8192 24.6 / 27.9, 32768 59 / 80; 2048
// columns, 1 row 11.6 / 5.6, 1024 14.5 / 12.3, 8192 59 / 37, 32768 134 / 102; in float32, 512
// columns, forward 1 row 3.3 / 2.7, 512 3.8 / 3.6, 1024 4.1 / 4.0, 2048 4.5 / 4.8, 32768 47 / 50, backward 1
// row 6.2 / 5.1, 512 7.9 / 7.1, 1024 7.5 / 9.1, 8192 18 / 22; 300 columns, 512 rows 3.7 / 3.7 and 7.7 /
// 7.2, 2048 4.4 / 5.5 and 8.8 / 10.6).
constexpr int64_t kFewForward = 1024, kFewBackward = 512;
template <typename F>
hipError_t by_rows(int64_t rows, int64_t vecs, int64_t few, F f) {
  if (vecs <= 8) return f.template run<8, 1>();
  if (vecs <= 16) return f.template run<16, 1>();
  if (vecs <= 32) return f.template run<32, 1>();
  if (vecs <= 64) return f.template run<64, 1>();
  if (vecs <= 128 && rows > few) return f.template run<64, 2>();
  if (vecs <= 256) return f.template run<256, 1>();
  if (vecs <= 512) return f.template run<256, 2>();
  if (vecs <= 1024) return f.template run<256, 4>();
  return f.template run<256, 0>();
}

// 1 / sqrt(var + eps), of ss squares around the mean: NaN where they pass float32's range, as the
// header has it (0 there would leave the bias as the row's values).
__device__ __forceinline__ float inverse_deviation(float ss, float count, float eps) {
  const float v = ss / count + eps;
  return v < INFINITY ? rsqrtf(v) : __builtin_nanf("");
}

// Four values in 8 bits; kOut is HG_DT_NONE (x's type), HG_DT_E4M3 or HG_DT_I8.
template <int kOut>
__device__ __forceinline__ uint32_t pack_8(const float *v) {
  return kOut == HG_DT_I8 ? pack_i8(v[0], v[1], v[2], v[3]) : pack_e4m3(v[0], v[1], v[2], v[3]);
}

// A row's values over its scale c (which goes to *scale), in 8 bits.  What is rounded is the float32
// quotient; it lies between the products with the neighbours of 1 / c, and so does its rounding:
// where the two agree, that is it, and only where they do not (one value in 10^5) is it divided.
// (150001 rows of 128 floats to e4m3: 29 us with the product by the reciprocal alone, which takes one
// value in 10^6 to the neighbour of its quotient's rounding; 30 so.)
template <int kOut>
struct Quotients {
  float c, below, above;
  bool zeros;  // a broken row of integers
  __device__ __forceinline__ Quotients(uint32_t amax, float *scale, bool write) {
    c = scale_of<kOut == HG_DT_I8>(amax);
    if (write) *scale = c;
    zeros = kOut == HG_DT_I8 && is_broken(amax);
    const uint32_t f = __float_as_uint(1.0f / c);  // (of an infinite scale `below` is a NaN: divided)
    below = __uint_as_float(f - 1);
    above = __uint_as_float(f + 1);
  }
  template <int V>
  __device__ __forceinline__ void store(uint8_t *p, const float *v, int n) const {
    uint32_t w[V / 4], other = 0;
#pragma unroll
    for (int k = 0; k < V; k += 4) {
      float lo[4], hi[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = v[k + j] * below;
        hi[j] = v[k + j] * above;
      }
      w[k / 4] = pack_8<kOut>(lo);
      other |= w[k / 4] ^ pack_8<kOut>(hi);
    }
    if (other) {
#pragma unroll
      for (int k = 0; k < V; k += 4) {
        float q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = v[k + j] / c;
        w[k / 4] = pack_8<kOut>(q);
      }
    }
#pragma unroll
    for (int k = 0; k < V / 4; ++k) w[k] = zeros ? 0 : w[k];
    store_words<V>(p, w, n);
  }
};

// NV vectors a lane hold the row.  Groups walk over the rows and load the next one while this one
// is reduced and written.
template <typename T, int G, int NV, int kOut>
__global__ __launch_bounds__(kBlock) void k_layer_norm(hg_layer_norm_args A) {
  constexpr int V = kVec<T>;
  constexpr int kRows = Group<G>::kRows;
  __shared__ float red[Group<G>::kLds];
  Group<G> grp(red);
  const int lane = threadIdx.x % G;
  const int dim = int(A.dim);
  // (divided by, not multiplied with its reciprocal: the mean of equal elements whose sums are exact,
  // as of up to 65536 in bfloat16, is the element)
  const float count = float(dim);
  const Source src{A.ids, A.x_rows};
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / G;
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) w[v][j] = b[v][j] = 0.0f;
    if (c < dim) {
      load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w[v]);
      load_columns<T>(A.bias, A.bias_dtype, 0.0f, c, dim - c, b[v]);
    }
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
    float h[NV][V];
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool in = (v * G + lane) * V < dim;  // (elements past the row's end are 0)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[v][j] = in ? float(x[v].e[j]) : 0.0f;
        if (A.residual && in) h[v][j] += float(r[v].e[j]);
        sum += h[v][j];
      }
    }
    if (i + step < A.rows) {
      load(i + step, next_at);
      next_at = i + 2 * step < A.rows ? src.at(i + 2 * step) : 0;
    }
    if (A.sum) {
      T *const to = static_cast<T *>(A.sum) + i * A.sum_stride;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        if (c < dim) store_row<T>(to + c, h[v], dim - c);
      }
    }
    const float mean = grp.sum(sum) / count;
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int n = dim - (v * G + lane) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[v][j] = j < n ? h[v][j] - mean : 0.0f;
        ss += h[v][j] * h[v][j];
      }
    }
    const float s = inverse_deviation(grp.sum(ss), count, A.eps);
    uint32_t amax = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[v][j] = h[v][j] * s * w[v][j] + b[v][j];
        if (kOut != HG_DT_NONE && c + j < dim) amax = max(amax, mag(h[v][j]));
      }
      if (kOut == HG_DT_NONE && c < dim)
        store_row<T>(static_cast<T *>(A.y) + i * A.y_stride + c, h[v], dim - c);
    }
    if constexpr (kOut != HG_DT_NONE) {
      const Quotients<kOut> over(grp.max(amax), A.scale + i, lane == 0);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * V;
        if (c < dim)
          over.template store<V>(static_cast<uint8_t *>(A.y) + i * A.y_stride + c, h[v], dim - c);
      }
    }
  }
}

// Rows that do not fit in a block's registers: a block reads its row three times (four for an
// 8-bit output).
template <typename T, int kOut>
__global__ __launch_bounds__(kBlock) void k_layer_norm_long(hg_layer_norm_args A) {
  constexpr int V = kVec<T>;
  __shared__ float red[Group<kBlock>::kLds];
  Group<kBlock> grp(red);
  // (counted without a sign: near the end of the longest rows a step passes 2^31)
  const uint32_t dim = uint32_t(A.dim);
  const float count = float(dim);
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
    float sum = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      float h[V];
      load_h(c, h);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += h[j];
    }
    const float mean = grp.sum(sum) / count;
    float ss = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      float h[V];
      load_h(c, h);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = uint32_t(j) < dim - c ? h[j] - mean : 0.0f;
        ss += d * d;
      }
    }
    const float s = inverse_deviation(grp.sum(ss), count, A.eps);
    auto value = [&](uint32_t c, const float *h, float *y) {
      float w[V], b[V];
      load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w);
      load_columns<T>(A.bias, A.bias_dtype, 0.0f, c, dim - c, b);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = (h[j] - mean) * s * w[j] + b[j];
    };
    uint32_t amax = 0;
    if constexpr (kOut != HG_DT_NONE) {
      for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
        float h[V], y[V];
        load_h(c, h);
        value(c, h, y);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (uint32_t(j) < dim - c) amax = max(amax, mag(y[j]));
      }
      amax = grp.max(amax);
    }
    const Quotients<kOut> over(amax, A.scale + i, kOut != HG_DT_NONE && threadIdx.x == 0);
    // (a lane reads what it overwrites before it does, and no other lane's)
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      const int n = dim - c;
      float h[V], y[V];
      load_h(c, h);
      value(c, h, y);
      if (A.sum) store_row<T>(static_cast<T *>(A.sum) + i * A.sum_stride + c, h, n);
      if constexpr (kOut != HG_DT_NONE) {
        over.template store<V>(static_cast<uint8_t *>(A.y) + i * A.y_stride + c, y, n);
      } else {
        store_row<T>(static_cast<T *>(A.y) + i * A.y_stride + c, y, n);
      }
    }
  }
}

// The parts of dweight and dbias: a block leaves one of each that is wanted, side by side.
struct Parts {
  float *w, *b;
  __device__ __forceinline__ explicit Parts(const hg_layer_norm_grad_args &A) {
    const int64_t wanted = (A.dweight != nullptr) + (A.dbias != nullptr);
    float *const at = static_cast<float *>(A.workspace) + int64_t(blockIdx.x) * wanted * A.dim;
    w = A.dweight ? at : nullptr;
    b = A.dbias ? at + (A.dweight ? A.dim : 0) : nullptr;
  }
};

// The backward pass.  Groups walk over the rows as going forward, and keep their lanes' columns'
// parts of dweight and dbias in registers; a block adds its groups' in LDS.  Two rounds of two
// sums: h and g, then d^2 and g d.
template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_layer_norm_grad(hg_layer_norm_grad_args A) {
  constexpr int V = kVec<T>;
  constexpr int kRows = Group<G>::kRows;
  __shared__ float red[Group<G>::kLds];
  __shared__ float wide[kRows > 1 ? kBlock * V : 1];
  Group<G> grp(red);
  const int lane = threadIdx.x % G;
  const int dim = int(A.dim);
  // (divided by, not multiplied with its reciprocal: the mean of equal elements whose sums are exact,
  // as of up to 65536 in bfloat16, is the element)
  const float count = float(dim);
  const Source src{A.ids, A.x_rows};
  const int64_t step = int64_t(gridDim.x) * kRows;
  float dw[NV][V], db[NV][V], w[NV][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) dw[v][j] = db[v][j] = w[v][j] = 0.0f;
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
    float sum = 0.0f, gsum = 0.0f;
    Vec<T> xc[NV], dc[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      xc[v] = x[v];
      dc[v] = d[v];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sum += float(xc[v].e[j]);
        gsum += float(dc[v].e[j]) * w[v][j];
      }
    }
    if (i + step < A.rows) {
      load(i + step, next_at);
      next_at = i + 2 * step < A.rows ? src.at(i + 2 * step) : 0;
    }
    grp.sum(sum, gsum);
    const float mean = sum / count, gmean = gsum / count;
    float ss = 0.0f, gd = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int n = dim - (v * G + lane) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float e = j < n ? float(xc[v].e[j]) - mean : 0.0f;
        ss += e * e;
        gd += float(dc[v].e[j]) * w[v][j] * e;
      }
    }
    grp.sum(ss, gd);
    const float s = inverse_deviation(ss, count, A.eps);
    const float k = gd / count * s * s;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float e = float(xc[v].e[j]) - mean, dy = float(dc[v].e[j]);
        dw[v][j] += dy * (e * s);
        db[v][j] += dy;
        o[j] = s * (dy * w[v][j] - gmean - e * k);
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
  const Parts to(A);
  const auto leave = [&](float(&part)[NV][V], float *out) {
    if (!out) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * V;
      if constexpr (kRows > 1) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) wide[threadIdx.x * V + j] = part[v][j];
        __syncthreads();
        if (threadIdx.x < G) {
          for (int r = 1; r < kRows; ++r)
#pragma unroll
            for (int j = 0; j < V; ++j) part[v][j] += wide[(r * G + lane) * V + j];
        }
      }
      if ((kRows == 1 || threadIdx.x < G) && c < dim) {
        Vec<float, V> t;
#pragma unroll
        for (int j = 0; j < V; ++j) t.e[j] = part[v][j];
        t.store(out + c, dim - c);
      }
    }
  };
  leave(dw, to.w);
  leave(db, to.b);
}

// The same for rows that do not fit: read three times, the parts kept in the workspace.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_layer_norm_grad_long(hg_layer_norm_grad_args A) {
  constexpr int V = kVec<T>;
  __shared__ float red[Group<kBlock>::kLds];
  Group<kBlock> grp(red);
  const uint32_t dim = uint32_t(A.dim);
  // (divided by, not multiplied with its reciprocal: the mean of equal elements whose sums are exact,
  // as of up to 65536 in bfloat16, is the element)
  const float count = float(dim);
  const Source src{A.ids, A.x_rows};
  const Parts to(A);
  for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V)
    for (int j = 0; j < V && uint32_t(j) < dim - c; ++j) {
      if (to.w) to.w[c + j] = 0.0f;
      if (to.b) to.b[c + j] = 0.0f;
    }
  for (int64_t i = blockIdx.x; i < A.rows; i += gridDim.x) {
    const int64_t at = src.at(i);
    const T *const dy = static_cast<const T *>(A.dy) + i * A.dy_stride;
    auto load = [&](uint32_t c, Vec<T> &x, Vec<T> &d, float *w) {
      d.load(dy + c, dim - c);
      load_x<T, Move::kCached>(A.x, A.x_stride, at, c, dim - c, x);
      load_columns<T>(A.weight, A.weight_dtype, 1.0f, c, dim - c, w);
    };
    float sum = 0.0f, gsum = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      float w[V];
      Vec<T> d, x;
      load(c, x, d, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sum += float(x.e[j]);
        gsum += uint32_t(j) < dim - c ? float(d.e[j]) * w[j] : 0.0f;
      }
    }
    grp.sum(sum, gsum);
    const float mean = sum / count, gmean = gsum / count;
    float ss = 0.0f, gd = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      float w[V];
      Vec<T> d, x;
      load(c, x, d, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (uint32_t(j) < dim - c) {
          const float e = float(x.e[j]) - mean;
          ss += e * e;
          gd += float(d.e[j]) * w[j] * e;
        }
      }
    }
    grp.sum(ss, gd);
    const float s = inverse_deviation(ss, count, A.eps);
    const float k = gd / count * s * s;
    for (uint32_t c = threadIdx.x * V; c < dim; c += kBlock * V) {
      const int n = dim - c;
      float w[V], o[V];
      Vec<T> d, x;
      load(c, x, d, w);
      for (int j = 0; j < V && j < n; ++j) {
        if (to.w) to.w[c + j] += float(d.e[j]) * ((float(x.e[j]) - mean) * s);
        if (to.b) to.b[c + j] += float(d.e[j]);
      }
      if (A.dx) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          o[j] = s * (float(d.e[j]) * w[j] - gmean - (float(x.e[j]) - mean) * k);
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

template <typename T, int kOut>
struct Forward {
  const hg_layer_norm_args &A;
  hipStream_t stream;
  template <int G, int NV>
  hipError_t run() const {
    const int64_t blocks = ceil_div<int64_t>(A.rows, Group<G>::kRows);
    if constexpr (NV == 0) {
      hipLaunchKernelGGL((k_layer_norm_long<T, kOut>),
                         dim3(unsigned(blocks < 65536 ? blocks : 65536)), dim3(kBlock), 0, stream,
                         A);
    } else {
      hipLaunchKernelGGL((k_layer_norm<T, G, NV, kOut>),
                         dim3(unsigned(blocks < kResident ? blocks : kResident)), dim3(kBlock), 0,
                         stream, A);
    }
    return hipGetLastError();
  }
};

template <typename T>
struct Backward {
  const hg_layer_norm_grad_args &A;
  hipStream_t stream;
  template <int G, int NV>
  hipError_t run() const {
    const int64_t blocks = ceil_div<int64_t>(A.rows, Group<G>::kRows);
    // (a block for each unit, then four rows for a block, before there are more parts to add)
    const int64_t most = std::min(rms_norm_grad_parts(A.rows), std::max(kUnits, A.rows / 4));
    const int64_t grid = blocks < most ? blocks : most;
    if constexpr (NV == 0)
      hipLaunchKernelGGL((k_layer_norm_grad_long<T>), dim3(unsigned(grid)), dim3(kBlock), 0, stream,
                         A);
    else
      hipLaunchKernelGGL((k_layer_norm_grad<T, G, NV>), dim3(unsigned(grid)), dim3(kBlock), 0,
                         stream, A);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : add(A, grid, stream);
  }
  // The parts' sums.
  static hipError_t add(const hg_layer_norm_grad_args &A, int64_t parts, hipStream_t stream) {
    return launch_sum_parts(static_cast<const float *>(A.workspace), parts, A.dweight ? A.dim : 0,
                            A.dweight, A.dbias ? A.dim : 0, A.dbias, stream);
  }
};

template <typename T, int kOut>
hipError_t forward(const hg_layer_norm_args &A, hipStream_t stream) {
  return by_rows(A.rows, ceil_div<int64_t>(A.dim, kVec<T>), kFewForward, Forward<T, kOut>{A, stream});
}
template <typename T>
hipError_t forward(const hg_layer_norm_args &A, hipStream_t stream) {
  if (A.out_dtype == HG_DT_E4M3) return forward<T, HG_DT_E4M3>(A, stream);
  if (A.out_dtype == HG_DT_I8) return forward<T, HG_DT_I8>(A, stream);
  return forward<T, HG_DT_NONE>(A, stream);
}

template <typename T>
hipError_t backward(const hg_layer_norm_grad_args &A, hipStream_t stream) {
  return by_rows(A.rows, ceil_div<int64_t>(A.dim, kVec<T>), kFewBackward, Backward<T>{A, stream});
}

}  // namespace

hipError_t launch_layer_norm(const hg_layer_norm_args &A, hipStream_t stream) {
  if (A.rows <= 0) return hipSuccess;
  switch (A.dtype) {
    case HG_DT_F32: return forward<float>(A, stream);
    case HG_DT_F16: return forward<_Float16>(A, stream);
    default: return forward<__bf16>(A, stream);
  }
}

hipError_t launch_layer_norm_grad(const hg_layer_norm_grad_args &A, hipStream_t stream) {
  if (A.rows <= 0) return Backward<float>::add(A, 0, stream);
  switch (A.dtype) {
    case HG_DT_F32: return backward<float>(A, stream);
    case HG_DT_F16: return backward<_Float16>(A, stream);
    default: return backward<__bf16>(A, stream);
  }
}

}  // namespace hg
