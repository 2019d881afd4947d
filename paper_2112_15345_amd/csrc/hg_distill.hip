// Distillation from a teacher's top logits: loss, gradient or both of a row.
//
//   p = softmax(teacher / T) over the listed classes, q = softmax(z / T) over all
//   loss = sum_j p_j (log p_j - log q_id(j)),  grad_v = a / T (q_v - sum_{id(j) = v} p_j)
//
// Bound by memory: the row of logits is read once (and its gradient written once).
// A wavefront or a block takes a row.  With a gradient the row stays in registers
// between the two sweeps (maximum and sum, then the gradient); without one, and for
// rows that do not fit, a single sweep keeps a running maximum and sum per thread.
// The listed classes' entries are written again after the sweep, from one thread
// each, so that no sum is made by atomics and each entry is rounded once.
#include "hg_dense.hpp"
#include "hg_device.hpp"

namespace hg {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

template <int G>
struct RowGroup {
  static constexpr int kBlock = G < 256 ? 256 : G;
  static constexpr int kRows = kBlock / G;
  float *red;  // LDS [G / 64]
  __device__ __forceinline__ void sync() const {
    if (G == 64)
      wave_sync();
    else
      __syncthreads();
  }
  // Over the group's threads; all get the result.
  template <typename F>
  __device__ __forceinline__ float reduce(float v, F f) const {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = f(v, __shfl_xor(v, d, 64));
    if (G > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      v = red[0];
#pragma unroll
      for (int i = 1; i < G / 64; ++i) v = f(v, red[i]);
    }
    return v;
  }
  __device__ __forceinline__ float sum(float v) const {
    return reduce(v, [](float a, float b) { return a + b; });
  }
  __device__ __forceinline__ float max(float v) const {
    return reduce(v, [](float a, float b) { return fmaxf(a, b); });
  }
};

// exp((z - m) / T), c = log2(e) / T
__device__ __forceinline__ float exp_of(float z, float m, float c) {
  return __builtin_amdgcn_exp2f((z - m) * c);
}

// NV vectors a thread hold the row; NV == 0: it is read twice (once without grad).
template <typename T, int G, int NV>
__global__ __launch_bounds__(RowGroup<G>::kBlock) void k_distill(hg_distill_args A) {
  constexpr int V = kVec<T>;
  constexpr int kRows = RowGroup<G>::kRows;
  extern __shared__ float lds[];
  __shared__ float red_all[G > 64 ? G / 64 : 1];
  const RowGroup<G> grp{red_all};
  const int sub = threadIdx.x / G;
  const int tid = threadIdx.x % G;
  const int top = A.top;
  float *const p = lds + sub * top;                      // [top] p_j, 0 where left out
  float *const zt = lds + (kRows + sub) * top;           // [top] z at id_j
  int *const id = reinterpret_cast<int *>(lds + 2 * kRows * top) + sub * top;  // [top], -1
  const int64_t i = int64_t(blockIdx.x) * kRows + sub;
  if (i >= A.rows) return;  // whole groups; with several a block there is no block barrier
  const int n = int(A.classes);
  const T *const z = static_cast<const T *>(A.logits) + i * A.logits_stride;
  T *const grad = A.grad ? static_cast<T *>(A.grad) + i * A.grad_stride : nullptr;
  const float a = A.row_weight ? A.row_weight[i] : 1.0f;
  const float inv_t = 1.0f / A.temperature;
  const float c = kLog2e * inv_t;

  // the teacher's entries
  float tm = -INFINITY, some = 0.0f, bad = 0.0f;
  for (int j = tid; j < top; j += G) {
    const int64_t v = A.ids[i * A.ids_stride + j];
    const float t = load_f32(A.teacher, A.teacher_dtype, i * A.teacher_stride + j);
    if (v < -1 || v >= n) bad = 1.0f;
    const bool in = v >= 0 && v < n && !(t == -INFINITY);
    id[j] = in ? int(v) : -1;
    p[j] = t;
    zt[j] = in ? float(z[v]) : 0.0f;
    if (in) {
      some = 1.0f;
      tm = fmaxf(tm, t);
    }
  }
  tm = grp.max(tm);
  some = grp.max(some);
  bad = grp.max(bad);
  float ts = 0.0f;
  for (int j = tid; j < top; j += G) {
    const float e = id[j] >= 0 ? exp_of(p[j], tm, c) : 0.0f;
    ts += e;
  }
  ts = grp.sum(ts);
  const bool nothing = some == 0.0f && bad == 0.0f;  // no entry left
  if (nothing || (a == 0.0f && !A.loss)) {
    if (A.loss && tid == 0) A.loss[i] = 0.0f;
    if (grad)
      for (int k = tid; k < n; k += G) grad[k] = T(0.0f);
    return;
  }

  // the student's maximum and sum
  float m = -INFINITY, s = 0.0f;
  Vec<T> r[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int k = (v * G + tid) * V;
      if (k < n) r[v].load(z + k, n - k);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int k = (v * G + tid) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (k + j < n) m = fmaxf(m, float(r[v].e[j]));
    }
    m = grp.max(m);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int k = (v * G + tid) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (k + j < n) s += exp_of(float(r[v].e[j]), m, c);
    }
  } else {
    for (int k = tid * V; k < n; k += G * V) {
      Vec<T> q;
      q.load(z + k, n - k);
      float f[V], mk = m;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        f[j] = k + j < n ? float(q.e[j]) : -INFINITY;
        mk = fmaxf(mk, f[j]);
      }
      float add = 0.0f;
      if (mk != -INFINITY) {
#pragma unroll
        for (int j = 0; j < V; ++j) add += exp_of(f[j], mk, c);
        s = (m == -INFINITY ? 0.0f : s * exp_of(m, mk, c)) + add;
        m = mk;
      } else {
        // only -inf so far, or NaN beside them, which has to reach the sum
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (f[j] != f[j]) s = f[j];
      }
    }
    const float all = grp.max(m);
    // (a thread that saw only -inf adds nothing, or its NaN)
    s = m == -INFINITY ? (s != s ? s : 0.0f) : s * exp_of(m, all, c);
    m = all;
  }
  s = grp.sum(s);
  if (m == -INFINITY || bad != 0.0f || ts != ts) s = __builtin_nanf("");

  const float ln_s = logf(s), ln_ts = logf(ts);
  float loss = 0.0f;
  for (int j = tid; j < top; j += G) {
    const float t = p[j];
    if (id[j] >= 0) {
      const float pj = exp_of(t, tm, c) / ts;
      const float lp = (t - tm) * inv_t - ln_ts;
      const float lq = (zt[j] - m) * inv_t - ln_s;
      p[j] = pj;
      if (!(pj == 0.0f)) loss += pj * (lp - lq);
    } else {
      p[j] = 0.0f;
    }
  }
  if (A.loss) {
    loss = grp.sum(loss);
    if (tid == 0) A.loss[i] = s != s ? s : loss;
  }
  if (!grad) return;

  const float f = a * inv_t / s;
  if (a == 0.0f) {
    for (int k = tid; k < n; k += G) grad[k] = T(0.0f);
    return;
  }
  if constexpr (NV > 0) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int k = (v * G + tid) * V;
      if (k < n) {
#pragma unroll
        for (int j = 0; j < V; ++j) r[v].e[j] = T(f * exp_of(float(r[v].e[j]), m, c));
        r[v].store(grad + k, n - k);
      }
    }
  } else {
    for (int k = tid * V; k < n; k += G * V) {
      Vec<T> q;
      q.load(z + k, n - k);
#pragma unroll
      for (int j = 0; j < V; ++j) q.e[j] = T(f * exp_of(float(q.e[j]), m, c));
      q.store(grad + k, n - k);
    }
  }
  // the listed classes, once each: p of every entry of the class off
  grp.sync();
  for (int j = tid; j < top; j += G) {
    const int v = id[j];
    if (v < 0) continue;
    float pv = 0.0f;
    bool first = true;
    for (int k = 0; k < top; ++k)
      if (id[k] == v) {
        first = first && k >= j;
        pv += p[k];
      }
    if (first) grad[v] = T(f * exp_of(zt[j], m, c) - a * inv_t * pv);
  }
}

template <typename T, int G, int NV>
hipError_t run(const hg_distill_args &A, hipStream_t stream) {
  constexpr int kRows = RowGroup<G>::kRows;
  const size_t lds = size_t(kRows) * size_t(A.top) * 12;
  hipLaunchKernelGGL((k_distill<T, G, NV>), dim3(unsigned(ceil_div<int64_t>(A.rows, kRows))),
                     dim3(RowGroup<G>::kBlock), lds, stream, A);
  return hipGetLastError();
}

template <typename T>
hipError_t by_classes(const hg_distill_args &A, hipStream_t stream) {
  const int64_t vecs = ceil_div<int64_t>(A.classes, kVec<T>);
  if (vecs <= 64) return run<T, 64, 1>(A, stream);
  if (vecs <= 256) return run<T, 64, 4>(A, stream);
  if (!A.grad) return run<T, 256, 0>(A, stream);
  if (vecs <= 1024) return run<T, 256, 4>(A, stream);
  if (vecs <= 4096) return run<T, 512, 8>(A, stream);
  if (vecs <= 8192) return run<T, 512, 16>(A, stream);
  return run<T, 1024, 0>(A, stream);
}

}  // namespace

hipError_t launch_distill(const hg_distill_args &A, hipStream_t stream) {
  if (A.rows <= 0) return hipSuccess;
  switch (A.dtype) {
    case HG_DT_F32: return by_classes<float>(A, stream);
    case HG_DT_F16: return by_classes<_Float16>(A, stream);
    default: return by_classes<__bf16>(A, stream);
  }
}

}  // namespace hg
