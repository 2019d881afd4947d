// Shared by the dense operators (hg_norm.hip, hg_linear.hip, hg_distill.hip) and
// their C entry points (hg_dense.cpp): element types, vector loads and stores,
// reductions, and the launchers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hg.h"
#include "hg_internal.hpp"

namespace hg {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
__host__ __device__ inline T ceil_div(T a, T b) {
  return (a + b - 1) / b;
}

// ---- launchers (all asynchronous on `stream`; arguments already checked) ----

hipError_t launch_rms_norm(const hg_norm_args &A, hipStream_t stream);
hipError_t launch_rms_norm_grad(const hg_norm_grad_args &A, hipStream_t stream);
int64_t rms_norm_grad_parts(int64_t rows, int64_t dim);

hipError_t launch_linear(const hg_linear_args &A, hipStream_t stream);
int64_t linear_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype);
hipError_t launch_linear_grad(const hg_linear_grad_args &A, hipStream_t stream);
int64_t linear_grad_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act);

hipError_t launch_distill(const hg_distill_args &A, hipStream_t stream);

// out[j] = sum over p < parts of part[p * n + j], in the order of p.
hipError_t launch_sum_parts(const float *part, int64_t parts, int64_t n, float *out,
                            hipStream_t stream);

// ---- device helpers ----------------------------------------------------------

// A 16-byte vector of elements and its 32-bit values.
template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

// n (1..kVec) elements from p, the rest zero.  Whole vectors are one load at any
// alignment of the element type (gfx950 loads need none of their own).
template <typename T, int V = kVec<T>>
struct Vec {
  T e[V];
  __device__ __forceinline__ void load(const T *p, int n) {
    if (n >= V) {
      __builtin_memcpy(e, p, sizeof(e));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = i < n ? p[i] : T(0.0f);
    }
  }
  __device__ __forceinline__ void store(T *p, int n) const {
    if (n >= V) {
      __builtin_memcpy(p, e, sizeof(e));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) p[i] = e[i];
    }
  }
};

__device__ __forceinline__ float load_f32(const void *p, int32_t dtype, int64_t i) {
  if (dtype == HG_DT_F32) return static_cast<const float *>(p)[i];
  if (dtype == HG_DT_F16) return float(static_cast<const _Float16 *>(p)[i]);
  return float(static_cast<const __bf16 *>(p)[i]);
}

template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int d = W / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
template <int W>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
  for (int d = W / 2; d >= 1; d >>= 1) v = max(v, uint32_t(__shfl_xor(int(v), d, 64)));
  return v;
}

}  // namespace hg
