// Shared by the dense operators (hg_norm.hip, hg_linear.hip, hg_distill.hip) and
// their C entry points (hg_dense.cpp): element types, vector loads and stores,
// reductions, and the launchers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "hg.h"
#include "hg_dense_plan.hpp"
#include "hg_internal.hpp"

namespace hg {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Blocks of a launch that walks over its work, at most.  (A grid has fewer than 2^32 threads.)
constexpr int64_t kMostBlocks = int64_t(1) << 20;

// ---- launchers (all asynchronous on `stream`; arguments already checked) ----

hipError_t launch_rms_norm(const hg_norm_args &A, hipStream_t stream);
hipError_t launch_rms_norm_grad(const hg_norm_grad_args &A, hipStream_t stream);
int64_t rms_norm_grad_parts(int64_t rows);

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

// How rows are moved.  Streamed: past the caches, for what is read or written once by
// a kernel (a residual norm of 65537 x 1024 in 16 bits: 136 us with cached stores and
// loads, 89 with streamed stores; its backward pass 184, 129, and 102 with both).
enum class Move { kCached, kStreamed };

// V elements, n (>= 1) of them in memory.  Whole vectors are one access at any
// alignment of the element type (gfx950 needs none of its own).
template <typename T, int V = kVec<T>>
struct Vec {
  T e[V];
  template <typename W>
  __device__ __forceinline__ static W *as(const T *p) {
    return reinterpret_cast<W *>(const_cast<T *>(p));
  }
  // Elements past n are `rest`.
  template <Move M = Move::kCached>
  __device__ __forceinline__ void load(const T *p, int n, T rest = T(0.0f)) {
    if (n >= V) {
      if constexpr (M == Move::kStreamed && sizeof(e) % 16 == 0) {
        typedef unsigned int W __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
        for (int h = 0; h < int(sizeof(e)) / 16; ++h) {
          const W w = __builtin_nontemporal_load(as<const W>(p) + h);
          __builtin_memcpy(reinterpret_cast<char *>(e) + 16 * h, &w, 16);
        }
      } else {
        __builtin_memcpy(e, p, sizeof(e));
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = i < n ? p[i] : rest;
    }
  }
  template <Move M = Move::kCached>
  __device__ __forceinline__ void store(T *p, int n) const {
    if (n >= V) {
      if constexpr (M == Move::kStreamed && sizeof(e) % 16 == 0) {
        typedef unsigned int W __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
        for (int h = 0; h < int(sizeof(e)) / 16; ++h) {
          W w;
          __builtin_memcpy(&w, reinterpret_cast<const char *>(e) + 16 * h, 16);
          __builtin_nontemporal_store(w, as<W>(p) + h);
        }
      } else {
        __builtin_memcpy(p, e, sizeof(e));
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) p[i] = e[i];
    }
  }
};

// A 16-byte vector as it came, for values that stay in registers: as an array of small
// elements the compiler would give each a register of its own.
template <typename T, Move M>
__device__ __forceinline__ u32x4 load_raw(const T *p) {
  Vec<T> t;
  t.template load<M>(p, kVec<T>);
  return __builtin_bit_cast(u32x4, t);
}
template <typename T>
__device__ __forceinline__ void unpack(u32x4 raw, float (&f)[kVec<T>]) {
  const Vec<T> t = __builtin_bit_cast(Vec<T>, raw);
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) f[j] = float(t.e[j]);
}
template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&f)[kVec<T>]) {
  Vec<T> t;
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) t.e[j] = T(f[j]);
  return __builtin_bit_cast(u32x4, t);
}
// The same value, of which the compiler knows nothing: what follows unpacks it anew
// instead of keeping what an earlier loop unpacked.  `after` orders it behind what made
// that value, so that a loop over vectors is not spread over as many registers.
__device__ __forceinline__ u32x4 forget(u32x4 v, float &after) {
  asm volatile("" : "+v"(v), "+v"(after));
  return v;
}

__device__ __forceinline__ float load_f32(const void *p, int32_t dtype, int64_t i) {
  if (dtype == HG_DT_F32) return static_cast<const float *>(p)[i];
  if (dtype == HG_DT_F16) return float(static_cast<const _Float16 *>(p)[i]);
  return float(static_cast<const __bf16 *>(p)[i]);
}

// f over the W neighbouring lanes that share a lane's position / W (W a power of
// two; all of them active); every lane gets the result.  By data-parallel moves within
// 16 lanes and row swaps past them: no trip through LDS.
template <int W, typename F>
__device__ __forceinline__ float lanes_reduce(float v, F f) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if constexpr (W >= 2) v = f(v, dpp(v, std::integral_constant<int, 0xb1>()));    // lane ^ 1
  if constexpr (W >= 4) v = f(v, dpp(v, std::integral_constant<int, 0x4e>()));    // lane ^ 2
  if constexpr (W >= 8) v = f(v, dpp(v, std::integral_constant<int, 0x141>()));   // the other 4 of 8
  if constexpr (W >= 16) v = f(v, dpp(v, std::integral_constant<int, 0x140>()));  // the other 8 of 16
  if constexpr (W >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (W >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_reduce<W>(v, [](float a, float b) { return a + b; });
}
// The larger of two bit patterns (of magnitudes: NaN is above infinity).
template <int W>
__device__ __forceinline__ uint32_t lanes_max_bits(uint32_t v) {
  return __float_as_uint(lanes_reduce<W>(__uint_as_float(v), [](float a, float b) {
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
  }));
}

}  // namespace hg
