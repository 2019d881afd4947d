// Matrix products with fused epilogues on the matrix cores, and their backward
// pass.
//
//   forward   y[m, n]  = act(x w^T + bias) + residual
//   backward  dx[m, k] = dz w,  dw[n, k] = dz^T x,  dz = dy act'(pre)
//
// All three are C[i, j] = sum_q P(j, q) Q(i, q) with C row-major; an operand is
// either stored with its rows along q ("plain": x and w going forward, dz for dx) or
// with q along its rows ("turned": w for dx, dz and x for dw).  A block makes a tile
// of C from slabs of kSlab bytes along q in LDS; a wavefront makes its part with
// 16 x 16 matrix instructions whose first operand is P, so that a lane ends with 4
// neighbours of a row of C.
#include "hg_dense.hpp"
#include "hg_device.hpp"

namespace hg {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// An element of 8 bits.  Products of 8-bit rows run on the bfloat16 instructions,
// with the elements converted (exactly) on their way into LDS: the 8-bit
// instructions of gfx950 keep only some 14 bits of a group of products (measured
// against exact sums: off by up to 1.3e-4 of the terms' sizes, where the bfloat16
// ones are within 2.4e-7), which is not a sum in 32 bits.
struct F8 {
  uint8_t b;
};
template <typename S>
struct ComputeOf {
  typedef S T;
};
template <>
struct ComputeOf<F8> {
  typedef __bf16 T;
};

// 8 elements of 8 bits as bfloat16.
__device__ __forceinline__ u32x4 widen(u32x2 v) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    o[2 * h] = __builtin_bit_cast(uint32_t, bf16x2(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[h], 1.0f, false)));
    o[2 * h + 1] = __builtin_bit_cast(uint32_t, bf16x2(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[h], 1.0f, true)));
  }
  return o;
}

constexpr int kSlab = 128;       // bytes of a plain operand's row in a slab

// Elements of q in a slab.
template <typename T>
constexpr int kDepth = kSlab / int(sizeof(T));

// One step: 16 x 16 of C over a slab, from two 16-byte fragments of each operand.
// A lane holds, of row (lane & 15), the pieces lane / 16 and lane / 16 + 4 of the
// slab; which q a position stands for does not matter as long as both operands
// agree.
__device__ __forceinline__ f32x4 mma(f32x4 c, const u32x4 (&p)[2], const u32x4 (&q)[2], __bf16) {
#pragma unroll
  for (int f = 0; f < 2; ++f)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p[f]),
                                                __builtin_bit_cast(bf16x8, q[f]), c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x4 mma(f32x4 c, const u32x4 (&p)[2], const u32x4 (&q)[2], _Float16) {
#pragma unroll
  for (int f = 0; f < 2; ++f)
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p[f]),
                                               __builtin_bit_cast(f16x8, q[f]), c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x4 mma(f32x4 c, const u32x4 (&p)[2], const u32x4 (&q)[2], float) {
#pragma unroll
  for (int f = 0; f < 2; ++f)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(p[f][e]), __uint_as_float(q[f][e]),
                                               c, 0, 0, 0);
  return c;
}
// ---- operands ------------------------------------------------------------------

struct Operand {
  const void *p;
  int64_t stride;  // elements between stored rows
  int64_t rows;    // extent along C's axis
};

// Where the 16-byte piece c of stored row r of an operand's slab lies in LDS
// (B: extent of the tile along C's axis).  The pieces of a row are permuted by
// the row so that the 64 lanes that read a fragment spread over all banks.
template <typename S, bool Turned, int B>
struct Slab {
  typedef typename ComputeOf<S>::T T;
  static constexpr int kRows = Turned ? kDepth<T> : B;           // stored rows
  static constexpr int kRowBytes = Turned ? B * int(sizeof(T)) : kSlab;
  static constexpr int kRowPieces = kRowBytes / 16;
  static constexpr int kBytes = kRows * kRowBytes;
  static constexpr int kTotal = kBytes / 16;

  __device__ static __forceinline__ int piece(int r, int c) {
    if (!Turned) return r * kRowBytes + ((c ^ ((r >> 1) & 7)) << 4);
    if (sizeof(T) == 2) {
      // a fragment read takes 32 bytes of each of 16 rows (4 neighbours, 8 apart)
      const int f = kRowBytes >= 256 ? (r & 3) | (((r >> 3) & 1) << 2)
                                     : ((r >> 1) & 1) | (((r >> 3) & 1) << 1);
      return r * kRowBytes + ((((c >> 1) ^ f) << 1 | (c & 1)) << 4);
    }
    // 64 bytes of each of 4 rows, 4 apart
    return r * kRowBytes + ((((c >> 2) ^ ((r >> 2) & 3)) << 2 | (c & 3)) << 4);
  }

  // The two fragments of the 16 C-positions from `at` on.
  __device__ static __forceinline__ void fragments(const char *lds, int at, u32x4 (&f)[2]) {
    const int lane = threadIdx.x & 63;
    const int g = lane >> 4, x = lane & 15;
    if constexpr (!Turned) {
      f[0] = *reinterpret_cast<const u32x4 *>(lds + piece(at + x, g));
      f[1] = *reinterpret_cast<const u32x4 *>(lds + piece(at + x, g + 4));
    } else if constexpr (sizeof(T) == 2) {
      // position e of piece P is row 8 P + e; a transposing read gives a lane 4 rows of
      // its column from 4 x 16 elements that 16 lanes address 4 by 4
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s16x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = 8 * (g + 4 * h) + 4 * u + (x >> 2);
          const int byte = (at + (x & 3) * 4) * 2;
          const char *a = lds + piece(r, byte >> 4) + (byte & 15);
          v[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4 *)(a));
        }
        const s16x8 w = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        f[h] = __builtin_bit_cast(u32x4, w);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * (g + 4 * h) + e;
          const int byte = (at + x) * 4;
          f[h][e] = *reinterpret_cast<const uint32_t *>(lds + piece(r, byte >> 4) + (byte & 15));
        }
    }
  }

  // The elements of piece `t` of the slab that starts at q0 (q < q_end): zeros outside.
  __device__ static __forceinline__ u32x4 load(const Operand &O, int64_t c0, int64_t q0,
                                               int64_t q_end, int t) {
    constexpr int E = 16 / int(sizeof(T));  // elements of a piece
    const int r = t / kRowPieces, c = t % kRowPieces;
    const int64_t row = (Turned ? q0 : c0) + r;
    const int64_t col = (Turned ? c0 : q0) + c * E;
    const int64_t row_end = Turned ? q_end : O.rows, col_end = Turned ? O.rows : q_end;
    S e[E];
    __builtin_memset(e, 0, sizeof(e));
    if (row < row_end && col < col_end) {
      const S *p = static_cast<const S *>(O.p) + row * O.stride + col;
      if (col + E <= col_end) {
        __builtin_memcpy(e, p, sizeof(e));
      } else {
        const int n = int(col_end - col);
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (k < n) e[k] = p[k];
      }
    }
    if constexpr (sizeof(S) == 1)
      return widen(__builtin_bit_cast(u32x2, e));
    else
      return __builtin_bit_cast(u32x4, e);
  }
};

// ---- epilogue ------------------------------------------------------------------

struct Epilogue {
  void *y;  // C, row-major
  int64_t y_stride;
  int64_t rows, cols;
  int32_t dtype;  // of y, pre and residual
  int32_t bias_dtype, act;
  const void *bias;  // [cols]
  const void *residual;
  int64_t residual_stride;
  void *pre;
  int64_t pre_stride;
  const float *row_scale, *col_scale;
  float *part;  // [splits, rows, cols] sums to be joined, instead of the rest
};

__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + __expf(-v)); }

__device__ __forceinline__ float act_of(float z, int act) {
  if (act == HG_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  // z sigmoid(v); an argument of -inf gives -0, not a NaN
  if (act == HG_ACT_NONE) return z;
  const float v = act == HG_ACT_SILU ? z : 1.5957691216057308f * (z + 0.044715f * z * z * z);
  return z == -INFINITY ? -0.0f : z * sigmoid(v);
}

__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == HG_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
  if (act == HG_ACT_NONE) return 1.0f;
  const float c = 1.5957691216057308f;
  const float v = act == HG_ACT_SILU ? z : c * (z + 0.044715f * z * z * z);
  const float dv = act == HG_ACT_SILU ? 1.0f : c * (1.0f + 0.134145f * z * z);
  const float s = sigmoid(v);
  const float rest = s * (1.0f - s);
  return rest == 0.0f ? s : s + z * rest * dv;  // (0 times an infinite dv far out)
}

template <typename T, int N>
__device__ __forceinline__ void put(void *base, int64_t at, const float *v, int n) {
  Vec<T, N> t;
#pragma unroll
  for (int j = 0; j < N; ++j) t.e[j] = T(v[j]);
  t.store(static_cast<T *>(base) + at, n);
}
template <int N>
__device__ __forceinline__ void put_as(void *base, int32_t dtype, int64_t at, const float *v,
                                       int n) {
  if (dtype == HG_DT_F32)
    put<float, N>(base, at, v, n);
  else if (dtype == HG_DT_F16)
    put<_Float16, N>(base, at, v, n);
  else
    put<__bf16, N>(base, at, v, n);
}
template <typename T, int N>
__device__ __forceinline__ void get(const void *base, int64_t at, float *v, int n) {
  Vec<T, N> t;
  t.load(static_cast<const T *>(base) + at, n);
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = float(t.e[j]);
}
template <int N>
__device__ __forceinline__ void get_as(const void *base, int32_t dtype, int64_t at, float *v,
                                       int n) {
  if (dtype == HG_DT_F32)
    get<float, N>(base, at, v, n);
  else if (dtype == HG_DT_F16)
    get<_Float16, N>(base, at, v, n);
  else
    get<__bf16, N>(base, at, v, n);
}

// N neighbours v of row i from column j on, n of them in C.
template <int N>
__device__ __forceinline__ void finish(const Epilogue &E, int64_t i, int64_t j, int n, float *v) {
  if (E.col_scale) {
    const float r = E.row_scale[i];
    float s[N];
    get<float, N>(E.col_scale, j, s, n);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] *= r * s[k];
  }
  if (E.bias) {
    float b[N];
    get_as<N>(E.bias, E.bias_dtype, j, b, n);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += b[k];
  }
  if (E.pre) put_as<N>(E.pre, E.dtype, i * E.pre_stride + j, v, n);
  if (E.act != HG_ACT_NONE) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = act_of(v[k], E.act);
  }
  if (E.residual) {
    float r[N];
    get_as<N>(E.residual, E.dtype, i * E.residual_stride + j, r, n);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += r[k];
  }
  put_as<N>(E.y, E.dtype, i * E.y_stride + j, v, n);
}

// ---- the tiled product ---------------------------------------------------------

struct Product {
  Operand P, Q;      // along C's columns, along its rows
  int64_t depth;     // extent of q
  int64_t per_split; // of it per part (a multiple of the slab's)
  int32_t tiles_i, tiles_j;
  Epilogue E;
};

template <typename S, bool TP, bool TQ, int BI, int BJ>
__global__ __launch_bounds__(256) void k_product(Product A) {
  typedef typename ComputeOf<S>::T T;
  constexpr int WI = BI / 2, WJ = BJ / 2;  // a wavefront's part: four, 2 x 2
  constexpr int NI = WI / 16, NJ = WJ / 16;
  using SP = Slab<S, TP, BJ>;
  using SQ = Slab<S, TQ, BI>;
  constexpr int kStage = SP::kBytes + SQ::kBytes;
  constexpr int kOut = 4 * 16 * (WJ + 4) * 4;
  __shared__ __align__(16) char lds[kStage > kOut ? kStage : kOut];
  const int wave = threadIdx.x >> 6;
  const int lane = threadIdx.x & 63;
  const int64_t tile = blockIdx.x;
  const int64_t j0 = (tile % A.tiles_j) * BJ, i0 = (tile / A.tiles_j) * BI;
  const int64_t q_begin = int64_t(blockIdx.y) * A.per_split;
  const int64_t q_end = min(A.depth, q_begin + A.per_split);
  const int wi = (wave >> 1) * WI, wj = (wave & 1) * WJ;

  f32x4 acc[NI][NJ];
#pragma unroll
  for (int a = 0; a < NI; ++a)
#pragma unroll
    for (int b = 0; b < NJ; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  constexpr int LP = SP::kTotal / 256, LQ = SQ::kTotal / 256;
  for (int64_t q = q_begin; q < q_end; q += kDepth<T>) {
    u32x4 vp[LP], vq[LQ];
#pragma unroll
    for (int u = 0; u < LP; ++u) vp[u] = SP::load(A.P, j0, q, q_end, u * 256 + threadIdx.x);
#pragma unroll
    for (int u = 0; u < LQ; ++u) vq[u] = SQ::load(A.Q, i0, q, q_end, u * 256 + threadIdx.x);
    __syncthreads();  // the last slab has been read
#pragma unroll
    for (int u = 0; u < LP; ++u) {
      const int t = u * 256 + threadIdx.x;
      *reinterpret_cast<u32x4 *>(lds + SP::piece(t / SP::kRowPieces, t % SP::kRowPieces)) = vp[u];
    }
#pragma unroll
    for (int u = 0; u < LQ; ++u) {
      const int t = u * 256 + threadIdx.x;
      *reinterpret_cast<u32x4 *>(lds + SP::kBytes +
                                 SQ::piece(t / SQ::kRowPieces, t % SQ::kRowPieces)) = vq[u];
    }
    __syncthreads();
    u32x4 fp[NJ][2], fq[NI][2];
#pragma unroll
    for (int b = 0; b < NJ; ++b) SP::fragments(lds, wj + 16 * b, fp[b]);
#pragma unroll
    for (int a = 0; a < NI; ++a) SQ::fragments(lds + SP::kBytes, wi + 16 * a, fq[a]);
#pragma unroll
    for (int a = 0; a < NI; ++a)
#pragma unroll
      for (int b = 0; b < NJ; ++b) acc[a][b] = mma(acc[a][b], fp[b], fq[a], T());
  }

  // 16 rows at a time through LDS: a lane's 4 neighbours in, 8 neighbours out, so that
  // whole rows of the part are read and written together
  __syncthreads();
  constexpr int LD = WJ + 4;  // floats; the 4 spread the rows over the banks
  float *const out = reinterpret_cast<float *>(lds) + wave * 16 * LD;
#pragma unroll
  for (int a = 0; a < NI; ++a) {
#pragma unroll
    for (int b = 0; b < NJ; ++b)
      *reinterpret_cast<f32x4 *>(out + (lane & 15) * LD + 16 * b + 4 * (lane >> 4)) = acc[a][b];
    wave_sync();
#pragma unroll
    for (int u = 0; u < 16 * WJ / 8 / 64; ++u) {
      const int t = u * 64 + lane;
      const int r = t / (WJ / 8), c = t % (WJ / 8) * 8;
      const int64_t i = i0 + wi + 16 * a + r, j = j0 + wj + c;
      if (i < A.E.rows && j < A.E.cols) {
        float v[8];
        *reinterpret_cast<f32x4 *>(v) = *reinterpret_cast<const f32x4 *>(out + r * LD + c);
        *reinterpret_cast<f32x4 *>(v + 4) = *reinterpret_cast<const f32x4 *>(out + r * LD + c + 4);
        const int n = int(min<int64_t>(8, A.E.cols - j));
        if (A.E.part)
          put<float, 8>(A.E.part, (int64_t(blockIdx.y) * A.E.rows + i) * A.E.cols + j, v, n);
        else
          finish<8>(A.E, i, j, n, v);
      }
    }
    wave_sync();
  }
}

// Adds the parts of a product in order, then the epilogue.
__global__ __launch_bounds__(256) void k_join(Epilogue E, int32_t splits) {
  const int64_t per_row = (E.cols + 7) / 8;
  const int64_t t = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (t >= E.rows * per_row) return;
  const int64_t i = t / per_row, j = t % per_row * 8;
  const int n = int(min<int64_t>(8, E.cols - j));
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int s = 0; s < splits; ++s) {
    float a[8];
    get<float, 8>(E.part, (s * E.rows + i) * E.cols + j, a, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += a[k];
  }
  finish<8>(E, i, j, n, v);
}

// ---- dz and its column sums ------------------------------------------------------

constexpr int kSumRows = 256;  // rows of C that one part of the column sums covers

// dz = dy act'(pre) in T (dz NULL: not written), and the sums over the block's rows.
// A wavefront takes 64 vectors of 8 columns; the block's four take turns over the rows.
// Block b: columns b % strips, rows b / strips.
template <typename T>
__global__ __launch_bounds__(256) void k_dz(const T *dy, int64_t dy_stride, const T *pre,
                                            int64_t pre_stride, int32_t act, int64_t m, int64_t n,
                                            int64_t strips, T *dz, float *part) {
  __shared__ float red[4][64 * 8 + 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t strip = blockIdx.x % strips, chunk = blockIdx.x / strips;
  const int64_t j = (strip * 64 + lane) * 8;
  const int64_t r0 = chunk * kSumRows, r1 = min(m, r0 + kSumRows);
  const int left = int(min<int64_t>(8, n - j));
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (left > 0)
    for (int64_t i = r0 + wave; i < r1; i += 4) {
      float v[8];
      get<T, 8>(dy, i * dy_stride + j, v, left);
      if (pre) {
        float z[8];
        get<T, 8>(pre, i * pre_stride + j, z, left);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= act_slope(z[k], act);
      }
      if (dz) put<T, 8>(dz, i * n + j, v, left);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += v[k];
    }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) red[wave][lane * 8 + k] = s[k];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += 256) {
    const int64_t col = strip * 512 + c;
    if (col < n)
      part[chunk * n + col] = red[0][c] + red[1][c] + red[2][c] + red[3][c];
  }
}

// ---- launches --------------------------------------------------------------------

constexpr int kTile = 128;

int64_t align16(int64_t b) { return (b + 15) / 16 * 16; }
int64_t size_of(int32_t dtype) {
  return dtype == HG_DT_F32 ? 4 : (dtype == HG_DT_E4M3 ? 1 : 2);
}
int64_t depth_of(int32_t dtype) { return kSlab / (dtype == HG_DT_F32 ? 4 : 2); }

// Into how many parts the depth is cut: enough for two blocks on each of 256 compute
// units, each of at least 8 slabs.
int64_t splits_of(int64_t tiles, int64_t depth, int64_t slab) {
  const int64_t want = tiles < 512 ? 512 / tiles : 1;
  const int64_t most = depth / (8 * slab);
  const int64_t s = want < most ? want : most;
  return s < 1 ? 1 : (s > 256 ? 256 : s);
}
int64_t splits_for(int64_t rows, int64_t cols, int64_t depth, int64_t slab) {
  if (rows <= 0 || cols <= 0) return 1;
  return splits_of(ceil_div<int64_t>(rows, kTile) * ceil_div<int64_t>(cols, kTile), depth, slab);
}

template <typename S, bool TP, bool TQ>
hipError_t product(Operand P, Operand Q, int64_t depth, Epilogue E, float *parts,
                   hipStream_t stream) {
  if (E.rows <= 0 || E.cols <= 0) return hipSuccess;
  Product A{};
  A.P = P;
  A.Q = Q;
  A.depth = depth;
  A.E = E;
  const int64_t ti = ceil_div<int64_t>(E.rows, kTile), tj = ceil_div<int64_t>(E.cols, kTile);
  if (ti * tj >= (int64_t(1) << 31)) return hipErrorInvalidConfiguration;
  A.tiles_i = int32_t(ti);
  A.tiles_j = int32_t(tj);
  const int64_t slab = kDepth<typename ComputeOf<S>::T>;
  int64_t splits = parts ? splits_for(E.rows, E.cols, depth, slab) : 1;
  A.per_split = ceil_div<int64_t>(ceil_div<int64_t>(depth, slab), splits) * slab;
  if (A.per_split < slab) A.per_split = slab;
  splits = depth > 0 ? ceil_div<int64_t>(depth, A.per_split) : 1;
  if (splits > 1) A.E.part = parts;
  hipLaunchKernelGGL((k_product<S, TP, TQ, kTile, kTile>), dim3(unsigned(ti * tj), unsigned(splits)),
                     dim3(256), 0, stream, A);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const int64_t threads = E.rows * ceil_div<int64_t>(E.cols, 8);
  hipLaunchKernelGGL(k_join, dim3(unsigned(ceil_div<int64_t>(threads, 256))), dim3(256), 0, stream,
                     A.E, int32_t(splits));
  return hipGetLastError();
}

int64_t parts_bytes(int64_t rows, int64_t cols, int64_t depth, int64_t slab) {
  const int64_t s = splits_for(rows, cols, depth, slab);
  return s > 1 ? s * rows * cols * 4 : 0;
}

template <typename T>
hipError_t linear(const hg_linear_args &A, hipStream_t stream) {
  Epilogue E{};
  E.y = A.y;
  E.y_stride = A.y_stride;
  E.rows = A.m;
  E.cols = A.n;
  E.dtype = A.out_dtype;
  E.bias = A.bias;
  E.bias_dtype = A.bias_dtype;
  E.act = A.act;
  E.residual = A.residual;
  E.residual_stride = A.residual_stride;
  E.pre = A.pre;
  E.pre_stride = A.pre_stride;
  if (A.dtype == HG_DT_E4M3) {
    E.row_scale = A.x_scale;
    E.col_scale = A.w_scale;
  }
  return product<T, false, false>(Operand{A.w, A.w_stride, A.n}, Operand{A.x, A.x_stride, A.m},
                                  A.k, E, static_cast<float *>(A.workspace), stream);
}

struct GradSpace {  // byte offsets in the workspace
  int64_t dz, sums, parts, total;
};
GradSpace grad_space(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act) {
  GradSpace g;
  const int64_t slab = depth_of(dtype);
  g.dz = 0;
  g.sums = align16(act == HG_ACT_NONE ? 0 : m * n * size_of(dtype));
  g.parts = g.sums + align16(ceil_div<int64_t>(m, kSumRows) * n * 4);
  const int64_t a = parts_bytes(m, k, n, slab), b = parts_bytes(n, k, m, slab);
  g.total = g.parts + align16(a > b ? a : b);
  return g;
}

template <typename T>
hipError_t linear_grad(const hg_linear_grad_args &A, hipStream_t stream) {
  const GradSpace g = grad_space(A.m, A.k, A.n, A.dtype, A.act);
  char *const ws = static_cast<char *>(A.workspace);
  const T *dz = static_cast<const T *>(A.dy);
  int64_t dz_stride = A.dy_stride;
  const bool has_act = A.act != HG_ACT_NONE;
  const int64_t chunks = ceil_div<int64_t>(A.m, kSumRows);
  const bool products = (A.dx || A.dw) && A.k > 0;
  if (A.m > 0 && A.n > 0 && ((has_act && products) || A.dbias)) {
    const int64_t strips = ceil_div<int64_t>(A.n, 512);
    if (strips * chunks >= (int64_t(1) << 31)) return hipErrorInvalidConfiguration;
    T *const to = has_act && products ? reinterpret_cast<T *>(ws + g.dz) : nullptr;
    float *const sums = A.dbias ? reinterpret_cast<float *>(ws + g.sums) : nullptr;
    hipLaunchKernelGGL((k_dz<T>), dim3(unsigned(strips * chunks)), dim3(256), 0, stream,
                       static_cast<const T *>(A.dy), A.dy_stride,
                       has_act ? static_cast<const T *>(A.pre) : nullptr, A.pre_stride, A.act, A.m,
                       A.n, strips, to, sums);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (to) {
      dz = to;
      dz_stride = A.n;
    }
  }
  if (A.dbias) {
    hipError_t e = launch_sum_parts(reinterpret_cast<const float *>(ws + g.sums), chunks, A.n,
                                    A.dbias, stream);
    if (e != hipSuccess) return e;
  }
  float *const parts = reinterpret_cast<float *>(ws + g.parts);
  if (A.dx) {
    Epilogue E{};
    E.y = A.dx;
    E.y_stride = A.dx_stride;
    E.rows = A.m;
    E.cols = A.k;
    E.dtype = A.dtype;
    hipError_t e = product<T, true, false>(Operand{A.w, A.w_stride, A.k},
                                           Operand{dz, dz_stride, A.m}, A.n, E, parts, stream);
    if (e != hipSuccess) return e;
  }
  if (A.dw) {
    Epilogue E{};
    E.y = A.dw;
    E.y_stride = A.dw_stride;
    E.rows = A.n;
    E.cols = A.k;
    E.dtype = A.dw_dtype;
    return product<T, true, true>(Operand{A.x, A.x_stride, A.k}, Operand{dz, dz_stride, A.n}, A.m,
                                  E, parts, stream);
  }
  return hipSuccess;
}

}  // namespace

int64_t linear_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype) {
  return parts_bytes(m, n, k, depth_of(dtype));
}

hipError_t launch_linear(const hg_linear_args &A, hipStream_t stream) {
  switch (A.dtype) {
    case HG_DT_F32: return linear<float>(A, stream);
    case HG_DT_F16: return linear<_Float16>(A, stream);
    case HG_DT_BF16: return linear<__bf16>(A, stream);
    default: return linear<F8>(A, stream);
  }
}

int64_t linear_grad_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act) {
  return grad_space(m, k, n, dtype, act).total;
}

hipError_t launch_linear_grad(const hg_linear_grad_args &A, hipStream_t stream) {
  switch (A.dtype) {
    case HG_DT_F32: return linear_grad<float>(A, stream);
    case HG_DT_F16: return linear_grad<_Float16>(A, stream);
    default: return linear_grad<__bf16>(A, stream);
  }
}

}  // namespace hg
