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
#include "hg_dense_plan.hpp"
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
// An element of 8-bit integers, whose products are summed exactly in 32-bit integers (of at most
// 131071 terms of up to 2^14).  The sums stay in the registers (and the parts of a depth that is cut in
// the places) of float32 ones until they are whole, and are rounded to float32 once.
// 16384 x 4096 x 4096 with bias and residual: 261 us, 2.1e15 operations a second (2.6e15 at a depth of
// 8192 without residual; the library's product of integers alone 281 us).
struct I8 {
  int8_t b;
};
// Elements that come with scales.
template <typename S>
constexpr bool kIs8 = std::is_same_v<S, F8> || std::is_same_v<S, I8>;
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

// A slab is 64 or 128 bytes (W) of a plain operand's row deep: 1 or 2 fragments (W / 64).
// Elements of q in it:
template <typename T, int W>
constexpr int kDepth = W / int(sizeof(T));

// One step: 16 x 16 of C over a 16-byte fragment of each operand.  A lane holds, of row
// (lane & 15), piece lane / 16 (for a slab's second fragment 4 more); which q a position
// stands for does not matter as long as both operands agree.
__device__ __forceinline__ f32x4 mma(f32x4 c, u32x4 p, u32x4 q, __bf16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                 __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 c, u32x4 p, u32x4 q, _Float16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p),
                                                __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 c, u32x4 p, u32x4 q, float) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(p[e]), __uint_as_float(q[e]), c, 0, 0,
                                             0);
  return c;
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 mma(f32x4 c, u32x4 p, u32x4 q, I8) {
  return __builtin_bit_cast(
      f32x4, __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, p),
                                                   __builtin_bit_cast(i32x4, q),
                                                   __builtin_bit_cast(i32x4, c), 0, 0, 0));
}
// Whether sums are integers, held as the bits of float32 values.
template <typename S>
constexpr bool kWhole = std::is_same_v<S, I8>;
// N such sums as float32 values.  (Where they are taken from LDS: a loop over the sums in registers,
// empty for other types, had the compiler spill those of 256 x 256 and 256 x 128 tiles in 16 bits and
// e4m3: the 8-bit batch of 16384 x 4096 x 4096 817 us, 417 so; 65537 x 512 x 1024 with gelu 234, 134.)
template <int N>
__device__ __forceinline__ void rounded(float *v) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = float(__float_as_int(v[k]));
}
// The sum of two sums.
template <bool kInt>
__device__ __forceinline__ float added(float a, float b) {
  return kInt ? __int_as_float(__float_as_int(a) + __float_as_int(b)) : a + b;
}

struct Plain32 {};

// Fragments as the matrix instructions take them, kPer of them at a time.
template <typename S>
struct Step {
  static constexpr int kPer = 1;
  u32x4 v;
  __device__ __forceinline__ Step() {}
  __device__ __forceinline__ explicit Step(const u32x4 *f) : v(f[0]) {}
  __device__ __forceinline__ f32x4 mma(const Step &q, f32x4 c) const {
    return hg::mma(c, v, q.v, S());
  }
};
template <>
struct Step<F8> {  // 16 elements: two steps of bfloat16
  static constexpr int kPer = 1;
  u32x4 v[2];
  __device__ __forceinline__ Step() {}
  __device__ __forceinline__ explicit Step(const u32x4 *f)
      : v{widen(u32x2{f[0][0], f[0][1]}), widen(u32x2{f[0][2], f[0][3]})} {}
  __device__ __forceinline__ f32x4 mma(const Step &q, f32x4 c) const {
    c = hg::mma(c, v[0], q.v[0], __bf16());
    return hg::mma(c, v[1], q.v[1], __bf16());
  }
};
// 32-bit elements as three bfloat16 that add up to them exactly, x = h + m + l with h rounded
// to nearest, |m| <= 2^-9 |x| and |l| <= 2^-16 |x|: six products of theirs give the product
// of two elements within 2^-24 of its size (m l, l m and l l are left out), and the 16-bit
// instructions are 16 times as fast as the 32-bit ones (16385 x 1024 x 4096: 771 us, by the
// 32-bit instructions 1303).  The pieces are made by integer operations: the conversion
// instruction is slower than the products it feeds (881 us with it).
// A result that is finite is one whose terms all were.  Infinities, NaN, values that round past
// the largest bfloat16 and products of pieces that pass the largest float32 (of either sign, also
// where the whole product stays below it) end in an infinity or a NaN: the caller makes those
// results again by the 32-bit instructions, and keeps the others.
template <>
struct Step<float> {
  static constexpr int kPer = 2;
  u32x4 h, m, l;
  __device__ __forceinline__ Step() {}
  __device__ __forceinline__ explicit Step(const u32x4 *f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // two elements to a register of each piece
      const uint32_t x = f[e / 2][e % 2 * 2], y = f[e / 2][e % 2 * 2 + 1];
      const uint32_t hx = (x + 0x8000u) & 0xffff0000u, hy = (y + 0x8000u) & 0xffff0000u;
      const float rx = __uint_as_float(x) - __uint_as_float(hx);
      const float ry = __uint_as_float(y) - __uint_as_float(hy);
      const uint32_t mx = __float_as_uint(rx) & 0xffff0000u, my = __float_as_uint(ry) & 0xffff0000u;
      h[e] = upper(hx, hy);
      m[e] = upper(__float_as_uint(rx), __float_as_uint(ry));
      l[e] = upper(__float_as_uint(rx - __uint_as_float(mx)),
                   __float_as_uint(ry - __uint_as_float(my)));
    }
  }
  // The upper halves of two values, as two bfloat16.
  __device__ __forceinline__ static uint32_t upper(uint32_t x, uint32_t y) {
    return __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
};
// 32-bit elements by the 32-bit instructions: 64 x 64 tiles, where latency counts, and results that
// the pieces do not give.
template <>
struct Step<Plain32> {
  static constexpr int kPer = 1;
  u32x4 v;
  __device__ __forceinline__ Step() {}
  __device__ __forceinline__ explicit Step(const u32x4 *f) : v(f[0]) {}
  __device__ __forceinline__ f32x4 mma(const Step &q, f32x4 c) const {
    return hg::mma(c, v, q.v, float());
  }
};

// One row of 16 x 16 parts.  (Pieces: product by product over the row, since an
// instruction that adds to what the last one has not finished waits for it.)
template <typename St, int NJ>
__device__ __forceinline__ void mma_row(const St (&p)[NJ], const St &q, f32x4 (&c)[NJ]) {
  if constexpr (St::kPer == 2) {
    const auto all = [&](u32x4 St::*a, u32x4 b) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) c[j] = mma(c[j], p[j].*a, b, __bf16());
    };
    all(&St::l, q.h);
    all(&St::h, q.l);
    all(&St::m, q.m);
    all(&St::m, q.h);
    all(&St::h, q.m);
    all(&St::h, q.h);
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j) c[j] = p[j].mma(q, c[j]);
  }
}

// ---- operands ------------------------------------------------------------------

struct Operand {
  const void *p;
  int64_t stride;  // elements between stored rows
  int64_t rows;    // extent along C's axis
  bool padded = false;  // rows of whole 16-byte pieces, the last one's rest zeros
};

// Where the 16-byte piece c of stored row r of an operand's slab lies in LDS
// (B: extent of the tile along C's axis).  The pieces of a row are permuted by
// the row so that the 64 lanes that read a fragment spread over all banks.
// T: the elements as they are in LDS.
template <typename T, bool Turned, int B, int W>
struct Slab {
  static constexpr int kFrags = W / 64;
  static constexpr int kRows = Turned ? kDepth<T, W> : B;        // stored rows
  static constexpr int kRowBytes = Turned ? B * int(sizeof(T)) : W;
  static constexpr int kRowPieces = kRowBytes / 16;
  static constexpr int kBytes = kRows * kRowBytes;
  static constexpr int kTotal = kBytes / 16;

  __device__ static __forceinline__ int piece(int r, int c) {
    if (!Turned) return r * kRowBytes + ((c ^ (W == 128 ? (r >> 1) & 7 : (r >> 2) & 3)) << 4);
    if (sizeof(T) == 2) {
      // a fragment read takes 32 bytes of each of 16 rows (4 neighbours, 8 apart)
      const int f = kRowBytes >= 256 ? (r & 3) | (((r >> 3) & 1) << 2)
                                     : ((r >> 1) & 1) | (((r >> 3) & 1) << 1);
      return r * kRowBytes + ((((c >> 1) ^ f) << 1 | (c & 1)) << 4);
    }
    // 64 bytes of each of 4 rows, 4 apart
    return r * kRowBytes + ((((c >> 2) ^ ((r >> 2) & 3)) << 2 | (c & 3)) << 4);
  }

  // The fragments of the 16 C-positions from `at` on.
  __device__ static __forceinline__ void fragments(const char *lds, int at, u32x4 (&f)[kFrags]) {
    const int lane = threadIdx.x & 63;
    const int g = lane >> 4, x = lane & 15;
    if constexpr (!Turned) {
#pragma unroll
      for (int h = 0; h < kFrags; ++h)
        f[h] = *reinterpret_cast<const u32x4 *>(lds + piece(at + x, g + 4 * h));
    } else if constexpr (sizeof(T) == 2) {
      // position e of piece P is row 8 P + e; a transposing read gives a lane 4 rows of
      // its column from 4 x 16 elements that 16 lanes address 4 by 4
#pragma unroll
      for (int h = 0; h < kFrags; ++h) {
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
      for (int h = 0; h < kFrags; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * (g + 4 * h) + e;
          const int byte = (at + x) * 4;
          f[h][e] = *reinterpret_cast<const uint32_t *>(lds + piece(r, byte >> 4) + (byte & 15));
        }
    }
  }

};

// The elements of piece `t` of an operand's slab that starts at q0 (q < q_end), as they
// go into LDS (L: its slab): zeros outside the operand.
template <typename S, typename L, bool Turned>
__device__ __forceinline__ u32x4 load_piece(const Operand &O, int64_t c0, int64_t q0,
                                            int64_t q_end, int t) {
  constexpr int E = 16 / int(sizeof(typename ComputeOf<S>::T));  // elements of a piece
  const int r = t / L::kRowPieces, c = t % L::kRowPieces;
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
  if constexpr (std::is_same_v<S, F8>)
    return widen(__builtin_bit_cast(u32x2, e));
  else
    return __builtin_bit_cast(u32x4, e);
}

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
  float *part;  // [splits, rows, cols] sums to be joined (of integers their bits), instead of the rest
};

// (a reciprocal within 1 unit of 2^-23, where a division would cost as much as the rest)
__device__ __forceinline__ float sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __expf(-v));
}

template <int kAct>
__device__ __forceinline__ float act_of(float z) {
  if (kAct == HG_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  if (kAct == HG_ACT_NONE) return z;
  // z sigmoid(v); an argument of -inf gives -0, not a NaN
  const float v = kAct == HG_ACT_SILU ? z : 1.5957691216057308f * (z + 0.044715f * z * z * z);
  return z == -INFINITY ? -0.0f : z * sigmoid(v);
}

template <int kAct>
__device__ __forceinline__ float act_slope(float z) {
  if (kAct == HG_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
  if (kAct == HG_ACT_NONE) return 1.0f;
  const float c = 1.5957691216057308f;
  const float v = kAct == HG_ACT_SILU ? z : c * (z + 0.044715f * z * z * z);
  const float dv = kAct == HG_ACT_SILU ? 1.0f : c * (1.0f + 0.134145f * z * z);
  const float s = sigmoid(v);
  const float rest = s * (1.0f - s);
  return rest == 0.0f ? s : s + z * rest * dv;  // (0 times an infinite dv far out)
}

// f(std::integral_constant of the activation): one branch outside a loop over values.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == HG_ACT_GELU)
    f(std::integral_constant<int, HG_ACT_GELU>());
  else if (act == HG_ACT_SILU)
    f(std::integral_constant<int, HG_ACT_SILU>());
  else if (act == HG_ACT_RELU)
    f(std::integral_constant<int, HG_ACT_RELU>());
}

template <typename T, int N, Move M = Move::kCached>
__device__ __forceinline__ void put(void *base, int64_t at, const float *v, int n) {
  Vec<T, N> t;
#pragma unroll
  for (int j = 0; j < N; ++j) t.e[j] = T(v[j]);
  t.template store<M>(static_cast<T *>(base) + at, n);
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

// Scales of rows and columns: none, mild ones (the product of any two is an ordinary number), or any.
enum class Scales { kNone, kMild, kAny };
__device__ __forceinline__ bool is_mild(float s) {
  return s >= 0x1p-62f && s < 0x1p62f;
}
// The product of two scales, which alone may leave float32's range: by mantissas in [1/2, 1) and
// exponents.  (Infinities and NaN are mantissas.)
struct Factor {
  float m;
  int e;
  __device__ __forceinline__ Factor() {}
  __device__ __forceinline__ Factor(float a, float b)
      : m(__builtin_amdgcn_frexp_mantf(a) * __builtin_amdgcn_frexp_mantf(b)),
        e(__builtin_amdgcn_frexp_expf(a) + __builtin_amdgcn_frexp_expf(b)) {}
  __device__ __forceinline__ float times(float v) const { return ldexpf(v * m, e); }
};

// N columns of C, from j on, n of them in C: what is the same for every row.
template <int N>
struct Columns {
  int64_t j;
  int n;
  float bias[N], scale[N];
  __device__ __forceinline__ Columns(const Epilogue &E, int64_t at) : j(at) {
    n = int(max<int64_t>(0, min<int64_t>(N, E.cols - j)));
#pragma unroll
    for (int k = 0; k < N; ++k) bias[k] = 0.0f, scale[k] = 1.0f;
    if (n > 0 && !E.part) {
      if (E.bias) get_as<N>(E.bias, E.bias_dtype, j, bias, n);
      if (E.col_scale) get<float, N>(E.col_scale, j, scale, n);
    }
  }
};

// The scales on the columns' sums v of R rows, i and every step-th after it.
// (By mantissas and exponents for all, the 8-bit batch took 422 us, with the mild ones apart 416.)
// by_row: the rows' scales, where they have been loaded.
template <Scales kScales, int N, int R>
__device__ __forceinline__ void scale(const Epilogue &E, const Columns<N> &C, int64_t i, int step,
                                      const float *by_row, float (&v)[R][N]) {
  if constexpr (kScales != Scales::kNone) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float by = by_row ? by_row[r] : E.row_scale[min<int64_t>(i + r * step, E.rows - 1)];
#pragma unroll
      for (int k = 0; k < N; ++k)
        v[r][k] = kScales == Scales::kMild ? v[r][k] * (by * C.scale[k])
                                           : Factor(by, C.scale[k]).times(v[r][k]);
    }
  }
}

// The columns' sums v of R rows, i and every step-th after it, to the result (n > 0; O: its
// type); `residual`: the rows'.
template <typename O, bool kPlain, Scales kScales, int N, int R>
__device__ __forceinline__ void finish(const Epilogue &E, const Columns<N> &C, int64_t i, int step,
                                       const Vec<O, N> *residual, float (&v)[R][N],
                                       const float *by_row = nullptr) {
  const auto write = [&](void *to, int64_t stride) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (i + r * step < E.rows)
        put<O, N, Move::kStreamed>(to, (i + r * step) * stride + C.j, v[r], C.n);
  };
  if (kPlain) {
    write(E.y, E.y_stride);
    return;
  }
  scale<kScales>(E, C, i, step, by_row, v);
  if (E.bias) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < N; ++k) v[r][k] += C.bias[k];
  }
  if (E.pre) write(E.pre, E.pre_stride);
  with_act(E.act, [&](auto act) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < N; ++k) v[r][k] = act_of<decltype(act)::value>(v[r][k]);
  });
  if (E.residual) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < N; ++k) v[r][k] += float(residual[r].e[k]);
  }
  write(E.y, E.y_stride);
}
template <typename O, int N>
__device__ __forceinline__ void load_residual(const Epilogue &E, const Columns<N> &C, int64_t i,
                                              Vec<O, N> &r) {
  if (E.residual)
    r.template load<Move::kStreamed>(static_cast<const O *>(E.residual) + i * E.residual_stride + C.j, C.n);
}
// f(O()) with the result's type.
template <typename F>
__device__ __forceinline__ void with_type(int32_t dtype, F f) {
  if (dtype == HG_DT_F32)
    f(float());
  else if (dtype == HG_DT_F16)
    f(_Float16());
  else
    f(__bf16());
}

// ---- the tiled product ---------------------------------------------------------

struct Product {
  Operand P, Q;      // along C's columns, along its rows
  int64_t depth;     // extent of q
  int64_t per_split; // of it per part (a multiple of the slab's)
  int32_t tiles_i, tiles_j;
  Epilogue E;
};

// Block b's tile.  Blocks go to the 8 XCDs in turn; each XCD is given a run of
// neighbouring tiles, kGroup tiles high, so that the slabs that they share are read
// through one L2.
constexpr int kGroup = 8;
__device__ __forceinline__ void tile_of(const Product &A, int64_t b, int64_t &ti, int64_t &tj) {
  const int64_t n = int64_t(A.tiles_i) * A.tiles_j, even = n / kXcds * kXcds;
  int64_t t = b < even ? xcd_block(b, even, true) : b;
  const int64_t g = t / (int64_t(kGroup) * A.tiles_j);
  const int64_t first = g * kGroup, high = min<int64_t>(kGroup, A.tiles_i - first);
  t -= first * A.tiles_j;
  ti = first + t % high;
  tj = t / high;
}

// The waves' parts of C through LDS, 16 rows at a time: a lane's 4 neighbours in, 16 bytes
// of neighbours out (N of them), so that a store's lanes write whole rows of the part: with
// 8 neighbours in 32 bits, two stores to a lane's 32 bytes, the halves of lines went out by
// themselves (the gradient of 4096 x 4096 weights over 8 rows: 36 us, now 20).  A lane keeps its columns; the residual
// is loaded 16 rows ahead.
// kPlain: nothing but the sums (the gradients).  kScaled: with scales, mild ones or not.
// kInt: the sums are integers.  kDeep: how many times 16 rows of the residual are in flight.  Where the products take little time
// (kDeep > 1) the scales of all rows are loaded first, too.
template <int N, int NJ>
struct Out {
  static constexpr int WJ = NJ * 16;
  static constexpr int LD = WJ + 4;  // floats; the 4 spread the rows over the banks
  static constexpr int kAcross = WJ / N, kDown = 64 / kAcross;  // lanes of a row, rows at a time
  static constexpr int U = 16 / kDown;
  float *const out;
  const int lane, r, c;
  __device__ __forceinline__ explicit Out(char *lds)
      : out(reinterpret_cast<float *>(lds) + (threadIdx.x >> 6) * 16 * LD),
        lane(threadIdx.x & 63), r(lane / kAcross), c(lane % kAcross * N) {}
  __device__ __forceinline__ void exchange(const f32x4 (&acc)[NJ]) const {
#pragma unroll
    for (int b = 0; b < NJ; ++b)
      *reinterpret_cast<f32x4 *>(out + (lane & 15) * LD + 16 * b + 4 * (lane >> 4)) = acc[b];
    wave_sync();
  }
  __device__ __forceinline__ void take(int u, float *v) const {
#pragma unroll
    for (int h = 0; h < N; h += 4)
      *reinterpret_cast<f32x4 *>(v + h) =
          *reinterpret_cast<const f32x4 *>(out + (u * kDown + r) * LD + c + h);
  }
};
template <bool kPlain, bool kScaled, bool kInt, int kDeep, int NI, int NJ>
__device__ __forceinline__ void write_out(const Product &A, char *lds, int64_t i0, int64_t j0,
                                          const f32x4 (&acc)[NI][NJ], bool mild) {
  const Epilogue &E = A.E;
  if (E.part) {
    const Out<4, NJ> L(lds);
    const Columns<4> C(E, j0 + L.c);
#pragma unroll
    for (int a = 0; a < NI; ++a) {
      L.exchange(acc[a]);
#pragma unroll
      for (int u = 0; u < L.U; ++u) {
        const int64_t i = i0 + 16 * a + u * L.kDown + L.r;
        float v[4];
        L.take(u, v);
        if (i < E.rows && C.n > 0)
          put<float, 4>(E.part, (int64_t(blockIdx.y) * E.rows + i) * E.cols + C.j, v, C.n);
      }
      wave_sync();
    }
    return;
  }
  const auto write = [&](auto type, auto scales) {
    typedef decltype(type) O;
    constexpr int N = 16 / int(sizeof(O));
    const Out<N, NJ> L(lds);
    // two rows for one pass through the epilogue's branches (150001 x 128 x 256 in bfloat16:
    // 36 us, one row each 39)
    constexpr int R = L.U < 2 ? L.U : 2;
    const Columns<N> C(E, j0 + L.c);
    Vec<O, N> res[kDeep][L.U];
    const auto ahead = [&](int a) {
#pragma unroll
      for (int u = 0; u < L.U; ++u) {
        const int64_t i = i0 + 16 * a + u * L.kDown + L.r;
        if (!kPlain && i < E.rows && C.n > 0) load_residual(E, C, i, res[a % kDeep][u]);
      }
    };
    constexpr bool kByRow = kDeep > 1 && decltype(scales)::value != Scales::kNone;
    float by[kByRow ? NI : 1][L.U];
    if constexpr (kByRow) {
#pragma unroll
      for (int a = 0; a < NI; ++a)
#pragma unroll
        for (int u = 0; u < L.U; ++u)
          by[a][u] = E.row_scale[min<int64_t>(i0 + 16 * a + u * L.kDown + L.r, E.rows - 1)];
    }
#pragma unroll
    for (int a = 0; a < kDeep && a < NI; ++a) ahead(a);
#pragma unroll
    for (int a = 0; a < NI; ++a) {
      L.exchange(acc[a]);
      Vec<O, N> now[L.U];
#pragma unroll
      for (int u = 0; u < L.U; ++u) {
        now[u] = res[a % kDeep][u];
        if (!kPlain) {  // (waited for here, not behind these rows' stores: 133 us, 138 without
                        // in 65537 x 512 x 1024 with residual and pre)
          u32x4 raw = __builtin_bit_cast(u32x4, now[u]);
          asm volatile("" : "+v"(raw));
          now[u] = __builtin_bit_cast(Vec<O, N>, raw);
        }
      }
      if (a + kDeep < NI) ahead(a + kDeep);
#pragma unroll
      for (int u = 0; u < L.U; u += R) {
        const int64_t i = i0 + 16 * a + u * L.kDown + L.r;
        float v[R][N];
#pragma unroll
        for (int t = 0; t < R; ++t) {
          L.take(u + t, v[t]);
          if constexpr (kInt) rounded<N>(v[t]);
        }
        if (i < E.rows && C.n > 0)
          finish<O, kPlain, decltype(scales)::value>(E, C, i, L.kDown, now + u, v,
                                                     kByRow ? by[a] + u : nullptr);
      }
      wave_sync();
    }
  };
  with_type(E.dtype, [&](auto type) {
    if constexpr (!kScaled)
      write(type, std::integral_constant<Scales, Scales::kNone>());
    else if (mild)
      write(type, std::integral_constant<Scales, Scales::kMild>());
    else
      write(type, std::integral_constant<Scales, Scales::kAny>());
  });
}

// (In 256 x 256 tiles of integers it spills: 16384 x 4096 x 4096 289 us by 4, 259 by 1; 512 x 4096 x
// 4096 17.8 and 20.1, 1001 x 2064 x 4099 22.2 and 23.7.)
template <typename S, int BI>
constexpr int kAheadOut = kWhole<S> && BI < 256 ? 4 : 1;

// Whether all scales of a wavefront's part of C are mild.
template <int NI, int NJ>
__device__ __forceinline__ bool all_mild(const Epilogue &E, int64_t i0, int64_t j0) {
  const int lane = threadIdx.x & 63;
  bool mild = true;
#pragma unroll
  for (int t = 0; t < 16 * NI; t += 64)
    mild = mild && is_mild(E.row_scale[min<int64_t>(i0 + t + lane, E.rows - 1)]);
#pragma unroll
  for (int t = 0; t < 16 * NJ; t += 64)
    mild = mild && is_mild(E.col_scale[min<int64_t>(j0 + t + lane, E.cols - 1)]);
  return __all(mild);
}

// Any operands: slabs through registers.
template <typename S, bool TP, bool TQ, int BI, int BJ>
__global__ __launch_bounds__(256) void k_product(Product A) {
  typedef typename ComputeOf<S>::T T;
  constexpr int WI = BI / 2, WJ = BJ / 2;  // a wavefront's part: four, 2 x 2
  constexpr int NI = WI / 16, NJ = WJ / 16;
  constexpr bool kScaled = kIs8<S>;
  using SP = Slab<T, TP, BJ, 128>;
  using SQ = Slab<T, TQ, BI, 128>;
  constexpr int kStage = SP::kBytes + SQ::kBytes;
  constexpr int kOut = 4 * 16 * (WJ + 4) * 4;
  __shared__ __align__(16) char lds[kStage > kOut ? kStage : kOut];
  const int wave = threadIdx.x >> 6;
  int64_t ti, tj;
  tile_of(A, blockIdx.x, ti, tj);
  const int64_t i0 = ti * BI, j0 = tj * BJ;
  const int64_t q_begin = int64_t(blockIdx.y) * A.per_split;
  const int64_t q_end = min(A.depth, q_begin + A.per_split);
  const int wi = (wave >> 1) * WI, wj = (wave & 1) * WJ;

  f32x4 acc[NI][NJ];
#pragma unroll
  for (int a = 0; a < NI; ++a)
#pragma unroll
    for (int b = 0; b < NJ; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  constexpr int LP = SP::kTotal / 256, LQ = SQ::kTotal / 256;
  u32x4 vp[LP], vq[LQ];
  const auto load = [&](int64_t q) {
#pragma unroll
    for (int u = 0; u < LP; ++u)
      vp[u] = load_piece<S, SP, TP>(A.P, j0, q, q_end, u * 256 + threadIdx.x);
#pragma unroll
    for (int u = 0; u < LQ; ++u)
      vq[u] = load_piece<S, SQ, TQ>(A.Q, i0, q, q_end, u * 256 + threadIdx.x);
  };
  if (q_begin < q_end) load(q_begin);
  for (int64_t q = q_begin; q < q_end; q += kDepth<T, 128>) {
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
    if (q + kDepth<T, 128> < q_end) load(q + kDepth<T, 128>);  // in flight meanwhile
    u32x4 fp[NJ][2], fq[NI][2];
#pragma unroll
    for (int b = 0; b < NJ; ++b) SP::fragments(lds, wj + 16 * b, fp[b]);
#pragma unroll
    for (int a = 0; a < NI; ++a) SQ::fragments(lds + SP::kBytes, wi + 16 * a, fq[a]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int a = 0; a < NI; ++a)
#pragma unroll
        for (int b = 0; b < NJ; ++b) acc[a][b] = mma(acc[a][b], fp[b][h], fq[a][h], T());
  }
  __syncthreads();
  bool mild = true;
  if constexpr (kScaled) mild = all_mild<NI, NJ>(A.E, i0 + wi, j0 + wj);
  write_out<TP, kScaled, kWhole<S>, kAheadOut<S, BI>>(A, lds, i0 + wi, j0 + wj, acc, mild);
}

// 16 bytes of zeros: where lanes past an operand's end load from.
__device__ __align__(16) const uint32_t g_zeros[4] = {0, 0, 0, 0};

// A wavefront's loads of an operand's slab straight into LDS: each moves 64 pieces to
// 1024 bytes in a row, and a lane picks the piece that belongs where its 16 bytes go.
template <typename S, bool Turned, int B, int W, int kWaves>
struct Stream {
  using L = Slab<S, Turned, B, W>;
  static constexpr int E = 16 / int(sizeof(S));
  static constexpr int kLoads = L::kBytes / 1024 / kWaves;
  static_assert(L::kBytes % (1024 * kWaves) == 0, "whole loads for every wavefront");
  const S *p[kLoads];
  int r[kLoads], c[kLoads];  // the piece's stored row and its first element, in the slab
  int64_t advance;

  __device__ __forceinline__ void begin(const Operand &O, int64_t c0, int64_t q0) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    advance = Turned ? int64_t(kDepth<S, W>) * O.stride : kDepth<S, W>;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int t = (u * kWaves + wave) * 64 + lane;
      r[u] = t / L::kRowPieces;
      // (the permutation of a row's pieces is its own inverse)
      c[u] = (L::piece(r[u], t % L::kRowPieces) - r[u] * L::kRowBytes) / 16 * E;
      int64_t row = (Turned ? q0 : c0) + r[u], col = (Turned ? c0 : q0) + c[u];
      // past the end along C: results there are not written, any row will do
      if (Turned)
        col = min<int64_t>(col, O.rows - E);
      else
        row = min<int64_t>(row, O.rows - 1);
      p[u] = static_cast<const S *>(O.p) + row * O.stride + col;
    }
  }
  // Starts the loads of the next slab, of which `left` of q are in the operand.
  template <bool kWhole>
  __device__ __forceinline__ void load(char *lds, int left) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const void *from = p[u];
      if (!kWhole) from = (Turned ? r[u] : c[u]) < left ? from : g_zeros;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void *)from,
          (__attribute__((address_space(3))) void *)(lds + (u * kWaves + wave) * 1024), 16, 0, 0);
      p[u] += advance;
    }
  }
};

// Waits until at most n of this wavefront's loads are in flight, and none of its reads of LDS: a
// slab is overwritten behind the barrier that follows, and the products that use the last
// fragments need not stand before it.  (As compiled they do, and the wait costs nothing.)
template <int n>
__device__ __forceinline__ void wait_loads() {
  static_assert(n < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | (n >> 4) << 14);
}

// Aligned operands: a ring of kStages slabs in LDS, the loads of the next ones in
// flight while one is multiplied.
template <typename S, int BI, int BJ, int W, int kStages>
constexpr int kRing = (BI + BJ) * W * kStages;  // bytes of LDS
template <typename S, bool TP, bool TQ, int BI, int BJ, int kWavesI, int kWavesJ, int W,
          int kStages>
__global__ __launch_bounds__(64 * kWavesI *kWavesJ,
                             (160 * 1024 / kRing<S, BI, BJ, W, kStages>) * kWavesI *kWavesJ / 4)  //
    void k_product_direct(Product A) {
  constexpr int kWaves = kWavesI * kWavesJ;
  constexpr int WI = BI / kWavesI, WJ = BJ / kWavesJ;
  constexpr int NI = WI / 16, NJ = WJ / 16;
  constexpr bool kScaled = kIs8<S>;
  using SP = Slab<S, TP, BJ, W>;
  using SQ = Slab<S, TQ, BI, W>;
  using LP = Stream<S, TP, BJ, W, kWaves>;
  using LQ = Stream<S, TQ, BI, W, kWaves>;
  constexpr int kFrags = W / 64;
  constexpr bool kPlain32 = sizeof(S) == 4 && BI < 128;
  constexpr int kStage = SP::kBytes + SQ::kBytes;
  constexpr int kOut = kWaves * 16 * (WJ + 4) * 4;
  static_assert(kOut <= kStages * kStage, "the parts of C fit where the slabs were");
  __shared__ __align__(1024) char lds[kStages * kStage];
  const int wave = threadIdx.x >> 6;
  int64_t ti, tj;
  tile_of(A, blockIdx.x, ti, tj);
  const int64_t i0 = ti * BI, j0 = tj * BJ;
  const int64_t q_begin = int64_t(blockIdx.y) * A.per_split;
  const int64_t depth = min(A.depth - q_begin, A.per_split);
  const int whole = int(depth / kDepth<S, W>), rest = int(depth % kDepth<S, W>);
  const int slabs = whole + (rest > 0);
  const int wi = wave / kWavesJ * WI, wj = wave % kWavesJ * WJ;

  bool mild = true;  // (found out here, before there is anything to wait for)
  if constexpr (kScaled) mild = all_mild<NI, NJ>(A.E, i0 + wi, j0 + wj);
  // no part of C for this wavefront (of integers it multiplies all the same: with this branch the
  // sums were copied and spilled in the loop, 948 us for 16384 x 4096 x 4096)
  const bool idle =
      !std::is_same_v<S, I8> && (i0 + wi >= A.E.rows || j0 + wj >= A.E.cols);

  f32x4 acc[NI][NJ];
  const auto multiply_all = [&](f32x4 (&acc)[NI][NJ], auto step) {
    typedef decltype(step) St;
#pragma unroll
    for (int a = 0; a < NI; ++a)
#pragma unroll
      for (int b = 0; b < NJ; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    LP lp;
    LQ lq;
    lp.begin(A.P, j0, q_begin);
    lq.begin(A.Q, i0, q_begin);
    const auto load = [&](int slab, char *to) {
      if (slab < whole) {
        lp.template load<true>(to, 0);
        lq.template load<true>(to + SP::kBytes, 0);
      } else if (slab < slabs) {
        lp.template load<false>(to, rest);
        lq.template load<false>(to + SP::kBytes, rest);
      }
    };
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) load(u, lds + u * kStage);
    int now = 0, ahead = kStages - 1;  // places in the ring
    for (int slab = 0; slab < slabs; ++slab) {
      // this wavefront's loads of the slab have landed (those of later ones may be in flight)
      if (slab + kStages - 1 <= slabs)
        wait_loads<(kStages - 2) * (LP::kLoads + LQ::kLoads)>();
      else
        wait_loads<0>();
      // now everyone's have, and the slab that the next loads overwrite has been read
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      load(slab + kStages - 1, lds + ahead * kStage);
      const char *const at = lds + now * kStage;
      ahead = now;
      now = now + 1 == kStages ? 0 : now + 1;
      if (idle) continue;
      u32x4 fp[NJ][kFrags], fq[NI][kFrags];
#pragma unroll
      for (int b = 0; b < NJ; ++b) SP::fragments(at, wj + 16 * b, fp[b]);
#pragma unroll
      for (int a = 0; a < NI; ++a) SQ::fragments(at + SP::kBytes, wi + 16 * a, fq[a]);
#pragma unroll
      for (int h = 0; h < kFrags; h += St::kPer) {
        St tp[NJ];
#pragma unroll
        for (int b = 0; b < NJ; ++b) tp[b] = St(&fp[b][h]);
#pragma unroll
        for (int a = 0; a < NI; ++a) {
          mma_row(tp, St(&fq[a][h]), acc[a]);
        }
      }
      // (of integers all fragments are read first, whose products take half as long as others': the
      // batch of 16384 x 4096 x 4096 took 267 us as the compiler mixes them, 259 so)
      if constexpr (std::is_same_v<S, I8>) {
        __builtin_amdgcn_sched_group_barrier(0x100, kFrags * (NI + NJ), 0);
        __builtin_amdgcn_sched_group_barrier(0x008, kFrags * NI * NJ, 0);
      }
    }
  };
  multiply_all(acc, Step<std::conditional_t<kPlain32, Plain32, S>>());
  if constexpr (sizeof(S) == 4 && !kPlain32) {
    const auto finite = [](float v) { return fabsf(v) < INFINITY; };
    bool all = true;
#pragma unroll
    for (int a = 0; a < NI; ++a)
#pragma unroll
      for (int b = 0; b < NJ; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) all = all && finite(acc[a][b][e]);
    // (the barrier also says that the ring has been read)
    if (__syncthreads_or(!all)) {
      f32x4 again[NI][NJ];
      multiply_all(again, Step<Plain32>());
#pragma unroll
      for (int a = 0; a < NI; ++a)
#pragma unroll
        for (int b = 0; b < NJ; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[a][b][e] = finite(acc[a][b][e]) ? acc[a][b][e] : again[a][b][e];
    }
  }
  __syncthreads();
  write_out<TP, kScaled, kWhole<S>, kAheadOut<S, BI>>(A, lds, i0 + wi, j0 + wj, acc, mild);
}

// Adds the parts of a product in a fixed order, then the epilogue.  kShare threads share N
// neighbours of a row (16 bytes of it): each adds every kShare-th part, the first adds theirs.
// kInt: the parts are integers, whose sum is exact, too.
template <int kShare, int N, Scales kScales, bool kInt>
__global__ __launch_bounds__(256) void k_join(Epilogue E, int32_t splits) {
  constexpr int kAt = 256 / kShare;
  __shared__ float red[kShare > 1 ? kShare : 1][kShare > 1 ? kAt : 1][N + 1];
  const int64_t per_row = (E.cols + N - 1) / N;
  const int share = threadIdx.x / kAt, at = threadIdx.x % kAt;
  const int64_t t = int64_t(blockIdx.x) * kAt + at;
  const bool in = t < E.rows * per_row;
  const int64_t i = in ? t / per_row : 0, j = in ? t % per_row * N : 0;
  float *const part = E.part;
  E.part = nullptr;
  const Columns<N> C(E, j);
  float sums[1][N];
  float *const v = sums[0];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.0f;
#pragma unroll 4
  for (int s = share; s < splits; s += kShare) {
    float a[N];
    get<float, N>(part, (s * E.rows + i) * E.cols + j, a, C.n);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = added<kInt>(v[k], a[k]);
  }
  if constexpr (kShare > 1) {
#pragma unroll
    for (int k = 0; k < N; ++k) red[share][at][k] = v[k];
    __syncthreads();
    if (share) return;
    for (int s = 1; s < kShare; ++s)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = added<kInt>(v[k], red[s][at][k]);
  }
  if (!in) return;
  if constexpr (kInt) rounded<N>(v);
  scale<kScales>(E, C, i, 0, nullptr, sums);
  with_type(E.dtype, [&](auto type) {
    Vec<decltype(type), N> r;
    load_residual(E, C, i, r);
    finish<decltype(type), false, Scales::kNone>(E, C, i, 0, &r, sums);
  });
}

// ---- few rows ------------------------------------------------------------------

// Products of at most kFew rows: bound by reading w once.  A wavefront takes 16 rows of w
// (columns of C) and every kWaves-th 128 bytes of them, straight from memory into the
// matrix instructions' registers, several loads ahead; a block's wavefronts are added in
// LDS.  G: 16-row parts of x.

// 16 bytes of a row of n elements from element c on; zeros past its end.
template <typename S>
__device__ __forceinline__ u32x4 row_piece(const S *row, int64_t c, int64_t n) {
  constexpr int E = 16 / int(sizeof(S));
  u32x4 v = {0, 0, 0, 0};
  if (c + E <= n) {
    __builtin_memcpy(&v, row + c, 16);
  } else if (c < n) {
    S e[E];
    __builtin_memset(e, 0, 16);
    for (int k = 0; k < E; ++k)
      if (c + k < n) e[k] = row[c + k];
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}

template <typename S, int G, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void k_few(Product A) {
  constexpr int D = 128 / int(sizeof(S));  // elements of a step
  constexpr int U = G == 1 ? 4 : 2;        // steps in flight
  __shared__ float red[kWaves][G][16][20];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int g = lane >> 4, x = lane & 15;
  const int64_t j0 = int64_t(blockIdx.x) * 16;
  // past the end: results that are not written, any row will do
  const S *const w = static_cast<const S *>(A.P.p) + min(j0 + x, A.P.rows - 1) * A.P.stride;
  const S *rows[G];
#pragma unroll
  for (int i = 0; i < G; ++i)
    rows[i] = static_cast<const S *>(A.Q.p) + min<int64_t>(16 * i + x, A.Q.rows - 1) * A.Q.stride;
  f32x4 acc[G];
#pragma unroll
  for (int i = 0; i < G; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t q0 = int64_t(blockIdx.y) * A.per_split;
  const int64_t n = min(A.depth, q0 + A.per_split);
  const int c = g * (16 / int(sizeof(S)));  // this lane's piece of 64 bytes
  for (int64_t q = q0 + int64_t(wave) * D; q < n; q += int64_t(kWaves) * D * U) {
    u32x4 fw[U][2], fx[U][G][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t at = q + int64_t(u) * kWaves * D + h * (D / 2) + c;
        fw[u][h] = row_piece(w, at, n);
#pragma unroll
        for (int i = 0; i < G; ++i) fx[u][i][h] = row_piece(rows[i], at, n);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (sizeof(S) == 4) {  // (bound by memory: the 32-bit instructions are enough)
#pragma unroll
          for (int i = 0; i < G; ++i) acc[i] = mma(acc[i], fw[u][h], fx[u][i][h], S());
        } else {
          const Step<S> p(&fw[u][h]);
#pragma unroll
          for (int i = 0; i < G; ++i) acc[i] = p.mma(Step<S>(&fx[u][i][h]), acc[i]);
        }
      }
  }
  // 8 neighbours of a row for a thread; what they meet is loaded before the sums are there
  const int t = threadIdx.x;
  const int64_t i = t >> 1;
  const bool in = t < G * 32 && i < A.E.rows;
  const Columns<8> C(A.E, in ? j0 + (t & 1) * 8 : A.E.cols);
  Factor scales[8];
  if constexpr (kIs8<S>) {
    const float by = in ? A.E.row_scale[i] : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) scales[k] = Factor(by, C.scale[k]);
  }
#pragma unroll
  for (int u = 0; u < G; ++u)
    *reinterpret_cast<f32x4 *>(&red[wave][u][x][4 * g]) = acc[u];
  __syncthreads();
  if (C.n <= 0) return;
  float sums[1][8] = {};
  float *const v = sums[0];
  for (int s = 0; s < kWaves; ++s)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = added<kWhole<S>>(v[k], red[s][i >> 4][i & 15][(t & 1) * 8 + k]);
  if (A.E.part) {
    put<float, 8>(A.E.part, (int64_t(blockIdx.y) * A.E.rows + i) * A.E.cols + C.j, v, C.n);
    return;
  }
  if constexpr (kWhole<S>) rounded<8>(v);
  if constexpr (kIs8<S>) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = scales[k].times(v[k]);
  }
  with_type(A.E.dtype, [&](auto type) {
    Vec<decltype(type), 8> r;
    load_residual(A.E, C, i, r);
    finish<decltype(type), false, Scales::kNone>(A.E, C, i, 0, &r, sums);
  });
}

// ---- dz and its column sums ------------------------------------------------------

// dz = dy act'(pre) in T (dz NULL: not written), zeros from column n to its stride, and the
// sums over the block's rows.  In T, because the products' instructions take 16-bit operands: the
// bits that go (the error of dx and dw against 64 bits is 0.0023 for it, 0.0017 without, of their
// sizes in bfloat16) would be a second piece of dz, and twice the time of both products.
// A wavefront takes 64 vectors of 8 columns; the block's four take turns over the rows.
// Place b: columns b % strips, rows b / strips; a block takes every gridDim.x-th place.
// The values before the activation (p NULL: none), 8 of them at a time: as they were, or kept in 8 bits.
template <typename T>
struct PreRows {
  const T *p;
  int64_t stride;
  struct Eight {
    Vec<T, 8> e;
    __device__ __forceinline__ void load(const PreRows &P, int64_t i, int64_t j, int n) {
      e.template load<Move::kStreamed>(P.p + i * P.stride + j, n);
    }
    __device__ __forceinline__ float value(int k) const { return float(e.e[k]); }
  };
};
struct PreKept : Kept {
  struct Eight {
    Vec<int8_t, 8> q;
    float s;
    __device__ __forceinline__ void load(const PreKept &P, int64_t i, int64_t j, int n) {
      q.load(static_cast<const int8_t *>(P.p) + i * P.stride + j, n);
      s = P.scale_of(i, j);
    }
    __device__ __forceinline__ float value(int k) const { return float(q.e[k]) * s; }
  };
};
template <typename T, typename Pre>
__global__ __launch_bounds__(256) void k_dz(const T *dy, int64_t dy_stride, Pre pre, int32_t act,
                                            int64_t m, int64_t n,
                                            int64_t strips, int64_t places, T *dz, int64_t dz_stride,
                                            float *part) {
  __shared__ float red[4][64 * 8 + 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t b = blockIdx.x; b < places; b += gridDim.x) {
    const int64_t strip = b % strips, chunk = b / strips;
    const int64_t j = (strip * 64 + lane) * 8;
    const int64_t r0 = chunk * kSumRows, r1 = min(m, r0 + kSumRows);
    const int left = int(min<int64_t>(8, n - j)), wide = int(min<int64_t>(8, dz_stride - j));
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    constexpr int U = 4;  // rows in flight
    if (left > 0)
      for (int64_t i0 = r0 + wave; i0 < r1; i0 += 4 * U) {
        Vec<T, 8> d[U];
        typename Pre::Eight z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t i = i0 + 4 * u;
          if (i < r1) {
            d[u].template load<Move::kStreamed>(dy + i * dy_stride + j, left);
            if (pre.p) z[u].load(pre, i, j, left);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t i = i0 + 4 * u;
          if (i >= r1) break;
          float v[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = float(d[u].e[k]);
          with_act(act, [&](auto a) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= act_slope<decltype(a)::value>(z[u].value(k));
          });
          if (left < 8) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < left ? v[k] : 0.0f;
          }
          if (dz) put<T, 8>(dz, i * dz_stride + j, v, wide);
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] += v[k];
        }
      }
    if (!part) continue;
    if (b != blockIdx.x) __syncthreads();  // the last place's sums have been read
#pragma unroll
    for (int k = 0; k < 8; ++k) red[wave][lane * 8 + k] = s[k];
    __syncthreads();
    for (int c = threadIdx.x; c < 512; c += 256) {
      const int64_t col = strip * 512 + c;
      if (col < n)
        part[chunk * n + col] = red[0][c] + red[1][c] + red[2][c] + red[3][c];
    }
  }
}

// ---- operands laid out anew ---------------------------------------------------------

// Rows of `cols` elements into rows of per_row 16-byte pieces, the last one's rest zeros.
struct Lay {
  const void *from;
  int64_t stride, cols;
  uint32_t per_row, pieces;
  u32x4 *to;
};
// Two operands by one launch (a launch of its own took each some 8 us, of 42 for 1001 x 2050 x 4099 in
// 8-bit integers): the first `blocks` blocks take A.
template <typename S>
__global__ __launch_bounds__(256) void k_lay(Lay A, Lay B, uint32_t blocks) {
  const bool first = blockIdx.x < blocks;
  const Lay &L = first ? A : B;
  const uint32_t b = first ? blockIdx.x : blockIdx.x - blocks;
  u32x4 v[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t t = b * 1024 + u * 256 + threadIdx.x;
    const int64_t row = t / L.per_row, c = int64_t(t % L.per_row) * (16 / int(sizeof(S)));
    if (t < L.pieces) v[u] = row_piece(static_cast<const S *>(L.from) + row * L.stride, c, L.cols);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t t = b * 1024 + u * 256 + threadIdx.x;
    if (t < L.pieces) L.to[t] = v[u];
  }
}

// ---- launches --------------------------------------------------------------------

// Whether every 16-byte piece of an operand is aligned, and lies in it or outside it, or
// ends in zeros.
template <typename S>
bool is_direct(const Operand &O, bool turned, int64_t depth) {
  constexpr int64_t E = 16 / int64_t(sizeof(S));
  return reinterpret_cast<uintptr_t>(O.p) % 16 == 0 && O.stride % E == 0 &&
         (O.padded || (turned ? O.rows : depth) % E == 0);
}

// The copy of an operand of rows x cols to `to`, which takes its place.
template <typename S>
Lay lay_of(Operand &O, int64_t rows, int64_t cols, bool turned, char *to) {
  const int64_t stride = padded(cols, sizeof(S));
  const uint32_t per_row = uint32_t(stride * sizeof(S) / 16);
  const Lay l{O.p, O.stride, cols, per_row, uint32_t(rows * per_row),  // (below 2^30)
              reinterpret_cast<u32x4 *>(to)};
  O = Operand{to, stride, turned ? stride : rows, true};
  return l;
}
template <typename S>
hipError_t lay(const Lay &A, const Lay &B, hipStream_t stream) {
  const uint32_t a = ceil_div<uint32_t>(A.pieces, 1024), b = ceil_div<uint32_t>(B.pieces, 1024);
  hipLaunchKernelGGL((k_lay<S>), dim3(a + b), dim3(256), 0, stream, A, B, a);
  return hipGetLastError();
}
template <typename S>
hipError_t lay(Operand &O, int64_t rows, int64_t cols, bool turned, char *to, hipStream_t stream) {
  const Lay l = lay_of<S>(O, rows, cols, turned, to);
  return lay<S>(l, Lay{l.from, 0, 0, 1, 0, nullptr}, stream);
}

template <typename S, bool TP, bool TQ, int BI, int BJ, int kWavesI, int kWavesJ, int W,
          int kStages>
void launch_direct(const Product &A, dim3 grid, hipStream_t stream) {
  hipLaunchKernelGGL((k_product_direct<S, TP, TQ, BI, BJ, kWavesI, kWavesJ, W, kStages>), grid,
                     dim3(64 * kWavesI * kWavesJ), 0, stream, A);
}

template <typename S, int G>
void launch_few(const Product &A, const FewPlan &p, hipStream_t stream) {
  const dim3 grid(unsigned(p.blocks), unsigned(p.splits));
  if (p.waves == 4)
    hipLaunchKernelGGL((k_few<S, G, 4>), grid, dim3(256), 0, stream, A);
  else
    hipLaunchKernelGGL((k_few<S, G, 16>), grid, dim3(1024), 0, stream, A);
}

template <int N, Scales kScales, bool kInt>
void launch_join(const Epilogue &E, int64_t splits, hipStream_t stream) {
  const int64_t vectors = E.rows * ceil_div<int64_t>(E.cols, N);
  if (splits > 4)
    hipLaunchKernelGGL((k_join<8, N, kScales, kInt>),
                       dim3(unsigned(ceil_div<int64_t>(vectors, 32))), dim3(256), 0, stream, E,
                       int32_t(splits));
  else
    hipLaunchKernelGGL((k_join<1, N, kScales, kInt>),
                       dim3(unsigned(ceil_div<int64_t>(vectors, 256))), dim3(256), 0, stream, E,
                       int32_t(splits));
}
template <typename S>
hipError_t join(const Epilogue &E, int64_t splits, hipStream_t stream) {
  constexpr Scales kScales = kIs8<S> ? Scales::kAny : Scales::kNone;
  E.dtype == HG_DT_F32 ? launch_join<4, kScales, kWhole<S>>(E, splits, stream)
                       : launch_join<8, kScales, kWhole<S>>(E, splits, stream);
  return hipGetLastError();
}

// The operand of C's rows (or columns) from `at` on, and the epilogue of n of them.
template <typename S>
Operand axis_from(Operand O, bool turned, int64_t at) {
  O.p = static_cast<const S *>(O.p) + (turned ? at : at * O.stride);
  O.rows -= at;
  return O;
}
void advance(const void *&p, int64_t elements, int32_t dtype) {
  if (p) p = static_cast<const char *>(p) + elements * size_of(dtype);
}
void advance(void *&p, int64_t elements, int32_t dtype) {
  if (p) p = static_cast<char *>(p) + elements * size_of(dtype);
}
Epilogue epilogue_of_rows(Epilogue E, int64_t at, int64_t n) {
  E.rows = n;
  advance(E.y, at * E.y_stride, E.dtype);
  advance(E.residual, at * E.residual_stride, E.dtype);
  advance(E.pre, at * E.pre_stride, E.dtype);
  if (E.row_scale) E.row_scale += at;
  return E;
}
Epilogue epilogue_of_cols(Epilogue E, int64_t at, int64_t n) {
  E.cols = n;
  advance(E.y, at, E.dtype);
  advance(E.residual, at, E.dtype);
  advance(E.pre, at, E.dtype);
  advance(E.bias, at, E.bias_dtype);
  if (E.col_scale) E.col_scale += at;
  return E;
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
  if constexpr (!TP && !TQ) {
    if (is_few(E.rows, E.cols)) {
      const FewPlan p = few_plan(E.cols, depth, sizeof(S));
      A.per_split = p.per_split;
      if (p.splits > 1) A.E.part = parts;
      if (E.rows <= 16)
        launch_few<S, 1>(A, p, stream);
      else
        launch_few<S, 2>(A, p, stream);
      const hipError_t e = hipGetLastError();
      return e != hipSuccess || p.splits == 1 ? e : join<S>(A.E, p.splits, stream);
    }
  }
  if (E.cols > kMostCols) {
    const int64_t half = E.cols / 2 / 256 * 256;
    const hipError_t e = product<S, TP, TQ>(P, Q, depth, epilogue_of_cols(E, 0, half), parts, stream);
    return e != hipSuccess ? e
                           : product<S, TP, TQ>(axis_from<S>(P, TP, half), Q, depth,
                                                epilogue_of_cols(E, half, E.cols - half), parts,
                                                stream);
  }
  const int64_t slab = kDepth<typename ComputeOf<S>::T, 128>;
  const bool direct = is_direct<S>(P, TP, depth) && is_direct<S>(Q, TQ, depth);
  for (int64_t done = 0; done < E.rows;) {
    const Plan p = plan_of(E.rows - done, E.cols, depth, slab, TP && TQ, direct);
    Product B = A;
    B.Q = axis_from<S>(Q, TQ, done);
    B.E = epilogue_of_rows(E, done, p.rows);
    const int64_t ti = ceil_div<int64_t>(p.rows, p.tile_i), tj = ceil_div<int64_t>(E.cols, p.tile_j);
    B.tiles_i = int32_t(ti);
    B.tiles_j = int32_t(tj);
    B.per_split = p.per_split;
    if (p.splits > 1) B.E.part = parts;
    const dim3 grid(unsigned(ti * tj), unsigned(p.splits));
    if (!direct && p.cut == Cut::kSmall)
      hipLaunchKernelGGL((k_product<S, TP, TQ, 64, 64>), grid, dim3(256), 0, stream, B);
    else if (!direct)
      hipLaunchKernelGGL((k_product<S, TP, TQ, 128, 128>), grid, dim3(256), 0, stream, B);
    else if (p.cut == Cut::kMedium)
      launch_direct<S, TP, TQ, 128, 128, 2, 2, 128, 2>(B, grid, stream);
    else if (p.cut == Cut::kSmall)
      launch_direct<S, TP, TQ, 64, 64, 2, 2, 128, 4>(B, grid, stream);
    else if constexpr (sizeof(S) == 4)
      return hipErrorInvalidConfiguration;  // (plan_of has no other cut in 32 bits)
    else if constexpr (TP && TQ)
      launch_direct<S, TP, TQ, 256, 128, 4, 2, 64, 3>(B, grid, stream);
    else
      launch_direct<S, TP, TQ, 256, 256, 2, 4, 128, 2>(B, grid, stream);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) e = join<S>(B.E, p.splits, stream);
    if (e != hipSuccess) return e;
    done += p.rows;
  }
  return hipSuccess;
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
  if (A.dtype == HG_DT_E4M3 || A.dtype == HG_DT_I8) {
    E.row_scale = A.x_scale;
    E.col_scale = A.w_scale;
  }
  Operand w{A.w, A.w_stride, A.n}, x{A.x, A.x_stride, A.m};
  const LinearSpace s = linear_space(A.m, A.k, A.n, A.dtype);
  char *const ws = static_cast<char *>(A.workspace);
  if (s.laid) {
    const Lay lw = lay_of<T>(w, A.n, A.k, false, ws + s.w);
    const Lay lx = lay_of<T>(x, A.m, A.k, false, ws + s.x);
    const hipError_t e = lay<T>(lw, lx, stream);
    if (e != hipSuccess) return e;
  }
  return product<T, false, false>(w, x, A.k, E, reinterpret_cast<float *>(ws + s.parts), stream);
}

template <typename T>
hipError_t linear_grad(const hg_linear_grad_args &A, const Kept &kept_x, const Kept &kept_pre,
                       hipStream_t stream) {
  const GradSpace g = grad_space(A.m, A.k, A.n, A.dtype, A.act, kept_x.p && A.dw);
  char *const ws = static_cast<char *>(A.workspace);
  Operand dz{A.dy, A.dy_stride, A.m}, dz_turned{A.dy, A.dy_stride, A.n};
  const bool has_act = A.act != HG_ACT_NONE;
  const int64_t chunks = ceil_div<int64_t>(A.m, kSumRows);
  const bool products = (A.dx || A.dw) && A.k > 0;
  if (A.m > 0 && A.n > 0 && ((g.dz_laid && products) || A.dbias)) {
    const int64_t strips = ceil_div<int64_t>(A.n, 512);
    const int64_t places = strips * chunks;
    T *const to = g.dz_laid && products ? reinterpret_cast<T *>(ws + g.dz) : nullptr;
    float *const sums = A.dbias ? reinterpret_cast<float *>(ws + g.sums) : nullptr;
    const auto launch = [&](auto pre) {
      hipLaunchKernelGGL((k_dz<T, decltype(pre)>), dim3(unsigned(std::min(places, kMostBlocks))),
                         dim3(256), 0, stream, static_cast<const T *>(A.dy), A.dy_stride, pre, A.act,
                         A.m, A.n, strips, places, to, g.dz_stride, sums);
    };
    if (has_act && kept_pre.p)
      launch(PreKept{kept_pre});
    else
      launch(PreRows<T>{has_act ? static_cast<const T *>(A.pre) : nullptr, A.pre_stride});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (to) {
      dz = Operand{to, g.dz_stride, A.m, true};
      dz_turned = Operand{to, g.dz_stride, g.dz_stride, true};
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
    Operand w{A.w, A.w_stride, A.k};
    hipError_t e = g.laid ? lay<T>(w, A.n, A.k, true, ws + g.w, stream) : hipSuccess;
    if (e == hipSuccess) e = product<T, true, false>(w, dz, A.n, E, parts, stream);
    if (e != hipSuccess) return e;
  }
  if (A.dw) {
    Epilogue E{};
    E.y = A.dw;
    E.y_stride = A.dw_stride;
    E.rows = A.n;
    E.cols = A.k;
    E.dtype = A.dw_dtype;
    Operand x{A.x, A.x_stride, A.k};
    hipError_t e = hipSuccess;
    if (kept_x.p && A.m > 0 && A.k > 0) {
      // what the rows stand for, in T (the products' instructions take it): a rounding more than
      // the integers and their scales have, of 2^-8 of each value at most (bfloat16; 2^-11 in float16)
      // where half their own step is 2^-8 of the largest value that shares the scale
      const int64_t stride = padded(A.k, sizeof(T));
      e = launch_dequantize(kept_x, A.m, A.k, stride, A.dtype, ws + g.x, stride, true, stream);
      x = Operand{ws + g.x, stride, stride, true};
    } else if (g.laid) {
      e = lay<T>(x, A.m, A.k, true, ws + g.x, stream);
    }
    return e != hipSuccess ? e : product<T, true, true>(x, dz_turned, A.m, E, parts, stream);
  }
  return hipSuccess;
}

}  // namespace

int64_t linear_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype) {
  return linear_space(m, k, n, dtype).total;
}

hipError_t launch_linear(const hg_linear_args &A, hipStream_t stream) {
  switch (A.dtype) {
    case HG_DT_F32: return linear<float>(A, stream);
    case HG_DT_F16: return linear<_Float16>(A, stream);
    case HG_DT_BF16: return linear<__bf16>(A, stream);
    case HG_DT_I8: return linear<I8>(A, stream);
    default: return linear<F8>(A, stream);
  }
}

int64_t linear_grad_workspace(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act,
                              bool kept_x) {
  return grad_space(m, k, n, dtype, act, kept_x).total;
}

hipError_t launch_linear_grad(const hg_linear_grad_args &A, const Kept &x, const Kept &pre,
                              hipStream_t stream) {
  switch (A.dtype) {
    case HG_DT_F32: return linear_grad<float>(A, x, pre, stream);
    case HG_DT_F16: return linear_grad<_Float16>(A, x, pre, stream);
    default: return linear_grad<__bf16>(A, x, pre, stream);
  }
}

}  // namespace hg
