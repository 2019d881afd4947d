// Distillation from a teacher's top logits: loss, gradient or both of a row.
//
//   p = softmax(teacher / T) over the listed classes, q = softmax(z / T) over all
//   loss = sum_j p_j (log p_j - log q_id(j)),  grad_v = a / T (q_v - sum_{id(j) = v} p_j)
//
// Bound by memory: a row of logits is read once, and its gradient written once.  A
// wavefront or a block takes a row.  With a gradient the row stays in registers, as it
// came, between the two sweeps (maximum and sum; the gradient), and each register is
// filled with the next row's values as soon as its gradient is written, so that loads
// are always in flight.  Without one a single sweep keeps a running maximum and sum.
// Each thread's sum is relative to its own maximum; they are brought together once.
// The group's first wavefront reads the teacher's list, for the next row while this
// one is swept, so that a row has two barriers and waits for no chain of loads (with
// the list read by all threads at the start of a row, 14 barriers and three loads
// that follow each other, a step of 8193 x 50001 in 16 bits took 670 us).
// The listed classes' entries are written again after the sweep, from one thread
// each, so that no sum is made by atomics and each entry is rounded once.
#include "hg_dense.hpp"
#include "hg_device.hpp"

namespace hg {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// exp((z - m) / T), c = log2(e) / T
__device__ __forceinline__ float exp_of(float z, float m, float c) {
  return __builtin_amdgcn_exp2f((z - m) * c);
}

// By halves: no long chain of additions.
template <int N>
__device__ __forceinline__ float sum_of(const float (&x)[N]) {
  if constexpr (N == 1) {
    return x[0];
  } else {
    float h[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) h[j] = x[j] + x[j + N / 2];
    return sum_of(h);
  }
}

__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.0f : m; }

template <int W>
__device__ __forceinline__ float lanes_top(float v) {
  return lanes_reduce<W>(v, [](float a, float b) { return fmaxf(a, b); });
}

// A sum of exp((z - m) / T) and its maximum m.  m = -inf: nothing but -inf so far, and
// then s is 0, or NaN where there was one.
struct Softmax {
  float m = -INFINITY, s = 0.0f;
  // Adds N logits, f (those that are not there: -inf).
  template <int N>
  __device__ __forceinline__ void add(const float (&f)[N], float c) {
    float top = m;
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, f[j]);
    const float at = finite_or_0(top);
    float e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) e[j] = exp_of(f[j], at, c);
    s = s * exp_of(m, at, c) + sum_of(e);  // (m = -inf: 0 times 0, or NaN kept)
    m = top;
  }
  // Over W neighbouring lanes.
  template <int W>
  __device__ __forceinline__ void join(float c) {
    const float top = lanes_top<W>(m);
    s = lanes_sum<W>(s * exp_of(m, finite_or_0(top), c));
    m = top;
  }
};

// Threads of a row's group, and rows of a block.
template <int G>
constexpr int kBlockOf = G < 256 ? 256 : G;
template <int G>
constexpr int kRowsOf = kBlockOf<G> / G;

// Entries of a list that a lane of the first wavefront holds ahead of their row; longer
// lists read the rest when the row begins.
constexpr int kAhead = 2;

constexpr int kScalars = 5;

// LDS of a group, twice: a row's is written while the last one's may still be read.
struct RowLds {
  float *p, *zt;      // [top]: p_j (0 where left out), z at its class
  int *id;            // [top]: the class, -1 where left out
  float *m, *s;       // [G / 64]: the wavefronts' sums
  float *scalars;     // [kScalars]
};
template <int G>
__host__ __device__ constexpr int lds_floats(int top) {
  return 3 * top + 2 * (G / 64) + kScalars;
}

template <typename T, int G>
struct Row {
  const hg_distill_args &A;
  float *lds;      // of this group
  uint32_t *seen;  // LDS: a bit for every class, all 0 between rows (NULL: not kept)
  int tid, top, n;
  int turn = 1;
  float inv_t, c;
  // the first wavefront's: the list of the row to come
  int64_t v[kAhead];
  float t[kAhead], z[kAhead], weight;
  // of the current row, for all
  float a;
  bool nothing;  // no entry is left: loss and gradient are 0
  bool repeats;  // a class may be listed twice

  __device__ __forceinline__ Row(const hg_distill_args &args, float *base, bool bits)
      : A(args), tid(threadIdx.x % G), top(args.top), n(int(args.classes)) {
    lds = base + (threadIdx.x / G) * 2 * lds_floats<G>(top);
    seen = nullptr;
    if (bits) {
      const int words = (n + 31) / 32;
      seen = reinterpret_cast<uint32_t *>(base + kRowsOf<G> * 2 * lds_floats<G>(top)) +
             (threadIdx.x / G) * words;
      for (int k = tid; k < words; k += G) seen[k] = 0;
      sync();
    }
    inv_t = 1.0f / A.temperature;
    c = kLog2e * inv_t;
  }
  __device__ __forceinline__ static void sync() {
    if (G == 64)
      wave_sync();
    else
      __syncthreads();
  }
  __device__ __forceinline__ bool first() const { return G == 64 || tid < 64; }
  __device__ __forceinline__ RowLds at() const {
    float *const b = lds + turn * lds_floats<G>(top);
    return RowLds{b, b + top, reinterpret_cast<int *>(b + 2 * top), b + 3 * top,
                  b + 3 * top + G / 64, b + 3 * top + 2 * (G / 64)};
  }
  __device__ __forceinline__ bool in(int64_t cls, float logit) const {
    return cls >= 0 && cls < n && !(logit == -INFINITY);
  }

  // The first wavefront, two steps ahead of a row's begin().
  __device__ __forceinline__ void fetch_list(int64_t i) {
    weight = A.row_weight ? A.row_weight[i] : 1.0f;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int j = (tid & 63) + 64 * e;
      v[e] = -1;
      t[e] = -INFINITY;
      if (j < top) {
        v[e] = A.ids[i * A.ids_stride + j];
        t[e] = load_f32(A.teacher, A.teacher_dtype, i * A.teacher_stride + j);
      }
    }
  }
  __device__ __forceinline__ float logit(int64_t i, int64_t cls) const {
    return float(static_cast<const T *>(A.logits)[i * A.logits_stride + cls]);
  }
  __device__ __forceinline__ void fetch_logits(int64_t i) {
#pragma unroll
    for (int e = 0; e < kAhead; ++e) z[e] = in(v[e], t[e]) ? logit(i, v[e]) : 0.0f;
  }

  // Row i begins: the first wavefront makes p from its list.
  __device__ __forceinline__ void begin(int64_t i) {
    turn ^= 1;
    if (!first()) return;
    const RowLds L = at();
    const int lane = tid & 63;
    float tm = -INFINITY, flags = 0.0f;  // 1: an entry, 2: an id out of range
    const auto see = [&](int j, int64_t cls, float logit, float at_z) {
      const bool ok = in(cls, logit);
      L.id[j] = ok ? int(cls) : -1;
      L.p[j] = logit;
      L.zt[j] = at_z;
      if (ok) tm = fmaxf(tm, logit);
      flags = fmaxf(flags, cls < -1 || cls >= n ? 2.0f : (ok ? 1.0f : 0.0f));
    };
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
      if (lane + 64 * e < top) see(lane + 64 * e, v[e], t[e], z[e]);
    for (int j = lane + 64 * kAhead; j < top; j += 64) {
      const int64_t cls = A.ids[i * A.ids_stride + j];
      const float x = load_f32(A.teacher, A.teacher_dtype, i * A.teacher_stride + j);
      see(j, cls, x, in(cls, x) ? logit(i, cls) : 0.0f);
    }
    tm = lanes_top<64>(tm);
    flags = lanes_top<64>(flags);
    float ts = 0.0f;
    for (int j = lane; j < top; j += 64)
      if (L.id[j] >= 0) ts += exp_of(L.p[j], tm, c);
    ts = lanes_sum<64>(ts);
    const float ln_ts = logf(ts);
    float h = 0.0f;  // sum_j p_j log p_j
    for (int j = lane; j < top; j += 64) {
      const float x = L.p[j];
      const float pj = L.id[j] >= 0 ? exp_of(x, tm, c) / ts : 0.0f;
      if (!(pj == 0.0f)) h += pj * ((x - tm) * inv_t - ln_ts);
      L.p[j] = pj;
    }
    h = lanes_sum<64>(h);
    // whether a class is listed twice: by a bit for every class, cleared again
    bool twice = !seen;
    if (seen) {
      for (int j = lane; j < top; j += 64) {
        const int cls = L.id[j];
        if (cls >= 0) twice = twice || (atomicOr(seen + (cls >> 5), 1u << (cls & 31)) >> (cls & 31) & 1);
      }
      for (int j = lane; j < top; j += 64)
        if (L.id[j] >= 0) seen[L.id[j] >> 5] = 0;
      twice = __any(twice);
    }
    if (lane == 0) {
      L.scalars[4] = twice ? 1.0f : 0.0f;
      L.scalars[0] = flags == 2.0f || ts != ts ? __builtin_nanf("") : 0.0f;
      L.scalars[1] = flags == 0.0f ? 1.0f : 0.0f;
      L.scalars[2] = weight;
      L.scalars[3] = h;
    }
  }

  // Brings the threads' sums together (NaN where the row's results are), learns what
  // begin() found, and writes the loss.
  __device__ __forceinline__ void join(int64_t i, Softmax &q) {
    const RowLds L = at();
    q.template join<64>(c);
    if constexpr (G > 64) {
      if ((threadIdx.x & 63) == 0) {
        L.m[threadIdx.x >> 6] = q.m;
        L.s[threadIdx.x >> 6] = q.s;
      }
      __syncthreads();
      q.m = L.m[threadIdx.x % (G / 64)];
      q.s = L.s[threadIdx.x % (G / 64)];
      q.template join<G / 64>(c);
    } else {
      sync();
    }
    nothing = L.scalars[1] != 0.0f;
    a = L.scalars[2];
    repeats = L.scalars[4] != 0.0f;
    q.s += L.scalars[0];
    if (q.m == -INFINITY) q.s = __builtin_nanf("");
    if (A.loss && first()) {
      float l = 0.0f;
      for (int j = tid; j < top; j += 64) {
        const float pj = L.p[j];
        if (!(pj == 0.0f)) l += pj * (L.zt[j] - q.m);
      }
      l = L.scalars[3] - lanes_sum<64>(l) * inv_t + logf(q.s);
      if (tid == 0) A.loss[i] = nothing ? 0.0f : l;
    }
  }

  // The gradient at the listed classes, once each: p of every entry of the class off.
  // Their entries were written by the sweep already, by other threads.
  __device__ __forceinline__ void listed_entries(T *grad, const Softmax &q) const {
    const RowLds L = at();
    const float f = a * inv_t / q.s;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);  // the sweep's stores are done (vmcnt 0)
    sync();
    if (nothing || a == 0.0f) return;
    if (!repeats) {
      for (int j = tid; j < top; j += G)
        if (L.id[j] >= 0)
          grad[L.id[j]] = T(f * exp_of(L.zt[j], q.m, c) - a * inv_t * L.p[j]);
      return;
    }
    // S neighbouring threads look for an entry's class in a part of the list each
    constexpr int S = G / 64 < 16 ? G / 64 : 16;
    const int share = tid % S;
    for (int j = tid / S; j < top; j += G / S) {
      const int cls = L.id[j];
      float pv = 0.0f;
      float before = 0.0f;  // whether an earlier entry has the class
#pragma unroll 4
      for (int k = share; k < top; k += S)
        if (L.id[k] == cls) {
          before = k < j ? 1.0f : before;
          pv += L.p[k];
        }
      pv = lanes_sum<S>(pv);
      before = lanes_sum<S>(before);
      if (share == 0 && cls >= 0 && before == 0.0f)
        grad[cls] = T(f * exp_of(L.zt[j], q.m, c) - a * inv_t * pv);
    }
  }
};

// How a row at p is cut into vectors that are aligned in memory: `head` elements, `whole`
// vectors, `last` elements (both below a vector).  Rows of an odd length start anywhere,
// and vectors across their boundaries cost a quarter more (rows of 50001 in 16 bits: the
// loss 166 us, 123 with the cut; rows of 50048: 123).
// (Not for short rows, where the ends cost more than they save: 32768 x 4001 in 16 bits,
// the loss 104 us with the cut and 76 without.)
template <typename T, bool kAlign>
struct Cut {
  int head, whole, last;
  __device__ __forceinline__ Cut(const T *p, int n) {
    constexpr int V = kVec<T>;
    head = kAlign ? int(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(T)) : 0;
    head = head < n ? head : n;
    whole = (n - head) / V;
    last = n - head - whole * V;
  }
};

// With a gradient: NV vectors a thread hold the row, and one more (of the first two
// threads) its ends.  Groups walk over the rows.
template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlockOf<G>, 4) void k_distill_step(hg_distill_args A) {
  constexpr int V = kVec<T>;
  // Past the caches for long rows; within them the listed classes' logits are found again,
  // and their gradients merge with the sweep's (32768 x 1000 in float32: 32 us cached, 46
  // streamed; 8193 x 50048 in 16 bits: 344 and 318).
  constexpr Move kLoad = G * NV > 3072 ? Move::kStreamed : Move::kCached;
  constexpr Move kStore = G > 64 ? Move::kStreamed : Move::kCached;
  extern __shared__ float lds[];
  Row<T, G> R(A, lds, true);
  const int n = int(A.classes);
  const uint32_t tid = R.tid;
  const int64_t step = int64_t(gridDim.x) * kRowsOf<G>;
  // (a wavefront's row is the same for its lanes: its address stays in scalar registers)
  int64_t i = int64_t(blockIdx.x) * kRowsOf<G> + __builtin_amdgcn_readfirstlane(threadIdx.x / G);
  const T *const logits = static_cast<const T *>(A.logits);
  float x[V];
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] = -INFINITY;
  const u32x4 none = pack<T>(x);
  u32x4 r[NV], end;
  const auto load = [&](const T *z, const Cut<T, (G > 64)> &C, int v) {
    r[v] = none;
    if (v * G + int(tid) < C.whole)
      r[v] = load_raw<T, kLoad>(z + C.head + v * G * V + tid * V);
  };
  const auto load_end = [&](const T *z, const Cut<T, (G > 64)> &C) {
    Vec<T> t = __builtin_bit_cast(Vec<T>, none);
    if (G > 64 && tid == 0 && C.head) t.load(z, C.head, T(-INFINITY));
    if (tid == 1 && C.last) t.load(z + n - C.last, C.last, T(-INFINITY));
    end = __builtin_bit_cast(u32x4, t);
  };
  if (i < A.rows) {
    if (R.first()) R.fetch_list(i);
    const T *const z = logits + i * A.logits_stride;
    const Cut<T, (G > 64)> C(z, n);
#pragma unroll
    for (int v = 0; v < NV; ++v) load(z, C, v);
    load_end(z, C);
    if (R.first()) R.fetch_logits(i);
  }
  // (a wavefront leaves on its own; a larger group is the block)
  for (; i < A.rows; i += step) {
    T *const grad = static_cast<T *>(A.grad) + i * A.grad_stride;
    const T *const z = logits + (i + step) * A.logits_stride;  // the next row
    const Cut<T, (G > 64)> C(logits + i * A.logits_stride, n), D(z, n);
    const bool more = i + step < A.rows;
    R.begin(i);
    if (more && R.first()) R.fetch_list(i + step);
    Softmax q;
    const auto top = [&](u32x4 raw) {
      unpack<T>(forget(raw, q.m), x);
#pragma unroll
      for (int j = 0; j < V; ++j) q.m = fmaxf(q.m, x[j]);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) top(r[v]);
    top(end);
    const float at = finite_or_0(q.m);
    const auto sum = [&](u32x4 raw) {
      unpack<T>(forget(raw, q.s), x);
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = exp_of(x[j], at, R.c);
      q.s += sum_of(x);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) sum(r[v]);
    sum(end);
    if (more && R.first()) R.fetch_logits(i + step);
    R.join(i, q);
    // rows whose gradient is 0 are written as such, whatever their logits
    const bool zero = R.nothing || R.a == 0.0f;
    float f = R.a * R.inv_t / q.s;
    const auto slope = [&](u32x4 raw) {
      unpack<T>(forget(raw, f), x);
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = f * exp_of(x[j], q.m, R.c);
      const u32x4 w = pack<T>(x);
      return __builtin_bit_cast(Vec<T>, zero ? u32x4{0, 0, 0, 0} : w);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v * G + int(tid) < C.whole)
        slope(r[v]).template store<kStore>(grad + C.head + v * G * V + tid * V, V);
      if (more) load(z, D, v);
    }
    if (tid < 2) {
      if (G > 64 && tid == 0 && C.head) slope(end).store(grad, C.head);
      if (tid == 1 && C.last) slope(end).store(grad + n - C.last, C.last);
      if (more) load_end(z, D);
    }
    R.listed_entries(grad, q);
  }
}

// The loss alone, or (with kGrad) rows too long for the kernel above, which are read a
// second time for their gradient.
template <typename T, int G, bool kGrad, bool kAlign>
__global__ __launch_bounds__(kBlockOf<G>) void k_distill(hg_distill_args A) {
  constexpr int V = kVec<T>;
  constexpr int U = 4;  // vectors of a thread in flight
  constexpr Move kMove = kGrad ? Move::kCached : Move::kStreamed;
  extern __shared__ float lds[];
  Row<T, G> R(A, lds, false);
  const int n = int(A.classes), tid = R.tid;
  // (a wavefront leaves on its own; a larger group is the block)
  for (int64_t i = int64_t(blockIdx.x) * kRowsOf<G> + threadIdx.x / G; i < A.rows;
       i += int64_t(gridDim.x) * kRowsOf<G>) {
    const T *const z = static_cast<const T *>(A.logits) + i * A.logits_stride;
    if (R.first()) {
      R.fetch_list(i);
      R.fetch_logits(i);
    }
    const Cut<T, kAlign> C(z, n);
    const T *const body = z + C.head;
    // (counted without a sign: near the end of the longest rows a step passes 2^31)
    const uint32_t end = C.whole * V;
    Softmax q;
    uint32_t k0 = 0;
    for (; k0 + G * V * U <= end; k0 += G * V * U) {
      Vec<T> r[U];
      float x[U * V];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u].template load<kMove>(body + k0 + (u * G + tid) * V, V);
#pragma unroll
      for (int u = 0; u < U * V; ++u) x[u] = float(r[u / V].e[u % V]);
      q.add(x, R.c);
    }
    const auto add = [&](const T *p, int m) {
      Vec<T> r;
      float x[V];
      r.template load<kMove>(p, m, T(-INFINITY));
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = float(r.e[j]);
      q.add(x, R.c);
    };
    for (uint32_t k = k0 + tid * V; k < end; k += G * V) add(body + k, V);
    if (kAlign && tid == 0 && C.head) add(z, C.head);
    if (tid == 1 && C.last) add(z + n - C.last, C.last);
    R.begin(i);
    R.join(i, q);
    if constexpr (kGrad) {
      T *const grad = static_cast<T *>(A.grad) + i * A.grad_stride;
      const bool zero = R.nothing || R.a == 0.0f;
      const float f = R.a * R.inv_t / q.s;
      const auto slope = [&](uint32_t k, int m) {
        Vec<T> r;
        r.load(z + k, m);
#pragma unroll
        for (int j = 0; j < V; ++j)
          r.e[j] = T(zero ? 0.0f : f * exp_of(float(r.e[j]), q.m, R.c));
        r.template store<Move::kStreamed>(grad + k, m);
      };
      for (uint32_t k = tid * V; k < end; k += G * V) slope(C.head + k, V);
      if (tid == 0 && C.head) slope(0, C.head);
      if (tid == 1 && C.last) slope(n - C.last, C.last);
      R.listed_entries(grad, q);
    }
  }
}

template <typename T, int G, int NV>
hipError_t step(const hg_distill_args &A, hipStream_t stream) {
  const size_t lds = size_t(kRowsOf<G>) *
                     (2 * lds_floats<G>(A.top) + (size_t(A.classes) + 31) / 32) * sizeof(float);
  const int64_t blocks = ceil_div<int64_t>(A.rows, kRowsOf<G>);
  const int64_t most = 256 * (2048 / kBlockOf<G>);  // as many threads as 256 compute units hold
  hipLaunchKernelGGL((k_distill_step<T, G, NV>), dim3(unsigned(blocks < most ? blocks : most)),
                     dim3(kBlockOf<G>), lds, stream, A);
  return hipGetLastError();
}

template <typename T, int G, bool kGrad, bool kAlign>
hipError_t sweep(const hg_distill_args &A, hipStream_t stream) {
  const size_t lds = size_t(kRowsOf<G>) * 2 * lds_floats<G>(A.top) * sizeof(float);
  const int64_t blocks = ceil_div<int64_t>(A.rows, kRowsOf<G>);
  hipLaunchKernelGGL((k_distill<T, G, kGrad, kAlign>),
                     dim3(unsigned(blocks < 65536 ? blocks : 65536)), dim3(kBlockOf<G>), lds,
                     stream, A);
  return hipGetLastError();
}

template <typename T>
hipError_t by_classes(const hg_distill_args &A, hipStream_t stream) {
  // (long lists take a block a row at least: four of them need as much LDS as two blocks have)
  int64_t vecs = A.classes / kVec<T>;  // whole ones
  if (A.top > 64 * kAhead && vecs <= 512) vecs = 513;
  if (!A.grad) {
    if (vecs <= 256) return sweep<T, 64, false, false>(A, stream);
    return vecs <= 2048 ? sweep<T, 256, false, false>(A, stream)
                        : sweep<T, 256, false, true>(A, stream);
  }
  if (vecs <= 64) return step<T, 64, 1>(A, stream);
  if (vecs <= 128) return step<T, 64, 2>(A, stream);
  if (vecs <= 256) return step<T, 64, 4>(A, stream);
  if (vecs <= 512) return step<T, 64, 8>(A, stream);
  if (vecs <= 1024) return step<T, 256, 4>(A, stream);
  if (vecs <= 2048) return step<T, 256, 8>(A, stream);
  if (vecs <= 3072) return step<T, 256, 12>(A, stream);
  if (vecs <= 4096) return step<T, 256, 16>(A, stream);
  if (vecs <= 7168) return step<T, 512, 14>(A, stream);
  if (vecs <= 8192) return step<T, 512, 16>(A, stream);
  if (vecs <= 12288) return step<T, 1024, 12>(A, stream);
  if (vecs <= 16384) return step<T, 1024, 16>(A, stream);
  return sweep<T, 1024, true, true>(A, stream);
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
